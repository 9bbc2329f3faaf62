"""wisp_verify_logprobs and wisp_verify_committed_tokens without a GPU: header, exports, refusals."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "wisp_logprobs.h")
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 4


@pytest.fixture(scope="module")
def lib():
    from paper_2601_11652_gb300 import binding, build
    build.build()
    return binding.load()


def test_header_and_exports(lib, tmp_path):
    from paper_2601_11652_gb300 import binding
    src = tmp_path / "t.c"
    src.write_text('#include "wisp_logprobs.h"\nint main(void){ return sizeof(wisp_logprobs_args) > 0 ? 0 : 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src),
                    "-o", str(tmp_path / "t.o")], check=True)
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(wisp_verify_\w+)\s*\(", text))
    assert len(names) == 3
    for n in names:
        assert hasattr(lib, n) and n in binding.EXPORTED, n


def _args(**kw):
    from paper_2601_11652_gb300 import binding as wb
    a = wb.wisp_logprobs_args()
    base = dict(rows=3, V=1000, row_stride=0, logits_dtype=1, logits=0x10000, tokens=0x2000, top_n=5, logprob=0x3000,
                entropy=0x4000, top_tokens=0x5000, top_logprobs=0x6000)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


BAD = [(dict(rows=-1), INVALID), (dict(V=0), INVALID), (dict(V=(1 << 24) + 1), UNSUPPORTED), (dict(row_stride=999), INVALID),
       (dict(row_stride=-5), INVALID), (dict(logits_dtype=2), INVALID), (dict(logits=None), INVALID), (dict(logits=0x10001), INVALID),
       (dict(logits=0x10002, logits_dtype=0), INVALID), (dict(tokens=None), INVALID), (dict(logprob=None), INVALID),
       (dict(top_n=-1), INVALID), (dict(top_n=33), UNSUPPORTED), (dict(top_tokens=None), INVALID), (dict(top_logprobs=None), INVALID)]


@pytest.mark.parametrize("kw,code", BAD, ids=[str(b[0]) for b in BAD])
def test_bad_arguments_are_refused(lib, kw, code):
    a = _args(**kw)
    assert lib.wisp_verify_logprobs(ctypes.byref(a), ctypes.c_void_p(0x100000), 1 << 30, None) == code
    assert lib.wisp_verify_logprobs_workspace_size(ctypes.byref(a)) == 0


def test_null_and_workspace(lib):
    assert lib.wisp_verify_logprobs(None, ctypes.c_void_p(0x100000), 1 << 30, None) == INVALID
    a = _args()
    n = lib.wisp_verify_logprobs_workspace_size(ctypes.byref(a))
    assert n > 0
    for ws, size in ((None, 1 << 30), (0x100010, 1 << 30), (0x100000, n - 1)):
        assert lib.wisp_verify_logprobs(ctypes.byref(a), ctypes.c_void_p(ws), size, None) == WORKSPACE


def test_committed_tokens_refusals(lib):
    from paper_2601_11652_gb300 import binding as wb
    def acc(**kw):
        c = wb.wisp_accept_args()
        for k, v in {**dict(B=2, total_q_rows=4, total_draft=2, draft_lens=0x1000, draft_tokens=0x2000, accepted_len=0x3000,
                            next_token=0x4000), **kw}.items():
            setattr(c, k, v)
        return c
    call = lambda c, out=0x5000: lib.wisp_verify_committed_tokens(ctypes.byref(c) if c else None, ctypes.c_void_p(out), None)
    assert call(None) == INVALID and call(acc(), None) == INVALID
    for kw in (dict(B=-1), dict(total_q_rows=1), dict(total_draft=-1), dict(draft_lens=None), dict(accepted_len=None),
               dict(next_token=None), dict(draft_tokens=None)):
        assert call(acc(**kw)) == INVALID, kw


def test_binding_refuses_rows_that_overlap():
    import torch

    from paper_2601_11652_gb300 import binding as wb
    out = dict(tokens=torch.zeros(3, dtype=torch.int32), logprob=torch.zeros(3))
    for z in (torch.zeros(1, 100).expand(3, 100), torch.zeros(1000).as_strided((3, 100), (99, 1)), torch.zeros(300)):
        with pytest.raises(ValueError) as e:
            wb.make_logprobs_args(logits=z, **out)
        assert "device tensors only" not in str(e.value)
    with pytest.raises(ValueError, match="device tensors only"):
        wb.make_logprobs_args(logits=torch.zeros(3, 100), **out)
