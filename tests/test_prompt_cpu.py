"""Prompt and shared attention without a GPU: the headers compile as C, bad arguments are refused before the device is touched, and
the binding refuses what the library cannot see."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2601_11652_gb300 import binding, build
    build.build()
    return binding.load()


def test_header_compiles_as_c_and_its_functions_are_exported(lib, tmp_path):
    from paper_2601_11652_gb300 import binding
    src = tmp_path / "t.c"
    src.write_text('#include "wisp_prompt.h"\nint main(void){ return sizeof(wisp_shared_args) > sizeof(wisp_prompt_args) ? 0 : 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-c", "-o", str(tmp_path / "t.o")],
                   check=True)
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "wisp_prompt.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(wisp_\w+)\s*\(const", text))
    assert names == {"wisp_prompt_workspace_size", "wisp_prompt_attention", "wisp_verify_shared_workspace_size", "wisp_verify_attention_shared"}
    for n in names:
        assert hasattr(lib, n) and n in binding.EXPORTED


def _args(attn=None, shared=None, **kw):
    from paper_2601_11652_gb300 import binding as wb
    s = wb.wisp_shared_args()
    base = dict(B=2, Hq=8, Hkv=2, D=128, block_size=16, max_blocks_per_seq=4, num_blocks=8, total_q_rows=40, draft_lens=0x1000,
                context_lens=0x2000, block_tables=0x3000, qkv_dtype=1, q=0x10000, k_cache=0x20000, v_cache=0x30000, out=0x40000)
    for k, v in {**base, **(attn or {})}.items():
        setattr(s.rows.attn, k, v)
    for k, v in {**dict(cache_dtype=2, k_scale=0x50000, v_scale=0x60000), **kw}.items():
        setattr(s.rows, k, v)
    for k, v in {**dict(shared_ids=0x70000, shared_pages=0x80000), **(shared or {})}.items():
        setattr(s, k, v)
    return s


BAD = [(dict(attn=dict(B=-1)), INVALID), (dict(attn=dict(Hq=0)), INVALID), (dict(attn=dict(Hq=9)), INVALID), (dict(attn=dict(Hkv=0)), INVALID),
       (dict(attn=dict(D=96)), UNSUPPORTED), (dict(attn=dict(block_size=32)), UNSUPPORTED), (dict(attn=dict(Hq=258)), UNSUPPORTED),
       (dict(attn=dict(qkv_dtype=2)), INVALID), (dict(cache_dtype=0), INVALID), (dict(cache_dtype=3), INVALID),
       (dict(attn=dict(qkv_dtype=0), cache_dtype=1), INVALID), (dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID),
       (dict(attn=dict(total_q_rows=1)), INVALID), (dict(attn=dict(num_blocks=0)), INVALID), (dict(attn=dict(max_blocks_per_seq=0)), INVALID),
       (dict(attn=dict(max_blocks_per_seq=1 << 27)), UNSUPPORTED), (dict(attn=dict(total_q_rows=(1 << 31) - 1)), UNSUPPORTED)] + \
      [(dict(attn={n: None}), INVALID) for n in ("draft_lens", "context_lens", "block_tables", "q", "k_cache", "v_cache", "out")] + \
      [(dict(attn={n: 0x10008}), INVALID) for n in ("q", "k_cache", "v_cache", "out")]


@pytest.mark.parametrize("kw,code", BAD, ids=[str(b[0]) for b in BAD])
def test_bad_arguments_are_refused(lib, kw, code):
    a, ws = _args(**kw), ctypes.c_void_p(0x100000)
    assert lib.wisp_prompt_attention(ctypes.byref(a.rows), ws, 1 << 40, None) == code
    assert lib.wisp_verify_attention_shared(ctypes.byref(a), ws, 1 << 40, None) == code
    assert lib.wisp_prompt_workspace_size(ctypes.byref(a.rows)) == 0 and lib.wisp_verify_shared_workspace_size(ctypes.byref(a)) == 0


def test_null_and_missing_groups(lib):
    ws = ctypes.c_void_p(0x100000)
    assert lib.wisp_prompt_attention(None, ws, 1 << 40, None) == INVALID and lib.wisp_prompt_workspace_size(None) == 0
    assert lib.wisp_verify_attention_shared(None, ws, 1 << 40, None) == INVALID and lib.wisp_verify_shared_workspace_size(None) == 0
    for n in ("shared_ids", "shared_pages"):
        a = _args(shared={n: None})
        assert lib.wisp_verify_attention_shared(ctypes.byref(a), ws, 1 << 40, None) == INVALID
        assert lib.wisp_verify_shared_workspace_size(ctypes.byref(a)) == 0


def _tensors(**kw):
    import torch
    t, i = torch.zeros, lambda *s: torch.zeros(s, dtype=torch.int32)
    base = dict(draft_lens=i(2), context_lens=i(2), block_tables=i(2, 4), q=t(9, 8, 64, dtype=torch.bfloat16), out=t(9, 8, 64, dtype=torch.bfloat16),
                k_cache=t(8, 2, 16, 64, dtype=torch.uint8), v_cache=t(8, 2, 16, 64, dtype=torch.uint8), k_scale=t(8, 2), v_scale=t(8, 2))
    return {**base, **kw}


def test_binding_refuses_what_would_be_read_out_of_range():
    import torch

    from paper_2601_11652_gb300 import binding as wb
    t, i, bf = torch.zeros, lambda *s: torch.zeros(s, dtype=torch.int32), dict(dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensors only"):  # (nothing else is wrong with these)
        wb.make_prompt_args(**_tensors())
    bad = [dict(out=t(8, 8, 64, **bf)), dict(out=t(9, 8, 64)), dict(q=t(9, 512, **bf), out=t(9, 512, **bf)), dict(q=t(9, 8, 128, **bf), out=t(9, 8, 128, **bf)),
           dict(v_cache=t(7, 2, 16, 64, dtype=torch.uint8)), dict(v_cache=t(8, 2, 16, 64, **bf)), dict(k_cache=t(8, 2, 64, dtype=torch.uint8)),
           dict(context_lens=i(1)), dict(block_tables=i(1, 4)), dict(block_tables=i(8)), dict(draft_lens=t(2, dtype=torch.int64)),
           dict(context_lens=t(2)), dict(block_tables=t(2, 4)), dict(request_ids=i(2)), dict(request_ids=t(1, dtype=torch.int64)),
           dict(num_blocks=9), dict(total_q_rows=10), dict(k_scale=None), dict(v_scale=t(8, 3)), dict(v_scale=t(8, 2, dtype=torch.float64)),
           dict(k_cache=t(8, 2, 16, 64), v_cache=t(8, 2, 16, 64))]
    for kw in bad:
        with pytest.raises(ValueError) as e:
            wb.make_prompt_args(**_tensors(**kw))
        assert "device tensors only" not in str(e.value) or "scale" in str(kw), kw
    for kw in (dict(shared_ids=i(1), shared_pages=i(2)), dict(shared_ids=i(2), shared_pages=t(2))):
        with pytest.raises(ValueError, match="shared_ids"):
            wb.make_shared_args(**_tensors(), **kw)


def test_sessions_that_may_not_share():
    import torch

    from paper_2601_11652_gb300 import serve
    s = serve.PagedSessions(4, 2, 64, "bf16", 16, 4, device="cpu")
    s.ctx[0] = 40
    s.tables[0, :3] = torch.tensor([4, 9, 2])
    for src, sids, tokens in ((0, [1], 20), (0, [1], 0), (0, [1], -16), (0, [1], 48), (0, [0], 16), (0, [1, 1], 16), (1, [2], 16), (2, [0], 16)):
        with pytest.raises(ValueError):
            s.share(src, sids, tokens)
    s.tables[3, 0] = 5
    with pytest.raises(ValueError):
        s.share(0, [3], 16)
    s.share(0, [1, 2], 32)
    assert s.tables[1].tolist() == s.tables[2].tolist() == [4, 9, -1, -1] and s.ctx.tolist() == [40, 32, 32, 0]
    assert s.prefix == [(0, 2)] * 3 + [(-1, 0)]
