"""wisp_kv_reserve_append_rope without a GPU: the header compiles as C, its symbols are exported, and arguments that the
host can judge are refused before the device is touched."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "wisp_kv8.h")


@pytest.fixture(scope="module")
def lib():
    from paper_2601_11652_gb300 import binding, build
    build.build()
    return binding.load()


def test_header_and_exports(lib, tmp_path):
    from paper_2601_11652_gb300 import binding
    src = tmp_path / "t.c"
    src.write_text('#include "wisp_kv8.h"\nint main(void){ return sizeof(wisp_kv_rope_args) > 0 ? 0 : 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src),
                    "-o", str(tmp_path / "t.o")], check=True)
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(wisp_(?:verify|kv)_\w+)\s*\(", text))
    assert {"wisp_kv_rope_workspace_size", "wisp_kv_reserve_append_rope"} <= names
    for n in names:
        assert hasattr(lib, n) and n in binding.EXPORTED, n


def _args(kv=None, **kw):
    from paper_2601_11652_gb300 import binding as wb
    a = wb.wisp_kv_rope_args()
    base_kv = dict(B=2, Hkv=2, D=128, block_size=16, max_blocks_per_seq=4, num_blocks=8, total_q_rows=4, draft_lens=0x1000,
                   context_lens=0x2000, block_tables=0x3000, free_blocks=0x4000, free_count=0x5000, kv_dtype=1,
                   k_cache=0x10000, v_cache=0x20000, k_new=0x30000, v_new=0x40000)
    base = dict(cache_dtype=2, k_scale=0x50000, v_scale=0x60000, rope=0x70000, rope_positions=64, rot_dim=128, interleaved=0,
                Hq=8, q=0x80000, q_out=0x90000, q_stride=0, k_stride=0, v_stride=0)
    for k, v in {**base_kv, **(kv or {})}.items():
        setattr(a.kv, k, v)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 4
BAD = [(dict(kv=dict(B=-1)), INVALID), (dict(kv=dict(D=96)), UNSUPPORTED), (dict(kv=dict(block_size=32)), UNSUPPORTED),
       (dict(kv=dict(kv_dtype=2)), INVALID), (dict(kv=dict(k_new=None)), INVALID), (dict(kv=dict(v_cache=0x20008)), INVALID),
       (dict(kv=dict(total_q_rows=1)), INVALID), (dict(cache_dtype=0), INVALID), (dict(cache_dtype=3), INVALID),
       (dict(k_scale=None), INVALID), (dict(rope=None), INVALID), (dict(rope=0x70004), INVALID),
       (dict(rope_positions=0), INVALID), (dict(rot_dim=24), UNSUPPORTED), (dict(rot_dim=144), INVALID),
       (dict(rot_dim=-16), INVALID), (dict(Hq=-1), INVALID), (dict(q=None), INVALID), (dict(q_out=0x90002), INVALID),
       (dict(q_stride=8 * 128 - 8), INVALID), (dict(k_stride=2 * 128 + 4), INVALID), (dict(v_stride=-256), INVALID)]


@pytest.mark.parametrize("kw,code", BAD, ids=[str(b[0]) for b in BAD])
def test_bad_arguments_are_refused(lib, kw, code):
    a = _args(**kw)
    assert lib.wisp_kv_reserve_append_rope(ctypes.byref(a), ctypes.c_void_p(0x100000), 1 << 30, None) == code


def test_null_and_workspace(lib):
    assert lib.wisp_kv_reserve_append_rope(None, ctypes.c_void_p(0x100000), 1 << 30, None) == INVALID
    assert lib.wisp_kv_rope_workspace_size(None) == 0
    a = _args()
    n = lib.wisp_kv_rope_workspace_size(ctypes.byref(a))
    assert n > 0
    for ws, size in ((None, 1 << 30), (0x100010, 1 << 30), (0x100000, n - 1)):
        assert lib.wisp_kv_reserve_append_rope(ctypes.byref(a), ctypes.c_void_p(ws), size, None) == WORKSPACE


def test_binding_refuses_what_it_can_see():
    import torch

    from paper_2601_11652_gb300 import binding as wb
    with pytest.raises(ValueError):
        wb._rows_ptr(torch.zeros(2, 2, 64))
    with pytest.raises(ValueError):
        wb._check_scales(torch.zeros(4, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 2), None)
    with pytest.raises(ValueError):
        wb._check_scales(torch.zeros(4, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 3))


def test_queries_that_overlap_their_output(lib):
    """In place means the same packed rows; any other overlap would have rows read after they were written."""
    size = 4 * 8 * 128 * 2
    call = lambda **kw: lib.wisp_kv_reserve_append_rope(ctypes.byref(_args(**kw)), ctypes.c_void_p(0x100000), 1, None)
    for kw in (dict(q_out=0x80000, q_stride=8 * 128 + 8), dict(q_out=0x80000 + 16), dict(q_out=0x80000 - 16),
               dict(q_out=0x80000 + size - 16), dict(q_out=0x80000 + size, q_stride=8 * 128 + 8)):
        assert call(**kw) == INVALID, kw
    # (these reach the check of the workspace, which is too small)
    for kw in (dict(q_out=0x80000), dict(q_out=0x80000, q_stride=8 * 128), dict(q_out=0x80000 + size), dict(q_out=0x80000 - size),
               dict(q_out=0x80000, Hq=0), dict(kv=dict(B=1, total_q_rows=1), q_out=0x80000, q_stride=16 * 128)):
        assert call(**kw) == WORKSPACE, kw


def test_commit_refusals(lib):
    call = lambda a, ws=0x100000, size=1: lib.wisp_kv_commit_rope(ctypes.byref(a) if a else None, ctypes.c_void_p(ws), size, None)
    new = dict(k_new=None, v_new=None, k_cache=None, v_cache=None)
    good = dict(kv=dict(accepted_len=0xa0000, **new), q=None, q_out=None, rope=None, k_scale=None, v_scale=None)
    assert call(_args(**good)) == WORKSPACE  # (taken, but for its workspace: it moves no rows)
    assert call(None) == INVALID and call(_args(**good), None, 1 << 30) == WORKSPACE
    for kw in (dict(kv=dict(new)), dict(rope_positions=0), dict(rot_dim=-16), dict(kv=dict(accepted_len=0xa0000, free_count=None))):
        assert call(_args(**{**good, **kw})) == INVALID, kw


def _tensors(**kw):
    import torch
    t, d = torch.zeros, dict(dtype=torch.bfloat16)
    i = lambda *s: t(s, dtype=torch.int32)
    base = dict(draft_lens=i(2), context_lens=i(2), block_tables=i(2, 4), free_blocks=i(8), free_count=i(1), k_new=t(4, 2, 64, **d),
                v_new=t(4, 2, 64, **d), q=t(4, 8, 64, **d), q_out=t(4, 8, 64, **d), k_cache=t(8, 2, 16, 64, dtype=torch.uint8),
                v_cache=t(8, 2, 16, 64, dtype=torch.uint8), k_scale=t(8, 2), v_scale=t(8, 2), rope=t(64, 64))
    return {**base, **kw}


def test_binding_refuses_rows_that_would_be_read_out_of_range():
    """Shapes, types and strides that the library cannot see are refused before any pointer is taken (so without a GPU, too)."""
    import torch

    from paper_2601_11652_gb300 import binding as wb
    t, d = torch.zeros, dict(dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensors only"):  # (nothing else is wrong with these)
        wb.make_kv_rope_args(**_tensors())
    bad = [dict(k_new=t(1, 2, 64, **d).expand(4, 2, 64)), dict(v_new=t(1, 2, 64, **d).expand(4, 2, 64)),
           dict(q=t(1, 8, 64, **d).expand(4, 8, 64)), dict(k_new=t(1000, **d).as_strided((4, 2, 64), (64, 64, 1))),
           dict(v_new=t(4, 2, 64)), dict(v_new=t(4, 1, 64, **d)), dict(v_new=t(4, 2, 128, **d)), dict(v_new=t(3, 2, 64, **d)),
           dict(q=t(3, 8, 64, **d), q_out=t(3, 8, 64, **d)), dict(q_out=None), dict(total_q_rows=5), dict(rope=t(64)),
           dict(k_cache=t(8, 2, 16, 128, dtype=torch.uint8)), dict(k_new=t(4, 128, **d))]
    for kw in bad:
        with pytest.raises(ValueError) as e:
            wb.make_kv_rope_args(**_tensors(**kw))
        assert "device tensors only" not in str(e.value), kw
    attn = dict(draft_lens=t(2, dtype=torch.int32), context_lens=t(2, dtype=torch.int32), block_tables=t(2, 4, dtype=torch.int32),
                q=t(4, 8, 64, **d), out=t(4, 8, 64, **d), **{n: _tensors()[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")})
    for kw in (dict(num_blocks=9), dict(total_q_rows=5)):
        with pytest.raises(ValueError) as e:
            wb.make_attn_kv8_args(**attn, **kw)
        assert "device tensors only" not in str(e.value), kw
