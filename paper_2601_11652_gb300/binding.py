"""ctypes binding of libwisp_verify.so (include/wisp_verify.h): argument marshalling only.

Every entry point of the C ABI has a Python function of the same name here.
Arguments are torch CUDA tensors (their data_ptr() is passed) or plain ints;
streams default to torch's current stream.  There is no CPU path: importing
this module without the built library, or calling it without a CUDA device,
raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import build as _build

WISP_OK, WISP_ERR_INVALID_ARG, WISP_ERR_UNSUPPORTED, WISP_ERR_CUDA, WISP_ERR_WORKSPACE = range(5)
WISP_F32, WISP_BF16, WISP_E4M3 = 0, 1, 2
DEVICE_CODES = {0: "ok", 1: "bad_length", 2: "bad_block", 3: "bad_token", 4: "bad_prob", 5: "unsupported",
                6: "timeout"}

_P = ctypes.c_void_p
_I32 = ctypes.c_int32


class wisp_attn_args(ctypes.Structure):
    _fields_ = [("B", _I32), ("Hq", _I32), ("Hkv", _I32), ("D", _I32), ("block_size", _I32),
                ("max_blocks_per_seq", _I32), ("num_blocks", _I32), ("total_q_rows", _I32),
                ("request_ids", _P), ("draft_lens", _P), ("context_lens", _P), ("block_tables", _P),
                ("qkv_dtype", ctypes.c_int), ("q", _P), ("k_cache", _P), ("v_cache", _P), ("out", _P)]


class wisp_accept_args(ctypes.Structure):
    _fields_ = [("B", _I32), ("V", _I32), ("total_q_rows", _I32), ("total_draft", _I32),
                ("request_ids", _P), ("draft_lens", _P), ("logits_dtype", ctypes.c_int),
                ("target_logits", _P), ("draft_tokens", _P), ("draft_probs", _P), ("accept_uniforms", _P),
                ("sample_uniforms", _P), ("accepted_len", _P), ("next_token", _P)]


class wisp_kv_args(ctypes.Structure):
    _fields_ = [("B", _I32), ("Hkv", _I32), ("D", _I32), ("block_size", _I32), ("max_blocks_per_seq", _I32),
                ("num_blocks", _I32), ("total_q_rows", _I32), ("request_ids", _P), ("draft_lens", _P),
                ("context_lens", _P), ("block_tables", _P), ("free_blocks", _P), ("free_count", _P),
                ("kv_dtype", ctypes.c_int), ("k_cache", _P), ("v_cache", _P), ("k_new", _P), ("v_new", _P),
                ("accepted_len", _P)]


class wisp_kv_rope_args(ctypes.Structure):
    _fields_ = [("kv", wisp_kv_args), ("cache_dtype", ctypes.c_int), ("k_scale", _P), ("v_scale", _P), ("rope", _P),
                ("rope_positions", _I32), ("rot_dim", _I32), ("interleaved", _I32), ("Hq", _I32), ("q", _P), ("q_out", _P),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


class wisp_attn_kv8_args(ctypes.Structure):
    _fields_ = [("attn", wisp_attn_args), ("k_scale", _P), ("v_scale", _P)]


class wisp_logprobs_args(ctypes.Structure):
    _fields_ = [("rows", _I32), ("V", _I32), ("row_stride", ctypes.c_int64), ("logits_dtype", ctypes.c_int), ("logits", _P),
                ("tokens", _P), ("top_n", _I32), ("logprob", _P), ("entropy", _P), ("top_tokens", _P), ("top_logprobs", _P)]


class wisp_prompt_args(ctypes.Structure):
    _fields_ = [("attn", wisp_attn_args), ("cache_dtype", ctypes.c_int), ("k_scale", _P), ("v_scale", _P)]


class wisp_shared_args(ctypes.Structure):
    _fields_ = [("rows", wisp_prompt_args), ("shared_ids", _P), ("shared_pages", _P)]


class WispError(RuntimeError):
    def __init__(self, fn: str, code: int, text: str):
        super().__init__(f"{fn}: {text} (status {code})")
        self.code = code


_lib = None

EXPORTED = ["wisp_verify_workspace_size", "wisp_verify_attention", "wisp_verify_accept", "wisp_verify_step",
            "wisp_verify_get_device_status", "wisp_verify_status_string", "wisp_verify_device_code_string",
            "wisp_verify_accept_noalloc", "wisp_verify_accept_greedy", "wisp_kv_workspace_size",
            "wisp_kv_reserve_append", "wisp_kv_commit", "wisp_kv_rope_workspace_size", "wisp_kv_reserve_append_rope",
            "wisp_kv_commit_rope", "wisp_verify_attention_kv8", "wisp_verify_step_kv8", "wisp_verify_logprobs_workspace_size", "wisp_verify_logprobs", "wisp_verify_committed_tokens",
            "wisp_prompt_workspace_size", "wisp_prompt_attention", "wisp_verify_shared_workspace_size",
            "wisp_verify_attention_shared"]


def lib_path() -> str:
    return _build.LIB_PATH


def load(path: str | None = None):
    """Load the shared library (built in-tree by build.py); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2601_11652_gb300.build` "
                           "(the verification step has no CPU implementation)")
    lib = ctypes.CDLL(path)
    AP, CP = ctypes.POINTER(wisp_attn_args), ctypes.POINTER(wisp_accept_args)
    lib.wisp_verify_workspace_size.argtypes = [AP, CP]
    lib.wisp_verify_workspace_size.restype = ctypes.c_size_t
    lib.wisp_verify_attention.argtypes = [AP, _P, ctypes.c_size_t, _P]
    lib.wisp_verify_attention.restype = ctypes.c_int
    lib.wisp_verify_accept.argtypes = [CP, _P, ctypes.c_size_t, _P]
    lib.wisp_verify_accept.restype = ctypes.c_int
    lib.wisp_verify_step.argtypes = [AP, CP, _P, ctypes.c_size_t, _P]
    lib.wisp_verify_step.restype = ctypes.c_int
    lib.wisp_verify_accept_greedy.argtypes = [CP, _P, ctypes.c_size_t, _P]
    lib.wisp_verify_accept_greedy.restype = ctypes.c_int
    lib.wisp_verify_accept_noalloc.argtypes = [CP, _P]
    lib.wisp_verify_accept_noalloc.restype = ctypes.c_int
    lib.wisp_verify_get_device_status.argtypes = [_P, ctypes.POINTER(_I32), ctypes.POINTER(ctypes.c_int64)]
    lib.wisp_verify_get_device_status.restype = ctypes.c_int
    lib.wisp_verify_status_string.argtypes = [ctypes.c_int]
    lib.wisp_verify_status_string.restype = ctypes.c_char_p
    lib.wisp_verify_device_code_string.argtypes = [_I32]
    lib.wisp_verify_device_code_string.restype = ctypes.c_char_p
    KP = ctypes.POINTER(wisp_kv_args)
    lib.wisp_kv_workspace_size.argtypes = [KP]
    lib.wisp_kv_workspace_size.restype = ctypes.c_size_t
    for fn in ("wisp_kv_reserve_append", "wisp_kv_commit"):
        getattr(lib, fn).argtypes = [KP, _P, ctypes.c_size_t, _P]
        getattr(lib, fn).restype = ctypes.c_int
    RP = ctypes.POINTER(wisp_kv_rope_args)
    lib.wisp_kv_rope_workspace_size.argtypes = [RP]
    lib.wisp_kv_rope_workspace_size.restype = ctypes.c_size_t
    for fn in ("wisp_kv_reserve_append_rope", "wisp_kv_commit_rope"):
        getattr(lib, fn).argtypes = [RP, _P, ctypes.c_size_t, _P]
        getattr(lib, fn).restype = ctypes.c_int
    A8 = ctypes.POINTER(wisp_attn_kv8_args)
    lib.wisp_verify_attention_kv8.argtypes = [A8, _P, ctypes.c_size_t, _P]
    lib.wisp_verify_attention_kv8.restype = ctypes.c_int
    lib.wisp_verify_step_kv8.argtypes = [A8, CP, _P, ctypes.c_size_t, _P]
    lib.wisp_verify_step_kv8.restype = ctypes.c_int
    LP = ctypes.POINTER(wisp_logprobs_args)
    lib.wisp_verify_logprobs_workspace_size.argtypes = [LP]
    lib.wisp_verify_logprobs_workspace_size.restype = ctypes.c_size_t
    lib.wisp_verify_logprobs.argtypes = [LP, _P, ctypes.c_size_t, _P]
    lib.wisp_verify_logprobs.restype = ctypes.c_int
    lib.wisp_verify_committed_tokens.argtypes = [CP, _P, _P]
    lib.wisp_verify_committed_tokens.restype = ctypes.c_int
    for fn, args in (("wisp_prompt_attention", wisp_prompt_args), ("wisp_verify_attention_shared", wisp_shared_args)):
        getattr(lib, fn).argtypes = [ctypes.POINTER(args), _P, ctypes.c_size_t, _P]
        getattr(lib, fn).restype = ctypes.c_int
    for fn, args in (("wisp_prompt_workspace_size", wisp_prompt_args), ("wisp_verify_shared_workspace_size", wisp_shared_args)):
        getattr(lib, fn).argtypes = [ctypes.POINTER(args)]
        getattr(lib, fn).restype = ctypes.c_size_t
    _lib = lib
    return lib


def _check(fn: str, code: int):
    if code != WISP_OK:
        raise WispError(fn, code, load().wisp_verify_status_string(code).decode())


def _ptr(t) -> int | None:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("device tensors only: the verification step runs on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _check_rows(t) -> None:
    if t.dim() != 3 or t.numel() and (t.stride(2) != 1 or t.shape[1] > 1 and t.stride(1) != t.shape[2]):
        raise ValueError("rows must be [rows, heads, D], the heads of a row contiguous")
    if t.shape[0] > 1 and t.stride(0) < t.shape[1] * t.shape[2]:  # (a stride of 0 would be read as packed rows)
        raise ValueError("rows must not overlap")


def _rows_ptr(t) -> tuple[int, int]:
    """Pointer and row stride (elements) of [rows, heads, D] rows that may lie apart, as parts of one projection output."""
    _check_rows(t)
    if not t.is_cuda:
        raise ValueError("device tensors only: the verification step runs on the GPU")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


def _cache_code(t: torch.Tensor) -> int:
    return WISP_E4M3 if t.dtype in (torch.float8_e4m3fn, torch.uint8) else _dtype_code(t)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return WISP_F32
    if t.dtype == torch.bfloat16:
        return WISP_BF16
    raise ValueError(f"unsupported dtype {t.dtype}")


def make_attn_args(*, draft_lens, context_lens, block_tables, q, k_cache, v_cache, out, request_ids=None,
                   num_blocks=None, total_q_rows=None) -> wisp_attn_args:
    """Fill wisp_attn_args from device tensors (shapes as in include/wisp_verify.h)."""
    B = draft_lens.shape[0]
    T_q, Hq, D = q.shape
    nb, Hkv, bs, D2 = k_cache.shape
    assert D2 == D and v_cache.shape == k_cache.shape and out.shape == q.shape and out.dtype == q.dtype
    a = wisp_attn_args()
    a.B, a.Hq, a.Hkv, a.D, a.block_size = B, Hq, Hkv, D, bs
    a.max_blocks_per_seq = block_tables.shape[1] if block_tables.dim() == 2 else 0
    a.num_blocks = nb if num_blocks is None else num_blocks
    a.total_q_rows = T_q if total_q_rows is None else total_q_rows
    a.request_ids, a.draft_lens, a.context_lens = _ptr(request_ids), _ptr(draft_lens), _ptr(context_lens)
    a.block_tables = _ptr(block_tables)
    a.qkv_dtype = _dtype_code(q)
    a.q, a.k_cache, a.v_cache, a.out = _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(out)
    return a


def make_accept_args(*, draft_lens, target_logits, draft_tokens, draft_probs, accept_uniforms,
                     sample_uniforms, accepted_len, next_token, request_ids=None, total_q_rows=None,
                     total_draft=None) -> wisp_accept_args:
    """Fill wisp_accept_args from device tensors (shapes as in include/wisp_verify.h)."""
    c = wisp_accept_args()
    c.B = draft_lens.shape[0]
    c.V = target_logits.shape[1]
    c.total_q_rows = target_logits.shape[0] if total_q_rows is None else total_q_rows
    c.total_draft = draft_tokens.shape[0] if total_draft is None else total_draft
    c.request_ids, c.draft_lens = _ptr(request_ids), _ptr(draft_lens)
    c.logits_dtype = _dtype_code(target_logits)
    c.target_logits = _ptr(target_logits)
    c.draft_tokens = _ptr(draft_tokens) if draft_tokens.numel() else None
    c.draft_probs = _ptr(draft_probs) if draft_probs.numel() else None
    c.accept_uniforms = _ptr(accept_uniforms) if accept_uniforms.numel() else None
    c.sample_uniforms, c.accepted_len, c.next_token = _ptr(sample_uniforms), _ptr(accepted_len), _ptr(next_token)
    return c


def wisp_verify_workspace_size(attn: wisp_attn_args | None, acc: wisp_accept_args | None) -> int:
    n = load().wisp_verify_workspace_size(ctypes.byref(attn) if attn else None, ctypes.byref(acc) if acc else None)
    if n == 0:
        raise WispError("wisp_verify_workspace_size", WISP_ERR_INVALID_ARG, "invalid arguments")
    return int(n)


def alloc_workspace(nbytes: int, device=None) -> torch.Tensor:
    """Caller-owned workspace (torch allocates; the library never does). 256-byte aligned."""
    t = torch.empty(nbytes + 256, dtype=torch.uint8, device=device or "cuda")
    off = (-t.data_ptr()) % 256
    return t[off: off + nbytes]


def wisp_verify_attention(attn: wisp_attn_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_verify_attention", load().wisp_verify_attention(
        ctypes.byref(attn), _ptr(workspace), workspace.numel(), _stream(stream)))


def wisp_verify_accept(acc: wisp_accept_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_verify_accept", load().wisp_verify_accept(
        ctypes.byref(acc), _ptr(workspace), workspace.numel(), _stream(stream)))


def wisp_verify_accept_greedy(acc: wisp_accept_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_verify_accept_greedy", load().wisp_verify_accept_greedy(
        ctypes.byref(acc), _ptr(workspace), workspace.numel(), _stream(stream)))


def wisp_verify_accept_noalloc(acc: wisp_accept_args, stream=None) -> None:
    _check("wisp_verify_accept_noalloc", load().wisp_verify_accept_noalloc(ctypes.byref(acc), _stream(stream)))


def wisp_verify_step(attn: wisp_attn_args, acc: wisp_accept_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_verify_step", load().wisp_verify_step(
        ctypes.byref(attn), ctypes.byref(acc), _ptr(workspace), workspace.numel(), _stream(stream)))


def wisp_verify_get_device_status(workspace: torch.Tensor) -> tuple[int, int]:
    code, rid = _I32(0), ctypes.c_int64(0)
    _check("wisp_verify_get_device_status",
           load().wisp_verify_get_device_status(_ptr(workspace), ctypes.byref(code), ctypes.byref(rid)))
    return int(code.value), int(rid.value)


# ---- paged KV maintenance (include/wisp_kv.h) ---------------------------------------------------
def make_kv_args(*, draft_lens, context_lens, block_tables, free_blocks, free_count, k_cache=None, v_cache=None,
                 k_new=None, v_new=None, accepted_len=None, request_ids=None, total_q_rows=None) -> wisp_kv_args:
    """Fill wisp_kv_args from device tensors (k_cache / v_cache [num_blocks, Hkv, 16, D])."""
    a = wisp_kv_args()
    a.B = draft_lens.shape[0]
    a.max_blocks_per_seq = block_tables.shape[1]
    a.num_blocks = free_blocks.shape[0]
    ref = k_cache if k_cache is not None else k_new
    a.Hkv = ref.shape[1] if ref is not None else 1
    a.D = ref.shape[-1] if ref is not None else 128
    a.block_size = 16
    a.total_q_rows = int(draft_lens.sum().item()) + a.B if total_q_rows is None else total_q_rows
    a.request_ids, a.draft_lens, a.context_lens = _ptr(request_ids), _ptr(draft_lens), _ptr(context_lens)
    a.block_tables, a.free_blocks, a.free_count = _ptr(block_tables), _ptr(free_blocks), _ptr(free_count)
    a.kv_dtype = _dtype_code(ref) if ref is not None else WISP_BF16
    a.k_cache, a.v_cache, a.k_new, a.v_new = _ptr(k_cache), _ptr(v_cache), _ptr(k_new), _ptr(v_new)
    a.accepted_len = _ptr(accepted_len)
    return a


def wisp_kv_workspace_size(kv: wisp_kv_args) -> int:
    n = load().wisp_kv_workspace_size(ctypes.byref(kv))
    if n == 0:
        raise WispError("wisp_kv_workspace_size", WISP_ERR_INVALID_ARG, "invalid arguments")
    return int(n)


def wisp_kv_reserve_append(kv: wisp_kv_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_kv_reserve_append", load().wisp_kv_reserve_append(
        ctypes.byref(kv), _ptr(workspace), workspace.numel(), _stream(stream)))


def wisp_kv_commit(kv: wisp_kv_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_kv_commit", load().wisp_kv_commit(ctypes.byref(kv), _ptr(workspace), workspace.numel(), _stream(stream)))


# ---- rotation on the way into the cache, 8-bit caches (include/wisp_kv8.h) ------------------------
def make_kv_rope_args(*, draft_lens, context_lens, block_tables, free_blocks, free_count, k_cache, v_cache, k_new, v_new,
                      rope=None, q=None, q_out=None, k_scale=None, v_scale=None, interleaved=False, request_ids=None,
                      total_q_rows=None, accepted_len=None) -> wisp_kv_rope_args:
    """Fill wisp_kv_rope_args from device tensors, for the append and (with accepted_len) the commit after it: k_new / v_new
    [rows, Hkv, D] and q [rows, Hq, D] (rows may lie apart), caches of their type or e4m3 (torch.float8_e4m3fn or uint8)
    with k_scale / v_scale [num_blocks, Hkv], rope [positions, rot_dim] of cosines and sines (None: no rotation)."""
    for t in (k_new, v_new, q):
        if t is not None:
            _check_rows(t)
    total = k_new.shape[0] if total_q_rows is None else total_q_rows
    if v_new.shape[1:] != k_new.shape[1:] or v_new.dtype != k_new.dtype:
        raise ValueError("k_new and v_new must be [rows, Hkv, D] of one type")
    if q is not None and (q_out is None or q.dtype != k_new.dtype or q_out.dtype != q.dtype or q_out.shape != q.shape or
                          q.shape[2:] != k_new.shape[2:]):
        raise ValueError("q and q_out go together, with the type and head dim of k_new")
    if min([t.shape[0] for t in (k_new, v_new, q) if t is not None]) < total:
        raise ValueError("k_new, v_new and q must have total_q_rows rows")
    if rope is not None and (rope.dtype != torch.float32 or rope.dim() != 2):
        raise ValueError("the rotation's table is float32 [positions, rot_dim]")
    if k_cache.dim() != 4 or k_cache.shape != v_cache.shape or k_cache.dtype != v_cache.dtype or k_cache.shape[1::2] != k_new.shape[1:]:
        raise ValueError("k_cache and v_cache must be [num_blocks, Hkv, 16, D] of one type")
    if k_cache.shape[0] < free_blocks.shape[0]:
        raise ValueError("free_blocks must not be longer than the pool")
    (kp, ks), (vp, vs) = _rows_ptr(k_new), _rows_ptr(v_new)
    a = wisp_kv_rope_args()
    a.kv = make_kv_args(draft_lens=draft_lens, context_lens=context_lens, block_tables=block_tables, free_blocks=free_blocks,
                        free_count=free_count, request_ids=request_ids, accepted_len=accepted_len,
                        total_q_rows=total)
    a.kv.Hkv, a.kv.D, a.kv.kv_dtype, a.cache_dtype = k_new.shape[1], k_new.shape[2], _dtype_code(k_new), _cache_code(k_cache)
    a.kv.block_size = k_cache.shape[2]
    a.kv.k_cache, a.kv.v_cache, a.kv.k_new, a.kv.v_new = _ptr(k_cache), _ptr(v_cache), kp, vp
    a.k_stride, a.v_stride = ks, vs
    if a.cache_dtype == WISP_E4M3:
        _check_scales(k_cache, k_scale, v_scale)
        a.k_scale, a.v_scale = _ptr(k_scale), _ptr(v_scale)
    if rope is not None:
        a.rope, a.rope_positions, a.rot_dim = _ptr(rope), rope.shape[0], rope.shape[1]
    a.interleaved = int(interleaved)
    if q is not None:
        a.Hq = q.shape[1]
        a.q, a.q_stride = _rows_ptr(q)
        a.q_out = _ptr(q_out)
    return a


def _check_scales(cache, *scales):
    for s in scales:
        if s is None or s.dtype != torch.float32 or tuple(s.shape) != tuple(cache.shape[:2]):
            raise ValueError("an 8-bit cache has float32 scales [num_blocks, Hkv]")


def wisp_kv_rope_workspace_size(a: wisp_kv_rope_args) -> int:
    n = load().wisp_kv_rope_workspace_size(ctypes.byref(a))
    if n == 0:
        raise WispError("wisp_kv_rope_workspace_size", WISP_ERR_INVALID_ARG, "invalid arguments")
    return int(n)


def wisp_kv_reserve_append_rope(a: wisp_kv_rope_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_kv_reserve_append_rope", load().wisp_kv_reserve_append_rope(
        ctypes.byref(a), _ptr(workspace), workspace.numel(), _stream(stream)))


def wisp_kv_commit_rope(a: wisp_kv_rope_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_kv_commit_rope", load().wisp_kv_commit_rope(ctypes.byref(a), _ptr(workspace), workspace.numel(), _stream(stream)))


def make_attn_kv8_args(*, draft_lens, context_lens, block_tables, q, k_cache, v_cache, k_scale, v_scale, out, request_ids=None,
                       num_blocks=None, total_q_rows=None) -> wisp_attn_kv8_args:
    """make_attn_args over an e4m3 cache (torch.float8_e4m3fn or uint8) with scales [num_blocks, Hkv]."""
    if _cache_code(k_cache) != WISP_E4M3 or v_cache.dtype != k_cache.dtype:
        raise ValueError("k_cache and v_cache must be e4m3 (torch.float8_e4m3fn or uint8)")
    if (num_blocks or 0) > k_cache.shape[0] or (total_q_rows or 0) > q.shape[0]:
        raise ValueError("num_blocks and total_q_rows must not be more than the pool and q have")
    _check_scales(k_cache, k_scale, v_scale)
    a = wisp_attn_kv8_args()
    a.attn = make_attn_args(draft_lens=draft_lens, context_lens=context_lens, block_tables=block_tables, q=q, k_cache=k_cache,
                            v_cache=v_cache, out=out, request_ids=request_ids, num_blocks=num_blocks, total_q_rows=total_q_rows)
    a.k_scale, a.v_scale = _ptr(k_scale), _ptr(v_scale)
    return a


def wisp_verify_attention_kv8(a: wisp_attn_kv8_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_verify_attention_kv8", load().wisp_verify_attention_kv8(
        ctypes.byref(a), _ptr(workspace), workspace.numel(), _stream(stream)))


def wisp_verify_step_kv8(a: wisp_attn_kv8_args, acc: wisp_accept_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_verify_step_kv8", load().wisp_verify_step_kv8(
        ctypes.byref(a), ctypes.byref(acc), _ptr(workspace), workspace.numel(), _stream(stream)))


# ---- log probabilities (include/wisp_logprobs.h) ----------------------------------------------------
def make_logprobs_args(*, logits, tokens, logprob, entropy=None, top_tokens=None, top_logprobs=None) -> wisp_logprobs_args:
    """Fill wisp_logprobs_args from device tensors: logits [rows, V] (rows may lie apart), tokens [rows] int32 (negative:
    the row is skipped), logprob / entropy [rows] float32, top_tokens int32 and top_logprobs float32 [rows, top_n]."""
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [rows, V], each row contiguous")
    rows, V = logits.shape
    if rows > 1 and logits.stride(0) < V:  # (expanded or overlapping: a stride of 0 would be read as packed rows)
        raise ValueError("the rows of logits must not overlap")
    if not logits.is_cuda:
        raise ValueError("device tensors only: the verification step runs on the GPU")
    if (top_tokens is None) != (top_logprobs is None):
        raise ValueError("top_tokens and top_logprobs go together")
    if tokens.dtype != torch.int32 or tokens.numel() != rows:
        raise ValueError("tokens must be [rows] int32")
    for t in (logprob, entropy):
        if t is not None and (t.dtype != torch.float32 or t.numel() != rows):
            raise ValueError("logprob and entropy must be [rows] float32")
    a = wisp_logprobs_args()
    a.rows, a.V = rows, V
    a.row_stride = logits.stride(0) if rows > 1 else 0
    a.logits_dtype = _dtype_code(logits)
    a.logits, a.tokens = logits.data_ptr(), _ptr(tokens)
    a.logprob, a.entropy = _ptr(logprob), _ptr(entropy)
    if top_tokens is not None:
        a.top_n = top_tokens.shape[1]
        if top_tokens.dtype != torch.int32 or top_logprobs.dtype != torch.float32 or top_tokens.shape[0] != rows or \
                top_logprobs.shape != top_tokens.shape:
            raise ValueError("top_tokens must be [rows, top_n] int32, top_logprobs the same in float32")
        a.top_tokens, a.top_logprobs = _ptr(top_tokens), _ptr(top_logprobs)
    return a


def wisp_verify_logprobs_workspace_size(a: wisp_logprobs_args) -> int:
    n = load().wisp_verify_logprobs_workspace_size(ctypes.byref(a))
    if n == 0:
        raise WispError("wisp_verify_logprobs_workspace_size", WISP_ERR_INVALID_ARG, "invalid arguments")
    return int(n)


def wisp_verify_logprobs(a: wisp_logprobs_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_verify_logprobs", load().wisp_verify_logprobs(
        ctypes.byref(a), _ptr(workspace), workspace.numel(), _stream(stream)))


def wisp_verify_committed_tokens(acc: wisp_accept_args, row_tokens: torch.Tensor, stream=None) -> None:
    if row_tokens.dtype != torch.int32 or row_tokens.numel() < acc.total_q_rows:
        raise ValueError("row_tokens must be [total_q_rows] int32")
    _check("wisp_verify_committed_tokens", load().wisp_verify_committed_tokens(
        ctypes.byref(acc), _ptr(row_tokens), _stream(stream)))


# ---- attention of whole prompts, and of batches that share pages (include/wisp_prompt.h) -------------
def make_prompt_args(*, draft_lens, context_lens, block_tables, q, k_cache, v_cache, out, k_scale=None, v_scale=None,
                     request_ids=None, num_blocks=None, total_q_rows=None) -> wisp_prompt_args:
    """Fill wisp_prompt_args from device tensors: as make_attn_args, without a limit on the query rows (draft_lens: rows - 1), over a
    cache of q's type or one in e4m3 (torch.float8_e4m3fn or uint8) with scales [num_blocks, Hkv]."""
    if q.dim() != 3 or out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("q and out must be [rows, Hq, D] of one type")
    if k_cache.dim() != 4 or k_cache.shape != v_cache.shape or k_cache.dtype != v_cache.dtype or k_cache.shape[3] != q.shape[2]:
        raise ValueError("k_cache and v_cache must be [num_blocks, Hkv, 16, D] of one type, with the head dim of q")
    B = draft_lens.numel()
    if block_tables.dim() != 2 or block_tables.shape[0] < B or context_lens.numel() < B or \
            any(t.dtype != torch.int32 for t in (draft_lens, context_lens, block_tables)):
        raise ValueError("draft_lens and context_lens must be [B], block_tables [B, max_blocks], int32")
    if request_ids is not None and (request_ids.dtype != torch.int64 or request_ids.numel() < B):
        raise ValueError("request_ids must be [B] int64")
    if (num_blocks or 0) > k_cache.shape[0] or (total_q_rows or 0) > q.shape[0]:
        raise ValueError("num_blocks and total_q_rows must not be more than the pool and q have")
    code = _cache_code(k_cache)
    if code != WISP_E4M3 and code != _dtype_code(q):
        raise ValueError("the cache has the queries' type or is e4m3")
    a = wisp_prompt_args()
    a.attn = make_attn_args(draft_lens=draft_lens, context_lens=context_lens, block_tables=block_tables, q=q, k_cache=k_cache,
                            v_cache=v_cache, out=out, request_ids=request_ids, num_blocks=num_blocks, total_q_rows=total_q_rows)
    a.cache_dtype = code
    if code == WISP_E4M3:
        _check_scales(k_cache, k_scale, v_scale)
        a.k_scale, a.v_scale = _ptr(k_scale), _ptr(v_scale)
    return a


def wisp_prompt_workspace_size(a: wisp_prompt_args) -> int:
    n = load().wisp_prompt_workspace_size(ctypes.byref(a))
    if n == 0:
        raise WispError("wisp_prompt_workspace_size", WISP_ERR_INVALID_ARG, "invalid arguments")
    return int(n)


def wisp_prompt_attention(a: wisp_prompt_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_prompt_attention", load().wisp_prompt_attention(
        ctypes.byref(a), _ptr(workspace), workspace.numel(), _stream(stream)))


def make_shared_args(*, shared_ids, shared_pages, draft_lens, **kw) -> wisp_shared_args:
    """Fill wisp_shared_args: make_prompt_args, and shared_ids / shared_pages [B] int32 (consecutive requests with the same id >= 0 and
    the same number of pages > 0 share their first pages)."""
    for t in (shared_ids, shared_pages):
        if t.dtype != torch.int32 or t.numel() < draft_lens.numel():
            raise ValueError("shared_ids and shared_pages must be [B] int32")
    a = wisp_shared_args()
    a.rows = make_prompt_args(draft_lens=draft_lens, **kw)
    a.shared_ids, a.shared_pages = _ptr(shared_ids), _ptr(shared_pages)
    return a


def wisp_verify_shared_workspace_size(a: wisp_shared_args) -> int:
    n = load().wisp_verify_shared_workspace_size(ctypes.byref(a))
    if n == 0:
        raise WispError("wisp_verify_shared_workspace_size", WISP_ERR_INVALID_ARG, "invalid arguments")
    return int(n)


def wisp_verify_attention_shared(a: wisp_shared_args, workspace: torch.Tensor, stream=None) -> None:
    _check("wisp_verify_attention_shared", load().wisp_verify_attention_shared(
        ctypes.byref(a), _ptr(workspace), workspace.numel(), _stream(stream)))
