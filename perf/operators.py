"""The operators around the verification step that a server runs beside it, as cases that can be timed and compared.

A case names one operator (`op`) and the shape of the batch it is called on:

  append     wisp_kv_reserve_append_rope: the new rows of the fused QKV projection, the position rotation, the write into
             the paged cache (of the rows' own type, or e4m3 with a power-of-two scale per page and KV head)
  attention  wisp_verify_attention_kv8: the k + 1 new queries of each request over a paged e4m3 cache with a scale per
             page and KV head
  logprobs   wisp_verify_logprobs: log probability of a given token of each row, the row's entropy, its top alternatives

`own` false: `run` computes the operator from elementary torch operations in fp32; true: through the library.  Lengths follow
from the case alone (every seed does the same amount of work); every tensor, the order of the requests and the placement of
the pages follow from the seed.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda"
E4M3_MAX = 448.0
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------ cases
def _append(name, *, B, heads=(32, 8, 128), dtype="bf16", cache="e4m3", k=(1, 8), ctx=(512, 4096), rot=None, interleaved=False,
            positions=131072):
    c = {"op": "append", "B": B, "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "dtype": dtype, "cache": cache, "k_lo": k[0],
         "k_hi": k[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1], "rot": heads[2] if rot is None else rot, "interleaved": interleaved,
         "positions": positions}
    return {"name": name, **c} if name else c


def _attention(name, *, B, heads=(32, 8, 128), k=(1, 8), ctx=(512, 4096), shuffle=False):
    c = {"op": "attention", "B": B, "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "k_lo": k[0], "k_hi": k[1], "ctx_lo": ctx[0],
         "ctx_hi": ctx[1], "shuffle": shuffle}
    return {"name": name, **c} if name else c


def _logprobs(name, *, rows, V=128256, dtype="bf16", top=5, skipped=0, pad=0, sd=2.0):
    c = {"op": "logprobs", "rows": rows, "V": V, "dtype": dtype, "top": top, "skipped": skipped, "pad": pad, "sd": sd}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one decode token of one request: launches and latency count
        _append("append_b1", B=1, k=(0, 0), ctx=(1000, 1000)),
        # an ordinary round of drafts into an 8-bit cache
        _append("append_b256", B=256, k=(1, 16), ctx=(64, 16384)),
        # chunks of prompts being prefilled
        _append("append_prompt", B=8, k=(700, 1023), ctx=(0, 30000)),
        # a model in fp32 with a cache of its own type and a rotation of half the head, pairs interleaved
        _append("append_f32_b64", B=64, heads=(28, 4, 128), dtype="f32", cache="f32", k=(0, 12), ctx=(256, 8192), rot=64,
                interleaved=True),
        # one request alone on a lightly loaded server
        _attention("attention_b1", B=1, k=(4, 4), ctx=(4096, 4096)),
        # an ordinary batch of a serving engine
        _attention("attention_b32", B=32),
        # a small model's heads of 64, plain decode requests (k = 0) among the drafts, pages in no order
        _attention("attention_d64_b64", B=64, heads=(32, 8, 64), k=(0, 8), ctx=(256, 8192), shuffle=True),
        # the largest: few requests with very long contexts on a fragmented pool
        _attention("attention_long_b16", B=16, k=(4, 8), ctx=(32768, 131072), shuffle=True),
        # the answer to one decode step of one request
        _logprobs("logprobs_r1", rows=1, top=20),
        # the rows of an ordinary round; those past a rejection are skipped
        _logprobs("logprobs_r176", rows=176, skipped=50),
        # a full server: every draft row of 256 requests
        _logprobs("logprobs_r2432", rows=2432, top=20),
        # fp32 logits of an odd vocabulary, rows padded apart, no alternatives asked for
        _logprobs("logprobs_f32_r300", rows=300, V=50257, dtype="f32", top=0, pad=47),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "logprobs"])
    heads = rng.choice([(32, 8, 128), (28, 4, 128), (8, 2, 128), (32, 8, 64), (8, 2, 64), (4, 4, 64)])
    g = heads[0] // heads[1]
    if op == "append":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        B = _log_int(rng, 1, 512)
        k_hi = min(1023, _log_int(rng, 1, max(2, 8192 // B)) - 1)
        ctx = _log_int(rng, 16, 30000)
        return _append(None, B=B, heads=heads, dtype=dtype, cache=rng.choice(["e4m3", "e4m3", dtype]),
                       k=(rng.randint(0, k_hi), k_hi), ctx=(rng.randint(0, ctx), ctx), rot=rng.choice([heads[2], heads[2] // 2]),
                       interleaved=rng.random() < 0.3)
    if op == "attention":
        B = _log_int(rng, 1, 256)
        k_hi = rng.randint(0, min(16, 128 // g - 1))
        most = min(131072, 1200000 * 8 * 128 // (B * heads[1] * heads[2]))
        hi = _log_int(rng, 32, most)
        return _attention(None, B=B, heads=heads, k=(rng.randint(0, k_hi), k_hi), ctx=(rng.randint(0, hi), hi),
                          shuffle=rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    rows = _log_int(rng, 1, 2432)
    V = _log_int(rng, 1000, min(152064, 300000000 // rows))
    if rng.random() < 0.6:  # most vocabularies are padded to a multiple of 64, some are not
        V = (V + 63) // 64 * 64
    return _logprobs(None, rows=rows, V=V, dtype=dtype, top=rng.choice([0, 1, 5, 8, 20, 32]), skipped=rng.randint(0, rows // 2),
                     pad=rng.choice([0, 0, 64, 47]), sd=rng.choice([1.0, 2.0, 4.0]))


def _lengths(c):
    """Draft and context lengths of the batch: of the case alone."""
    r = np.random.default_rng([c["B"], c["k_hi"], c["ctx_hi"], c["D"], 7])
    return r.integers(c["k_lo"], c["k_hi"] + 1, c["B"]), r.integers(c["ctx_lo"], c["ctx_hi"] + 1, c["B"])


def _touched(c):
    """Per request: pages that its new rows touch, and slots of its first one that are in use already."""
    k, ctx = _lengths(c)
    return (ctx + k) // PAGE - ctx // PAGE + 1, ctx % PAGE


def work(case):
    c = case
    if c["op"] == "logprobs":
        n = c["rows"] - c["skipped"]
        es = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": n * (c["V"] * es + 4) + c["rows"] * (8 + 8 * c["top"]), "flops": 5 * n * c["V"]}
    k, ctx = _lengths(c)
    T, H, D = int(k.sum()) + c["B"], c["Hkv"], c["D"]
    if c["op"] == "append":
        es, cs = (2 if c["dtype"] == "bf16" else 4), (1 if c["cache"] == "e4m3" else 2 if c["cache"] == "bf16" else 4)
        b = T * (2 * c["Hq"] + 2 * H) * D * es + T * 2 * H * D * cs + T * 4 * c["rot"]
        if c["cache"] == "e4m3":
            pages, old = _touched(c)
            b += 2 * H * (int(pages.sum()) * 4 + int((old * D).sum()) + int((old > 0).sum()) * 4)
        return {"bytes": b, "flops": 3 * T * (c["Hq"] + H) * c["rot"]}
    L = ctx + k + 1
    b = int(L.sum()) * 2 * H * D + int(((L + PAGE - 1) // PAGE).sum()) * (2 * H * 4 + 4) + 2 * T * c["Hq"] * D * 2
    seen = (k + 1) * (ctx + 1) + k * (k + 1) // 2  # visible (query, key) pairs
    return {"bytes": b, "flops": 4 * int(seen.sum()) * c["Hq"] * D}


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _scale_of(amax):
    """The power of two 2^e with the least e such that amax <= 448 2^e (1 for amax = 0)."""
    m, e = torch.frexp(amax)
    e = (e - 9 + (m > 0.875).to(e.dtype)).clamp(-96, 120)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.ones_like(amax))


def _channels(gen, H, D, dtype=torch.float32):
    """Standard deviations of a cache's channels: 1, a few outliers of 4 (keys have such channels)."""
    return 1.0 + 3.0 * (torch.rand((H, 1, D), generator=gen, device=DEV) < 0.03).to(dtype)


def _cache8(gen, pages, H, D, sd):
    """A pool of `pages` full e4m3 pages and their scales."""
    codes = torch.empty((pages, H, PAGE, D), dtype=torch.uint8, device=DEV)
    scale = torch.empty((pages, H), dtype=torch.float32, device=DEV)
    step = max(1, (64 << 20) // (H * PAGE * D))
    for a in range(0, pages, step):
        x = torch.randn((min(step, pages - a), H, PAGE, D), generator=gen, device=DEV) * sd
        s = _scale_of(x.abs().amax(dim=(2, 3)))
        scale[a:a + step] = s
        codes[a:a + step] = (x / s[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.view(torch.float8_e4m3fn), scale


def _prepare_logprobs(c, seed):
    gen = _gen(seed)
    wide = torch.randn((c["rows"], c["V"] + c["pad"]), generator=gen, device=DEV, dtype=DT[c["dtype"]]).mul_(c["sd"])
    tokens = torch.randint(0, c["V"], (c["rows"],), generator=gen, device=DEV, dtype=torch.int32)
    # some tokens are likely ones
    likely = wide[:, :c["V"]].argmax(dim=1).to(torch.int32)
    tokens = torch.where(torch.rand(c["rows"], generator=gen, device=DEV) < 0.5, likely, tokens)
    tokens[torch.randperm(c["rows"], generator=gen, device=DEV)[:c["skipped"]]] = -1
    f = lambda *s: torch.empty(s, dtype=torch.float32, device=DEV)  # noqa: E731
    t = {"logits": wide[:, :c["V"]], "tokens": tokens, "logprob": f(c["rows"]), "entropy": f(c["rows"])}
    if c["top"]:
        t["top_tokens"], t["top_logprobs"] = torch.empty((c["rows"], c["top"]), dtype=torch.int32, device=DEV), f(c["rows"], c["top"])
    return {"op": "logprobs", "top": c["top"], "t": t}


def _prepare_append(c, seed):
    gen, host = _gen(seed), np.random.default_rng([int(seed), 11])
    k, ctx = _lengths(c)
    order = host.permutation(c["B"])
    k, ctx = k[order], ctx[order]
    B, T, H, D, dt = c["B"], int(k.sum()) + c["B"], c["Hkv"], c["D"], DT[c["dtype"]]
    first, last = ctx // PAGE, (ctx + k) // PAGE
    # pages in front of the new rows: 64 pages of a prefix that the requests share; from there on each has its own
    mine = last - first + 1
    shared, num = 64, 64 + int(mine.sum())
    ids = shared + host.permutation(num - shared)
    bt = np.full((B, int(last.max()) + 1), -1, dtype=np.int32)
    at = 0
    for r in range(B):
        bt[r, :first[r]] = host.integers(0, shared, first[r])
        bt[r, first[r]:last[r] + 1] = ids[at:at + mine[r]]
        at += int(mine[r])
    qkv = torch.randn((T, (c["Hq"] + 2 * H) * D), generator=gen, device=DEV, dtype=dt)
    sd = _channels(gen, H, D).reshape(1, H * D)
    qkv[:, c["Hq"] * D:(c["Hq"] + H) * D] *= sd.to(dt)
    q, kn, vn = qkv.split([c["Hq"] * D, H * D, H * D], dim=1)
    t = {"draft_lens": _i32(k), "context_lens": _i32(ctx), "block_tables": _i32(bt), "free_blocks": _i32(np.zeros(num)),
         "free_count": _i32([0]), "q": q.unflatten(1, (c["Hq"], D)), "k_new": kn.unflatten(1, (H, D)),
         "v_new": vn.unflatten(1, (H, D)), "q_out": torch.empty((T, c["Hq"], D), dtype=dt, device=DEV)}
    if c["cache"] == "e4m3":
        t["k_cache"], t["k_scale"] = _cache8(gen, num, H, D, sd.reshape(H, 1, D))
        t["v_cache"], t["v_scale"] = _cache8(gen, num, H, D, 1.0)
    else:
        t["k_cache"] = torch.randn((num, H, PAGE, D), generator=gen, device=DEV, dtype=DT[c["cache"]])
        t["v_cache"] = torch.randn((num, H, PAGE, D), generator=gen, device=DEV, dtype=DT[c["cache"]])
    # cosines and sines of every position, as a model makes them once
    inv = 500000.0 ** (-torch.arange(0, c["rot"], 2, device=DEV, dtype=torch.float64) / c["rot"])
    angle = torch.arange(c["positions"], device=DEV, dtype=torch.float64)[:, None] * inv
    t["rope"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    return {"op": "append", "t": t, "T": T, "pages": int(max(mine)), "interleaved": c["interleaved"], "rot": c["rot"]}


def _prepare_attention(c, seed):
    gen, host = _gen(seed), np.random.default_rng([int(seed), 11])
    k, ctx = _lengths(c)
    order = host.permutation(c["B"])
    k, ctx = k[order], ctx[order]
    B, T, H, D = c["B"], int(k.sum()) + c["B"], c["Hkv"], c["D"]
    nblk = (ctx + k + PAGE) // PAGE
    num = int(nblk.sum())
    ids = host.permutation(num) if c["shuffle"] else np.arange(num)
    bt = np.full((B, int(nblk.max())), -1, dtype=np.int32)
    at = 0
    for r in range(B):
        bt[r, :nblk[r]] = ids[at:at + nblk[r]]
        at += int(nblk[r])
    t = {"draft_lens": _i32(k), "context_lens": _i32(ctx), "block_tables": _i32(bt),
         "q": torch.randn((T, c["Hq"], D), generator=gen, device=DEV, dtype=torch.bfloat16)}
    t["k_cache"], t["k_scale"] = _cache8(gen, num, H, D, _channels(gen, H, D))
    t["v_cache"], t["v_scale"] = _cache8(gen, num, H, D, 1.0)
    t["out"] = torch.empty_like(t["q"])
    return {"op": "attention", "t": t, "k_max": int(k.max())}


def prepare(case, seed):
    return {"append": _prepare_append, "attention": _prepare_attention, "logprobs": _prepare_logprobs}[case["op"]](case, seed)


# ------------------------------------------------------------------------------------------ plain forms
def _plain_logprobs(s):
    t = s["t"]
    z, tok = t["logits"].float(), t["tokens"].long()
    m = z.amax(dim=1, keepdim=True)
    d = z - m
    e = d.exp()
    tot = e.sum(dim=1, keepdim=True)
    lse = tot.log()
    on = tok >= 0
    zero = torch.zeros_like(m[:, 0])
    out = {"logprob": torch.where(on, d.gather(1, tok.clamp(min=0)[:, None])[:, 0] - lse[:, 0], zero),
           "entropy": torch.where(on, lse[:, 0] - (e * d).sum(dim=1) / tot[:, 0], zero)}
    if s["top"]:
        best, ids = torch.sort(d, dim=1, descending=True, stable=True)
        out["top_tokens"] = torch.where(on[:, None], ids[:, :s["top"]], -1).to(torch.int32)
        out["top_logprobs"] = torch.where(on[:, None], best[:, :s["top"]] - lse, zero[:, None])
    return out


def _rows(t, T):
    """Request and index within the request of every query row."""
    n = t["draft_lens"].long() + 1
    r = torch.repeat_interleave(torch.arange(n.numel(), device=n.device), n, output_size=T)
    return r, torch.arange(T, device=n.device) - (n.cumsum(0) - n)[r]


def _rotate(x, cos, sin, rot, interleaved):
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    cos, sin = cos[:, None, :], sin[:, None, :]
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], dim=-1).flatten(-2) if interleaved else torch.cat([u, v], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_append(s):
    t = s["t"]
    T, rot = s["T"], s["rot"]
    r, j = _rows(t, T)
    ctx = t["context_lens"].long()
    pos = ctx[r] + j
    cos, sin = t["rope"][pos].split([rot // 2, rot // 2], dim=1)
    t["q_out"].copy_(_rotate(t["q"], cos, sin, rot, s["interleaved"]))
    new = {"k": _rotate(t["k_new"], cos, sin, rot, s["interleaved"]), "v": t["v_new"].float()}
    bt = t["block_tables"].long()
    out = {"q_out": t["q_out"]}
    if "k_scale" not in t:
        page = bt[r, pos // PAGE]
        t["k_cache"][page, :, pos % PAGE] = new["k"].to(t["k_cache"].dtype)
        t["v_cache"][page, :, pos % PAGE] = new["v"].to(t["v_cache"].dtype)
        return {**out, "k_cache": t["k_cache"], "v_cache": t["v_cache"]}
    # the pages that new rows touch, padded to s["pages"] per request
    B, P = bt.shape[0], s["pages"]
    first, used = ctx // PAGE, ctx % PAGE
    slot = torch.arange(P * PAGE, device=DEV)
    filled = slot[None] < (used + t["draft_lens"].long() + 1)[:, None]
    ids = bt.gather(1, (first[:, None] + torch.arange(P, device=DEV)).clamp(max=bt.shape[1] - 1))

    def write(cache, scale, x):
        H, D = x.shape[1:]
        raw = cache.view(torch.uint8)
        buf = torch.zeros((B, P * PAGE, H, D), device=DEV)
        old = raw[ids[:, 0]].view(torch.float8_e4m3fn).float() * scale[ids[:, 0]][:, :, None, None]
        keep = (slot[None, :PAGE] < used[:, None])[:, :, None, None]
        buf[:, :PAGE] = torch.where(keep, old.transpose(1, 2), buf[:, :PAGE])
        buf[r, used[r] + j] = x
        buf = buf.view(B, P, PAGE, H, D)
        sc = _scale_of(buf.abs().amax(dim=(2, 4)))
        codes = (buf / sc[:, :, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        live = filled.view(B, P, PAGE)
        touched = live[:, :, 0]
        scale[ids[touched]] = sc[touched]
        raw[ids[:, :, None].expand(B, P, PAGE)[live], :, (slot % PAGE)[None].expand(B, -1)[filled]] = codes[live]

    write(t["k_cache"], t["k_scale"], new["k"])
    write(t["v_cache"], t["v_scale"], new["v"])
    return {**out, "k_cache": t["k_cache"], "v_cache": t["v_cache"], "k_scale": t["k_scale"], "v_scale": t["v_scale"]}


def _plain_attention(s):
    t = s["t"]
    T, Hq, D = t["q"].shape
    bt = t["block_tables"].long().clamp(min=0)
    B, H, n = bt.shape[0], t["k_cache"].shape[1], s["k_max"] + 1
    g = Hq // H

    def paged(cache, scale):
        x = cache.view(torch.uint8)[bt].view(torch.float8_e4m3fn).float()
        return (x * scale[bt][..., None, None]).transpose(1, 2).flatten(2, 3)

    k, v = paged(t["k_cache"], t["k_scale"]), paged(t["v_cache"], t["v_scale"])
    r, j = _rows(t, T)
    q = torch.zeros((B, n, Hq, D), device=DEV)
    q[r, j] = t["q"].float()
    q = q.view(B, n, H, g, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * g, D)
    sc = q @ k.transpose(2, 3) / math.sqrt(D)
    seen = torch.arange(k.shape[2], device=DEV) <= (t["context_lens"].long()[:, None] + torch.arange(n, device=DEV))[:, :, None]
    seen = seen[:, None, :, None].expand(B, 1, n, g, k.shape[2]).reshape(B, 1, n * g, k.shape[2])
    sc = torch.where(seen, sc, -math.inf)
    e = (sc - sc.amax(dim=3, keepdim=True)).exp()
    o = e @ v / e.sum(dim=3, keepdim=True)
    o = o.view(B, H, n, g, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    t["out"].copy_(o[r, j])
    return t["out"]


# ------------------------------------------------------------------------------------------ the library's calls
def _handle(s):
    """Argument struct and workspace of the call: a user's program fills them once for its buffers."""
    from paper_2601_11652_gb300 import binding as wb

    t = s["t"]
    if s["op"] == "append":
        a = wb.make_kv_rope_args(**t, total_q_rows=s["T"], interleaved=s["interleaved"])
        return a, wb.alloc_workspace(wb.wisp_kv_rope_workspace_size(a)), wb.wisp_kv_reserve_append_rope
    if s["op"] == "attention":
        a = wb.make_attn_kv8_args(**t)
        return a, wb.alloc_workspace(wb.wisp_verify_workspace_size(a.attn, None)), wb.wisp_verify_attention_kv8
    a = wb.make_logprobs_args(**t)
    return a, wb.alloc_workspace(wb.wisp_verify_logprobs_workspace_size(a)), wb.wisp_verify_logprobs


def run(state):
    s = state
    if not own:
        return {"append": _plain_append, "attention": _plain_attention, "logprobs": _plain_logprobs}[s["op"]](s)
    if "handle" not in s:
        s["handle"] = _handle(s)
    args, ws, call = s["handle"]
    call(args, ws)
    t = s["t"]
    if s["op"] == "append":
        return {n: t[n] for n in ("q_out", "k_cache", "v_cache", "k_scale", "v_scale") if n in t}
    if s["op"] == "attention":
        return t["out"]
    return {n: t[n] for n in ("logprob", "entropy", "top_tokens", "top_logprobs") if n in t}


# ------------------------------------------------------------------------------------------ in 64 bits
def _exact_logprobs(c, t):
    out = {n: [] for n in ("logprob", "entropy", "top_logprobs")}
    tokens = t["tokens"].tolist()
    for i, tok in enumerate(tokens):
        z = t["logits"][i].double()
        lse = torch.logsumexp(z, 0)
        lp = z - lse
        out["logprob"].append(lp[tok] if tok >= 0 else torch.zeros_like(lse))
        out["entropy"].append(-(lp.exp() * lp).sum() if tok >= 0 else torch.zeros_like(lse))
        if c["top"]:
            out["top_logprobs"].append(torch.topk(lp, c["top"]).values if tok >= 0 else torch.zeros_like(lp[:c["top"]]))
    got = {n: torch.stack(v) for n, v in out.items() if v}
    return {**got, "top_tokens": None} if c["top"] else got


def _exact_append(c, t):
    k, ctx = t["draft_lens"].tolist(), t["context_lens"].tolist()
    half, D = c["rot"] // 2, c["D"]
    first = torch.arange(half, device=DEV) * 2 if c["interleaved"] else torch.arange(half, device=DEV)
    second = first + (1 if c["interleaved"] else half)
    pos = torch.cat([torch.arange(a, a + n + 1, device=DEV) for a, n in zip(ctx, k)])
    table = t["rope"][pos].double()
    turn = torch.complex(table[:, :half], table[:, half:])[:, None]

    def turned(x):
        x = x.double()
        w = torch.complex(x[..., first], x[..., second]) * turn
        y = x.clone()
        y[..., first], y[..., second] = w.real, w.imag
        return y

    out = {"q_out": turned(t["q"])}
    rows = {"k": turned(t["k_new"]), "v": t["v_new"].double()}
    tables = t["block_tables"].cpu().numpy()
    for n in "kv":
        eight = n + "_scale" in t
        cache = t[n + "_cache"].double()
        scale = t[n + "_scale"].double() if eight else None
        at = 0
        for r in range(c["B"]):
            p, end = ctx[r], ctx[r] + k[r] + 1
            while p < end:
                page, lo = int(tables[r, p // PAGE]), p % PAGE
                hi = min(PAGE, lo + end - p)
                fresh = rows[n][at:at + hi - lo].transpose(0, 1)
                if eight:
                    live = torch.cat([cache[page, :, :lo] * scale[page][:, None, None], fresh], dim=1)
                    peak = live.abs().amax(dim=(1, 2))
                    s = torch.pow(2.0, torch.ceil(torch.log2(torch.clamp(peak, min=1e-300) / E4M3_MAX)))
                    s = torch.where(peak <= s / 2 * E4M3_MAX, s / 2, s)  # a logarithm of 2^n that comes out above n
                    s = torch.where(peak > 0, s, torch.ones_like(s))
                    scale[page] = s
                    cache[page, :, :hi] = live / s[:, None, None]
                else:
                    cache[page, :, lo:hi] = fresh
                at += hi - lo
                p += hi - lo
        if eight:
            out[n + "_scale"] = scale
        out[n + "_cache"] = cache
    return out


def _exact_attention(c, t):
    g, at = c["Hq"] // c["Hkv"], 0
    out = torch.empty(t["q"].shape, dtype=torch.float64, device=DEV)
    for r, (k, ctx) in enumerate(zip(t["draft_lens"].tolist(), t["context_lens"].tolist())):
        L = ctx + k + 1
        ids = t["block_tables"][r, :(L + PAGE - 1) // PAGE].long()
        val = {}
        for n in "kv":
            x = t[n + "_cache"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * t[n + "_scale"][ids].double()[:, :, None, None]
            val[n] = x.permute(1, 0, 2, 3).reshape(c["Hkv"], -1, c["D"])[:, :L]
        for i in range(k + 1):
            n = ctx + i + 1
            q = t["q"][at + i].double().view(c["Hkv"], g, c["D"])
            p = torch.softmax(torch.einsum("hgd,htd->hgt", q, val["k"][:, :n]) * c["D"] ** -0.5, dim=2)
            out[at + i] = torch.einsum("hgt,htd->hgd", p, val["v"][:, :n]).reshape(c["Hq"], c["D"])
        at += k + 1
    return out


def exact(case, seed):
    if case["op"] == "append" and case["B"] * (case["k_hi"] + 1) > 40000:
        return None
    t = prepare(case, seed)["t"]
    return {"append": _exact_append, "attention": _exact_attention, "logprobs": _exact_logprobs}[case["op"]](case, t)
