"""The attention that a server runs beside the verification step, as cases that can be timed and compared.

A case names one operator (`op`) and the shape of the batch it is called on:

  prompt     wisp_prompt_attention: the queries of whole prompts, or of chunks of prompts behind a cached prefix, packed one
             after the other, over the paged cache that holds their keys and values; causal, grouped heads
  shared     wisp_verify_attention_shared: the k + 1 new queries of each request of a batch whose requests begin with the same
             pages (a system prompt), run by run

The cache has the queries' type, or holds e4m3 codes with a scale per page and KV head.

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
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
MOST_SCORES = 9_000_000_000      # scores that a drawn case's plain form holds at once
MOST_CACHE = 11_000_000_000      # elements of the keys that it gathers
MOST_FLOPS = 2.2e12
MOST_BYTES = 3.2e9


# ------------------------------------------------------------------------------------------ cases
def _prompt(name, *, B, n, ctx=(0, 0), heads=(32, 8, 128), dtype="bf16", cache=None, shuffle=False):
    c = {"op": "prompt", "B": B, "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "dtype": dtype, "cache": cache or dtype, "n_lo": n[0],
         "n_hi": n[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1], "shuffle": shuffle}
    return {"name": name, **c} if name else c


def _shared(name, *, B, prefix, runs=1, n=(1, 9), ctx=(64, 1024), heads=(32, 8, 128), dtype="bf16", cache=None, shuffle=True):
    c = {"op": "shared", "B": B, "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "dtype": dtype, "cache": cache or dtype, "n_lo": n[0],
         "n_hi": n[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1], "prefix": prefix, "runs": runs, "shuffle": shuffle}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the shortest prompt that is worth a call of its own: latency counts
        _prompt("prompt_n64", B=1, n=(64, 64)),
        # one user's prompt on an idle server
        _prompt("prompt_n2000", B=1, n=(2000, 2000)),
        # chunks of prompts behind what is cached already, as a chunked prefill packs them
        _prompt("prompt_chunks_b8", B=8, n=(700, 1024), ctx=(0, 30000), shuffle=True),
        # a batch of short prompts of different lengths, from one token on, heads of 64
        _prompt("prompt_d64_b48", B=48, n=(1, 1500), heads=(32, 8, 64), shuffle=True),
        # the largest: one long document
        _prompt("prompt_n16384", B=1, n=(16384, 16384)),
        # prompts into an 8-bit cache, seven query heads to a KV head
        _prompt("prompt_kv8_b6", B=6, n=(500, 4000), ctx=(0, 2000), heads=(28, 4, 128), cache="e4m3"),
        # a small model in fp32
        _prompt("prompt_f32_b5", B=5, n=(100, 900), heads=(8, 2, 64), dtype="f32"),
        # two requests behind a short system prompt
        _shared("shared_b2", B=2, prefix=1024, n=(1, 1), ctx=(40, 200)),
        # an ordinary batch of drafts behind a long system prompt
        _shared("shared_b64", B=64, prefix=8192),
        # four system prompts, decode steps and drafts among each other
        _shared("shared_b256_runs4", B=256, prefix=4096, runs=4, n=(1, 13), ctx=(16, 3000), heads=(28, 4, 128)),
        # the largest: many requests behind a book's worth of instructions
        _shared("shared_b256", B=256, prefix=16384, n=(1, 9), ctx=(128, 2048)),
        # an 8-bit cache and heads of 64
        _shared("shared_kv8_b100", B=100, prefix=6000, runs=3, n=(1, 5), ctx=(1, 1500), heads=(32, 8, 64), cache="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    while True:
        heads = rng.choice([(32, 8, 128), (28, 4, 128), (8, 2, 128), (32, 8, 64), (8, 2, 64), (4, 4, 64), (16, 1, 128)])
        kind = rng.choice([("bf16", None), ("bf16", None), ("bf16", None), ("bf16", "e4m3"), ("f32", None), ("f32", "e4m3")])
        if rng.random() < 0.5:
            B, n, ctx = _log_int(rng, 1, 64), _log_int(rng, 1, 16384), rng.choice([0, _log_int(rng, 1, 30000)])
            c = _prompt(None, B=B, n=(rng.randint(1, n), n), ctx=(rng.randint(0, ctx), ctx), heads=heads, dtype=kind[0], cache=kind[1],
                        shuffle=rng.random() < 0.5)
        else:
            B, n, ctx = _log_int(rng, 2, 256), rng.randint(1, 16), _log_int(rng, 1, 4000)
            c = _shared(None, B=B, prefix=_log_int(rng, 16, 16384), runs=rng.randint(1, max(1, min(6, B // 2))), n=(rng.randint(1, n), n),
                        ctx=(rng.randint(0, ctx), ctx), heads=heads, dtype=kind[0], cache=kind[1], shuffle=rng.random() < 0.7)
        L = c["ctx_hi"] + c["n_hi"] + c.get("prefix", 0)
        scores, cached, w = c["B"] * c["Hq"] * c["n_hi"] * L, c["B"] * c["Hkv"] * c["D"] * L, work(c)
        slower = 20 if c["dtype"] == "f32" else 1  # (fp32 products)
        if scores <= MOST_SCORES and cached <= MOST_CACHE and w["flops"] * slower <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


def _lengths(c):
    """New rows, keys in front of them (behind the shared pages, where there are any) and shared pages of each request."""
    r = np.random.default_rng([c["B"], c["n_hi"], c["ctx_hi"], c["D"], 7])
    n, ctx = r.integers(c["n_lo"], c["n_hi"] + 1, c["B"]), r.integers(c["ctx_lo"], c["ctx_hi"] + 1, c["B"])
    if c["op"] == "prompt":
        return n, ctx, np.zeros(c["B"], dtype=np.int64), np.zeros(c["B"], dtype=np.int64)
    # runs of about equal size; their prefixes shorter from run to run
    run = np.arange(c["B"]) * c["runs"] // c["B"]
    pages = np.maximum(1, c["prefix"] // PAGE - run * (c["prefix"] // PAGE // 8))
    return n, ctx, run, pages


def work(case):
    c = case
    n, ctx, run, pages = _lengths(c)
    T, H, D = int(n.sum()), c["Hkv"], c["D"]
    es, cs = (2 if c["dtype"] == "bf16" else 4), {"bf16": 2, "f32": 4, "e4m3": 1}[c["cache"]]
    first = np.array([pages[run == i][0] for i in np.unique(run)])
    keys = int((ctx + n).sum()) + int(first.sum()) * PAGE
    b = 2 * T * c["Hq"] * D * es + 2 * keys * H * D * cs + (keys // PAGE) * (4 + (8 * H if cs == 1 else 0))
    seen = n * (ctx + pages * PAGE) + n * (n + 1) // 2
    return {"bytes": b, "flops": 4 * int(seen.sum()) * c["Hq"] * D}


# ------------------------------------------------------------------------------------------ inputs
def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _cache(gen, c, pages, sd):
    """A pool of `pages` full pages, and scales of an 8-bit one: the least powers of two that keep a page's values in range."""
    shape = (pages, c["Hkv"], PAGE, c["D"])
    if c["cache"] != "e4m3":
        return torch.randn(shape, generator=gen, device=DEV, dtype=DT[c["cache"]]).mul_(sd.to(DT[c["cache"]])), None
    codes = torch.empty(shape, dtype=torch.float8_e4m3fn, device=DEV)
    scale = torch.empty(shape[:2], device=DEV)
    step = max(1, (64 << 20) // (c["Hkv"] * PAGE * c["D"]))
    for a in range(0, pages, step):
        x = torch.randn((min(step, pages - a), *shape[1:]), generator=gen, device=DEV) * sd
        scale[a:a + step] = torch.exp2(torch.ceil(torch.log2(x.abs().amax(dim=(2, 3)) / 448.0)))
        codes[a:a + step] = (x / scale[a:a + step, :, None, None]).to(torch.float8_e4m3fn)
    return codes, scale


def prepare(case, seed):
    c = case
    gen, host = torch.Generator(device=DEV), np.random.default_rng([int(seed), 11])
    gen.manual_seed(int(seed) * 1000003 + 31)
    n, ctx, run, pages = _lengths(c)
    # the order within a run is the seed's
    order = np.concatenate([host.permutation(np.flatnonzero(run == i)) for i in np.unique(run)])
    n, ctx = n[order], ctx[order]
    B, T, D = c["B"], int(n.sum()), c["D"]
    mine = (ctx + n + PAGE - 1) // PAGE
    first = [int(pages[run == i][0]) for i in np.unique(run)]
    num = int(mine.sum()) + sum(first)
    ids = host.permutation(num) if c["shuffle"] else np.arange(num)
    bt = np.full((B, int((mine + pages).max())), -1, dtype=np.int32)
    at = 0
    for i, r in enumerate(np.unique(run)):
        bt[run == r, :first[i]] = ids[at:at + first[i]]
        at += first[i]
    for r in range(B):
        bt[r, pages[r]:pages[r] + mine[r]] = ids[at:at + mine[r]]
        at += int(mine[r])
    t = {"draft_lens": _i32(n - 1), "context_lens": _i32(ctx + pages * PAGE), "block_tables": _i32(bt),
         "q": torch.randn((T, c["Hq"], D), generator=gen, device=DEV, dtype=DT[c["dtype"]])}
    # a few channels of the keys are larger than the others
    sd = 1.0 + 3.0 * (torch.rand((c["Hkv"], 1, D), generator=gen, device=DEV) < 0.03)
    t["k_cache"], ks = _cache(gen, c, num, sd)
    t["v_cache"], vs = _cache(gen, c, num, torch.ones((), device=DEV))
    if ks is not None:
        t["k_scale"], t["v_scale"] = ks, vs
    t["out"] = torch.empty_like(t["q"])
    if c["op"] == "shared":
        t["shared_ids"], t["shared_pages"] = _i32(run), _i32(pages)
    return {"op": c["op"], "t": t, "n_max": int(n.max())}


# ------------------------------------------------------------------------------------------ plain form
def _plain(s):
    t = s["t"]
    T, Hq, D = t["q"].shape
    bt = t["block_tables"].long().clamp(min=0)
    B, H, n = bt.shape[0], t["k_cache"].shape[1], s["n_max"]
    g = Hq // H

    def paged(name):
        cache = t[name + "_cache"]
        if name + "_scale" not in t:
            return cache[bt].transpose(1, 2).flatten(2, 3).float()
        x = cache.view(torch.uint8)[bt].view(torch.float8_e4m3fn).float().mul_(t[name + "_scale"][bt][..., None, None])
        return x.transpose(1, 2).flatten(2, 3)

    rows = t["draft_lens"].long() + 1
    r = torch.repeat_interleave(torch.arange(B, device=DEV), rows, output_size=T)
    j = torch.arange(T, device=DEV) - (rows.cumsum(0) - rows)[r]
    q = torch.zeros((B, n, Hq, D), device=DEV)
    q[r, j] = t["q"].float()
    q = q.view(B, n, H, g, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * g, D)
    sc = (q / math.sqrt(D)) @ paged("k").transpose(2, 3)
    behind = torch.arange(sc.shape[3], device=DEV) > (t["context_lens"].long()[:, None] + torch.arange(n, device=DEV))[:, :, None]
    sc.view(B, H, n, g, -1).masked_fill_(behind[:, None, :, None], -math.inf)
    sc.sub_(sc.amax(dim=3, keepdim=True)).exp_()
    o = sc @ paged("v") / sc.sum(dim=3, keepdim=True)
    o = o.view(B, H, n, g, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    t["out"].copy_(o[r, j])
    return t["out"]


# ------------------------------------------------------------------------------------------ the library's calls
def _handle(s):
    """Argument struct and workspace of the call: a user's program fills them once for its buffers."""
    from paper_2601_11652_gb300 import binding as wb

    if s["op"] == "prompt":
        a = wb.make_prompt_args(**s["t"])
        return a, wb.alloc_workspace(wb.wisp_prompt_workspace_size(a)), wb.wisp_prompt_attention
    a = wb.make_shared_args(**s["t"])
    return a, wb.alloc_workspace(wb.wisp_verify_shared_workspace_size(a)), wb.wisp_verify_attention_shared


def run(state):
    s = state
    if not own:
        return _plain(s)
    if "handle" not in s:
        s["handle"] = _handle(s)
    args, ws, call = s["handle"]
    call(args, ws)
    return s["t"]["out"]


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    c = case
    t = prepare(c, seed)["t"]
    g, at = c["Hq"] // c["Hkv"], 0
    out = torch.empty(t["q"].shape, dtype=torch.float64, device=DEV)
    for r, (k, ctx) in enumerate(zip(t["draft_lens"].tolist(), t["context_lens"].tolist())):
        L = ctx + k + 1
        ids = t["block_tables"][r, :(L + PAGE - 1) // PAGE].long()
        val = {}
        for x in "kv":
            y = t[x + "_cache"].view(torch.uint8)[ids].view(t[x + "_cache"].dtype).double()
            if x + "_scale" in t:
                y *= t[x + "_scale"][ids].double()[:, :, None, None]
            val[x] = y.permute(1, 0, 2, 3).reshape(c["Hkv"], 1, -1, c["D"])[:, :, :L]
        # blocks of rows, each over the keys that its last one sees
        for a in range(0, k + 1, 256):
            b = min(k + 1, a + 256)
            q = t["q"][at + a:at + b].double().view(b - a, c["Hkv"], g, c["D"]).permute(1, 2, 0, 3)
            p = q @ val["k"][:, :, :ctx + b].transpose(2, 3) * c["D"] ** -0.5
            p += torch.cat([p.new_zeros((b - a, ctx + a)), p.new_full((b - a, b - a), -math.inf).triu(1)], dim=1)
            o = torch.softmax(p, dim=3) @ val["v"][:, :, :ctx + b]
            out[at + a:at + b] = o.permute(2, 0, 1, 3).reshape(b - a, c["Hq"], c["D"])
        at += k + 1
    return out
