"""wisp_prompt_attention and wisp_verify_attention_shared against their definition in 64 bits.

Bounds.  With A = sum_t w_t |v_t| (w the row's softmax weights) an output is off by at most 2^-8 |out| where it is rounded to bf16, and by
the weights' relative error times A.  With bf16 queries a weight is rounded to bf16 for the product: 2^-8.  A score's error d changes a
weight by a factor of up to exp(2 d): sums of |q k| / sqrt(D) stay below 64 here, so sums of up to 128 products in fp32 leave
d < 128 * 2^-24 * 64 = 2^-11, and 2^-10 covers it; the scaled score's rounding (below 93 * 2^-23) and the exponential's 2^-22 are far below.
With fp32 queries everything together stays below 2^-9.  A code * scale that is no bf16 value moves K and V by 2^-8 of themselves: for V
another 2^-8 A, for K a score by 2^-8 sum |q k| / sqrt(D), counted from the inputs."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
PAGE = 16
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2601_11652_gb300 import build
    build.build()


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype))).cuda()


class Case:
    """k, ctx: per request; runs: per request (id, pages) or None for the prompt operator.  Slots past the requests' tokens and
    pages of nobody hold NaN."""

    def __init__(self, seed, *, k, ctx, Hq=8, Hkv=2, D=128, dtype=BF, cache=None, runs=None, shuffle=True, sd=1.0, exact_scales=True,
                 spare=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.k, self.ctx, self.Hq, self.Hkv, self.D, self.runs = list(k), list(ctx), Hq, Hkv, D, runs
        self.exact_scales = exact_scales
        B, T = len(self.k), sum(self.k) + len(self.k)
        n = [(c + kk + PAGE) // PAGE for c, kk in zip(self.ctx, self.k)]
        lead = list(range(B))  # whose first pages a request has
        if runs:
            for r in range(1, B):
                if runs[r] == runs[r - 1] and runs[r][0] >= 0 and runs[r][1] > 0:
                    lead[r] = lead[r - 1]
        own = [n[r] - (runs[r][1] if lead[r] != r else 0) for r in range(B)]
        nb = sum(own) + 3
        ids = (rng.permutation(nb) if shuffle else np.arange(nb)).tolist()
        bt = np.full((B, max(n) + spare), -1, np.int32)
        at = 0
        for r in range(B):
            s = n[r] - own[r]
            bt[r, s:n[r]] = ids[at:at + own[r]]
            bt[r, :s] = bt[lead[r], :s]
            at += own[r]
        self.bt = bt.copy()
        if runs:  # entries that are not read
            for r in range(B):
                if lead[r] != r:
                    bt[r, :runs[r][1]] = 1 << 30
        self.t = dict(draft_lens=dev(self.k), context_lens=dev(self.ctx), block_tables=dev(bt),
                      q=(torch.randn((T, Hq, D), generator=g, device="cuda") * sd).to(dtype))
        if runs:
            self.t["shared_ids"], self.t["shared_pages"] = dev([x[0] for x in runs]), dev([x[1] for x in runs])
        self.val = {}
        for x in "kv":
            v = torch.randn((nb, Hkv, PAGE, D), generator=g, device="cuda")
            if cache == "e4m3":
                s = torch.exp2(torch.ceil(torch.log2(v.abs().amax((2, 3)) / 448)))
                if not exact_scales:
                    s = s * (1.0 + torch.rand((nb, Hkv), generator=g, device="cuda"))
                    s[torch.rand((nb, Hkv), generator=g, device="cuda") < 0.1] = 0
                code = (v / torch.where(s > 0, s, torch.ones_like(s))[:, :, None, None]).to(torch.float8_e4m3fn)
                self.t[x + "_cache"], self.t[x + "_scale"] = code, s
                self.val[x] = code.double() * s.double()[:, :, None, None]
            else:
                self.t[x + "_cache"] = v.to(dtype)
                self.val[x] = self.t[x + "_cache"].double()
            bits = self.t[x + "_cache"].view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[self.t[x + "_cache"].element_size()])
            nan = -1 if cache == "e4m3" else {BF: 0x7fc0, F32: 0x7fc00000}[dtype]
            if cache == "e4m3":
                nan = 0x7f
            for r in range(B):
                L = self.ctx[r] + self.k[r] + 1
                if L % PAGE and L > 0:
                    bits[int(self.bt[r, n[r] - 1]), :, L % PAGE:] = nan
            bits[torch.tensor(ids[at:], device="cuda")] = nan
        self.t["out"] = torch.full_like(self.t["q"], 77)

    def args(self):
        from paper_2601_11652_gb300 import binding as wb
        if self.runs:
            a = wb.make_shared_args(**self.t)
            return a, wb.wisp_verify_shared_workspace_size(a), wb.wisp_verify_attention_shared
        a = wb.make_prompt_args(**self.t)
        return a, wb.wisp_prompt_workspace_size(a), wb.wisp_prompt_attention

    def run(self, expect=0, stream=None):
        from paper_2601_11652_gb300 import binding as wb
        a, n, call = self.args()
        ws = wb.alloc_workspace(n)
        ws.fill_(0xA5)
        call(a, ws, stream)
        torch.cuda.synchronize()
        code, rid = wb.wisp_verify_get_device_status(ws)
        assert code == expect, (code, rid)
        return rid

    def row_of(self, r):
        return sum(self.k[:r]) + r

    def reference(self, r, a, b):
        """Rows a .. b of request r: outputs, weighted magnitudes, and how far a score may be off for its scale's sake."""
        t, g, c = self.t, self.Hq // self.Hkv, self.ctx[r]
        L = c + b
        ids = torch.from_numpy(self.bt[r, :(L + PAGE - 1) // PAGE].astype(np.int64)).cuda()
        K, V = (self.val[x][ids].permute(1, 0, 2, 3).reshape(self.Hkv, 1, -1, self.D)[:, :, :L] for x in "kv")
        at = self.row_of(r)
        q = t["q"][at + a:at + b].double().view(b - a, self.Hkv, g, self.D).permute(1, 2, 0, 3)
        see = torch.arange(L, device="cuda") <= c + torch.arange(a, b, device="cuda")[:, None]
        w = torch.softmax((q @ K.transpose(2, 3) / math.sqrt(self.D)).masked_fill(~see, -math.inf), dim=3)
        ref, mag = w @ V, w @ V.abs()
        off = 0.0
        if not self.exact_scales:
            off = 2.0 ** -8 * (q.abs() @ K.abs().transpose(2, 3)).amax(3, keepdim=True) / math.sqrt(self.D)
        back = lambda y: y.permute(2, 0, 1, 3).reshape(b - a, self.Hq, -1)
        return back(ref), back(mag), back(torch.expm1(2 * off)) if not self.exact_scales else 0.0

    def check(self, skipped=()):
        bf = self.t["out"].dtype == BF
        worst = 0.0
        for r, k in enumerate(self.k):
            if r in skipped or k < 0:
                continue
            at = self.row_of(r)
            for a in range(0, k + 1, 512):
                b = min(k + 1, a + 512)
                ref, mag, far = self.reference(r, a, b)
                got = self.t["out"][at + a:at + b].double()
                assert torch.isfinite(got).all(), (r, a)
                bound = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -10 + far + (0 if self.exact_scales else 2.0 ** -8)) * mag if bf \
                    else 2.0 ** -9 * mag
                worst = max(worst, ((got - ref).abs() / bound.clamp(min=1e-30)).max().item())
                assert worst <= 1, (r, a, worst)
        return worst


TYPES = [(BF, None), (BF, "e4m3"), (F32, None), (F32, "e4m3")]
HEADS = [(32, 8, 128), (28, 4, 128), (8, 8, 64), (32, 8, 64), (5, 1, 128), (16, 1, 64)]
SHAPES = {"one_token": ([0], [0]), "one_row_each": ([0, 0, 0, 0], [0, 1, 15, 300]), "small": ([1, 2, 15, 16, 17], [0, 0, 0, 0, 0]),
          "tiles": ([30, 31, 32, 63, 64, 65], [0, 1, 127, 128, 64, 63]), "mixed": ([199, 0, 500, 7, 128], [0, 700, 33, 1000, 129]),
          "chunk": ([40], [5000])}


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_prompts_match_the_definition(shape, heads, dtype, cache):
    k, ctx = SHAPES[shape]
    c = Case(len(shape) + sum(heads), k=k, ctx=ctx, Hq=heads[0], Hkv=heads[1], D=heads[2], dtype=dtype, cache=cache)
    c.run()
    c.check()


@pytest.mark.parametrize("g", [1, 2, 3, 7, 12, 43, 65, 127, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_heads_per_group(g, D, dtype):
    c = Case(g + D, k=[140, 3], ctx=[0, 260], Hq=2 * g, Hkv=2, D=D, dtype=dtype)
    c.run()
    c.check()


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 128, 129, 130, 192, 257])
@pytest.mark.parametrize("D", [64, 128])
def test_lengths_around_tiles(n, D):
    for Hq, Hkv in ((8, 2), (2, 2)):
        c = Case(n, k=[n - 1, n - 1], ctx=[0, 100], Hq=Hq, Hkv=Hkv, D=D, shuffle=False)
        c.run()
        c.check()


@pytest.mark.parametrize("n,ctx,Hq,Hkv,D", [(3000, 0, 8, 2, 128), (2047, 2049, 4, 4, 64), (1500, 9000, 4, 1, 128)])
def test_long_prompts(n, ctx, Hq, Hkv, D):
    c = Case(n, k=[n - 1], ctx=[ctx], Hq=Hq, Hkv=Hkv, D=D)
    c.run()
    c.check()


def runs_of(*groups):
    """(id, pages, requests) -> per request"""
    return [(i, p) for i, p, n in groups for _ in range(n)]


SHARED = {
    "two": (runs_of((0, 3, 2)), [0, 0], [48, 60]),
    "pages": (runs_of((5, 1, 3), (6, 7, 2), (6, 9, 3)), [0, 3, 1, 2, 0, 5, 0, 1], [16, 17, 31, 112, 127, 144, 145, 300]),
    "alone": (runs_of((0, 4, 1), (-1, 4, 2), (1, 0, 2), (2, 2, 1)), [1, 0, 2, 3, 0, 1], [64, 64, 70, 10, 0, 32]),
    "mixed": (runs_of((-1, 0, 1), (3, 40, 9), (-1, 0, 1), (4, 130, 5), (0, 2, 2)), list(range(9)) + [4, 0, 15, 1, 1, 7, 2, 0, 70],
              [5] + [640 + 37 * i for i in range(9)] + [800] + [2080, 2081, 2500, 2095, 2096] + [32, 33]),
    "many": (runs_of((0, 20, 70)), [i % 5 for i in range(70)], [320 + (i * 53) % 700 for i in range(70)]),
    "long": (runs_of((0, 500, 3)), [4, 0, 2], [8000, 8010, 8500])}


@pytest.mark.parametrize("shape", list(SHARED))
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_shared_prefixes_match_the_definition(shape, heads, dtype, cache):
    runs, k, ctx = SHARED[shape]
    c = Case(len(shape) + sum(heads), k=k, ctx=ctx, runs=runs, Hq=heads[0], Hkv=heads[1], D=heads[2], dtype=dtype, cache=cache)
    c.run()
    c.check()


def test_more_requests_than_the_planner_has_threads():
    B = 1100
    runs = runs_of((0, 2, 500), (1, 3, 530), (-1, 0, 30), (2, 1, 40))
    rng = np.random.default_rng(4)
    c = Case(4, k=rng.integers(0, 3, B).tolist(), ctx=[max(0, p) * PAGE + int(x) for (i, p), x in zip(runs, rng.integers(0, 90, B))], runs=runs,
             Hq=4, Hkv=2, D=64)
    c.run()
    c.check()
    p = Case(5, k=rng.integers(0, 40, B).tolist(), ctx=rng.integers(0, 90, B).tolist(), Hq=4, Hkv=2, D=64)
    p.run()
    p.check()


@pytest.mark.parametrize("B", [16, 17, 32, 33, 64, 65, 128, 129, 256, 257, 511, 512, 513])
@pytest.mark.parametrize("shared", [False, True])
def test_batches_around_the_planners_sizes(B, shared):
    """As many requests, and requests and runs, as the planner has threads, and one more; every run has one to three requests."""
    rng = np.random.default_rng(B)
    runs = None
    if shared:
        runs = [(i, 1 + i % 3) for i in range(B) for _ in range(1 + (i * 7) % 3)][:B]
    k = rng.integers(0, 4, B).tolist()
    c = Case(B, k=k, ctx=[(runs[r][1] * PAGE if shared else 0) + int(x) for r, x in enumerate(rng.integers(0, 40, B))], runs=runs, Hq=4, Hkv=2, D=64)
    c.run()
    c.check()


@pytest.mark.parametrize("B", [17, 33, 130])
def test_runs_of_one_request_each(B):
    """As many runs as requests, none of which shares anything."""
    c = Case(B, k=[r % 3 for r in range(B)], ctx=[16 + r for r in range(B)], runs=[(r, 1) for r in range(B)], Hq=2, Hkv=1, D=128)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("k,ctx", [([3], [40000]), ([0, 700, 2], [17000, 5, 33000])])
def test_more_chunks_than_the_planner_has_threads(dtype, cache, k, ctx):
    c = Case(11, k=k, ctx=ctx, Hq=4, Hkv=1, D=64, dtype=dtype, cache=cache)
    nan = ctx[0] + k[0]  # only the last row sees it, and its chunk is one of many
    c.run()
    c.check()
    before = c.t["out"].clone()
    put(c, "v", 0, nan, 7, math.nan)
    c.run()
    same = torch.ones_like(before, dtype=torch.bool)
    same[k[0], :, 7] = False
    assert torch.isnan(c.t["out"][k[0], :, 7]).all() and torch.equal(c.t["out"][same], before[same])


def bits_of(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def put(c, x, r, token, d, value):
    """Element d of all heads of token `token` of request r; returns the value as the cache holds it."""
    cache = c.t[x + "_cache"]
    page, slot = int(c.bt[r, token // PAGE]), token % PAGE
    if cache.dtype == torch.float8_e4m3fn:
        assert math.isnan(value)
        bits_of(cache)[page, :, slot, d] = 0x7f
    else:
        cache[page, :, slot, d] = value
    c.val[x][page, :, slot, d] = value


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (4, 4, 64), (14, 2, 64)])
@pytest.mark.parametrize("shared", [False, True])
def test_values_that_are_not_finite(dtype, cache, Hq, Hkv, D, shared):
    """They reach the rows that see them and no others, in their element; everything else is as without them."""
    k, ctx = [200, 3, 150], [96 + 70, 96, 96 + 1]
    c = Case(7, k=k, ctx=ctx, runs=runs_of((0, 6, 3)) if shared else None, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, cache=cache)
    inf, nan = math.inf, math.nan
    odd = [(0, ctx[0] + 50, 5, nan), (0, 100, 3, nan), (1, ctx[1] + 2, 1, nan), (2, ctx[2] + 149, 40, nan), (2, ctx[2] + 150, 41, nan)]
    if not cache:
        odd += [(0, ctx[0] + 60, 7, inf), (0, ctx[0] + 90, 7, -inf), (0, ctx[0] + 200, 63, -inf), (2, ctx[2], 8, inf), (2, ctx[2] + 128, 9, -inf)]
    if shared:
        odd.append((0, 17, 11, nan))  # in the pages of all
    clean = {x: c.val[x].clone() for x in "kv"}
    for r, t, d, v in odd:
        put(c, "v", r, t, d, v)
    c.val = clean
    for r, t, d, v in odd:
        c.val["v"][int(c.bt[r, t // PAGE]), :, t % PAGE, d] = 0
    c.run()
    bf = dtype == BF
    for r in range(3):
        at = c.row_of(r)
        ref, mag, _ = c.reference(r, 0, k[r] + 1)
        got = c.t["out"][at:at + k[r] + 1].double()
        want = ref.clone()
        pos = ctx[r] + torch.arange(k[r] + 1, device="cuda")
        for rr, t, d, v in odd:
            if rr == r or t < 96 and shared:
                sees = (pos >= t)[:, None].expand(-1, Hq)
                col = want[:, :, d]
                want[:, :, d] = torch.where(sees, torch.where(torch.isinf(col) & (col != v), nan, v if math.isnan(v) else v + 0 * col), col)
        fine = torch.isfinite(want)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
        bound = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -10) * mag if bf else 2.0 ** -9 * mag
        assert ((got - want).abs()[fine] <= bound[fine]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_keys_that_are_not_finite(dtype, D):
    """A NaN key makes the rows that see it NaN; scores of -inf weigh nothing, and a row that has no other is NaN."""
    k, ctx = [300], [0]
    c = Case(8, k=k, ctx=ctx, Hq=4, Hkv=2, D=D, dtype=dtype)
    c.t["q"][:, :, 0] = 1
    for t in range(130):
        put(c, "k", 0, t, 0, -math.inf)
    put(c, "k", 0, 280, 2, math.nan)
    c.run()
    got = c.t["out"].double()
    assert torch.isnan(got[:130]).all() and torch.isnan(got[280:]).all()
    c.val["k"][torch.isnan(c.val["k"])] = 0
    ref, mag, _ = c.reference(0, 130, 280)
    bound = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -10) * mag if dtype == BF else 2.0 ** -9 * mag
    assert ((got[130:280] - ref).abs() <= bound).all()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("grow", [1, -1])
def test_scores_that_grow_and_fall(dtype, cache, grow):
    """Maxima that move from tile to tile, by little and by hundreds of powers of two.  Scores are larger than elsewhere, so their error is
    counted from the inputs: 2^-17 of sum |q k| / sqrt(D) for the sums, as much again for scaling, both in numerator and denominator."""
    k, ctx = [700, 90], [0, 600]
    c = Case(9, k=k, ctx=ctx, Hq=4, Hkv=2, D=128, dtype=dtype, cache=cache, runs=None)
    for r in range(2):
        L = ctx[r] + k[r] + 1
        t = torch.arange((L + PAGE - 1) // PAGE * PAGE, device="cuda").view(-1, PAGE)
        pages = torch.from_numpy(c.bt[r, :len(t)].astype(np.int64)).cuda()
        e = torch.div(t[:, :1] if cache else t, 40, rounding_mode="floor")
        f = torch.exp2((e if grow > 0 else e[-1, -1] - e).float() * 0.5)
        if cache:
            c.t["k_scale"][pages] *= torch.exp2(torch.floor(torch.log2(f)))
            c.val["k"][pages] = c.t["k_cache"][pages].double() * c.t["k_scale"][pages].double()[:, :, None, None]
        else:
            x = (c.t["k_cache"][pages].float() * f[:, None, :, None]).to(dtype)
            c.t["k_cache"][pages], c.val["k"][pages] = x, x.double()
    c.run()
    for r in range(2):
        at, L = c.row_of(r), ctx[r] + k[r] + 1
        ref, mag, _ = c.reference(r, 0, k[r] + 1)
        ids = torch.from_numpy(c.bt[r, :(L + PAGE - 1) // PAGE].astype(np.int64)).cuda()
        K = c.val["k"][ids].permute(1, 0, 2, 3).reshape(2, 1, -1, 128)[:, :, :L].abs()
        q = c.t["q"][at:at + k[r] + 1].double().view(-1, 2, 2, 128).permute(1, 2, 0, 3).abs()
        see = torch.arange(L, device="cuda") <= ctx[r] + torch.arange(k[r] + 1, device="cuda")[:, None]
        S = (q @ K.transpose(2, 3) / math.sqrt(128)).masked_fill(~see, 0).amax(3).permute(2, 0, 1).reshape(k[r] + 1, 4, 1)
        far = torch.expm1(2 * 2.0 ** -16 * S)
        got = c.t["out"][at:at + k[r] + 1].double()
        bound = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -20 + far) * mag if dtype == BF else (2.0 ** -18 + far) * mag
        # (where the largest weights meet zeros of V.)  A weight below 2^-126 of the row's largest is no normal number and counts as zero: fewer
        # than 2^10 keys of |v| < 2^3 then leave out less than 2^-113.  With fp32 queries a weight has steps of 2^-36 of the row's largest: 2^-23
        bound = bound + (2.0 ** -113 if dtype == BF else 2.0 ** -23)
        assert torch.isfinite(got).all() and bool(((got - ref).abs() <= bound).all())


@pytest.mark.parametrize("D", [64, 128])
def test_scales_that_are_no_powers_of_two(D):
    for dtype in (BF, F32):
        c = Case(10, k=[150, 20], ctx=[30, 400], Hq=8, Hkv=2, D=D, dtype=dtype, cache="e4m3", exact_scales=dtype == F32)
        if dtype == F32:  # (any scale is exact in fp32)
            f = 1.0 + torch.rand(c.t["k_scale"].shape, device="cuda")
            c.t["k_scale"] *= f
            c.val["k"] *= f.double()[:, :, None, None]
        c.run()
        c.check()


def test_refused_requests_leave_the_others():
    from paper_2601_11652_gb300 import binding as wb
    # (too long for its table; a negative length; a block outside the pool; a prefix that is shorter than its shared pages)
    for bad, code in ((dict(ctx=100000), 1), (dict(k=-3), 1), (dict(block=1 << 29), 2), (dict(block=-5), 2), (dict(pages=40), 1)):
        for dtype in (BF, F32):
            runs = runs_of((1, 4, 2), (2, 40 if "pages" in bad else 5, 1), (1, 4, 2))
            c = Case(11, k=[5, 70, 9, 0, 30], ctx=[64, 200, 90, 70, 64], runs=runs if "pages" not in bad else runs_of((1, 4, 2), (2, 5, 1), (1, 4, 2)),
                     Hq=4, Hkv=2, D=64, dtype=dtype)
            skipped = [2]
            if "pages" in bad:
                c.t["shared_pages"][2] = 40
            if "ctx" in bad:
                c.t["context_lens"][2] = bad["ctx"]
            if "block" in bad:
                c.t["block_tables"][2, 3] = bad["block"]
            if "k" in bad:  # its one row stays in the offsets
                c = Case(11, k=[5, 70, 0, 0, 30], ctx=[64, 200, 90, 70, 64], runs=runs, Hq=4, Hkv=2, D=64, dtype=dtype)
                c.t["draft_lens"][2] = bad["k"]
            c.t["request_ids"] = torch.arange(900, 905, device="cuda")
            assert c.run(expect=code) == 902
            c.check(skipped=skipped)
    # a run whose first request is refused takes its pages from the next
    c = Case(12, k=[3, 4, 5], ctx=[64, 70, 80], runs=runs_of((1, 4, 3)), Hq=4, Hkv=2, D=64)
    c.t["block_tables"][1, :4] = torch.from_numpy(c.bt[0, :4]).cuda()
    c.t["context_lens"][0] = 1 << 20
    c.run(expect=1)
    c.check(skipped=[0])
    # rows that the caller's buffers do not have, and rows of nobody
    c = Case(13, k=[3, 40, 5], ctx=[64, 70, 80], Hq=4, Hkv=2, D=64)
    a = wb.make_prompt_args(**c.t, total_q_rows=4 + 41)
    ws = wb.alloc_workspace(wb.wisp_prompt_workspace_size(a))
    wb.wisp_prompt_attention(a, ws)
    assert wb.wisp_verify_get_device_status(ws)[0] == 1
    c.check(skipped=[2])
    assert (c.t["out"][45:] == 77).all()


def test_outputs_behind_the_last_request_stay():
    from paper_2601_11652_gb300 import binding as wb
    for runs in (None, runs_of((0, 2, 2))):
        c = Case(14, k=[3, 40], ctx=[64, 70], Hq=4, Hkv=2, D=128, runs=runs)
        rows = c.t["q"].shape[0]
        for n in ("q", "out"):
            c.t[n] = torch.cat([c.t[n], torch.full((300, 4, 128), 77, dtype=BF, device="cuda")])
        a = (wb.make_shared_args if runs else wb.make_prompt_args)(**c.t, total_q_rows=rows)
        size, call = (wb.wisp_verify_shared_workspace_size, wb.wisp_verify_attention_shared) if runs else \
            (wb.wisp_prompt_workspace_size, wb.wisp_prompt_attention)
        ws = wb.alloc_workspace(size(a))
        call(a, ws)
        assert wb.wisp_verify_get_device_status(ws)[0] == 0
        c.check()
        assert (c.t["out"][rows:] == 77).all()


def test_an_empty_batch():
    from paper_2601_11652_gb300 import binding as wb
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    t = dict(draft_lens=i(0), context_lens=i(0), block_tables=i(0, 1), q=torch.zeros((0, 4, 64), dtype=BF, device="cuda"),
             k_cache=torch.zeros((1, 2, 16, 64), dtype=BF, device="cuda"), v_cache=torch.zeros((1, 2, 16, 64), dtype=BF, device="cuda"))
    t["out"] = torch.empty_like(t["q"])
    a = wb.make_prompt_args(**t)
    ws = wb.alloc_workspace(wb.wisp_prompt_workspace_size(a))
    wb.wisp_prompt_attention(a, ws)
    assert wb.wisp_verify_get_device_status(ws)[0] == 0


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_repeats_to_the_bit_on_streams_and_in_graphs(dtype, cache):
    """Two cases on two streams at once, each with its workspace, then both captured and replayed on other inputs in the same buffers."""
    from paper_2601_11652_gb300 import binding as wb
    cases = [Case(15, k=[900, 3], ctx=[200, 5000], Hq=8, Hkv=2, D=128, dtype=dtype, cache=cache),
             Case(16, k=[3, 0, 7], ctx=[4000, 3900, 4100], runs=runs_of((0, 240, 3)), Hq=8, Hkv=2, D=64, dtype=dtype, cache=cache)]
    for c in cases:
        c.run()
        c.check()
    want = [c.t["out"].clone() for c in cases]
    calls = []
    for c in cases:
        c.t["out"].fill_(0)
        a, n, call = c.args()
        calls.append((a, wb.alloc_workspace(n), call))
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for (a, ws, call), s in zip(calls, streams):
            call(a, ws, s)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert torch.equal(c.t["out"], w)
    for c, (a, ws, call) in zip(cases, calls):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(a, ws)
        for f in (0.5, -1.0):
            c.t["q"].mul_(f)
            c.t["out"].fill_(0)
            g.replay()
            torch.cuda.synchronize()
            assert wb.wisp_verify_get_device_status(ws)[0] == 0
            c.check()


@pytest.mark.parametrize("shared", [False, True])
def test_a_graph_follows_lengths_and_runs(shared):
    """A captured call reads lengths, tables, runs and rows anew: replayed on another batch of as many requests and rows, in the same buffers."""
    from paper_2601_11652_gb300 import binding as wb
    pages = [8, 8, 3, 3, 3, 0]
    first = Case(18, k=[200, 3, 0, 9, 31, 1], ctx=[200, 129, 50, 48, 70, 0], Hq=8, Hkv=2, D=128, spare=600,
                 runs=list(zip([0, 0, 1, 1, 1, -1], pages)) if shared else None)
    then = Case(19, k=[0, 120, 0, 60, 60, 4], ctx=[17, 900, 64, 7000, 7001, 300], Hq=8, Hkv=2, D=128,
                runs=list(zip([3, -1, 2, 7, 7, 7], [1, 0, 4, 430, 430, 2])) if shared else None)
    have = then.t["k_cache"].shape[0]
    for x in "kv":  # (one pool that is large enough for both)
        pool = torch.full((have, 2, PAGE, 128), math.nan, dtype=BF, device="cuda")
        pool[:first.t[x + "_cache"].shape[0]] = first.t[x + "_cache"]
        first.t[x + "_cache"] = pool
    tables = torch.full_like(first.t["block_tables"], -1)
    tables[:, :then.t["block_tables"].shape[1]] = then.t["block_tables"]
    then.t["block_tables"] = tables
    inputs = [{n: t.clone() for n, t in c.t.items()} for c in (first, then)]
    a, n, call = first.args()
    buffers, ws = first.t, wb.alloc_workspace(n)
    call(a, ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(a, ws)
    for c, t in ((then, inputs[1]), (first, inputs[0]), (then, inputs[1])):
        for n in buffers:
            buffers[n].copy_(t[n])
        g.replay()
        torch.cuda.synchronize()
        assert wb.wisp_verify_get_device_status(ws)[0] == 0
        c.t = dict(t, out=buffers["out"])
        c.check()


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes, its pages from the far end."""
    nb = (1 << 32) // (8 * PAGE * 128 * 2) + 400
    for cache in (None, "e4m3"):
        c = Case(17, k=[300, 2], ctx=[40, 900], Hq=16, Hkv=8, D=128, cache=cache)
        have = c.t["k_cache"].shape[0]
        for x in "kv":
            big = torch.zeros((nb, 8, PAGE, 128), dtype=c.t["k_cache"].dtype, device="cuda")
            bits_of(big)[-have:] = bits_of(c.t[x + "_cache"])
            c.t[x + "_cache"] = big
            if cache:
                s = torch.zeros((nb, 8), device="cuda")
                s[-have:] = c.t[x + "_scale"]
                c.t[x + "_scale"] = s
        c.t["block_tables"] = torch.where(c.t["block_tables"] >= 0, c.t["block_tables"] + (nb - have), c.t["block_tables"])
        c.run()
        c.check()
        del big
        c.t.clear()
        torch.cuda.empty_cache()
