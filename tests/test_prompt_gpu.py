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
