"""wisp_verify_attention_kv8 against its definition in 64 bits.

Bounds.  With A = sum_t w_t |v_t| (w the row's softmax weights) an output is off by at most 2^-8 |out| where it is rounded
to bf16, and by the weights' relative error times A.  With bf16 queries a weight enters the product with 8 significant
bits: 2^-8.  A score's error d changes weights by up to 2 d, and scores here stay below 40 with sums of |q k| / sqrt(D) below
60, so fp32 sums of up to 128 products leave d < 128 * 2^-24 * 60 < 2^-11: another 2^-8 covers it.  In fp32 the two
together stay below 2^-9: the score's part is 2 * 2^-11 at the worst and 2^-13 in all cases here."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
PAGE = 16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2601_11652_gb300 import build
    build.build()


class Case:
    def __init__(self, seed, *, k, ctx, Hq=32, Hkv=8, D=128, dtype=torch.bfloat16, shuffle=True, garbage=True, scales="append", sd=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.k, self.ctx, self.Hq, self.Hkv, self.D = list(k), list(ctx), Hq, Hkv, D
        B, T = len(self.k), sum(self.k) + len(self.k)
        n = [(c + kk + PAGE) // PAGE for c, kk in zip(self.ctx, self.k)]
        nb = sum(n) + 3
        ids = (rng.permutation(nb) if shuffle else np.arange(nb)).tolist()
        bt = np.full((B, max(n) + 2), -1, np.int32)
        at = 0
        for r in range(B):
            bt[r, :n[r]] = ids[at:at + n[r]]
            at += n[r]
        d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.t = dict(draft_lens=d(np.array(self.k, np.int32)), context_lens=d(np.array(self.ctx, np.int32)), block_tables=d(bt),
                      q=(torch.randn((T, Hq, D), generator=g, device="cuda") * sd).to(dtype))
        for x in "kv":
            v = torch.randn((nb, Hkv, PAGE, D), generator=g, device="cuda")
            if scales == "append":
                s = torch.exp2(torch.ceil(torch.log2(v.abs().amax((2, 3)) / 448)))
            else:  # any finite value that is not negative
                s = torch.rand((nb, Hkv), generator=g, device="cuda") * 0.02
                s[torch.rand((nb, Hkv), generator=g, device="cuda") < 0.1] = 0
            code = (v / torch.where(s > 0, s, torch.ones_like(s))[:, :, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
            self.t[x + "_cache"], self.t[x + "_scale"] = code, s
        if garbage:  # slots past the requests' tokens and pages of nobody hold NaN codes
            for r in range(B):
                L = self.ctx[r] + self.k[r] + 1
                if L % PAGE:
                    for x in "kv":
                        self.t[x + "_cache"].view(torch.uint8)[int(bt[r, n[r] - 1]), :, L % PAGE:] = 0x7f
            for x in "kv":
                self.t[x + "_cache"].view(torch.uint8)[torch.tensor(ids[at:], device="cuda")] = 0xff
        self.t["out"] = torch.full_like(self.t["q"], 77)

    def run(self, expect=0, stream=None, acc=None):
        from paper_2601_11652_gb300 import binding as wb
        a = wb.make_attn_kv8_args(**self.t)
        ws = wb.alloc_workspace(wb.wisp_verify_workspace_size(a.attn, acc))
        if acc is None:
            wb.wisp_verify_attention_kv8(a, ws, stream)
        else:
            wb.wisp_verify_step_kv8(a, acc, ws, stream)
        torch.cuda.synchronize()
        code, rid = wb.wisp_verify_get_device_status(ws)
        assert code == expect, (code, rid)
        return rid

    def check(self, skipped=(), nan_ok=False):
        t, g = self.t, self.Hq // self.Hkv
        bf = t["out"].dtype == torch.bfloat16
        at, worst = 0, 0.0
        for r, (k, c) in enumerate(zip(self.k, self.ctx)):
            L = c + k + 1
            ids = t["block_tables"][r, :(L + PAGE - 1) // PAGE].long()
            rows = slice(at, at + k + 1)
            at += k + 1
            if r in skipped:
                continue
            def load(x):
                y = t[x + "_cache"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * t[x + "_scale"][ids].double()[:, :, None, None]
                return y.permute(1, 0, 2, 3).reshape(self.Hkv, -1, self.D)[:, :L]
            K, V = load("k"), load("v")
            q = t["q"][rows].double().view(k + 1, self.Hkv, g, self.D)
            s = torch.einsum("jhgd,htd->jhgt", q, K) / math.sqrt(self.D)
            seen = torch.arange(L, device="cuda") <= c + torch.arange(k + 1, device="cuda")[:, None]
            s = torch.where(seen[:, None, None], s, -math.inf)
            w = torch.softmax(s, dim=3)
            ref = torch.einsum("jhgt,htd->jhgd", w, V)
            A = torch.einsum("jhgt,htd->jhgd", w, V.abs())
            got = t["out"][rows].double().view(ref.shape)
            bound = (2.0 ** -8 * ref.abs() + 2.0 ** -7 * A) if bf else 2.0 ** -9 * A
            assert torch.isfinite(got).all()
            worst = max(worst, ((got - ref).abs() / bound.clamp(min=1e-30)).max().item())
            assert worst <= 1, (r, worst)
        return worst


SHAPES = {"one_token": ([0], [0]), "one_key_each": ([0, 0, 0], [0, 1, 15]), "pages": ([0, 1, 2, 3], [15, 16, 17, 14]),
          "tiles": ([3, 0, 4, 1, 2], [127, 128, 124, 255, 126]), "mixed": ([4, 0, 15, 7, 1], [1000, 4096, 333, 0, 2050]),
          "split": ([4], [20000])}


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (28, 4, 128), (8, 8, 64), (32, 8, 64), (5, 1, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matches_the_definition(shape, Hq, Hkv, D, dtype):
    k, ctx = SHAPES[shape]
    c = Case(len(shape) + Hq + D, k=k, ctx=ctx, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype)
    c.run()
    c.check()


@pytest.mark.parametrize("rows", [1, 7, 8, 9, 16, 17, 31, 33, 40, 48, 57, 63, 64, 65, 100, 128])
@pytest.mark.parametrize("D", [64, 128])
def test_row_counts(rows, D):
    # `rows` heads per KV head with one token each, and one head with `rows` tokens
    c = Case(rows, k=[0, 0], ctx=[700, 129], Hq=2 * rows, Hkv=2, D=D)
    c.run()
    c.check()
    c = Case(rows + 1, k=[rows - 1, rows - 1], ctx=[0, 300], Hq=2, Hkv=2, D=D)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_any_scales(dtype):
    c = Case(3, k=[5, 0, 9], ctx=[700, 90, 1], scales="any", dtype=dtype)
    c.run()
    c.check()


def test_pages_in_order_and_a_batch():
    c = Case(4, k=list(range(9)) * 4, ctx=[37 * i for i in range(36)], shuffle=False)
    c.run()
    c.check()


@pytest.mark.parametrize("D", [64, 128])
def test_many_items_of_mixed_row_counts(D):
    # several items per SM, of 4 to 64 query rows and one to a few dozen tiles, in one order after the other
    rng = np.random.default_rng(D)
    c = Case(40 + D, k=rng.integers(0, 16, 96), ctx=np.where(rng.random(96) < 0.5, rng.integers(0, 300, 96), rng.integers(0, 5000, 96)), D=D)
    c.run()
    c.check()
    a = c.t["out"].clone()
    c.run()
    assert torch.equal(a, c.t["out"])


@pytest.mark.parametrize("order", ["rising", "falling", "one_late", "one_early"])
def test_scores_far_apart(order):
    # keys whose scores rise or fall by hundreds along the sequence, or one key that takes nearly all
    c = Case(5, k=[3, 0], ctx=[3000, 900], Hq=4, Hkv=1, shuffle=False)
    t = c.t
    u = torch.randn(c.D, generator=torch.Generator().manual_seed(1)).cuda()
    t["q"] = (u + 0.1 * torch.randn(t["q"].shape, device="cuda")).to(torch.bfloat16)
    n = t["k_cache"].shape[0] * PAGE
    ramp = torch.linspace(-3, 3, n, device="cuda")
    if order == "falling":
        ramp = -ramp
    elif order.startswith("one"):
        ramp = torch.zeros(n, device="cuda")
        ramp[[60, 3100] if order == "one_early" else [2900, 3850]] = 2.0
    x = (ramp[:, None] * u).view(-1, 1, PAGE, c.D)
    t["k_scale"] = torch.full_like(t["k_scale"], 2.0 ** -5)
    t["k_cache"] = (x / 2.0 ** -5).to(torch.float8_e4m3fn)
    c.run()
    c.check()


def test_many_small_weights_beside_a_large_one():
    # one key with half of the weight and a value of zero: the output is the mean of the 60000 others
    c = Case(6, k=[0], ctx=[60000], Hq=4, Hkv=1, garbage=False, shuffle=False)
    t = c.t
    t["q"][:] = 1
    t["k_cache"].view(torch.uint8)[:] = 0
    t["k_scale"][:] = 2.0 ** -5
    t["v_scale"][:] = 2.0 ** -5
    gap = math.log(60000) * math.sqrt(c.D) / c.D
    t["k_cache"][0, 0, 3] = torch.full((c.D,), gap / 2.0 ** -5, device="cuda").to(torch.float8_e4m3fn)
    t["v_cache"] = ((1 + 0.3 * torch.randn(t["v_cache"].shape, device="cuda")) / 2.0 ** -5).to(torch.float8_e4m3fn)
    t["v_cache"].view(torch.uint8)[0, 0, 3] = 0
    c.run()
    c.check()


def test_a_nan_value_reaches_only_rows_that_see_it():
    c = Case(7, k=[6, 2], ctx=[250, 31], Hq=8, Hkv=2)
    bt = c.t["block_tables"]
    hit = {}
    for r, j, h, d in ((0, 3, 1, 17), (0, 5, 1, 17), (0, 6, 0, 100), (1, 0, 0, 0)):
        tok = c.ctx[r] + j
        c.t["v_cache"].view(torch.uint8)[int(bt[r, tok // PAGE]), h, tok % PAGE, d] = 0x7f
        hit[(r, h, d)] = min(j, hit.get((r, h, d), 99))
    # a NaN key: rows that see it have no softmax
    tok = c.ctx[1] + 2
    c.t["k_cache"].view(torch.uint8)[int(bt[1, tok // PAGE]), 1, tok % PAGE, 5] = 0xff
    c.run()
    out = c.t["out"].float().cpu().numpy().reshape(-1, 2, 4, c.D)
    want = np.zeros(out.shape, bool)
    for (r, h, d), j in hit.items():
        row = 7 * r
        want[row + j: row + c.k[r] + 1, h, :, d] = True
    want[7 + 2, 1] = True
    assert np.array_equal(np.isnan(out), want)


def test_a_nan_value_with_fp32_queries():
    # row 0 of request 1 sees its NaN value with a weight that underflows to zero
    c = Case(17, k=[6, 2], ctx=[250, 31], Hq=8, Hkv=2, dtype=torch.float32)
    bt, hit = c.t["block_tables"], {}
    for r, j, h, d in ((0, 3, 1, 17), (0, 5, 1, 17), (0, 6, 0, 100), (1, 0, 0, 0)):
        tok = c.ctx[r] + j
        c.t["v_cache"].view(torch.uint8)[int(bt[r, tok // PAGE]), h, tok % PAGE, d] = 0x7f
        hit[(r, h, d)] = min(j, hit.get((r, h, d), 99))
    c.t["q"][7:] *= 1e4
    c.run()
    out = c.t["out"].cpu().numpy().reshape(-1, 2, 4, c.D)
    want = np.zeros(out.shape, bool)
    for (r, h, d), j in hit.items():
        want[7 * r + j: 7 * r + c.k[r] + 1, h, :, d] = True
    assert np.array_equal(np.isnan(out), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite_reaches_only_its_own_row(dtype, value):
    c = Case(18, k=[6, 2, 12], ctx=[250, 31, 400], Hq=8, Hkv=2, dtype=dtype)
    at = ((3, 5, 77), (8, 0, 0), (8, 7, 127), (20, 2, 64))  # query row, head, element
    for row, h, d in at:
        c.t["q"][row, h, d] = 0
    c.run()
    before = c.t["out"].clone()
    for row, h, d in at:
        c.t["q"][row, h, d] = value
    c.run()
    hit = torch.zeros(c.t["out"].shape[:2], dtype=torch.bool, device="cuda")
    for row, h, d in at:
        hit[row, h] = True
    assert torch.isnan(c.t["out"][hit]).all() and torch.equal(c.t["out"][~hit], before[~hit])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("first", [0.0, 2.0 ** -90, 2.0 ** 60])
def test_value_scales_far_apart(first, D):
    # the first page's values have a scale of their own, and the rows' maxima fall by 2^29 from the first tile to the second
    c = Case(19, k=[10, 3, 15], ctx=[119, 300, 2000], Hq=8, Hkv=2, D=D)
    t, g = c.t, 4
    t["q"][:] = 0
    t["q"][..., 0] = 16  # a key's score is 16 * its element 0 / sqrt(D)
    for r, ctx in enumerate(c.ctx):
        ids = t["block_tables"][r].long()
        t["v_scale"][ids[0]] = first
        n = (ctx + c.k[r] + PAGE) // PAGE
        t["k_cache"].view(torch.uint8)[ids[:n], :, :, 0] = 0
        t["k_scale"][ids[:n]] = 1.0
        peak = torch.tensor(20.0 / math.log2(math.e) * math.sqrt(D) / 16).to(torch.float8_e4m3fn).view(torch.uint8).item()
        low = torch.tensor(-9.0 / math.log2(math.e) * math.sqrt(D) / 16).to(torch.float8_e4m3fn).view(torch.uint8).item()
        t["k_cache"].view(torch.uint8)[ids[2], :, 6, 0] = peak          # key 38
        t["k_cache"].view(torch.uint8)[ids[8:n], :, :, 0] = low         # keys from 128 on
    c.run()
    at = 0
    for r, (k, ctx) in enumerate(zip(c.k, c.ctx)):
        L = ctx + k + 1
        ids = t["block_tables"][r, :(L + PAGE - 1) // PAGE].long()
        load = lambda x: (t[x + "_cache"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() *
                          t[x + "_scale"][ids].double()[:, :, None, None]).permute(1, 0, 2, 3).reshape(2, -1, D)[:, :L]
        K, W = load("k"), load("v")
        s = torch.einsum("jhgd,htd->jhgt", t["q"][at:at + k + 1].double().view(k + 1, 2, g, D), K) / math.sqrt(D)
        seen = torch.arange(L, device="cuda") <= ctx + torch.arange(k + 1, device="cuda")[:, None]
        w = torch.softmax(torch.where(seen[:, None, None], s, -math.inf), dim=3)
        ref, A = torch.einsum("jhgt,htd->jhgd", w, W), torch.einsum("jhgt,htd->jhgd", w, W.abs())
        got = t["out"][at:at + k + 1].double().view(ref.shape)
        at += k + 1
        # besides the usual bound, half of P's least step for every key, against the least P of the largest product's tile
        top = (w.unsqueeze(-1) * W.abs()[None, :, None]).amax((3, 4))[..., None]
        assert ((got - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -7 * A + 2.0 ** -9 * top * math.sqrt(L)).all()


def test_extreme_magnitudes():
    for kf, vf, qf in ((2.0 ** -40, 2.0 ** 60, 1.0), (2.0 ** 30, 2.0 ** -60, 2.0 ** -30), (1.0, 2.0 ** -90, 1.0), (1.0, 2.0 ** 100, 1.0)):
        c = Case(8, k=[3], ctx=[400], Hq=4, Hkv=2)
        c.t["k_scale"] *= kf
        c.t["v_scale"] *= vf
        c.t["q"] *= qf
        c.run()
        c.check()


def test_queries_of_mixed_size():
    c = Case(9, k=[7, 0], ctx=[500, 100], Hq=8, Hkv=2)
    c.t["q"] *= torch.exp2(torch.randint(-12, 3, c.t["q"].shape[:2] + (1,), device="cuda").float()).to(torch.bfloat16)
    c.t["q"][3] = 0
    c.run()
    c.check()


def test_repeats_to_the_bit_and_streams():
    c = Case(10, k=[4, 8, 0] * 5, ctx=[1000, 30, 5000] * 5)
    c.run()
    a = c.t["out"].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.t["out"].fill_(3)
    s.wait_stream(torch.cuda.current_stream())
    c.run(stream=s)
    assert torch.equal(a, c.t["out"])


def test_bad_requests_are_skipped():
    c = Case(11, k=[3, 2, 1], ctx=[100, 50, 300], Hq=8, Hkv=2)
    c.t["context_lens"][1] = -4
    assert c.run(expect=1) == 1
    c.check(skipped=[1])
    c = Case(12, k=[3, 2, 1], ctx=[100, 50, 300], Hq=8, Hkv=2)
    c.t["block_tables"][2, 7] = 10 ** 6
    assert c.run(expect=2) == 2
    c.check(skipped=[2])
    c = Case(13, k=[3, 40, 1], ctx=[100, 50, 300], Hq=8, Hkv=2)
    assert c.run(expect=5) == 1          # 4 * 41 rows
    c.check(skipped=[1])


def test_offsets_past_32_bits():
    # the sequences' pages lie at the end of a pool of more than 2^32 bytes
    c = Case(14, k=[4, 1], ctx=[300, 40], Hq=32, Hkv=8)
    t, nb = c.t, (1 << 32) // (8 * PAGE * 128) + 500
    lo = nb - t["k_cache"].shape[0]
    for x in "kv":
        big = torch.full((nb, 8, PAGE, 128), 0x7f, dtype=torch.uint8, device="cuda")
        big[lo:] = t[x + "_cache"].view(torch.uint8)
        s = torch.ones((nb, 8), device="cuda")
        s[lo:] = t[x + "_scale"]
        t[x + "_cache"], t[x + "_scale"] = big.view(torch.float8_e4m3fn), s
    t["block_tables"] = torch.where(t["block_tables"] >= 0, t["block_tables"] + lo, -1)
    c.run()
    c.check()


def test_step_gives_the_results_of_its_parts():
    from paper_2601_11652_gb300 import binding as wb
    k, V = [3, 0, 8, 5] * 8, 5000
    c = Case(15, k=k, ctx=[500, 10, 2000, 77] * 8)
    T, Td, B = sum(k) + len(k), sum(k), len(k)
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randn((T, V), generator=g, device="cuda").to(torch.bfloat16) * 2
    row = torch.cat([torch.arange(n) + i + sum(k[:i]) for i, n in enumerate(k)]).cuda()
    qd = torch.softmax(z[row].float() + 0.5 * torch.randn((Td, V), generator=g, device="cuda"), 1)
    out = lambda: dict(accepted_len=torch.full((B,), -7, dtype=torch.int32, device="cuda"),
                       next_token=torch.full((B,), -7, dtype=torch.int32, device="cuda"))
    common = dict(draft_lens=c.t["draft_lens"], target_logits=z, draft_tokens=qd.argmax(1).int(), draft_probs=qd,
                  accept_uniforms=torch.rand(Td, generator=g, device="cuda"), sample_uniforms=torch.rand(B, generator=g, device="cuda"))
    o1, o2 = out(), out()
    c.run()
    a = c.t["out"].clone()
    acc = wb.make_accept_args(**common, **o1)
    ws = wb.alloc_workspace(wb.wisp_verify_workspace_size(None, acc))
    wb.wisp_verify_accept(acc, ws)
    c.t["out"].fill_(3)
    c.run(acc=wb.make_accept_args(**common, **o2))
    assert torch.equal(a, c.t["out"]) and all(torch.equal(o1[n], o2[n]) for n in o1) and (o1["accepted_len"] >= 0).all()


def test_empty_batch_and_refusals():
    from paper_2601_11652_gb300 import binding as wb
    c = Case(16, k=[0], ctx=[5])
    t = {n: v[:0] if n in ("draft_lens", "context_lens", "block_tables", "q", "out") else v for n, v in c.t.items()}
    a = wb.make_attn_kv8_args(**t)
    ws = wb.alloc_workspace(wb.wisp_verify_workspace_size(a.attn, None))
    wb.wisp_verify_attention_kv8(a, ws)
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        wb.make_attn_kv8_args(**{**c.t, "k_cache": c.t["k_cache"].float()})
    with pytest.raises(ValueError):
        wb.make_attn_kv8_args(**{**c.t, "v_scale": c.t["v_scale"][:, :1]})
    for change in (dict(k_scale=None), dict(v_scale=None)):
        a = wb.make_attn_kv8_args(**c.t)
        for n, v in change.items():
            setattr(a, n, v)
        with pytest.raises(wb.WispError):
            wb.wisp_verify_attention_kv8(a, ws)


def _set_scores(c, want, scale=2.0 ** -5):
    """Keys of request r get scores want[r] (log2 units, [L]) for every query: carried by the first two elements, whose codes leave an
    error of some 2^-7 relative (the checks take the scores from the codes)."""
    t, D = c.t, c.D
    t["q"][:] = 0
    t["q"][..., :2] = 16
    t["k_scale"][:] = scale
    for r, s in enumerate(want):
        x = torch.as_tensor(s, dtype=torch.float64, device="cuda") * math.log(2) * math.sqrt(D) / 16 / scale
        assert x.abs().max() <= 448
        hi = x.to(torch.float8_e4m3fn)
        lo = (x - hi.double()).to(torch.float8_e4m3fn)
        n = x.numel()
        tok = torch.arange(n, device="cuda")
        page = t["block_tables"][r].long()[tok // PAGE]
        raw = t["k_cache"].view(torch.uint8)
        for d, y in ((0, hi), (1, lo)):
            raw[page, :, tok % PAGE, d] = y.view(torch.uint8)[:, None]


@pytest.mark.parametrize("cache", ["e4m3", "own"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_nan_value_in_a_chunk_of_no_weight(dtype, cache):
    # 20005 keys of one request are cut; all keys but the first 64 weigh 2^-200: their chunks add nothing but a value that is NaN
    from paper_2601_11652_gb300 import binding as wb
    c = Case(50, k=[4], ctx=[20000], Hq=8, Hkv=2, dtype=dtype, garbage=False)
    s = torch.full((20005,), -200.0)
    s[:64] = 0
    _set_scores(c, [s], scale=0.25)
    c.run()
    c.check()
    want = np.zeros((5, 2, 4, c.D), bool)
    for tok, h, d in ((5000, 0, 17), (12345, 1, 3)) + (((20003, 1, 99),) if cache == "e4m3" else ()):
        c.t["v_cache"].view(torch.uint8)[int(c.t["block_tables"][0, tok // PAGE]), h, tok % PAGE, d] = 0x7f
        want[max(0, tok - 20000):, h, :, d] = True
    if cache == "e4m3":
        c.run()
    else:  # the same values in a cache of the queries' type
        t = {n: v for n, v in c.t.items() if not n.endswith("_scale")}
        for x in "kv":
            t[x + "_cache"] = (c.t[x + "_cache"].float() * c.t[x + "_scale"][:, :, None, None]).to(dtype)
        a = wb.make_attn_args(**t)
        ws = wb.alloc_workspace(wb.wisp_verify_workspace_size(a, None))
        wb.wisp_verify_attention(a, ws)
        torch.cuda.synchronize()
        assert wb.wisp_verify_get_device_status(ws)[0] == 0
    out = c.t["out"].float().cpu().numpy().reshape(-1, 2, 4, c.D)
    assert np.array_equal(np.isnan(out), want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("strong,gap,sd", [(-5.9, 9.2, 0.0), (-5.9, 9.2, 0.3), (-3.75, 15.25, 0.0), (-3.9, 13.0, 0.0), (-2.0, 9.0, 0.3),
                                           (-8.0, 10.0, 0.0)])
def test_small_weights_beside_a_strong_key_in_every_tile(strong, gap, sd, D):
    # a first key with the largest weight, and in every 128 keys one `strong` octaves from it, the others `gap` octaves below that one:
    # each weighs little, together they carry up to a fifth.  Values of mean 1, so that nothing averages out.
    B, ctx = 20, 4095  # 160 (request, head) pairs: no sequence is cut
    c = Case(30, k=[0] * B, ctx=[ctx] * B, D=D, garbage=False)
    g = torch.Generator(device="cuda").manual_seed(5)
    want = []
    for r in range(B):
        s = torch.full((ctx + 1,), strong - gap, dtype=torch.float64, device="cuda")
        s += sd * torch.randn(s.shape, generator=g, device="cuda", dtype=torch.float64)
        s[5 + r::128] = strong
        s[0] = 0
        want.append(s)
    _set_scores(c, want)
    c.t["v_scale"][:] = 2.0 ** -6
    c.t["v_cache"] = ((1 + 0.3 * torch.randn(c.t["v_cache"].shape, generator=g, device="cuda")) * 64).to(torch.float8_e4m3fn)
    c.run()
    c.check()


def _split_scales(c, pages_of):
    """Sets the V scale of page i of request r to pages_of(r, i), with codes of magnitude at most 1."""
    t = c.t
    raw, x = t["v_cache"].view(torch.uint8), t["v_cache"].float()
    nan = torch.isnan(x)
    x = torch.sign(x) * (0.25 + 0.75 * torch.rand(x.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9)))
    codes = x.to(torch.float8_e4m3fn).view(torch.uint8)
    raw[~nan] = codes[~nan]
    for r, (k, ctx) in enumerate(zip(c.k, c.ctx)):
        for i in range((ctx + k + PAGE) // PAGE):
            t["v_scale"][int(t["block_tables"][r, i])] = pages_of(r, i)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name,of", [
    ("largest", lambda r, i: 2.0 ** 127), ("subnormal_beside_large", lambda r, i: 2.0 ** 100 if i % 3 == 0 else 2.0 ** -140),
    ("as_the_append_writes", lambda r, i: 2.0 ** 118 if i == 2 else 2.0 ** -96), ("one_page", lambda r, i: 2.0 ** 90 if (r, i) == (2, 9) else 0.01),
    ("zero_beside_large", lambda r, i: 0.0 if i % 2 else 2.0 ** 40), ("zero_first", lambda r, i: 0.0 if i < 9 else 0.02),
    ("at_the_edges", lambda r, i: (2.0 ** -41, 2.0 ** 29, 0.0, 2.0 ** -42, 2.0 ** 30)[(i + r) % 5]),
    ("zero_beside_small", lambda r, i: 0.0 if i % 2 else 2.0 ** -25), ("zero_beside_not_so_small", lambda r, i: 0.0 if i % 2 else 2.0 ** -15),
    ("rising", lambda r, i: 2.0 ** (min(118, 3 * i - 96))), ("falling", lambda r, i: 2.0 ** max(-96, 118 - 3 * i))])
def test_any_value_scales(name, of, D, dtype):
    c = Case(40, k=[10, 3, 15, 0, 8], ctx=[119, 300, 2000, 0, 700], Hq=8, Hkv=2, D=D, dtype=dtype)
    _split_scales(c, of)
    c.run()
    c.check()
    a = c.t["out"].clone()
    c.run()
    assert torch.equal(a, c.t["out"])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_value_scales_far_apart_in_a_cut_sequence(dtype):
    # 20001 keys of one request are cut: chunks with ordinary scales, with large ones and with both are merged
    for of in (lambda r, i: 2.0 ** 110 if i > 900 else 0.01, lambda r, i: 2.0 ** 110 if i % 400 == 7 else 0.01, lambda r, i: 2.0 ** -96 if i % 2 else 2.0 ** -20):
        c = Case(41, k=[4], ctx=[20000], Hq=8, Hkv=2, dtype=dtype)
        _split_scales(c, of)
        c.run()
        c.check()


@pytest.mark.parametrize("D", [64, 128])
def test_value_scales_far_apart_and_values_or_queries_that_are_not_finite(D):
    c = Case(42, k=[6, 2, 12], ctx=[250, 31, 400], Hq=8, Hkv=2, D=D)
    _split_scales(c, lambda r, i: 2.0 ** 100 if i % 2 else 2.0 ** -90)
    bt, want = c.t["block_tables"], np.zeros((23, 2, 4, D), bool)
    for r, j, h, d in ((0, 3, 1, 17), (0, 6, 0, 50), (1, 0, 0, 0), (2, 12, 1, 63)):
        tok = c.ctx[r] + j
        c.t["v_cache"].view(torch.uint8)[int(bt[r, tok // PAGE]), h, tok % PAGE, d] = 0x7f
        want[(0, 7, 10)[r] + j:(7, 10, 23)[r], h, :, d] = True
    for row, head, v in ((1, 2, math.inf), (9, 0, math.nan), (12, 7, -math.inf)):
        c.t["q"][row, head, 3] = v
        want[row, head // 4, head % 4] = True
    c.run()
    out = c.t["out"].float().cpu().numpy().reshape(-1, 2, 4, D)
    assert np.array_equal(np.isnan(out), want)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gap", [8, 14, 20])
def test_values_of_a_page_with_a_small_scale(gap, D):
    """Nearly all of the weight is on pages with a small V scale; pages with a scale 2^gap as large and little weight hold zeros in every
    second element, which thus come from the small ones alone.

    Bound: as in test_matches_the_definition for the scores and the output's rounding, and a key's weight * V scale off by at most 2^-8 of
    itself or 2^-15 of the largest such product among its 128 keys, whichever is more (in fewer than 128 rows the keys' tiles start at
    key 0: no sequence is cut)."""
    B, L = 20, 2048
    c = Case(31, k=[0] * B, ctx=[L - 1] * B, D=D, garbage=False)
    t = c.t
    tok = torch.arange(L, device="cuda")
    big = tok // PAGE % 4 == 3
    _set_scores(c, [torch.where(big, -4.0, 0.0).double()] * B)
    for r in range(B):
        ids = t["block_tables"][r, :L // PAGE].long()
        t["v_scale"][ids] = torch.where(big[::PAGE], 2.0 ** (gap - 10), 2.0 ** -10)[:, None]
        v = 1 + 0.3 * torch.randn((L // PAGE, 8, PAGE, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(r))
        v[big[::PAGE], :, :, ::2] = 0
        t["v_cache"].view(torch.uint8)[ids] = (v * 8).to(torch.float8_e4m3fn).view(torch.uint8)
    c.run()
    for r in range(B):
        ids = t["block_tables"][r, :L // PAGE].long()
        load = lambda x, s: (t[x + "_cache"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() *
                             (t[x + "_scale"][ids].double()[:, :, None, None] if s else 1)).permute(1, 0, 2, 3).reshape(8, L, D)
        K, V, code = load("k", True), load("v", True), load("v", False)
        w = torch.softmax(torch.einsum("hgd,htd->hgt", t["q"][r].double().view(8, 4, D), K) / math.sqrt(D), dim=2)
        prod = w * t["v_scale"][ids].double().T.repeat_interleave(PAGE, 1)[:, None]
        top = prod.view(8, 4, -1, 128).amax(3).repeat_interleave(128, 2)
        ref, A = torch.einsum("hgt,htd->hgd", w, V), torch.einsum("hgt,htd->hgd", w, V.abs())
        step = torch.einsum("hgt,htd->hgd", torch.maximum(2.0 ** -8 * prod, 2.0 ** -15 * top), code.abs())
        got = t["out"][r].double().view(ref.shape)
        assert ((got - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -8 * A + step).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("e", [-126, -110, -96, -70, -60, 40, 60, 100, 118])
def test_one_scale_for_all_values(e, D, dtype):
    """Outputs scale with V: with 2^e in the place of 2^-6 they are 2^(e + 6) times the same, to the bounds of the definition.  (The
    codes go up to 448, so that outputs stay normal, but for elements below 2^-8 of the largest at the smallest scale.)"""
    c = Case(60, k=[4, 0, 15], ctx=[700, 20, 5000], Hq=8, Hkv=2, D=D, dtype=dtype)
    c.t["v_cache"].view(torch.uint8)[:] = torch.where((c.t["v_cache"].view(torch.uint8) & 0x7f) == 0x7f, c.t["v_cache"].view(torch.uint8),
                                                      (c.t["v_cache"].float().nan_to_num() / 2).to(torch.float8_e4m3fn).view(torch.uint8))
    c.t["v_scale"][:] = 2.0 ** e
    c.run()
    c.t["out"].copy_((c.t["out"].double() * 2.0 ** (-6 - e)).to(dtype))
    c.t["v_scale"][:] = 2.0 ** -6
    c.check()
