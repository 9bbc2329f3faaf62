"""The attention of prompts and of shared prefixes at the ends of what its types hold: finite inputs give finite outputs, and what a row
does not see changes none of its bits.  Definition and bounds as in test_prompt_gpu.py."""
import math

import numpy as np
import pytest
import torch

from test_prompt_gpu import BF, F32, PAGE, TYPES, Case, _lib, bits_of, runs_of  # noqa: F401 (_lib builds the library)

pytestmark = pytest.mark.gpu


def scale_tokens(c, x, a, b, e):
    """K or V (x) of tokens a .. b - 1 of every request times 2^e: in the cache, or in the scales of an e4m3 cache (whole pages)."""
    for r in range(len(c.k)):
        L = c.ctx[r] + c.k[r] + 1
        for p in range(a // PAGE, (min(b, L) + PAGE - 1) // PAGE):
            page = int(c.bt[r, p])
            if x + "_scale" in c.t:
                assert a % PAGE == 0 and (b % PAGE == 0 or b >= L)
                c.t[x + "_scale"][page] *= 2.0 ** e
                c.val[x][page] = c.t[x + "_cache"][page].double() * c.t[x + "_scale"][page].double()[:, None, None]
            else:
                s = slice(max(a - p * PAGE, 0), min(b - p * PAGE, PAGE))
                y = c.t[x + "_cache"]
                y[page, :, s] = (y[page, :, s].double() * 2.0 ** e).to(y.dtype)
                c.val[x][page, :, s] = y[page, :, s].double()


def far_scores(c, e):
    """Scores of up to 2^e sqrt(D), in steps of a quarter of that.  Every sum is a whole number of small powers of two, exact in any order, so
    that equal scores are equal, and a row is the mean of V over the keys of its largest score; other weights are below 2^-126 but where e is
    small, and there check()'s bounds hold as anywhere."""
    g = torch.Generator(device="cuda").manual_seed(e)
    a = e // 2
    c.t["q"].fill_(2.0 ** a)
    shape = c.t["k_cache"].shape[:3]
    u = torch.tensor([1.0, 0.75, 0.5, -1.0], device="cuda")[torch.randint(0, 4, shape, generator=g, device="cuda")]
    u[:, :, 0] = 0.5
    u[torch.rand(shape[0], generator=g, device="cuda") < 0.7] = -1.0  # (whole tiles without the largest, too)
    u = u[..., None].expand(*shape, c.D)
    if "k_scale" in c.t:
        c.t["k_cache"] = u.to(torch.float8_e4m3fn).contiguous()
        c.t["k_scale"].fill_(2.0 ** (e - a))
    else:
        c.t["k_cache"] = (u * 2.0 ** (e - a)).to(c.t["q"].dtype).contiguous()
    c.val["k"] = u.double() * 2.0 ** (e - a)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("e", [13, 15, 16, 17, 18, 24, 26, 28, 30, 33, 40, 100])
def test_scores_far_from_zero(dtype, cache, D, e):
    c = Case(e + D, k=[250, 3, 61], ctx=[0, 70, 500], Hq=4, Hkv=2, D=D, dtype=dtype, cache=cache)
    far_scores(c, e)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads", [(8, 8, 64), (28, 4, 128)])
@pytest.mark.parametrize("k,ctx,runs", [([3], [40000], None), ([9, 0, 30, 2], [3000, 700, 5000, 2000], None),
                                        ([1, 0, 4, 2, 7], [350, 320, 900, 64, 3000], runs_of((0, 20, 3), (-1, 0, 1), (1, 7, 1)))])
def test_scores_far_from_zero_in_chunks(dtype, cache, heads, k, ctx, runs):
    c = Case(5, k=k, ctx=ctx, Hq=heads[0], Hkv=heads[1], D=heads[2], dtype=dtype, cache=cache, runs=runs)
    far_scores(c, 40)
    c.t["q"][2:4] *= 2.0 ** -40  # (a row whose scores are small beside them)
    c.run()
    c.check()


SPLIT = ([250, 3, 190, 61], [0, 70, 33, 500])  # rows and contexts; what changes lies in the middle of tiles


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [16, 48, 160, 528])
@pytest.mark.parametrize("e", [40, 100])
def test_values_behind_a_row_change_none_of_its_bits(dtype, cache, D, at, e):
    k, ctx = SPLIT
    c = Case(at + D, k=k, ctx=ctx, Hq=4, Hkv=2, D=D, dtype=dtype, cache=cache)
    c.run()
    c.check()
    before = c.t["out"].clone()
    scale_tokens(c, "v", at, 1 << 20, e)
    c.run()
    for r in range(len(k)):
        n = min(max(at - ctx[r], 0), k[r] + 1)  # rows that do not see them
        row = c.row_of(r)
        assert torch.equal(c.t["out"][row:row + n], before[row:row + n]), r
    assert torch.isfinite(c.t["out"]).all()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [16, 160, 528])
@pytest.mark.parametrize("e", [30, 100])
def test_keys_behind_a_row_change_none_of_its_bits(dtype, cache, D, at, e):
    k, ctx = SPLIT
    c = Case(at + D, k=k, ctx=ctx, Hq=4, Hkv=2, D=D, dtype=dtype, cache=cache)
    c.run()
    before = c.t["out"].clone()
    scale_tokens(c, "k", at, 1 << 20, e)
    c.run()
    for r in range(len(k)):
        n = min(max(at - ctx[r], 0), k[r] + 1)  # rows that do not see them
        row = c.row_of(r)
        assert torch.equal(c.t["out"][row:row + n], before[row:row + n]), r
    assert torch.isfinite(c.t["out"]).all()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("runs", [None, runs_of((0, 20, 3))])
@pytest.mark.parametrize("e", [-110, -80, -45, -30, 30, 45, 80, 100, 112])
def test_scores_do_not_depend_on_where_their_magnitude_lies(dtype, cache, runs, e):
    """Keys times 2^e and queries times 2^-e: the same scores.  Powers of two are exact in every step, so that the outputs are equal to the bit,
    but for fp32 queries past 2^45, which are computed apart (check()'s bound)."""
    c = Case(24, k=[140, 9, 30], ctx=[320, 350, 2000], Hq=8, Hkv=2, D=128, dtype=dtype, cache=cache, runs=runs)
    c.run()
    before = c.t["out"].clone()
    q = c.t["q"].double()
    c.t["q"] = (q * 2.0 ** -e).to(dtype)
    exact = torch.equal(c.t["q"].double() * 2.0 ** e, q)  # (queries below 2^-14 times 2^-112 are no normal numbers and lose bits)
    if cache:
        c.t["k_scale"] = (c.t["k_scale"].double() * 2.0 ** e).float()
    else:
        c.t["k_cache"] = (c.t["k_cache"].double() * 2.0 ** e).to(dtype)
    c.val["k"] = c.val["k"] * 2.0 ** e
    c.run()
    assert exact or e == 112
    if exact and (dtype == BF or e > -42):
        assert torch.equal(c.t["out"], before)
    c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("q,k", [(0, 113), (0, 118), (-100, 110), (60, 60), (118, 0)])
def test_equal_scores_of_any_size(dtype, cache, q, k):
    """Queries of 2^q, keys of 2^k: every row is the mean of the V that it sees."""
    c = Case(25, k=[140, 9, 30], ctx=[320, 350, 2000], Hq=8, Hkv=2, D=128, dtype=dtype, cache=cache)
    c.t["q"].fill_(2.0 ** q)
    if cache:
        c.t["k_cache"] = torch.ones_like(c.val["k"]).to(torch.float8_e4m3fn)
        c.t["k_scale"].fill_(2.0 ** k)
    else:
        c.t["k_cache"].fill_(2.0 ** k)
    c.val["k"] = torch.full_like(c.val["k"], 2.0 ** k)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("runs", [None, runs_of((0, 20, 3))])
@pytest.mark.parametrize("e", [-80, -40, 30, 44, 60, 80])
def test_outputs_scale_with_values(dtype, cache, runs, e):
    """Powers of two in all of V are powers of two in the outputs, bit by bit."""
    c = Case(23, k=[140, 9, 30], ctx=[320, 350, 2000], Hq=8, Hkv=2, D=128, dtype=dtype, cache=cache, runs=runs)
    c.run()
    before = c.t["out"].clone()
    if cache:
        c.t["v_scale"] *= 2.0 ** e
    else:
        c.t["v_cache"] = (c.t["v_cache"].double() * 2.0 ** e).to(dtype)
    c.run()
    assert torch.equal(c.t["out"].double(), before.double() * 2.0 ** e)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads", [(8, 8, 64), (28, 4, 128)])
@pytest.mark.parametrize("k,ctx,runs", [([140, 9, 30], [320, 350, 2000], None), ([3], [40000], None), ([700, 0], [0, 5000], None),
                                        ([1, 0, 4, 2, 7], [350, 320, 900, 64, 3000], runs_of((0, 20, 3), (-1, 0, 1), (1, 7, 1)))])
@pytest.mark.parametrize("alike", [False, True])
def test_values_near_the_largest(dtype, cache, heads, k, ctx, runs, alike):
    """V of up to 2^127; alike: all of them so, and the outputs their mean."""
    c = Case(31, k=k, ctx=ctx, Hq=heads[0], Hkv=heads[1], D=heads[2], dtype=dtype, cache=cache, runs=runs)
    v = c.val["v"]
    if alike:
        v = torch.where(torch.isnan(v), v, torch.ones_like(v))
    e = 126 - math.floor(math.log2(v[~torch.isnan(v)].abs().max()))
    if cache:
        if alike:
            c.t["v_cache"] = v.to(torch.float8_e4m3fn)
            c.t["v_scale"].fill_(2.0 ** e)
        else:
            c.t["v_scale"] = (c.t["v_scale"].double() * 2.0 ** e).float()
    else:
        c.t["v_cache"] = (v * 2.0 ** e).to(dtype)
    c.val["v"] = v * 2.0 ** e
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_a_value_near_the_largest_among_others(dtype, cache):
    """One token's V (one page's scales) of 2^120 times the others'; rows in front of it keep their bits."""
    c = Case(32, k=[250, 100, 30], ctx=[0, 70, 3000], Hq=4, Hkv=2, D=128, dtype=dtype, cache=cache)
    c.run()
    before = c.t["out"].clone()
    scale_tokens(c, "v", 96, 112 if cache else 97, 120)
    c.run()
    for r in range(2):
        n = 96 - c.ctx[r]
        row = c.row_of(r)
        assert torch.equal(c.t["out"][row:row + n], before[row:row + n]), r
    c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("e", [0, -60, -100, -118, 80])
@pytest.mark.parametrize("zeros", [1, 5, 70])
def test_zero_values_in_front(dtype, cache, e, zeros):
    """The first tokens' V is zero and the others' 2^e: rows that see zeros only are zero, others as everywhere (e4m3: whole pages, by their
    scales).  Outputs below fp32's normal numbers have steps of 2^-149: with weights of up to 2^14 in front of them, 2^-135."""
    c = Case(33, k=[150, 40, 3], ctx=[0, 20, 2000], Hq=4, Hkv=2, D=64, dtype=dtype, cache=cache)
    scale_tokens(c, "v", 0, 1 << 20, e)
    for r in range(3):
        n = (zeros + 15) // 16 * 16 if cache else zeros
        for t in range(min(n, c.ctx[r] + c.k[r] + 1)):
            page, slot = int(c.bt[r, t // PAGE]), t % PAGE
            if cache:
                c.t["v_scale"][page] = 0
            else:
                c.t["v_cache"][page, :, slot] = 0
            c.val["v"][page, :, slot] = 0
    c.run()
    bf = dtype == BF
    for r in range(3):
        at = c.row_of(r)
        ref, mag, _ = c.reference(r, 0, c.k[r] + 1)
        got = c.t["out"][at:at + c.k[r] + 1].double()
        bound = (2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -10) * mag if bf else 2.0 ** -9 * mag) + 2.0 ** -133
        assert bool(((got - ref).abs() <= bound).all()), r


def test_workspace_follows_what_can_be_cut():
    """Partials are reserved for sequences that are long enough to be cut (sizes in bytes, D + 2 floats a row)."""
    from paper_2601_11652_gb300 import binding as wb
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    for rows, pages, most in ((64, 4, 1 << 20), (128, 8, 1 << 20), (2000, 125, 120 << 20), (64, 16, 3 * 2 * 8 * 256 * 130 * 4 + (1 << 20))):
        q = torch.empty((rows, 32, 128), dtype=BF, device="cuda")
        kv = torch.empty((pages, 8, 16, 128), dtype=BF, device="cuda")
        a = wb.make_prompt_args(draft_lens=i(1), context_lens=i(1), block_tables=i(1, pages), q=q, k_cache=kv, v_cache=kv, out=q)
        assert wb.wisp_prompt_workspace_size(a) < most, (rows, pages)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,ctx", [(1, 127), (1, 128), (1, 129), (1, 255), (1, 256), (1, 257), (1, 1024), (3, 2047), (200, 0), (300, 800), (70, 1300), (500, 560)])
@pytest.mark.parametrize("copies", [1, 3, 40])
def test_tables_as_wide_as_their_sequences(dtype, n, ctx, copies):
    """The workspace is sized by the table's width: no longer sequence fits behind it."""
    runs = runs_of((0, ctx // 16, copies)) if ctx >= 16 else None
    for r in (None, runs):
        c = Case(n + ctx, k=[n - 1] * copies, ctx=[ctx] * copies, Hq=8, Hkv=2, D=64, dtype=dtype, runs=r, spare=0)
        c.run()
        c.check()


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_rows_computed_apart_repeat_and_leave_refused_requests(dtype, cache):
    """Rows with scores far from zero, some of them in a run with a refused request; they repeat to the bit, whatever is computed beside them."""
    k, ctx, runs = [30, 2, 0, 5, 200], [64, 70, 64, 300, 64], runs_of((1, 4, 3), (-1, 0, 1), (2, 4, 1))
    c = Case(34, k=k, ctx=ctx, Hq=8, Hkv=2, D=128, dtype=dtype, cache=cache, runs=runs)
    far_scores(c, 50)
    c.t["q"][3::7] *= 2.0 ** -50
    c.run()
    c.check()
    first = c.t["out"].clone()
    for _ in range(5):
        c.t["out"].fill_(77)
        c.run()
        assert torch.equal(c.t["out"], first)
    c.t["context_lens"][1] = 1 << 20
    c.t["out"].fill_(77)
    c.run(expect=1)
    c.check(skipped=[1])
    assert (c.t["out"][31:34] == 77).all()
    same = [r for r in range(238) if not 31 <= r < 34]
    assert torch.equal(c.t["out"][same], first[same])


def test_workspace_of_many_heads():
    """What is reserved for rows that are computed apart follows the rows, not the tiles that they are in: 1024 requests of one row, 64 heads."""
    from paper_2601_11652_gb300 import binding as wb
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    q = torch.empty((1024, 64, 64), dtype=BF, device="cuda")
    kv = torch.empty((8, 64, 16, 64), dtype=BF, device="cuda")
    t = dict(draft_lens=i(1024), context_lens=i(1024), block_tables=i(1024, 8), q=q, k_cache=kv, v_cache=kv, out=q)
    assert wb.wisp_prompt_workspace_size(wb.make_prompt_args(**t)) < 4 << 20
    rows = 1024 * 64  # a partial for the run's keys and one for the request's own
    assert wb.wisp_verify_shared_workspace_size(wb.make_shared_args(**t, shared_ids=i(1024), shared_pages=i(1024))) < 2 * rows * 66 * 4 + (12 << 20)
