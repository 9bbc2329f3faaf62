"""wisp_verify_logprobs against its definition in 64 bits, wisp_verify_committed_tokens against plain Python.

Bounds.  exp(z - m) is taken in fp32 with a relative error below 2^-20 (the rounding of the exponent's argument, at most
2^-24 times 126 log2 units where a weight still counts in a sum, makes most of it); sums of one sign keep that and add their
roundings, at most 2^-19 in all with the splits used here.  So log s is off by at most 2^-18 plus its rounding, and a log
probability by 2^-18 + 2^-23 (|z| + |lse|).  The entropy's second term is a mean of (z - m): off by 2^-18 (1 + |H| + log V)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2601_11652_gb300 import build
    build.build()


def call(logits, tokens, top, entropy=True, expect=0, stream=None):
    from paper_2601_11652_gb300 import binding as wb
    rows = logits.shape[0]
    f = lambda *s: torch.full(s, 77.0, device="cuda")
    out = dict(logprob=f(rows), entropy=f(rows) if entropy else None,
               top_tokens=torch.full((rows, top), 77, dtype=torch.int32, device="cuda") if top else None,
               top_logprobs=f(rows, top) if top else None)
    a = wb.make_logprobs_args(logits=logits, tokens=tokens, **out)
    ws = wb.alloc_workspace(wb.wisp_verify_logprobs_workspace_size(a))
    ws.fill_(0xff)
    wb.wisp_verify_logprobs(a, ws, stream)
    torch.cuda.synchronize()
    code, row = wb.wisp_verify_get_device_status(ws)
    assert code == expect, (code, row)
    return {n: v.cpu().numpy() for n, v in out.items() if v is not None}


def check_row(z, tok, got, i, top):
    """z: the row in 64 bits (numpy)."""
    V = z.size
    if tok < 0:
        assert got["logprob"][i] == 0 and got.get("entropy", [0] * (i + 1))[i] == 0
        if top:
            assert np.all(got["top_tokens"][i] == -1) and np.all(got["top_logprobs"][i] == 0)
        return
    m = z.max()
    with np.errstate(invalid="ignore"):
        lse = m + math.log(np.exp(z - m).sum())
        lp = z - lse
        p = np.exp(lp)
        H = -np.where(p > 0, p * lp, 0).sum()
    tol = lambda x: 2.0 ** -18 + 2.0 ** -23 * (np.abs(x) + abs(lse))
    if z[tok] == -math.inf:
        assert got["logprob"][i] == -math.inf
    else:
        assert abs(got["logprob"][i] - lp[tok]) <= tol(z[tok])
    if "entropy" in got:
        assert abs(got["entropy"][i] - H) <= 2.0 ** -18 * (1 + abs(H) + math.log(V)) + 2.0 ** -23 * abs(lse)
    if top:
        n = min(top, V)
        order = np.lexsort((np.arange(V), -z))[:n]
        assert np.array_equal(got["top_tokens"][i][:n], order)
        want = lp[order]
        fin = np.isfinite(want)
        assert np.array_equal(np.isfinite(got["top_logprobs"][i][:n]), fin)
        assert np.all(np.abs(got["top_logprobs"][i][:n] - want)[fin] <= tol(z[order])[fin])
        assert np.all(got["top_tokens"][i][n:] == -1) and np.all(got["top_logprobs"][i][n:] == -math.inf)


def check(logits, tokens, top, got):
    z = logits.double().cpu().numpy()
    for i, t in enumerate(tokens.tolist()):
        check_row(z[i], t, got, i, top)


def make(seed, rows, V, dtype, pad=0, sd=2.0, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randn(rows * (V + pad) + offset, generator=g, device="cuda") * sd
    wide = wide.to(dtype)[offset:].view(rows, V + pad)
    tok = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    return wide[:, :V], tok


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,V,pad,offset", [(1, 1, 0, 0), (3, 2, 0, 0), (5, 31, 0, 1), (4, 1000, 24, 0), (7, 4099, 0, 3), (2, 32768, 0, 0),
                                               (1, 128256, 0, 0), (9, 50257, 47, 1), (33, 8192, 8, 0), (200, 1031, 0, 0), (3, 152064, 0, 5)])
@pytest.mark.parametrize("top", [0, 1, 20, 32])
def test_matches_the_definition(dtype, rows, V, pad, offset, top):
    z, tok = make(rows + V + top, rows, V, dtype, pad, offset=offset)
    if rows > 2:
        tok[rows // 2] = -1
    got = call(z, tok, top, entropy=top != 1)
    check(z, tok, top, got)


def test_ties_go_to_the_lowest_id():
    for V in (100, 5000, 128256):
        z = torch.zeros((4, V), dtype=torch.bfloat16, device="cuda")
        z[1] = -0.0
        z[1, 7] = 0.0
        z[2] = (torch.arange(V, device="cuda") % 3).to(torch.bfloat16)
        z[3] = (torch.arange(V, device="cuda") >= V - 40).to(torch.bfloat16)
        tok = torch.tensor([0, V - 1, 2, 5], dtype=torch.int32, device="cuda")
        check(z, tok, 32, call(z, tok, 32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sorted_rows(dtype):
    V = 20011
    up = torch.linspace(-40, 40, V, device="cuda")
    z = torch.stack([up, up.flip(0), up[torch.randperm(V, device="cuda")], up / 1000]).to(dtype)
    tok = torch.tensor([0, 0, 3, V - 1], dtype=torch.int32, device="cuda")
    check(z, tok, 32, call(z, tok, 32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_and_extreme_logits(dtype):
    V, lowest = 9001, torch.finfo(dtype).min
    z, _ = make(5, 8, V, dtype)
    z = z.clone()
    z[0, :] = -math.inf
    z[0, V - 1] = 3.0                       # one token left: probability 1, entropy 0
    z[1, : V - 5] = -math.inf               # fewer finite logits than alternatives
    z[2, 4:] = lowest                       # masked with the type's lowest value
    z[3, 100:] = -math.inf                  # masked from some place on
    z[4] *= 1e4                             # one token takes all
    z[5] = lowest                           # uniform at the lowest value
    z[6, 17] = torch.finfo(dtype).max       # the largest value
    tok = torch.tensor([V - 1, 0, 1, 50, 7, 8, 17, 11], dtype=torch.int32, device="cuda")
    check(z, tok, 20, call(z, tok, 20))


def test_rows_without_a_softmax_and_bad_tokens():
    for dtype in (torch.bfloat16, torch.float32):
        z, tok = make(6, 6, 3001, dtype)
        z = z.clone()
        for row, at, v in ((1, 2999, math.nan), (2, 0, math.inf), (4, slice(None), -math.inf)):
            z[row, at] = v
            t = tok.clone()
            got = call(z, t, 8, expect=4)
            for i in range(6):
                if math.isnan(got["logprob"][i]):
                    assert np.isnan(got["entropy"][i]) and np.all(got["top_tokens"][i] == -1) and np.all(np.isnan(got["top_logprobs"][i]))
                else:
                    check_row(z[i].double().cpu().numpy(), int(t[i]), got, i, 8)
            assert math.isnan(got["logprob"][row])
            t[row] = -1                          # skipped rows are not judged
            check(z, t, 8, call(z, t, 8))
            z[row] = 0
        t = tok.clone()
        t[3] = 3001
        got = call(z, t, 8, expect=3)
        assert math.isnan(got["logprob"][3]) and np.all(got["top_tokens"][3] == -1)


def test_repeats_to_the_bit_and_runs_on_another_stream():
    z, tok = make(8, 64, 128256, torch.bfloat16)
    a = call(z, tok, 20)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = call(z, tok, 20, stream=s)
    for n in a:
        assert np.array_equal(a[n], b[n]), n


def test_offsets_past_31_bits():
    rows, V, stride = 3, 1000, (1 << 30) + 8     # row 2 starts past 2^31 elements
    big = torch.zeros(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    z = big.as_strided((rows, V), (stride, 1))
    x, tok = make(9, rows, V, torch.bfloat16)
    z.copy_(x)
    check(x, tok, 5, call(z, tok, 5))


def test_no_rows():
    call(torch.zeros((0, 100), device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), 3)


@pytest.mark.parametrize("B,k_hi", [(1, 0), (1, 40), (37, 9), (1024, 3), (1500, 16)])
def test_committed_tokens(B, k_hi):
    from paper_2601_11652_gb300 import binding as wb
    rng = np.random.default_rng(B)
    k = rng.integers(0, k_hi + 1, B)
    L = np.array([rng.integers(0, x + 1) for x in k])
    L[rng.random(B) < 0.1] = -1
    T, extra = int(k.sum()) + B, 5
    draft, nxt = rng.integers(0, 1000, int(k.sum())), rng.integers(1000, 2000, B)
    want, d0 = [], 0
    for r in range(B):
        want += [-1 if L[r] < 0 or i > L[r] else nxt[r] if i == L[r] else draft[d0 + i] for i in range(k[r] + 1)]
        d0 += k[r]
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    t = dict(draft_lens=d(k), draft_tokens=d(draft), accepted_len=d(L), next_token=d(nxt))
    acc = wb.make_accept_args(**t, target_logits=torch.zeros((T, 8), device="cuda"), draft_probs=torch.zeros((0, 8), device="cuda"),
                              accept_uniforms=torch.zeros(0, device="cuda"), sample_uniforms=torch.zeros(B, device="cuda"),
                              total_q_rows=T + extra)
    out = torch.full((T + extra,), 77, dtype=torch.int32, device="cuda")
    wb.wisp_verify_committed_tokens(acc, out)
    torch.cuda.synchronize()
    assert out.cpu().numpy().tolist() == want + [-1] * extra
