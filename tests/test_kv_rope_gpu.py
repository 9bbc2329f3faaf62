"""wisp_kv_reserve_append_rope against its definition in 64 bits.

Bounds.  A rotated element is two products and a sum, each rounded to fp32: its error is at most 3 * 2^-24 of |a| + |b|,
taken as 2^-22 of the pair's magnitude.  Rounding to bf16 (8 significant bits) adds 2^-8 relative; to e4m3 2^-4 relative, or half of the
lowest subnormal, 2^-10 scales, whichever is more.  Magnitudes here keep bf16 and fp32 out of their subnormals."""
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


def _e4m3_table():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn)
    return t.double().numpy()


E4M3 = _e4m3_table()


def scale_of(amax):
    """The least power of two 2^e, -96 <= e <= 120, with amax <= 448 2^e (1 for 0)."""
    if amax == 0:
        return 1.0
    m, e = math.frexp(amax)
    return 2.0 ** min(max(e - 9 + (m > 0.875), -96), 120)


class Case:
    def __init__(self, seed, *, k, ctx, dtype=torch.bfloat16, cache="e4m3", D=128, Hq=8, Hkv=2, rot=None, interleaved=False,
                 fused=True, missing=True, positions=2048, extra_free=0):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.k, self.ctx, self.D, self.Hq, self.Hkv = list(k), list(ctx), D, Hq, Hkv
        self.rot = D if rot is None else rot
        self.interleaved, self.cache = interleaved, cache
        B, T = len(self.k), sum(self.k) + len(self.k)
        have = [(c + PAGE - 1) // PAGE for c in self.ctx]
        need = [(c + kk + PAGE) // PAGE for c, kk in zip(self.ctx, self.k)]
        if not missing:
            have = need
        nb = sum(need) + extra_free
        ids = rng.permutation(nb).tolist()
        width = max(need) + 1
        tables = np.full((B, width), -1, np.int32)
        for r in range(B):
            for b in range(have[r]):
                tables[r, b] = ids.pop()
        self.free = ids[:]
        stack = np.array(ids + [0] * (nb - len(ids)), np.int32)
        d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        rand = lambda *s: torch.randn(s, generator=g).to(dtype).cuda()
        if fused:
            qkv = rand(T, (Hq + 2 * Hkv) * D + 16)
            q, kn, vn = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hkv) * D], qkv[:, (Hq + Hkv) * D:(Hq + 2 * Hkv) * D]
        else:
            q, kn, vn = rand(T, Hq * D), rand(T, Hkv * D), rand(T, Hkv * D)
        self.t = dict(draft_lens=d(np.array(self.k, np.int32)), context_lens=d(np.array(self.ctx, np.int32)), block_tables=d(tables),
                      free_blocks=d(stack), free_count=d(np.array([len(self.free)], np.int32)), q=q.unflatten(1, (Hq, D)),
                      k_new=kn.unflatten(1, (Hkv, D)), v_new=vn.unflatten(1, (Hkv, D)),
                      q_out=torch.full((T, Hq, D), -7.0, dtype=dtype, device="cuda"))
        if cache == "e4m3":
            for n in "kv":
                self.t[n + "_cache"] = torch.randint(0, 256, (nb, Hkv, PAGE, D), generator=g, dtype=torch.uint8).cuda()
                self.t[n + "_cache"][(self.t[n + "_cache"] & 0x7f) == 0x7f] = 0x30
                self.t[n + "_scale"] = torch.exp2(torch.randint(-12, -6, (nb, Hkv), generator=g).float()).cuda()
        else:
            self.t["k_cache"], self.t["v_cache"] = rand(nb, Hkv, PAGE, D), rand(nb, Hkv, PAGE, D)
        if self.rot:
            ang = torch.rand((positions, self.rot // 2), generator=g, dtype=torch.float64) * 6.3
            self.t["rope"] = torch.cat([ang.cos(), ang.sin()], 1).float().cuda()

    def args(self, **kw):
        from paper_2601_11652_gb300 import binding as wb
        return wb.make_kv_rope_args(**{**self.t, **kw}, interleaved=self.interleaved)

    def run(self, stream=None, expect=0, **kw):
        from paper_2601_11652_gb300 import binding as wb
        a = self.args(**kw)
        ws = wb.alloc_workspace(wb.wisp_kv_rope_workspace_size(a))
        wb.wisp_kv_reserve_append_rope(a, ws, stream)
        torch.cuda.synchronize()
        code, rid = wb.wisp_verify_get_device_status(ws)
        assert code == expect, (code, rid)
        return rid

    def snapshot(self):
        return {n: v.clone() for n, v in self.t.items()}

    def rotated(self, x, pos):
        """x [rows, H, D] in 64 bits, and the pairs' magnitudes |a| + |b| of each element."""
        x = x.double().cpu().numpy()
        mag = np.abs(x)
        if self.rot == 0:
            return x, mag
        half = self.rot // 2
        ang = self.t["rope"].double().cpu().numpy()[pos]
        c, s = ang[:, None, :half], ang[:, None, half:]
        ia = np.arange(0, self.rot, 2) if self.interleaved else np.arange(half)
        ib = ia + 1 if self.interleaved else ia + half
        y, a, b = x.copy(), x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        mag[..., ia] = mag[..., ib] = np.abs(a) + np.abs(b)
        return y, mag

    def check(self, before, skipped=()):
        t, D = self.t, self.D
        tables = t["block_tables"].cpu().numpy()
        pos = np.concatenate([np.arange(c, c + k + 1) for c, k in zip(self.ctx, self.k)])
        safe = np.minimum(pos, (t["rope"].shape[0] if self.rot else 1 << 30) - 1)
        req = np.repeat(np.arange(len(self.k)), np.array(self.k) + 1)
        on = ~np.isin(req, list(skipped))
        q, qm = self.rotated(before["q"], safe)
        got = t["q_out"].double().cpu().numpy()
        half_ulp = 2.0 ** -8 if t["q_out"].dtype == torch.bfloat16 else 2.0 ** -24
        assert np.all(np.abs(got - q)[on] <= (half_ulp * np.abs(q) + 2.0 ** -22 * qm)[on])
        assert torch.equal(t["context_lens"], before["context_lens"])
        for n in "kv":
            x, mag = self.rotated(before[n + "_new"], safe) if n == "k" else (before["v_new"].double().cpu().numpy(),) * 2
            old, new = before[n + "_cache"].cpu(), t[n + "_cache"].cpu()
            same = torch.ones(new.shape, dtype=torch.bool)
            if self.cache == "e4m3":
                sc0, sc1 = before[n + "_scale"].double().cpu().numpy(), t[n + "_scale"].double().cpu().numpy()
                scale_same = np.ones(sc1.shape, bool)
            row = 0
            for r, (c, k) in enumerate(zip(self.ctx, self.k)):
                p = c
                while p <= c + k:
                    lo, hi = p % PAGE, min(PAGE, p % PAGE + c + k + 1 - p)
                    fresh, m = x[row:row + hi - lo].transpose(1, 0, 2), np.abs(mag[row:row + hi - lo]).transpose(1, 0, 2)
                    row, p = row + hi - lo, p + hi - lo
                    if r in skipped:
                        continue
                    page = tables[r, (p - 1) // PAGE]
                    assert 0 <= page < new.shape[0]
                    if self.cache != "e4m3":
                        same[page, :, lo:hi] = False
                        u = 2.0 ** -8 if new.dtype == torch.bfloat16 else 2.0 ** -24
                        assert np.all(np.abs(new[page, :, lo:hi].double().numpy() - fresh) <= u * np.abs(fresh) + 2.0 ** -22 * m)
                        continue
                    same[page, :, :hi] = False
                    scale_same[page] = False
                    live = np.concatenate([E4M3[old[page, :, :lo].numpy()] * sc0[page][:, None, None], fresh], 1)
                    slack = np.concatenate([np.zeros((self.Hkv, lo, D)), 2.0 ** -22 * m], 1)
                    peak = np.abs(live).max(axis=(1, 2))
                    for h in range(self.Hkv):
                        s = sc1[page, h]
                        assert s in (scale_of(peak[h] * (1 - 2.0 ** -21)), scale_of(peak[h] * (1 + 2.0 ** -21)))
                    s = sc1[page][:, None, None]
                    got = E4M3[new[page, :, :hi].numpy()] * s
                    assert np.all(np.abs(got - live) <= np.maximum(2.0 ** -4 * np.abs(live), 2.0 ** -10 * s) + slack)
            assert torch.equal(new[same], old[same]), "slots that belong to nobody's new rows keep their values"
            if self.cache == "e4m3":
                assert np.array_equal(sc0[scale_same], sc1[scale_same])


K_CTX = {"single_tokens": ([0] * 7, [0, 1, 15, 16, 17, 31, 500]),
         "drafts": ([0, 3, 8, 1, 15, 16, 40, 5], [0, 13, 16, 31, 1, 15, 7, 1000]),
         "one_prompt": ([777], [0]),
         "prompts": ([100, 0, 300, 63], [5, 0, 129, 16])}


@pytest.mark.parametrize("shape", list(K_CTX))
@pytest.mark.parametrize("dtype,cache", [("bf16", "e4m3"), ("f32", "e4m3"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("D,rot,interleaved,fused", [(128, 128, False, True), (128, 64, True, False), (64, 32, False, True),
                                                     (64, 64, True, True), (128, 0, False, True), (128, 16, False, False)])
def test_matches_the_definition(shape, dtype, cache, D, rot, interleaved, fused):
    k, ctx = K_CTX[shape]
    c = Case(len(shape) + D + rot, k=k, ctx=ctx, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, cache=cache, D=D,
             rot=rot, interleaved=interleaved, fused=fused)
    before = c.snapshot()
    c.run()
    c.check(before)
    # once more on the same inputs: the pages are there and the codes repeat to the bit
    after = c.snapshot()
    c.run()
    for n, v in c.t.items():
        assert torch.equal(v, after[n]), n


@pytest.mark.parametrize("Hq,Hkv", [(28, 4), (1, 1), (40, 40), (71, 1), (32, 17)])
def test_head_counts(Hq, Hkv):
    c = Case(Hq, k=[2, 0, 17], ctx=[30, 16, 3], Hq=Hq, Hkv=Hkv)
    before = c.snapshot()
    c.run()
    c.check(before)


def test_without_queries_and_queries_in_place():
    c = Case(3, k=[4, 9], ctx=[12, 100])
    before = c.snapshot()
    c.run(q=None, q_out=None)
    assert torch.equal(c.t["q_out"], before["q_out"])
    q = before["q"].clone(memory_format=torch.contiguous_format)
    c.run(q=q, q_out=q)
    c.t["q_out"] = q
    c.check(before)


def test_the_scale_shrinks_after_a_large_row_went():
    c = Case(5, k=[3], ctx=[5], missing=False)
    c.t["k_new"][0] *= 1000
    c.run()
    big = c.t["k_scale"].clone()
    c.t["k_new"][0] /= 1000  # the same positions once more, as after a rejection of all drafts
    before = c.snapshot()
    c.run()
    c.check(before)
    assert (c.t["k_scale"] < big).any()


def test_infinities_nan_and_zeros():
    c = Case(6, k=[0, 5, 0, 20], ctx=[16, 32, 33, 0], rot=0, missing=False)
    c.t["v_new"][0] = 0                      # a page of zeros: scale 1, codes 0
    c.t["v_new"][1, 0, 3] = math.inf
    c.t["v_new"][2, 0, 4] = -math.inf
    c.t["v_new"][3, 1, 5] = math.nan
    v = c.t["v_new"].double().cpu().numpy()
    c.run()
    pages = c.t["block_tables"].cpu().numpy()
    code = lambda page, h, s, d: E4M3[int(c.t["v_cache"][page, h, s, d])]
    p0, p1 = pages[0, 1], pages[1, 2]
    assert torch.all(c.t["v_scale"][p0] == 1) and torch.all(c.t["v_cache"][p0, :, 0] == 0)
    fin = np.where(np.isfinite(v[1:7]), np.abs(v[1:7]), 0).max(axis=(0, 2))
    assert [c.t["v_scale"][p1, h].item() for h in range(2)] == [scale_of(f) for f in fin]
    assert code(p1, 0, 0, 3) == 448 and code(p1, 0, 1, 4) == -448 and math.isnan(code(p1, 1, 2, 5))
    ok = np.isfinite(v[1:7]).transpose(1, 0, 2)
    got = E4M3[c.t["v_cache"][p1, :, :6].cpu().numpy()] * c.t["v_scale"][p1].double().cpu().numpy()[:, None, None]
    want = v[1:7].transpose(1, 0, 2)
    s = c.t["v_scale"][p1].double().cpu().numpy()[:, None, None]
    assert np.all(np.abs(got - want)[ok] <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * s)[ok])


@pytest.mark.parametrize("factor", [2.0 ** -110, 2.0 ** -60, 2.0 ** 60, 2.0 ** 118])
def test_extreme_magnitudes(factor):
    c = Case(7, k=[18], ctx=[0], dtype=torch.float32, rot=0)
    c.t["v_new"] *= factor
    c.t["k_new"] *= factor
    before = c.snapshot()
    c.run()
    if factor > 2.0 ** -100:
        c.check(before)
    else:  # under the least scale: rounded to its lowest codes
        s = c.t["v_scale"][c.t["block_tables"][0, :2].long()]
        assert torch.all(s == 2.0 ** -96)


def test_requests_past_the_table_or_without_pages_are_skipped():
    from paper_2601_11652_gb300 import binding as wb
    c = Case(8, k=[3, 4, 2], ctx=[40, 62, 9], positions=66)
    before = c.snapshot()
    c.t["q_out"][:] = -7
    assert c.run(expect=1) == 1          # 62 + 5 > 66: bad length, request 1
    c.check(before, skipped=[1])
    assert torch.all(c.t["q_out"][4:9] == -7)
    c = Case(9, k=[3, 40, 2], ctx=[40, 62, 9])
    c.t["free_count"][0] = 2             # request 1 wants three pages: it and those after it get none
    before = c.snapshot()
    assert c.run(expect=7) in (1, 2)     # whichever reports first
    c.check(before, skipped=[1, 2])
    c = Case(10, k=[3], ctx=[40], missing=False)
    c.t["block_tables"][0, 2] = 10 ** 6
    assert c.run(expect=2) == 0
    assert wb.DEVICE_CODES[2] == "bad_block"


def test_on_another_stream_and_captured():
    c = Case(11, k=[3, 8, 0], ctx=[40, 62, 9])
    before = c.snapshot()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.run(stream=s)
    c.check(before)
    from paper_2601_11652_gb300 import binding as wb
    c = Case(12, k=[3, 8, 0], ctx=[40, 62, 9])
    before = c.snapshot()
    a = c.args()
    ws = wb.alloc_workspace(wb.wisp_kv_rope_workspace_size(a))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wb.wisp_kv_reserve_append_rope(a, ws)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    c.check(before)


def test_empty_batch():
    from paper_2601_11652_gb300 import binding as wb
    c = Case(13, k=[0], ctx=[0])
    z = lambda n: c.t[n][:0]
    a = wb.make_kv_rope_args(**{**c.t, **{n: z(n) for n in ("draft_lens", "context_lens", "block_tables", "q", "k_new", "v_new", "q_out")}})
    ws = wb.alloc_workspace(4096)
    before = c.t["k_cache"].clone()
    wb.wisp_kv_reserve_append_rope(a, ws)
    torch.cuda.synchronize()
    assert wb.wisp_verify_get_device_status(ws)[0] == 0 and torch.equal(before, c.t["k_cache"])


@pytest.mark.parametrize("B", [3, 1023, 1024, 1025, 1500])
@pytest.mark.parametrize("why", ["no_blocks", "bad_block"])
def test_queries_of_a_request_refused_for_its_pages_stay(why, B):
    """Whatever the batch's size: a refused request's queries are not written, so that in place they may be sent again."""
    k = [3, 40, 2] + [0] * (B - 3)
    ctx = [40, 62, 9] + [17] * (B - 3)

    def refuse(c):
        if why == "no_blocks":  # request 1 wants three pages: it gets none, and those after it that need one neither
            c.t["free_count"][0] = 2
            return 7, [1, 2] + list(range(3, B))
        c.t["block_tables"][1, 0] = 10 ** 6
        return 2, [1]

    for in_place in (False, True):
        c = Case(B, k=k, ctx=ctx, D=64, Hq=2, Hkv=1, rot=32)
        code, skipped = refuse(c)
        if in_place:
            c.t["q"] = c.t["q"].clone(memory_format=torch.contiguous_format)
            c.t["q_out"] = c.t["q"]
        before = c.snapshot()
        c.run(expect=code)
        rows = torch.from_numpy(np.isin(np.repeat(np.arange(B), np.array(k) + 1), skipped)).cuda()
        assert torch.equal(c.t["q_out"][rows], before["q_out"][rows])
        c.check(before, skipped=skipped)
        if in_place and why == "no_blocks":  # pages are freed: the refused requests' own queries, sent again, are rotated once
            c.t["free_count"][0] = len(c.free)
            c.t["free_blocks"][:] = torch.tensor(c.free + [0] * (c.t["free_blocks"].numel() - len(c.free)), dtype=torch.int32)
            c.t["block_tables"].copy_(before["block_tables"])
            c.t["q"][~rows] = before["q"][~rows]
            c.run()
            c.check(before)


@pytest.mark.parametrize("B", [1023, 1024, 1025, 1500])
def test_many_requests(B):
    rng = np.random.default_rng(B)
    c = Case(B, k=rng.integers(0, 6, B), ctx=rng.integers(0, 60, B), D=64, Hq=2, Hkv=1)
    before = c.snapshot()
    c.run()
    c.check(before)


@pytest.mark.parametrize("B", [5, 1025])
def test_a_negative_length_and_rows_of_nobody(B):
    # request 1's length is negative: it counts as 0 where the rows of those after it begin
    c = Case(B, k=[2, 0, 7] + [1] * (B - 3), ctx=[20, 30, 9] + [33] * (B - 3), D=64, Hq=2, Hkv=1)
    c.t["draft_lens"][1] = -3
    before = c.snapshot()
    assert c.run(expect=1) == 1
    c.check(before, skipped=[1])
    assert torch.all(c.t["q_out"][3] == -7)
    # more rows than the requests have
    c = Case(B + 1, k=[2, 5, 7] + [1] * (B - 2), ctx=[20, 30, 9] + [33] * (B - 2), D=64, Hq=2, Hkv=1)
    before = c.snapshot()
    short = {n: c.t[n][:-1] for n in ("draft_lens", "context_lens", "block_tables")}
    c.run(expect=1, **short)
    c.check(before, skipped=[B])
    assert torch.all(c.t["q_out"][-2:] == -7)


def _round_past_the_rotation(rot):
    """Request 1 has pages for 80 tokens and wants positions 62 .. 66 of a table for 66: the append refuses it.  Then a step over the
    pool and the commit."""
    from paper_2601_11652_gb300 import binding as wb
    c = Case(8, k=[3, 4, 2], ctx=[40, 62, 9], positions=66, missing=False, Hq=8, Hkv=2, rot=rot)
    t, B, T, Td, V = c.t, 3, 12, 9, 1000
    g = torch.Generator(device="cuda").manual_seed(3)
    acc_len, tok = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    a = c.args(accepted_len=acc_len)
    ws = wb.alloc_workspace(wb.wisp_kv_rope_workspace_size(a))
    wb.wisp_kv_reserve_append_rope(a, ws)
    attn = wb.make_attn_kv8_args(draft_lens=t["draft_lens"], context_lens=t["context_lens"], block_tables=t["block_tables"], q=t["q_out"],
                                 k_cache=t["k_cache"], v_cache=t["v_cache"], k_scale=t["k_scale"], v_scale=t["v_scale"],
                                 out=torch.empty_like(t["q_out"]))
    acc = wb.make_accept_args(draft_lens=t["draft_lens"], target_logits=torch.randn((T, V), generator=g, device="cuda"),
                              draft_tokens=torch.arange(Td, dtype=torch.int32, device="cuda"),
                              draft_probs=torch.full((Td, V), 1 / V, device="cuda"), accept_uniforms=torch.zeros(Td, device="cuda"),
                              sample_uniforms=torch.full((B,), 0.5, device="cuda"), accepted_len=acc_len, next_token=tok)
    vws = wb.alloc_workspace(wb.wisp_verify_workspace_size(attn.attn, acc))
    wb.wisp_verify_step_kv8(attn, acc, vws)
    cws = wb.alloc_workspace(wb.wisp_kv_rope_workspace_size(a))
    wb.wisp_kv_commit_rope(a, cws)
    torch.cuda.synchronize()
    return c, acc_len.tolist(), [wb.wisp_verify_get_device_status(w)[0] for w in (ws, vws, cws)], wb.wisp_verify_get_device_status(cws)[1]


def test_commit_leaves_a_request_past_the_rotation():
    c, L, codes, who = _round_past_the_rotation(rot=64)
    assert codes == [1, 0, 1] and who == 1 and min(L) >= 0
    assert c.t["context_lens"].tolist() == [40 + 1 + L[0], 62, 9 + 1 + L[2]]
    # a cache without a rotation: the block table alone limits it
    c, L, codes, _ = _round_past_the_rotation(rot=0)
    assert codes == [0, 0, 0]
    assert c.t["context_lens"].tolist() == [40 + 1 + L[0], 62 + 1 + L[1], 9 + 1 + L[2]]
