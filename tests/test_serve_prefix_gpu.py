"""GPU: sessions behind a common prompt.  The prompt is prefilled with its attention, its whole pages are shared, each session gets the rest of
its own prompt, and rounds of a server run over them; beside it a server whose sessions each have everything for themselves.  Accepted
lengths and tokens depend on the logits alone and have to be equal; attention outputs are compared with 64-bit formulas over the pool as
it is (bounds as in test_serve_kv8_gpu.py)."""
import numpy as np
import pytest
import torch

from paper_2601_11652_gb300 import workload as wl
from test_serve_kv8_gpu import rotate, values

pytestmark = pytest.mark.gpu

V, NB, MB = 2000, 260, 40
PROMPT, TAILS = 270, [0, 5, 40, 2, 100, 17]   # 16 whole pages and 14 tokens; what each session has behind the whole pages
KS = [[3, 0, 5, 1, 8, 2], [2, 4, 0, 6, 1, 0]]


def check(sess, out, table, ctx, q, pos, rot_table, interleaved):
    """Attention outputs [rows, Hq, D] of queries at positions `pos` of one session, against the pool."""
    Hq, D, Hkv = q.shape[1], q.shape[2], sess.Hkv
    L = int(pos[-1]) + 1
    pages = torch.from_numpy(table[: (L + 15) // 16].astype(np.int64)).cuda()
    kv = {}
    for n in "kv":
        x = getattr(sess, n + "_cache")[pages].double()
        if sess.kv8:
            x = x * sess.scales[n + "_scale"][pages].double()[:, :, None, None]
        kv[n] = x.transpose(1, 2).reshape(-1, Hkv, D)[:L].cpu().repeat_interleave(Hq // Hkv, 1)
    qr = rotate(q, pos, rot_table, interleaved) if rot_table is not None else q
    s = torch.einsum("jhd,thd->hjt", qr.to(torch.bfloat16).double(), kv["k"]) / D ** 0.5
    p = torch.softmax(s.masked_fill(torch.arange(L)[None, :] > pos[:, None], -np.inf), -1)
    ref, mag = torch.einsum("hjt,thd->jhd", p, kv["v"]), torch.einsum("hjt,thd->jhd", p, kv["v"].abs())
    e = 2.0 ** -7 * q.abs().amax((1, 2)) * kv["k"].abs().max() / D ** 0.5 if rot_table is not None else torch.zeros(len(pos))
    far = torch.expm1(2.0 * e)[:, None, None]
    assert ((out.double().cpu() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -7 + far) * mag).all()


@pytest.mark.parametrize("cache,Hq,Hkv,D,rot", [(None, 8, 2, 128, 0), (None, 4, 4, 64, 64), ("e4m3", 8, 2, 128, 64), ("e4m3", 14, 2, 64, 0)])
def test_sessions_behind_one_prompt(cache, Hq, Hkv, D, rot):
    from paper_2601_11652_gb300 import build, serve
    build.build()
    n = len(TAILS)
    ang = torch.arange(MB * 16)[:, None].double() * 10000.0 ** (-torch.arange(rot // 2).double() / max(1, rot // 2))
    table = torch.cat([ang.cos(), ang.sin()], 1).float() if rot else None
    make = lambda: serve.PagedSessions(n + 1, Hkv, D, "bf16", NB, MB, cache=cache, rope=table)
    sess, alone = make(), make()
    draw = lambda key, m: wl.make_round(key, k=m - 1, Hq=Hq, Hkv=Hkv, D=D, V=8)
    prompt = draw((51, 0), PROMPT)
    kn, vn, qn = prompt["k_new"], prompt["v_new"], prompt["q"]
    # the prompt in two chunks, with its attention
    out = torch.cat([sess.prefill([0], [kn[a:b]], [vn[a:b]], q_rows=[qn[a:b]]) for a, b in ((0, 100), (100, PROMPT))])
    check(sess, out, sess.tables[0].cpu().numpy(), 0, values(qn), torch.arange(PROMPT), table, False)
    with pytest.raises(ValueError):
        sess.prefill([1], [kn[:4]], [vn[:4]], q_rows=[qn[:3]])
    whole = PROMPT // 16 * 16
    free = int(sess.free_count)
    sess.share(0, list(range(1, n + 1)), whole)
    assert int(sess.free_count) == free
    # the rest of each session's prompt, all in one call
    tails = {s: draw((52, s), TAILS[s - 1]) for s in range(1, n + 1) if TAILS[s - 1]}
    sids = list(tails)
    out = sess.prefill(sids, [tails[s]["k_new"] for s in sids], [tails[s]["v_new"] for s in sids], q_rows=[tails[s]["q"] for s in sids])
    row = 0
    for s in sids:
        m = TAILS[s - 1]
        check(sess, out[row:row + m], sess.tables[s].cpu().numpy(), 0, values(tails[s]["q"]), whole + torch.arange(m), table, False)
        row += m
    for s in range(1, n + 1):
        parts = [(kn[:whole], vn[:whole])] + ([(tails[s]["k_new"], tails[s]["v_new"])] if s in tails else [])
        assert alone.prefill([s], [np.concatenate([p[0] for p in parts])], [np.concatenate([p[1] for p in parts])]) is None
    server, other = serve.VerifyServer(sess, Hq, V, top_n=3), serve.VerifyServer(alone, Hq, V, top_n=3)
    order = [4, 1, 0, 6, 2, 5, 3]  # (0, the prompt's own session, has its tokens behind the whole pages)
    alone.prefill([0], [kn], [vn])
    for rnd, ks in enumerate(KS):
        d = [wl.make_round((53, rnd, s), k=ks[s - 1] if s else 1, Hq=Hq, Hkv=Hkv, D=D, V=V) for s in order]
        pay = [serve.Payload(x["q"], x["k_new"], x["v_new"], x["logits"], x["draft_tokens"], x["draft_probs"], x["accept_u"],
                             x["sample_u"]) for x in d]
        want, got = other.run_batch(order, pay), server.run_batch(order, pay)
        assert server.shared_ws is not None and other.shared_ws is None
        assert got.sids == order
        for f in ("accepted_len", "next_token", "context_lens", "row_tokens", "logprob", "entropy", "top_tokens", "top_logprobs"):
            assert np.array_equal(getattr(want, f), getattr(got, f)), f
        row = 0
        for i, s in enumerate(order):
            m = len(d[i]["q"])
            check(sess, got.out[row:row + m], got.block_tables[i], 0, values(d[i]["q"]), int(got.context_lens[i]) + torch.arange(m), table, False)
            row += m
        assert torch.equal(sess.ctx, alone.ctx)
        for s in range(1, n + 1):
            assert torch.equal(sess.tables[s, :whole // 16], sess.tables[0, :whole // 16])
    # a batch with one of them alone takes the ordinary step
    server.shared_ws = None
    x = wl.make_round((54, 0), k=2, Hq=Hq, Hkv=Hkv, D=D, V=V)
    server.run_batch([3], [serve.Payload(x["q"], x["k_new"], x["v_new"], x["logits"], x["draft_tokens"], x["draft_probs"], x["accept_u"],
                                         x["sample_u"])])
    assert server.shared_ws is None


def payload_of(x):
    from paper_2601_11652_gb300 import serve
    return serve.Payload(x["q"], x["k_new"], x["v_new"], x["logits"], x["draft_tokens"], x["draft_probs"], x["accept_u"], x["sample_u"])


@pytest.mark.parametrize("rounds", [6])
def test_rounds_without_log_probabilities(rounds):
    """Nothing but the batch's own buffers lies between its arguments and the attention, so that one given back too early would be written over."""
    from paper_2601_11652_gb300 import build, serve
    build.build()
    Hq, Hkv, D, n = 8, 2, 64, 5
    sess = serve.PagedSessions(n, Hkv, D, "bf16", NB, MB)
    x = wl.make_round((61, 0), k=99, Hq=Hq, Hkv=Hkv, D=D, V=8)
    sess.prefill([0], [x["k_new"]], [x["v_new"]])
    sess.share(0, [1, 2, 3, 4], 96)
    server = serve.VerifyServer(sess, Hq, V)
    for i in range(rounds):
        d = [wl.make_round((62, i, s), k=s, Hq=Hq, Hkv=Hkv, D=D, V=V) for s in range(n)]
        got = server.run_batch(list(range(n)), [payload_of(y) for y in d])
        row = 0
        for s in range(n):
            m = s + 1
            check(sess, got.out[row:row + m], got.block_tables[s], 0, values(d[s]["q"]), int(got.context_lens[s]) + torch.arange(m), None, False)
            row += m


@pytest.mark.parametrize("filled_by", ["prefill", "rows"])
def test_a_session_used_anew_reads_its_own_pages(filled_by):
    from paper_2601_11652_gb300 import build, serve
    build.build()
    Hq, Hkv, D, n = 8, 2, 64, 4
    sess = serve.PagedSessions(n, Hkv, D, "bf16", NB, MB)
    x = wl.make_round((63, 0), k=99, Hq=Hq, Hkv=Hkv, D=D, V=8)
    sess.prefill([0], [x["k_new"]], [x["v_new"]])
    sess.share(0, [1, 2, 3], 64)
    sess.tables[2], sess.ctx[2] = -1, 0
    y = wl.make_round((63, 1), k=79, Hq=Hq, Hkv=Hkv, D=D, V=8)
    if filled_by == "prefill":
        sess.prefill([2], [y["k_new"]], [y["v_new"]])
    else:  # (the rows of a session that somebody filled elsewhere)
        extra = serve.PagedSessions(1, Hkv, D, "bf16", 8, MB)
        extra.prefill([0], [y["k_new"]], [y["v_new"]])
        to = torch.arange(NB - 60, NB - 55, device="cuda")
        for name in ("k_cache", "v_cache"):
            getattr(sess, name)[to] = getattr(extra, name)[extra.tables[0, :5].long()]
        sess.tables[2, :5], sess.ctx[2] = to.int(), 80
        keep = sess.free_blocks[:int(sess.free_count)]
        keep = keep[~torch.isin(keep, to.int())]
        sess.free_blocks[:len(keep)] = keep
        sess.free_count.fill_(len(keep))
    server = serve.VerifyServer(sess, Hq, V)
    d = [wl.make_round((64, s), k=2, Hq=Hq, Hkv=Hkv, D=D, V=V) for s in range(n)]
    got = server.run_batch(list(range(n)), [payload_of(z) for z in d])
    for s in range(n):
        check(sess, got.out[3 * s:3 * s + 3], got.block_tables[s], 0, values(d[s]["q"]), int(got.context_lens[s]) + torch.arange(3), None, False)
    assert got.context_lens.tolist() == [100, 64, 80, 64]
