"""GPU: the serving loop over an 8-bit cache, with rotation on the way in and log probabilities beside the tokens.

Sessions are served twice on the same payloads: with the plain pool, for the accepted lengths and tokens (they depend on
the logits alone, and have to be equal), and with an e4m3 pool, a rotation table and `top_n`.  The second's pool, attention
outputs and log probabilities are compared with 64-bit formulas of what went in.
"""
import numpy as np
import pytest
import torch

from paper_2601_11652_gb300 import workload as wl

pytestmark = pytest.mark.gpu

V, NB, MB, TOP = 3000, 300, 40, 4
PREFIX = [40, 1, 333, 16, 127]
KS = [[3, 0, 5, 1, 8], [2, 4, 0, 6, 1], [1, 3, 8, 0, 5]]


def bits(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16).double()


def values(a):
    return bits(a) if a.dtype == np.uint16 else torch.from_numpy(a).double()


def rotate(x, pos, table, interleaved):
    """x [rows, heads, D] rotated by the rows' positions, in 64 bits."""
    half = table.shape[1] // 2
    c, s = table[pos, None, :half].double(), table[pos, None, half:].double()
    x = x.clone()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    u, v = x[..., a].clone(), x[..., b].clone()
    x[..., a], x[..., b] = u * c - v * s, v * c + u * s
    return x


@pytest.mark.parametrize("cache,Hq,Hkv,D,rot,interleaved", [
    ("e4m3", 8, 2, 128, 64, False), ("e4m3", 4, 4, 64, 64, True), ("e4m3", 8, 2, 64, 0, False),
    (None, 8, 2, 128, 64, False), (None, 4, 4, 64, 64, True)])
def test_rounds_of_a_server(cache, Hq, Hkv, D, rot, interleaved):
    from paper_2601_11652_gb300 import build, serve
    build.build()
    n = len(PREFIX)
    sids = list(range(n))
    ang = torch.arange(MB * 16)[:, None].double() * 10000.0 ** (-torch.arange(rot // 2).double() / max(1, rot // 2))
    table = torch.cat([ang.cos(), ang.sin()], 1).float() if rot else None
    plain = serve.PagedSessions(n, Hkv, D, "bf16", NB, MB)
    sess = serve.PagedSessions(n, Hkv, D, "bf16", NB, MB, cache=cache, rope=table, interleaved=interleaved)
    first = [wl.make_round((31, s), k=0, Hq=Hq, Hkv=Hkv, D=D, V=V, prefix=PREFIX[s]) for s in sids]
    for x in (plain, sess):
        x.prefill(sids, [f["prefix_k"] for f in first], [f["prefix_v"] for f in first])
    keys = [rotate(values(f["prefix_k"]), torch.arange(p), table, interleaved) if rot else values(f["prefix_k"])
            for f, p in zip(first, PREFIX)]
    vals = [values(f["prefix_v"]) for f in first]
    server = serve.VerifyServer(sess, Hq, V, top_n=TOP)
    other = serve.VerifyServer(plain, Hq, V)
    for rnd, ks in enumerate(KS):
        d = [wl.make_round((32, rnd, s), k=ks[s], Hq=Hq, Hkv=Hkv, D=D, V=V) for s in sids]
        pay = [serve.Payload(x["q"], x["k_new"], x["v_new"], x["logits"], x["draft_tokens"], x["draft_probs"], x["accept_u"],
                             x["sample_u"]) for x in d]
        want, got = other.run_batch(sids, pay), server.run_batch(sids, pay)
        assert want.logprob is None
        assert np.array_equal(want.accepted_len, got.accepted_len) and np.array_equal(want.next_token, got.next_token)
        assert (got.accepted_len >= 0).all()
        row = 0
        for s in sids:
            k, L = ks[s], int(got.accepted_len[s])
            ctx = len(keys[s])
            pos = torch.arange(ctx, ctx + k + 1)
            kn, q = values(d[s]["k_new"]), values(d[s]["q"])
            if rot:
                kn, q = rotate(kn, pos, table, interleaved), rotate(q, pos, table, interleaved)
            kall, vall = torch.cat([keys[s], kn]), torch.cat([vals[s], values(d[s]["v_new"])])
            # the pool: a code is within 2^-4 of its value, or half of the least step, 2^-9 of the scale; and of what it was
            # before where its page has been encoded again since.  A page's scales are at most a factor of 4 apart (the largest of
            # 64 normal values or more; a rejected one may have had the largest): 2^-8 and 2^-10 of the last, 2^-7 allowed.
            # Rows of the queries' type are rounded once.  2^-20: the rotation in 32 bits
            pages = torch.from_numpy(got.block_tables[s][: (ctx + k) // 16 + 1]).long().cuda()
            dec = {}
            for name, x in (("k", kall), ("v", vall)):
                pool = getattr(sess, name + "_cache")[pages].double()
                big = x.abs().max() * 2.0 ** -20
                if cache:
                    sc = sess.scales[name + "_scale"][pages].double()[:, :, None, None]
                    pool, step = pool * sc, (sc * 2.0 ** -7).expand(pool.shape)
                flat = lambda y: y.transpose(1, 2).reshape(-1, Hkv, D)[: ctx + k + 1].cpu()
                dec[name] = flat(pool)
                allowed = 2.0 ** -4 * x.abs() + flat(step) + big if cache else 2.0 ** -8 * x.abs() + big
                assert ((dec[name] - x).abs() <= allowed).all()
            # the attention over the pool as it is: 2^-8 of the outputs and 2^-7 of the weighted magnitudes.  A query element whose
            # rounding to bf16 the rotation in 32 bits tips (one in 2^15) moves by 2^-8 of itself: with two of them in a row
            # its scores move by e, its weights by a factor of exp(2 e)
            out = got.out[row:row + k + 1].double().cpu()
            g = Hq // Hkv
            K, W = dec["k"].repeat_interleave(g, 1), dec["v"].repeat_interleave(g, 1)
            qb = q.to(torch.bfloat16).double() if rot else q
            sc = torch.einsum("jhd,thd->hjt", qb, K) / D ** 0.5
            see = torch.arange(ctx + k + 1)[None, :] <= pos[:, None]
            p = torch.softmax(sc.masked_fill(~see, -np.inf), -1)
            ref, mag = torch.einsum("hjt,thd->jhd", p, W), torch.einsum("hjt,thd->jhd", p, W.abs())
            e = 2.0 ** -7 * q.abs().amax((1, 2)) * K.abs().max() / D ** 0.5 if rot else torch.zeros(k + 1)
            far = torch.expm1(2.0 * e)[:, None, None]
            assert ((out - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -7 + far) * mag).all()
            # the log probabilities of what the rows committed
            tokens = list(d[s]["draft_tokens"][:L]) + [got.next_token[s]] + [-1] * (k - L)
            assert got.row_tokens[row:row + k + 1].tolist() == [int(t) for t in tokens]
            z = values(d[s]["logits"])
            lp = torch.log_softmax(z, 1)
            for i in range(k + 1):
                at = row + i
                if tokens[i] < 0:
                    assert got.logprob[at] == 0 and got.entropy[at] == 0 and (got.top_tokens[at] == -1).all()
                    continue
                tol = 2.0 ** -16 + 2.0 ** -22 * z[i].abs().max().item()
                assert abs(got.logprob[at] - lp[i, tokens[i]].item()) <= tol
                assert abs(got.entropy[at] + (lp[i].exp() * lp[i]).sum().item()) <= 16 * tol
                best = sorted(range(V), key=lambda t: (-z[i, t].item(), t))[:TOP]
                assert got.top_tokens[at].tolist() == best
                assert np.abs(got.top_logprobs[at] - lp[i, best].numpy()).max() <= tol
            keys[s], vals[s] = kall[: ctx + 1 + L], vall[: ctx + 1 + L]
            row += k + 1
        assert torch.equal(sess.ctx, plain.ctx) and torch.equal(sess.free_count, plain.free_count)
        assert sess.ctx.tolist() == [len(x) for x in keys]


def test_refusals():
    from paper_2601_11652_gb300 import binding as wb, build, serve
    build.build()
    with pytest.raises(ValueError):
        serve.PagedSessions(1, 2, 128, "bf16", 8, 4, cache="fp8")
    sess = serve.PagedSessions(1, 2, 128, "bf16", 8, 4, cache="e4m3", rope=torch.zeros((8, 64)))
    f = wl.make_round((33, 0), k=0, Hq=4, Hkv=2, D=128, V=64, prefix=9)
    with pytest.raises(RuntimeError):  # nine positions, eight in the table
        sess.prefill([0], [f["prefix_k"]], [f["prefix_v"]])
    server = serve.VerifyServer(serve.PagedSessions(1, 2, 128, "bf16", 8, 4), 4, 64, top_n=33)
    pay = serve.Payload(f["q"], f["k_new"], f["v_new"], f["logits"], f["draft_tokens"], f["draft_probs"], f["accept_u"], f["sample_u"])
    with pytest.raises(wb.WispError):
        server.run_batch([0], [pay])
