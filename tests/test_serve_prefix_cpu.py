"""Batches of sessions that share pages, without a GPU: what the server hands to the library, and for how long.  The library's calls are
stood in for; what they would read is looked at when they are called."""
import contextlib
import types
import weakref

import numpy as np
import pytest
import torch

from paper_2601_11652_gb300 import serve

HQ, HKV, D, V = 4, 2, 64, 8


class Stream:
    def __init__(self, log, name):
        self.log, self.name = log, name

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))

    def synchronize(self):
        pass


@pytest.fixture
def fake(monkeypatch):
    """Calls in order (.log), and per attention call over shared pages the ids and pages that it would have read (.read)."""
    f = types.SimpleNamespace(log=[], read=[], refs=None)

    def make_shared(**kw):
        f.refs = {n: weakref.ref(kw[n]) for n in ("shared_ids", "shared_pages", "draft_lens", "context_lens", "block_tables", "q", "out")}
        return types.SimpleNamespace()

    def shared_call(args, ws, stream=None):
        alive = {n: r() for n, r in f.refs.items()}
        gone = [n for n, t in alive.items() if t is None]
        assert not gone, f"{gone}: freed before the call that reads them"
        f.log.append(("attention", getattr(stream, "name", None)))
        f.read.append((alive["shared_ids"].tolist(), alive["shared_pages"].tolist()))

    def called(name):
        return lambda *a, **kw: f.log.append((name, getattr(a[-1], "name", None)))

    wb = serve.wb
    for n in ("make_kv_args", "make_attn_args", "make_accept_args", "make_prompt_args"):
        monkeypatch.setattr(wb, n, lambda **kw: types.SimpleNamespace())
    monkeypatch.setattr(wb, "make_shared_args", make_shared)
    monkeypatch.setattr(wb, "wisp_verify_attention_shared", shared_call)
    for n in ("wisp_kv_reserve_append", "wisp_kv_commit", "wisp_verify_step", "wisp_verify_accept", "wisp_prompt_attention"):
        monkeypatch.setattr(wb, n, called(n))
    for n in ("wisp_kv_workspace_size", "wisp_verify_workspace_size", "wisp_verify_shared_workspace_size", "wisp_prompt_workspace_size"):
        monkeypatch.setattr(wb, n, lambda *a: 1)
    monkeypatch.setattr(wb, "alloc_workspace", lambda n, dev=None: torch.zeros(1))
    monkeypatch.setattr(wb, "wisp_verify_get_device_status", lambda ws: (0, 0))
    f.current = Stream(f.log, "current")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: f.current)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "synchronize", lambda dev=None: None)
    monkeypatch.setattr(torch.cuda, "Event", lambda **kw: types.SimpleNamespace(record=lambda s: None, elapsed_time=lambda o: 0.0))
    return f


def payload(k):
    z = lambda *s: np.zeros(s, np.float32)
    return serve.Payload(z(k + 1, HQ, D), z(k + 1, HKV, D), z(k + 1, HKV, D), z(k + 1, V), np.zeros(k, np.int32), z(k, V), z(k), 0.5)


def sessions(n, shared, pages):
    """Session 0 with 100 tokens in pages 20 .. 26, `shared` behind its first pages."""
    s = serve.PagedSessions(n, HKV, D, "f32", 64, 8, device="cpu")
    s.ctx[0] = 100
    s.tables[0, :7] = torch.arange(20, 27)
    s.share(0, shared, pages * 16)
    return s


def test_what_the_attention_reads_lives_until_it_is_called(fake):
    s = sessions(4, [1, 3], 2)
    server = serve.VerifyServer(s, HQ, V)
    server.run_batch([3, 2, 0, 1], [payload(k) for k in (1, 0, 2, 0)])
    ids, pages = fake.read[0]
    assert ids.count(0) == 3 and [p for i, p in zip(ids, pages) if i == 0] == [2, 2, 2]


@pytest.mark.parametrize("shared", [False, True])
def test_another_stream_waits_for_the_batch_that_it_reads(fake, shared):
    """Rows, lengths and tables of a batch are written on the current stream."""
    s = sessions(4, [1, 3], 2)
    other = Stream(fake.log, "other")
    server = serve.VerifyServer(s, HQ, V, stream=other)
    server.run_batch([3, 1] if shared else [2], [payload(1) for _ in range(2 if shared else 1)])
    assert fake.log.index(("other", "waits for", "current")) < fake.log.index(("wisp_kv_reserve_append", "other"))
    assert (("attention", "other") in fake.log) == shared


@pytest.mark.parametrize("queries", [False, True])
def test_a_prefill_on_another_stream_waits_for_its_rows(fake, queries):
    s = sessions(4, [1], 2)
    z = lambda *x: np.zeros(x, np.float32)
    s.prefill([2], [z(5, HKV, D)], [z(5, HKV, D)], stream=Stream(fake.log, "other"), q_rows=[z(5, HQ, D)] if queries else None)
    assert fake.log.index(("other", "waits for", "current")) < fake.log.index(("wisp_kv_reserve_append", "other"))
    assert (("wisp_prompt_attention", "other") in fake.log) == queries


def test_a_session_used_anew_leaves_its_run(fake):
    """The block tables say what is shared: a session that has been emptied and given other pages reads its own."""
    s = sessions(6, [1, 2, 3], 2)
    server = serve.VerifyServer(s, HQ, V)
    s.tables[2], s.ctx[2] = -1, 0            # emptied, and ...
    s.tables[2, :3] = torch.tensor([40, 41, 42])
    s.ctx[2] = 45                            # ... filled again
    s.tables[3], s.ctx[3] = -1, 0            # emptied
    server.run_batch([0, 1, 2, 3], [payload(1) for _ in range(4)])
    assert fake.read[-1] == ([0, 0, -1, -1], [2, 2, 2, 2])
    s.tables[0], s.ctx[0] = -1, 0            # now the run's own source
    s.tables[0, :3] = torch.tensor([50, 51, 52])
    s.ctx[0] = 48
    server.run_batch([0, 1, 2, 3], [payload(1) for _ in range(4)])
    assert fake.read[-1][0][1:] == [-1, -1, -1]   # (a run of one is computed alone)


def test_a_prefill_of_an_empty_session_ends_its_sharing(fake):
    s = sessions(6, [1, 2], 2)
    s.tables[1], s.ctx[1] = -1, 0
    z = lambda *x: np.zeros(x, np.float32)
    s.prefill([1, 2], [z(5, HKV, D)] * 2, [z(5, HKV, D)] * 2)
    assert s.prefix[:3] == [(0, 2), (-1, 0), (0, 2)]  # (session 2 has its shared pages and gets its next tokens)
