"""A bounded decoding session's bookkeeping (CPU tensors, no kernels): a call that raises takes back what it counted, a cut frees the
pages behind the budget, and only sequences beyond it are cut."""
from contextlib import nullcontext
from types import SimpleNamespace

import pytest
import torch

from paper_2511_03983_b200 import engine as E


def session(monkeypatch, S=2, n=2, page_size=4, max_len=24, keep=8, slack=3):
    s = E.DecodeSession.__new__(E.DecodeSession)
    s.S, s.n, s.page_size, s.max_len, s.keep, s.slack, s.recent = S, n, page_size, max_len, keep, slack, 2
    s.max_pages = -(-max_len // page_size)
    s.n_pages = S * n * s.max_pages
    s.free = list(range(s.n_pages - 1, -1, -1))
    s.lens, s.seen = [[0] * n for _ in range(S)], [[0] * n for _ in range(S)]
    s.pages = [[[] for _ in range(n)] for _ in range(S)]
    s.page_table = torch.zeros(S, n, s.max_pages, dtype=torch.int32)
    s.kv_len, s.new_len, s.seen_len, s.keep_len, s.new_pos = (torch.zeros(S, n, dtype=torch.int32) for _ in range(5))
    s.x = [torch.zeros(S, n, 8), torch.zeros(S, n, 8)]
    s.use_graph, s.graph = False, None
    s.weights = s.slot_pos = [None, None]
    s.evict_ws = None
    s.pools = [torch.zeros(1, 2, 1)] * 2
    s.eng = SimpleNamespace(w=SimpleNamespace(n_layers=2, d_model=8, d_head=8, dtype=1), _bind=lambda l: None, kv_max=1, kv_count=[None, None],
                            launches=0, _timed=lambda name: nullcontext())
    calls = []
    monkeypatch.setattr(E.B, "kv_evict_args", lambda *a, **k: k)
    monkeypatch.setattr(E.B, "twist_kv_evict", lambda k: calls.append((k["keep"].tolist(), k["kv_len"].tolist())))
    s._layers = lambda: None
    return s, calls


def test_steps_cut_what_has_grown_beyond_the_budget_and_free_its_pages(monkeypatch):
    s, calls = session(monkeypatch)
    x = torch.zeros(2, 2, 8)
    with s._growing([[10, 3], [0, 12]]):
        pass
    s.step(x)                                                     # 12 tokens are beyond 8 + 3, 10 are not
    assert calls == [([[10, 3], [0, 8]], [[10, 3], [0, 12]])] * 2
    assert s.lens == [[11, 4], [1, 9]] and s.seen == [[11, 4], [1, 13]]
    assert [[len(p) for p in r] for r in s.pages] == [[3, 1], [1, 3]]
    assert s.kv_len.tolist() == s.lens and s.seen_len.tolist() == s.seen and s.new_pos.tolist() == [[10, 3], [0, 12]]
    s.evict()                                                     # by hand: all that is beyond the budget
    assert s.lens == [[8, 4], [1, 8]] and [[len(p) for p in r] for r in s.pages] == [[2, 1], [1, 2]]
    assert s.seen == [[11, 4], [1, 13]] and len(calls) == 4
    s.evict()
    assert len(calls) == 4
    assert sorted(s.free + [p for r in s.pages for q in r for p in q]) == list(range(s.n_pages))
    s.release(1, 1)
    assert s.seen[1][1] == 0 and s.kv_len.tolist()[1][1] == 0 and s.seen_len.tolist()[1][1] == 0


def test_a_call_that_raises_takes_back_what_it_counted(monkeypatch):
    s, calls = session(monkeypatch)
    with s._growing([[5, 6], [7, 8]]):
        pass
    state = lambda: ([list(r) for r in s.lens], [list(r) for r in s.seen], [[list(p) for p in r] for r in s.pages], list(s.free), s.kv_len.tolist(),
                     s.seen_len.tolist())
    before = state()

    def fails():
        raise IndexError("list index out of range")
    s._layers = fails
    with pytest.raises(IndexError):
        s.step(torch.zeros(2, 2, 8))
    assert state() == before and not calls
    with pytest.raises(ValueError):                               # more than the cache's room
        with s._growing([[1, 30], [0, 0]]):
            pass
    assert state() == before

    def refuses(k):
        raise E.B.TwistError(-2, "twist_kv_evict")
    monkeypatch.setattr(E.B, "twist_kv_evict", refuses)
    with s._growing([[6, 0], [0, 0]]):
        pass
    before = state()
    with pytest.raises(E.B.TwistError):
        s.step(torch.zeros(2, 2, 8))
    assert state() == before
