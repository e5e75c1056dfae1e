"""Cuts of a bounded decoding session that fail, and what they are launched with (CPU tensors, no kernels)."""
import pytest
import torch

from paper_2511_03983_b200 import engine as E
from test_small_cache_session_cpu import session


def grown(monkeypatch, lens=((12, 3), (0, 14))):
    s, calls = session(monkeypatch)
    with s._growing([list(r) for r in lens]):
        pass
    return s, calls


def state(s):
    return [list(r) for r in s.lens], [list(r) for r in s.seen], [[list(p) for p in r] for r in s.pages], list(s.free), s.kv_len.tolist()


def failing(monkeypatch, at):
    """The `at`-th call of twist_kv_evict raises."""
    calls = []

    def evict(k):
        if len(calls) == at:
            raise E.B.TwistError(-2, "twist_kv_evict")
        calls.append(k)
    monkeypatch.setattr(E.B, "twist_kv_evict", evict)
    return calls


def test_a_cut_that_fails_behind_its_first_layer_closes_the_session_until_all_is_released(monkeypatch):
    s, _ = grown(monkeypatch)
    calls = failing(monkeypatch, 1)
    before = state(s)
    with pytest.raises(E.B.TwistError):
        s.step(torch.zeros(2, 2, 8))
    assert len(calls) == 1 and state(s) == before
    for call in (lambda: s.step(torch.zeros(2, 2, 8)), s.evict, lambda: s.evict(3)):
        with pytest.raises(RuntimeError, match="1 of 2 layers"):
            call()
    assert len(calls) == 1
    s.release(0, 0)
    s.release(1, 1)
    with pytest.raises(RuntimeError):                             # one sequence is left
        s.step(torch.zeros(2, 2, 8))
    s.release(0, 1)
    s.step(torch.zeros(2, 2, 8))
    assert s.lens == [[1, 1], [1, 1]]


def test_a_cut_that_is_refused_before_anything_was_cut_changes_nothing(monkeypatch):
    s, _ = grown(monkeypatch)
    calls = failing(monkeypatch, 0)
    before = state(s)
    with pytest.raises(E.B.TwistError):
        s.evict()
    assert state(s) == before and not calls and s.broken is None
    built = []

    def refused(*a, **k):                                         # the second layer's arguments: the first is not launched
        built.append(k)
        if len(built) == 2:
            raise ValueError("weights")
        return k
    calls = failing(monkeypatch, 10)
    monkeypatch.setattr(E.B, "kv_evict_args", refused)
    with pytest.raises(ValueError):
        s.evict()
    assert state(s) == before and not calls and s.broken is None
    monkeypatch.setattr(E.B, "kv_evict_args", lambda *a, **k: k)
    s.evict()
    assert len(calls) == 2 and s.lens == [[8, 3], [0, 8]]


def test_a_cut_is_laid_out_for_the_longest_sequence_not_for_the_room(monkeypatch):
    s, _ = grown(monkeypatch)
    bounds = []
    monkeypatch.setattr(E.B, "kv_evict_args", lambda *a, **k: bounds.append(k.get("max_len", a[6] if len(a) > 6 else 0)) or k)
    s.evict()
    with s._growing([[1, 6], [0, 3]]):
        pass
    s.evict()
    assert bounds == [14, 14, 11, 11]                             # of 24
