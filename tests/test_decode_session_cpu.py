"""A call of a decoding session that raises counts for nothing: lengths, pages, the free list and the device's lengths are
as before it, whatever step it failed at (CPU tensors in the place of the device's, no kernels)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2511_03983_b200 import engine as E


def session(forward=None, layers=None, S=2, n=2, page_size=4, max_len=10, n_pages=12, n_layers=0):
    """A session without a model: `forward` stands for the engine's forward pass, `layers` for the layers of a step."""
    s = E.DecodeSession.__new__(E.DecodeSession)
    s.S, s.n, s.page_size, s.max_len, s.n_pages = S, n, page_size, max_len, n_pages
    s.max_pages = -(-max_len // page_size)
    s.free = list(range(n_pages - 1, -1, -1))
    s.lens = [[0] * n for _ in range(S)]
    s.pages = [[[] for _ in range(n)] for _ in range(S)]
    s.page_table = torch.zeros(S, n, s.max_pages, dtype=torch.int32)
    s.kv_len, s.new_len = torch.zeros(S, n, dtype=torch.int32), torch.zeros(S, n, dtype=torch.int32)
    s.x = [torch.zeros(S, n, 8), torch.zeros(S, n, 8)]
    s.use_graph, s.graph = False, None
    s.eng = SimpleNamespace(seq_len=6, n_seqs=n, x=[torch.zeros(S, n * 6, 8)], w=SimpleNamespace(n_layers=n_layers, d_model=8), forward=forward,
                            _bind=lambda l: (_ for _ in ()).throw(RuntimeError("layer %d" % l)))
    s._layers = layers
    return s


def state(s):
    return [list(r) for r in s.lens], [[list(p) for p in r] for r in s.pages], list(s.free), s.kv_len.tolist()


def fails(*a, **k):
    raise IndexError("list index out of range")


def works(*a, **k):
    return None


def test_a_prompt_that_fails_in_the_forward_pass_can_be_given_again():
    s = session(forward=fails)
    before = state(s)
    with pytest.raises(IndexError):
        s.prefill(7, [[6, 2], [0, 5]])
    assert state(s) == before
    s.eng.forward = works
    s.prefill(0, [[6, 2], [0, 5]])
    assert s.kv_len.tolist() == [[6, 2], [0, 5]] and len(s.free) == 12 - (2 + 1 + 0 + 2)
    for r, row in enumerate(s.pages):
        for b, held in enumerate(row):
            assert s.page_table[r, b, :len(held)].tolist() == held


def test_a_prompt_that_fails_at_the_append_can_be_given_again():
    s = session(forward=works, n_layers=1)
    before = state(s)
    with pytest.raises(RuntimeError):
        s.prefill(0)
    assert state(s) == before


@pytest.mark.parametrize("fresh", [False, True])
def test_a_step_that_fails_leaves_the_lengths(fresh):
    s = session(layers=fails)
    if not fresh:
        s._extend([[4, 3], [0, 1]])                    # the next token of the first sequence needs a page
    before = state(s)
    with pytest.raises(IndexError):
        s.step(torch.zeros(2, 2, 8))
    assert state(s) == before
    s._layers = lambda: s.x[0]
    s.step(torch.ones(2, 2, 8))
    assert s.kv_len.tolist() == [[v + 1 for v in r] for r in before[0]]
    held = [p for row in s.pages for q in row for p in q]
    assert len(set(held)) == len(held) and not set(held) & set(s.free) and len(held) + len(s.free) == 12
    for r, row in enumerate(s.pages):
        for b, q in enumerate(row):
            assert s.page_table[r, b, :len(q)].tolist() == q


def test_a_step_whose_input_cannot_be_copied_leaves_the_lengths():
    s = session(layers=works)
    s.x = [None, None]
    before = state(s)
    with pytest.raises(AttributeError):
        s.step(torch.zeros(2, 2, 8))
    assert state(s) == before


def test_lengths_that_cannot_be_copied_to_the_device_leave_the_session():
    s = session(layers=works)
    s.page_table = torch.zeros(1, 1, 1, dtype=torch.int32).expand(3, 3, 3)[..., :2]        # a copy that raises
    before = state(s)
    with pytest.raises(RuntimeError):
        s.step(torch.zeros(2, 2, 8))
    assert state(s) == before
