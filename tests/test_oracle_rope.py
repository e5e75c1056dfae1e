"""Pins for the oracle's rotation by position: complex multiplication, the relative-position property of the scores, the
gradient through a whole rotated stack by finite differences.  CPU only.  Also the host bookkeeping of a decode session."""
from types import SimpleNamespace

import numpy as np
import pytest

from oracle import twist_oracle as o


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dims", [8, 4])
def test_rope_is_multiplication_by_unit_complex_numbers(layout, dims):
    r = np.random.default_rng(1)
    d, H, g, n, N = 8, 3, 2, 2, 5
    kvw = g * d
    X = r.standard_normal((n * N, (H + 2 * g) * d))
    Y = o.rope(X, N, d, kvw, 100.0, dims, layout, False, first=3)
    assert np.array_equal(Y[:, (H + g) * d:], X[:, (H + g) * d:])                # V as it was
    for t in range(n * N):
        for h in range(H + g):
            x, y = X[t, h * d:(h + 1) * d], Y[t, h * d:(h + 1) * d]
            zx = x[:dims // 2] + 1j * x[dims // 2:dims] if layout == 0 else x[0:dims:2] + 1j * x[1:dims:2]
            zy = y[:dims // 2] + 1j * y[dims // 2:dims] if layout == 0 else y[0:dims:2] + 1j * y[1:dims:2]
            f = 100.0 ** (-np.arange(0, dims, 2) / dims)
            assert np.allclose(zy, zx * np.exp(1j * (3 + t % N) * f), rtol=1e-13, atol=1e-13)
            assert np.array_equal(y[dims:], x[dims:])
    back = o.rope(Y, N, d, kvw, 100.0, dims, layout, False, sign=-1.0, first=3)
    assert np.allclose(back, X, rtol=1e-13, atol=1e-13)                          # the transpose is the inverse


def test_rotated_scores_depend_on_the_distance_only():
    r = np.random.default_rng(2)
    d, N = 16, 12
    row = r.standard_normal(3 * d)
    X = np.tile(row, (N, 1))                                                     # the same token at every position
    Y = o.rope(X, N, d, d, 10000.0, d, 0, False)
    S = Y[:, :d] @ Y[:, d:2 * d].T
    for k in range(-N + 1, N):
        diag = np.diagonal(S, k)
        assert np.allclose(diag, diag[0], rtol=1e-12)


def test_gradient_through_a_rotated_stack_by_finite_differences():
    r = np.random.default_rng(3)
    d, dh, H, N, f = 6, 4, 2, 4, 5
    spec = SimpleNamespace(n_heads=H, n_kv_heads=1, d_head=dh, d_ff=f, ffn_kind=2, rope_base=50.0, rot_dims=4, rope_layout=1)
    W = {"qkv": r.standard_normal((H * dh + 2 * dh, d)), "o": r.standard_normal((H * dh, d)), "up": r.standard_normal((f, d)),
         "gate": r.standard_normal((f, d)), "down": r.standard_normal((f, d))}
    layers, head_kv = [W, {k: v * 0.7 for k, v in W.items()}], [[0, 0], [0, 0]]
    X, G = r.standard_normal((2 * N, d)), r.standard_normal((2 * N, d))
    loss = lambda ls, x: float(np.sum(o.stack_fwd(spec, ls, head_kv, x, 2, N, False)[0] * G))
    _, saved = o.stack_fwd(spec, layers, head_kv, X, 2, N, False)
    grads, dX = o.stack_bwd(spec, layers, head_kv, saved, G, 2, N, False)
    eps = 1e-6
    for l in range(2):
        for i, j in ((0, 0), (3, 2), (9, 5), (14, 1)):
            pert = []
            for sgn in (1, -1):
                ls = [{k: v.copy() for k, v in w.items()} for w in layers]
                ls[l]["qkv"][i, j] += sgn * eps
                pert.append(loss(ls, X))
            want = (pert[0] - pert[1]) / (2 * eps)
            assert abs(grads[l]["qkv"][i, j] - want) <= 1e-5 * max(1.0, abs(want))
    for i, j in ((0, 0), (5, 3)):
        pert = []
        for sgn in (1, -1):
            x = X.copy()
            x[i, j] += sgn * eps
            pert.append(loss(layers, x))
        want = (pert[0] - pert[1]) / (2 * eps)
        assert abs(dX[i, j] - want) <= 1e-5 * max(1.0, abs(want))


def _session(S=2, n=2, page_size=4, max_len=10, n_pages=7):
    """A DecodeSession's bookkeeping without buffers of a model (CPU tensors, no kernels)."""
    import torch
    from paper_2511_03983_b200.engine import DecodeSession
    s = DecodeSession.__new__(DecodeSession)
    s.S, s.n, s.page_size, s.max_len, s.n_pages = S, n, page_size, max_len, n_pages
    s.max_pages = -(-max_len // page_size)
    s.free = list(range(n_pages - 1, -1, -1))
    s.lens = [[0] * n for _ in range(S)]
    s.pages = [[[] for _ in range(n)] for _ in range(S)]
    s.page_table = torch.zeros(S, n, s.max_pages, dtype=torch.int32)
    s.kv_len = torch.zeros(S, n, dtype=torch.int32)
    return s


def test_session_hands_out_pages_once_and_takes_them_back():
    s = _session()
    s._extend([[5, 0], [1, 4]])
    assert s.kv_len.tolist() == [[5, 0], [1, 4]] and len(s.free) == 7 - (2 + 0 + 1 + 1)
    held = [p for row in s.pages for q in row for p in q]
    assert len(set(held)) == len(held) and not set(held) & set(s.free)
    assert [s.page_table[0, 0, k].item() for k in range(2)] == s.pages[0][0]
    before = ([list(r) for r in s.lens], list(s.free))
    with pytest.raises(RuntimeError):
        s._extend([[4, 4], [4, 5]])                                   # 1 + 1 + 1 + 2 pages, 3 are free
    with pytest.raises(ValueError):
        s._extend([[6, 0], [0, 0]])                                   # beyond max_len
    with pytest.raises(ValueError):
        s._extend([[-1, 0], [0, 0]])
    assert before == ([list(r) for r in s.lens], list(s.free))        # a refused request changes nothing
    s.release(0, 0)
    assert s.kv_len.tolist() == [[0, 0], [1, 4]] and len(s.free) == 5
    s._extend([[3, 3], [3, 4]])
    held = [p for row in s.pages for q in row for p in q]
    assert len(set(held)) == len(held) == 1 + 1 + 1 + 2


def test_workload_rotation_is_off_unless_asked_for():
    from dataclasses import replace
    from paper_2511_03983_b200 import inputs as I
    from paper_2511_03983_b200.engine import rope_frequencies
    for k in (2, 3, 4):
        assert I.PRESETS[k].rot_dims == 0 and rope_frequencies(I.PRESETS[k], "cpu") is None
    w = replace(I.PRESETS[3], rope_base=10000.0)
    f = rope_frequencies(w, "cpu")
    assert w.rot_dims == 64 and f.numel() == 32 and f[0] == 1.0 and abs(f[16].item() - 0.01) < 1e-15
    assert replace(w, rope_dims=16).rot_dims == 16
