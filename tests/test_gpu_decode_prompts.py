"""Decoding sessions: what the padding rows of a prompt, and the pages of sequences that ended, hold must not reach other tokens."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from paper_2511_03983_b200 import inputs as I
from test_gpu_decode_session import dev, fill_model

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("d_head,ln", [(64, False), (64, True), (16, True)])
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), torch.finfo(torch.bfloat16).min])
def test_rows_behind_a_prompt_may_hold_anything(B, d_head, ln, fill):
    """The same bits for the prompt's tokens, and for tokens decoded after it, whatever the padding rows hold; the batch
    itself is not written."""
    from paper_2511_03983_b200.engine import DecodeSession, StackEngine
    N, n = 140, 3
    w = replace(I.scaled_twin(I.PRESETS[3], d_model=256, d_ff=688, d_head=d_head, tokens=n * N, n_layers=2, local_steps=1), rope_base=10000.0,
                layer_norm=ln)
    S = w.n_subnets
    eng = StackEngine(w, n, N)
    fill_model(eng, w)
    eng.extract(0)
    lengths = [[[N, 1, 70], [0, 64, 139], [128, 65, 3], [20, 0, 137]][s % 4] for s in range(S)]
    live = torch.zeros(S, n, N, dtype=torch.bool)
    for s in range(S):
        for b in range(n):
            live[s, b, :lengths[s][b]] = True
    live = live.view(S, n * N, 1).cuda()
    tok = dev(np.stack([I.normal(7, s, (n * N, w.d_model), 1.0, I.DTYPE_BF16) for s in range(S)]))
    new = dev(I.normal(78, 0, (3, S, n, w.d_model), 1.0, I.DTYPE_BF16))
    outs = []
    for k, pad in enumerate((0.0, fill)):
        given = torch.where(live, tok, torch.tensor(pad, dtype=tok.dtype, device="cuda"))
        eng.X.append(given.clone())
        ses = DecodeSession(eng, max_len=N + 3)
        y = ses.prefill(k, lengths)
        outs.append([torch.where(live, y, torch.zeros_like(y))] + [ses.step(t).clone() for t in new])
        torch.cuda.synchronize()
        assert B.twist_device_status() == 0
        assert torch.equal(eng.X[k].view(torch.int16), given.view(torch.int16))
    for i, (want, got) in enumerate(zip(*outs)):
        assert bool(torch.isfinite(want).all())
        assert torch.equal(want, got), i


@pytest.mark.parametrize("graph", [False, True])
def test_pages_that_change_hands_on_a_side_stream(B, graph):
    """Sequences that end and start again in a pool with few spare pages, on a stream of the caller: every output has the bits
    that a fresh session gives for the same tokens alone."""
    from paper_2511_03983_b200.engine import DecodeSession, StackEngine
    n, most, steps = 3, 40, 70
    w = replace(I.scaled_twin(I.PRESETS[3], d_model=256, d_ff=688, d_head=64, tokens=n * 8, n_layers=2, local_steps=1), rope_base=10000.0)
    S = w.n_subnets
    eng = StackEngine(w, n, 8)
    fill_model(eng, w)
    eng.extract(0)
    gen = torch.Generator().manual_seed(5)
    new = dev(I.normal(79, 0, (steps, S, n, w.d_model), 1.0, I.DTYPE_BF16))
    ends = torch.randint(1, most, (steps, S, n), generator=gen)          # a sequence that is this long ends before the step
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    runs, got, started = {}, [], [[0] * n for _ in range(S)]
    with torch.cuda.stream(side):
        ses = DecodeSession(eng, max_len=most, n_pages=S * n * 3 - 2, graph=graph)
        for i in range(steps):
            for s in range(S):
                for b in range(n):
                    if ses.lens[s][b] >= int(ends[i, s, b]) or ses.lens[s][b] == 32:
                        ses.release(s, b)
                        started[s][b] = i
                    runs[(i, s, b)] = started[s][b]
            got.append(ses.step(new[i]).clone())
    side.synchronize()
    assert B.twist_device_status() == 0
    assert len({v for v in runs.values()}) > 20                          # many sequences began in pages that others had held
    for s, b, last in ((0, 0, steps - 1), (1, 2, 50), (S - 1, 1, 33), (2, 0, 12)):
        first = runs[(last, s, b)]
        fresh = DecodeSession(eng, max_len=most)
        for i in range(first, last + 1):
            y = fresh.step(new[i])
            assert torch.equal(y[s, b], got[i][s, b]), (s, b, i)
