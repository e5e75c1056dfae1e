"""Padded prompts of a decoding session: what the rows behind a sequence's length hold must not reach its tokens."""
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
