"""An 8-bit session over tokens whose input is zero (padding that is part of the sequence): blocks without keys and values between large
ones.  Attention against the cache's own values in 64 bits, tolerances as in test_gpu_small_cache_session."""
import pytest
import torch

from test_gpu_small_cache_session import B, check_attention, make, rows, tokens  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("keep", [None, 1040])
def test_tokens_without_values(B, keep):  # noqa: F811
    from paper_2511_03983_b200.engine import DecodeSession
    eng = make(seq_len=1024)
    x = eng.X[0].view(eng.w.n_subnets, eng.n_seqs, 1024, -1)
    x.copy_(x.abs() * 400)                                        # one sign: large sums
    x[:, :, 512:560] = 0
    x[:, 0, 64:80] = 0
    x[:, 1, 1008:] = 0
    ses = DecodeSession(eng, max_len=1100, cache_bits=8, **({} if keep is None else dict(keep=keep)))
    ses.prefill(0)
    empty = rows(ses, 0, 0, 0, 1)[:, 512:560]
    assert (empty == 0).all() and abs(rows(ses, 0, 0, 0, 1)).max() > 100
    new = tokens(eng, 40) * 400
    new[:, 3:24] = 0
    for i in range(40):
        y = ses.step(new[:, i])
        assert torch.isfinite(y).all()
        if i in (0, 2, 10, 23, 39):
            check_attention(eng, ses)
    assert B.twist_device_status() == 0
