"""What the split 8-bit decode leaves behind when warps give up (a copy that did not come): the time-out is reported, the join takes nothing
from entries that were never written, and the next call is as good as ever.  The scratch holds nonsense before every call."""
import pytest
import torch

from test_gpu_small_cache import attention_case, decode_args

pytestmark = pytest.mark.gpu
EDGE = 4096                                          # elements on both sides of the results


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


def guarded(shape, dtype):
    """(whole buffer, the results' part of it)."""
    n = 1
    for v in shape:
        n *= v
    whole = torch.full((n + 2 * EDGE,), 3.0, dtype=dtype, device="cuda")
    return whole, whole[EDGE:EDGE + n].view(shape)


@pytest.mark.parametrize("fill", [0xFF, 0x7F, 0x00, 0x11])
@pytest.mark.parametrize("lens,H,NH,NKV", [([3000, 0, 17, 1200], 4, 8, 2),                 # an entry for every item
                                           ([900, 64, 2001], 12, 16, 1),                   # two passes over a position's keys
                                           ([40 + 7 * i % 90 for i in range(1300)], 4, 8, 2)])       # one for every warp
def test_warps_that_give_up(B, lens, H, NH, NKV, fill):
    gen = torch.Generator().manual_seed(len(lens))
    c = attention_case(gen, 64, 16, 1, lens, H, NH, NKV)
    ws = torch.empty(B.twist_attn_decode_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    n = len(lens)

    def call(every, tile):
        ws.fill_(fill)
        (out_all, out), (lse_all, lse) = guarded((1, n, H * 64), torch.bfloat16), guarded((1, H, n), torch.float32)
        args = decode_args(B, c, out, lse, ws)
        B.twist_selftest_decode_quit(args, every, tile)
        status = B.twist_device_status()
        for t in (out_all, lse_all):
            assert torch.all(t[:EDGE] == 3.0) and torch.all(t[-EDGE:] == 3.0)
        return out, lse, status

    want, want_lse, status = call(1, 1 << 20)        # nobody gives up
    assert status == 0
    empty = torch.tensor([v == 0 for v in lens], device="cuda")
    out, lse, status = call(1, 0)                    # everybody, at once: nothing is written (but for warps that only had empty sequences)
    assert status == B.ERR_DEVICE_TIMEOUT
    assert torch.all(out[0, ~empty] == 3.0) and torch.all(lse[0][:, ~empty] == 3.0)
    for every, tile in ((1, 1), (2, 0), (3, 0), (2, 1), (7, 1)):
        assert call(every, tile)[2] == B.ERR_DEVICE_TIMEOUT
        assert B.twist_device_status() == 0
    out, lse, status = call(1, 1 << 20)
    assert status == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)
