"""twist_attn_decode refuses an output that lies over its queries (other CTAs still read them); nothing is launched."""
import ctypes as C

import pytest

BASE = 0x100000


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


def call(B, q, out, q_stride):
    """6 rows of 256 elements (512 bytes)."""
    other = 0x10000000
    a = B.AttnDecodeArgs(dtype=B.BF16, n_subnets=2, n_seqs=3, head_keep=4, kv_max=2, d_head=64, n_heads=8, n_kv_heads=2, page_size=16,
                         n_pages=9, max_pages=2, max_len=0, page_stride=2 * 16 * 64, q_stride=q_stride, q=q, k_cache=other,
                         v_cache=other, page_table=other, kv_len=other, head_idx=other, kv_pos=other, out=out, lse=None, ws=other,
                         ws_bytes=1 << 30)
    return B.lib().twist_attn_decode(C.byref(a), None)


@pytest.mark.parametrize("q_stride", [256, 512, 2048])
@pytest.mark.parametrize("shift", [0, 16, 496, -16, -512, -3056])
def test_an_output_over_the_queries_is_refused(B, q_stride, shift):
    assert call(B, BASE, BASE + shift, q_stride) == B.ERR_SHAPE
    # over the last row alone
    assert call(B, BASE, BASE + 5 * 2 * q_stride + 496, q_stride) == B.ERR_SHAPE
