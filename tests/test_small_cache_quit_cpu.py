"""Refusals of the decode's self-test and of head sizes that an 8-bit cache does not have; no GPU is touched."""
import ctypes as C

from test_small_cache_cpu import P, decode


def test_refusals():
    from paper_2511_03983_b200 import binding as B
    f = lambda every=1, tile=0, **kw: B.lib().twist_selftest_decode_quit(C.byref(decode(B, **kw)), every, tile, None)
    assert B.lib().twist_selftest_decode_quit(None, 1, 0, None) == B.ERR_NULL
    assert f(every=0) == B.ERR_SHAPE and f(tile=-1) == B.ERR_SHAPE
    assert f(d_head=128, page_stride=2 * 16 * 128, q_stride=512) == B.ERR_UNSUPPORTED
    assert f(scales=None) == B.ERR_NULL and f(scales=P + 8) == B.ERR_SHAPE and f(ws=None) == B.ERR_WORKSPACE


def test_an_8_bit_cache_has_heads_of_16_to_128_everywhere():
    from paper_2511_03983_b200 import binding as B
    from test_small_cache_cpu import append, evict, weights
    h = B.lib()
    for d in (8, 48, 96, 112, 256):
        big = dict(d_head=d, page_stride=2 * 16 * d)
        assert h.twist_kv_evict(C.byref(evict(B, cache=B.CACHE_E4M3, scales=P, **big)), None) == B.ERR_UNSUPPORTED
        assert h.twist_kv_append_q8(C.byref(append(B, rot_dims=0, q_stride=4 * d, **big)), None) == B.ERR_UNSUPPORTED
        assert h.twist_attn_decode_q8(C.byref(decode(B, q_stride=4 * d, **big)), None) == B.ERR_UNSUPPORTED
        assert h.twist_attn_weights(C.byref(weights(B, cache=B.CACHE_E4M3, scales=P, q_stride=4 * d, **big)), None) == B.ERR_UNSUPPORTED
