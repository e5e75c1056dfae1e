"""Refusals of the decode's self-test; no GPU is touched."""
import ctypes as C

from test_small_cache_cpu import P, decode


def test_refusals():
    from paper_2511_03983_b200 import binding as B
    f = lambda every=1, tile=0, **kw: B.lib().twist_selftest_decode_quit(C.byref(decode(B, **kw)), every, tile, None)
    assert B.lib().twist_selftest_decode_quit(None, 1, 0, None) == B.ERR_NULL
    assert f(every=0) == B.ERR_SHAPE and f(tile=-1) == B.ERR_SHAPE
    assert f(d_head=128, page_stride=2 * 16 * 128, q_stride=512) == B.ERR_UNSUPPORTED
    assert f(scales=None) == B.ERR_NULL and f(scales=P + 8) == B.ERR_SHAPE and f(ws=None) == B.ERR_WORKSPACE
