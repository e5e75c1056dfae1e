"""Refusals of the 8-bit cache, weight and eviction entry points: every bad argument comes back as its documented status before
anything is launched (no GPU is touched), and the Python side refuses tensors that do not describe the layout."""
import ctypes as C

import pytest
import torch

P = 0x100000                       # an aligned address that nothing dereferences


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


def append(B, **kw):
    f = dict(dtype=B.BF16, n_subnets=2, n_seqs=3, tokens=6, head_keep=4, kv_max=2, d_head=64, page_size=16, n_pages=9,
             max_pages=2, rot_dims=64, layout=B.ROPE_HALF, page_stride=2 * 16 * 64, q_stride=256, qkv=P, q_out=2 * P, k_cache=P,
             v_cache=P, scales=P, page_table=P, kv_len=P, seen=None, new_begin=None, new_len=None, kv_count=None, inv_freq=P)
    f.update(kw)
    return B.KvAppendQ8Args(**f)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), "ERR_UNSUPPORTED"), (dict(d_head=8, rot_dims=8), "ERR_UNSUPPORTED"), (dict(d_head=48), "ERR_UNSUPPORTED"),
    (dict(d_head=256), "ERR_UNSUPPORTED"), (dict(n_seqs=0), "ERR_SHAPE"), (dict(tokens=0), "ERR_SHAPE"), (dict(tokens=7), "ERR_SHAPE"),
    (dict(kv_max=0), "ERR_SHAPE"), (dict(rot_dims=65), "ERR_SHAPE"), (dict(rot_dims=66), "ERR_SHAPE"), (dict(rot_dims=-2), "ERR_SHAPE"),
    (dict(layout=3), "ERR_SHAPE"), (dict(page_size=8), "ERR_UNSUPPORTED"), (dict(page_size=48), "ERR_UNSUPPORTED"),
    (dict(page_stride=2 * 16 * 64 - 16), "ERR_SHAPE"), (dict(page_stride=2 * 16 * 64 + 8), "ERR_SHAPE"), (dict(q_stride=252), "ERR_SHAPE"),
    (dict(qkv=None), "ERR_NULL"), (dict(k_cache=None), "ERR_NULL"), (dict(v_cache=None), "ERR_NULL"), (dict(scales=None), "ERR_NULL"),
    (dict(page_table=None), "ERR_NULL"), (dict(kv_len=None), "ERR_NULL"), (dict(inv_freq=None), "ERR_NULL"),
    (dict(k_cache=P + 8), "ERR_SHAPE"), (dict(scales=P + 4), "ERR_SHAPE"), (dict(inv_freq=P + 4), "ERR_SHAPE"),
    (dict(new_begin=P, new_len=P), "ERR_SHAPE"), (dict(q_out=P + 16), "ERR_SHAPE"), (dict(max_pages=1 << 27), "ERR_UNSUPPORTED"),
])
def test_append_refusals(B, kw, status):
    h = B.lib()
    assert h.twist_kv_append_q8(C.byref(append(B, **kw)), None) == getattr(B, status)
    assert h.twist_kv_append_q8(None, None) == B.ERR_NULL


def decode(B, **kw):
    f = dict(dtype=B.BF16, n_subnets=2, n_seqs=3, head_keep=4, kv_max=2, d_head=64, n_heads=8, n_kv_heads=2, page_size=16,
             n_pages=9, max_pages=2, max_len=0, page_stride=2 * 16 * 64, q_stride=256, q=P, k_cache=P, v_cache=P, scales=P,
             page_table=P, kv_len=P, head_idx=P, kv_pos=P, out=2 * P, lse=None, ws=P, ws_bytes=1 << 30)
    f.update(kw)
    return B.AttnDecodeQ8Args(**f)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), "ERR_UNSUPPORTED"), (dict(d_head=8), "ERR_UNSUPPORTED"), (dict(d_head=256), "ERR_UNSUPPORTED"),
    (dict(d_head=0), "ERR_SHAPE"), (dict(n_seqs=0), "ERR_SHAPE"), (dict(n_subnets=33), "ERR_UNSUPPORTED"), (dict(max_len=-1), "ERR_SHAPE"),
    (dict(page_size=17), "ERR_UNSUPPORTED"), (dict(page_stride=64), "ERR_SHAPE"), (dict(page_stride=2 * 16 * 64 + 8), "ERR_SHAPE"),
    (dict(q_stride=128), "ERR_SHAPE"), (dict(n_heads=7), "ERR_SHAPE"), (dict(kv_pos=None), "ERR_SHAPE"), (dict(head_idx=None), "ERR_SHAPE"),
    (dict(q=None), "ERR_NULL"), (dict(scales=None), "ERR_NULL"), (dict(k_cache=None), "ERR_NULL"), (dict(out=None), "ERR_NULL"),
    (dict(scales=P + 8), "ERR_SHAPE"), (dict(v_cache=P + 8), "ERR_SHAPE"), (dict(ws=None), "ERR_WORKSPACE"), (dict(ws_bytes=64), "ERR_WORKSPACE"),
    (dict(out=P), "ERR_SHAPE"),                                # over the queries
    (dict(n_seqs=4096, max_pages=1 << 22), "ERR_UNSUPPORTED"),
])
def test_decode_refusals(B, kw, status):
    h = B.lib()
    assert h.twist_attn_decode_q8(C.byref(decode(B, **kw)), None) == getattr(B, status)
    assert h.twist_attn_decode_q8(None, None) == B.ERR_NULL


def weights(B, **kw):
    f = dict(dtype=B.BF16, n_subnets=2, n_seqs=3, head_keep=4, kv_max=2, d_head=64, n_heads=8, n_kv_heads=2, page_size=16,
             n_pages=9, max_pages=2, max_len=0, cache=B.CACHE_BF16, page_stride=2 * 16 * 64, q_stride=256, q=P, lse=P, k_cache=P,
             scales=None, page_table=P, kv_len=P, new_len=None, seen=None, head_idx=P, kv_pos=P, prior=2 * P, weights=3 * P,
             slot_pos=4 * P)
    f.update(kw)
    return B.AttnWeightsArgs(**f)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), "ERR_UNSUPPORTED"), (dict(cache=2), "ERR_SHAPE"), (dict(cache=1), "ERR_SHAPE"), (dict(scales=P), "ERR_SHAPE"),
    (dict(cache=1, scales=P, d_head=8), "ERR_UNSUPPORTED"), (dict(d_head=24), "ERR_UNSUPPORTED"), (dict(n_seqs=-1), "ERR_SHAPE"),
    (dict(cache=1, scales=P, page_stride=2 * 16 * 64 + 8), "ERR_SHAPE"), (dict(page_stride=2 * 16 * 64 - 8), "ERR_SHAPE"),
    (dict(max_len=-1), "ERR_SHAPE"), (dict(page_size=2048), "ERR_UNSUPPORTED"), (dict(head_idx=None), "ERR_SHAPE"),
    (dict(n_subnets=33), "ERR_UNSUPPORTED"), (dict(n_heads=2048), "ERR_UNSUPPORTED"), (dict(n_seqs=40000), "ERR_UNSUPPORTED"),
    (dict(q=None), "ERR_NULL"), (dict(lse=None), "ERR_NULL"), (dict(k_cache=None), "ERR_NULL"), (dict(weights=None), "ERR_NULL"),
    (dict(lse=P + 4), "ERR_SHAPE"), (dict(weights=P + 4), "ERR_SHAPE"), (dict(prior=P + 8), "ERR_SHAPE"),
    (dict(prior=3 * P + 16), "ERR_SHAPE"), (dict(slot_pos=3 * P), "ERR_SHAPE"), (dict(slot_pos=2 * P + 32), "ERR_SHAPE"),
    (dict(n_seqs=4096, max_pages=1 << 22), "ERR_UNSUPPORTED"),
])
def test_weights_refusals(B, kw, status):
    h = B.lib()
    assert h.twist_attn_weights(C.byref(weights(B, **kw)), None) == getattr(B, status)
    assert h.twist_attn_weights(None, None) == B.ERR_NULL


def core(B, **kw):
    f = dict(dtype=B.BF16, n_subnets=2, n_seqs=3, seq_len=20, head_keep=4, kv_max=2, d_head=64, n_heads=8, n_kv_heads=2,
             page_size=16, n_pages=12, max_pages=2, last_queries=0, qkv=P, lse=P, page_table=P, new_len=None, head_idx=P, kv_pos=P,
             weights=2 * P, slot_pos=3 * P, plan=None)
    f.update(kw)
    return B.AttnCoreWeightsArgs(**f)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), "ERR_UNSUPPORTED"), (dict(d_head=24), "ERR_UNSUPPORTED"), (dict(seq_len=0), "ERR_SHAPE"),
    (dict(last_queries=-1), "ERR_SHAPE"), (dict(page_size=5), "ERR_UNSUPPORTED"), (dict(n_heads=9), "ERR_SHAPE"),
    (dict(head_idx=None), "ERR_SHAPE"), (dict(n_subnets=33), "ERR_UNSUPPORTED"), (dict(qkv=None), "ERR_NULL"), (dict(lse=None), "ERR_NULL"),
    (dict(page_table=None), "ERR_NULL"), (dict(weights=None), "ERR_NULL"), (dict(qkv=P + 8), "ERR_SHAPE"), (dict(slot_pos=P + 4), "ERR_SHAPE"),
    (dict(slot_pos=2 * P), "ERR_SHAPE"),
])
def test_core_weights_refusals(B, kw, status):
    h = B.lib()
    assert h.twist_attn_core_weights(C.byref(core(B, **kw)), None) == getattr(B, status)
    assert h.twist_attn_core_weights(None, None) == B.ERR_NULL


def evict(B, **kw):
    f = dict(dtype=B.BF16, n_subnets=2, n_seqs=3, kv_max=2, d_head=64, page_size=16, n_pages=9, max_pages=2, max_len=0, recent=4,
             cache=B.CACHE_BF16, page_stride=2 * 16 * 64, k_cache=P, v_cache=P, scales=None, page_table=P, kv_len=P, keep=P, seen=None,
             kv_count=None, weights=2 * P, slot_pos=3 * P, weights_out=2 * P, slot_pos_out=3 * P, ws=P, ws_bytes=1 << 30)
    f.update(kw)
    return B.KvEvictArgs(**f)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), "ERR_UNSUPPORTED"), (dict(cache=-1), "ERR_SHAPE"), (dict(cache=1), "ERR_SHAPE"), (dict(scales=P), "ERR_SHAPE"),
    (dict(d_head=12), "ERR_UNSUPPORTED"), (dict(d_head=264, page_stride=1 << 20), "ERR_UNSUPPORTED"),
    (dict(cache=1, scales=P, d_head=24), "ERR_UNSUPPORTED"), (dict(recent=-1), "ERR_SHAPE"), (dict(max_len=-1), "ERR_SHAPE"),
    (dict(page_stride=2 * 16 * 64 - 8), "ERR_SHAPE"), (dict(page_size=30), "ERR_UNSUPPORTED"), (dict(max_pages=1 << 23), "ERR_UNSUPPORTED"),
    (dict(n_seqs=1 << 20), "ERR_UNSUPPORTED"), (dict(k_cache=None), "ERR_NULL"), (dict(keep=None), "ERR_NULL"),
    (dict(weights=None), "ERR_NULL"), (dict(slot_pos_out=None), "ERR_NULL"), (dict(weights=P + 4), "ERR_SHAPE"),
    (dict(weights_out=4 * P), "ERR_SHAPE"),                    # one in place, the other not
    (dict(weights_out=2 * P + 64, slot_pos_out=4 * P), "ERR_SHAPE"), (dict(slot_pos=2 * P, slot_pos_out=2 * P), "ERR_SHAPE"),
    (dict(weights_out=3 * P, slot_pos_out=4 * P), "ERR_SHAPE"), (dict(ws=None), "ERR_WORKSPACE"), (dict(ws_bytes=100), "ERR_WORKSPACE"),
])
def test_evict_refusals(B, kw, status):
    h = B.lib()
    assert h.twist_kv_evict(C.byref(evict(B, **kw)), None) == getattr(B, status)
    assert h.twist_kv_evict(None, None) == B.ERR_NULL


def test_evict_workspace_grows_with_its_arguments_and_refuses_nonsense(B):
    f = B.twist_kv_evict_workspace_bytes
    assert 0 < f(1, 1, 1, 1) <= f(1, 1, 1, 1000) < f(1, 2, 1, 1000) < f(3, 2, 4, 1000)
    assert f(4, 16, 4, 16384) == 4 * 16 * 4 * f(1, 1, 1, 16384)
    for bad in ((0, 1, 1, 1), (1, -1, 1, 1), (1, 1, 1, 0), (1, 1, 1, 1 << 40), (1 << 16, 1 << 16, 1, 1)):
        assert f(*bad) == 0


def test_layout_checks_of_the_python_side(B):
    f8 = torch.float8_e4m3fn
    pool = torch.zeros(5, 2, 3, 16, 32).to(f8)
    assert B._cache(pool[:, 0], pool[:, 1], 3, 32, f8) == (16, 5, 2 * 3 * 16 * 32)
    with pytest.raises(ValueError):
        B._cache(pool[:, 0], pool[:, 1], 3, 32)                       # an 8-bit cache is no bf16 cache
    with pytest.raises(ValueError):
        B._cache(pool[:, 0].float(), pool[:, 1].float(), 3, 32, f8)
    f32 = torch.float32
    assert B._addresses(-1, ("seen", None, f32, 30), ("scales", pool.float(), f32, pool.numel()))[0] == 0
    with pytest.raises(ValueError, match="scales"):
        B._addresses(-1, ("seen", None, f32, 30), ("scales", torch.zeros(5, 3, 1), f32, 30))    # K's and V's side by side are expected
    with pytest.raises(ValueError, match="scales"):
        B._addresses(-1, ("scales", torch.zeros(5, 3, 1, 2, dtype=torch.float64), f32, 30))
    assert B._cache_kind(pool, torch.zeros(1)) == B.CACHE_E4M3 and B._cache_kind(pool.float().bfloat16(), None) == B.CACHE_BF16
    with pytest.raises(ValueError):
        B._cache_kind(pool, None)
    with pytest.raises(ValueError):
        B._cache_kind(pool.float().bfloat16(), torch.zeros(1))
