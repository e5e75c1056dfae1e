"""Refusals of the position, cache and decode entry points: every bad argument comes back as its documented status before
anything is launched (no GPU is touched), and the Python side refuses tensors that do not describe the layout."""
import ctypes as C

import pytest
import torch

OK_PTR = 0x10000


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


def rope(B, **kw):
    f = dict(dtype=B.BF16, n_subnets=2, tokens=6, head_keep=4, kv_max=2, d_head=64, rot_dims=64, layout=B.ROPE_HALF, seq_len=3,
             in_=OK_PTR, out=OK_PTR, inv_freq=OK_PTR, pos=None)
    f.update(kw)
    return B.RopeArgs(**f)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), "ERR_UNSUPPORTED"), (dict(n_subnets=0), "ERR_SHAPE"), (dict(tokens=0), "ERR_SHAPE"),
    (dict(head_keep=0), "ERR_SHAPE"), (dict(kv_max=0), "ERR_SHAPE"), (dict(d_head=60), "ERR_SHAPE"),
    (dict(d_head=264), "ERR_UNSUPPORTED"), (dict(rot_dims=0), "ERR_SHAPE"), (dict(rot_dims=63), "ERR_SHAPE"),
    (dict(rot_dims=66), "ERR_SHAPE"), (dict(layout=2), "ERR_SHAPE"), (dict(seq_len=0), "ERR_SHAPE"),
    (dict(in_=None), "ERR_NULL"), (dict(out=None), "ERR_NULL"), (dict(inv_freq=None), "ERR_NULL"),
    (dict(in_=OK_PTR + 8), "ERR_SHAPE"), (dict(out=OK_PTR + 4), "ERR_SHAPE"), (dict(inv_freq=OK_PTR + 4), "ERR_SHAPE"),
    (dict(out=OK_PTR + 32), "ERR_SHAPE"),                      # overlaps the input without being it
])
def test_rope_refusals(B, kw, status):
    h = B.lib()
    for f in (h.twist_rope_fwd, h.twist_rope_bwd):
        assert f(C.byref(rope(B, **kw)), None) == getattr(B, status)
        assert f(None, None) == B.ERR_NULL


def append(B, **kw):
    f = dict(dtype=B.BF16, n_subnets=2, n_seqs=3, tokens=6, head_keep=4, kv_max=2, d_head=64, page_size=16, n_pages=9,
             max_pages=2, rot_dims=64, layout=B.ROPE_HALF, page_stride=2 * 16 * 64, q_stride=256, qkv=OK_PTR,
             q_out=0x40000, k_cache=OK_PTR, v_cache=OK_PTR, page_table=OK_PTR, kv_len=OK_PTR, new_begin=None, new_len=None,
             kv_count=None, inv_freq=OK_PTR)
    f.update(kw)
    return B.KvAppendArgs(**f)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), "ERR_UNSUPPORTED"), (dict(n_seqs=0), "ERR_SHAPE"), (dict(n_pages=0), "ERR_SHAPE"),
    (dict(max_pages=0), "ERR_SHAPE"), (dict(page_size=24), "ERR_UNSUPPORTED"), (dict(page_size=8), "ERR_UNSUPPORTED"),
    (dict(page_size=2048), "ERR_UNSUPPORTED"), (dict(page_stride=2 * 16 * 64 - 8), "ERR_SHAPE"),
    (dict(page_stride=2 * 16 * 64 + 4), "ERR_SHAPE"), (dict(tokens=7), "ERR_SHAPE"),   # neither one per sequence nor a padded batch
    (dict(q_stride=248), "ERR_SHAPE"), (dict(q_stride=260), "ERR_SHAPE"), (dict(qkv=None), "ERR_NULL"),
    (dict(k_cache=None), "ERR_NULL"), (dict(v_cache=None), "ERR_NULL"), (dict(page_table=None), "ERR_NULL"),
    (dict(kv_len=None), "ERR_NULL"), (dict(inv_freq=None), "ERR_NULL"), (dict(k_cache=OK_PTR + 8), "ERR_SHAPE"),
    (dict(v_cache=OK_PTR + 2), "ERR_SHAPE"), (dict(qkv=OK_PTR + 8), "ERR_SHAPE"), (dict(q_out=OK_PTR + 64), "ERR_SHAPE"),
    (dict(new_begin=OK_PTR, new_len=OK_PTR), "ERR_SHAPE"), (dict(max_pages=1 << 27), "ERR_UNSUPPORTED"),
    (dict(rot_dims=65), "ERR_SHAPE"),
])
def test_append_refusals(B, kw, status):
    h = B.lib()
    assert h.twist_kv_append(C.byref(append(B, **kw)), None) == getattr(B, status)
    assert h.twist_kv_append(None, None) == B.ERR_NULL


def decode(B, **kw):
    f = dict(dtype=B.BF16, n_subnets=2, n_seqs=3, head_keep=4, kv_max=2, d_head=64, n_heads=8, n_kv_heads=2, page_size=16,
             n_pages=9, max_pages=2, max_len=0, page_stride=2 * 16 * 64, q_stride=256, q=OK_PTR, k_cache=OK_PTR,
             v_cache=OK_PTR, page_table=OK_PTR, kv_len=OK_PTR, head_idx=OK_PTR, kv_pos=OK_PTR, out=OK_PTR, lse=None,
             ws=OK_PTR, ws_bytes=1 << 30)
    f.update(kw)
    return B.AttnDecodeArgs(**f)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), "ERR_UNSUPPORTED"), (dict(d_head=48), "ERR_UNSUPPORTED"), (dict(d_head=256), "ERR_UNSUPPORTED"),
    (dict(d_head=0), "ERR_SHAPE"), (dict(n_seqs=0), "ERR_SHAPE"), (dict(n_subnets=33), "ERR_UNSUPPORTED"),
    (dict(max_len=-1), "ERR_SHAPE"), (dict(page_size=17), "ERR_UNSUPPORTED"), (dict(page_stride=64), "ERR_SHAPE"),
    (dict(q_stride=128), "ERR_SHAPE"), (dict(n_heads=7), "ERR_SHAPE"), (dict(kv_pos=None), "ERR_SHAPE"),
    (dict(head_idx=None), "ERR_SHAPE"),                        # without sharing every head has a KV position of its own
    (dict(q=None), "ERR_NULL"), (dict(k_cache=None), "ERR_NULL"), (dict(v_cache=None), "ERR_NULL"),
    (dict(page_table=None), "ERR_NULL"), (dict(kv_len=None), "ERR_NULL"), (dict(out=None), "ERR_NULL"),
    (dict(q=OK_PTR + 2), "ERR_SHAPE"), (dict(out=OK_PTR + 8), "ERR_SHAPE"), (dict(ws=OK_PTR + 8), "ERR_SHAPE"),
    (dict(ws=None), "ERR_WORKSPACE"), (dict(ws_bytes=64), "ERR_WORKSPACE"),
    (dict(max_pages=1 << 27), "ERR_UNSUPPORTED"), (dict(n_heads=2048), "ERR_UNSUPPORTED"),
    (dict(n_seqs=32768), "ERR_UNSUPPORTED"), (dict(n_seqs=4096, max_pages=1 << 22), "ERR_UNSUPPORTED"),          # more work than the kernel's counters hold
])
def test_decode_refusals(B, kw, status):
    h = B.lib()
    assert h.twist_attn_decode(C.byref(decode(B, **kw)), None) == getattr(B, status)
    assert h.twist_attn_decode(None, None) == B.ERR_NULL


def test_decode_workspace_grows_with_the_head_and_refuses_nonsense(B):
    sizes = [B.twist_attn_decode_workspace_bytes(d) for d in (8, 16, 32, 64, 128)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and sizes[-1] < 64 << 20
    assert B.twist_attn_decode_workspace_bytes(0) == 0 and B.twist_attn_decode_workspace_bytes(256) == 0


def test_layout_checks_of_the_python_side(B):
    bf = torch.bfloat16
    pool = torch.zeros(5, 2, 3, 16, 32, dtype=bf)                     # K and V of a page side by side
    assert B._cache(pool[:, 0], pool[:, 1], 3, 32) == (16, 5, 2 * 3 * 16 * 32)
    assert B._cache(pool[:1, 0], pool[:1, 1], 3, 32)[1] == 1
    with pytest.raises(ValueError):
        B._cache(pool[:, 0], pool[:, 1].contiguous(), 3, 32)          # spaced differently
    with pytest.raises(ValueError):
        B._cache(pool[:, 0].transpose(1, 2), pool[:, 1].transpose(1, 2), 3, 32)
    with pytest.raises(ValueError):
        B._cache(pool[:, 0].float(), pool[:, 1].float(), 3, 32)
    qkv = torch.zeros(2, 5, 96, dtype=bf)
    assert B._rows("q", qkv[..., :32], 2, 5, 32) == 96
    assert B._rows("q", qkv[:, :1, :32].contiguous(), 2, 1, 32) == 32
    assert B._rows("q", qkv[:1, :1, :32], 1, 1, 32) == 32             # a single row has no spacing
    with pytest.raises(ValueError):
        B._rows("q", qkv[:, :4, :32], 2, 4, 32)                       # a gap between the subnets
    with pytest.raises(ValueError):
        B._rows("q", qkv[..., :32].float(), 2, 5, 32)
    with pytest.raises(ValueError):
        B._tensor("kv_len", torch.zeros(3, dtype=torch.int64), torch.int32, 3, -1)
    with pytest.raises(ValueError):
        B._tensor("kv_len", torch.zeros(6, dtype=torch.int32)[::2], torch.int32, 3, -1)
    with pytest.raises(ValueError):
        B._tensor("kv_len", torch.zeros(3, dtype=torch.int32), torch.int32, 3, 0)      # not on the current device
