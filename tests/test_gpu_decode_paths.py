"""Attention of one new token on both ways its work can go: one cluster of CTAs per item, and the line of tiles that is cut
over all warps and joined.  Which way a call goes follows from the bound on the lengths, so every test here chooses it by
the bound (a table far wider than the sequences, and the bound that the caller gives) and asserts from the scratch buffer
that it was taken: the short way does not touch it, the line leaves a descriptor of every item that was cut.

Values and tolerances as in test_gpu_decode: the definition in 64 bits."""
import numpy as np
import pytest
import torch

from test_gpu_decode import BF, Case, host

pytestmark = pytest.mark.gpu

WIDE = 20480         # keys that the widened table has room for: beyond what the short way takes, whatever the head size
SHORT, LINE = 16, 0  # max_len that makes a call go the short way / through the line (0: the table's room)


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


def widened(table, page):
    """The page table with room for WIDE keys; the entries that no key needs lie outside the pool."""
    S, n, m = table.shape
    out = torch.full((S, n, max(m, WIDE // page)), 1 << 24, dtype=torch.int32)
    out[..., :m] = table
    return out.cuda()


def cut_items(ws):
    """None: the call did not use its scratch (the short way); else how many items were cut between warps."""
    if bool((ws == 0xFF).all()):
        return None
    n = torch.cuda.get_device_properties(0).multi_processor_count * 16
    desc = ws[:16 * n].view(torch.int32).view(n, 4)
    return int(((desc[:, 2] > 0) & (desc[:, 0] >= 0)).sum())


def call(B, c, bound, **kw):
    """One call from freshly filled outputs and scratch; returns (out, lse, items that were cut)."""
    c.out.fill_(9.0)
    c.lse.fill_(9.0)
    c.ws.fill_(0xFF)
    B.twist_attn_decode(c.args(B, **dict(dict(max_len=bound, page_table=widened(c.table, c.page)), **kw)))
    torch.cuda.synchronize()
    return c.out.clone(), c.lse.clone(), cut_items(c.ws)


# heads of a group, heads of the call, the list of heads, kv_pos, how many heads the one position takes
CROWDED = [
    (1, 2, [3, 3], [0, 0, 0, 0], 1),
    (2, 5, [0, 1, 0, 1, 1], [0, 1, 2], 2),
    (4, 5, [0, 1, 2, 3, 3], [0, 1], 4),
    (4, 6, [4, 4, 4, 5, 6, 7], [1, 0], 4),
    (4, 8, [0, 1, 2, 3, 4, 5, 6, 7], [0, 0], 4),                     # two groups sent to one position
    (8, 11, [0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10], [0, 0], 8),
    (12, 14, list(range(12)) + [0, 1], [0, 1], 12),                  # two row tiles, the second with room for four more
]


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("bound", [SHORT, LINE])
@pytest.mark.parametrize("group,H,heads,kv_pos,fit", CROWDED)
def test_heads_beyond_a_group_are_reported_and_left_on_both_ways(B, group, H, heads, kv_pos, fit, bound, d):
    """A position takes as many heads as a group has, in the order of the list; the rest keep their output whichever way the
    call goes, and the call is reported."""
    nkv = len(kv_pos)
    c = Case(B, 1, [700, 3, 40], H, (group * nkv, nkv), d, 16, seed=group)
    c.kv_max = min(nkv, H)
    idx = lambda v: torch.tensor([v], dtype=torch.int32, device="cuda")
    fine, pos = idx(heads[:fit]), idx(kv_pos)
    # the heads that fit, alone: a proper call over the same cache
    q = c.q.view(1, 3, H, d)[:, :, :fit].reshape(1, 3, fit * d).contiguous().cuda()
    want = torch.full((1, 3, fit * d), 7.0, dtype=BF, device="cuda")
    want_lse = torch.full((1, fit, 3), 7.0, dtype=torch.float32, device="cuda")
    if len(set(heads[:fit])) < fit:                                   # (repeats read the position of the head they repeat)
        fine = idx([heads[0] // group * group + i for i in range(fit)])
    B.twist_attn_decode(B.attn_decode_args(
        B.BF16, 1, 3, fit, c.kv_max, d, c.nh, c.nkv, bound, q=q, k_cache=c.k, v_cache=c.v, page_table=widened(c.table, 16),
        kv_len=c.dlens, head_idx=fine, kv_pos=pos, out=want, lse=want_lse, ws=c.ws))
    torch.cuda.synchronize()
    assert B.twist_device_status() == 0
    out, lse, cut = call(B, c, bound, head_idx=idx(heads), kv_pos=pos)
    assert B.twist_device_status() == B.ERR_BAD_INDEX
    assert cut is None if bound == SHORT else cut > 0
    out = out.view(1, 3, H, d)
    assert torch.equal(out[:, :, :fit], want.view(1, 3, fit, d)) and torch.equal(lse[:, :fit], want_lse)
    assert bool((out[:, :, fit:] == 9.0).all()) and bool((lse[:, fit:] == 9.0).all())


@pytest.mark.parametrize("bound", [SHORT, LINE])
@pytest.mark.parametrize("q_stride,shift", [
    (4 * 64, -6 * 256), (4 * 64, 6 * 256),           # right before the queries, right behind them
    (12 * 256, 256), (12 * 256, 4 * 12 * 256 + 6 * 256 - 8),     # between two rows of queries that lie far apart
    (12 * 256, 5 * 12 * 256 + 256),                  # right behind the last row
])
def test_an_output_beside_the_queries_is_taken(B, q_stride, shift, bound):
    """Queries and output in one buffer: only an output over the queries is refused (there, nothing is written)."""
    c = Case(B, 2, [40, 0, 700, 9, 33, 1], 4, (8, 2), 64, 16)
    want, want_lse, _ = call(B, c, bound)
    room = 6 * 256
    buf = torch.full((2 * room + 6 * q_stride,), 5.0, dtype=BF, device="cuda")
    q = torch.as_strided(buf, (2, 3, 256), (3 * q_stride, q_stride, 1), room)
    q.copy_(c.dq)
    before = buf.clone()
    out = buf[room + shift:room + shift + 6 * 256].view(2, 3, 256)
    _, lse, _ = call(B, c, bound, q=q, out=out)
    assert B.twist_device_status() == 0
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.equal(q, c.dq)
    out.copy_(before[room + shift:room + shift + 6 * 256].view(2, 3, 256))
    assert torch.equal(buf, before)
    for over in (0, 8, -8):
        with pytest.raises(B.TwistError):
            call(B, c, bound, q=q, out=buf[room + over:room + over + 6 * 256].view(2, 3, 256))
    torch.cuda.synchronize()
    assert torch.equal(buf, before)
