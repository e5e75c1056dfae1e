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


# ------------------------------------------------------------------------------------------------ the line of work

def twice(B, c, bound, **kw):
    """The same call two times: the same bits, checked against the definition; returns what one call returns."""
    out, lse, cut = call(B, c, bound, **kw)
    again, again_lse, again_cut = call(B, c, bound, **kw)
    assert torch.equal(out, again) and torch.equal(lse, again_lse) and cut == again_cut
    assert B.twist_device_status() == 0
    c.check(out, lse)
    return out, lse, cut


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129]
rng = lambda seed, n, top: [int(x) for x in np.random.default_rng(seed).integers(0, top, n)]
ROUTES = [
    # S, lens, H, (NH, NKV), d, page
    (1, EDGES, 1, None, 8, 16), (2, EDGES * 2, 2, None, 16, 32), (1, EDGES, 3, None, 32, 16), (2, EDGES * 2, 3, None, 64, 64), (1, EDGES, 2, None, 128, 128),
    (1, [0, 0, 0], 2, None, 64, 16),                                  # nothing cached anywhere
    (1, [0, 0, 900, 0, 1], 2, (4, 2), 16, 16),                        # empty sequences around the only long one
    # every head size: shared keys, several subnets, sequences that change inside a warp's work
    (2, rng(1, 10, 700), 5, (8, 2), 8, 16), (3, rng(2, 9, 2500), 5, (8, 4), 16, 16), (2, rng(3, 12, 2500), 4, (8, 2), 32, 64),
    (2, rng(4, 12, 900), 5, (8, 2), 64, 16), (2, rng(5, 16, 900), 5, (8, 4), 128, 32), (1, [5000, 1, 4999], 2, (4, 2), 128, 1024),
    # more than eight heads on a position: one and two row tiles, few items (a table of all of them) and many
    (1, [2500, 600], 12, (12, 1), 64, 64), (2, [900, 0, 3000, 17], 10, (48, 4), 64, 32), (1, [5000, 3], 13, (48, 4), 16, 16),
    (1, [2600, 31], 9, (36, 3), 128, 16), (2, rng(6, 6, 900), 30, (40, 2), 32, 16), (4, rng(7, 4 * 120, 300), 10, (48, 4), 32, 16),
    # more heads, and more sequences, than a CTA keeps
    (8, rng(8, 8 * 3, 1500), 70, (96, 8), 16, 16), (8, rng(9, 8 * 2, 300), 66, (80, 20), 64, 16), (32, rng(10, 32, 200), 9, (18, 9), 128, 16),
    (1, rng(11, 700, 40), 4, (8, 2), 64, 16), (2, rng(12, 2 * 700, 90), 2, None, 16, 16), (1, rng(13, 3000, 40), 1, None, 32, 16),
]


@pytest.mark.parametrize("case", range(len(ROUTES)))
def test_decode_through_the_line_of_work(B, case):
    """The cut of the line, the parts and their join: unused slots hold NaN, unused table entries lie outside the pool.  The
    short way gives the same within the tolerance of both."""
    S, lens, H, gqa, d, page = ROUTES[case]
    c = Case(B, S, lens, H, gqa, d, page, seed=case + 100, fill=float("nan"), interleaved=case % 2 == 1, q_wide=case % 3 == 1)
    _, _, cut = twice(B, c, LINE)
    assert cut is not None
    if max(lens) > 600:
        assert cut > 0


@pytest.mark.parametrize("d", [8, 16, 32, 64, 128])
def test_decode_the_short_way(B, d):
    c = Case(B, 2, [700, 0, 33, 1, 64, 129], 5, (8, 2), d, 16, seed=d, fill=float("nan"))
    assert twice(B, c, SHORT)[2] is None
    # a bound that the lengths pass: the same call, only the way its work is split is another
    assert twice(B, c, 1)[2] is None


@pytest.mark.parametrize("d", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("fill", [float("inf"), float("-inf"), torch.finfo(BF).min, torch.finfo(BF).max])
def test_decode_in_the_line_ignores_what_unused_slots_hold(B, fill, d):
    c = Case(B, 1, [33, 0, 700, 1], 4, (8, 2), d, 32, fill=fill)
    assert twice(B, c, LINE)[2] > 0
    assert twice(B, c, SHORT)[2] is None


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("bound", [SHORT, LINE])
def test_decode_scores_that_grow_along_a_cut_sequence(B, bound, d):
    """The reference maximum moves many times, and the parts of an item have maxima far from each other."""
    c = Case(B, 1, [3000, 513], 2, None, d, 16, sharp=3.0)
    ramp = (torch.arange(c.k.shape[0] * c.page) % 97).view(c.k.shape[0], 1, c.page, 1).float().cuda() / 8
    c.k = (c.k.float() * ramp).to(BF)
    cut = twice(B, c, bound)[2]
    assert cut is None if bound == SHORT else cut == 4


@pytest.mark.parametrize("d", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("bound", [SHORT, LINE])
def test_decode_non_finite_values_on_both_ways(B, bound, d):
    """Key -inf: no weight.  Key +inf, or NaN in a key or a query: NaN in the heads that read it.  NaN or an infinity in V:
    not finite in its own element only (an infinity may come out as NaN: its weight is the sum of two terms)."""
    n, key = 700, 333
    c = Case(B, 1, [n] * 8, 1, None, d, 16)
    q = torch.zeros(1, 8, d, dtype=BF)
    q[..., 0] = 1.0
    q[0, 4, d - 1] = float("nan")
    c.q, c.dq = q, q.cuda()
    slot = lambda cache, b, i: cache[c.table[0, b, i // 16].item(), 0, i % 16]
    for b, val in ((0, float("-inf")), (1, float("inf")), (3, float("nan"))):
        slot(c.k, b, key)[0] = val
    for b, val in ((2, float("nan")), (5, float("inf")), (6, float("-inf"))):
        slot(c.v, b, key)[d - 2] = val
    slot(c.v, 7, n - 1)[d - 2] = float("inf")                         # the last key, which stands in for those behind it
    out, lse, cut = call(B, c, bound)
    assert B.twist_device_status() == 0
    assert cut is None if bound == SHORT else cut == 8
    out, lse = host(out)[0], host(lse)[0, 0]
    for b in (1, 3, 4):
        assert np.all(np.isnan(out[b]))
    for b in (2, 5, 6, 7):
        assert not np.isfinite(out[b, d - 2]) and np.all(np.isfinite(np.delete(out[b], d - 2))) and np.isfinite(lse[b])
    assert np.isnan(out[2, d - 2])
    K, V = host(c.k), host(c.v)
    for b in (0, 2, 5, 6, 7):
        pages = c.table[0, b].numpy()[:-(-n // 16)]
        k, v = K[pages, 0].reshape(-1, d)[:n], V[pages, 0].reshape(-1, d)[:n]
        keep = np.arange(n) != key if b == 0 else np.ones(n, dtype=bool)
        p = np.exp(k[keep, 0] / np.sqrt(d))
        p, total = p / p.sum(), p.sum()
        cols = [j for j in range(d) if b == 0 or j != d - 2]
        want, size = p @ v[keep][:, cols], p @ np.abs(v[keep][:, cols])
        # one product: a score is exact up to its scaling (2^-21 with the exponential), the two-term weight adds 2^-16, n sums
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -19 + 2.0 ** -16 + 2 * n * 2.0 ** -23) * size
        assert np.all(np.abs(out[b, cols] - want) <= tol)
        assert abs(lse[b] - np.log(total)) <= 2.0 ** -19 + n * 2.0 ** -23 + 2.0 ** -22 * abs(np.log(total))


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("bound", [SHORT, LINE])
def test_decode_reports_bad_index_data_on_both_ways(B, bound, d):
    """A page outside the pool is read as page 0, lengths are clamped, a head or a position that does not exist reads
    position 0; the other sequences and heads are what they are without it."""
    c = Case(B, 1, [700, 900, 40], 4, (8, 2), d, 16)
    want, want_lse, cut = call(B, c, bound)
    assert B.twist_device_status() == 0 and (cut is None if bound == SHORT else cut > 0)
    table = widened(c.table, 16)
    for at, bad in ((3, c.k.shape[0]), (56, -1), (0, 1 << 30)):
        t = table.clone()
        t[0, 1, at] = bad
        out, lse, _ = call(B, c, bound, page_table=t)
        assert B.twist_device_status() == B.ERR_BAD_INDEX
        assert torch.equal(out[0, 0], want[0, 0]) and torch.equal(out[0, 2], want[0, 2])
        t[0, 1, at] = 0
        zero, zero_lse, _ = call(B, c, bound, page_table=t)
        assert B.twist_device_status() == 0 and torch.equal(out, zero) and torch.equal(lse, zero_lse)
    lens = c.dlens.clone()
    lens[0, 1] = -1
    out, lse, _ = call(B, c, bound, kv_len=lens)
    assert B.twist_device_status() == B.ERR_BAD_INDEX
    assert bool((out[0, 1] == 0).all()) and bool((lse[0, :, 1] == -float("inf")).all())
    lens[0, 1] = 0
    zero, zero_lse, _ = call(B, c, bound, kv_len=lens)
    assert B.twist_device_status() == 0 and torch.equal(out, zero) and torch.equal(lse, zero_lse)
    full = torch.where(table < c.k.shape[0], table, torch.zeros_like(table)).clamp_min(0)     # a length beyond the table is read as its room
    lens[0, 1] = WIDE
    most, most_lse, _ = call(B, c, bound, kv_len=lens, page_table=full)
    assert B.twist_device_status() == 0
    lens[0, 1] = WIDE + 1
    out, lse, _ = call(B, c, bound, kv_len=lens, page_table=full)
    assert B.twist_device_status() == B.ERR_BAD_INDEX and torch.equal(out, most) and torch.equal(lse, most_lse)
    heads = c.extra["head_idx"].clone()
    group = [h for h in range(4) if c.of[0][h] == 0]                  # heads that read position 0
    for bad in (8, -1, 1 << 30):
        heads[0, group[0]] = bad
        out, lse, _ = call(B, c, bound, head_idx=heads)
        assert B.twist_device_status() == B.ERR_BAD_INDEX and torch.equal(out, want) and torch.equal(lse, want_lse)
    pos = c.extra["kv_pos"].clone()
    pos[pos == 0] = 2                                                 # a position that the cache does not have
    out, lse, _ = call(B, c, bound, kv_pos=pos)
    assert B.twist_device_status() == B.ERR_BAD_INDEX and torch.equal(out, want) and torch.equal(lse, want_lse)


def test_decode_in_the_line_beyond_32_bit_offsets(B):
    """Pages more than 2^31 elements into the pool, in items that are cut."""
    d, page, kv = 64, 64, 2
    stride = (1 << 30) + 8 * 123
    flat = torch.zeros(3 * stride, dtype=BF, device="cuda")
    k = torch.as_strided(flat, (3, kv, page, d), (stride, page * d, d, 1), 0)
    v = torch.as_strided(flat, (3, kv, page, d), (stride, page * d, d, 1), kv * page * d)
    c = Case(B, 1, [190], 2, None, d, page)
    order = torch.tensor([2, 0, 1])
    for j in range(3):
        k[order[j]] = c.k[c.table[0, 0, j].item()]
        v[order[j]] = c.v[c.table[0, 0, j].item()]
    table = widened(order.to(torch.int32).view(1, 1, 3), page)
    for bound in (SHORT, LINE):
        out, lse, cut = call(B, c, bound, k_cache=k, v_cache=v, page_table=table)
        assert B.twist_device_status() == 0 and (cut is None if bound == SHORT else cut == 2)
        c.check(out, lse)


def test_calls_through_the_line_on_two_streams_and_in_two_graphs(B):
    """Overlapping calls with scratch of their own, launched and replayed, give what each gives alone."""
    cases = [Case(B, 1, [6000, 40, 700], 4, (8, 4), 64, 16, seed=s) for s in (1, 2)]
    tables = [widened(c.table, 16) for c in cases]
    want = [call(B, c, LINE)[:2] for c in cases]
    graphs = []
    for c, t in zip(cases, tables):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.twist_attn_decode(c.args(B, page_table=t))
        graphs.append(g)
    for replay in (False, True):
        for c in cases:
            c.out.fill_(9.0)
            c.lse.fill_(9.0)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in cases]
        for _ in range(20):
            for c, t, st, g in zip(cases, tables, streams, graphs):
                with torch.cuda.stream(st):
                    if replay:
                        g.replay()
                    else:
                        B.twist_attn_decode(c.args(B, page_table=t))
        torch.cuda.synchronize()
        for c, (out, lse) in zip(cases, want):
            assert torch.equal(c.out, out) and torch.equal(c.lse, lse) and cut_items(c.ws) > 0
    assert B.twist_device_status() == 0
