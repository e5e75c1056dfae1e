"""The 8-bit cache (append, decode), the attention weight that cached tokens gather, and eviction by it, against the definitions in
64 bits.

Tolerances (derived, per element).
 * append: numbers and scales of what is not rotated are exact.  Rotated K has an error of 2^-20 (|x| + |y|) before it is rounded
   (the reduced angle is exact to 1.9e-7 rad, sincospif to a few 2^-24, two products and a sum to 2^-23), which may move it to the
   neighbouring number: half a step of e4m3 is 2^-4 of the value, at least 2^-10 of the scale, so
   |error| <= 2^-4 (|want| + r) + 2^-10 scale + r, r = 2^-20 (|x| + |y|).  Q: 2^-8 |want| + r.
 * decode: a score is a sum of d exact products in fp32 (queries in fp16 keep 29 binary digits against the head's largest: less
   than the sum's own rounding): its error is at most e_s = (d + 4) 2^-23 sum|q k| / sqrt(d), which with 2^-21 for the
   exponential is the relative error of its probability.  A probability as fp16, times at most 2^4 and at least 2^-4: half a
   step is 2^-12 of it, at least 2^-25 * 2^4 in units of the reference, against a sum of at least 1 in them.  Sums over n keys
   n 2^-23 each:
   |error| <= 2^-8 |want| + (2 e_s + 2^-20 + 2^-12 + 2 n 2^-23) sum p|v| + 2^-21 sum |v|;  log-sum-exp: e_s + 2^-20 + n 2^-23 + 2^-22 |want|.
 * weights: every term p = exp(s - lse) has the relative error e_s + 2^-22 |s - lse| + 2^-21, a sum of m terms m 2^-24 of itself.
 * evict: which tokens stay, where they go and all numbers are exact."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
F8 = torch.float8_e4m3fn
BLOCK = 16


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


def f64(t):
    """Numbers of an e4m3 tensor."""
    return t.detach().cpu().float().double().numpy()


def need(a):
    """The scale that magnitudes up to a need."""
    e = -110
    while e < 119 and a > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def code(x, scale):
    """e4m3 numbers nearest to x / scale (float64 array of numbers), saturating; NaN for what is not finite."""
    y = torch.from_numpy(np.where(np.isfinite(x), np.clip(np.where(np.isfinite(x), x, 0) / scale, -448, 448), np.nan))
    return y.float().to(F8).float().double().numpy()


def paged(gen, lens, page, spare=3, max_pages=None):
    """(table [n][max_pages] int32, pages of the pool): scattered pages; unused entries hold nonsense."""
    need_ = [-(-v // page) for v in lens]
    most = max(1, max(need_)) if max_pages is None else max_pages
    pool = sum(need_) + spare
    order = torch.randperm(pool, generator=gen).tolist()
    table, at = [], 0
    for k in need_:
        table.append(order[at:at + k] + [10 ** 6] * (most - k))
        at += k
    return table, pool


def pools(gen, pool, KV, page, D, spread=2):
    """(K, V, scales) on the GPU: blocks of different spread, some subnormal numbers."""
    c = lambda: (torch.randn(pool, KV, page, D, generator=gen) * 60).clamp(-448, 448).to(F8)
    s = torch.exp2(torch.randint(-6 - spread, -5 + spread, (pool, KV, page // BLOCK, 2), generator=gen).float())
    return c().cuda(), c().cuda(), s.cuda()


def values(cache, scales, which):
    """Cached values [pool][KV][page][D] in 64 bits."""
    x = f64(cache)
    s = host(scales)[..., which]
    return (x.reshape(*s.shape, BLOCK, -1) * s[..., None, None]).reshape(x.shape)


# ------------------------------------------------------------------------------------------------ append

def rotate64(x, pos, rot, layout):
    """x [rows][heads][D]; also |x| + |y| of every element's pair (0 where nothing is rotated)."""
    half = rot // 2
    y, slack = x.copy(), np.zeros_like(x)
    if rot:
        a = pos[:, None, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
        i, j = (slice(0, half), slice(half, rot)) if layout == 0 else (slice(0, rot, 2), slice(1, rot, 2))
        y[..., i] = x[..., i] * np.cos(a) - x[..., j] * np.sin(a)
        y[..., j] = x[..., i] * np.sin(a) + x[..., j] * np.cos(a)
        slack[..., i] = slack[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return y, slack


class Blocks:
    """The definition: a sequence's blocks of one KV position of K or of V."""

    def __init__(self):
        self.num, self.scale = {}, {}

    def append(self, slot, x):
        """Rows x [n][D] from `slot` on."""
        i = 0
        while i < len(x):
            blk, row = divmod(slot + i, BLOCK)
            take = min(BLOCK - row, len(x) - i)
            part = x[i:i + take]
            s = need(np.max(np.abs(np.where(np.isfinite(part), part, 0))))
            if row:
                s = max(s, self.scale[blk])
                for r in range(row):
                    self.num[blk, r] = code(self.num[blk, r] * self.scale[blk], s)
            self.scale[blk] = s
            for r in range(take):
                self.num[blk, row + r] = code(part[r], s)
            i += take


def call_append(B, S, n, T, H, KV, D, rot, layout, **t):
    freq = torch.tensor(10000.0 ** (-np.arange(0, max(rot, 1), 2) / max(rot, 1)), device="cuda") if rot else None
    B.twist_kv_append_q8(B.kv_append_q8_args(B.BF16, S, n, T, H, KV, D, rot, layout, inv_freq=freq, **t))


@pytest.mark.parametrize("D,page,H,KV", [(16, 16, 3, 2), (32, 64, 2, 1), (64, 32, 4, 4), (128, 128, 1, 1), (128, 16, 6, 3)])
def test_append_unrotated_is_exact_over_many_calls(B, D, page, H, KV):
    """Tokens in portions of every size: block borders inside and between portions, scales that grow, blocks of zeros, values from
    subnormal to the type's largest, infinities and NaN."""
    gen = torch.Generator().manual_seed(D + page)
    S, n = 2, 3
    most, w = 150, (H + 2 * KV) * D
    table, pool = paged(gen, [most] * (S * n), page)
    k = torch.full((pool, KV, page, D), 3.0).to(F8).cuda()
    v = torch.full((pool, KV, page, D), -5.0).to(F8).cuda()
    scales = torch.full((pool, KV, page // BLOCK, 2), 0.25, device="cuda")
    ref = {(s, b, g, j): Blocks() for s in range(S) for b in range(n) for g in range(KV) for j in (0, 1)}
    lens = [[0] * n for _ in range(S)]
    for step, portion in enumerate([1, 1, 14, 3, 37, 16, 5, 30, 1, 15]):
        new = [[(portion * (s + 2 * b + 1)) % (portion + 1) for b in range(n)] for s in range(S)]
        x = torch.randn(S, n, portion, w, generator=gen) * torch.exp2(torch.randint(-8, 9, (S, n, portion, 1), generator=gen).float())
        if step == 2:
            x[0, 0] = 0
        if step == 4:
            x[1, :, ::3] *= 2.0 ** 100
            x[0, 1] *= 2.0 ** -126
            x[0, 2, 5::7, ::5] = float("inf")
            x[1, 0, 3::5, 1::6] = float("nan")
        if step == 5:
            x[0, 0, 0] = torch.finfo(BF).max
        x = x.to(BF)
        for s in range(S):
            for b in range(n):
                lens[s][b] += new[s][b]
                rows = host(x[s, b, :new[s][b]]).reshape(new[s][b], H + 2 * KV, D)
                for g in range(KV):
                    for j in (0, 1):
                        ref[s, b, g, j].append(lens[s][b] - new[s][b], rows[:, H + j * KV + g])
        call_append(B, S, n, n * portion, H, KV, D, 0, 0, qkv=x.view(S, n * portion, w).cuda(), k_cache=k, v_cache=v, scales=scales,
                    page_table=i32(table).view(S, n, -1), kv_len=i32(lens), new_len=i32(new))
    assert B.twist_device_status() == 0
    num, sc = [f64(k), f64(v)], host(scales)
    touched = np.zeros((pool, KV, page), bool)
    for (s, b, g, j), blocks in ref.items():
        for (blk, r), want in blocks.num.items():
            slot = blk * BLOCK + r
            pg = table[s * n + b][slot // page]
            touched[pg, g, slot % page] = True
            assert np.array_equal(num[j][pg, g, slot % page], want, equal_nan=True), (s, b, g, j, slot)
            assert sc[pg, g, slot % page // BLOCK, j] == blocks.scale[blk]
    assert np.all(num[0][~touched] == 3.0) and np.all(num[1][~touched] == -5.0)
    blocks_touched = touched.reshape(pool, KV, -1, BLOCK).any(-1)
    assert np.all(sc[~blocks_touched] == 0.25)


@pytest.mark.parametrize("form", ["one", "padded", "packed"])
@pytest.mark.parametrize("D,rot,layout,page,H,KV", [
    (64, 64, 0, 32, 3, 2), (64, 64, 1, 16, 2, 2), (128, 128, 0, 64, 2, 1), (128, 64, 1, 16, 5, 3), (32, 32, 0, 16, 4, 1),
    (32, 20, 0, 32, 2, 2), (32, 22, 1, 16, 1, 1), (16, 16, 0, 16, 2, 1), (16, 8, 0, 64, 2, 2), (64, 36, 0, 16, 1, 1), (128, 2, 1, 128, 1, 1)])
def test_append_rotated(B, D, rot, layout, page, H, KV, form):
    gen = torch.Generator().manual_seed(17 * D + rot + layout)
    S, n, w = 2, 5, (H + 2 * KV) * D
    rows = 1 if form == "one" else 43
    new = [[1] * n, [1] * n] if form == "one" else [[0, 43, 1, 17, 16], [5, 0, 0, 31, 43]]
    past = [[0, 5, 16, 31, 200], [1, 15, 0, 33, 64]]
    lens = [[a + b for a, b in zip(x, y)] for x, y in zip(new, past)]
    seen = [[v + 1000 * (i + 1) for i, v in enumerate(r)] for r in lens]
    table, pool = paged(gen, [v for r in lens for v in r], page)
    k, v, scales = pools(gen, pool, KV, page, D)
    before = [values(k, scales, 0), values(v, scales, 1)]
    s_before = host(scales)
    T = n * rows if form != "packed" else max(sum(r) for r in new) + 3
    x = (torch.randn(S, T, w, generator=gen) * 2).to(BF)
    begin = [[sum(r[:i]) for i in range(n + 1)] for r in new]
    kw = dict(new_begin=i32(begin)) if form == "packed" else dict(new_len=i32(new)) if form == "padded" else {}
    dx = x.cuda()
    q_out = torch.full((S, T, H * D), 7.0, dtype=BF, device="cuda")
    held = [KV, max(1, KV - 1)]
    call_append(B, S, n, T, H, KV, D, rot, layout, qkv=dx, q_out=q_out, k_cache=k, v_cache=v, scales=scales,
                page_table=i32(table).view(S, n, -1), kv_len=i32(lens), seen=i32(seen), kv_count=i32(held), **kw)
    assert B.twist_device_status() == 0
    got, sc, gq = [values(k, scales, 0), values(v, scales, 1)], host(scales), host(q_out)
    written = np.zeros((pool, KV, page), bool)
    owned = np.zeros((S, T), bool)
    for s in range(S):
        for b in range(n):
            m = new[s][b]
            r0 = begin[s][b] if form == "packed" else b * rows
            owned[s, r0:r0 + m] = True
            z = host(x[s, r0:r0 + m]).reshape(m, H + 2 * KV, D)
            y, slack = rotate64(z[:, :H + KV], np.arange(seen[s][b] - m, seen[s][b], dtype=np.float64), rot, layout)
            r = 2.0 ** -20 * slack
            assert np.all(np.abs(gq[s, r0:r0 + m].reshape(m, H, D) - y[:, :H]) <= 2.0 ** -8 * np.abs(y[:, :H]) + r[:, :H])
            for i in range(m):
                slot = lens[s][b] - m + i
                pg, at = table[s * n + b][slot // page], slot % page
                written[pg, :held[s], at // BLOCK * BLOCK:at // BLOCK * BLOCK + BLOCK] = True
                for g in range(held[s]):
                    sk, sv = sc[pg, g, at // BLOCK]
                    want, tol = y[i, H + g], r[i, H + g]
                    assert np.all(np.abs(got[0][pg, g, at] - want) <= 2.0 ** -4 * (np.abs(want) + tol) + 2.0 ** -10 * sk + tol)
                    want = z[i, H + KV + g]
                    assert np.all(np.abs(got[1][pg, g, at] - want) <= 2.0 ** -4 * np.abs(want) + 2.0 ** -10 * sv)
            # what the blocks held before keeps its value to the new scale's rounding
            for slot in range((lens[s][b] - m) // BLOCK * BLOCK, lens[s][b] - m if m else 0):
                pg, at = table[s * n + b][slot // page], slot % page
                for j in (0, 1):
                    old, now = before[j][pg, :held[s], at], got[j][pg, :held[s], at]
                    assert np.all(np.abs(now - old) <= 2.0 ** -10 * sc[pg, :held[s], at // BLOCK, j][:, None])
                    assert np.all(sc[pg, :held[s], at // BLOCK, j] >= s_before[pg, :held[s], at // BLOCK, j])
    assert np.all(gq[~owned] == 7.0)
    for j in (0, 1):
        assert np.array_equal(got[j][~written], before[j][~written])
    same = dx.clone()                                            # Q rotated in place: the same bits
    call_append(B, S, n, T, H, KV, D, rot, layout, qkv=same, q_out=same[..., :H * D], k_cache=k, v_cache=v, scales=scales,
                page_table=i32(table).view(S, n, -1), kv_len=i32(lens), seen=i32(seen), kv_count=i32(held), **kw)
    own = torch.from_numpy(owned).cuda()
    assert torch.equal(same[..., :H * D][own], q_out[own]) and torch.equal(same[..., H * D:], dx[..., H * D:])
    assert torch.equal(same[~own], dx[~own])


@pytest.mark.parametrize("form", ["one", "padded"])
@pytest.mark.parametrize("D", [16, 64, 128])
def test_append_to_blocks_of_any_scale(B, D, form):
    """A block whose scale is no power of two (another program's): the next power of two counts, its tokens are rounded to the new scale."""
    gen = torch.Generator().manual_seed(D)
    olds = [1.5 * 2.0 ** -3, 3.7, 2.0 ** -2, 0.3, 1e-3, 1.0000001, 5e-36]
    n, KV, page, held = len(olds), 2, 16, 5
    fresh = 1 if form == "one" else 6
    k, v, scales = pools(gen, n, KV, page, D)
    scales[:] = torch.tensor(olds, dtype=torch.float32, device="cuda")[:, None, None, None] * torch.tensor([1.0, 1.25], device="cuda")
    before = [f64(k), f64(v)]
    old = host(scales)
    x = (torch.randn(1, n * fresh, 3 * KV * D, generator=gen) * 20).to(BF)
    call_append(B, 1, n, n * fresh, KV, KV, D, 0, 0, qkv=x.cuda(), q_out=None, k_cache=k, v_cache=v, scales=scales,
                page_table=i32([[[b] for b in range(n)]]), kv_len=i32([[held + fresh] * n]))
    assert B.twist_device_status() == 0
    new = host(scales)
    rows = host(x).reshape(n, fresh, 3 * KV, D)
    for b in range(n):
        for g in range(KV):
            for which, cache in enumerate((k, v)):
                part = rows[b, :, KV + which * KV + g]
                was = old[b, g, 0, which]
                s = max(need(np.abs(part).max()), 2.0 ** max(-110, math.ceil(math.log2(was))))
                assert new[b, g, 0, which] == s
                got = f64(cache)[b, g]
                assert np.array_equal(got[held:held + fresh], code(part, s))
                mine = (before[which][b, g, :held].astype(np.float32) * np.float32(was / s)).astype(np.float64)
                assert np.array_equal(got[:held], code(mine, 1.0))


def test_append_bad_index_data_is_skipped_and_reported(B):
    gen = torch.Generator().manual_seed(5)
    S, n, H, KV, D, page = 1, 4, 2, 1, 64, 16
    table, pool = paged(gen, [40] * 4, page)
    w = (H + 2 * KV) * D
    x = torch.randn(S, n * 9, w, generator=gen).to(BF).cuda()

    def call(lens, table=table, **kw):
        k, v, scales = pools(torch.Generator().manual_seed(1), pool, KV, page, D)
        first = [t.clone() for t in (k, v, scales)]
        q = torch.full((S, n * 9, H * D), 7.0, dtype=BF, device="cuda")
        call_append(B, S, n, n * 9, H, KV, D, 0, 0, qkv=x, q_out=q, k_cache=k, v_cache=v, scales=scales, page_table=i32([table]),
                    kv_len=i32([lens]), **kw)
        status = B.twist_device_status()
        rows = [b for b in range(n) if not torch.all(q[0, b * 9:b * 9 + 9] == 7.0)]
        same = all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(first, (k, v, scales)))
        return status, rows, same

    assert call([9, 20, 40, 48]) == (0, [0, 1, 2, 3], False)
    assert call([8, 8, 8, 8])[:2] == (B.ERR_BAD_INDEX, [])                 # fewer cached tokens than new ones
    assert call([49, 20, 8, 49]) == (B.ERR_BAD_INDEX, [1], False)          # more than the table has slots
    assert call([20] * 4, new_len=i32([[10, 9, -1, 0]])) == (B.ERR_BAD_INDEX, [1], False)
    assert call([20] * 4, seen=i32([[19, 20, 500, 0]])) == (B.ERR_BAD_INDEX, [1, 2], False)
    bad = [[10 ** 6, -1, pool]] * 4
    assert call([20] * 4, table=bad) == (B.ERR_BAD_INDEX, [], True)
    for begin in ([0, 9, 5, 18, 20], [-1, 9, 10, 11, 12], [0, 9, 18, 27, 37]):
        assert call([20] * 4, new_begin=i32([begin])) == (B.ERR_BAD_INDEX, [], True)


# ------------------------------------------------------------------------------------------------ decode and weights

def heads_of(gen, S, NH, NKV, H):
    """(head_idx, kv_pos, KV position of every kept head, kv_max)."""
    per = NH // NKV
    idx = [sorted(torch.randperm(NH, generator=gen)[:H].tolist()) for _ in range(S)]
    kv_pos, of = [], []
    for hs in idx:
        held = sorted({h // per for h in hs})
        kv_pos.append([held.index(g) if g in held else -1 for g in range(NKV)])
        of.append([held.index(h // per) for h in hs])
    return idx, kv_pos, of, min(NKV, H)


def sequence(vals, table, m, page):
    """[KV][m][D]"""
    pages = table[:-(-m // page)]
    return np.concatenate([vals[p] for p in pages], axis=1)[:, :m]


SHAPES = [
    # D, page, S, lens, H, NH, NKV
    (16, 16, 2, [0, 1, 15, 16, 17, 63, 64, 65], 3, 4, 2),
    (32, 32, 1, [33, 1, 500, 129], 8, 8, 1),
    (64, 16, 2, [1, 31, 32, 33, 0, 700], 6, 8, 2),
    (64, 128, 1, [2000, 5], 12, 12, 1),            # twelve heads on a position: two passes
    (128, 16, 3, [17, 48, 0, 1, 333], 2, 4, 4),
    (128, 64, 1, [1029], 1, 1, 1),
    (64, 64, 1, [30011], 2, 2, 2),                 # long enough to be split
    (128, 16, 1, [9000, 1], 3, 8, 2),
    (32, 16, 2, [4097, 40, 0, 12000], 4, 8, 4),
    (16, 16, 1, [7001], 10, 10, 1),
]


def attention_case(gen, D, page, S, lens, H, NH, NKV, q8=True, spread=2):
    n = len(lens)
    idx, kv_pos, of, KV = heads_of(gen, S, NH, NKV, H)
    table, pool = paged(gen, lens * S, page)
    q = (torch.randn(S, n, H * D, generator=gen) * torch.rand(S, n, 1, generator=gen) * 2).to(BF)
    if q8:
        k, v, scales = pools(gen, pool, KV, page, D, spread)
        vals = [values(k, scales, 0), values(v, scales, 1)]
    else:
        k, v, scales = (torch.randn(pool, KV, page, D, generator=gen).to(BF) for _ in range(2)), None, None
        k, v = k
        vals = [host(k), host(v)]
        k, v = k.cuda(), v.cuda()
    return dict(S=S, n=n, D=D, page=page, lens=lens, H=H, NH=NH, NKV=NKV, KV=KV, idx=idx, kv_pos=kv_pos, of=of, table=table, pool=pool,
                q=q, k=k, v=v, scales=scales, vals=vals)


def decode_args(B, c, out, lse, ws, q=None, **kw):
    return B.attn_decode_q8_args(B.BF16, c["S"], c["n"], c["H"], c["KV"], c["D"], c["NH"], c["NKV"], q=c["q"].cuda() if q is None else q,
                                 k_cache=c["k"], v_cache=c["v"], scales=c["scales"], page_table=i32(c["table"]).view(c["S"], c["n"], -1),
                                 kv_len=i32([c["lens"]] * c["S"]), head_idx=i32(c["idx"]), kv_pos=i32(c["kv_pos"]), out=out, lse=lse, ws=ws, **kw)


def scores64(c, s, b):
    """(scores [H][m], their error bound, V by head)."""
    m, D, H = c["lens"][b], c["D"], c["H"]
    k = sequence(c["vals"][0], c["table"][s * c["n"] + b], m, c["page"])[c["of"][s]]
    q = host(c["q"][s, b]).reshape(H, D)
    x = np.einsum("hkd,hd->hk", k, q) / math.sqrt(D)
    e = (D + 4) * 2.0 ** -23 * np.einsum("hkd,hd->hk", np.abs(k), np.abs(q)) / math.sqrt(D)
    return x, e


def check_decode(c, out, lse):
    out, lse = host(out), host(lse)
    for s in range(c["S"]):
        for b in range(c["n"]):
            m = c["lens"][b]
            got = out[s, b].reshape(c["H"], c["D"])
            if m == 0:
                assert np.all(got == 0) and np.all(lse[s, :, b] == -np.inf)
                continue
            x, e = scores64(c, s, b)
            v = sequence(c["vals"][1], c["table"][s * c["n"] + b], m, c["page"])[c["of"][s]]
            top = x.max(1, keepdims=True)
            p = np.exp(x - top)
            l = p.sum(1, keepdims=True)
            want = np.einsum("hk,hkd->hd", p / l, v)
            e_s = e.max(1, keepdims=True)
            mass = np.einsum("hk,hkd->hd", p / l, np.abs(v))
            tol = 2.0 ** -8 * np.abs(want) + (2 * e_s + 2.0 ** -20 + 2.0 ** -12 + 2 * m * 2.0 ** -23) * mass + 2.0 ** -21 * np.abs(v).sum(1)
            assert np.all(np.abs(got - want) <= tol), (s, b, np.max(np.abs(got - want) / tol))
            wl = (top + np.log(l))[:, 0]
            assert np.all(np.abs(lse[s, :, b] - wl) <= e_s[:, 0] + 2.0 ** -20 + m * 2.0 ** -23 + 2.0 ** -22 * np.abs(wl))


@pytest.mark.parametrize("D,page,S,lens,H,NH,NKV", SHAPES)
def test_decode_q8(B, D, page, S, lens, H, NH, NKV):
    gen = torch.Generator().manual_seed(D * 31 + len(lens))
    c = attention_case(gen, D, page, S, lens, H, NH, NKV)
    # slots behind the ends hold NaN, and so do the scales of blocks that nothing has been written to
    num = c["k"].view(torch.uint8).cpu(), c["v"].view(torch.uint8).cpu()
    sc = c["scales"].cpu()
    used = np.zeros((c["pool"], page), bool)
    for i, row in enumerate(c["table"]):
        for slot in range(lens[i % len(lens)]):
            used[row[slot // page], slot % page] = True
    free = torch.from_numpy(~used)
    for x in num:
        x.permute(0, 2, 1, 3)[free] = 0x7F
    sc.permute(0, 2, 1, 3)[torch.from_numpy(~used.reshape(c["pool"], -1, BLOCK).any(-1))] = float("nan")
    c["k"].copy_(num[0].view(F8))
    c["v"].copy_(num[1].view(F8))
    c["scales"].copy_(sc)
    ws = torch.empty(B.twist_attn_decode_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    runs = []
    for _ in range(2):
        out = torch.full((S, c["n"], H * D), 3.0, dtype=BF, device="cuda")
        lse = torch.full((S, H, c["n"]), 3.0, device="cuda")
        B.twist_attn_decode_q8(decode_args(B, c, out, lse, ws))
        runs.append((out, lse))
    assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1])       # the same bits
    assert B.twist_device_status() == 0
    check_decode(c, *runs[0])
    for bound in (max(lens), 1):                                     # the bound chooses the way, not the result
        B.twist_attn_decode_q8(decode_args(B, c, out, lse, ws, max_len=bound))
        check_decode(c, out, lse)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_decode_q8_scales_far_apart(B, D):
    """Neighbouring blocks whose scales differ by up to 2^40, and scales that are no powers of two."""
    gen = torch.Generator().manual_seed(D)
    c = attention_case(gen, D, 16, 1, [50, 257, 3000], 4, 4, 2, spread=20)
    c["scales"][..., 0] = torch.rand(c["scales"].shape[:-1], generator=gen).cuda() * 0.02 + 0.001
    c["scales"][..., 1] *= 0.7
    c["vals"] = [values(c["k"], c["scales"], 0), values(c["v"], c["scales"], 1)]
    ws = torch.empty(B.twist_attn_decode_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(1, 3, 4 * D, dtype=BF, device="cuda"), torch.empty(1, 4, 3, device="cuda")
    B.twist_attn_decode_q8(decode_args(B, c, out, lse, ws))
    check_decode(c, out, lse)


@pytest.mark.parametrize("D", [16, 64, 128])
def test_decode_q8_queries_of_any_size_and_moving_maxima(B, D):
    """Queries from 2^-120 to 2^100 (fp16 alone would lose them), keys so small that scores stay finite, scores that grow along the
    cache, and a row of zeros."""
    gen = torch.Generator().manual_seed(D + 1)
    c = attention_case(gen, D, 16, 1, [700, 40], 4, 4, 4)
    q = torch.randn(1, 2, 4, D, generator=gen)
    q[:, :, 0] *= 2.0 ** -120
    q[:, :, 1] *= 2.0 ** 100
    q[:, :, 2] = 0
    q[:, :, 3] *= 3
    c["q"] = q.to(BF).view(1, 2, 4 * D)
    sc = c["scales"].cpu()
    sc[:, 1, :, 0] = 2.0 ** -105
    for i, row in enumerate(c["table"]):                              # growing scores of head 3
        for j, pg in enumerate(p for p in row if p < c["pool"]):
            sc[pg, 3, :, 0] = 2.0 ** -9 * (1 + j / 8)
    c["scales"].copy_(sc)
    c["vals"] = [values(c["k"], c["scales"], 0), values(c["v"], c["scales"], 1)]
    ws = torch.empty(B.twist_attn_decode_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(1, 2, 4 * D, dtype=BF, device="cuda"), torch.empty(1, 4, 2, device="cuda")
    B.twist_attn_decode_q8(decode_args(B, c, out, lse, ws))
    check_decode(c, out, lse)


def test_decode_q8_nan_touches_its_element_only(B):
    gen = torch.Generator().manual_seed(9)
    c = attention_case(gen, 64, 16, 1, [100], 2, 2, 2)
    num = c["v"].view(torch.uint8)
    num[c["table"][0][1], 0, 3, 5] = 0x7F
    ws = torch.empty(B.twist_attn_decode_workspace_bytes(64), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(1, 1, 128, dtype=BF, device="cuda"), torch.empty(1, 2, 1, device="cuda")
    B.twist_attn_decode_q8(decode_args(B, c, out, lse, ws))
    bad = torch.isnan(out[0, 0]).nonzero().flatten().tolist()
    assert bad == [5] and torch.isfinite(lse).all()


def test_decode_q8_cache_in_one_buffer_beyond_32_bits(B):
    """K and V pages side by side, pages beyond element 2^31, no sharing of heads."""
    gen = torch.Generator().manual_seed(3)
    D, page, KV = 128, 16, 2
    per = 2 * KV * page * D
    n_pages = (1 << 31) // per + 40
    buf = torch.zeros(n_pages, 2, KV, page, D, dtype=torch.uint8, device="cuda").view(F8)
    scales = torch.zeros(n_pages, KV, 1, 2, device="cuda")
    lens, use = [70, 33], [n_pages - 1 - i for i in range(8)]
    table = [use[:5], use[5:] + [0, 0]]
    q = torch.randn(1, 2, KV * D, generator=gen).to(BF)
    x = torch.randn(1, 103, 3 * KV * D, generator=gen).to(BF).cuda()
    B.twist_kv_append_q8(B.kv_append_q8_args(B.BF16, 1, 2, 103, KV, KV, D, qkv=x, k_cache=buf[:, 0], v_cache=buf[:, 1], scales=scales,
                                             page_table=i32([table]), kv_len=i32([lens]), new_begin=i32([[0, 70, 103]])))
    ws = torch.empty(B.twist_attn_decode_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(1, 2, KV * D, dtype=BF, device="cuda"), torch.empty(1, KV, 2, device="cuda")
    B.twist_attn_decode_q8(B.attn_decode_q8_args(B.BF16, 1, 2, KV, KV, D, q=q.cuda(), k_cache=buf[:, 0], v_cache=buf[:, 1], scales=scales,
                                                 page_table=i32([table]), kv_len=i32([lens]), out=out, lse=lse, ws=ws))
    assert B.twist_device_status() == 0
    few = torch.tensor(sorted(use), device="cuda")
    again = [[sorted(use).index(p) for p in t if p] for t in table]
    sub = [buf.view(torch.uint8)[few][:, j].contiguous().view(F8) for j in (0, 1)]
    c = dict(S=1, n=2, D=D, page=page, lens=lens, H=KV, of=[[0, 1]], table=again, q=q,
             vals=[values(sub[j], scales[few], j) for j in (0, 1)])
    check_decode(c, out, lse)
    want = host(x[0, :70]).reshape(70, 3 * KV, D)
    got = sequence(c["vals"][0], again[0], 70, page).transpose(1, 0, 2)
    assert np.all(np.abs(got - want[:, KV:2 * KV]) <= 2.0 ** -4 * np.abs(want[:, KV:2 * KV]) + 2.0 ** -10 * 2.0 ** -6)


def check_weights(c, lse, prior, fresh, got, slot_pos, seen, old_pos):
    lse = host(lse)
    got, pos = host(got), slot_pos.cpu().numpy()
    written = np.zeros(got.shape, bool)
    for s in range(c["S"]):
        for b in range(c["n"]):
            m = c["lens"][b]
            if m == 0:
                continue
            x, e = scores64(c, s, b)
            d = x - lse[s, :, b][:, None]
            p = np.exp(d)
            err = p * (e + 2.0 ** -22 * np.abs(d) + 2.0 ** -21)
            for g in sorted(set(c["of"][s])):
                mine = [h for h in range(c["H"]) if c["of"][s][h] == g]
                for j in range(m):
                    pg, at = c["table"][s * c["n"] + b][j // c["page"]], j % c["page"]
                    written[pg, g, at] = True
                    new = j >= m - fresh[s][b]
                    want = p[mine, j].sum() + (0.0 if new or prior is None else prior[pg, g, at])
                    assert abs(got[pg, g, at] - want) <= err[mine, j].sum() + (len(mine) + 1) * 2.0 ** -24 * want, (s, b, g, j)
                    assert pos[pg, g, at] == (seen[s][b] - m + j if new else old_pos)
    assert np.all(got[~written] == -3.0) and np.all(pos[~written] == old_pos)


@pytest.mark.parametrize("q8", [True, False])
@pytest.mark.parametrize("D,page,S,lens,H,NH,NKV", [s for s in SHAPES if max(s[3]) < 8000] + [(8, 16, 1, [100, 3], 10, 10, 1)])
def test_weights(B, D, page, S, lens, H, NH, NKV, q8):
    if q8 and D == 8:
        pytest.skip("an 8-bit cache has heads of 16 and more")
    gen = torch.Generator().manual_seed(D * 7 + len(lens))
    c = attention_case(gen, D, page, S, lens, H, NH, NKV, q8)
    lse = torch.full((S, H, c["n"]), float("-inf"))
    for s in range(S):
        for b in range(c["n"]):
            if lens[b]:
                x, _ = scores64(c, s, b)
                lse[s, :, b] = torch.logsumexp(torch.from_numpy(x), 1).float()
    lse = lse.cuda()
    prior = torch.rand(c["pool"], c["KV"], page, generator=gen).cuda()
    fresh = [[min(m, (3 * b + s) % 5) for b, m in enumerate(lens)] for s in range(S)]
    seen = [[m + 10 * b for b, m in enumerate(lens)] for _ in range(S)]

    def call(weights, slot_pos, prior, max_len=0, **kw):
        B.twist_attn_weights(B.attn_weights_args(
            B.BF16, S, c["n"], H, c["KV"], D, NH, NKV, max_len, q=c["q"].cuda(), lse=lse, k_cache=c["k"], scales=c["scales"],
            page_table=i32(c["table"]).view(S, c["n"], -1), kv_len=i32([lens] * S), head_idx=i32(c["idx"]), kv_pos=i32(c["kv_pos"]),
            weights=weights, slot_pos=slot_pos, prior=prior, **kw))

    fill = lambda: (torch.full_like(prior, -3.0), torch.full(prior.shape, -9, dtype=torch.int32, device="cuda"))
    for max_len in (0, max(lens), 1):
        got, pos = fill()
        call(got, pos, prior, max_len, new_len=i32(fresh), seen=i32(seen))
        check_weights(c, lse, host(prior), fresh, got, pos, seen, -9)
    ones = [[min(m, 1) for m in lens]] * S
    got, pos = fill()
    call(got, pos, None)                                       # no prior; one new token each; positions are slots
    check_weights(c, lse, None, ones, got, pos, [lens] * S, -9)
    mine = torch.where(got == -3.0, got, prior)                # in place
    want, pos2 = fill()
    call(want, pos2, prior, new_len=i32(fresh))
    call(mine, None, mine, new_len=i32(fresh))
    assert torch.equal(mine, want)
    assert B.twist_device_status() == 0


def test_weights_bad_index_data(B):
    gen = torch.Generator().manual_seed(2)
    c = attention_case(gen, 64, 16, 1, [40, 33], 4, 8, 2)
    lse = torch.zeros(1, 4, 2, device="cuda")
    w = lambda: torch.zeros(c["pool"], c["KV"], 16, device="cuda")

    def call(table=None, lens=None, **kw):
        B.twist_attn_weights(B.attn_weights_args(
            B.BF16, 1, 2, 4, c["KV"], 64, 8, 2, q=c["q"].cuda(), lse=lse, k_cache=c["k"], scales=c["scales"],
            page_table=i32(table or c["table"]).view(1, 2, -1), kv_len=i32([lens or c["lens"]]), head_idx=i32(kw.pop("idx", c["idx"])),
            kv_pos=i32(c["kv_pos"]), weights=w(), **kw))
        return B.twist_device_status()

    assert call() == 0
    assert call(new_len=i32([[1, -1]])) == B.ERR_BAD_INDEX and call(new_len=i32([[41, 1]])) == B.ERR_BAD_INDEX
    assert call(lens=[49, 1]) == B.ERR_BAD_INDEX and call(lens=[-1, 1]) == B.ERR_BAD_INDEX
    assert call(table=[[-5, 10 ** 6, c["pool"]]] * 2) == B.ERR_BAD_INDEX
    assert call(idx=[[0, 1, 2, 99]]) == B.ERR_BAD_INDEX
    assert call() == 0


@pytest.mark.parametrize("D", [8, 16, 64, 128])
def test_weights_of_keys_that_are_not_finite(B, D):
    """A key with an infinity in a bf16 cache gives what its heads' scores say (here all of them -inf: nothing), also where fewer than
    eight heads read it; a NaN gives NaN, and neither touches other keys."""
    gen = torch.Generator().manual_seed(D)
    H, page, m = 3, 16, 40
    k = torch.randn(3, 1, page, D, generator=gen).to(BF)
    k[0, 0, 5, 0] = float("inf")
    k[1, 0, 7, 1] = float("nan")
    q = torch.randn(1, 1, H, D, generator=gen).to(BF)
    q[..., 0] = -1.0
    weights, lse = torch.full((3, 1, page), -3.0, device="cuda"), torch.full((1, H, 1), 2.0, device="cuda")
    B.twist_attn_weights(B.attn_weights_args(
        B.BF16, 1, 1, H, 1, D, H, 1, q=q.view(1, 1, H * D).cuda(), lse=lse, k_cache=k.cuda(), page_table=i32([[[0, 1, 2]]]), kv_len=i32([[m]]),
        head_idx=i32([[0, 1, 2]]), kv_pos=i32([[0]]), weights=weights))
    got, x, y = host(weights).reshape(-1), host(q)[0, 0], host(k).reshape(-1, D)[:m]
    with np.errstate(invalid="ignore"):
        s = x @ y.T / math.sqrt(D)
        want = np.exp(s - 2.0).sum(0)
        e = (D + 4) * 2.0 ** -23 * (np.abs(x) @ np.abs(y).T) / math.sqrt(D) + 2.0 ** -22 * np.abs(s - 2.0) + 2.0 ** -21
        bound = (np.exp(s - 2.0) * e).sum(0) + (H + 1) * 2.0 ** -24 * want
    assert got[5] == 0.0 and np.isnan(got[16 + 7])
    fine = [j for j in range(m) if j not in (5, 16 + 7)]
    assert np.all(np.abs(got[fine] - want[fine]) <= bound[fine])
    assert np.all(got[m:] == -3.0)
    assert B.twist_device_status() == 0


# ------------------------------------------------------------------------------------------------ prompts

@pytest.mark.parametrize("last", [0, 1, 50])
@pytest.mark.parametrize("D,page,S,n,N,H,NH,NKV", [
    (8, 16, 1, 2, 37, 3, 4, 2), (16, 32, 2, 3, 70, 2, 2, 1), (32, 16, 1, 2, 300, 4, 8, 2), (64, 16, 2, 2, 129, 6, 8, 2),
    (64, 64, 1, 1, 513, 9, 9, 1), (64, 16, 1, 3, 1, 2, 2, 2), (128, 16, 1, 2, 200, 3, 4, 4), (128, 128, 1, 1, 385, 2, 2, 1),
    (64, 16, 1, 2, 1024, 2, 2, 2)])
def test_core_weights(B, D, page, S, n, N, H, NH, NKV, last):
    gen = torch.Generator().manual_seed(D + N)
    idx, kv_pos, of, KV = heads_of(gen, S, NH, NKV, H)
    lens = [[N - (s + b) % 2 * (N // 3) if (s, b) != (0, 1) else min(N, 0 if N < 100 else 17) for b in range(n)] for s in range(S)]
    table, pool = paged(gen, [v for r in lens for v in r], page)
    x = (torch.randn(S, n, N, (H + 2 * KV) * D, generator=gen) * 1.5).to(BF)
    lse = torch.full((S, H, n, N), float("nan"))
    for s in range(S):
        for b in range(n):
            x[s, b, lens[s][b]:] = float("nan")                 # rows behind the end may hold anything
    z = host(x)
    stats = {}
    for s in range(S):
        for b in range(n):
            m = lens[s][b]
            for h in range(H):
                if m:
                    q, k = z[s, b, :m, h * D:(h + 1) * D], z[s, b, :m, (H + of[s][h]) * D:(H + of[s][h] + 1) * D]
                    y = q @ k.T / math.sqrt(D)
                    e = (D + 4) * 2.0 ** -23 * (np.abs(q) @ np.abs(k).T) / math.sqrt(D)
                    y[np.triu_indices(m, 1)] = -np.inf
                    top = y.max(1)
                    lse[s, h, b, :m] = torch.from_numpy(top + np.log(np.exp(y - top[:, None]).sum(1))).float()
                    stats[s, b, h] = y, e
    weights, pos = torch.full((pool, KV, page), -3.0, device="cuda"), torch.full((pool, KV, page), -9, dtype=torch.int32, device="cuda")

    def call(weights, pos):
        B.twist_attn_core_weights(B.attn_core_weights_args(
            B.BF16, S, n, N, H, KV, D, NH, NKV, last, qkv=x.view(S, n * N, -1).cuda(), lse=lse.view(S, H, n * N).cuda(),
            page_table=i32(table).view(S, n, -1), new_len=i32(lens), head_idx=i32(idx), kv_pos=i32(kv_pos), weights=weights, slot_pos=pos))

    call(weights, pos)
    assert B.twist_device_status() == 0
    again = torch.full_like(weights, -3.0)
    call(again, None)
    assert torch.equal(again, weights)                          # the same bits
    got, where = host(weights), pos.cpu().numpy()
    written = np.zeros(got.shape, bool)
    for s in range(S):
        for b in range(n):
            m = lens[s][b]
            first = max(0, m - last) if last else 0
            for g in sorted(set(of[s])):
                want, err, terms = np.zeros(m), np.zeros(m), 0
                for h in (h for h in range(H) if of[s][h] == g and m):
                    y, e = stats[s, b, h]
                    d = (y - lse[s, h, b, :m].double().numpy()[:, None])[first:]
                    p = np.exp(d)
                    want += p.sum(0)
                    err += np.where(p > 0, p * (e[first:] + 2.0 ** -22 * np.where(np.isfinite(d), np.abs(d), 0) + 2.0 ** -21), 0).sum(0)
                    terms += m - first
                for j in range(m):
                    pg, at = table[s * n + b][j // page], j % page
                    written[pg, g, at] = True
                    assert abs(got[pg, g, at] - want[j]) <= err[j] + terms * 2.0 ** -24 * want[j], (s, b, g, j)
                    assert where[pg, g, at] == j
    assert np.all(got[~written] == -3.0) and np.all(where[~written] == -9)


@pytest.mark.parametrize("last", [0, 1, 129, 400])
@pytest.mark.parametrize("D,page,S,n,N,H,NH,NKV", [
    (16, 16, 1, 2, 900, 1, 1, 1), (16, 64, 2, 2, 700, 3, 4, 2), (32, 32, 1, 2, 700, 5, 12, 4), (32, 16, 2, 1, 1025, 1, 2, 1),
    (32, 16, 1, 3, 130, 12, 12, 1), (16, 128, 1, 1, 257, 8, 8, 1)])
def test_core_weights_small_heads(B, D, page, S, n, N, H, NH, NKV, last):
    """Rows narrower than the tile that is copied, neighbours in it, few and many queries a key."""
    test_core_weights(B, D, page, S, n, N, H, NH, NKV, last)


@pytest.mark.parametrize("row", [400, 401, 403, 640, 1100])
@pytest.mark.parametrize("D", [16, 64, 128])
def test_core_weights_of_a_query_that_is_not_a_number(B, D, row):
    """Its head's keys up to it are NaN, the keys behind it and the other position's are not."""
    gen = torch.Generator().manual_seed(D)
    N, page = 1200, 64
    x = torch.randn(1, N, 6 * D, generator=gen).to(BF)
    x[0, row, 3] = float("nan")                                 # of head 0
    z = host(x)[0]
    lse = torch.empty(1, 2, N)
    want = np.zeros((2, N))
    for h in range(2):
        with np.errstate(invalid="ignore"):
            y = z[:, h * D:(h + 1) * D] @ z[:, (2 + h) * D:(3 + h) * D].T / math.sqrt(D)
            y[np.triu_indices(N, 1)] = -np.inf
            l = np.log(np.exp(y).sum(1))                        # the scores are small
            want[h] = np.where(np.tril(np.ones((N, N))) > 0, np.exp(y - l[:, None]), 0).sum(0)
        lse[0, h] = torch.from_numpy(l).float()
    pages = -(-N // page)
    weights = torch.full((pages, 2, page), -3.0, device="cuda")
    B.twist_attn_core_weights(B.attn_core_weights_args(
        B.BF16, 1, 1, N, 2, 2, D, qkv=x.cuda(), lse=lse.cuda(), page_table=i32([[list(range(pages))]]), weights=weights,
        slot_pos=torch.zeros(weights.shape, dtype=torch.int32, device="cuda")))
    got = host(weights).transpose(1, 0, 2).reshape(2, -1)[:, :N]
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).sum() == row + 1
    fine = ~np.isnan(want)
    # scores below 16 in magnitude: the tolerance of a weight's terms, with sum |q k| / sqrt(d) <= 6 sqrt(d) for these numbers
    bound = (D + 4) * 2.0 ** -23 * 6 * math.sqrt(D) + 2.0 ** -22 * 32 + 2.0 ** -21 + N * 2.0 ** -24
    assert np.all(np.abs(got - want)[fine] <= bound * want[fine])
    assert B.twist_device_status() == 0


# ------------------------------------------------------------------------------------------------ eviction

def evict64(num, scales, w, pos, table, lens, keeps, seens, recent, held, page, q8):
    """The definition, on copies; returns (k, v, scales, weights, positions) and a mask of the slots below min(len, keep)."""
    k, v = num[0].copy(), num[1].copy()
    sc = None if scales is None else scales.copy()
    w_out, p_out = w.copy(), pos.copy()
    here = np.zeros(w.shape, bool)
    for i, m in enumerate(lens):
        keep, seen = keeps[i], seens[i]
        at = lambda slot: (table[i][slot // page], slot % page)
        for g in range(held[i]):
            W = np.array([w[at(j)[0], g, at(j)[1]] for j in range(m)], np.float64)
            P = [int(pos[at(j)[0], g, at(j)[1]]) for j in range(m)]
            guard = seen - min(recent, keep)
            def rank(j):
                if P[j] >= guard:
                    return (0, 0.0, j)
                return (2, 0.0, j) if np.isnan(W[j]) else (1, -W[j], j)
            best = set(sorted(range(m), key=rank)[:keep])
            source = list(range(m))
            movers = iter([j for j in range(keep, m) if j in best])
            taken = [j for j in range(min(keep, m)) if j not in best]
            for j in taken:
                source[j] = next(movers)
            for j in range(min(keep, m)):
                a, b = at(j), at(source[j])
                here[a[0], g, a[1]] = True
                w_out[a[0], g, a[1]], p_out[a[0], g, a[1]] = w[b[0], g, b[1]], pos[b[0], g, b[1]]
            if not q8:
                for j in taken:
                    a, b = at(j), at(source[j])
                    k[a[0], g, a[1]], v[a[0], g, a[1]] = num[0][b[0], g, b[1]], num[1][b[0], g, b[1]]
                continue
            for blk in sorted({j // BLOCK for j in taken}):
                rows = [j for j in range(blk * BLOCK, min(m, blk * BLOCK + BLOCK))]
                for c, (old, new) in enumerate(((num[0], k), (num[1], v))):
                    true = [old[at(source[j])[0], g, at(source[j])[1]] * scales[at(source[j])[0], g, at(source[j])[1] // BLOCK, c] for j in rows]
                    s = need(max(np.max(np.abs(np.where(np.isfinite(x), x, 0))) for x in true))
                    for j, x in zip(rows, true):
                        new[at(j)[0], g, at(j)[1]] = code(x, s)
                    sc[at(rows[0])[0], g, at(rows[0])[1] // BLOCK, c] = s
    return k, v, sc, w_out, p_out, here


EVICTIONS = [
    # D, page, KV, lens, keeps, recent
    (64, 16, 2, [40, 17, 16, 0, 1], [20, 16, 16, 5, 0], 4),
    (16, 16, 1, [33, 100, 64], [32, 1, 63], 0),
    (32, 64, 3, [500, 129], [255, 128], 1000),
    (128, 16, 1, [1040, 1025], [1024, 1024], 256),
    (128, 128, 2, [700], [333], 100),
    (64, 32, 1, [3000, 2500, 31], [777, 2499, 30], 64),
    (64, 16, 1, [9000], [4001], 1000),                    # several CTAs
    (16, 1024, 1, [20000], [9999], 7),
]


@pytest.mark.parametrize("q8", [True, False])
@pytest.mark.parametrize("D,page,KV,lens,keeps,recent", EVICTIONS)
def test_evict(B, D, page, KV, lens, keeps, recent, q8):
    gen = torch.Generator().manual_seed(D + page + len(lens))
    n = len(lens)
    table, pool = paged(gen, lens, page)
    if q8:
        k, v, scales = pools(gen, pool, KV, page, D, spread=4)
        k.view(torch.uint8)[:, :, 3, 0] = 0x7F
        num = [f64(k), f64(v)]
    else:
        k, v, scales = (torch.randn(pool, KV, page, D, generator=gen).to(BF).cuda() for _ in range(2)), None, None
        k, v = k
        num = [host(k), host(v)]
    # many equal weights, and some that are no numbers
    w = torch.randint(0, 30, (pool, KV, page), generator=gen).float() / 8
    dice = torch.rand(pool, KV, page, generator=gen)
    w = torch.where(dice < 0.02, float("nan"), torch.where(dice < 0.04, float("inf"), torch.where(dice < 0.06, -float("inf"), torch.where(dice < 0.3, torch.rand(w.shape, generator=gen), w))))
    w = torch.where((dice > 0.97), -0.0, w)
    seen = [m + 100 * i for i, m in enumerate(lens)]
    pos = torch.full((pool, KV, page), -1, dtype=torch.int32)
    for i, m in enumerate(lens):
        for g in range(KV):
            where = torch.randperm(seen[i], generator=gen)[:m].tolist() if seen[i] else []
            for j in range(m):
                pos[table[i][j // page], g, j % page] = where[j]
    held = [max(1, KV - 1)] * n if KV > 1 else [1] * n
    ref = evict64(num, None if not q8 else host(scales), w.numpy(), pos.numpy(), table, lens, keeps, seen, recent, held, page, q8)
    table_ = i32([[x if x < 10 ** 6 else 0 for x in r] for r in table]).view(1, n, -1)
    max_len = max(lens)
    for in_place in (False, True):
        k2, v2, w2, p2 = k.clone(), v.clone(), w.cuda(), pos.cuda()
        s2 = None if scales is None else scales.clone()
        wo, po = (w2, p2) if in_place else (torch.full_like(w2, -3.0), torch.full_like(p2, -9))
        ws = torch.empty(B.twist_kv_evict_workspace_bytes(1, n, KV, max_len), dtype=torch.uint8, device="cuda")
        B.twist_kv_evict(B.kv_evict_args(
            B.BF16, 1, n, KV, D, recent, max_len, k_cache=k2, v_cache=v2, scales=s2, weights=w2, slot_pos=p2, weights_out=wo, slot_pos_out=po,
            page_table=table_, kv_len=i32([lens]), keep=i32([keeps]), seen=i32([seen]), kv_count=i32([held[0]]), ws=ws))
        assert B.twist_device_status() == 0
        got = (f64(k2), f64(v2)) if q8 else (host(k2), host(v2))
        here = ref[5]
        assert np.array_equal(po.cpu().numpy()[here], ref[4][here])
        assert np.array_equal(wo.cpu().numpy()[here], ref[3][here], equal_nan=True)
        if q8:
            assert np.array_equal(host(s2), ref[2])
        for a, b in zip(got, ref[:2]):
            assert np.array_equal(a, b, equal_nan=True)
        if in_place:
            assert torch.equal(w2.cpu()[torch.from_numpy(~here)].view(torch.int32), w[torch.from_numpy(~here)].view(torch.int32))
        else:
            assert torch.all(wo[torch.from_numpy(~here).cuda()] == -3.0) and torch.all(po[torch.from_numpy(~here).cuda()] == -9)


def test_evict_more_slots_than_shared_memory_keeps(B):
    """A position of 250 000 tokens over a cluster: part of the keys are formed again in every pass."""
    gen = torch.Generator().manual_seed(1)
    m, keep, page, D = 250_001, 100_003, 1024, 8
    pages = -(-m // page)
    k = torch.arange(pages * page, dtype=torch.int32).view(1, 1, -1)
    cache = torch.zeros(pages, 1, page, D, dtype=BF, device="cuda")
    bits = cache.view(torch.int32)                                   # the token's number in the row itself
    bits[..., 0] = k.view(pages, 1, page).cuda()
    w = torch.rand(pages, 1, page, generator=gen).mul_(50000).floor_()
    pos = k.view(pages, 1, page).clone()
    want = torch.argsort(torch.where(k.flatten()[:m] >= m - 5000, float("inf"), w.flatten()[:m]), descending=True, stable=True)[:keep]
    w2, p2 = w.cuda(), pos.cuda()
    ws = torch.empty(B.twist_kv_evict_workspace_bytes(1, 1, 1, m), dtype=torch.uint8, device="cuda")
    B.twist_kv_evict(B.kv_evict_args(B.BF16, 1, 1, 1, D, 5000, m, k_cache=cache, v_cache=cache.clone(), weights=w2, slot_pos=p2,
                                     page_table=torch.arange(pages, dtype=torch.int32, device="cuda").view(1, 1, -1), kv_len=i32([[m]]),
                                     keep=i32([[keep]]), ws=ws))
    assert B.twist_device_status() == 0
    got = p2.flatten()[:keep].cpu()
    assert torch.equal(got.sort().values.long(), want.sort().values)
    assert torch.equal(cache.view(torch.int32)[..., 0].flatten()[:keep].cpu(), got)
    assert torch.equal(w2.flatten()[:keep].cpu(), w.flatten()[got.long()])
    stays = torch.zeros(m, dtype=torch.bool)
    stays[want] = True
    low = stays[:keep]
    assert torch.equal(got[low], torch.arange(keep, dtype=torch.int32)[low])               # who stays is not touched
    assert torch.equal(got[~low].long(), (keep + stays[keep:].nonzero().flatten()))        # movers in ascending order


@pytest.mark.parametrize("m,keep,recent", [(1040, 1024, 0), (1040, 1024, 256), (300, 1, 0), (3000, 777, 100), (9000, 4001, 0), (9000, 8999, 50)])
@pytest.mark.parametrize("kind", ["equal", "two", "low bits", "last bits", "some equal", "descending", "one bin"])
def test_evict_weights_close_together(B, kind, m, keep, recent):
    """The threshold among weights that differ late or not at all; a KV position whose other half has the weights in reverse."""
    gen = torch.Generator().manual_seed(m + keep)
    page, D = 64, 16
    pages = -(-m // page)
    one = {"equal": lambda: torch.full((m,), 0.75), "two": lambda: 1 + torch.randint(0, 2, (m,), generator=gen) * 2.0 ** -23,
           "low bits": lambda: 1 + torch.randint(0, 8000, (m,), generator=gen) * 2.0 ** -23,
           "last bits": lambda: 1 + torch.randint(0, 900, (m,), generator=gen) * 2.0 ** -23,
           "some equal": lambda: torch.where(torch.rand(m, generator=gen) < 0.6, torch.tensor(0.5), torch.rand(m, generator=gen)),
           "descending": lambda: 2.0 - torch.arange(m) / m, "one bin": lambda: 1 + 0.2 * torch.rand(m, generator=gen)}[kind]().float()
    w = torch.zeros(2, pages * page)
    w[0, :m], w[1, :m] = one, one.flip(0)
    seq = torch.stack([torch.randperm(m, generator=gen) for _ in range(2)]).int()
    pos = torch.full((2, pages * page), -1, dtype=torch.int32)
    pos[:, :m] = seq
    lay = lambda t: t.view(2, pages, page).transpose(0, 1).contiguous().cuda()
    back = lambda t: t.cpu().transpose(0, 1).reshape(2, -1)
    cache = torch.zeros(pages, 2, page, D, dtype=BF, device="cuda")
    cache.view(torch.int32)[..., 3] = lay(pos)                       # the token's number in the row itself
    w2, p2, v = lay(w), lay(pos), cache.clone()
    ws = torch.empty(B.twist_kv_evict_workspace_bytes(1, 1, 2, m), dtype=torch.uint8, device="cuda")
    B.twist_kv_evict(B.kv_evict_args(B.BF16, 1, 1, 2, D, recent, m, k_cache=cache, v_cache=v, weights=w2, slot_pos=p2,
                                     page_table=torch.arange(pages, dtype=torch.int32, device="cuda").view(1, 1, -1), kv_len=i32([[m]]),
                                     keep=i32([[keep]]), ws=ws))
    assert B.twist_device_status() == 0
    for g in range(2):
        rank = torch.where(seq[g] >= m - min(recent, keep), float("inf"), w[g, :m])
        stays = torch.zeros(m, dtype=torch.bool)
        stays[torch.argsort(rank, descending=True, stable=True)[:keep]] = True
        source = torch.arange(m)[:keep].clone()
        source[~stays[:keep]] = keep + stays[keep:].nonzero().flatten()
        assert torch.equal(back(p2)[g, :keep], pos[g, source])
        assert torch.equal(back(w2)[g, :keep], w[g, source])
        for t in (cache, v):
            assert torch.equal(back(t.view(torch.int32)[..., 3])[g, :keep], pos[g, source])


def test_evict_bad_index_data(B):
    gen = torch.Generator().manual_seed(4)
    page, D, KV = 16, 64, 2
    table, pool = paged(gen, [60, 60], page)
    first = pools(gen, pool, KV, page, D)
    w = torch.rand(pool, KV, page, generator=gen).cuda()
    pos = torch.zeros(pool, KV, page, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.twist_kv_evict_workspace_bytes(1, 2, KV, 64), dtype=torch.uint8, device="cuda")

    def call(table, lens, keep):
        t = [x.clone() for x in (*first, w, pos)]
        B.twist_kv_evict(B.kv_evict_args(B.BF16, 1, 2, KV, D, 0, k_cache=t[0], v_cache=t[1], scales=t[2], weights=t[3], slot_pos=t[4],
                                         page_table=i32([table]), kv_len=i32([lens]), keep=i32([keep]), ws=ws))
        status = B.twist_device_status()
        rows = [b for b in range(2) if not torch.equal(t[3][table[b]] if max(table[b]) < pool and min(table[b]) >= 0 else t[3][:0],
                                                       w[table[b]] if max(table[b]) < pool and min(table[b]) >= 0 else w[:0])]
        return status, rows

    assert call(table, [60, 60], [30, 30]) == (0, [0, 1])
    assert call([table[0], [table[1][0], -1, *table[1][2:]]], [60, 60], [30, 30]) == (B.ERR_BAD_INDEX, [0])
    assert call([table[0], [*table[1][:3], pool]], [60, 60], [30, 30]) == (B.ERR_BAD_INDEX, [0])
    assert call(table, [60, -1], [30, 30]) == (B.ERR_BAD_INDEX, [0])
    assert call(table, [65, 60], [64, -3])[0] == B.ERR_BAD_INDEX
    assert call(table, [60, 60], [60, 61]) == (0, [])


# ------------------------------------------------------------------------------------------------ together

def test_a_step_of_all_of_them_captured_and_replayed(B):
    """Append, decode, weights and eviction as one graph on a side stream, replayed with new lengths and inputs, against the same
    calls one by one; and two such steps at once on two streams."""
    gen = torch.Generator().manual_seed(8)
    S, n, H, KV, D, page, budget = 2, 3, 4, 2, 64, 16, 32

    class Step:
        def __init__(self, seed):
            g = torch.Generator().manual_seed(seed)
            pool = S * n * 4
            self.table = torch.randperm(pool, generator=g).to(torch.int32).view(S, n, 4).cuda()
            self.k, self.v = (torch.zeros(pool, KV, page, D, device="cuda").to(F8) for _ in range(2))
            self.scales = torch.ones(pool, KV, 1, 2, device="cuda")
            self.w, self.pos = torch.zeros(pool, KV, page, device="cuda"), torch.zeros(pool, KV, page, dtype=torch.int32, device="cuda")
            self.len, self.seen, self.keep = (torch.zeros(S, n, dtype=torch.int32, device="cuda") for _ in range(3))
            self.x = torch.zeros(S, n, (H + 2 * KV) * D, dtype=BF, device="cuda")
            self.out, self.lse = torch.zeros(S, n, H * D, dtype=BF, device="cuda"), torch.zeros(S, H, n, device="cuda")
            self.ws = torch.zeros(B.twist_attn_decode_workspace_bytes(D), dtype=torch.uint8, device="cuda")
            self.ws2 = torch.zeros(B.twist_kv_evict_workspace_bytes(S, n, KV, 64), dtype=torch.uint8, device="cuda")
            self.idx, self.kv_pos = i32([[0, 1, 2, 3]] * S), i32([[0, 1]] * S)
            self.freq = torch.tensor(10000.0 ** (-np.arange(0, D, 2) / D), device="cuda")

        def run(self):
            cache = dict(k_cache=self.k, v_cache=self.v, scales=self.scales, page_table=self.table, kv_len=self.len)
            q = self.x[..., :H * D]
            B.twist_kv_append_q8(B.kv_append_q8_args(B.BF16, S, n, n, H, KV, D, D, qkv=self.x, q_out=q, seen=self.seen, inv_freq=self.freq, **cache))
            B.twist_attn_decode_q8(B.attn_decode_q8_args(B.BF16, S, n, H, KV, D, 4, 2, q=q, out=self.out, lse=self.lse, ws=self.ws,
                                                         head_idx=self.idx, kv_pos=self.kv_pos, **cache))
            B.twist_attn_weights(B.attn_weights_args(B.BF16, S, n, H, KV, D, 4, 2, q=q, lse=self.lse, k_cache=self.k, scales=self.scales,
                                                     page_table=self.table, kv_len=self.len, prior=self.w, weights=self.w, slot_pos=self.pos,
                                                     seen=self.seen, head_idx=self.idx, kv_pos=self.kv_pos))
            B.twist_kv_evict(B.kv_evict_args(B.BF16, S, n, KV, D, 8, weights=self.w, slot_pos=self.pos, keep=self.keep, seen=self.seen,
                                             ws=self.ws2, **cache))

        def data(self, x, length, seen, keep):
            self.x.copy_(x)
            self.len.copy_(length)
            self.seen.copy_(seen)
            self.keep.copy_(keep)

        def state(self):
            return [t.clone() for t in (self.k.view(torch.uint8), self.v.view(torch.uint8), self.scales, self.w, self.pos, self.out, self.lse)]

    plain, captured, other = Step(1), Step(1), Step(2)
    captured.len.fill_(1)
    captured.seen.fill_(1)
    captured.keep.fill_(1)
    captured.run()                                                     # loads the kernels
    fresh = Step(1)
    for name in ("k", "v", "scales", "w", "pos"):
        getattr(captured, name).copy_(getattr(fresh, name))
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        captured.run()
    length = torch.zeros(S, n, dtype=torch.int32)
    for t in range(60):
        length = torch.clamp(length + 1, max=64)
        x = torch.randn(S, n, (H + 2 * KV) * D, generator=gen).to(BF)
        seen = torch.full((S, n), t + 1, dtype=torch.int32)
        keep = torch.where(length > budget + 3, budget, length)
        for st in (plain, captured, other):
            st.data(x, length, seen, keep)
        torch.cuda.synchronize()
        plain.run()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        other.run()                                                    # at the same time, on the default stream
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(plain.state(), captured.state())), t
        assert torch.equal(plain.out, other.out) and torch.equal(plain.lse, other.lse)      # other pages, the same bits
        length = keep.clone()
    assert B.twist_device_status() == 0
    assert int(plain.pos.max()) == 59 and torch.isfinite(plain.out.float()).all()
