"""Rotation by position, the paged cache and the attention that reads it, against the definitions in 64 bits.

Tolerances (derived, per element).  u = 2^-8 is half a bf16 step relative to the value.
 * rotation: the reduced angle is exact to 2^-25 turns (1.9e-7 rad), sincospif to a few 2^-24, the two products and
   their difference to 2^-23 each: |error| <= u |want| + 2^-20 (|x| + |y|).
 * decode: a score is a sum of d products in fp32: its error is at most e_s = (d + 2) 2^-23 sum|q k| / sqrt(d), which
   (with 2^-21 for the exponential) is the relative error of its probability; the two-term bf16 probability adds 2^-16,
   the sums over n keys n 2^-23 each: |error| <= u |want| + (2 e_s + 2^-20 + 2^-16 + 2 n 2^-23) sum p|v|;
   log-sum-exp: e_s + 2^-20 + n 2^-23 + 2^-22 |want|."""
import numpy as np
import pytest
import torch

from oracle import twist_oracle as o

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
BF = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


def rng_bf16(gen, *shape, std=1.0):
    return (torch.randn(*shape, generator=gen) * std).to(BF)


def host(t):
    return t.detach().cpu().to(torch.float64).numpy()


def freqs(rot, base=10000.0):
    return base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)


def rotate64(x, pos, rot, layout, inv, sign=1.0):
    """x [.., heads, d] float64, pos [..]."""
    half = rot // 2
    a = pos[..., None, None].astype(np.float64) * inv
    c, s = np.cos(a), sign * np.sin(a)
    y = x.copy()
    i, j = (slice(0, half), slice(half, rot)) if layout == 0 else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., i] * s + x[..., j] * c
    slack = np.zeros_like(x)
    slack[..., i] = slack[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return y, U * np.abs(y) + 2.0 ** -20 * slack


# ------------------------------------------------------------------------------------------------ rotation

ROPE_SHAPES = [
    # S, n_seqs, N, H, KV, d, rot
    (1, 1, 1, 1, 1, 8, 8),            # half of the rotation is not a whole 16-byte chunk: element by element
    (2, 3, 5, 3, 2, 8, 2),
    (2, 1, 33, 2, 1, 16, 16),
    (1, 2, 77, 5, 2, 24, 12),
    (3, 2, 40, 4, 4, 64, 64),
    (2, 1, 130, 6, 1, 64, 32),        # half of every head rotated
    (1, 3, 501, 8, 8, 128, 128),
    (1, 1, 9, 2, 2, 256, 256),
    (2, 4, 1024, 16, 4, 64, 64),      # many rows: whole tiles of rows
    (1, 1, 3001, 3, 3, 40, 38),
]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("S,n_seqs,N,H,KV,d,rot", ROPE_SHAPES)
def test_rope_forward_and_backward(B, S, n_seqs, N, H, KV, d, rot, layout):
    gen = torch.Generator().manual_seed(7 * d + rot)
    T, w = n_seqs * N, (H + 2 * KV) * d
    x = rng_bf16(gen, S, T, w)
    inv = freqs(rot)
    dx, dinv = x.cuda(), torch.from_numpy(inv).cuda()
    pos = np.broadcast_to(np.arange(T) % N, (S, T))
    for sign, call in ((1.0, B.twist_rope_fwd), (-1.0, B.twist_rope_bwd)):
        out = torch.full_like(dx, 9.0)
        call(B.rope_args(B.BF16, S, T, H, KV, d, rot, N, layout, in_=dx, out=out, inv_freq=dinv))
        same = dx.clone()
        call(B.rope_args(B.BF16, S, T, H, KV, d, rot, N, layout, in_=same, out=same, inv_freq=dinv))
        assert torch.equal(out, same)                                  # in place: the same bits
        z = host(x).reshape(S, T, H + 2 * KV, d)
        want, tol = rotate64(z[:, :, :H + KV], pos, rot, layout, inv, sign)
        got = host(out).reshape(S, T, H + 2 * KV, d)
        assert np.all(np.abs(got[:, :, :H + KV] - want) <= tol)
        assert np.array_equal(got[:, :, H + KV:], z[:, :, H + KV:])    # V as it was
        assert np.array_equal(got[..., :H + KV, rot:], z[..., :H + KV, rot:])


def test_rope_explicit_and_far_positions(B):
    """Positions up to 2^31 - 1: the angle must be reduced in 64 bits."""
    S, T, H, KV, d = 2, 9, 2, 1, 64
    gen = torch.Generator().manual_seed(1)
    x = rng_bf16(gen, S, T, (H + 2 * KV) * d)
    pos = torch.randint(0, 1 << 20, (S, T), generator=gen, dtype=torch.int32)
    pos[0, :4] = torch.tensor([0, 1, 2 ** 31 - 1, 123456789], dtype=torch.int32)
    inv = freqs(d, 500000.0)
    out = torch.empty_like(x, device="cuda")
    B.twist_rope_fwd(B.rope_args(B.BF16, S, T, H, KV, d, d, in_=x.cuda(), out=out, inv_freq=torch.from_numpy(inv).cuda(), pos=pos.cuda()))
    z = host(x).reshape(S, T, H + 2 * KV, d)
    want, tol = rotate64(z[:, :, :H + KV], pos.numpy(), d, 0, inv)
    got = host(out).reshape(S, T, H + 2 * KV, d)
    # the angle is rounded four times in 64 bits, here and in the kernel: 4 * 2^31 * 2^-53 = 2^-20 rad more
    tol = tol + (tol - U * np.abs(want))
    assert np.all(np.abs(got[:, :, :H + KV] - want) <= tol)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("d,rot", [(16, 16), (32, 16), (8, 6)])
def test_rope_gradient_is_the_transpose_of_the_forward_differences(B, layout, d, rot):
    """The forward is linear, so its difference quotients are its values at unit vectors: column i is fwd(e_i), exact up to
    one rounding.  bwd(w) must be R^T w."""
    inv = torch.from_numpy(freqs(rot)).cuda()
    eye = torch.zeros(1, d, 3 * d, dtype=BF)
    eye[0, :, :d] = torch.eye(d)                                        # row i: unit vector i in the one Q head
    pos = torch.full((1, d), 5, dtype=torch.int32).cuda()
    col = torch.empty_like(eye, device="cuda")
    B.twist_rope_fwd(B.rope_args(B.BF16, 1, d, 1, 1, d, rot, layout=layout, in_=eye.cuda(), out=col, inv_freq=inv, pos=pos))
    R = host(col)[0, :, :d].T                                           # R[j, i] = d out_j / d in_i
    gen = torch.Generator().manual_seed(3)
    wgt = rng_bf16(gen, 1, 1, 3 * d)
    grad = torch.empty_like(wgt, device="cuda")
    B.twist_rope_bwd(B.rope_args(B.BF16, 1, 1, 1, 1, d, rot, layout=layout, in_=wgt.cuda(), out=grad, inv_freq=inv, pos=pos[:, :1].contiguous()))
    w = host(wgt)[0, 0, :d]
    want = R.T @ w
    # R's entries carry one bf16 rounding each, the result another
    assert np.all(np.abs(host(grad)[0, 0, :d] - want) <= U * np.abs(want) + (U + 2.0 ** -20) * (np.abs(R.T) @ np.abs(w)))


# ------------------------------------------------------------------------------------------------ append

def scattered_pages(gen, counts, page, spare=2):
    """Page table [n][most] over a shuffled pool; returns (table, pool size)."""
    need = [-(-c // page) for c in counts]
    pool = sum(need) + spare
    order = torch.randperm(pool, generator=gen)
    table = torch.zeros(len(counts), max(1, max(need)), dtype=torch.int32)
    at = 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k].to(torch.int32)
        at += k
    return table, pool


def append64(qkv, table, lens, new, first, H, KV, d, page, rot, layout, inv, held=None):
    """[(s, row, q, tol_q, [(page, slot, k, tol_k, v)])] of every new token."""
    S, n = lens.shape
    for s in range(S):
        for b in range(n):
            for i in range(new[s, b]):
                r = first[s, b] + i
                pos = lens[s, b] - new[s, b] + i
                z = qkv[s, r].reshape(H + 2 * KV, d)
                qk, tol = rotate64(z[:H + KV], np.array(pos), rot, layout, inv) if rot else (z[:H + KV], np.zeros((H + KV, d)))
                yield s, r, qk[:H], tol[:H], table[s, b, pos // page], pos % page, qk[H:], tol[H:], z[H + KV:]


APPEND = [
    # form, S, n_seqs, rows, past, H, KV, d, page, rot
    ("one", 1, 1, 1, 0, 1, 1, 8, 16, 8),
    ("one", 2, 5, 1, 63, 4, 2, 64, 16, 64),
    ("one", 3, 70, 1, 40, 2, 2, 16, 32, 8),
    ("padded", 2, 3, 37, 20, 3, 1, 32, 16, 32),
    ("padded", 1, 4, 130, 0, 6, 6, 64, 64, 64),
    ("packed", 2, 4, 50, 9, 4, 2, 128, 32, 64),
    ("packed", 3, 37, 11, 100, 2, 1, 64, 128, 0),       # no rotation
    ("packed", 1, 2, 700, 0, 8, 2, 64, 1024, 64),
    ("packed", 2, 3, 5, 3, 3, 2, 24, 16, 20),           # a head of odd size, rotated element by element
]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("form,S,n,rows,past,H,KV,d,page,rot", APPEND)
def test_append(B, form, S, n, rows, past, H, KV, d, page, rot, layout):
    gen = torch.Generator().manual_seed(rows * 13 + d)
    new = torch.randint(0, rows + 1, (S, n), generator=gen) if form != "one" else torch.ones(S, n, dtype=torch.int64)
    old = torch.randint(0, past + 1, (S, n), generator=gen)
    lens = (new + old).to(torch.int32)
    table, pool = scattered_pages(gen, lens.flatten().tolist(), page)
    table = table.view(S, n, -1)
    begin = torch.zeros(S, n + 1, dtype=torch.int32)
    begin[:, 1:] = torch.cumsum(new, 1)
    T = n if form == "one" else n * rows if form == "padded" else int(begin[:, -1].max()) + 3     # rows behind the last sequence
    first = begin[:, :-1] if form == "packed" else (torch.arange(n) * (T // n)).expand(S, n)
    w = (H + 2 * KV) * d
    qkv = rng_bf16(gen, S, T, w)
    inv = freqs(max(rot, 2))
    both = rng_bf16(gen, pool, 2, KV, page, d).cuda()                   # K and V of a page side by side: a strided cache
    before = both.clone()
    q_out = torch.full((S, T, H * d), 5.0, dtype=BF, device="cuda")
    dev = lambda t: t.contiguous().cuda()
    kw = dict(new_begin=dev(begin)) if form == "packed" else dict(new_len=dev(new.to(torch.int32))) if form == "padded" else {}
    args = lambda src, q: B.kv_append_args(
        B.BF16, S, n, T, H, KV, d, rot, layout, qkv=src, q_out=q, k_cache=both[:, 0], v_cache=both[:, 1],
        page_table=dev(table), kv_len=dev(lens), inv_freq=torch.from_numpy(inv).cuda()[:rot // 2] if rot else None, **kw)
    src = dev(qkv)
    B.twist_kv_append(args(src, q_out))
    torch.cuda.synchronize()
    assert B.twist_device_status() == 0
    got_q, got = host(q_out).reshape(S, T, H, d), host(both)
    ref = host(before)
    seen = np.zeros((S, T), dtype=bool)
    for s, r, q, tq, pg, slot, k, tk, v in append64(host(qkv), table.numpy(), lens.numpy(), new.numpy(), first.numpy(), H, KV, d,
                                                     page, rot, layout, inv[:rot // 2]):
        assert np.all(np.abs(got_q[s, r] - q) <= tq), (s, r)
        assert np.all(np.abs(got[pg, 0, :, slot] - k) <= tk), (s, r)
        assert np.array_equal(got[pg, 1, :, slot], v)
        seen[s, r] = True
        ref[pg, :, :, slot] = got[pg, :, :, slot]
    assert np.array_equal(got, ref)                                     # every other slot as it was
    assert np.all(got_q[~seen] == 5.0)                                  # rows of no sequence as they were
    # Q rotated in place gives the same bits and leaves K and V columns alone
    again = src.clone()
    B.twist_kv_append(args(again, again[..., :H * d]))
    mask = torch.from_numpy(seen).cuda()[..., None]
    assert torch.equal(again[..., :H * d], torch.where(mask, q_out, src[..., :H * d]))
    assert torch.equal(again[..., H * d:], src[..., H * d:])
    # without a place for Q the cache is the same
    one = both.clone()
    both.copy_(before)
    B.twist_kv_append(args(src, None))
    assert torch.equal(one, both)


def test_append_skips_positions_a_subnet_does_not_hold(B):
    S, n, H, KV, d, page = 3, 2, 2, 3, 16, 16
    gen = torch.Generator().manual_seed(0)
    qkv = rng_bf16(gen, S, n, (H + 2 * KV) * d).cuda()
    k = torch.full((S * n, KV, page, d), 3.0, dtype=BF, device="cuda")
    v = k.clone()
    held = torch.tensor([0, 2, 3], dtype=torch.int32).cuda()
    table = torch.arange(S * n, dtype=torch.int32).view(S, n, 1).cuda()
    lens = torch.ones(S, n, dtype=torch.int32).cuda()
    B.twist_kv_append(B.kv_append_args(B.BF16, S, n, n, H, KV, d, qkv=qkv, k_cache=k, v_cache=v, page_table=table, kv_len=lens, kv_count=held))
    z = qkv.view(S, n, H + 2 * KV, d)
    for s, c in enumerate(held.tolist()):
        for b in range(n):
            for cache, off in ((k, H), (v, H + KV)):
                page_ = cache[s * n + b]
                assert torch.equal(page_[:c, 0], z[s, b, off:off + c])
                assert bool((page_[c:] == 3.0).all()) and bool((page_[:, 1:] == 3.0).all())


def test_append_reports_bad_index_data_and_writes_nothing_for_it(B):
    S, n, H, KV, d, page = 1, 6, 1, 1, 32, 16
    gen = torch.Generator().manual_seed(0)
    qkv = rng_bf16(gen, S, n, 3 * d).cuda()
    k = torch.zeros(8, KV, page, d, dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    q = torch.full((S, n, d), 5.0, dtype=BF, device="cuda")
    table = torch.arange(6, dtype=torch.int32).view(S, n, 1)
    table[0, 1], table[0, 2] = 8, -1                                    # pages outside the pool
    lens = torch.tensor([[1, 1, 1, 17, 0, 16]], dtype=torch.int32)      # one beyond the table, one before its beginning
    B.twist_kv_append(B.kv_append_args(B.BF16, S, n, n, H, KV, d, qkv=qkv, q_out=q, k_cache=k, v_cache=v, page_table=table.cuda(), kv_len=lens.cuda()))
    torch.cuda.synchronize()
    assert B.twist_device_status() == B.ERR_BAD_INDEX and B.twist_device_status() == 0
    good = [0, 5]
    for b in range(n):
        assert torch.equal(q[0, b], qkv[0, b, :d] if b in good else torch.full_like(q[0, b], 5.0))
    want = torch.zeros_like(k)
    want[0, 0, 0], want[5, 0, 15] = qkv[0, 0, d:2 * d], qkv[0, 5, d:2 * d]
    assert torch.equal(k, want)
    # rows that contradict the layout
    for kw in (dict(new_begin=torch.tensor([[0, 2, 1, 3, 4, 5, 6]], dtype=torch.int32).cuda()),
               dict(new_begin=torch.tensor([[0, 1, 2, 3, 4, 5, 7]], dtype=torch.int32).cuda()),         # more rows than there are
               dict(new_begin=torch.tensor([[-1, 1, 2, 3, 4, 5, 6]], dtype=torch.int32).cuda()),
               dict(new_len=torch.tensor([[1, 1, 2, 1, 1, -1]], dtype=torch.int32).cuda())):
        lens6 = torch.ones(S, n, dtype=torch.int32).cuda()
        tab = torch.arange(6, dtype=torch.int32).view(S, n, 1).cuda()
        B.twist_kv_append(B.kv_append_args(B.BF16, S, n, n, H, KV, d, qkv=qkv, q_out=q, k_cache=k, v_cache=v, page_table=tab, kv_len=lens6, **kw))
        torch.cuda.synchronize()
        assert B.twist_device_status() == B.ERR_BAD_INDEX


# ------------------------------------------------------------------------------------------------ decode

class Case:
    def __init__(self, B, S, lens, H, gqa, d, page, seed=0, sharp=1.5, fill=None, interleaved=False, q_wide=False):
        gen = torch.Generator().manual_seed(seed + 17 * d + page)
        lens = torch.tensor(lens, dtype=torch.int32).view(S, -1)
        n = lens.shape[1]
        self.S, self.n, self.H, self.d, self.page = S, n, H, d, page
        if gqa is None:
            self.nh, self.nkv, self.kv_max = 0, 0, H
            self.of = np.tile(np.arange(H), (S, 1))
            self.extra = {}
        else:
            nh, nkv = gqa
            rng = np.random.default_rng(seed)
            idx = np.stack([np.sort(rng.choice(nh, H, replace=False)) for _ in range(S)]).astype(np.int32)
            kv_idx, kv_count = o.kv_groups(idx, nh, nkv)
            _, _, kv_pos = o.cover_and_pos(kv_idx, nkv, counts=kv_count)
            self.nh, self.nkv, self.kv_max = nh, nkv, min(nkv, H)
            self.of = np.stack([[kv_pos[s][h // (nh // nkv)] for h in idx[s]] for s in range(S)])
            self.extra = dict(head_idx=torch.from_numpy(idx).cuda(), kv_pos=torch.from_numpy(kv_pos.astype(np.int32)).cuda())
        table, pool = scattered_pages(gen, lens.flatten().tolist(), page)
        for i, m in enumerate(lens.flatten().tolist()):                  # entries that no key needs may hold anything
            table[i, -(-m // page):] = (1 << 24) if i % 2 else -7
        self.table, self.lens = table.view(S, n, -1), lens
        both = rng_bf16(gen, pool, 2, self.kv_max, page, d)
        if fill is not None:                                             # whatever the unused slots hold must not matter
            used = torch.zeros(pool, page, dtype=torch.bool)
            for i, m in enumerate(lens.flatten().tolist()):
                for k in range(-(-m // page)):
                    used[table[i, k], :min(page, m - k * page)] = True
            both = torch.where(used[:, None, None, :, None], both, torch.tensor(fill, dtype=BF))
        self.q = (torch.randn(S, n, H, d, generator=gen) * torch.rand(S, n, H, 1, generator=gen) * 2 * sharp).to(BF).view(S, n, H * d)
        self.pool = both.cuda()
        self.k, self.v = (self.pool[:, 0], self.pool[:, 1]) if interleaved else (self.pool[:, 0].contiguous(), self.pool[:, 1].contiguous())
        wide = torch.full((S, n, (H + 3) * d), 7.0, dtype=BF)
        wide[..., :H * d] = self.q
        self.dq = wide.cuda()[..., :H * d] if q_wide else self.q.cuda()
        self.out = torch.full((S, n, H * d), 9.0, dtype=BF, device="cuda")
        self.lse = torch.full((S, H, n), 9.0, dtype=torch.float32, device="cuda")
        self.ws = torch.empty(B.twist_attn_decode_workspace_bytes(d), dtype=torch.uint8, device="cuda").fill_(0xFF)
        self.dtable, self.dlens = self.table.contiguous().cuda(), lens.cuda()

    def args(self, B, **kw):
        f = dict(q=self.dq, k_cache=self.k, v_cache=self.v, page_table=self.dtable, kv_len=self.dlens, out=self.out, lse=self.lse,
                 ws=self.ws, **self.extra)
        f.update(kw)
        return B.attn_decode_args(B.BF16, self.S, self.n, self.H, self.kv_max, self.d, self.nh, self.nkv, **f)

    def check(self, out=None, lse=None):
        out, lse = host(self.out if out is None else out), host(self.lse if lse is None else lse)
        K, V, q = host(self.k), host(self.v), host(self.q).reshape(self.S, self.n, self.H, self.d)
        d = self.d
        for s in range(self.S):
            for b in range(self.n):
                m = int(self.lens[s, b])
                if m == 0:
                    assert np.all(out[s, b] == 0) and np.all(lse[s, :, b] == -np.inf)
                    continue
                pages = self.table[s, b, :-(-m // self.page)].numpy()
                k = K[pages].transpose(1, 0, 2, 3).reshape(self.kv_max, -1, d)[:, :m]
                v = V[pages].transpose(1, 0, 2, 3).reshape(self.kv_max, -1, d)[:, :m]
                for h in range(self.H):
                    g = self.of[s][h]
                    sc = k[g] @ q[s, b, h] / np.sqrt(d)
                    e_s = (d + 2) * 2.0 ** -23 * np.max(np.abs(k[g]) @ np.abs(q[s, b, h])) / np.sqrt(d)
                    top = sc.max()
                    p = np.exp(sc - top)
                    p, total = p / p.sum(), p.sum()
                    want = p @ v[g]
                    tol = U * np.abs(want) + (2 * e_s + 2.0 ** -20 + 2.0 ** -16 + 2 * m * 2.0 ** -23) * (p @ np.abs(v[g]))
                    got = out[s, b, h * d:(h + 1) * d]
                    assert np.all(np.abs(got - want) <= tol), (s, b, h, m, float(np.max(np.abs(got - want) / tol)))
                    wl = top + np.log(total)
                    assert abs(lse[s, h, b] - wl) <= e_s + 2.0 ** -20 + m * 2.0 ** -23 + 2.0 ** -22 * abs(wl), (s, b, h, m)


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129]
DECODE = [
    # S, lens, H, (NH, NKV), d, page
    (1, EDGES, 1, None, 8, 16),
    (2, EDGES, 2, None, 16, 32),
    (1, EDGES, 3, None, 32, 16),
    (2, EDGES, 3, None, 64, 64),
    (1, EDGES, 2, None, 128, 128),
    (1, [0, 0, 0], 2, None, 64, 16),                    # nothing cached anywhere
    (1, [700], 4, None, 128, 16),                       # a single sequence, split
    (2, [5000, 3, 0, 1300], 4, (8, 2), 64, 32),         # ragged, split, shared keys
    (3, [1, 900, 0, 20, 77, 2000], 5, (8, 4), 16, 16),
    (1, [2500, 600], 12, (12, 1), 64, 64),              # twelve heads on one KV position: two passes over its keys
    (2, [640, 1025], 20, (24, 1), 32, 16),
    (2, [1500, 1], 7, (32, 4), 128, 1024),              # one page holds most of a sequence
    (4, [int(x) for x in np.random.default_rng(3).integers(0, 600, 4 * 60)], 6, (12, 4), 64, 16),      # a big ragged batch
    (1, [40000], 2, (4, 2), 8, 256),
    (1, [9000, 8999], 2, None, 32, 16),
    # sharing by up to twelve heads: positions with one and with two passes over their keys, few items and many
    (2, [900, 0, 3000, 17], 10, (48, 4), 64, 32),
    (1, [5000], 13, (48, 4), 16, 16),
    (1, [2600, 31], 9, (36, 3), 128, 16),
    (4, [int(x) for x in np.random.default_rng(4).integers(0, 900, 4 * 120)], 10, (48, 4), 32, 16),
    (8, [int(x) for x in np.random.default_rng(5).integers(0, 1500, 8 * 3)], 70, (96, 8), 16, 16),     # more heads than the kernel caches
    (1, [int(x) for x in np.random.default_rng(6).integers(0, 40, 700)], 4, (8, 2), 64, 16),           # more sequences than it caches
    # one cluster of CTAs per item: 2, 4 and 8 of them, lengths that leave some without keys
    (1, [300, 5, 0], 2, None, 64, 16), (1, [1000, 40], 4, (8, 2), 64, 64), (1, [513], 1, None, 128, 16), (2, [700, 64], 3, (4, 2), 32, 32),
    (1, [1500], 5, (24, 2), 16, 16), (1, [900], 2, None, 8, 16),
]


@pytest.mark.parametrize("case", range(len(DECODE)))
def test_decode(B, case):
    S, lens, H, gqa, d, page = DECODE[case]
    if len(lens) % S:
        lens = (lens * S)[:S * len(lens)]
    if gqa is None and S > 1 and lens is EDGES:
        lens = EDGES * S
    c = Case(B, S, lens, H, gqa, d, page, seed=case, fill=float("nan"), interleaved=case % 2 == 0, q_wide=case % 3 == 0)
    B.twist_attn_decode(c.args(B))
    torch.cuda.synchronize()
    assert B.twist_device_status() == 0
    c.check()
    # the caller's bound on the lengths only chooses the split: both ways are right, and each repeats its own bits
    out, lse = c.out.clone(), c.lse.clone()
    for bound in (1, 1 << 30, 0):
        for _ in range(2):
            c.out.fill_(9.0)
            B.twist_attn_decode(c.args(B, max_len=bound))
            c.check()
    assert torch.equal(c.out, out) and torch.equal(c.lse, lse)
    # the log-sum-exp is optional
    c.out.fill_(9.0)
    B.twist_attn_decode(c.args(B, lse=None))
    assert torch.equal(c.out, out)


@pytest.mark.parametrize("fill", [float("inf"), float("-inf"), torch.finfo(BF).min, torch.finfo(BF).max])
def test_decode_ignores_what_unused_slots_hold(B, fill):
    c = Case(B, 1, [33, 0, 700, 1], 4, (8, 2), 64, 32, fill=fill)
    for bound in (1, 0):
        B.twist_attn_decode(c.args(B, max_len=bound))
        c.check()


def test_decode_scores_that_grow_along_the_sequence(B):
    """The running reference maximum has to move many times; the largest scores are far beyond exp's range in fp32."""
    c = Case(B, 1, [3000, 513], 2, None, 64, 16, sharp=3.0)
    ramp = (torch.arange(c.k.shape[0] * c.page) % 97).view(c.k.shape[0], 1, c.page, 1).float().cuda() / 8
    c.k = (c.k.float() * ramp).to(BF)
    for bound in (1, 0):
        B.twist_attn_decode(c.args(B, max_len=bound))
        c.check()


def test_decode_non_finite_values_behave_as_the_formula(B):
    """An infinite key score takes all the weight of nothing finite: NaN as in the formula; keys whose score is -inf count
    for nothing; a NaN in V reaches its own element only."""
    c = Case(B, 1, [40, 40, 40], 1, None, 64, 16)
    q = torch.zeros(64)
    q[0] = 1.0
    c.q = q.to(BF).view(1, 1, 64).expand(1, 3, 64).contiguous()
    c.dq = c.q.cuda()
    for b, val in ((0, float("-inf")), (1, float("inf"))):
        c.k[c.table[0, b, 1].item(), 0, 3, 0] = val                      # key 19 of sequence b
    c.v[c.table[0, 2, 0].item(), 0, 5, 7] = float("nan")
    for bound in (1, 0):
        B.twist_attn_decode(c.args(B, max_len=bound))
        out = host(c.out)[0]
        assert np.all(np.isfinite(out[0])) and np.all(np.isnan(out[1]))
        assert np.isnan(out[2, 7]) and np.all(np.isfinite(np.delete(out[2], 7)))
        pages = c.table[0, 0].numpy()
        k, v = host(c.k)[pages, 0].reshape(-1, 64)[:40], host(c.v)[pages, 0].reshape(-1, 64)[:40]
        keep = np.arange(40) != 19
        p = np.exp(k[keep, 0] / 8)
        want = (p / p.sum()) @ v[keep]
        assert np.all(np.abs(out[0] - want) <= U * np.abs(want) + 2.0 ** -15 * np.abs(v[keep]).max())


def test_decode_reports_bad_index_data(B):
    c = Case(B, 1, [40, 40], 4, (8, 2), 32, 16)
    good = c.args(B)
    B.twist_attn_decode(good)
    assert B.twist_device_status() == 0
    want = c.out.clone()
    table = c.dtable.clone()
    table[0, 1, 1] = c.k.shape[0]                                        # a page outside the pool is read as page 0
    B.twist_attn_decode(c.args(B, page_table=table))
    assert B.twist_device_status() == B.ERR_BAD_INDEX
    assert torch.equal(c.out[0, 0], want[0, 0])
    table[0, 1, 1] = 0
    got = c.out.clone()
    B.twist_attn_decode(c.args(B, page_table=table))
    assert B.twist_device_status() == 0 and torch.equal(got, c.out)
    for bad in (-1, 49):                                                 # lengths outside the table (3 pages of 16) are clamped
        lens = c.dlens.clone()
        lens[0, 1] = bad
        B.twist_attn_decode(c.args(B, kv_len=lens))
        assert B.twist_device_status() == B.ERR_BAD_INDEX
        assert torch.equal(c.out[0, 0], want[0, 0])
        if bad < 0:
            assert bool((c.out[0, 1] == 0).all())
    heads = c.extra["head_idx"].clone()
    heads[0, 3] = 64                                                     # a head that does not exist reads position 0
    B.twist_attn_decode(c.args(B, head_idx=heads))
    assert B.twist_device_status() == B.ERR_BAD_INDEX


def test_decode_more_heads_than_a_group_has_are_reported(B):
    """Kept heads are distinct; a list that repeats one more often than a group has heads is reported."""
    c = Case(B, 1, [40], 12, (12, 12), 32, 16)
    heads = torch.zeros(1, 12, dtype=torch.int32, device="cuda")
    B.twist_attn_decode(c.args(B, head_idx=heads))
    assert B.twist_device_status() == B.ERR_BAD_INDEX
    assert bool((c.out.view(12, 32)[8:] == 9.0).all())                   # beyond one row tile: left as they were


def test_decode_cache_beyond_32_bit_offsets(B):
    """Pages more than 2^31 elements into the pool."""
    d, page, kv = 64, 64, 2
    stride = (1 << 30) + 8 * 123                                          # elements between pages
    flat = torch.zeros(3 * stride, dtype=BF, device="cuda")               # 6.4 GB
    k = torch.as_strided(flat, (3, kv, page, d), (stride, page * d, d, 1), 0)
    v = torch.as_strided(flat, (3, kv, page, d), (stride, page * d, d, 1), kv * page * d)
    c = Case(B, 1, [190], 2, None, d, page)
    order = torch.tensor([2, 0, 1])
    for j in range(3):
        k[order[j]] = c.k[c.table[0, 0, j].item()]
        v[order[j]] = c.v[c.table[0, 0, j].item()]
    table = order.to(torch.int32).view(1, 1, 3).cuda()
    for bound in (1, 1 << 20):
        B.twist_attn_decode(c.args(B, k_cache=k, v_cache=v, page_table=table, max_len=bound))
        c.check()
    # and appending there
    qkv = rng_bf16(torch.Generator().manual_seed(1), 1, 1, 6 * d).cuda()
    lens = torch.full((1, 1), 3, dtype=torch.int32).cuda()
    B.twist_kv_append(B.kv_append_args(B.BF16, 1, 1, 1, 2, kv, d, qkv=qkv, k_cache=k, v_cache=v, page_table=table, kv_len=lens))
    assert torch.equal(k[2, :, 2].reshape(-1), qkv[0, 0, 2 * d:4 * d]) and torch.equal(v[2, :, 2].reshape(-1), qkv[0, 0, 4 * d:])


def test_decode_long_cache_split_over_the_whole_gpu(B):
    c = Case(B, 1, [70001], 2, (4, 2), 128, 64)
    B.twist_attn_decode(c.args(B))
    c.check()


def test_append_and_decode_in_a_captured_graph_replay_with_new_lengths(B):
    """One decoding step captured once and replayed: lengths and projected rows change between replays, the graph does not."""
    S, n, H, KV, d, page, pages = 2, 3, 4, 2, 64, 16, 40
    gen = torch.Generator().manual_seed(4)
    nh, nkv = 8, 2
    head_idx = torch.tensor([[0, 1, 4, 7], [2, 3, 5, 6]], dtype=torch.int32).cuda()
    kv_pos = torch.tensor([[0, 1], [0, 1]], dtype=torch.int32).cuda()
    of = np.array([[0, 0, 1, 1], [0, 0, 1, 1]])
    table = torch.randperm(S * n * pages, generator=gen).to(torch.int32).view(S, n, pages).cuda()
    k = torch.full((S * n * pages, KV, page, d), float("nan"), dtype=BF, device="cuda")
    v = k.clone()
    lens = torch.zeros(S, n, dtype=torch.int32, device="cuda")
    given = torch.zeros(S, n, (H + 2 * KV) * d, dtype=BF, device="cuda")
    qkv = torch.zeros_like(given)
    out = torch.zeros(S, n, H * d, dtype=BF, device="cuda")
    lse = torch.zeros(S, H, n, device="cuda")
    ws = torch.empty(B.twist_attn_decode_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    inv = freqs(d)
    dinv = torch.from_numpy(inv).cuda()
    q = qkv[..., :H * d]

    def step():
        qkv.copy_(given)                                                  # (a copy and a fill beside the kernels of the graph)
        out.zero_()
        B.twist_kv_append(B.kv_append_args(B.BF16, S, n, n, H, KV, d, d, qkv=qkv, q_out=q, k_cache=k, v_cache=v, page_table=table,
                                           kv_len=lens, inv_freq=dinv))
        B.twist_attn_decode(B.attn_decode_args(B.BF16, S, n, H, KV, d, nh, nkv, q=q, k_cache=k, v_cache=v, page_table=table, kv_len=lens,
                                               head_idx=head_idx, kv_pos=kv_pos, out=out, lse=lse, ws=ws))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lens.fill_(1)
        step()                                                            # warm-up outside the capture
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rows = rng_bf16(gen, 30, S, n, (H + 2 * KV) * d)
    k.fill_(float("nan"))
    v.fill_(float("nan"))
    z = host(rows).reshape(30, S, n, H + 2 * KV, d)
    rk, _ = rotate64(z[:, :, :, H:H + KV], np.broadcast_to(np.arange(30)[:, None, None], (30, S, n)), d, 0, inv)
    rk = torch.from_numpy(rk).to(BF).to(torch.float64).numpy()            # as the cache stores it
    for i in range(30):
        given.copy_(rows[i])
        lens.fill_(i + 1)
        graph.replay()
        torch.cuda.synchronize()
        if i not in (0, 1, 16, 29):
            continue
        rq, _ = rotate64(z[i][:, :, :H], np.full((S, n), i), d, 0, inv)
        got = host(out).reshape(S, n, H, d)
        for s in range(S):
            for b in range(n):
                for h in range(H):
                    g = of[s][h]
                    x = rk[:i + 1, s, b, g] @ rq[s, b, h] / np.sqrt(d)
                    p = np.exp(x - x.max())
                    p /= p.sum()
                    vv = z[:i + 1, s, b, H + KV + g]
                    want = p @ vv
                    # query and keys carry one bf16 rounding each: a score is off by 2 u sum|q k| / sqrt(d), its weight by that
                    # relative to itself, and the softmax by twice it; a rounded key may fall to the other side of a tie
                    e = 4 * U * np.max(np.abs(rk[:i + 1, s, b, g]) @ np.abs(rq[s, b, h])) / np.sqrt(d)
                    assert np.all(np.abs(got[s, b, h] - want) <= U * np.abs(want) + (2 * e + 2.0 ** -14) * (p @ np.abs(vv))), (i, s, b, h)
    assert B.twist_device_status() == 0


def test_calls_on_two_streams_at_once(B):
    """Two overlapping calls, each with scratch of its own, give what each gives alone."""
    cases = [Case(B, 1, [6000, 40], 4, (8, 4), 64, 16, seed=s) for s in (1, 2)]
    want = []
    for c in cases:
        B.twist_attn_decode(c.args(B))
        want.append((c.out.clone(), c.lse.clone()))
        c.out.fill_(9.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(20):
        for c, st in zip(cases, streams):
            with torch.cuda.stream(st):
                B.twist_attn_decode(c.args(B))
    torch.cuda.synchronize()
    for c, (out, lse) in zip(cases, want):
        assert torch.equal(c.out, out) and torch.equal(c.lse, lse)


def test_tensors_that_do_not_fit_the_call_are_refused(B):
    c = Case(B, 1, [40, 9], 4, (8, 2), 32, 16)
    for kw in (dict(kv_len=c.dlens.long()), dict(kv_len=c.dlens[:, :1].contiguous()), dict(page_table=c.dtable.cpu()),
               dict(lse=c.lse.double()), dict(lse=c.lse[:, :3].contiguous()), dict(head_idx=c.extra["head_idx"].long()),
               dict(kv_pos=c.extra["kv_pos"][:, :1].contiguous()), dict(out=c.out.float()), dict(q=c.dq.cpu()), dict(ws=c.ws.cpu()),
               dict(k_cache=c.k[:, :1]), dict(v_cache=c.v.float()), dict(q=c.dq[..., ::2])):
        with pytest.raises(ValueError):
            c.args(B, **kw)
    with pytest.raises(B.TwistError):
        B.twist_attn_decode(c.args(B, ws=c.ws[:64]))
    x = torch.zeros(1, 4, 96, dtype=BF, device="cuda")
    inv = torch.ones(16, dtype=torch.float64, device="cuda")
    good = dict(in_=x, out=x, inv_freq=inv)
    B.twist_rope_fwd(B.rope_args(B.BF16, 1, 4, 1, 1, 32, 32, 4, **good))
    for kw in (dict(in_=x.float()), dict(out=x[:, :2]), dict(inv_freq=inv.float()), dict(inv_freq=inv[:8]), dict(in_=x.cpu()),
               dict(pos=torch.zeros(1, 4, device="cuda"))):
        with pytest.raises(ValueError):
            B.rope_args(B.BF16, 1, 4, 1, 1, 32, 32, 4, **dict(good, **kw))
    k = torch.zeros(2, 1, 16, 32, dtype=BF, device="cuda")
    good = dict(qkv=x, k_cache=k, v_cache=k.clone(), page_table=torch.zeros(1, 4, 1, dtype=torch.int32, device="cuda"),
                kv_len=torch.ones(1, 4, dtype=torch.int32, device="cuda"), inv_freq=inv)
    B.kv_append_args(B.BF16, 1, 4, 4, 1, 1, 32, 32, **good)
    for kw in (dict(qkv=x[..., :64]), dict(q_out=x[..., :33]), dict(new_len=torch.ones(1, 3, dtype=torch.int32, device="cuda")),
               dict(new_begin=torch.ones(1, 4, dtype=torch.int32, device="cuda")), dict(kv_count=torch.ones(2, dtype=torch.int32, device="cuda")),
               dict(kv_len=good["kv_len"].cpu())):
        with pytest.raises(ValueError):
            B.kv_append_args(B.BF16, 1, 4, 4, 1, 1, 32, 32, **dict(good, **kw))
