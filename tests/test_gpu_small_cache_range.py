"""The 8-bit decode over its whole range: sums that are large in units of a block whose values are all zero, scales at both ends of fp32,
probabilities far below the largest, and keys whose scale is large beside products that are zero.

Tolerance of a result (the definition in 64 bits, p = exp(s - max), l = sum p, mass = sum p |v| / l):
 * its own rounding to bf16: half a step is 2^-8 of it, and 2^-134 where it is subnormal;
 * a score's error e_s = (d + 4) 2^-23 sum|q k| / sqrt(d) and 2^-20 for the exponential are relative errors of p, once in the sum and once in l;
 * a probability as fp16: half a step is 2^-11 of it, or, below fp16's normal numbers, 2^-25 of numbers scaled so that the largest p * scale so
   far is 2^13 at least: 2^-38 of max(p * scale) for every key, times its number, at most 448;
 * probabilities, and factors of parts that are joined, below 2^-126 are zero: 2^-126 |v| of every key, twice;
 * sums over n keys in fp32, 2 n 2^-23, and 2^-16 for sums brought to other units (an exponent of up to 2^7, 2^-24 of it, a few times)."""
import math

import numpy as np
import pytest
import torch

from test_gpu_small_cache import BF, BLOCK, F8, code, f64, host, i32, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


# (sequences, keys of the longest): one launch for all of an item, or the line cut into pieces (many keys of one item to a warp)
WAYS = {"whole": (3, 900), "split": (12, 6000)}


def cache_of(k, v, ks, vs, page):
    """Dense sequences of numbers k, v [n][KV][m][D] and scales [n][KV][m / 16] as pages: (k, v, scales, table)."""
    n, KV, m, D = k.shape
    per = -(-m // page)
    fill = lambda x, to, value: np.concatenate([x, np.full((*x.shape[:2], to - x.shape[2], *x.shape[3:]), value)], 2)
    pages = lambda x: torch.from_numpy(fill(x, per * page, 0.0).reshape(n, KV, per, page, D).transpose(0, 2, 1, 3, 4).reshape(n * per, KV, page, D)
                                       .astype(np.float32, order="C")).to(F8).cuda()
    sc = np.stack([fill(s, per * page // BLOCK, 1.0).reshape(n, KV, per, page // BLOCK).transpose(0, 2, 1, 3).reshape(n * per, KV, -1)
                   for s in (ks, vs)], -1)
    return pages(k), pages(v), torch.from_numpy(sc.astype(np.float32, order="C")).cuda(), np.arange(n * per).reshape(n, per)


def run(B, q, k, v, ks, vs, lens, page=64):
    """Decode with two heads on each KV position: (out [n][H][D], lse [H][n], q, K, V, weights), in 64 bits."""
    n, KV, m, D = k.shape
    H = 2 * KV
    dk, dv, scales, table = cache_of(k, v, ks, vs, page)
    ws = torch.empty(B.twist_attn_decode_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(1, n, H * D, dtype=BF, device="cuda"), torch.empty(1, H, n, device="cuda")
    heads = dict(head_idx=i32([list(range(H))]), kv_pos=i32([list(range(KV))]))
    cache = dict(k_cache=dk, scales=scales, page_table=i32([table.tolist()]), kv_len=i32([lens]))
    dq = torch.from_numpy(q).to(BF).cuda().view(1, n, H * D)
    B.twist_attn_decode_q8(B.attn_decode_q8_args(B.BF16, 1, n, H, KV, D, H, KV, q=dq, v_cache=dv, out=out, lse=lse, ws=ws, **cache, **heads))
    assert B.twist_device_status() == 0
    weights = torch.zeros(*dk.shape[:3], device="cuda")
    B.twist_attn_weights(B.attn_weights_args(B.BF16, 1, n, H, KV, D, H, KV, q=dq, lse=lse, weights=weights, **cache, **heads))
    assert B.twist_device_status() == 0
    full = lambda x, s: x * np.repeat(s, BLOCK, 2)[:, :, :m, None]
    w = host(weights).reshape(n, -1, KV, page).transpose(0, 2, 1, 3).reshape(n, KV, -1)
    return host(out).reshape(n, H, D), host(lse)[0], host(dq).reshape(n, H, D), full(k, ks), full(v, vs), w


def check(got, lse, q, k, v, weights, lens, vs):
    n, H, D = got.shape
    worst = 0.0
    for b in range(n):
        m = lens[b]
        for h in range(H):
            kk, vv = k[b, h // 2, :m], v[b, h // 2, :m]
            x = kk @ q[b, h] / math.sqrt(D)
            e = ((D + 4) * 2.0 ** -23 * (np.abs(kk) @ np.abs(q[b, h])) / math.sqrt(D)).max()
            p = np.exp(x - x.max())
            l = p.sum()
            want, mass = p @ vv / l, p @ np.abs(vv) / l
            scale = np.repeat(vs[b, h // 2], BLOCK)[:m]
            tiny = m * 2.0 ** -38 * (p * scale).max() * 448 / l + 2.0 ** -125 * np.abs(vv).sum(0) / l
            tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -134 + (2 * e + 2.0 ** -20 + 2.0 ** -11 + 2.0 ** -16 + 2 * m * 2.0 ** -23) * mass + tiny
            assert np.all(np.isfinite(got[b, h])), (b, h)
            worst = max(worst, np.max(np.abs(got[b, h] - want) / tol))
            assert worst <= 1, (b, h, worst)
            assert abs(lse[h, b] - (x.max() + np.log(l))) <= e + 2.0 ** -20 + m * 2.0 ** -23 + 2.0 ** -22 * abs(x.max() + np.log(l))
        for g in range(H // 2):                     # the weights of the same step: every term within e + 2^-22 |s - lse| + 2^-21 of itself
            terms = []
            for h in (2 * g, 2 * g + 1):
                x = k[b, g, :m] @ q[b, h] / math.sqrt(D)
                e = (D + 4) * 2.0 ** -23 * (np.abs(k[b, g, :m]) @ np.abs(q[b, h])) / math.sqrt(D)
                d = x - lse[h, b]
                terms.append((np.exp(d), np.exp(d) * (e + 2.0 ** -22 * np.abs(d) + 2.0 ** -21)))
            w = terms[0][0] + terms[1][0]
            assert np.all(np.abs(weights[b, g, :m] - w) <= terms[0][1] + terms[1][1] + 3 * 2.0 ** -24 * w + 2 * 2.0 ** -126)   # (a term below 2^-126 is 0)


def case(rng, way, D, KV=2):
    n, m = WAYS[way]
    lens = [m - int(rng.integers(0, m // 3)) for _ in range(n)]
    k = code(rng.standard_normal((n, KV, m, D)) * 60, 1.0)
    v = code(rng.standard_normal((n, KV, m, D)) * 100, 1.0)
    q = rng.standard_normal((n, 2 * KV, D))
    blocks = -(-m // BLOCK)
    return n, m, lens, q, k, v, np.full((n, KV, blocks), 2.0 ** -7), np.full((n, KV, blocks), 2.0 ** -8)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("scale", [-9, 0, 4, 60])
@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_blocks_of_zeros_between_values_of_any_size(B, D, scale, way):
    """Tokens without values (their scale is 2^-110) behind long runs of values of one sign, the scores of one position rising by nearly
    2^8 behind its first keys."""
    rng = np.random.default_rng(D + scale)
    n, m, lens, q, k, v, ks, vs = case(rng, way, D)
    v = np.abs(v) * 2
    v = code(v, 1.0)
    vs[:] = 2.0 ** scale
    zero = rng.random(vs.shape) < 0.05
    zero[:, :, 20] = True
    vs[zero] = 2.0 ** -110
    v[np.repeat(zero, BLOCK, 2)[:, :, :m]] = 0
    k[:, 0] = 0                                      # position 0: scores 0, then 7.9 in powers of two, exactly the same for all keys
    k[:, 0, 64:, 0] = 1
    ks[:, 0] = 1
    q[:, :2, 0] = 7.9 * math.log(2) * math.sqrt(D)
    check(*run(B, q, k, v, ks, vs, lens), lens, vs)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_scales_at_both_ends(B, D, way):
    """Blocks a hundred powers of two apart in both orders, and the smallest and largest scales there are."""
    rng = np.random.default_rng(D)
    n, m, lens, q, k, v, ks, vs = case(rng, way, D)
    vs[:] = 2.0 ** rng.choice([-126.0, -110.0, -100.0, -50.0, 0.0, 50.0, 78.0], vs.shape)
    vs[0] = 2.0 ** -126                              # a sequence of the smallest alone, one of them and zeros, one without extremes
    vs[1] = np.where(rng.random(vs[1].shape) < 0.5, 2.0 ** -126, 2.0 ** -100)
    vs[2] = np.where(np.arange(vs.shape[2]) % 2 == 0, 2.0 ** 60, 2.0 ** -60)
    v[2][:, np.repeat(np.arange(vs.shape[2]) % 2 == 0, BLOCK)[:m]] = 0           # large scales over nothing
    check(*run(B, q, k, v, ks, vs, lens), lens, vs)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("below", [18.3, 20.3, 21.2, 24.0, 27.7])
@pytest.mark.parametrize("D", [16, 64, 128])
def test_probabilities_far_below_the_largest(B, D, below, way):
    """In every 256 keys one takes nearly all of the weight and has next to no value: the result is what the others give.  The heavy
    key's block has a smaller scale (position 0) or the others' (position 1)."""
    rng = np.random.default_rng(int(10 * below) + D)
    n, m, lens, q, k, v, ks, vs = case(rng, way, D)
    heavy = np.arange(m) % 256 == 5
    k[:] = 0
    k[:, :, heavy, 0] = 256
    ks[:] = 2.0 ** -8
    q[:, :, 0] = below * math.log(2) * math.sqrt(D)
    v = code(np.abs(rng.standard_normal(v.shape)) * 20 + 100, 1.0)
    v[:, :, heavy] = 0
    blocks = np.arange(vs.shape[2]) % 16 == 0
    vs[:] = 0.7
    vs[:, 0, blocks] = 2.0 ** -40
    check(*run(B, q, k, v, ks, vs, lens), lens, vs)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("D", [16, 64, 128])
def test_scores_that_are_zero_beside_a_large_scale(B, D, way):
    """Keys of zeros in blocks whose scale times the queries' size is beyond fp32: their scores are zero."""
    rng = np.random.default_rng(D)
    n, m, lens, q, k, v, ks, vs = case(rng, way, D)
    ks[:] = 2.0 ** -50
    big = rng.random(ks.shape) < 0.3
    ks[big] = 2.0 ** 119
    k[np.repeat(big, BLOCK, 2)[:, :, :m]] = 0
    q *= 2.0 ** 42
    check(*run(B, q, k, v, ks, vs, lens), lens, vs)
