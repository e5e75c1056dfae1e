"""Decoding sessions whose cache is held in 8 bits or bounded by eviction: what a step's attention computes, which tokens are kept,
and that both leave a session's other results as they are.

Tolerances: the attention's output against softmax(q k / sqrt(d)) v over the cache's own values in 64 bits as for the decode call
(bf16 rounding 2^-8, fp16 probabilities 2^-12, scores (d + 4) 2^-23 sum|q k| / sqrt(d)); weights as for the weight calls (2^-20
for what the log-sum-exp, itself within 2^-20, and the exponential add to that)."""
import math
from dataclasses import replace

import numpy as np
import pytest
import torch

from paper_2511_03983_b200 import inputs as I

pytestmark = pytest.mark.gpu

MATS = {"gate": I.MAT_GATE, "up": I.MAT_UP, "down": I.MAT_DOWN, "qkv": I.MAT_QKV, "o": I.MAT_O}


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


def make(layers=1, n_seqs=2, seq_len=24, d_head=64, cfg=3, **extra):
    from paper_2511_03983_b200.engine import StackEngine
    w = replace(I.scaled_twin(I.PRESETS[cfg], d_model=256, d_ff=512, d_head=d_head, tokens=n_seqs * seq_len, n_layers=layers, local_steps=1),
                **dict(dict(rope_base=10000.0), **extra))
    eng = StackEngine(w, n_seqs, seq_len)
    for l in range(w.n_layers):
        for m in eng.full:                                        # larger projections than at the start of training: sharper scores
            x = I.weight(w, l, MATS[m]) * (8.0 if m == "qkv" else 1.0)
            eng.full[m][l].copy_(torch.from_numpy(x).to(torch.bfloat16))
    eng.X.append(torch.from_numpy(np.stack([I.normal(11, s, (w.tokens, w.d_model), 1.0, I.DTYPE_BF16) for s in range(w.n_subnets)])).to(torch.bfloat16).cuda())
    eng.extract(0)
    return eng


def tokens(eng, count, seed=21):
    w = eng.w
    x = np.stack([I.normal(seed, s, (count, eng.n_seqs, w.d_model), 1.0, I.DTYPE_BF16) for s in range(w.n_subnets)])
    return torch.from_numpy(x).to(torch.bfloat16).cuda()          # [S][count][n_seqs][d]


def rows(ses, l, s, b, which):
    """[kv_max][len][d_head] of a sequence in 64 bits."""
    x = ses.pools[l][:, which].float().double()
    if ses.cache_bits == 8:
        x = x * ses.scales[l][..., which].double().repeat_interleave(16, -1)[..., None]
    return torch.cat([x[p] for p in ses.pages[s][b]], 1)[:, :ses.lens[s][b]].cpu().numpy()


def paged(ses, t, s, b):
    return torch.cat([t[p] for p in ses.pages[s][b]], 1)[:, :ses.lens[s][b]].cpu().numpy()


def held(eng, l, s):
    return int(eng.kv_count[l][s])


def check_attention(eng, ses, l=0):
    """The last layer's attention of the last step against the cache as it is; returns the probabilities by (s, b, position)."""
    w = eng.w
    kind = eng.kind_of(l)
    q, out = ses.qkv[kind], ses.a[kind].double().cpu().numpy()
    per = w.n_heads // w.n_kv_heads
    given = {}
    for s in range(w.n_subnets):
        heads = eng.idx_head[l][s].tolist()
        pos = [int(eng.kv_pos[l][s][h // per]) if eng.gqa else i for i, h in enumerate(heads)]
        for b in range(eng.n_seqs):
            k, v = rows(ses, l, s, b, 0), rows(ses, l, s, b, 1)
            x = q[s, b, :eng.a_sub].double().cpu().numpy().reshape(-1, w.d_head)
            for i, p in enumerate(pos):
                y = k[p] @ x[i] / math.sqrt(w.d_head)
                e = ((w.d_head + 4) * 2.0 ** -23 * (np.abs(k[p]) @ np.abs(x[i])) / math.sqrt(w.d_head)).max()
                pr = np.exp(y - y.max())
                pr /= pr.sum()
                want = pr @ v[p]
                tol = 2.0 ** -8 * np.abs(want) + (2 * e + 2.0 ** -11) * (pr @ np.abs(v[p])) + 2.0 ** -21 * np.abs(v[p]).sum(0)
                got = out[s, b].reshape(-1, w.d_head)[i]
                assert np.all(np.abs(got - want) <= tol), (s, b, i)
                sums, err = given.setdefault((s, b, p), [np.zeros(len(pr)), np.zeros(len(pr))])
                sums += pr
                err += pr * (2 * e + 2.0 ** -20)
    return given


@pytest.mark.parametrize("cfg,d_head", [(3, 64), (3, 16), (2, 32), (4, 128)])
def test_an_8_bit_session_attends_over_what_it_holds(B, cfg, d_head):
    from paper_2511_03983_b200.engine import DecodeSession
    eng = make(cfg=cfg, d_head=d_head)
    full, small = DecodeSession(eng, max_len=40), DecodeSession(eng, max_len=40, cache_bits=8)
    lengths = [[24, 7]] * eng.w.n_subnets
    full.prefill(0, lengths)
    small.prefill(0, lengths)
    x = tokens(eng, 6)
    for i in range(6):
        full.step(x[:, i])
        small.step(x[:, i])
        check_attention(eng, small)
    assert B.twist_device_status() == 0
    for s in range(eng.w.n_subnets):                               # half a step of e4m3, and of the scale's smallest number
        for b in range(2):
            for j in (0, 1):
                a, c = rows(full, 0, s, b, j)[:held(eng, 0, s)], rows(small, 0, s, b, j)[:held(eng, 0, s)]
                # (rotated K is rounded to bf16 on the one side: 2^-8; blocks keep the largest of 16 tokens)
                top = np.abs(a).max()
                assert np.all(np.abs(c - a) <= (2.0 ** -4 + 2.0 ** -7) * np.abs(a) + 2.0 ** -10 * top / 224)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("extra", [dict(), dict(rope_base=0.0), dict(rope_dims=32, rope_layout=1, layer_norm=True)])
def test_a_budget_that_is_not_reached_changes_nothing_and_weights_add_up(B, bits, extra):
    from paper_2511_03983_b200.engine import DecodeSession
    eng = make(**extra)
    plain, kept = DecodeSession(eng, max_len=64, cache_bits=bits), DecodeSession(eng, max_len=64, cache_bits=bits, keep=48)
    lengths = [[24, 9]] * eng.w.n_subnets
    want = plain.prefill(0, lengths).clone()
    assert torch.equal(kept.prefill(0, lengths), want)
    w = eng.w
    sums = {}
    for s in range(w.n_subnets):
        for b in range(2):
            for p in range(held(eng, 0, s)):
                sums[s, b, p] = [paged(kept, kept.weights[0], s, b)[p].astype(np.float64), 0.0]
                # of a prompt's queries every one gives each of its heads one unit
                heads = sum(1 for h in eng.idx_head[0][s].tolist() if (int(eng.kv_pos[0][s][h // (w.n_heads // w.n_kv_heads)]) if eng.gqa else 0) == p)
                assert abs(sums[s, b, p][0].sum() - heads * lengths[s][b]) <= 2.0 ** -8 * heads * lengths[s][b]
    x = tokens(eng, 8)
    for i in range(8):
        assert torch.equal(kept.step(x[:, i]), plain.step(x[:, i]))
        for key, (pr, err) in check_attention(eng, kept).items():
            sums[key][0] = np.append(sums[key][0], 0.0) + pr
            sums[key][1] = np.append(sums[key][1], 0.0) + err if i else err
    for (s, b, p), (want, err) in sums.items():
        got = paged(kept, kept.weights[0], s, b)[p]
        assert np.all(np.abs(got - want) <= err + 16 * 2.0 ** -24 * want)
        assert paged(kept, kept.slot_pos[0], s, b)[p].tolist() == list(range(lengths[s][b] + 8))
    assert B.twist_device_status() == 0


@pytest.mark.parametrize("bits,graph,page_size", [(8, False, 16), (8, True, 16), (16, True, 32), (16, False, 16)])
def test_sequences_run_on_beyond_their_budget(B, bits, graph, page_size):
    """Forty steps with a budget of 20 tokens: every cut keeps the tokens that the weights before it name, a token's keys follow it,
    pages come back, and the attention is over what is held."""
    from paper_2511_03983_b200.engine import DecodeSession
    eng = make(layers=2)
    w = eng.w
    ses = DecodeSession(eng, max_len=32, page_size=page_size, cache_bits=bits, keep=20, recent=6, slack=5, graph=graph)
    other = DecodeSession(eng, max_len=32, page_size=page_size, cache_bits=bits, keep=20, recent=6, slack=5, graph=not graph)
    lengths = [[24, 13]] * w.n_subnets
    for z in (ses, other):
        z.prefill(0, lengths)
    x = tokens(eng, 40)
    cuts = 0
    for i in range(40):
        before = [list(r) for r in ses.lens]
        state = [[[(paged(ses, ses.weights[l], s, b), paged(ses, ses.slot_pos[l], s, b), rows(ses, l, s, b, 0)) for l in range(2)]
                  for b in range(2)] for s in range(w.n_subnets)]
        y = ses.step(x[:, i]).clone()
        assert torch.equal(other.step(x[:, i]), y)                # captured or not: the same bits
        for s in range(w.n_subnets):
            for b in range(2):
                n = before[s][b]
                if n < 25:
                    assert ses.lens[s][b] == n + 1
                    continue
                cuts += 1
                assert ses.lens[s][b] == 21 and len(ses.pages[s][b]) == -(-21 // page_size)
                for l in range(2):
                    wt, pos, k = state[s][b][l]
                    new_pos, new_k = paged(ses, ses.slot_pos[l], s, b), rows(ses, l, s, b, 0)
                    for p in range(held(eng, l, s)):
                        guard = lengths[s][b] + i - 6
                        order = sorted(range(n), key=lambda j: (pos[p][j] < guard, 0.0 if pos[p][j] >= guard else -wt[p][j], j))
                        assert sorted(new_pos[p][:20]) == sorted(pos[p][j] for j in order[:20])
                        assert new_pos[p][20] == lengths[s][b] + i
                        if bits == 16:
                            at = {int(v): j for j, v in enumerate(pos[p])}
                            assert all(np.array_equal(new_k[p][j], k[p][at[int(new_pos[p][j])]]) for j in range(20))
        check_attention(eng, ses, 1)
    assert cuts > 10 and B.twist_device_status() == 0
    assert len(ses.free) + sum(len(p) for r in ses.pages for p in r) == ses.n_pages
    ses.release(0, 1)
    assert ses.lens[0][1] == 0 and ses.seen[0][1] == 0
    ses.step(x[:, 0])
    assert paged(ses, ses.slot_pos[0], 0, 1)[:held(eng, 0, 0)].tolist() == [[0]] * held(eng, 0, 0)


def test_options_that_a_session_refuses(B):
    from paper_2511_03983_b200.engine import DecodeSession
    eng = make()
    for kw in (dict(cache_bits=4), dict(keep=0), dict(keep=40), dict(keep=20, slack=0), dict(keep=10, recent=-1), dict(keep=10, last_queries=-1),
               dict(keep=25, slack=16)):
        with pytest.raises(ValueError):
            DecodeSession(eng, max_len=40, **kw)
    with pytest.raises(ValueError):
        DecodeSession(eng, max_len=40).evict()
    with pytest.raises(ValueError):
        DecodeSession(make(d_head=8), max_len=40, cache_bits=8)
