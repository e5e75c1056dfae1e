"""Rotation by position inside training rounds, and extracted subnets answering token by token (prefill, then one token at a
time through the paged cache), against the fp64 oracle that mirrors the bf16 rounding points.  Tolerances as for the other
chained compositions: 2e-2 relative Frobenius for activations, 5e-2 for the change of the weights, 2e-2 for losses."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import twist_oracle as o
from paper_2511_03983_b200 import inputs as I

pytestmark = pytest.mark.gpu

MATS = {"gate": I.MAT_GATE, "up": I.MAT_UP, "down": I.MAT_DOWN, "qkv": I.MAT_QKV, "o": I.MAT_O}


@pytest.fixture(scope="module")
def B():
    from paper_2511_03983_b200 import binding
    binding.lib()
    return binding


def dev(x, dtype=torch.bfloat16):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


def rel_fro(got, want):
    return float(np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300))


def fill_model(eng, w):
    full = []
    for l in range(w.n_layers):
        layer = {m: I.weight(w, l, MATS[m]) for m in eng.full}
        for m, v in layer.items():
            eng.full[m][l].copy_(dev(v))
        if w.layer_norm:
            for n in I.LN_PARAMS:
                layer[n] = I.ln_param(w, l, n)
                eng.full_ln[n][l].copy_(dev(layer[n], torch.float32))
        full.append(layer)
    return full


@pytest.mark.parametrize("cfg,dims,n_seqs,extra", [
    (2, dict(d_model=192, d_ff=528, d_head=16, tokens=192, n_layers=2, local_steps=2), 2, dict(rope_base=100.0)),
    (3, dict(d_model=256, d_ff=688, d_head=64, tokens=200, n_layers=2, local_steps=1), 2,
     dict(rope_base=10000.0, rope_dims=32, rope_layout=1, layer_norm=True, lr=1.0)),
    (3, dict(d_model=256, d_ff=688, d_head=8, tokens=200, n_layers=3, local_steps=2), 2, dict(rope_base=30.0, shared_layers=(0, 2))),
])
def test_training_round_with_rotation_matches_the_oracle(B, cfg, dims, n_seqs, extra):
    from paper_2511_03983_b200.engine import StackEngine
    w = replace(I.scaled_twin(I.PRESETS[cfg], **dims), **extra)
    seq_len = w.tokens // n_seqs
    eng = StackEngine(w, n_seqs, seq_len, keep_f32_full=True)
    full = fill_model(eng, w)
    store = {}
    for k in range(w.local_steps):
        for kind, dst in ((I.BATCH_X, eng.X), (I.BATCH_TGT_D, eng.Td)):
            arr = np.stack([I.batch(w, kind, 0, s, k, w.d_model) for s in range(w.n_subnets)])
            store[(kind, k)] = arr
            dst.append(dev(arr))
    eng.run_round(0)
    torch.cuda.synchronize()
    assert B.twist_device_status() == 0
    full64 = [{m: v.astype(np.float64) for m, v in layer.items()} for layer in full]
    new, _, losses = o.round_stack(w, full64, lambda kind, rnd, s, k, width: store[(kind, k)][s], 0, n_seqs, seq_len, True)
    assert np.allclose(eng.stack_loss[: w.local_steps].cpu().numpy(), np.array(losses).T, rtol=2e-2)
    for l in range(w.n_layers):
        for m in eng.full:
            res = eng.full_f32[m][l].cpu().numpy().astype(np.float64)
            err = rel_fro(res - full64[l][m], new[l][m] - full64[l][m])
            assert err < 5e-2, (l, m, err)


@pytest.mark.parametrize("cfg,dims,n_seqs,extra,page", [
    (2, dict(d_model=192, d_ff=528, d_head=64, tokens=64, n_layers=2), 2, dict(rope_base=100.0), 16),
    (3, dict(d_model=256, d_ff=688, d_head=64, tokens=99, n_layers=2), 3, dict(rope_base=10000.0, layer_norm=True), 32),
    (3, dict(d_model=256, d_ff=688, d_head=8, tokens=40, n_layers=3), 1, dict(rope_base=30.0, rope_layout=1, shared_layers=(0,)), 16),
    (4, dict(d_model=256, d_ff=512, d_head=128, tokens=36, n_layers=1), 2, {}, 16),              # no rotation
])
def test_extracted_subnets_answer_token_by_token(B, cfg, dims, n_seqs, extra, page):
    from paper_2511_03983_b200.engine import DecodeSession, StackEngine
    w = replace(I.scaled_twin(I.PRESETS[cfg], local_steps=1, **dims), **extra)
    S, N, d, steps = w.n_subnets, w.tokens // n_seqs, w.d_model, 5
    eng = StackEngine(w, n_seqs, N)
    full = fill_model(eng, w)
    rng = np.random.default_rng(8)
    lengths = [[int(x) for x in rng.integers(0 if n_seqs > 1 else 1, N + 1, n_seqs)] for _ in range(S)]
    lengths[0][0] = N
    tok = np.stack([I.normal(77, s, (n_seqs, N + steps, d), 1.0, I.DTYPE_BF16) for s in range(S)])      # every sequence's tokens
    prompt = np.zeros((S, n_seqs, N, d), dtype=np.float32)
    for s in range(S):
        for b in range(n_seqs):
            prompt[s, b, :lengths[s][b]] = tok[s, b, :lengths[s][b]]
    eng.X.append(dev(prompt.reshape(S, n_seqs * N, d)))
    eng.extract(0)
    ses = DecodeSession(eng, max_len=N + steps, page_size=page)
    pre = ses.prefill(0, lengths).float().cpu().numpy().reshape(S, n_seqs, N, d).copy()
    outs = []
    for i in range(steps):
        x = np.stack([np.stack([tok[s, b, lengths[s][b] + i] for b in range(n_seqs)]) for s in range(S)])
        outs.append(ses.step(dev(x)).float().cpu().numpy().copy())
    torch.cuda.synchronize()
    assert B.twist_device_status() == 0
    bps = [o.layer_blueprints(w, 0, l) for l in range(w.n_layers)]
    for s in range(S):
        layers = [{m: np.asarray(v, dtype=np.float64) for m, v in o.gather_layer(w, full[l], bps[l], s).items()} for l in range(w.n_layers)]
        head_kv = [o.head_kv_positions(bps[l], w, s) for l in range(w.n_layers)]
        for b in range(n_seqs):
            m = lengths[s][b]
            want, _ = o.stack_fwd(w, layers, head_kv, tok[s, b, :m + steps].astype(np.float64), 1, m + steps, True)
            if m:
                assert rel_fro(pre[s, b, :m], want[:m]) < 2e-2, (s, b)
            for i in range(steps):
                assert rel_fro(outs[i][s, b], want[m + i]) < 2e-2, (s, b, i)
    # a full cache refuses, a released sequence starts again at position 0
    with pytest.raises(ValueError):
        ses.step(dev(x))
    ses.release(0, 0)
    for s in range(S):
        for b in range(n_seqs):
            if (s, b) != (0, 0):
                ses.release(s, b)
    y = ses.step(dev(tok[:, :, 0])).float().cpu().numpy()
    want, _ = o.stack_fwd(w, [{m: np.asarray(v, dtype=np.float64) for m, v in o.gather_layer(w, full[l], bps[l], 0).items()} for l in range(w.n_layers)],
                          [o.head_kv_positions(bps[l], w, 0) for l in range(w.n_layers)], tok[0, 0, :1].astype(np.float64), 1, 1, True)
    assert rel_fro(y[0, 0], want[0]) < 2e-2


@pytest.mark.parametrize("layers,ln", [(2, False), (3, True)])
def test_a_session_as_a_replayed_graph_gives_the_same_bits(B, layers, ln):
    """The layers of a step captured once: the steps give what the steps without a graph give, also after a sequence was
    released and started again."""
    from paper_2511_03983_b200.engine import DecodeSession, StackEngine
    w = replace(I.scaled_twin(I.PRESETS[3], d_model=256, d_ff=688, d_head=64, tokens=42, n_layers=layers, local_steps=1), rope_base=10000.0,
                layer_norm=ln)
    eng = StackEngine(w, 2, 21)
    fill_model(eng, w)
    eng.X.append(dev(np.stack([I.normal(7, s, (42, w.d_model), 1.0, I.DTYPE_BF16) for s in range(w.n_subnets)])))
    eng.extract(0)
    tok = dev(I.normal(78, 0, (20, w.n_subnets, 2, w.d_model), 1.0, I.DTYPE_BF16))
    outs = []
    for graph in (False, True):
        ses = DecodeSession(eng, max_len=48, graph=graph)
        ses.prefill(0, [[21, 3]] * w.n_subnets)
        got = [ses.step(tok[i]).clone() for i in range(12)]
        ses.release(1, 0)
        got += [ses.step(tok[i]).clone() for i in range(12, 20)]
        outs.append(got)
        torch.cuda.synchronize()
        assert B.twist_device_status() == 0
    for i, (x, y) in enumerate(zip(*outs)):
        assert torch.equal(x, y), i
