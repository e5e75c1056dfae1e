"""Cases of the position rotation, the paged key-value cache and the attention that reads it.

Operators (binding names): twist_rope_fwd / twist_rope_bwd, twist_kv_append, twist_attn_decode.  Shapes follow the
framework: S subnets of H kept heads each; a row of projected activations is [Q of the kept heads | K of the kept
KV positions | V of the same].  Lengths of sequences are a function of the case alone, values come from the seed.
"""
import random

import torch

own = False          # True: run() calls the framework's kernels; False: the plain form

BF = torch.bfloat16


# ------------------------------------------------------------------------------------------------ cases

def _rope(name, S, n_seqs, seq_len, H, KV, D, rot, layout, bwd):
    c = dict(op="rope", S=S, n_seqs=n_seqs, seq_len=seq_len, H=H, KV=KV, D=D, rot=rot, layout=layout, bwd=bwd)
    return dict(c, name=name) if name else c


def _append(name, S, n_seqs, rows, form, past, H, KV, D, page, rot, layout):
    c = dict(op="append", S=S, n_seqs=n_seqs, rows=rows, form=form, past=past, H=H, KV=KV, D=D, page=page, rot=rot,
             layout=layout)
    return dict(c, name=name) if name else c


def _decode(name, S, n_seqs, longest, ragged, H, NH, NKV, D, page):
    c = dict(op="decode", S=S, n_seqs=n_seqs, longest=longest, ragged=ragged, H=H, NH=NH, NKV=NKV, D=D, page=page)
    return dict(c, name=name) if name else c


def listed():
    return [
        # forward rotation of one short prompt through a GPT-2-small-shaped subnet: the smallest call
        _rope("rope fwd, short prompt", 1, 1, 37, 6, 6, 64, 64, "half", False),
        # forward rotation of a training step, TinyLlama-shaped: 4 subnets, 16 sequences of 2048 tokens
        _rope("rope fwd, training step", 4, 16, 2048, 16, 4, 64, 64, "half", False),
        # backward of the rotation, all 32 heads of a 7B-shaped layer, interleaved pairs, odd sequence length
        _rope("rope bwd, wide heads", 2, 3, 4093, 32, 32, 128, 128, "pairs", True),
        # one new token of one sequence: what every step of a single answer does per layer
        _append("append, one token", 1, 1, 1, "one", 700, 8, 8, 128, 16, 128, "half"),
        # one new token of each of 128 sequences in 4 extracted subnets (grouped-query heads)
        _append("append, batch of tokens", 4, 128, 1, "one", 1500, 16, 4, 64, 32, 64, "half"),
        # prompts of different lengths, packed, half of each head rotated
        _append("append, packed prompts", 4, 13, 2311, "packed", 0, 12, 12, 64, 64, 32, "pairs"),
        # one sequence, a short cache: latency
        _decode("decode, short cache", 1, 1, 97, 0, 6, 12, 12, 64, 16),
        # ragged batch of a TinyLlama-shaped group of subnets: heads share KV positions unevenly, an empty sequence
        _decode("decode, ragged subnets", 4, 16, 2048, 1, 16, 32, 4, 64, 16),
        # one answer far into a long context: the length is all there is to split
        _decode("decode, one long cache", 1, 1, 131071, 0, 8, 32, 32, 128, 64),
        # whole model with 8 query heads per KV head, a serving batch of ragged lengths
        _decode("decode, shared keys", 1, 64, 16000, 1, 32, 32, 4, 64, 32),
        # 8 subnets of a 7B-shaped layer, 16 sequences each: the largest
        _decode("decode, eight subnets", 8, 16, 8192, 1, 8, 32, 32, 128, 16),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["rope", "append", "decode", "decode"])
    D = rng.choice([16, 32, 64, 64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    NKV = rng.choice([1, 2, 4, 8, 12])
    NH = NKV * rng.choice([1, 1, 2, 4, 8, 12])
    H = rng.randint(1, NH)
    KV = min(NKV, H)
    S = rng.choice([1, 1, 2, 3, 4, 8])
    width = (H + 2 * KV) * D
    rot = rng.choice([D, D, D // 2])
    layout = rng.choice(["half", "pairs"])
    if op == "rope":
        room = max(1, 200_000_000 // (S * width))
        tokens = _log(rng, 1, room)
        n_seqs = _log(rng, 1, min(tokens, 64))
        return _rope(None, S, n_seqs, max(1, tokens // n_seqs), H, KV, D, rot, layout, rng.random() < 0.5)
    if op == "append":
        room = max(1, 60_000_000 // (S * width))
        form = rng.choice(["one", "padded", "packed"])
        n_seqs = _log(rng, 1, max(1, min(256, room)))
        rows = 1 if form == "one" else _log(rng, 1, max(1, min(4000, room // n_seqs)))
        return _append(None, S, n_seqs, rows, form, rng.choice([0, 5, _log(rng, 1, 1000)]), H, KV, D, page, rot, layout)
    n_seqs = _log(rng, 1, 128)
    room = max(1, 1_000_000_000 // (S * n_seqs * KV * 2 * D * 2))
    return _decode(None, S, n_seqs, _log(rng, 1, min(room, 140_000)), rng.choice([0, 1, 1]), H, NH, NKV, D, page)


# ------------------------------------------------------------------------------------------------ shapes that a case fixes

def _lens(c):
    """Keys of every (subnet, sequence) of a decode case: all the longest, or ragged with an empty one among several."""
    n = c["S"] * c["n_seqs"]
    if not c["ragged"]:
        return [c["longest"]] * n
    r = random.Random(n * 7919 + c["longest"])
    v = [r.randint(1, c["longest"]) for _ in range(n)]
    v[0] = c["longest"]
    if n > 4:
        v[n // 2] = 0
    return v


def _heads(c):
    """Per subnet: the sorted kept heads (of c["NH"])."""
    r = random.Random(c["S"] * 31 + c["H"])
    return [sorted(r.sample(range(c["NH"]), c["H"])) for _ in range(c["S"])]


def _new(c):
    """New tokens of every (subnet, sequence) of an append case."""
    n = c["S"] * c["n_seqs"]
    if c["form"] == "one":
        return [1] * n
    r = random.Random(n * 104729 + c["rows"])
    v = [r.randint(0 if n > 2 else 1, c["rows"]) for _ in range(n)]
    v[-1] = c["rows"]
    return v


def _past(c):
    """Tokens already cached per (subnet, sequence) of an append case."""
    n = c["S"] * c["n_seqs"]
    r = random.Random(n * 15485863 + c["past"])
    return [r.randint(0, c["past"]) for _ in range(n)]


def _freq(rot, device):
    """The customary frequencies 10000^(-2j / rot), in 64 bits."""
    return 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)


def _normal(shape, gen, std=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * std).to(BF)


def _paged(lens, page, gen):
    """(page table [n][pages], pages of the pool): every sequence's pages scattered over the pool."""
    need = [-(-v // page) for v in lens]
    most = max(1, max(need))
    pool = sum(need) + 3
    table = torch.zeros(len(lens), most, dtype=torch.int64)
    order = torch.randperm(pool, generator=gen, device="cuda").cpu()
    at = 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    return table.to(torch.int32).cuda(), pool


def _groups(heads, NH, NKV):
    """(kv_pos [S][NKV], KV position of every kept head [S][H]): kept KV groups of a subnet in ascending order."""
    per = NH // NKV
    pos, of = [], []
    for hs in heads:
        held = sorted({h // per for h in hs})
        pos.append([held.index(g) if g in held else -1 for g in range(NKV)])
        of.append([held.index(h // per) for h in hs])
    return pos, of


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    st = dict(c)
    S, H, D = c["S"], c["H"], c["D"]
    if c["op"] == "rope":
        w = (H + 2 * c["KV"]) * D
        st["x"] = _normal((S, c["n_seqs"] * c["seq_len"], w), gen)
        st["out"] = torch.empty_like(st["x"])
        st["freq"] = _freq(c["rot"], "cuda")
        return st
    if c["op"] == "append":
        new, past, KV, n = _new(c), _past(c), c["KV"], c["n_seqs"]
        lens = [a + b for a, b in zip(new, past)]
        table, pool = _paged(lens, c["page"], gen)
        per_s = [new[s * n:(s + 1) * n] for s in range(S)]
        tokens = n * c["rows"] if c["form"] != "packed" else max(1, max(sum(v) for v in per_s))
        st["tokens"] = tokens
        st["qkv"] = _normal((S, tokens, (H + 2 * KV) * D), gen)
        st["q_out"] = torch.zeros(S, tokens, H * D, dtype=BF, device="cuda")
        st["k"] = _normal((pool, KV, c["page"], D), gen)
        st["v"] = _normal((pool, KV, c["page"], D), gen)
        st["table"] = table.view(S, n, -1)
        st["len"] = i32(lens).view(S, n)
        st["new_len"] = i32(new).view(S, n)
        begin = [[sum(v[:i]) for i in range(n + 1)] for v in per_s]
        st["begin"] = i32(begin)
        st["freq"] = _freq(c["rot"], "cuda")
        return st
    lens, heads = _lens(c), _heads(c)
    table, pool = _paged(lens, c["page"], gen)
    pos, of = _groups(heads, c["NH"], c["NKV"])
    KV = min(c["NKV"], H)
    n = c["n_seqs"]
    st["KV"] = KV
    # queries of different sharpness: some heads attend broadly, some to a few keys
    sharp = torch.rand(S, n, H, 1, generator=gen, device="cuda") * 3
    st["q"] = (torch.randn(S, n, H, D, generator=gen, device="cuda") * sharp).to(BF).view(S, n, H * D)
    st["k"] = _normal((pool, KV, c["page"], D), gen)
    st["v"] = _normal((pool, KV, c["page"], D), gen)
    st["table"] = table.view(S, n, -1)
    st["len"] = i32(lens).view(S, n)
    st["head_idx"], st["kv_pos"], st["of"] = i32(heads), i32(pos), torch.tensor(of, device="cuda")
    st["out"] = torch.empty(S, n, H * D, dtype=BF, device="cuda")
    st["lse"] = torch.empty(S, H, n, dtype=torch.float32, device="cuda")
    st["ws"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ the calls

def run(state):
    return _run_own(state) if own else _PLAIN[state["op"]](state)


def _run_own(st):
    from paper_2511_03983_b200 import binding as B
    if st["op"] == "rope":
        a = B.rope_args(B.BF16, st["S"], st["n_seqs"] * st["seq_len"], st["H"], st["KV"], st["D"], st["rot"], st["seq_len"],
                        layout=B.ROPE_HALF if st["layout"] == "half" else B.ROPE_PAIRS, in_=st["x"], out=st["out"],
                        inv_freq=st["freq"])
        (B.twist_rope_bwd if st["bwd"] else B.twist_rope_fwd)(a)
        return st["out"]
    if st["op"] == "append":
        rows = dict(new_begin=st["begin"]) if st["form"] == "packed" else dict(new_len=st["new_len"]) \
            if st["form"] == "padded" else {}
        a = B.kv_append_args(B.BF16, st["S"], st["n_seqs"], st["tokens"], st["H"], st["KV"], st["D"], rot_dims=st["rot"],
                             layout=B.ROPE_HALF if st["layout"] == "half" else B.ROPE_PAIRS, qkv=st["qkv"],
                             q_out=st["q_out"], k_cache=st["k"], v_cache=st["v"], page_table=st["table"],
                             kv_len=st["len"], inv_freq=st["freq"], **rows)
        B.twist_kv_append(a)
        return {"q": st["q_out"], "k": st["k"], "v": st["v"]}
    a = B.attn_decode_args(B.BF16, st["S"], st["n_seqs"], st["H"], st["KV"], st["D"], st["NH"], st["NKV"],
                           q=st["q"], k_cache=st["k"], v_cache=st["v"], page_table=st["table"], kv_len=st["len"],
                           head_idx=st["head_idx"], kv_pos=st["kv_pos"], out=st["out"], lse=st["lse"], ws=st["ws"])
    B.twist_attn_decode(a)
    return {"out": st["out"], "lse": st["lse"]}


# ------------------------------------------------------------------------------------------------ plain forms

def _rotate(x, pos, freq, rot, layout, sign):
    """x [.., heads, D] float, pos [..]: the first `rot` elements of every head rotated (angles in 64 bits)."""
    angle = pos.to(torch.float64)[..., None, None] * freq
    cos, sin = torch.cos(angle).float(), (sign * torch.sin(angle)).float()
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., :rot // 2], r[..., rot // 2:]) if layout == "half" else (r[..., 0::2], r[..., 1::2])
    ra, rb = a * cos - b * sin, a * sin + b * cos
    r = torch.cat([ra, rb], -1) if layout == "half" else torch.stack([ra, rb], -1).flatten(-2)
    return torch.cat([r, rest], -1)


def _plain_rope(st):
    S, H, KV, D = st["S"], st["H"], st["KV"], st["D"]
    x = st["x"]
    T = x.shape[1]
    pos = (torch.arange(T, device=x.device) % st["seq_len"]).expand(S, T)
    qk = x[..., :(H + KV) * D].float().view(S, T, H + KV, D)
    qk = _rotate(qk, pos, st["freq"], st["rot"], st["layout"], -1.0 if st["bwd"] else 1.0)
    st["out"][..., :(H + KV) * D] = qk.view(S, T, -1).to(BF)
    st["out"][..., (H + KV) * D:] = x[..., (H + KV) * D:]
    return st["out"]


def _plain_append(st):
    S, H, KV, D, n, page = st["S"], st["H"], st["KV"], st["D"], st["n_seqs"], st["page"]
    T = st["tokens"]
    dev = st["qkv"].device
    t = torch.arange(T, device=dev)
    if st["form"] == "packed":
        seq = torch.searchsorted(st["begin"][:, 1:].contiguous(), t.to(torch.int32).expand(S, T).contiguous(), right=True)
        valid = seq < n
        seq = seq.clamp(max=n - 1)
        first = torch.gather(st["begin"].long(), 1, seq)
        i = t - first
    else:
        seq = (t // st["rows"]).expand(S, T)
        i = (t % st["rows"]).expand(S, T)
        valid = i < torch.gather(st["new_len"].long(), 1, seq)
    pos = torch.gather(st["len"].long(), 1, seq) - torch.gather(st["new_len"].long(), 1, seq) + i
    qk = st["qkv"][..., :(H + KV) * D].float().view(S, T, H + KV, D)
    qk = _rotate(qk, pos, st["freq"], st["rot"], st["layout"], 1.0).to(BF)
    q = qk[:, :, :H].reshape(S, T, H * D)
    st["q_out"].copy_(torch.where(valid[..., None], q, st["q_out"]))
    s_of = torch.arange(S, device=dev)[:, None].expand(S, T)
    s_of, seq, pos = s_of[valid], seq[valid], pos[valid]
    at = st["table"].long()[s_of, seq, pos // page]
    st["k"][at, :, pos % page] = qk[:, :, H:][valid]
    st["v"][at, :, pos % page] = st["qkv"][..., (H + KV) * D:].view(S, T, KV, D)[valid]
    return {"q": st["q_out"], "k": st["k"], "v": st["v"]}


def _plain_decode(st):
    S, H, D, n, page = st["S"], st["H"], st["D"], st["n_seqs"], st["page"]
    table = st["table"].long()
    head = st["of"][:, None, :].expand(S, n, H)

    def rows(cache):             # [S][n][H][keys][D] of the KV position that each head reads
        got = cache[table[:, :, None, :], head[..., None]]
        return got.reshape(S, n, H, -1, D).float()

    q = st["q"].float().view(S, n, H, 1, D)
    score = (q @ rows(st["k"]).transpose(-1, -2)).squeeze(-2) * (D ** -0.5)
    live = torch.arange(score.shape[-1], device=score.device) < st["len"].long()[..., None, None]
    score = torch.where(live, score, torch.full((), float("-inf"), device=score.device))
    top = score.amax(-1, keepdim=True)
    p = torch.where(live, torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top)),
                    torch.zeros((), device=score.device))
    total = p.sum(-1, keepdim=True)
    v = rows(st["v"])
    o = (p[..., None, :] @ v).squeeze(-2) / torch.where(total > 0, total, torch.ones_like(total))
    st["out"].copy_(o.reshape(S, n, H * D).to(BF))
    st["lse"].copy_((torch.log(total) + torch.where(torch.isinf(top), torch.zeros_like(top), top)).squeeze(-1).transpose(1, 2))
    return {"out": st["out"], "lse": st["lse"]}


_PLAIN = {"rope": _plain_rope, "append": _plain_append, "decode": _plain_decode}


# ------------------------------------------------------------------------------------------------ cost and exact values

def work(case):
    c = case
    S, H, D = c["S"], c["H"], c["D"]
    if c["op"] == "rope":
        rows = S * c["n_seqs"] * c["seq_len"]
        return {"bytes": rows * (H + 2 * c["KV"]) * D * 4 + 8 * (c["rot"] // 2), "flops": rows * (H + c["KV"]) * c["rot"] * 3}
    if c["op"] == "append":
        new = sum(_new(c))
        pages = sum(-(-a // c["page"]) for a in _new(c))
        return {"bytes": new * (H + 2 * c["KV"]) * D * 4 + 4 * (pages + 2 * S * c["n_seqs"]) + 8 * (c["rot"] // 2),
                "flops": new * (H + c["KV"]) * c["rot"] * 3}
    lens, heads = _lens(c), _heads(c)
    per, n = c["NH"] // c["NKV"], c["n_seqs"]
    held = [len({h // per for h in hs}) for hs in heads]
    keys = [sum(lens[s * n:(s + 1) * n]) for s in range(S)]
    size = sum(k * g for k, g in zip(keys, held)) * 2 * D * 2
    pages = sum(-(-v // c["page"]) for v in lens)
    return {"bytes": size + S * n * H * (4 * D + 4) + 4 * (pages + S * n), "flops": sum(keys) * H * 4 * D}


def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    S, H, D, n = st["S"], st["H"], st["D"], st["n_seqs"]

    def turn(x, pos, sign):      # x [rows][heads][D] in 64 bits; pairs as complex numbers times exp(i angle)
        rot, half = st["rot"], st["rot"] // 2
        w = torch.polar(torch.ones((), dtype=f64, device=x.device).expand(len(pos), half),
                        sign * pos.to(f64)[:, None] * st["freq"][None, :])[:, None]
        x = x.clone()
        lo, hi = (slice(0, half), slice(half, rot)) if st["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(x[..., lo], x[..., hi]) * w
        x[..., lo], x[..., hi] = z.real, z.imag
        return x

    if st["op"] == "rope":
        KV = st["KV"]
        out = torch.empty(st["x"].shape, dtype=f64, device="cuda")
        pos = torch.arange(st["seq_len"], device="cuda")
        N = st["seq_len"]
        for s in range(S):
            for b in range(n):
                z = st["x"][s, b * N:(b + 1) * N].to(f64).view(N, H + 2 * KV, D)
                z[:, :H + KV] = turn(z[:, :H + KV], pos, -1.0 if st["bwd"] else 1.0)
                out[s, b * N:(b + 1) * N] = z.view(N, -1)
        return out
    if st["op"] == "append":
        KV, page = st["KV"], st["page"]
        q, k, v = st["q_out"].to(f64), st["k"].to(f64), st["v"].to(f64)
        begin, new, lens, table = st["begin"].tolist(), st["new_len"].tolist(), st["len"].tolist(), st["table"].long()
        for s in range(S):
            for b in range(n):
                m = new[s][b]
                if m == 0:
                    continue
                r0 = begin[s][b] if st["form"] == "packed" else b * st["rows"]
                z = st["qkv"][s, r0:r0 + m].to(f64).view(m, H + 2 * KV, D)
                pos = torch.arange(lens[s][b] - m, lens[s][b], device="cuda")
                qk = turn(z[:, :H + KV], pos, 1.0)
                q[s, r0:r0 + m] = qk[:, :H].reshape(m, -1)
                at = table[s, b][pos // page]
                k[at, :, pos % page] = qk[:, H:]
                v[at, :, pos % page] = z[:, H + KV:]
        return {"q": q, "k": k, "v": v}
    out = torch.zeros(S, n, H * D, dtype=f64, device="cuda")
    lse = torch.full((S, H, n), float("-inf"), dtype=f64, device="cuda")
    lens, table = st["len"].tolist(), st["table"].long()
    for s in range(S):
        of = st["of"][s]
        for b in range(n):
            m = lens[s][b]
            if m == 0:
                continue
            pages = table[s, b, :-(-m // st["page"])]
            k = st["k"][pages].to(f64).permute(1, 0, 2, 3).reshape(st["KV"], -1, D)[:, :m]
            v = st["v"][pages].to(f64).permute(1, 0, 2, 3).reshape(st["KV"], -1, D)[:, :m]
            q = st["q"][s, b].to(f64).view(H, D)
            step = max(1, (1 << 27) // (m * D))       # heads at a time
            for h in range(0, H, step):
                g = of[h:h + step]
                x = torch.einsum("hkd,hd->hk", k[g], q[h:h + step]) / D ** 0.5
                lse[s, h:h + step, b] = torch.logsumexp(x, 1)
                out[s, b].view(H, D)[h:h + step] = torch.einsum("hk,hkd->hd", torch.softmax(x, 1), v[g])
    return {"out": out, "lse": lse}
