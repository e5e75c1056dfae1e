"""Cases of the smaller key-value cache: 8-bit append and decode, the attention weight that cached keys gather, and eviction
by it.

Operators (binding names): twist_kv_append_q8, twist_attn_decode_q8, twist_attn_weights, twist_attn_core_weights,
twist_kv_evict.  Shapes follow the framework: S subnets of H kept heads each; a row of projected activations is [Q of the kept
heads | K of the kept KV positions | V of the same].  An 8-bit cache holds e4m3 numbers and a pair of scales (K, V) for each
block of 16 tokens and KV position; run() returns the numbers as float8 tensors beside their scales.  Lengths of sequences are a
function of the case alone, values come from the seed.
"""
import random

import torch

own = False          # True: run() calls the framework's kernels; False: the plain form

BF = torch.bfloat16
F8 = torch.float8_e4m3fn
BLOCK = 16           # tokens that share a scale
LOW, HIGH = -110, 119          # exponents that a scale may have


# ------------------------------------------------------------------------------------------------ cases

def _append(name, S, n_seqs, rows, form, past, H, KV, D, page, rot, layout):
    c = dict(op="append", S=S, n_seqs=n_seqs, rows=rows, form=form, past=past, H=H, KV=KV, D=D, page=page, rot=rot,
             layout=layout)
    return dict(c, name=name) if name else c


def _decode(name, S, n_seqs, longest, ragged, H, NH, NKV, D, page):
    c = dict(op="decode", S=S, n_seqs=n_seqs, longest=longest, ragged=ragged, H=H, NH=NH, NKV=NKV, D=D, page=page)
    return dict(c, name=name) if name else c


def _weights(name, S, n_seqs, longest, ragged, H, NH, NKV, D, page, q8):
    c = dict(op="weights", S=S, n_seqs=n_seqs, longest=longest, ragged=ragged, H=H, NH=NH, NKV=NKV, D=D, page=page, q8=q8)
    return dict(c, name=name) if name else c


def _core(name, S, n_seqs, longest, ragged, last, H, NH, NKV, D, page):
    c = dict(op="core", S=S, n_seqs=n_seqs, longest=longest, ragged=ragged, last=last, H=H, NH=NH, NKV=NKV, D=D, page=page)
    return dict(c, name=name) if name else c


def _evict(name, S, n_seqs, longest, ragged, keep, recent, again, KV, D, page, q8):
    c = dict(op="evict", S=S, n_seqs=n_seqs, longest=longest, ragged=ragged, keep=keep, recent=recent, again=again, KV=KV,
             D=D, page=page, q8=q8)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token of each of 128 sequences in 4 extracted subnets (grouped-query heads): a decoding step
        _append("append, batch of tokens", 4, 128, 1, "one", 1500, 16, 4, 64, 32, 64, "half"),
        # prompts of different lengths, packed, behind a few cached tokens, half of each head rotated
        _append("append, packed prompts", 4, 13, 2311, "packed", 5, 12, 12, 64, 64, 32, "pairs"),
        # one sequence, a short cache: latency, the smallest decode
        _decode("decode, short cache", 1, 1, 97, 0, 6, 12, 12, 64, 16),
        # ragged batch of a TinyLlama-shaped group of subnets: heads share KV positions unevenly, an empty sequence
        _decode("decode, ragged subnets", 4, 16, 2048, 1, 16, 32, 4, 64, 16),
        # whole model with 8 query heads per KV head, a serving batch of ragged lengths
        _decode("decode, shared keys", 1, 64, 16000, 1, 32, 32, 4, 64, 32),
        # 8 subnets of a 7B-shaped layer, 16 sequences each: the largest
        _decode("decode, eight subnets", 8, 16, 8192, 1, 8, 32, 32, 128, 16),
        # the weights of a step of the ragged subnets, 8-bit cache
        _weights("weights, ragged subnets", 4, 16, 2048, 1, 16, 32, 4, 64, 16, True),
        # the weights of one answer far into a long context, bf16 cache
        _weights("weights, one long cache", 1, 1, 131071, 0, 8, 32, 32, 128, 64, False),
        # the weights of a few short ragged prompts, the last 32 queries of each
        _core("prompt weights, short", 2, 3, 77, 1, 32, 8, 16, 4, 32, 16),
        # the weights of whole prompts of a TinyLlama-shaped group of subnets
        _core("prompt weights, long", 4, 4, 2048, 0, 0, 16, 32, 4, 64, 16),
        # a cache that is one page over its budget, evicted every 16 tokens: the steady state of a serving batch
        _evict("evict, a page over", 4, 16, 1040, 0, 1024, 256, True, 4, 64, 16, True),
        # long ragged prompts cut to a quarter after their prefill, 7B-shaped heads, bf16 cache
        _evict("evict, long prompts", 1, 8, 16000, 1, 4099, 1024, False, 8, 128, 64, False),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "weights", "core", "evict"])
    D = rng.choice([16, 32, 64, 64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    NKV = rng.choice([1, 2, 4, 8, 12])
    NH = NKV * rng.choice([1, 1, 2, 4, 8, 12])
    H = rng.randint(1, NH)
    KV = min(NKV, H)
    S = rng.choice([1, 1, 2, 3, 4, 8])
    width = (H + 2 * KV) * D
    if op == "append":
        room = max(1, 60_000_000 // (S * width))
        form = rng.choice(["one", "padded", "packed"])
        n_seqs = _log(rng, 1, max(1, min(256, room)))
        rows = 1 if form == "one" else _log(rng, 1, max(1, min(4000, room // n_seqs)))
        return _append(None, S, n_seqs, rows, form, rng.choice([0, 5, _log(rng, 1, 1000)]), H, KV, D, page, rng.choice([D, D, D // 2]),
                       rng.choice(["half", "pairs"]))
    n_seqs = _log(rng, 1, 64 if op == "evict" else 128)
    if op in ("decode", "weights"):
        room = max(1, 900_000_000 // (S * n_seqs * KV * 2 * D))
        longest, ragged = _log(rng, 1, min(room, 140_000)), rng.choice([0, 1, 1])
        if op == "decode":
            return _decode(None, S, n_seqs, longest, ragged, H, NH, NKV, D, page)
        return _weights(None, S, n_seqs, longest, ragged, H, NH, NKV, D, page, rng.random() < 0.5)
    if op == "core":
        H = min(H, 32)
        room = max(1, int((1_000_000_000 / (S * n_seqs * H)) ** 0.5))
        longest = _log(rng, 1, min(room, 4000))
        return _core(None, S, n_seqs, longest, rng.choice([0, 1, 1]), rng.choice([0, 0, 32, longest]), H, NH, NKV, D, page)
    room = max(1, 130_000_000 // (S * n_seqs * KV * D))
    longest = _log(rng, 1, min(room, 60_000))
    keep = rng.choice([_log(rng, 1, longest), max(1, longest - rng.randint(0, 64)), max(1, longest // 2)])
    return _evict(None, S, n_seqs, longest, rng.choice([0, 1, 1]), keep, rng.choice([0, keep // 4, _log(rng, 1, longest)]),
                  rng.random() < 0.5, KV, D, page, rng.random() < 0.6)


# ------------------------------------------------------------------------------------------------ shapes that a case fixes

def _lens(c):
    """Keys of every (subnet, sequence): all the longest, or ragged with an empty one among several."""
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


def _gone(c):
    """Tokens of each sequence of an append case that were evicted before (its positions run ahead of its slots)."""
    r = random.Random(c["past"] + 17)
    return [r.randint(0, 900) for _ in range(c["S"] * c["n_seqs"])]


def _groups(heads, NH, NKV):
    """(kv_pos [S][NKV], KV position of every kept head [S][H]): kept KV groups of a subnet in ascending order."""
    per = NH // NKV
    pos, of = [], []
    for hs in heads:
        held = sorted({h // per for h in hs})
        pos.append([held.index(g) if g in held else -1 for g in range(NKV)])
        of.append([held.index(h // per) for h in hs])
    return pos, of


# ------------------------------------------------------------------------------------------------ inputs

def _freq(rot, device):
    """The customary frequencies 10000^(-2j / rot), in 64 bits."""
    return 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)


def _normal(shape, gen, std=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * std).to(BF)


def _coded(shape, gen):
    """(e4m3 numbers [pool][KV][page][D], their scales [pool][KV][page / 16]): values of about unit size, blocks of different
    spread."""
    pool, KV, page, _ = shape
    code = (torch.randn(*shape, generator=gen, device="cuda") * 90).clamp_(-448, 448).to(F8)
    return code, torch.exp2(torch.randint(-8, -4, (pool, KV, page // BLOCK), generator=gen, device="cuda").float())


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


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _attention(st, c, gen):
    """Queries, heads, pages and lengths of a decode or weights case."""
    S, H, D, n = c["S"], c["H"], c["D"], c["n_seqs"]
    lens, heads = _lens(c), _heads(c)
    table, pool = _paged(lens, c["page"], gen)
    pos, of = _groups(heads, c["NH"], c["NKV"])
    st["KV"] = min(c["NKV"], H)
    # queries of different sharpness: some heads attend broadly, some to a few keys
    sharp = torch.rand(S, n, H, 1, generator=gen, device="cuda") * 3
    st["q"] = (torch.randn(S, n, H, D, generator=gen, device="cuda") * sharp).to(BF).view(S, n, H * D)
    st["table"] = table.view(S, n, -1)
    st["len"] = _i32(lens).view(S, n)
    st["head_idx"], st["kv_pos"], st["of"] = _i32(heads), _i32(pos), torch.tensor(of, device="cuda")
    return pool


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = dict(c)
    S, D, n, page = c["S"], c["D"], c["n_seqs"], c["page"]
    if c["op"] == "append":
        H, KV = c["H"], c["KV"]
        new, past, gone = _new(c), _past(c), _gone(c)
        lens = [a + b for a, b in zip(new, past)]
        table, pool = _paged(lens, page, gen)
        per_s = [new[s * n:(s + 1) * n] for s in range(S)]
        tokens = n * c["rows"] if c["form"] != "packed" else max(1, max(sum(v) for v in per_s))
        st["tokens"] = tokens
        st["qkv"] = _normal((S, tokens, (H + 2 * KV) * D), gen)
        st["q_out"] = torch.zeros(S, tokens, H * D, dtype=BF, device="cuda")
        st["k"], ks = _coded((pool, KV, page, D), gen)
        st["v"], vs = _coded((pool, KV, page, D), gen)
        st["scales"] = torch.stack([ks, vs], -1)
        st["table"] = table.view(S, n, -1)
        st["len"] = _i32(lens).view(S, n)
        st["seen"] = _i32([a + b for a, b in zip(lens, gone)]).view(S, n)
        st["new_len"] = _i32(new).view(S, n)
        st["begin"] = _i32([[sum(v[:i]) for i in range(n + 1)] for v in per_s])
        st["freq"] = _freq(c["rot"], "cuda")
        return st
    if c["op"] == "evict":
        KV, lens = c["KV"], _lens(c)
        table, pool = _paged(lens, page, gen)
        st["table"] = table.view(S, n, -1)
        st["len"] = _i32(lens).view(S, n)
        st["keep"] = _i32([min(v, c["keep"]) for v in lens]).view(S, n)
        st["kv_count"] = _i32([max(1, KV - s % 2) for s in range(S)])
        if c["q8"]:
            st["k"], ks = _coded((pool, KV, page, D), gen)
            st["v"], vs = _coded((pool, KV, page, D), gen)
            st["scales"] = torch.stack([ks, vs], -1)
        else:
            st["k"], st["v"], st["scales"] = _normal((pool, KV, page, D), gen), _normal((pool, KV, page, D), gen), None
        # heavy-tailed weights, some keys that nothing ever looked at
        w = torch.rand(pool, KV, page, generator=gen, device="cuda").clamp_(min=1e-6).reciprocal_()
        st["weights"] = torch.where(torch.rand(pool, KV, page, generator=gen, device="cuda") < 0.05, torch.zeros_like(w), w)
        # positions: as the slots, or (again) those of a cache whose first slots were evicted and filled before
        room = table.shape[1] * page
        i = torch.arange(room, device="cuda")
        length = st["len"].view(-1, 1, 1)
        if c["again"]:
            m = torch.clamp(length, max=c["keep"])
            dice = torch.where(i < m, torch.rand(S * n, KV, room, generator=gen, device="cuda"), 2.0 + i / room)
            pos = torch.where(i < m, 2 * dice.argsort(-1), i + m)
            st["seen"] = (st["len"] + st["keep"]).contiguous()
        else:
            pos = i.expand(S * n, KV, room)
            st["seen"] = st["len"].clone()
        st["slot_pos"] = torch.zeros(pool, KV, page, dtype=torch.int32, device="cuda")
        used = (torch.arange(table.shape[1], device="cuda") * page < length[:, 0]).reshape(-1)
        st["slot_pos"][table.long().reshape(-1)[used]] = \
            pos.reshape(S * n, KV, -1, page).transpose(1, 2).reshape(-1, KV, page)[used].to(torch.int32)
        st["weights_out"], st["slot_pos_out"] = torch.zeros_like(st["weights"]), torch.zeros_like(st["slot_pos"])
        st["ws"] = torch.empty(S * n * KV * (4 * room + 1024) + (1 << 20), dtype=torch.uint8, device="cuda")
        return st
    H = c["H"]
    if c["op"] == "core":
        lens, heads = _lens(c), _heads(c)
        table, pool = _paged(lens, page, gen)
        pos, of = _groups(heads, c["NH"], c["NKV"])
        KV = st["KV"] = min(c["NKV"], H)
        st["table"], st["new_len"] = table.view(S, n, -1), _i32(lens).view(S, n)
        st["head_idx"], st["kv_pos"], st["of"] = _i32(heads), _i32(pos), torch.tensor(of, device="cuda")
        st["qkv"] = _normal((S, n * c["longest"], (H + 2 * KV) * D), gen, 1.3)
        st["lse"] = torch.logsumexp(_prompt_scores(st), -1).permute(0, 2, 1, 3).reshape(S, H, -1).contiguous()
        st["weights"] = torch.zeros(pool, KV, page, device="cuda")
        st["slot_pos"] = torch.zeros(pool, KV, page, dtype=torch.int32, device="cuda")
        return st
    pool = _attention(st, c, gen)
    KV = st["KV"]
    if c["op"] == "decode":
        st["k"], ks = _coded((pool, KV, page, D), gen)
        st["v"], vs = _coded((pool, KV, page, D), gen)
        st["scales"] = torch.stack([ks, vs], -1)
        st["out"] = torch.empty(S, n, H * D, dtype=BF, device="cuda")
        st["lse"] = torch.empty(S, H, n, dtype=torch.float32, device="cuda")
        st["ws"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        return st
    if c["q8"]:
        st["k"], ks = _coded((pool, KV, page, D), gen)
        st["scales"] = torch.stack([ks, ks], -1)
    else:
        st["k"], st["scales"] = _normal((pool, KV, page, D), gen), None
    st["lse"] = torch.logsumexp(_scores(st), -1).transpose(1, 2).contiguous()
    st["seen"] = st["len"] + 100
    st["prior"] = torch.rand(pool, KV, page, generator=gen, device="cuda").square_() * 4
    st["weights"] = torch.zeros_like(st["prior"])
    st["slot_pos"] = torch.zeros(pool, KV, page, dtype=torch.int32, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ the calls

def run(state):
    return _run_own(state) if own else _PLAIN[state["op"]](state)


def _run_own(st):
    from paper_2511_03983_b200 import binding as B
    S, n, D = st["S"], st["n_seqs"], st["D"]
    if st["op"] == "append":
        rows = dict(new_begin=st["begin"]) if st["form"] == "packed" else dict(new_len=st["new_len"]) \
            if st["form"] == "padded" else {}
        B.twist_kv_append_q8(B.kv_append_q8_args(
            B.BF16, S, n, st["tokens"], st["H"], st["KV"], D, rot_dims=st["rot"],
            layout=B.ROPE_HALF if st["layout"] == "half" else B.ROPE_PAIRS, qkv=st["qkv"], q_out=st["q_out"], k_cache=st["k"],
            v_cache=st["v"], scales=st["scales"], page_table=st["table"], kv_len=st["len"], seen=st["seen"], inv_freq=st["freq"],
            **rows))
        return {"q": st["q_out"], "k": st["k"], "v": st["v"], "scales": st["scales"]}
    if st["op"] == "evict":
        B.twist_kv_evict(B.kv_evict_args(
            B.BF16, S, n, st["KV"], D, st["recent"], k_cache=st["k"], v_cache=st["v"], scales=st["scales"],
            weights=st["weights"], slot_pos=st["slot_pos"], weights_out=st["weights_out"], slot_pos_out=st["slot_pos_out"],
            page_table=st["table"], kv_len=st["len"], keep=st["keep"], seen=st["seen"], kv_count=st["kv_count"], ws=st["ws"]))
        return _evicted(st)
    share = dict(head_idx=st["head_idx"], kv_pos=st["kv_pos"])
    if st["op"] == "core":
        B.twist_attn_core_weights(B.attn_core_weights_args(
            B.BF16, S, n, st["longest"], st["H"], st["KV"], D, st["NH"], st["NKV"], last_queries=st["last"], qkv=st["qkv"],
            lse=st["lse"], page_table=st["table"], new_len=st["new_len"], weights=st["weights"], slot_pos=st["slot_pos"], **share))
        return {"weights": st["weights"], "slot_pos": st["slot_pos"]}
    if st["op"] == "weights":
        B.twist_attn_weights(B.attn_weights_args(
            B.BF16, S, n, st["H"], st["KV"], D, st["NH"], st["NKV"], q=st["q"], lse=st["lse"], k_cache=st["k"],
            scales=st["scales"], page_table=st["table"], kv_len=st["len"], seen=st["seen"], prior=st["prior"],
            weights=st["weights"], slot_pos=st["slot_pos"], **share))
        return {"weights": st["weights"], "slot_pos": st["slot_pos"]}
    B.twist_attn_decode_q8(B.attn_decode_q8_args(
        B.BF16, S, n, st["H"], st["KV"], D, st["NH"], st["NKV"], q=st["q"], k_cache=st["k"], v_cache=st["v"],
        scales=st["scales"], page_table=st["table"], kv_len=st["len"], out=st["out"], lse=st["lse"], ws=st["ws"], **share))
    return {"out": st["out"], "lse": st["lse"]}


def _evicted(st):
    out = {"k": st["k"], "v": st["v"], "weights": st["weights_out"], "slot_pos": st["slot_pos_out"]}
    return dict(out, scales=st["scales"]) if st["q8"] else out


# ------------------------------------------------------------------------------------------------ plain forms

def _rotate(x, pos, freq, rot, layout):
    """x [.., heads, D] float, pos [..]: the first `rot` elements of every head rotated (angles in 64 bits)."""
    angle = pos.to(torch.float64)[..., None, None] * freq
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., :rot // 2], r[..., rot // 2:]) if layout == "half" else (r[..., 0::2], r[..., 1::2])
    ra, rb = a * cos - b * sin, a * sin + b * cos
    r = torch.cat([ra, rb], -1) if layout == "half" else torch.stack([ra, rb], -1).flatten(-2)
    return torch.cat([r, rest], -1)


def _need(amax):
    """The smallest power of two (of those that a scale may be) whose 448-fold is not below amax."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.exp2(torch.where(amax > 0, e.clamp(LOW, HIGH), LOW).to(amax.dtype))


def _finite(x):
    """Magnitudes; of what is not finite, nothing."""
    return torch.where(torch.isfinite(x), x.abs(), torch.zeros((), device=x.device))


def _code(x, scale):
    y = x / scale
    return torch.where(torch.isfinite(x), y.clamp(-448, 448), torch.full((), float("nan"), device=x.device)).to(F8)


def _tokens(st):
    """Of an append case: (row valid [S][T], its sequence, its slot, its position)."""
    S, n, T = st["S"], st["n_seqs"], st["tokens"]
    t = torch.arange(T, device="cuda")
    if st["form"] == "packed":
        seq = torch.searchsorted(st["begin"][:, 1:].contiguous(), t.to(torch.int32).expand(S, T).contiguous(), right=True)
        valid = seq < n
        seq = seq.clamp(max=n - 1)
        i = t - torch.gather(st["begin"].long(), 1, seq)
    else:
        seq = (t // st["rows"]).expand(S, T)
        i = (t % st["rows"]).expand(S, T)
        valid = i < torch.gather(st["new_len"].long(), 1, seq)
    back = i - torch.gather(st["new_len"].long(), 1, seq)
    return valid, seq, torch.gather(st["len"].long(), 1, seq) + back, torch.gather(st["seen"].long(), 1, seq) + back


def _plain_append(st):
    S, H, KV, D, page = st["S"], st["H"], st["KV"], st["D"], st["page"]
    T, per = st["tokens"], page // BLOCK
    valid, seq, slot, pos = _tokens(st)
    qk = st["qkv"][..., :(H + KV) * D].float().view(S, T, H + KV, D)
    qk = _rotate(qk, pos, st["freq"], st["rot"], st["layout"])
    st["q_out"].copy_(torch.where(valid[..., None], qk[:, :, :H].reshape(S, T, H * D).to(BF), st["q_out"]))
    s_of = torch.arange(S, device="cuda")[:, None].expand(S, T)
    s_of, seq, slot = s_of[valid], seq[valid], slot[valid]
    at = st["table"].long()[s_of, seq, slot // page] * per + slot % page // BLOCK      # block of the pool
    touched, which = torch.unique(at, return_inverse=True)
    row = slot % BLOCK
    first = torch.full((len(touched),), BLOCK, device="cuda").scatter_reduce(0, which, row, "amin")
    held = (torch.arange(BLOCK, device="cuda") < first[:, None])[:, None, :, None]     # rows that held tokens before
    for j, (name, x) in enumerate((("k", qk[:, :, H:][valid]), ("v", st["qkv"][..., (H + KV) * D:].view(S, T, KV, D)[valid].float()))):
        top = torch.zeros(len(touched), KV, device="cuda").index_reduce(0, which, _finite(x).amax(-1), "amax")
        scales = st["scales"][touched // per, :, touched % per, j]
        scale = torch.where(first[:, None] > 0, torch.maximum(scales, _need(top)), _need(top))
        cache = st[name].view(torch.uint8).view(-1, KV, per, BLOCK, D)
        old = cache[touched // per, :, touched % per].view(F8)
        again = _code(old.float() * scales[..., None, None], scale[..., None, None])
        block = torch.where(held, again.view(torch.uint8), old.view(torch.uint8))
        block[which, :, row] = _code(x, scale[which][..., None]).view(torch.uint8)
        cache[touched // per, :, touched % per] = block
        st["scales"][touched // per, :, touched % per, j] = scale
    return {"q": st["q_out"], "k": st["k"], "v": st["v"], "scales": st["scales"]}


def _values(st, name):
    """The cache's values [pool][KV][page][D] in 32 bits."""
    x = st[name]
    if st["scales"] is None:
        return x.float()
    s = st["scales"][..., 0 if name == "k" else 1]
    return (x.float().view(*s.shape, BLOCK, -1) * s[..., None, None]).view(x.shape)


def _rows(st, name):
    """[S][n][H][keys][D] of the KV position that each head reads."""
    S, n, H = st["S"], st["n_seqs"], st["H"]
    head = st["of"][:, None, :].expand(S, n, H)
    got = _values(st, name)[st["table"].long()[:, :, None, :], head[..., None]]
    return got.reshape(S, n, H, -1, st["D"])


def _scores(st):
    """[S][n][H][keys], minus infinity behind a sequence's end."""
    S, H, D, n = st["S"], st["H"], st["D"], st["n_seqs"]
    score = (st["q"].float().view(S, n, H, 1, D) @ _rows(st, "k").transpose(-1, -2)).squeeze(-2) * (D ** -0.5)
    live = torch.arange(score.shape[-1], device="cuda") < st["len"].long()[..., None, None]
    return torch.where(live, score, torch.full((), float("-inf"), device="cuda"))


def _plain_decode(st):
    S, H, D, n = st["S"], st["H"], st["D"], st["n_seqs"]
    score = _scores(st)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    o = (p[..., None, :] @ _rows(st, "v")).squeeze(-2) / torch.where(total > 0, total, torch.ones_like(total))
    st["out"].copy_(o.reshape(S, n, H * D).to(BF))
    st["lse"].copy_((torch.log(total) + top).squeeze(-1).transpose(1, 2))
    return {"out": st["out"], "lse": st["lse"]}


def _of_positions(st, x):
    """x [S][n][H][keys] added up over the heads that read a KV position: [S][n][KV][keys]; and which positions are read."""
    reads = torch.nn.functional.one_hot(st["of"], st["KV"]).float()                    # [S][H][KV]
    return torch.einsum("snhk,shp->snpk", x, reads), reads.sum(1) > 0


def _store(st, name, x, read, lens):
    """x [S][n][KV][keys] into the paged array `name`, for keys before the end and positions that heads read."""
    keys = torch.arange(x.shape[-1], device="cuda")
    live = (keys < lens.long()[..., None, None]) & read[:, None, :, None]
    s, b, p, k = live.nonzero(as_tuple=True)
    st[name][st["table"].long()[s, b, k // st["page"]], p, k % st["page"]] = x[s, b, p, k].to(st[name].dtype)


def _plain_weights(st):
    score = _scores(st)
    live = torch.isfinite(score)
    lse = st["lse"].transpose(1, 2)[..., None]
    p = torch.where(live, torch.exp(score - torch.where(live, lse, torch.zeros_like(lse))), torch.zeros((), device="cuda"))
    got, read = _of_positions(st, p)
    S, n = st["S"], st["n_seqs"]
    keys = torch.arange(got.shape[-1], device="cuda")
    fresh = (keys == st["len"].long()[..., None, None] - 1).expand(got.shape)          # the step's own token starts from nothing
    prior = st["prior"][st["table"].long()].transpose(2, 3).reshape(S, n, st["KV"], -1)
    _store(st, "weights", torch.where(fresh, got, prior + got), read, st["len"])
    s, b, pos = (fresh & (st["len"] > 0)[..., None, None] & read[:, None, :, None]).nonzero(as_tuple=True)[:3]
    k = st["len"].long()[s, b] - 1
    st["slot_pos"][st["table"].long()[s, b, k // st["page"]], pos, k % st["page"]] = st["seen"][s, b] - 1
    return {"weights": st["weights"], "slot_pos": st["slot_pos"]}


def _prompt_scores(st):
    """[S][n][H][query][key] of a prompt, minus infinity above the diagonal."""
    S, H, D, n, KV, N = st["S"], st["H"], st["D"], st["n_seqs"], st["KV"], st["longest"]
    x = st["qkv"].float().view(S, n, N, -1)
    q = x[..., :H * D].view(S, n, N, H, D).transpose(2, 3)
    k = x[..., H * D:(H + KV) * D].reshape(S, n, N, KV, D).transpose(2, 3)
    k = torch.gather(k, 2, st["of"][:, None, :, None, None].expand(S, n, H, N, D))
    i = torch.arange(N, device="cuda")
    return torch.where(i[:, None] >= i, q @ k.transpose(-1, -2) * (D ** -0.5), torch.full((), float("-inf"), device="cuda"))


def _plain_core(st):
    S, H, n, N = st["S"], st["H"], st["n_seqs"], st["longest"]
    i, length = torch.arange(N, device="cuda"), st["new_len"].long()[..., None]
    asks = (i < length) & (i >= length - (st["last"] or N))                            # [S][n][query]
    lse = st["lse"].view(S, H, n, N).transpose(1, 2)
    p = torch.exp(_prompt_scores(st) - lse[..., None])
    p = torch.where(asks[:, :, None, :, None], p, torch.zeros((), device="cuda")).sum(-2)
    got, read = _of_positions(st, p)
    _store(st, "weights", got, read, st["new_len"])
    _store(st, "slot_pos", i.expand(got.shape), read, st["new_len"])
    return {"weights": st["weights"], "slot_pos": st["slot_pos"]}


def _plain_evict(st):
    S, n, KV, D, page = st["S"], st["n_seqs"], st["KV"], st["D"], st["page"]
    table = st["table"].long()
    room = table.shape[-1] * page
    flat = lambda x: x[table].transpose(2, 3).reshape(S, n, KV, room)                  # a paged array by sequence
    w, pos = flat(st["weights"]), flat(st["slot_pos"])
    i = torch.arange(room, device="cuda")
    length, keep = (st[k].long()[..., None, None] for k in ("len", "keep"))
    held = (torch.arange(KV, device="cuda") < st["kv_count"][:, None])[:, None, :, None]
    guarded = pos >= st["seen"].long()[..., None, None] - keep.clamp(max=st["recent"])
    rank = torch.where(i < length, torch.where(guarded, float("inf"), w), -float("inf"))
    order = torch.argsort(rank, dim=-1, descending=True, stable=True)
    stays = torch.zeros(rank.shape, dtype=torch.bool, device="cuda").scatter_(-1, order, (i < keep).expand(rank.shape))
    stays &= i < length
    into = held & ~stays & (i < torch.minimum(keep, length))
    moves = held & stays & (i >= keep)
    number = into.cumsum(-1) - 1
    movers = torch.argsort(torch.where(moves, i, room + i), dim=-1)                    # ascending slots of those that move
    source = torch.where(into, torch.gather(movers, -1, number.clamp(min=0)), i.expand(into.shape))
    live = held & (i < torch.minimum(keep, length))
    s, b, p, k = live.nonzero(as_tuple=True)
    at, from_ = table[s, b, k // page], source[s, b, p, k]
    src = table[s, b, from_ // page]
    for name in ("weights", "slot_pos"):
        st[name + "_out"][at, p, k % page] = st[name][src, p, from_ % page]
    if not st["q8"]:
        s, b, p, k = into.nonzero(as_tuple=True)
        from_ = source[s, b, p, k]
        at, src = table[s, b, k // page], table[s, b, from_ // page]
        for name in ("k", "v"):
            st[name][at, p, k % page] = st[name][src, p, from_ % page]
        return _evicted(st)
    # blocks that take tokens in are coded anew, all their rows before the old end
    s, b, p, blk = into.view(S, n, KV, -1, BLOCK).any(-1).nonzero(as_tuple=True)
    k = blk[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    row = k < length[s, b, 0]
    from_ = source[s[:, None], b[:, None], p[:, None], k]
    src = table[s[:, None], b[:, None], from_ // page]
    at, line = table[s, b, blk * BLOCK // page], blk % (page // BLOCK)
    new = []
    for j, name in enumerate(("k", "v")):
        code = st[name].view(torch.uint8)[src, p[:, None], from_ % page].view(F8).float()
        x = code * st["scales"][src, p[:, None], from_ % page // BLOCK, j][..., None]
        scale = _need(torch.where(row[..., None], _finite(x), torch.zeros((), device="cuda")).amax((-1, -2)))
        cache = st[name].view(torch.uint8).view(-1, KV, page // BLOCK, BLOCK, D)
        new.append((cache, torch.where(row[..., None], _code(x, scale[:, None, None]).view(torch.uint8), cache[at, p, line]), scale))
    for j, (cache, block, scale) in enumerate(new):
        cache[at, p, line] = block
        st["scales"][at, p, line, j] = scale
    return _evicted(st)


_PLAIN = {"append": _plain_append, "decode": _plain_decode, "weights": _plain_weights, "core": _plain_core, "evict": _plain_evict}


# ------------------------------------------------------------------------------------------------ cost and exact values

def work(case):
    c = case
    S, D, n = c["S"], c["D"], c["n_seqs"]
    if c["op"] == "append":
        H, KV, new = c["H"], c["KV"], _new(c)
        blocks = sum(-(-a // BLOCK) for a in new)
        pages = sum(-(-a // c["page"]) for a in new)
        return {"bytes": sum(new) * D * (2 * (H + 2 * KV) + 2 * H + 2 * KV) + 8 * KV * blocks + 4 * (pages + 3 * S * n) + 8 * (c["rot"] // 2),
                "flops": sum(new) * ((H + KV) * c["rot"] * 3 + 2 * KV * D * 2)}
    lens = _lens(c)
    pages = sum(-(-v // c["page"]) for v in lens)
    if c["op"] == "evict":
        # a weight and a position of every slot, and of every one kept; the tokens that have to move: the recent ones behind
        # the budget, and of the others as many as chance puts there
        size = slots = kept = 0
        for i, v in enumerate(lens):
            held, keep = max(1, c["KV"] - (i // n) % 2), min(c["keep"], v)
            recent = min(c["recent"], keep)
            moved = min(recent, v - keep)
            if v - recent > keep:
                moved += (keep - recent) * (v - recent - keep) / (v - recent)
            size += held * moved * 2 * 2 * D * (1 if c["q8"] else 2)
            slots += held * v
            kept += held * keep
        return {"bytes": int(size) + 8 * slots + 8 * kept + 4 * (pages + 3 * S * n), "flops": slots}
    heads = _heads(c)
    per = c["NH"] // c["NKV"]
    held = [len({h // per for h in hs}) for hs in heads]
    H = c["H"]
    if c["op"] == "core":
        pairs = sum(v * (v + 1) // 2 - (max(0, v - c["last"]) * (max(0, v - c["last"]) + 1) // 2 if c["last"] else 0) for v in lens)
        rows = [sum(lens[s * n:(s + 1) * n]) for s in range(S)]
        size = sum(r * (H * (2 * D + 4) + g * (2 * D + 8)) for r, g in zip(rows, held))
        return {"bytes": size + 4 * (pages + S * n), "flops": pairs * H * (2 * D + 3)}
    keys = [sum(lens[s * n:(s + 1) * n]) for s in range(S)]
    slots = sum(k * g for k, g in zip(keys, held))
    index = S * n * H * 2 * D + 4 * (pages + S * n)
    if c["op"] == "weights":
        size = slots * (D + 4 / BLOCK if c["q8"] else 2 * D) + slots * 8
        return {"bytes": int(size) + index + 4 * S * n * H, "flops": sum(keys) * H * (2 * D + 3)}
    return {"bytes": int(slots * (2 * D + 8 / BLOCK)) + index + S * n * H * (2 * D + 4), "flops": sum(keys) * H * 4 * D}


def _power(a):
    """Exponent of the scale that values up to `a` (a number) need."""
    e = LOW
    while e < HIGH and a > 448 * 2.0 ** e:
        e += 1
    return e


def _powers(a):
    return torch.tensor([2.0 ** _power(v) for v in a.tolist()], dtype=torch.float64, device="cuda")


def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    S, D, n, page = st["S"], st["D"], st["n_seqs"], st["page"]
    return {"append": _exact_append, "decode": _exact_decode, "weights": _exact_weights, "core": _exact_core,
            "evict": _exact_evict}[st["op"]](st, f64, S, D, n, page)


def _exact_append(st, f64, S, D, n, page):
    H, KV, rot, half = st["H"], st["KV"], st["rot"], st["rot"] // 2
    if S * n > 600:                 # the loops below would take long
        return None

    def turn(x, pos):               # x [rows][heads][D] in 64 bits; pairs as complex numbers times exp(i angle)
        w = torch.polar(torch.ones((), dtype=f64, device=x.device).expand(len(pos), half), pos.to(f64)[:, None] * st["freq"][None, :])[:, None]
        x = x.clone()
        lo, hi = (slice(0, half), slice(half, rot)) if st["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(x[..., lo], x[..., hi]) * w
        x[..., lo], x[..., hi] = z.real, z.imag
        return x

    q, k, v, scales = (st[name].to(f64) for name in ("q_out", "k", "v", "scales"))
    begin, new, lens, seen, table = (st[name].tolist() for name in ("begin", "new_len", "len", "seen", "table"))
    for s in range(S):
        for b in range(n):
            m = new[s][b]
            if m == 0:
                continue
            r0 = begin[s][b] if st["form"] == "packed" else b * st["rows"]
            z = st["qkv"][s, r0:r0 + m].to(f64).view(m, H + 2 * KV, D)
            z[:, :H + KV] = turn(z[:, :H + KV], torch.arange(seen[s][b] - m, seen[s][b], device="cuda"))
            q[s, r0:r0 + m] = z[:, :H].reshape(m, -1)
            at = lens[s][b] - m
            done = 0
            while done < m:         # block by block
                slot = at + done
                take, row, pg = min(m - done, BLOCK - slot % BLOCK), slot % page, table[s][b][slot // page]
                lo = row - row % BLOCK
                for j, cache in enumerate((k, v)):
                    x = z[done:done + take, H + j * KV:H + (j + 1) * KV]
                    e = _powers(x.abs().amax((0, 2)))
                    if slot % BLOCK:
                        e = torch.maximum(e, scales[pg, :, lo // BLOCK, j])
                        cache[pg, :, lo:row] *= (scales[pg, :, lo // BLOCK, j] / e)[:, None, None]
                    scales[pg, :, lo // BLOCK, j] = e
                    cache[pg, :, row:row + take] = x.transpose(0, 1) / e[:, None, None]
                done += take
    return {"q": q, "k": k, "v": v, "scales": scales}


def _sequence(st, name, s, b, m, f64):
    """[KV][m][D]: a sequence's cached values in 64 bits."""
    pages = st["table"][s, b, :-(-m // st["page"])].long()
    x = st[name][pages].to(f64)
    if st["scales"] is not None:
        x = x * st["scales"][pages, :, :, 0 if name == "k" else 1].to(f64).repeat_interleave(BLOCK, -1)[..., None]
    return x.permute(1, 0, 2, 3).reshape(st["KV"], -1, st["D"])[:, :m]


def _exact_decode(st, f64, S, D, n, page):
    H = st["H"]
    out = torch.zeros(S, n, H * D, dtype=f64, device="cuda")
    lse = torch.full((S, H, n), float("-inf"), dtype=f64, device="cuda")
    lens = st["len"].tolist()
    for s in range(S):
        for b in range(n):
            m = lens[s][b]
            if m == 0:
                continue
            k, v = _sequence(st, "k", s, b, m, f64), _sequence(st, "v", s, b, m, f64)
            q = st["q"][s, b].to(f64).view(H, D)
            step = max(1, (1 << 27) // (m * D))       # heads at a time
            for h in range(0, H, step):
                g = st["of"][s, h:h + step]
                x = torch.einsum("hkd,hd->hk", k[g], q[h:h + step]) / D ** 0.5
                lse[s, h:h + step, b] = torch.logsumexp(x, 1)
                out[s, b].view(H, D)[h:h + step] = torch.einsum("hk,hkd->hd", torch.softmax(x, 1), v[g])
    return {"out": out, "lse": lse}


def _put(st, into, s, b, p, x):
    """x [m] into position p of a sequence's slots."""
    k = torch.arange(len(x), device="cuda")
    into[st["table"][s, b].long()[k // st["page"]], p, k % st["page"]] = x.to(into.dtype)


def _exact_weights(st, f64, S, D, n, page):
    H = st["H"]
    weights, pos = st["weights"].to(f64), st["slot_pos"].clone()
    lens, of = st["len"].tolist(), st["of"].tolist()
    for s in range(S):
        for b in range(n):
            m = lens[s][b]
            if m == 0:
                continue
            k = _sequence(st, "k", s, b, m, f64)
            at = torch.arange(m, device="cuda")
            pages = st["table"][s, b].long()[at // page]
            for p in sorted(set(of[s])):
                heads = [h for h in range(H) if of[s][h] == p]
                x = st["q"][s, b].to(f64).view(H, D)[heads] @ k[p].T / D ** 0.5
                w = torch.exp(x - st["lse"][s, heads, b].to(f64)[:, None]).sum(0)
                w[:-1] += st["prior"][pages, p, at % page].to(f64)[:-1]
                weights[pages, p, at % page] = w
                pos[pages[-1], p, at[-1] % page] = st["seen"][s, b] - 1
    return {"weights": weights, "slot_pos": pos}


def _exact_core(st, f64, S, D, n, page):
    H, KV, N = st["H"], st["KV"], st["longest"]
    weights, pos = st["weights"].to(f64), st["slot_pos"].clone()
    lens, of = st["new_len"].tolist(), st["of"].tolist()
    for s in range(S):
        for b in range(n):
            m = lens[s][b]
            if m == 0:
                continue
            x = st["qkv"][s, b * N:b * N + m].to(f64)
            first = max(0, m - st["last"]) if st["last"] else 0
            i = torch.arange(m, device="cuda")
            for p in sorted(set(of[s])):
                w = torch.zeros(m, dtype=f64, device="cuda")
                k = x[:, (H + p) * D:(H + p + 1) * D]
                for h in (h for h in range(H) if of[s][h] == p):
                    y = x[first:, h * D:(h + 1) * D] @ k.T / D ** 0.5 - st["lse"][s, h, b * N + first:b * N + m].to(f64)[:, None]
                    w += torch.exp(y).masked_fill_(i > i[first:, None], 0).sum(0)
                _put(st, weights, s, b, p, w)
                _put(st, pos, s, b, p, i)
    return {"weights": weights, "slot_pos": pos}


def _exact_evict(st, f64, S, D, n, page):
    k_v = [st["k"].to(f64), st["v"].to(f64)]
    scales = st["scales"].to(f64) if st["q8"] else None
    weights, pos = st["weights_out"].to(f64), st["slot_pos_out"].clone()
    lens, keeps, seen, held = (st[name].tolist() for name in ("len", "keep", "seen", "kv_count"))
    if sum(map(sum, lens)) * st["KV"] > 4_000_000 or S * n * st["KV"] > 600:
        return None
    for s in range(S):
        for b in range(n):
            m, keep = lens[s][b], keeps[s][b]
            pages, at = st["table"][s, b].long(), torch.arange(m, device="cuda")
            for p in range(held[s]):
                if m == 0:
                    continue
                w, where = st["weights"][pages[at // page], p, at % page], st["slot_pos"][pages[at // page], p, at % page]
                guarded = (where >= seen[s][b] - min(st["recent"], keep)).tolist()
                w_ = w.tolist()
                best = sorted(range(m), key=lambda i: (not guarded[i], 0.0 if guarded[i] else -w_[i], i))[:keep]
                there = [False] * m
                for i in best:
                    there[i] = True
                source = list(range(min(keep, m)))
                movers = iter([i for i in range(keep, m) if there[i]])
                taken = [i for i in range(min(keep, m)) if not there[i]]
                for i in taken:
                    source[i] = next(movers)
                src = torch.tensor(source, device="cuda", dtype=torch.int64)
                _put(st, weights, s, b, p, w[src])
                _put(st, pos, s, b, p, where[src])
                if not taken:
                    continue
                if not st["q8"]:
                    t = torch.tensor(taken, device="cuda")
                    for x in k_v:
                        x[pages[t // page], p, t % page] = x[pages[src[t] // page], p, src[t] % page]
                    continue
                whole = torch.arange(m, device="cuda")
                whole[:len(source)] = src
                blocks = torch.tensor(sorted({i // BLOCK for i in taken}), device="cuda")
                for j, x in enumerate(k_v):
                    true = x[pages[at // page], p, at % page] * scales[pages[at // page], p, at % page // BLOCK, j][:, None]
                    pad = torch.zeros(-(-m // BLOCK) * BLOCK, D, dtype=f64, device="cuda")
                    pad[:m] = true[whole]
                    rows = pad.view(-1, BLOCK, D)[blocks]
                    e = _powers(rows.abs().amax((1, 2)))
                    t = (blocks[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")).reshape(-1)
                    live = t < m
                    val = (rows / e[:, None, None]).reshape(-1, D)[live]
                    t = t[live]
                    x[pages[t // page], p, t % page] = val
                    scales[pages[blocks * BLOCK // page], p, blocks * BLOCK % page // BLOCK, j] = e
    out = {"k": k_v[0], "v": k_v[1], "weights": weights, "slot_pos": pos}
    return dict(out, scales=scales) if st["q8"] else out
