"""Measured cases of the serving and training operators around attention.

Four operators: the per-head norm of queries and keys with the rotation of positions in the same
pass ("norm"), its gradients ("norm_bwd"), the paged 4-bit cache of keys and values written and
read back ("cache"), and attention over that cache ("attn").  A case is a dict of plain values;
prepare() makes its inputs on the GPU from a seed, run() makes one pass: in elementary torch
operations in 32 bits where `own` is false, through the framework's entry points where it is true.
exact() gives the same outputs from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6
GROUP = 32     # features that share one scale in the cache
BLOCK = 16     # tokens of one cache block


# ---------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # one decoding step of a few sequences: the shortest call, all latency
        dict(name="norm_step", op="norm", dtype="bf16", B=8, Hq=16, Hk=4, N=1, d=64, rot=64,
             style="half", P=4096),
        # a training batch with as many key heads as query heads
        dict(name="norm_train_d64", op="norm", dtype="bf16", B=4, Hq=16, Hk=16, N=2048, d=64,
             rot=64, style="half", P=2048),
        # single precision, an odd length, part of each head rotated in neighbouring pairs
        dict(name="norm_odd_fp32", op="norm", dtype="fp32", B=3, Hq=10, Hk=2, N=1021, d=96,
             rot=32, style="pairs", P=5000),
        # gradients of a long training batch with shared key heads: the largest of its kind
        dict(name="bwd_long_d128", op="norm_bwd", dtype="bf16", B=2, Hq=32, Hk=8, N=8192, d=128,
             rot=128, style="half", P=8192),
        # gradients in single precision at an odd length
        dict(name="bwd_odd_fp32", op="norm_bwd", dtype="fp32", B=2, Hq=6, Hk=3, N=517, d=128,
             rot=64, style="pairs", P=1000),
        # every sequence of a serving batch appends one token to the cache
        dict(name="cache_step", op="cache", dtype="bf16", B=64, Hk=8, N=1, dk=128, dv=128,
             page=64, L=4000),
        # long prompts go into the cache and are read back
        dict(name="cache_prompt", op="cache", dtype="bf16", B=3, Hk=8, N=16001, dk=128, dv=128,
             page=32, L=16384),
        # one short conversation, one token: latency
        dict(name="attn_one", op="attn", dtype="bf16", B=1, Hq=16, Hk=4, N=1, dk=128, dv=128,
             page=16, L=1000, causal=True),
        # a serving batch of uneven lengths, the empty and the one-token sequence among them
        dict(name="attn_batch", op="attn", dtype="bf16", B=48, Hq=32, Hk=8, N=1, dk=128, dv=128,
             page=64, L=16384, causal=True),
        # two very long contexts, eight queries to a key head
        dict(name="attn_long", op="attn", dtype="bf16", B=2, Hq=64, Hk=8, N=1, dk=128, dv=128,
             page=128, L=131072, causal=True),
        # a chunk of a prompt against what is cached before it: the most arithmetic
        dict(name="attn_chunk", op="attn", dtype="bf16", B=1, Hq=32, Hk=8, N=2048, dk=128, dv=128,
             page=64, L=16384, causal=True),
        # a few draft tokens verified in single precision, odd page size, narrow values
        dict(name="attn_draft_fp32", op="attn", dtype="fp32", B=5, Hq=12, Hk=4, N=5, dk=128,
             dv=64, page=48, L=3001, causal=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_bwd", "cache", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op in ("norm", "norm_bwd"):
        d = rng.choice([64, 96, 128, 128])
        rot = rng.choice([d, d, 32])
        Hk = rng.choice([1, 2, 4, 8])
        Hq = Hk * rng.choice([1, 3, 4])
        N = _log(rng, 1, 8192)
        most = (1 << 26) // (2 * (Hq + Hk) * d * N)     # about the elements of the largest case
        B = _log(rng, 1, max(1, min(32, most)))
        return dict(op=op, dtype=dtype, B=B, Hq=Hq, Hk=Hk, N=N, d=d, rot=rot,
                    style=rng.choice(["half", "pairs"]), P=N + rng.randrange(1, 3000))
    dk, dv = rng.choice([(64, 64), (128, 128), (128, 128), (128, 64)])
    page = rng.choice([16, 32, 48, 64, 128, 256])
    Hk = rng.choice([1, 2, 4, 8])
    if op == "cache":
        N = _log(rng, 1, 16000)
        B = _log(rng, 1, max(1, min(64, 48000 // N)))
        return dict(op=op, dtype=dtype, B=B, Hk=Hk, N=N, dk=dk, dv=dv, page=page,
                    L=N + rng.randrange(1, 2000))
    G = rng.choice([1, 2, 4, 5, 8])
    if rng.random() < 0.75:                              # decoding: few queries, any context
        N = rng.choice([1, 1, 1, 2, 4])
        L = _log(rng, 100, 65536)
        B = _log(rng, 1, max(1, min(64, 262144 // L)))
    else:                                                # a chunk of a prompt
        dtype = "bf16"
        N = _log(rng, 16, 2048)
        L = N + _log(rng, 100, 14000)
        B = _log(rng, 1, max(1, min(8, (1 << 25) // (N * L))))
    return dict(op=op, dtype=dtype, B=B, Hq=Hk * G, Hk=Hk, N=N, dk=dk, dv=dv, page=page, L=L,
                causal=rng.random() < 0.8)


def _lens(case):
    """The lengths of the case's sequences: one of the full length, an empty one and one of a
    single token in larger batches, the others spread between a sixteenth of it and the whole."""
    B, L = case["B"], case["L"]
    rng = random.Random(B * 1000003 + L)
    lens = [L] + [_log(rng, max(1, L // 16), L) for _ in range(B - 1)]
    if B >= 8:
        lens[1], lens[2] = 0, 1
    return lens


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------
def _rand(gen, *shape, dtype=torch.float32, scale=1.0):
    x = torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)
    return (x * scale if scale != 1.0 else x).to(dtype)


def _angles(P, rot):
    """cos and sin of position * 10000^(-2 i / rot), from 64 bits, [P, rot / 2]."""
    i = torch.arange(rot // 2, device=DEV, dtype=torch.float64)
    a = torch.arange(P, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * i / rot)
    return a.cos().float(), a.sin().float()


def _pages(gen, lens, page, L):
    """A table of shuffled pages for sequences of up to L tokens, and how many pages there are:
    the last one belongs to no sequence.  Places past a sequence's last page hold -1."""
    per = [-(-n // page) for n in lens]
    width = max(1, -(-L // page))
    order = torch.randperm(sum(per), generator=gen, device=DEV).to(torch.int32)
    first = torch.tensor([sum(per[:b]) for b in range(len(per))], device=DEV)
    count = torch.tensor(per, device=DEV)
    at = torch.arange(width, device=DEV)
    live = at[None] < count[:, None]
    where = (first[:, None] + at[None]).clamp(max=max(0, sum(per) - 1))
    table = torch.where(live, order[where] if sum(per) else torch.zeros_like(where, dtype=torch.int32),
                        torch.full_like(where, -1, dtype=torch.int32))
    return table.to(torch.int32).contiguous(), sum(per) + 1


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dt, B, N = TYPES[case["dtype"]], case["B"], case["N"]
    s = {"op": case["op"], "case": dict(case), "dtype": dt}
    if case["op"] in ("norm", "norm_bwd"):
        Hq, Hk, d = case["Hq"], case["Hk"], case["d"]
        # projections of a trained layer: heads of different sizes, weights near one
        head = torch.exp(0.5 * _rand(gen, Hq + Hk, 1, 1))
        s["q"] = (_rand(gen, B, Hq, N, d) * head[:Hq]).to(dt)
        s["k"] = (_rand(gen, B, Hk, N, d) * head[Hq:]).to(dt)
        s["wq"], s["wk"] = (1.0 + 0.2 * _rand(gen, d)).to(dt), (1.0 + 0.2 * _rand(gen, d)).to(dt)
        s["cos"], s["sin"] = _angles(case["P"], case["rot"])
        start = torch.randint(0, case["P"] - N + 1, (B, 1), generator=gen, device=DEV)
        s["pos"] = (start + torch.arange(N, device=DEV)).to(torch.int32)
        if case["op"] == "norm_bwd":
            s["dq"] = _rand(gen, B, Hq, N, d, dtype=dt, scale=0.01)
            s["dk"] = _rand(gen, B, Hk, N, d, dtype=dt, scale=0.01)
        return s
    Hk, dk, dv, page, L = case["Hk"], case["dk"], case["dv"], case["page"], case["L"]
    if case["op"] == "cache":
        s["table"], n = _pages(gen, [L] * B, page, L)
        s["pool"] = torch.zeros(n, Hk, page // BLOCK, 9 * (dk + dv), dtype=torch.uint8, device=DEV)
        start = torch.randint(0, L - N + 1, (B, 1), generator=gen, device=DEV)
        s["pos"] = (start + torch.arange(N, device=DEV)).to(torch.int32)
        channel = torch.exp(0.5 * _rand(gen, Hk, 1, dk))     # some key channels are larger
        s["k"] = (_rand(gen, B, Hk, N, dk) * channel).to(dt)
        s["v"] = _rand(gen, B, Hk, N, dv, dtype=dt)
        return s
    lens = _lens(case)
    order = torch.randperm(B, generator=gen, device=DEV).tolist()
    lens = [lens[i] for i in order]
    s["table"], n = _pages(gen, lens, page, L)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    channel = torch.exp(0.3 * _rand(gen, Hk, 1, dk))
    k = _rand(gen, n, Hk, page, dk) * channel
    v = _rand(gen, n, Hk, page, dv)
    # what lies past a sequence's end is whatever the page held before: here, not numbers at all
    end = (torch.tensor([n_ - 1 for n_ in lens], device=DEV).clamp(min=0) // page)[:, None]
    last = s["table"].long().gather(1, end)[:, 0]
    for b, length in enumerate(lens):
        if length % page:
            k[last[b], :, length % page:] = float("nan")
            v[last[b], :, length % page:] = float("nan")
    s["pool"] = _pack(_quantise(k), _quantise(v))
    s["q"] = _rand(gen, B, case["Hq"], N, dk, dtype=dt, scale=1.5)
    return s


# ---------------------------------------------------------------------------------------------
# The cache's format, in elementary operations
# ---------------------------------------------------------------------------------------------
def _quantise(x):
    """(codes + 8 as uint8, scales in bf16) of [..., d]: 32 neighbouring features share the scale
    bf16(max / 7), a feature is rint(x / scale) in [-7, 7]."""
    x = x.float().unflatten(-1, (-1, GROUP))
    m = x.abs().amax(-1, keepdim=True)
    scale = (m / torch.full_like(m, 7.0)).to(torch.bfloat16)
    scale = torch.where(torch.isfinite(m), scale, torch.full_like(scale, float("nan")))
    code = torch.round(x / scale.float()).clamp(-7.0, 7.0)
    code = torch.where(torch.isfinite(m) & (scale != 0), code, torch.zeros_like(code))
    return (code + 8.0).to(torch.uint8).flatten(-2), scale.squeeze(-1)


def _halfwords(code, value):
    """Codes [..., d] of one token as its 16-bit words in a block's order: [..., d / 4] int16.
    Keys: chunk t of 4, group, then the even and the odd four of eight features 32 g + 8 t + e.
    Values: eight chunks of four features 4 c .. 4 c + 3 of each group."""
    c = code.to(torch.int32).unflatten(-1, (-1, 4, 8))               # group, t, e
    if value:
        c = c.flatten(-2).unflatten(-1, (8, 4)).transpose(-3, -2)    # c, group, feature
    else:
        c = c.transpose(-3, -2).unflatten(-1, (4, 2)).transpose(-2, -1)  # t, group, odd, e / 2
    w = c[..., 0] | c[..., 1] << 4 | c[..., 2] << 8 | c[..., 3] << 12
    return torch.where(w >= 32768, w - 65536, w).to(torch.int16).flatten(-3 if not value else -2)


def _places(dk, dv, device):
    """Where a token's 16-bit words lie in a block, by token: for key codes, value codes, key
    scales and value scales, [16, words]."""
    t = torch.arange(BLOCK, device=device)[:, None]
    nk, nv = dk // 4, dv // 4
    kw = torch.arange(nk, device=device)[None] + t * nk
    w = torch.arange(nv, device=device)[None]
    c, g, groups = w // (nv // 8), w % (nv // 8), nv // 8
    chunk = (t // 8 * 8 + c) * 4 + t % 8 // 2
    vw = BLOCK * nk + (chunk * groups + g) * 2 + t % 2
    ks = BLOCK * (nk + nv) + t * (nk // 8) + torch.arange(nk // 8, device=device)[None]
    vs = BLOCK * (nk + nv + nk // 8) + t * groups + torch.arange(groups, device=device)[None]
    return kw, vw, ks, vs


def _pack(kq, vq):
    """The pool [pages, heads, blocks, bytes] of quantised keys and values [pages, heads, page, d]."""
    (kc, ks), (vc, vs) = kq, vq
    n, H, page, dk = kc.shape
    dv = vc.shape[-1]
    pool = torch.empty(n, H, page // BLOCK, 9 * (dk + dv) // 2, dtype=torch.int16, device=kc.device)
    words = (_halfwords(kc, False), _halfwords(vc, True), ks.view(torch.int16), vs.view(torch.int16))
    for at, w in zip(_places(dk, dv, kc.device), words):
        pool[..., at.flatten()] = w.unflatten(2, (-1, BLOCK)).flatten(-2)
    return pool.view(torch.uint8)


def _codes(words, value):
    """The codes [..., d] of a token's 16-bit words (the reverse of _halfwords)."""
    w = words.to(torch.int32) & 0xFFFF
    c = torch.stack([w & 15, w >> 4 & 15, w >> 8 & 15, w >> 12], -1)
    if value:
        return c.unflatten(-2, (8, -1)).transpose(-3, -2).flatten(-3) - 8
    return c.unflatten(-2, (4, -1, 2)).transpose(-4, -3).transpose(-2, -1).flatten(-4) - 8


def _values(words, scales, value):
    c = _codes(words, value).float().unflatten(-1, (-1, GROUP))
    return (c * scales.contiguous().view(torch.bfloat16).float()[..., None]).flatten(-2)


def _gather(pool, table, dk, dv):
    """Keys and values [B, H, tokens, d] in 32 bits of all pages that the table names (places that
    hold -1 read page 0)."""
    p = pool.view(torch.int16)[table.long().clamp(min=0)].transpose(1, 2)   # B, H, pages, blocks, words
    kw, vw, ks, vs = (p[..., at] for at in _places(dk, dv, pool.device))
    return _values(kw, ks, False).flatten(2, 4), _values(vw, vs, True).flatten(2, 4)


# ---------------------------------------------------------------------------------------------
# The operators in plain form
# ---------------------------------------------------------------------------------------------
def _pairs(x, rot, style):
    """The two members of each rotated pair, [..., rot / 2]."""
    if style == "half":
        return x[..., :rot // 2], x[..., rot // 2:rot]
    return x[..., 0:rot:2], x[..., 1:rot:2]


def _unpair(a, b, rest, style):
    front = torch.cat([a, b], -1) if style == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([front, rest], -1) if rest.shape[-1] else front


def _norm(x, w, c, s, rot, style):
    x = x.float()
    u = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    a, b = _pairs(u, rot, style)
    return _unpair(a * c - b * s, b * c + a * s, u[..., rot:], style)


def _norm_bwd(x, w, c, s, g, rot, style):
    x, g, w = x.float(), g.float(), w.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    a, b = _pairs(g, rot, style)
    t = _unpair(a * c + b * s, b * c - a * s, g[..., rot:], style)
    wt = w * t
    return r * (wt - n * (wt * n).mean(-1, keepdim=True)), (t * n).sum((0, 1, 2))


def _plain_norm(s):
    rot, style, dt = s["case"]["rot"], s["case"]["style"], s["dtype"]
    c, n = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    if s["op"] == "norm":
        return [_norm(s["q"], s["wq"], c, n, rot, style).to(dt), _norm(s["k"], s["wk"], c, n, rot, style).to(dt)]
    dq, dwq = _norm_bwd(s["q"], s["wq"], c, n, s["dq"], rot, style)
    dk, dwk = _norm_bwd(s["k"], s["wk"], c, n, s["dk"], rot, style)
    return [dq.to(dt), dk.to(dt), dwq, dwk]


def _plain_cache(s):
    dk, dv, page = s["case"]["dk"], s["case"]["dv"], s["case"]["page"]
    H = s["k"].shape[1]
    pos = s["pos"].long()
    where = s["table"].long().gather(1, pos // page)
    blocks = page // BLOCK
    # the 16-token block of each token and head, [B, H, N, 1], and the token's place in it
    at = ((where[:, None] * H + torch.arange(H, device=DEV)[:, None]) * blocks + (pos % page // BLOCK)[:, None])[..., None]
    place = [p[pos % BLOCK][:, None] + at * (9 * (dk + dv) // 2) for p in _places(dk, dv, DEV)]
    pool = s["pool"].view(torch.int16).view(-1)
    (kc, ks), (vc, vs) = _quantise(s["k"]), _quantise(s["v"])
    pool[place[0]], pool[place[1]] = _halfwords(kc, False), _halfwords(vc, True)
    pool[place[2]], pool[place[3]] = ks.view(torch.int16), vs.view(torch.int16)
    k, v = _values(pool[place[0]], pool[place[2]], False), _values(pool[place[1]], pool[place[3]], True)
    return [k.to(s["dtype"]), v.to(s["dtype"])]


def _plain_attn(s):
    case = s["case"]
    B, N, Hk, dk, dv = case["B"], case["N"], case["Hk"], case["dk"], case["dv"]
    G = case["Hq"] // Hk
    k, v = _gather(s["pool"], s["table"], dk, dv)
    T = k.shape[2]
    key = torch.arange(T, device=DEV)
    v = torch.where((key[None] < s["lens"][:, None])[:, None, :, None], v, torch.zeros((), device=DEV))
    # the last position that a query may see
    upto = s["lens"][:, None] - 1 + torch.zeros(1, N, dtype=torch.int64, device=DEV)
    if case["causal"]:
        upto = upto - (N - 1) + torch.arange(N, device=DEV)[None]
    seen = (key[None, None] <= upto[..., None])[:, None]                 # B, 1, N, T
    p = torch.matmul(s["q"].float().view(B, Hk, G * N, dk), k.transpose(-2, -1)) / math.sqrt(dk)
    p = torch.where(seen, p.view(B, Hk * G, N, T), torch.full((), -math.inf, device=DEV))
    m = p.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(p - torch.where(m == -math.inf, torch.zeros_like(m), m)), torch.zeros((), device=DEV))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hk, G * N, T), v).view(B, Hk * G, N, dv)
    return (o / torch.where(total == 0, torch.ones_like(total), total)).to(s["dtype"])


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------
def run(state):
    s = state
    if not own:
        return {"norm": _plain_norm, "norm_bwd": _plain_norm, "cache": _plain_cache, "attn": _plain_attn}[s["op"]](s)
    import paper_2606_07713_gb300 as moa
    if s["op"] == "norm":
        return moa.qk_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["pos"], eps=EPS,
                                interleaved=s["case"]["style"] == "pairs")
    if s["op"] == "norm_bwd":
        return moa.qk_norm_rope_bwd(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["pos"], s["dq"],
                                    s["dk"], eps=EPS, interleaved=s["case"]["style"] == "pairs")
    if s["op"] == "cache":
        moa.kv4_write(s["k"], s["v"], s["pool"], s["table"], s["pos"])
        return moa.kv4_read(s["pool"], s["table"], s["pos"], s["case"]["dk"], dtype=s["dtype"])
    return moa.kv4_attn(s["q"], s["pool"], s["table"], s["lens"], max_len=s["case"]["L"], causal=s["case"]["causal"])


# ---------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    B, N = case["B"], case["N"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("norm", "norm_bwd"):
        rows, d = B * N * (case["Hq"] + case["Hk"]), case["d"]
        table = min(B * N, case["P"]) * case["rot"] * 4 + 4 * B * N
        if case["op"] == "norm":
            return {"bytes": 2 * rows * d * size + table + 2 * d * size, "flops": 7 * rows * d}
        return {"bytes": 3 * rows * d * size + table + 2 * d * (size + 4), "flops": 14 * rows * d}
    d = case["dk"] + case["dv"]
    if case["op"] == "cache":
        rows = B * N * case["Hk"]
        return {"bytes": rows * d * (2 * size + 2 * 9 / 16) + 4 * B * N, "flops": 5 * rows * d}
    held = pairs = 0
    for n in _lens(case):
        held += n
        if case["causal"]:
            first = max(0, n - N + 1)                    # keys of the first query that sees any
            rows = min(N, n)
            pairs += rows * (max(first, 1) + n) // 2 if rows else 0
        else:
            pairs += N * n
    return {"bytes": held * case["Hk"] * d * 9 / 16 + B * N * case["Hq"] * d * size + held // case["page"] * 4 + 4 * B,
            "flops": 2 * case["Hq"] * pairs * d}


# ---------------------------------------------------------------------------------------------
# The same outputs from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_norm(case, s):
    rot, half = case["rot"], case["rot"] // 2
    i = torch.arange(half, device=DEV)
    first, second = (i, i + half) if case["style"] == "half" else (2 * i, 2 * i + 1)
    angle = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].long()][:, None]
    got = []
    for x, w, g in ((s["q"], s["wq"], s.get("dq")), (s["k"], s["wk"], s.get("dk"))):
        x, w = x.double(), w.double()
        d = x.shape[-1]
        root = (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt()

        def turn(y, by):
            z = torch.complex(y[..., first], y[..., second]) * by
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
            return y

        if g is None:
            got.append(turn(x / root * w, angle))
            continue
        t = turn(g.double(), angle.conj())
        a = t * w
        got.append((a / root - x * (a * x).sum(-1, keepdim=True) / (d * root.pow(3)), (t * x / root).sum((0, 1, 2))))
    return got if case["op"] == "norm" else [got[0][0], got[1][0], got[0][1], got[1][1]]


def _exact_cache(s):
    got = []
    for x in (s["k"], s["v"]):
        y = x.double().reshape(*x.shape[:-1], -1, GROUP)
        scale = (y.abs().max(-1, keepdim=True).values / 7).to(torch.bfloat16).double()
        got.append((torch.round(y / scale).clamp(-7, 7) * scale).reshape(x.shape))
    return got


def _exact_read(block, dk, dv):
    """Keys [16, dk] and values [16, dv] in 64 bits of blocks [..., bytes], feature by feature."""
    def nibble(byte, high):
        x = block[..., byte].to(torch.int64)
        return torch.where(high, x >> 4, x & 15).double() - 8

    def bf16(byte):
        return (block[..., byte].to(torch.int32) << 16 | block[..., byte + 1].to(torch.int32) << 24).view(torch.float32).double()

    t = torch.arange(BLOCK, device=DEV)[:, None]
    out, base = [], BLOCK * (dk + dv) // 2
    for d, value in ((dk, False), (dv, True)):
        f = torch.arange(d, device=DEV)[None]
        g, e = f // GROUP, f % GROUP
        if value:
            word = (((t // 8) * 8 + e // 4) * 4 + t % 8 // 2) * (d // GROUP) + g
            bit = 16 * (t % 2) + 4 * (e % 4)
            start = BLOCK * dk // 2
        else:
            word = (t * 4 + e // 8) * (d // GROUP) + g
            bit = 16 * (e % 2) + 4 * (e % 8 // 2)
            start = 0
        code = nibble(start + word * 4 + bit // 8, bit % 8 == 4)
        out.append(code * bf16(base + 2 * (t * (d // GROUP) + g)))
        base += 2 * BLOCK * (d // GROUP)
    return out


def _exact_attn(case, s):
    N, G, page = case["N"], case["Hq"] // case["Hk"], case["page"]
    o = torch.zeros(case["B"], case["Hq"], N, case["dv"], dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        if not n:
            continue
        pages = s["table"][b, :-(-n // page)].long()
        for h in range(case["Hk"]):
            k, v = _exact_read(s["pool"][pages, h], case["dk"], case["dv"])
            k, v = k.reshape(-1, case["dk"])[:n], v.reshape(-1, case["dv"])[:n]
            for j in range(h * G, h * G + G):
                score = s["q"][b, j].double() @ k.T * case["dk"] ** -0.5
                if case["causal"]:
                    late = torch.arange(n, device=DEV)[None] > torch.arange(n - N, n, device=DEV)[:, None]
                    score = score.masked_fill(late, -math.inf)
                o[b, j] = torch.nan_to_num(torch.softmax(score, -1), nan=0.0) @ v
    return o


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "norm_bwd"):
        return _exact_norm(case, s)
    return _exact_cache(s) if case["op"] == "cache" else _exact_attn(case, s)
