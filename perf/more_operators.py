"""Measured cases of windowed attention and of the 16- and 32-bit paged cache.

Four operators: causal attention with a sliding window and a few first tokens that stay visible
("fwd"), its gradients ("bwd"), new keys and values appended to a paged cache with the rotation of
their positions, queries rotated beside them ("append"), and attention of new tokens over that cache
("attn").  A case is a dict of plain values; prepare() makes its inputs on the GPU from a seed, run()
makes one pass: in elementary torch operations in 32 bits where `own` is false, through the
framework's entry points where it is true.  exact() gives the same outputs from the definitions in 64
bits.

Visibility, the same everywhere: of a sequence's L tokens the N queries are the last N, query i stands
at position p = L - N + i and sees token j if j <= p (causal), and j > p - W or j < S: W is the window
(0: none), S the number of first tokens that stay visible.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # a long document in training or prefill, four query heads to a key head: the most arithmetic
        dict(name="fwd_long", op="fwd", dtype="bf16", B=1, Hq=32, Hk=8, N=32768, M=32768, dk=128, dv=128, W=4096, S=4),
        # a training batch of a causal layer without a window, as many key heads as query heads
        dict(name="fwd_causal_d64", op="fwd", dtype="bf16", B=4, Hq=16, Hk=16, N=2048, M=2048, dk=64, dv=64, W=0, S=0),
        # single precision, an odd length, more keys than queries, narrow values
        dict(name="fwd_odd_fp32", op="fwd", dtype="fp32", B=2, Hq=6, Hk=3, N=517, M=700, dk=128, dv=64, W=100, S=3),
        # gradients of a windowed layer with shared key heads
        dict(name="bwd_long", op="bwd", dtype="bf16", B=2, Hq=32, Hk=8, N=8192, M=8192, dk=128, dv=128, W=1024, S=4),
        # gradients of the causal layer
        dict(name="bwd_causal_d64", op="bwd", dtype="bf16", B=4, Hq=16, Hk=16, N=2048, M=2048, dk=64, dv=64, W=0, S=0),
        # gradients in single precision at an odd length
        dict(name="bwd_odd_fp32", op="bwd", dtype="fp32", B=2, Hq=6, Hk=3, N=517, M=517, dk=128, dv=64, W=100, S=3),
        # every sequence of a serving batch appends one token: all latency
        dict(name="append_step", op="append", dtype="bf16", B=64, Hq=32, Hk=8, N=1, dk=128, dv=128, rot=128,
             style="half", page=64, L=4000),
        # long prompts go into the cache, half of each head rotated in neighbouring pairs
        dict(name="append_prompt", op="append", dtype="bf16", B=3, Hq=16, Hk=8, N=16001, dk=128, dv=128, rot=64,
             style="pairs", page=32, L=16384),
        # one conversation of a windowed layer, one token: latency
        dict(name="attn_one", op="attn", dtype="bf16", B=1, Hq=16, Hk=4, N=1, dk=128, dv=128, page=16, L=5000,
             W=1024, S=4, causal=True),
        # a serving batch of uneven lengths, the empty and the one-token sequence among them
        dict(name="attn_batch", op="attn", dtype="bf16", B=48, Hq=32, Hk=8, N=1, dk=128, dv=128, page=64, L=16384,
             W=0, S=0, causal=True),
        # a chunk of a prompt against what is cached before it
        dict(name="attn_chunk", op="attn", dtype="bf16", B=1, Hq=32, Hk=8, N=2048, dk=128, dv=128, page=64, L=16384,
             W=0, S=0, causal=True),
        # a few draft tokens verified in single precision, odd page size, narrow values, a window
        dict(name="attn_draft_fp32", op="attn", dtype="fp32", B=5, Hq=12, Hk=4, N=5, dk=128, dv=64, page=48, L=3001,
             W=1000, S=4, causal=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["fwd", "bwd", "append", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    dk, dv = rng.choice([(64, 64), (128, 128), (128, 128), (128, 64), (64, 128)])
    Hk = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 3, 4, 5, 8])
    if op in ("fwd", "bwd"):
        top = 16384 if op == "fwd" and dtype == "bf16" else 8192 if dtype == "bf16" else 2048
        N = _log(rng, 1, top)
        M = N + (_log(rng, 1, 2000) if rng.random() < 0.3 else 0)
        B = _log(rng, 1, max(1, min(8, (1 << (32 if dtype == "bf16" else 28)) // (Hk * G * N * M))))
        W = 0 if rng.random() < 0.3 else _log(rng, 1, 4096)
        return dict(op=op, dtype=dtype, B=B, Hq=Hk * G, Hk=Hk, N=N, M=M, dk=dk, dv=dv, W=W,
                    S=rng.choice([0, 1, 4, 4, 130]) if W else 0)
    page = rng.choice([16, 32, 48, 64, 128, 256])
    if op == "append":
        N = _log(rng, 1, 16000)
        B = _log(rng, 1, max(1, min(64, 32000 // N)))
        return dict(op=op, dtype=dtype, B=B, Hq=Hk * min(G, 4), Hk=Hk, N=N, dk=dk, dv=dv, rot=rng.choice([dk, dk, 32]),
                    style=rng.choice(["half", "pairs"]), page=page, L=N + rng.randrange(1, 2000))
    W = 0 if rng.random() < 0.5 else _log(rng, 1, 8192)
    S = rng.choice([0, 1, 4, 4, 130]) if W else 0
    if rng.random() < 0.7:                               # decoding: few queries, any context
        N = rng.choice([1, 1, 1, 2, 4])
        L = _log(rng, 100, 65536)
        B = _log(rng, 1, max(1, min(64, 131072 // L)))
    else:                                                # a chunk of a prompt
        dtype = "bf16"
        N = _log(rng, 16, 2048)
        L = N + _log(rng, 100, 14000)
        B = _log(rng, 1, max(1, min(8, (1 << 25) // (N * L))))
    return dict(op=op, dtype=dtype, B=B, Hq=Hk * G, Hk=Hk, N=N, dk=dk, dv=dv, page=page, L=L, W=W, S=S,
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
    dt, B, N, Hk, dk, dv = TYPES[case["dtype"]], case["B"], case["N"], case["Hk"], case["dk"], case["dv"]
    s = {"op": case["op"], "case": dict(case), "dtype": dt}
    channel = torch.exp(0.3 * _rand(gen, Hk, 1, dk))     # some key channels are larger
    if case["op"] in ("fwd", "bwd"):
        s["q"] = _rand(gen, B, case["Hq"], N, dk, dtype=dt, scale=1.5)
        s["k"] = (_rand(gen, B, Hk, case["M"], dk) * channel).to(dt)
        s["v"] = _rand(gen, B, Hk, case["M"], dv, dtype=dt)
        if case["op"] == "bwd":
            s["do"] = _rand(gen, B, case["Hq"], N, dv, dtype=dt, scale=0.01)
            # what the forward pass left behind
            s["o"] = torch.empty(B, case["Hq"], N, dv, dtype=dt, device=DEV)
            s["lse"] = torch.empty(B, case["Hq"], N, dtype=torch.float32, device=DEV)
            for b in range(B):
                o, s["lse"][b] = _plain_rows(s["q"][b].float(), s["k"][b].float(), s["v"][b].float(), case, case["M"])
                s["o"][b] = o.to(dt)
        return s
    page, L = case["page"], case["L"]
    if case["op"] == "append":
        s["table"], n = _pages(gen, [L] * B, page, L)
        s["pool"] = torch.zeros(n, Hk, page, dk + dv, dtype=dt, device=DEV)
        start = torch.randint(0, L - N + 1, (B, 1), generator=gen, device=DEV)
        s["pos"] = (start + torch.arange(N, device=DEV)).to(torch.int32)
        s["cos"], s["sin"] = _angles(L, case["rot"])
        s["q"] = _rand(gen, B, case["Hq"], N, dk, dtype=dt, scale=1.5)
        s["k"] = (_rand(gen, B, Hk, N, dk) * channel).to(dt)
        s["v"] = _rand(gen, B, Hk, N, dv, dtype=dt)
        return s
    lens = _lens(case)
    order = torch.randperm(B, generator=gen, device=DEV).tolist()
    lens = [lens[i] for i in order]
    s["table"], n = _pages(gen, lens, page, L)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["pool"] = torch.cat([_rand(gen, n, Hk, page, dk) * channel, _rand(gen, n, Hk, page, dv)], -1).to(dt)
    # what lies past a sequence's end is whatever the page held before: here, not numbers at all
    end = (torch.tensor([n_ - 1 for n_ in lens], device=DEV).clamp(min=0) // page)[:, None]
    last = s["table"].long().gather(1, end)[:, 0]
    for b, length in enumerate(lens):
        if length % page:
            s["pool"][last[b], :, length % page:] = float("nan")
    if case["W"]:
        # pages between the first tokens and the first query's window have been given back
        at = torch.arange(s["table"].shape[1], device=DEV)[None]
        first = (s["lens"].long() - N - case["W"] + 1)[:, None]       # the first token that a window reaches
        gone = (at * page >= case["S"]) & ((at + 1) * page <= first)
        s["table"] = torch.where(gone, torch.full_like(s["table"], -1), s["table"])
    s["q"] = _rand(gen, B, case["Hq"], N, dk, dtype=dt, scale=1.5)
    return s


# ---------------------------------------------------------------------------------------------
# The operators in plain form
# ---------------------------------------------------------------------------------------------
def _seen(N, T, length, W, S, causal):
    """[N, T]: which of T places each of the last N of `length` tokens sees."""
    p = length - N + torch.arange(N, device=DEV)[:, None]
    j = torch.arange(T, device=DEV)[None]
    seen = (j <= p) if causal else (j < length)
    if W:
        seen = seen & ((j > p - W) | (j < S))
    return seen


def _plain_weights(q, k, case, length):
    """(weights, log of the sums) of one sequence: q [Hq, N, dk], k [Hk, T, dk] in 32 bits; a row that
    sees nothing has no weights."""
    Hq, N, dk = q.shape
    Hk, T = k.shape[:2]
    seen = _seen(N, T, length, case["W"], case["S"], case.get("causal", True))
    p = torch.matmul(q.view(Hk, Hq // Hk * N, dk), k.transpose(-2, -1)).view(Hq, N, T)
    p = torch.where(seen, p.mul_(dk ** -0.5), torch.full((), -math.inf, device=DEV))
    m = p.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = p.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total == 0, torch.ones_like(total), total))
    return p, (torch.log(total) + m)[..., 0]


def _plain_rows(q, k, v, case, length):
    Hq, N, _ = q.shape
    Hk, T, dv = v.shape
    p, lse = _plain_weights(q, k, case, length)
    return torch.matmul(p.view(Hk, Hq // Hk * N, T), v).view(Hq, N, dv), lse


def _plain_fwd(s):
    o = torch.empty(*s["q"].shape[:3], s["v"].shape[3], dtype=s["dtype"], device=DEV)
    step = 8 if s["q"].shape[2] > 16384 else s["q"].shape[1]      # heads of a long sequence at a time
    G = s["case"]["Hq"] // s["case"]["Hk"]
    step = max(G, step // G * G)
    for b in range(o.shape[0]):
        for h in range(0, o.shape[1], step):
            kv = slice(h // G, (h + step) // G)
            o[b, h:h + step] = _plain_rows(s["q"][b, h:h + step].float(), s["k"][b, kv].float(), s["v"][b, kv].float(),
                                           s["case"], s["case"]["M"])[0].to(s["dtype"])
    return o


def _plain_bwd(s):
    case = s["case"]
    dq, dk, dv = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
    Hk, T = case["Hk"], case["M"]
    rows = case["Hq"] // Hk * case["N"]
    scale = case["dk"] ** -0.5
    for b in range(case["B"]):
        q, k, v, o, do = (s[n][b].float() for n in ("q", "k", "v", "o", "do"))
        seen = _seen(case["N"], T, T, case["W"], case["S"], True)
        p = torch.matmul(q.view(Hk, rows, -1), k.transpose(-2, -1)).view(case["Hq"], case["N"], T)
        p = torch.where(seen, p.mul_(scale).sub_(s["lse"][b][..., None]).exp_(), torch.zeros((), device=DEV))
        g = do.view(Hk, rows, -1)
        dv[b] = torch.matmul(p.view(Hk, rows, T).transpose(-2, -1), g).to(s["dtype"])
        d = torch.matmul(g, v.transpose(-2, -1)).view_as(p).sub_((o * do).sum(-1, keepdim=True)).mul_(p)
        d = d.view(Hk, rows, T)
        dq[b] = (torch.matmul(d, k) * scale).view_as(q).to(s["dtype"])
        dk[b] = (torch.matmul(d.transpose(-2, -1), q.view(Hk, rows, -1)) * scale).to(s["dtype"])
    return [dq, dk, dv]


def _turn(x, c, n, rot, style):
    """x with its first rot features rotated, rounded to its type."""
    y = x.float()
    a, b = (y[..., :rot // 2], y[..., rot // 2:rot]) if style == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
    a, b = a * c - b * n, b * c + a * n
    front = torch.cat([a, b], -1) if style == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([front, y[..., rot:]], -1).to(x.dtype)


def _plain_append(s):
    case, pos = s["case"], s["pos"].long()
    c, n = s["cos"][pos][:, None], s["sin"][pos][:, None]
    where = s["table"].long().gather(1, pos // case["page"])
    row = torch.cat([_turn(s["k"], c, n, case["rot"], case["style"]), s["v"]], -1)
    s["pool"][where, :, pos % case["page"]] = row.transpose(1, 2)
    return [_turn(s["q"], c, n, case["rot"], case["style"]), s["pool"]]


def _plain_attn(s):
    case = s["case"]
    B, N, Hq, Hk, dk, dv = case["B"], case["N"], case["Hq"], case["Hk"], case["dk"], case["dv"]
    kv = s["pool"][s["table"].long().clamp(min=0)].transpose(1, 2).flatten(2, 3).float()     # B, Hk, places, dk + dv
    k, v = kv[..., :dk], kv[..., dk:]
    T = kv.shape[2]
    p = s["lens"][:, None] - N + torch.arange(N, device=DEV)
    j = torch.arange(T, device=DEV)
    seen = j <= (p if case["causal"] else s["lens"][:, None] - 1 + 0 * p)[..., None]
    if case["W"]:
        seen = seen & ((j > p[..., None] - case["W"]) | (j < case["S"]))
    v = torch.where(seen.any(1)[:, None, :, None], v, torch.zeros((), device=DEV))
    seen = seen[:, None]
    w = torch.matmul(s["q"].float().view(B, Hk, Hq // Hk * N, dk), k.transpose(-2, -1)) * dk ** -0.5
    w = torch.where(seen, w.view(B, Hq, N, T), torch.full((), -math.inf, device=DEV))
    m = w.amax(-1, keepdim=True)
    w = torch.where(seen, torch.exp(w - torch.where(m == -math.inf, torch.zeros_like(m), m)), torch.zeros((), device=DEV))
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(B, Hk, Hq // Hk * N, T), v).view(B, Hq, N, dv)
    return (o / torch.where(total == 0, torch.ones_like(total), total)).to(s["dtype"])


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------
def run(state):
    s = state
    if not own:
        return {"fwd": _plain_fwd, "bwd": _plain_bwd, "append": _plain_append, "attn": _plain_attn}[s["op"]](s)
    import paper_2606_07713_gb300 as moa
    c = s["case"]
    if s["op"] == "append":
        q = moa.kv_append(s["k"], s["v"], s["pool"], s["table"], s["pos"], s["cos"], s["sin"], q=s["q"],
                          interleaved=c["style"] == "pairs")
        return [q, s["pool"]]
    window = c["W"] or None
    if s["op"] == "fwd":
        return moa.window_attn(s["q"], s["k"], s["v"], window=window, sinks=c["S"])
    if s["op"] == "bwd":
        return list(moa.window_attn_bwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], window=window, sinks=c["S"]))
    return moa.kv_attn(s["q"], s["pool"], s["table"], s["lens"], max_len=c["L"], window=window, sinks=c["S"],
                       causal=c["causal"])


# ---------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------
def _counts(N, length, W, S, causal):
    """(pairs of a query and a token that it sees, tokens that any query sees)."""
    p = length - N + np.arange(N, dtype=np.int64)
    end = np.maximum(p + 1, 0) if causal else np.full(N, length, dtype=np.int64)
    first = np.clip(p - W + 1, 0, end) if W else np.zeros(N, dtype=np.int64)
    held = np.minimum(first, S)
    live = end > 0
    if not live.any():
        return 0, 0
    low = int(first[live].min())
    return int((end - first + held)[live].sum()), int(end.max()) - low + min(low, S)


def work(case):
    B, N, Hq, Hk, dk, dv = case["B"], case["N"], case["Hq"], case["Hk"], case["dk"], case["dv"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "append":
        rows = Hq * dk + Hk * (dk + dv)
        return {"bytes": 2 * B * N * rows * size + B * N * (4 * case["rot"] + 4), "flops": 3 * B * N * (Hq + Hk) * case["rot"]}
    if case["op"] == "attn":
        pairs = seen = 0
        for n in _lens(case):
            a, b = _counts(N, n, case["W"], case["S"], case["causal"])
            pairs, seen = pairs + a, seen + b
        return {"bytes": seen * Hk * (dk + dv) * size + B * N * Hq * (dk + dv) * size + seen // case["page"] * 4 + 4 * B,
                "flops": 2 * Hq * pairs * (dk + dv)}
    pairs, seen = _counts(N, case["M"], case["W"], case["S"], True)
    query, key = B * Hq * N * size, B * Hk * seen * (dk + dv) * size
    if case["op"] == "fwd":
        return {"bytes": query * (dk + dv) + key, "flops": 2 * B * Hq * pairs * (dk + dv)}
    # scores, weights times dO, dO V^T, dS K, dS^T Q
    return {"bytes": query * (2 * dk + 2 * dv) + 4 * B * Hq * N + 2 * key, "flops": 2 * B * Hq * pairs * (3 * dk + 2 * dv)}


# ---------------------------------------------------------------------------------------------
# The same outputs from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------
_BLOCK = 1024      # queries at a time


def _exact_blocks(N, length, W, S, causal):
    """For blocks of queries: (first, last, the tokens that they may see, what is hidden of those)."""
    for a in range(0, N, _BLOCK):
        z = min(N, a + _BLOCK)
        stop = max(0, length - N + z) if causal else length
        start = max(0, length - N + a - W + 1) if W else 0
        start = min(start, stop)
        tokens = torch.cat([torch.arange(min(S, start), device=DEV), torch.arange(start, stop, device=DEV)])
        gap = torch.arange(length - N + a, length - N + z, device=DEV)[:, None] - tokens[None]     # how far back
        hidden = (gap < 0) if causal else torch.zeros_like(gap, dtype=torch.bool)
        if W:
            hidden = hidden | ((gap >= W) & (tokens[None] >= S))
        yield a, z, tokens, hidden


def _exact_softmax(q, k, hidden, scale):
    x = (q @ k.T) * scale
    x = x.masked_fill(hidden, -math.inf)
    return torch.nan_to_num(torch.softmax(x, -1), nan=0.0) if x.shape[1] else x


def _exact_dense(case, s):
    N, M, G, scale = case["N"], case["M"], case["Hq"] // case["Hk"], 1.0 / math.sqrt(case["dk"])
    zeros = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=DEV)
    o = torch.zeros(case["B"], case["Hq"], N, case["dv"], dtype=torch.float64, device=DEV)
    grads = [zeros(s["q"]), zeros(s["k"]), zeros(s["v"])] if case["op"] == "bwd" else None
    for b in range(case["B"]):
        for h in range(case["Hq"]):
            k, v = s["k"][b, h // G].double(), s["v"][b, h // G].double()
            q = s["q"][b, h].double()
            for a, z, tokens, hidden in _exact_blocks(N, M, case["W"], case["S"], True):
                p = _exact_softmax(q[a:z], k[tokens], hidden, scale)
                o[b, h, a:z] = p @ v[tokens]
                if grads is None:
                    continue
                g = s["do"][b, h, a:z].double()
                e = g @ v[tokens].T
                e = p * (e - (p * e).sum(-1, keepdim=True)) * scale
                grads[0][b, h, a:z] = e @ k[tokens]
                grads[1][b, h // G].index_add_(0, tokens, e.T @ q[a:z])
                grads[2][b, h // G].index_add_(0, tokens, p.T @ g)
    return o if grads is None else grads


def _exact_append(case, s):
    half = case["rot"] // 2
    i = torch.arange(half, device=DEV)
    first, second = (i, i + half) if case["style"] == "half" else (2 * i, 2 * i + 1)
    angle = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].long()][:, None]

    def turn(x):
        x = x.double()
        z = torch.complex(x[..., first], x[..., second]) * angle
        x[..., first], x[..., second] = z.real, z.imag
        return x

    pool = s["pool"].double()
    rows = torch.cat([turn(s["k"]), s["v"].double()], -1)
    for b in range(case["B"]):
        at = s["pos"][b].long()
        pool[s["table"][b].long()[at // case["page"]], :, at % case["page"]] = rows[b].transpose(0, 1)
    return [turn(s["q"]), pool]


def _exact_attn(case, s):
    N, G, page, scale = case["N"], case["Hq"] // case["Hk"], case["page"], 1.0 / math.sqrt(case["dk"])
    o = torch.zeros(case["B"], case["Hq"], N, case["dv"], dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        pages = s["table"][b].long()
        for a, z, tokens, hidden in _exact_blocks(N, n, case["W"], case["S"], case["causal"]):
            if not len(tokens):
                continue
            for h in range(case["Hk"]):
                rows = s["pool"][pages[tokens // page], h, tokens % page].double()
                k, v = rows[:, :case["dk"]], rows[:, case["dk"]:]
                for j in range(h * G, h * G + G):
                    o[b, j, a:z] = _exact_softmax(s["q"][b, j, a:z].double(), k, hidden, scale) @ v
    return o


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("fwd", "bwd"):
        return _exact_dense(case, s)
    return _exact_append(case, s) if case["op"] == "append" else _exact_attn(case, s)
