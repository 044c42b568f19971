"""Attention over the 4-bit cache where a CTA works long on one item, and where there are more items than
CTAs: rings that turn over many times, several batches of pages, pieces of many CTAs.

The reference is computed in 64 bits on the device from what kv4_read gives back in fp32 (exact, see
test_kv4.py).  Bounds: those of test_kv4.py.  An accumulator's chain is at most 100 products of 16 tokens
in the longest share here, then 4 warps and 80 pieces: 200 * 2^-24 is below the 2^-15 that they allow.
"""
import math

import numpy as np
import pytest

import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib
from test_kv4 import check, table_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def turns(dtype, Hq, Hk, N, dk, dv, lens):
    """(tiles that a warp takes of an item cut by its share, stages of its ring, tiles whose pages it looks
    up at once, whether there are more items than CTAs): kv4_attn.cu's division of the work."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    rows = Hq // Hk * N
    tile = 8 if rows <= 8 else 16 if rows <= 16 else 32
    ctas = sms * (3 if tile == 8 and dtype == "bf16" else 2)
    n_tiles = -(-rows // tile)
    total = sum(max(1, -(-n // 64)) + 6 for n in lens) * n_tiles * Hk
    sub = 1 if tile == 32 else 2
    stages = (13824 if tile == 8 and dtype == "bf16" else 18432) // (sub * 9 * (dk + dv))
    return (total // ctas - 6) // sub, stages, 32 // sub, len(lens) * Hk * n_tiles > ctas


def problem(dtype, Hq, Hk, N, dk, dv, page, lens, seed):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    table, n_pages = table_of(np.random.default_rng(seed), lens, page)
    pool = torch.full((n_pages, Hk, page // 16, 9 * (dk + dv)), 255, dtype=torch.uint8, device="cuda:0")
    pages = torch.from_numpy(table).cuda()
    channel = torch.exp(0.3 * torch.randn(dk, generator=g, device="cuda:0"))
    for b, n in enumerate(lens):
        for at in range(0, n, 16384):
            m = min(16384, n - at)
            k = (torch.randn(1, Hk, m, dk, generator=g, device="cuda:0") * channel).bfloat16()
            v = torch.randn(1, Hk, m, dv, generator=g, device="cuda:0").bfloat16()
            pos = torch.arange(at, at + m, dtype=torch.int32, device="cuda:0")[None]
            pkg.kv4_write(k, v, pool, pages[b:b + 1].contiguous(), pos)
    q = torch.randn(len(lens), Hq, N, dk, generator=g, device="cuda:0").to(DT[dtype])
    return q, pool, pages


def reference(q, pool, pages, lens, b, heads, dk, causal, gone=()):
    """(o, lse, sum p |v|, largest sum |q k|) of sequence b's key heads, [heads * G, N, ...], in 64 bits;
    `gone`: tokens that are not there."""
    n, N = lens[b], q.shape[2]
    G = q.shape[1] // pool.shape[1]
    out = []
    for h in heads:
        if n == 0:
            dv = pool.shape[3] // 9 - dk
            out.append([np.zeros((G, N, dv)), np.full((G, N), -np.inf), np.zeros((G, N, dv)), np.zeros((G, N))])
            continue
        pos = torch.arange(n, dtype=torch.int32, device="cuda:0")[None]
        k, v = (x[0, 0].double() for x in pkg.kv4_read(pool[:, h:h + 1].contiguous(), pages[b:b + 1].contiguous(), pos,
                                                       dk, dtype=torch.float32))
        x = q[b, h * G:(h + 1) * G].double()
        at = torch.arange(n, device="cuda:0")
        seen = at[None] < (n - N + 1 + torch.arange(N, device="cuda:0")[:, None] if causal else n)
        seen = seen.expand(N, n).clone()
        for lo, hi in gone:
            seen[:, lo:hi] = False
        k, v = (torch.where(seen.any(0)[:, None], y, torch.zeros_like(y)) for y in (k, v))
        s = torch.where(seen, x @ k.T * dk ** -0.5, -math.inf)
        m = s.amax(-1, keepdim=True)
        p = torch.where(seen, torch.exp(s - torch.where(torch.isfinite(m), m, 0.0)), 0.0)
        total = p.sum(-1, keepdim=True)
        lse = (m + torch.log(total))[..., 0]
        p = p / torch.where(total == 0, 1.0, total)
        size = torch.where(seen, x.abs() @ k.abs().T * dk ** -0.5, 0.0).amax(-1)
        out.append([y.cpu().numpy() for y in (p @ v, lse, p @ v.abs(), size)])
    return [np.concatenate(y) for y in zip(*out)]


LONG = [  # dtype, Hq, Hk, N, d_k, d_v, page, lens
    ("bf16", 32, 8, 1, 128, 128, 64, [131072, 90001]),      # 8-row tiles
    ("bf16", 8, 8, 3, 64, 64, 48, [150000, 120007]),
    ("bf16", 16, 8, 6, 128, 64, 32, [100000, 70001]),       # 16-row tiles
    ("bf16", 16, 4, 5, 64, 128, 128, [90000, 70000, 60007]),  # 32-row tiles
    ("fp32", 8, 4, 2, 128, 128, 64, [140001, 131072]),
    ("fp32", 4, 2, 7, 128, 64, 16, [230000, 180003]),
    ("fp32", 8, 2, 8, 64, 64, 256, [220000, 180001]),
]


@pytest.mark.parametrize("case", LONG, ids=lambda c: "x".join(map(str, c)).replace(" ", ""))
def test_long_shares(case):
    dtype, Hq, Hk, N, dk, dv, page, lens = case
    tiles, stages, batch, _ = turns(dtype, Hq, Hk, N, dk, dv, lens)
    assert tiles > stages and tiles > batch
    q, pool, pages = problem(dtype, Hq, Hk, N, dk, dv, page, lens, seed=Hq + N)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda:0")
    heads, G = (0, Hk - 1), Hq // Hk
    mine = [h * G + g for h in heads for g in range(G)]
    for causal in (True, False):
        o, lse = pkg.kv4_attn_lse(q, pool, pages, n, max_len=max(lens), causal=causal)
        assert pkg.get_device_status() == _lib.MOA_OK
        for b in range(len(lens)):
            check(o[b, mine], lse[b, mine], reference(q, pool, pages, lens, b, heads, dk, causal), dk, dtype, b)
        assert torch.equal(o, pkg.kv4_attn(q, pool, pages, n, max_len=max(lens), causal=causal))
    # pages that are not there, all along the first sequence: every batch has some
    wrong = pages.clone()
    lost = list(range(5, lens[0] // page, max(1, 3001 // page)))
    for i, slot in enumerate(lost):
        wrong[0, slot] = -1 if i % 2 else len(pool)
    o, lse = pkg.kv4_attn_lse(q, pool, wrong, n, max_len=max(lens))
    assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
    ref = reference(q, pool, pages, lens, 0, heads, dk, True, gone=[(s * page, (s + 1) * page) for s in lost])
    check(o[0, mine], lse[0, mine], ref, dk, dtype, "pages gone")


MANY = [  # dtype, Hq, Hk, N, d_k, d_v, page, sequences
    ("bf16", 32, 8, 1, 128, 128, 16, 64),
    ("bf16", 8, 8, 9, 64, 64, 32, 41),        # 16-row tiles
    ("bf16", 16, 8, 20, 64, 128, 64, 23),     # two 32-row tiles a head
    ("fp32", 8, 8, 2, 128, 64, 48, 40),
    ("fp32", 16, 8, 19, 64, 64, 16, 21),
]


@pytest.mark.parametrize("most", [700, 40])
@pytest.mark.parametrize("case", MANY, ids=lambda c: "x".join(map(str, c)))
def test_more_items_than_ctas(case, most):
    dtype, Hq, Hk, N, dk, dv, page, B = case
    lens = [int(x) for x in np.random.default_rng(B).integers(0, most, size=B)]
    lens[3], lens[4], lens[-1] = 0, 1, most
    assert turns(dtype, Hq, Hk, N, dk, dv, lens)[3]
    q, pool, pages = problem(dtype, Hq, Hk, N, dk, dv, page, lens, seed=B)
    o, lse = pkg.kv4_attn_lse(q, pool, pages, torch.tensor(lens, dtype=torch.int32, device="cuda:0"), max_len=most)
    assert pkg.get_device_status() == _lib.MOA_OK
    ref = [reference(q, pool, pages, lens, b, range(Hk), dk, True) for b in range(B)]
    check(o, lse, [np.stack(x) for x in zip(*ref)], dk, dtype)
