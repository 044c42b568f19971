"""Writes and reads of the 4-bit cache so long that a CTA takes several heads, and whole blocks cross at
once: exact, as in test_kv4.py, codes, scales and the bytes that are not named.
"""
import numpy as np
import pytest

import ops_reference as R
import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib
from test_kv4 import cast, dev, host, table_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def heads_of_a_cta(B, H, N, dk, dv):
    """The kernels' rule: all heads, halved until there are eight CTAs an SM."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    units = B * ((N + 30) // 16)
    ctas = -(-units // (2 if dk <= 64 and dv <= 64 else 1))
    hp = H
    while hp > 1 and ctas * -(-H // hp) < 8 * sms:
        hp = (hp + 1) // 2
    return hp


# B, H, N, d_k, d_v, page, heads a CTA takes
CASES = [
    (1, 3, 9800, 128, 128, 64, 2),
    (1, 5, 9801, 128, 64, 48, 3),
    (2, 8, 9999, 64, 128, 32, 8),
    (1, 8, 19700, 64, 64, 256, 4),
    (3, 7, 13000, 64, 64, 16, 7),
]


def problem(case, dtype, start, seed):
    B, H, N, dk, dv, page, _ = case
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    size = torch.exp(2 * torch.randn(B, 1, N, 1, generator=g, device="cuda:0"))
    k = (torch.randn(B, H, N, dk, generator=g, device="cuda:0") * size).to(kind)
    v = torch.randn(B, H, N, dv, generator=g, device="cuda:0").to(kind)
    table, n_pages = table_of(np.random.default_rng(seed), [start + N + 40] * B, page)
    pos = np.tile(np.arange(start, start + N, dtype=np.int32), (B, 1))
    pool = torch.randint(0, 256, (n_pages, H, page // 16, 9 * (dk + dv)), generator=g, device="cuda:0", dtype=torch.uint8)
    return k, v, table, pos, pool


def check_blocks(pool, before, k, v, table, pos, dk, dv, seed):
    """Bytes of seeded blocks, the first and the last of every sequence among them, and of all pages that
    belong to nobody."""
    page = 16 * before.shape[2]
    r = np.random.default_rng(seed)
    for b in range(len(pos)):
        live = np.flatnonzero(pos[b] >= 0)
        first, last = pos[b, live[0]] // 16, pos[b, live[-1]] // 16
        blocks = np.unique(np.r_[first, last, first + 1, last - 1, r.integers(first, last + 1, size=12)])
        at = (torch.from_numpy(table[b, blocks * 16 // page].astype(np.int64)), slice(None),
              torch.from_numpy(blocks * 16 % page // 16))
        # advanced indices apart put the blocks first: [blocks, heads, bytes]
        got = R.unpack(pool[at].cpu().numpy(), dk, dv)
        want = R.unpack(before[at].cpu().numpy(), dk, dv)
        where = {p: n for n, p in enumerate(pos[b]) if p >= 0}
        for i, block in enumerate(blocks):
            for token in range(16):
                n = where.get(block * 16 + token)
                if n is None:
                    continue
                (kc, ks), (vc, vs) = R.quantise(host(k[b, :, n])), R.quantise(host(v[b, :, n]))
                for w, x in zip(want, (kc, ks, vc, vs)):
                    w[i, :, token] = x
        for x, y in zip(got, want):
            assert np.array_equal(x, y, equal_nan=True)
    nobody = np.setdiff1d(np.arange(len(before)), table[table >= 0])
    assert len(nobody) and torch.equal(pool[torch.from_numpy(nobody)], before[torch.from_numpy(nobody)])


def widened(x, dtype):
    """What the cache gives back for rows x, computed by the definition in the float32 operations that it
    rounds by, on the device."""
    y = x.float().unflatten(-1, (-1, 32))
    m = y.abs().amax(-1, keepdim=True)
    s = (m / torch.full_like(m, 7.0)).bfloat16().float()
    code = torch.round(y / s).clamp(-7, 7)
    return torch.where(s > 0, code * s, torch.zeros_like(y)).flatten(-2).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


@pytest.mark.parametrize("start", [0, 5])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_long_consecutive_positions(case, dtype, start):
    B, H, N, dk, dv, page, hp = case
    assert heads_of_a_cta(B, H, N, dk, dv) == hp > 1
    k, v, table, pos, before = problem(case, dtype, start, seed=N + start)
    pool = before.clone()
    pkg.kv4_write(k, v, pool, dev(table), dev(pos))
    check_blocks(pool, before, k, v, table, pos, dk, dv, seed=N)
    # the same rows in another order, token by token: the same bytes
    order = torch.randperm(N, device="cuda:0")
    other = before.clone()
    pkg.kv4_write(k[:, :, order], v[:, :, order], other, dev(table), dev(pos)[:, order].contiguous())
    assert torch.equal(pool, other)
    # read back whole, from inside a block, and in another order
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    want = widened(k, dtype), widened(v, dtype)
    for rows in (slice(None), slice(7, N - 3), order):
        at = dev(pos)[:, rows].contiguous()
        for x, y in zip(pkg.kv4_read(pool, dev(table), at, dk, dtype=kind), want):
            assert torch.equal(x, y[:, :, rows])
    assert pkg.get_device_status() == _lib.MOA_OK


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("left,right", [(1, 0), (37, 0), (0, 21), (16, 5)])
def test_padded_rows_among_long_ones(left, right, dtype):
    """Sequences of different lengths side by side, padded in front (queries being the last tokens) or
    behind, one of them all padding."""
    case = B, H, N, dk, dv, page, hp = (3, 5, 6600, 128, 128, 64, 5)
    assert heads_of_a_cta(B, H, N, dk, dv) == hp > 1
    k, v, table, pos, before = problem(case, dtype, 3, seed=left + right)
    pos[0, :left] = -1
    pos[0, N - right:] = -1
    pos[1, :2 * left + 3] = -1
    pos[2] = -1
    pool = before.clone()
    pkg.kv4_write(k, v, pool, dev(table), dev(pos))
    check_blocks(pool, before, k[:2], v[:2], table[:2], pos[:2], dk, dv, seed=1)
    mine = torch.from_numpy(table[2].astype(np.int64))
    assert torch.equal(pool[mine], before[mine])
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    live = dev(pos >= 0)[:, None, :, None]
    for x, y in zip(pkg.kv4_read(pool, dev(table), dev(pos), dk, dtype=kind), (widened(k, dtype), widened(v, dtype))):
        assert torch.equal(x, torch.where(live, y, torch.zeros_like(y)))
    assert pkg.get_device_status() == _lib.MOA_OK


def test_padding_in_front_costs_no_time():
    """Rows of a prompt that begin with padding still cross in whole blocks.  The fastest of 30 calls each
    way, in turn: the two take the same 50 us within a few per cent; in pieces of two and four bytes it was
    27 % more."""
    B, H, N, d, page = 3, 8, 16001, 128, 64
    per = N // page + 2
    pool, pages = pkg.kv4_pool(B * per, H, page, d, d), torch.arange(B * per, dtype=torch.int32, device="cuda:0").view(B, per)
    flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda:0")
    plain = torch.arange(N, dtype=torch.int32, device="cuda:0").repeat(B, 1)
    padded = torch.where(plain < 7, -1, plain - 7).int().contiguous()
    out = [torch.empty(B, H, N, d, dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    times = {}
    for _ in range(30):
        for name, pos in (("plain", plain), ("padded", padded)):
            flush.zero_()
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            pkg.kv4_read(pool, pages, pos, d, out=out)
            b.record()
            torch.cuda.synchronize()
            times[name] = min(times.get(name, 1e9), a.elapsed_time(b))
    assert times["padded"] <= 1.15 * times["plain"], times
