"""moa_kv4_attn with so many query rows that the library widens the cache once and attends on the
tensor cores, against the plain 64-bit implementation: the bounds of test_kv4.py (bf16: weights and
values rounded once each)."""
import math

import numpy as np
import pytest

import ops_reference as R
import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib
from test_kv4 import cast, check, dev, table_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def widened(B, Hq, Hk, N, dk, dv, max_len):
    """Whether the call takes this path: its workspace holds the keys and values in 16 bits."""
    need = pkg.moa_kv4_attn_workspace_bytes(B, Hq, Hk, N, dk, dv, max_len, pkg.MOA_BF16)
    return need >= min(B * Hk * max_len * (dk + dv) * 2, 1 << 30)


def problem(lens, Hq, Hk, N, dk, dv, page, seed, q_scale=1.0, spread=0.3):
    """As in test_kv4.py, with the cache filled by the library's own write (checked there), and bytes
    of 255 (scales that are not numbers) wherever it holds no token."""
    r = np.random.default_rng(seed)
    table, n_pages = table_of(r, lens, page)
    T = max(1, max(lens))
    k = cast(r.normal(size=(len(lens), Hk, T, dk)) * np.exp(spread * r.normal(size=dk)), "bf16")
    v = cast(r.normal(size=(len(lens), Hk, T, dv)), "bf16")
    pos = np.where(np.arange(T)[None] < np.array(lens)[:, None], np.arange(T)[None], -1).astype(np.int32)
    pool = torch.full((n_pages, Hk, page // 16, 9 * (dk + dv)), 255, dtype=torch.uint8, device="cuda:0")
    pkg.kv4_write(dev(k, "bf16"), dev(v, "bf16"), pool, dev(table), dev(pos))
    q = cast(q_scale * r.normal(size=(len(lens), Hq, N, dk)), "bf16")
    return q, pool, table, R.values(*R.quantise(k)), R.values(*R.quantise(v))


def reference(q, k, v, lens, scale, causal):
    return [np.stack(x) for x in zip(*(R.attention_dense(q[b], k[b], v[b], n, scale, causal) for b, n in enumerate(lens)))]


CHUNKS = [  # lens, Hq, Hk, N, d_k, d_v, page, causal
    ([3300], 4, 1, 512, 128, 128, 64, True),
    ([2500, 100, 0, 1], 12, 4, 129, 64, 64, 16, True),          # queries before a sequence's first token
    ([5000, 129], 5, 1, 300, 128, 64, 48, True),
    ([700, 640, 128], 16, 2, 260, 64, 128, 128, False),
    ([2049, 2048], 8, 8, 700, 128, 128, 256, True),
    ([1537], 24, 3, 513, 64, 64, 32, True),
    ([9000, 300], 2, 1, 257, 128, 128, 64, False),
]


@pytest.mark.parametrize("case", CHUNKS, ids=lambda c: "x".join(map(str, c)).replace(" ", ""))
def test_chunk(case):
    lens, Hq, Hk, N, dk, dv, page, causal = case
    assert widened(len(lens), Hq, Hk, N, dk, dv, max(lens))
    q, pool, table, k, v = problem(lens, Hq, Hk, N, dk, dv, page, seed=sum(lens) + N)
    ref = reference(q, k, v, lens, 1 / math.sqrt(dk), causal)
    t = [dev(q, "bf16"), pool, dev(table), dev(np.array(lens, dtype=np.int32))]
    o, lse = pkg.kv4_attn_lse(*t, max_len=max(lens), causal=causal)
    assert pkg.get_device_status() == _lib.MOA_OK
    check(o, lse, ref, dk, "bf16")
    again, lse2 = pkg.kv4_attn_lse(*t, max_len=max(lens), causal=causal)
    assert torch.equal(o, again) and torch.equal(lse, lse2)
    # token-major queries and output, no LSE, a looser bound of the lengths
    out = torch.zeros(len(lens), N, Hq, dv, dtype=torch.bfloat16, device="cuda:0")
    pkg.kv4_attn(t[0].transpose(1, 2).contiguous().transpose(1, 2), *t[1:], causal=causal, out=out.transpose(1, 2))
    check(out.transpose(1, 2), None, ref, dk, "bf16", "token-major")


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_chunk_scales_and_magnitudes(scale):
    """Weights from uniform to one-hot, a negative scale, and rows and keys of very different sizes
    (the powers of two taken out of queries and key tiles)."""
    lens, Hq, Hk, N, dk, dv, page = [4100], 4, 1, 512, 64, 64, 64
    assert widened(1, Hq, Hk, N, dk, dv, max(lens))
    q, pool, table, k, v = problem(lens, Hq, Hk, N, dk, dv, page, seed=5, q_scale=0.5)
    q[:, :, ::7] = cast(q[:, :, ::7] * 2.0 ** -40, "bf16")
    q[:, 1, 3] = 0.0
    ref = reference(q, k, v, lens, scale, True)
    o, lse = pkg.kv4_attn_lse(dev(q, "bf16"), pool, dev(table), dev(np.array(lens, dtype=np.int32)), scale=scale)
    check(o, lse, ref, dk, "bf16", scale)


def test_chunk_of_large_and_small_keys():
    """Keys of 2^60 in some tiles and 2^-60 in others against queries of 2^-59: the small ones weigh
    as zeros, exactly."""
    lens, Hq, Hk, N, dk, dv, page = [4096], 4, 1, 512, 128, 128, 64
    r = np.random.default_rng(9)
    table, n_pages = table_of(r, lens, page)
    size = np.where(np.arange(4096) // 512 % 2 == 0, 2.0 ** 60, 2.0 ** -60)[None, None, :, None]
    k = cast(r.normal(size=(1, Hk, 4096, dk)) * size, "bf16")
    v = cast(r.normal(size=(1, Hk, 4096, dv)), "bf16")
    q = cast(r.normal(size=(1, Hq, N, dk)) * 2.0 ** -59, "bf16")
    pool = pkg.kv4_pool(n_pages, Hk, page, dk, dv)
    pkg.kv4_write(dev(k, "bf16"), dev(v, "bf16"), pool, dev(table), dev(np.arange(4096, dtype=np.int32)[None]))
    ref = reference(q, R.values(*R.quantise(k)), R.values(*R.quantise(v)), lens, dk ** -0.5, True)
    o, lse = pkg.kv4_attn_lse(dev(q, "bf16"), pool, dev(table), dev(np.array(lens, dtype=np.int32)))
    check(o, lse, ref, dk, "bf16")


def test_chunk_lengths_and_pages_outside_their_tables():
    lens, Hq, Hk, N, dk, dv, page = [2000, 1800], 4, 2, 512, 64, 64, 16
    q, pool, table, k, v = problem(lens, Hq, Hk, N, dk, dv, page, seed=6)
    t = [dev(q, "bf16"), pool]
    assert widened(2, Hq, Hk, N, dk, dv, 2000)
    good = pkg.kv4_attn(*t, dev(table), dev(np.array(lens, dtype=np.int32)))
    assert pkg.get_device_status() == _lib.MOA_OK
    o = pkg.kv4_attn(*t, dev(table), dev(np.array([2000, -7], dtype=np.int32)))
    assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
    assert bool((o[1] == 0).all())
    check(o[:1], None, [x[:1] for x in reference(q[:1], k[:1], v[:1], lens[:1], dk ** -0.5, True)], dk, "bf16")
    # tokens of a page that is not there are hidden
    for wrong in (len(pool), -1):
        tb = table.copy()
        tb[0, 20] = wrong
        o = pkg.kv4_attn(*t, dev(tb), dev(np.array(lens, dtype=np.int32)), causal=False)
        assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
        rest = [np.delete(x[:1, :, :2000], np.s_[320:336], axis=2) for x in (k, v)]
        check(o[:1], None, reference(q[:1], *rest, [1984], dk ** -0.5, False), dk, "bf16")
        assert torch.equal(o[1], pkg.kv4_attn(*t, dev(table), dev(np.array(lens, dtype=np.int32)), causal=False)[1])
    assert pkg.get_device_status() == _lib.MOA_OK
    assert bool(torch.isfinite(good).all())


@pytest.mark.parametrize("value", [False, True])
def test_chunk_visible_nan_reaches_its_queries_only(value):
    """A key or value that is not a number: the rows that see it are NaN (all features, or at least the
    value's group), the others as ever."""
    lens, Hq, Hk, N, dk, dv, page = [3000, 2900], 4, 2, 512, 64, 64, 64
    q, pool, table, k, v = problem(lens, Hq, Hk, N, dk, dv, page, seed=13)
    assert widened(2, Hq, Hk, N, dk, dv, 3000)
    t = [dev(q, "bf16"), pool, dev(table), dev(np.array(lens, dtype=np.int32))]
    good = pkg.kv4_attn(*t)
    at, token = R.scale_place(dk, dv, 2900 % 16, 1, value), 2900
    pool[int(table[0, token // page]), 1, token % page // 16, at:at + 2] = 255
    o = pkg.kv4_attn(*t)
    first = token - (3000 - N)            # the first query that sees it
    assert bool(torch.isnan(o[0, 2:, first:, 32:]).all())
    o[0, 2:, first:] = good[0, 2:, first:]
    assert torch.equal(o, good)


def test_chunk_heads_in_several_groups():
    """More widened keys and values than one pass holds (1 GB): the heads are taken in groups."""
    lens, Hq, Hk, N, dk, dv, page = [600, 40, 333], 16, 8, 256, 128, 128, 64
    max_len = 1 << 18
    assert 3 * Hk * max_len * (dk + dv) * 2 > 1 << 30
    q, pool, table, k, v = problem(lens, Hq, Hk, N, dk, dv, page, seed=1)
    wide = np.full((3, max_len // page), -1, dtype=np.int32)
    wide[:, :table.shape[1]] = table
    o, lse = pkg.kv4_attn_lse(dev(q, "bf16"), pool, dev(wide), dev(np.array(lens, dtype=np.int32)), max_len=max_len)
    assert pkg.get_device_status() == _lib.MOA_OK
    check(o, lse, reference(q, k, v, lens, dk ** -0.5, True), dk, "bf16")
