"""Attention with a window, its gradients and the 16- and 32-bit cache at sizes where work is divided: many
work items, items cut between CTAs, clusters, long contexts, places past 32 bits.  The references are 64-bit
sums in torch operations on the GPU; the bounds are those of window_reference.py, with the magnitudes that
they are made of computed beside the outputs."""
import math

import pytest

import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib
from window_reference import HALF, SUMS, WEIGHT

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}


def rand(g, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(TORCH[dtype])


def seen(N, T, length, window, sinks, causal=True):
    p = length - N + torch.arange(N, device="cuda")[:, None]
    j = torch.arange(T, device="cuda")[None]
    see = (j <= p) if causal else (j < length) & (p == p)
    return see & ((j > p - window) | (j < sinks)) if window else see


def reference(q, k, v, see, dtype):
    """(o, its bound, lse and its bound) of one head in 64 bits: q [N, d], k [T, d], v [T, dv]."""
    q, k, v = q.double(), k.double(), v.double()
    scale, u = q.shape[1] ** -0.5, HALF[dtype]
    s = (q @ k.T * scale).masked_fill(~see, -math.inf)
    size = (q.abs() @ k.abs().T * scale).masked_fill(~see, 0).amax(1)
    lse = torch.logsumexp(s, 1)
    p = torch.nan_to_num(torch.softmax(s, 1), nan=0.0)
    o, av = p @ v, p @ v.abs()
    e = (q.shape[1] + 8) * 2.0 ** -24 * size[:, None]
    bound = (2 * e + WEIGHT + SUMS + (u if dtype == "bf16" else 0.0)) * av * 1.02 + u * o.abs() * 1.02 + 1e-30
    return o, bound, lse, e[:, 0] + 2.0 ** -17 + 2.0 ** -20 * lse.abs()


def check(o, lse, q, k, v, see, dtype):
    ro, bound, rl, slack = reference(q, k, v, see, dtype)
    assert bool(((o.double() - ro).abs() <= bound).all())
    if lse is not None:
        live = see.any(1)
        assert bool((torch.isfinite(lse) == live).all())
        assert bool(((lse.double() - rl).abs() <= slack)[live].all())


@pytest.mark.parametrize("dtype,B,Hq,Hk,N,M,dk,dv,window,sinks", [
    ("bf16", 1, 8, 2, 4000, 4000, 128, 128, 700, 4),        # more items than CTAs, cut between them
    ("bf16", 3, 16, 16, 1025, 1025, 64, 64, 0, 0),
    ("bf16", 1, 3, 1, 6000, 6100, 64, 128, 0, 0),
    ("bf16", 2, 4, 4, 3001, 3001, 128, 64, 50, 200),
    ("bf16", 1, 2, 2, 40, 9000, 128, 128, 0, 0),            # few rows, many pieces
    ("fp32", 2, 4, 2, 1500, 1500, 64, 64, 300, 3),
    ("fp32", 1, 2, 1, 3, 5000, 128, 128, 0, 0),
])
def test_window(dtype, B, Hq, Hk, N, M, dk, dv, window, sinks):
    g = torch.Generator(device="cuda").manual_seed(N + M)
    q, k, v = (rand(g, B, Hq, N, dk, dtype=dtype, scale=1.5), rand(g, B, Hk, M, dk, dtype=dtype), rand(g, B, Hk, M, dv, dtype=dtype))
    o, lse = pkg.window_attn_lse(q, k, v, window=window or None, sinks=sinks)
    assert pkg.get_device_status() == _lib.MOA_OK
    see = seen(N, M, M, window, sinks)
    for b in range(B):
        for h in (0, Hq // 2, Hq - 1):
            check(o[b, h], lse[b, h], q[b, h], k[b, h // (Hq // Hk)], v[b, h // (Hq // Hk)], see, dtype)


@pytest.mark.parametrize("dtype,B,Hq,Hk,N,M,dk,dv,window,sinks", [
    ("bf16", 1, 8, 2, 3000, 3000, 128, 128, 400, 4),        # sinks in pieces
    ("bf16", 1, 2, 1, 2500, 2500, 64, 64, 0, 0),            # every token tile in pieces
    ("bf16", 4, 12, 12, 1100, 1100, 64, 64, 0, 0),          # more items than CTAs
    ("bf16", 1, 6, 2, 1500, 2000, 128, 64, 100, 300),       # sinks over several tiles
    ("bf16", 1, 4, 4, 700, 700, 64, 128, 9, 700),           # every token a sink
    ("bf16", 1, 4, 2, 30, 3000, 128, 128, 0, 0),            # few rows: their tokens in pieces
    ("bf16", 2, 2, 2, 5, 2500, 64, 64, 2000, 100),
    ("fp32", 1, 2, 1, 30, 1900, 128, 64, 0, 0),
    ("fp32", 2, 6, 2, 3, 1000, 64, 128, 700, 5),
    ("fp32", 1, 4, 2, 1400, 1400, 64, 64, 200, 3),
    ("fp32", 1, 1, 1, 1200, 1200, 128, 128, 0, 0),
])
def test_gradients(dtype, B, Hq, Hk, N, M, dk, dv, window, sinks):
    g = torch.Generator(device="cuda").manual_seed(N + M + 1)
    q, k, v = (rand(g, B, Hq, N, dk, dtype=dtype, scale=1.5), rand(g, B, Hk, M, dk, dtype=dtype), rand(g, B, Hk, M, dv, dtype=dtype))
    do = rand(g, B, Hq, N, dv, dtype=dtype, scale=0.1)
    o, lse = pkg.window_attn_lse(q, k, v, window=window or None, sinks=sinks)
    got = pkg.window_attn_bwd(q, k, v, o, lse, do, window=window or None, sinks=sinks)
    assert pkg.get_device_status() == _lib.MOA_OK
    see, scale, G = seen(N, M, M, window, sinks), dk ** -0.5, Hq // Hk
    u = HALF[dtype]
    ub = u if dtype == "bf16" else 0.0
    for b in range(B):
        for hk in {0, Hk - 1}:
            dk_, dv_ = torch.zeros(M, dk, dtype=torch.float64, device="cuda"), torch.zeros(M, dv, dtype=torch.float64, device="cuda")
            ek, ev = torch.zeros_like(dk_), torch.zeros_like(dv_)
            kk, vv = k[b, hk].double(), v[b, hk].double()
            for h in range(hk * G, hk * G + G):
                qq, gg, oo, ll = q[b, h].double(), do[b, h].double(), o[b, h].double(), lse[b, h].double()
                base = torch.where(torch.isfinite(ll), ll, 0.0)[:, None]
                p = torch.exp((qq @ kk.T * scale - base).masked_fill(~see, -math.inf))
                size = (qq.abs() @ kk.abs().T * scale).masked_fill(~see, 0).amax(1, keepdim=True)
                w = 2 * (dk + 8) * 2.0 ** -24 * size + WEIGHT + 2.0 ** -22 * base.abs()
                ds = p * (gg @ vv.T - (gg * oo).sum(1, keepdim=True))
                dot = (dv + 8) * 2.0 ** -24 * (gg.abs() @ vv.abs().T + (gg * oo).abs().sum(1, keepdim=True))
                eds = (w + ub + SUMS) * ds.abs() + p * dot * 1.02
                want = scale * ds @ kk
                bound = scale * (eds @ kk.abs()) * 1.02 + u * want.abs() * 1.02 + 1e-30
                assert bool(((got[0][b, h].double() - want).abs() <= bound).all()), "dq"
                dk_ += scale * ds.T @ qq
                ek += scale * eds.T @ qq.abs()
                dv_ += p.T @ gg
                ev += ((w + ub + SUMS) * p).T @ gg.abs()
            assert bool(((got[1][b, hk].double() - dk_).abs() <= 1.02 * (ek + u * dk_.abs()) + 1e-30).all()), "dk"
            assert bool(((got[2][b, hk].double() - dv_).abs() <= 1.02 * (ev + u * dv_.abs()) + 1e-30).all()), "dv"


def cache(g, lens, Hk, page, dk, dv, dtype, n_pages=None, first=0):
    """(pool, table, rows by sequence [Hk, n, dk + dv]); pages from `first` on, in any order; junk past the ends."""
    per = [-(-n // page) for n in lens]
    order = (torch.randperm(sum(per), generator=g, device="cuda") + first).to(torch.int32)
    pool = torch.empty(n_pages or sum(per), Hk, page, dk + dv, dtype=TORCH[dtype], device="cuda")
    table = torch.full((len(lens), max(per) or 1), -1, dtype=torch.int32, device="cuda")
    rows, at = [], 0
    for b, n in enumerate(lens):
        mine = order[at:at + per[b]].long()
        at += per[b]
        x = rand(g, Hk, per[b] * page, dk + dv, dtype=dtype)
        x[:, n:] = float("nan")
        pool[mine] = x.view(Hk, per[b], page, dk + dv).transpose(0, 1)
        table[b, :per[b]] = mine.to(torch.int32)
        rows.append(x[:, :n])
    return pool, table, rows


def check_cache(o, lse, q, rows, lens, dk, window, sinks, causal, dtype):
    Hq, N = q.shape[1:3]
    for b, n in enumerate(lens):
        if n == 0:
            assert bool((o[b] == 0).all())
            continue
        see = seen(N, n, n, window, sinks, causal)
        for h in {0, Hq - 1}:
            x = rows[b][h // (Hq // rows[b].shape[0])]
            check(o[b, h], lse[b, h], q[b, h], x[:, :dk], x[:, dk:], see, dtype)


@pytest.mark.parametrize("lens,Hq,Hk,N,dk,dv,page,window,sinks,causal,dtype", [
    ([20000], 8, 1, 1, 128, 128, 64, 0, 0, True, "bf16"),                    # one sequence on all SMs
    ([30000, 7, 12345], 4, 2, 3, 64, 64, 16, 0, 0, False, "bf16"),
    ([900 + 37 * i for i in range(40)] + [0, 1], 16, 8, 1, 128, 64, 32, 0, 0, True, "bf16"),   # more items than CTAs
    ([5000, 4000], 8, 2, 1, 128, 128, 16, 1024, 4, True, "bf16"),             # clusters
    ([300, 250, 1], 4, 2, 60, 64, 128, 48, 0, 0, True, "bf16"),               # clusters, many rows
    ([130], 2, 1, 1, 64, 64, 64, 0, 0, True, "bf16"),
    ([3000, 2000, 100], 32, 8, 700, 128, 128, 64, 0, 0, True, "bf16"),         # chunks
    ([9000, 500], 8, 2, 333, 64, 64, 32, 2000, 130, True, "bf16"),
    ([20000, 3], 4, 1, 1, 128, 128, 64, 0, 0, True, "fp32"),
    ([3000, 2500], 6, 2, 5, 128, 64, 48, 1000, 4, True, "fp32"),              # clusters of 16
    ([1200], 4, 2, 300, 64, 64, 16, 0, 0, True, "fp32"),
])
def test_cache(lens, Hq, Hk, N, dk, dv, page, window, sinks, causal, dtype):
    g = torch.Generator(device="cuda").manual_seed(sum(lens))
    pool, table, rows = cache(g, lens, Hk, page, dk, dv, dtype)
    q = rand(g, len(lens), Hq, N, dk, dtype=dtype, scale=1.5)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = pkg.kv_attn_lse(q, pool, table, ln, max_len=max(lens), window=window or None, sinks=sinks, causal=causal)
    assert pkg.get_device_status() == _lib.MOA_OK
    check_cache(o, lse, q, rows, lens, dk, window, sinks, causal, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_pool_of_more_than_2_31_elements(dtype):
    """Rows appended to, and read from, the last pages of a pool of 2.4 * 10^9 elements."""
    Hk, page, d, n_pages = 8, 128, 128, 9200
    g = torch.Generator(device="cuda").manual_seed(1)
    pool = torch.empty(n_pages, Hk, page, 2 * d, dtype=TORCH[dtype], device="cuda")
    assert pool.numel() > 2 ** 31
    lens, N = [300, 140], 300
    table = torch.tensor([[n_pages - 1, n_pages - 3, 8300], [n_pages - 2, 8301, 0]], dtype=torch.int32, device="cuda")
    k, v = rand(g, 2, Hk, N, d, dtype=dtype), rand(g, 2, Hk, N, d, dtype=dtype)
    pos = torch.arange(N, dtype=torch.int32, device="cuda").repeat(2, 1)
    pos[1, 140:] = -1
    pkg.kv_append(k, v, pool, table, pos)
    q = rand(g, 2, 16, 2, d, dtype=dtype, scale=1.5)
    o, lse = pkg.kv_attn_lse(q, pool, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    assert pkg.get_device_status() == _lib.MOA_OK
    rows = [torch.cat([k[b, :, :n], v[b, :, :n]], -1) for b, n in enumerate(lens)]
    check_cache(o, lse, q, rows, lens, d, 0, 0, True, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_dense_strides_past_32_bits(dtype):
    """A sequence's keys and values 2^31 elements apart from the next one's."""
    N, d, B = 70, 64, 2
    g = torch.Generator(device="cuda").manual_seed(4)
    step = 2 ** 31 + 4096
    big = torch.empty(step + 4 * N * d, dtype=TORCH[dtype], device="cuda")
    q = rand(g, B, 2, N, d, dtype=dtype)
    k, v = (big.as_strided((B, 1, N, d), (step, N * d, d, 1), at) for at in (0, 2 * N * d))
    k.copy_(rand(g, B, 1, N, d, dtype=dtype))
    v.copy_(rand(g, B, 1, N, d, dtype=dtype))
    o, lse = pkg.window_attn_lse(q, k, v, window=20, sinks=1)
    grads = pkg.window_attn_bwd(q, k, v, o, lse, q, window=20, sinks=1)
    kc, vc = k.contiguous(), v.contiguous()
    want = pkg.window_attn_lse(q, kc, vc, window=20, sinks=1)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    assert all(torch.equal(a, b) for a, b in zip(grads, pkg.window_attn_bwd(q, kc, vc, o, lse, q, window=20, sinks=1)))
    assert pkg.get_device_status() == _lib.MOA_OK


@pytest.mark.parametrize("N", [1, 2, 50, 400])
def test_values_that_are_not_numbers_in_whole_and_cut_items(N):
    """A value that is not finite in each tile, seen and not seen, with items on one CTA, cut, and in clusters: the
    rows that do not see it are bit for bit what they are without it, or within the bound where they are computed
    again."""
    Hq, Hk, d, page, L, window = 8, 4, 64, 32, 5000, 600
    g = torch.Generator(device="cuda").manual_seed(N)
    for w in (window, 0):
        pool, table, rows = cache(g, [L, 900], Hk, page, d, d, "bf16")
        q = rand(g, 2, Hq, N, d, dtype="bf16")
        ln = torch.tensor([L, 900], dtype=torch.int32, device="cuda")
        t = L - N // 2 - 1                                # seen by half of the queries
        pool[table[0, t // page].long(), 1, t % page, d + 3] = float("inf")
        o, lse = pkg.kv_attn_lse(q, pool, table, ln, window=w or None)
        assert pkg.get_device_status() == _lib.MOA_OK
        see = seen(N, L, L, w, 0)
        hit = see[:, t]
        for h in range(Hq):
            x = rows[0][h // 2]
            ro, bound, _, _ = reference(q[0, h], x[:, :d], x[:, d:], see, "bf16")
            ok = (o[0, h].double() - ro).abs() <= bound
            if h // 2 == 1:
                assert bool(torch.isinf(o[0, h, hit, 3]).all())
                ok[hit, 3] = True
            assert bool(ok.all())


def test_two_streams_at_once():
    """Calls under way at the same time, each with its own outputs and workspaces."""
    g = torch.Generator(device="cuda").manual_seed(8)
    sets = []
    for i in range(2):
        q, k, v = rand(g, 1, 8, 2000, 64, dtype="bf16"), rand(g, 1, 2, 2000, 64, dtype="bf16"), rand(g, 1, 2, 2000, 64, dtype="bf16")
        sets.append((q, k, v))

    def both(t, stream=None):
        o, lse = pkg.window_attn_lse(*t, window=300, sinks=2, stream=stream)
        return [o, lse, *pkg.window_attn_bwd(*t, o, lse, t[0], window=300, sinks=2, stream=stream)]

    want = [both(t) for t in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[both(t, s) for t, s in zip(sets, streams)] for _ in range(4)]
    torch.cuda.synchronize()
    for r in got:
        for x, y in zip(r, want):
            assert all(torch.equal(a, b) for a, b in zip(x, y))


@pytest.mark.parametrize("N,M,window,sinks", [(27000, 27000, 3000, 4), (5000, 26000, 0, 0)])
def test_more_keys_and_values_than_l2_holds(N, M, window, sinks):
    """Work items are then taken in another order; rows at the beginning, the end and in between."""
    Hq, Hk, d = 16, 8, 128
    g = torch.Generator(device="cuda").manual_seed(N)
    q, k, v = (rand(g, 1, h, n, d, dtype="bf16") for h, n in ((Hq, N), (Hk, M), (Hk, M)))
    o, lse = pkg.window_attn_lse(q, k, v, window=window or None, sinks=sinks)
    assert pkg.get_device_status() == _lib.MOA_OK
    rows = torch.cat([torch.arange(70, device="cuda"), torch.randint(0, N, (200,), generator=g, device="cuda"),
                      torch.arange(N - 70, N, device="cuda")])
    p, j = (M - N + rows)[:, None], torch.arange(M, device="cuda")[None]
    see = (j <= p) & ((j > p - window) | (j < sinks)) if window else j <= p
    for h in range(Hq):
        check(o[0, h, rows], lse[0, h, rows], q[0, h, rows], k[0, h // 2], v[0, h // 2], see, "bf16")
    # every row was written: values of one give the sum of its weights, each rounded by 2^-8 at most, and the output once
    ones = pkg.window_attn(q, k, torch.ones_like(v), window=window or None, sinks=sinks)
    assert bool(((ones.float() - 1).abs() <= 2.0 ** -7 * 1.02).all())


def test_kernels_longer_than_the_limit_of_a_wait():
    """Forward and gradients of 40000 tokens and 32 heads take some 20 and 100 ms; with waits limited to 5 ms no wait runs out: each is for
    one tile, or lasts with the length of the context."""
    import os
    import subprocess
    import sys
    code = (
        "import torch, paper_2606_07713_gb300 as p\n"
        "q = torch.randn(1, 32, 40000, 128, device='cuda').bfloat16()\n"
        "k, v = (torch.randn(1, 4, 40000, 128, device='cuda').bfloat16() for _ in range(2))\n"
        "o, lse = p.window_attn_lse(q, k, v)\n"
        "g = p.window_attn_bwd(q, k, v, o, lse, q)\n"
        "v[:, :, 5, 7] = float('inf')\n"
        "p.window_attn(q[:, :, :300], k[:, :, :300].contiguous(), v[:, :, :300].contiguous())\n"
        "print('status', p.get_device_status(), all(bool(torch.isfinite(x).all()) for x in (o, *g)))\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, MOA_WAIT_LIMIT_NS="5000000", PYTHONPATH=root))
    assert r.returncode == 0 and "status 0 True" in r.stdout, r.stdout + r.stderr


@pytest.mark.parametrize("lens,Hq,Hk,N,dk,dv,page,window,sinks,causal", [
    ([16384], 8, 2, 1, 128, 128, 64, 0, 0, True),                    # 16 CTAs, eight tiles each
    ([5000, 16300], 2, 2, 3, 64, 128, 16, 0, 0, True),               # 16, lengths apart
    ([8100], 32, 8, 4, 128, 128, 16, 0, 0, True),                    # 8
    ([7000, 8192], 12, 6, 2, 128, 64, 48, 0, 0, False),              # 8, later tokens seen
    ([100000], 32, 8, 1, 128, 128, 128, 7500, 130, True),            # 8, a window
    ([2100], 32, 2, 8, 64, 64, 32, 0, 0, True),                      # 16, all 128 rows
    ([4096, 1, 0, 3000], 32, 8, 1, 128, 128, 16, 0, 0, True),        # 4
    ([1800, 2000, 5, 1999, 129, 2048], 16, 8, 5, 64, 64, 48, 0, 0, True),          # 2
    ([1000, 512, 900, 3, 128, 0, 640, 1024] * 2, 16, 8, 2, 128, 128, 16, 0, 0, True),   # 1: no clusters
    ([1000, 512, 900, 3, 128, 0, 640, 1025] * 2, 16, 8, 2, 128, 128, 16, 0, 0, True),   # more tiles: equal shares
    ([700] * 20, 16, 8, 2, 128, 64, 16, 200, 3, True),               # more items than SMs: equal shares
])
def test_few_query_rows(lens, Hq, Hk, N, dk, dv, page, window, sinks, causal):
    """Every size of a cluster and its neighbours, at the most tiles a CTA."""
    test_cache(lens, Hq, Hk, N, dk, dv, page, window, sinks, causal, "bf16")


@pytest.mark.parametrize("B,L", [(1, 8000), (4, 4000), (8, 2000), (16, 1000), (10, 4000)])
def test_hidden_values_that_are_not_numbers_in_clusters_and_shares(B, L):
    """The last token's values: not numbers, seen by the second of two queries only."""
    Hq, Hk, N, d, page = 16, 8, 2, 128, 16
    g = torch.Generator(device="cuda").manual_seed(B)
    pool, table, rows = cache(g, [L] * B, Hk, page, d, d, "bf16")
    q = rand(g, B, Hq, N, d, dtype="bf16", scale=1.5)
    ln = torch.full((B,), L, dtype=torch.int32, device="cuda")
    t = L - 1
    pool[table[B - 1, t // page].long(), 2, t % page, d:] = float("nan")
    o, lse = pkg.kv_attn_lse(q, pool, table, ln)
    assert pkg.get_device_status() == _lib.MOA_OK
    assert bool(torch.isnan(o[B - 1, 4:6, 1]).all()) and int(torch.isnan(o).sum()) == 2 * d
    see = seen(N, L, L, 0, 0)
    for b, h in ((B - 1, 4), (B - 1, 5), (B - 1, 6), (0, 0)):
        x = rows[b][h // 2]
        clean = torch.nan_to_num(x[:, d:].double())
        ro, bound, rl, _ = reference(q[b, h], x[:, :d], clean, see, "bf16")
        assert bool(((o[b, h, :1].double() - ro[:1]).abs() <= bound[:1]).all())
        if h != 4 and h != 5:
            assert bool(((o[b, h].double() - ro).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens", [[100], [300, 100], [1500, 40, 129], [200] * 20])
def test_queries_that_are_not_numbers(lens, dtype):
    """One such query of a head: its output and log-sum-exp are not numbers, in tiles that it sees in part too (their maximum
    is then that of the hidden scores), and no other row changes."""
    Hq, Hk, N, d = 8, 4, 3, 64
    g = torch.Generator(device="cuda").manual_seed(len(lens))
    pool, table, _ = cache(g, lens, Hk, 32, d, d, dtype)
    q = rand(g, len(lens), Hq, N, d, dtype=dtype)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    good, good_lse = pkg.kv_attn_lse(q, pool, table, ln, window=50, sinks=2)
    q[-1, 5, 1, 7] = float("nan")
    o, lse = pkg.kv_attn_lse(q, pool, table, ln, window=50, sinks=2)
    assert bool(torch.isnan(o[-1, 5, 1]).all()) and bool(torch.isnan(lse[-1, 5, 1]))
    o[-1, 5, 1], lse[-1, 5, 1] = good[-1, 5, 1], good_lse[-1, 5, 1]
    assert torch.equal(o, good) and torch.equal(lse, good_lse)


@pytest.mark.parametrize("lens,Hq,Hk,N,dk,dv,page,window,sinks,causal", [
    ([8192], 32, 8, 64, 128, 128, 16, 0, 0, True),           # clusters: 4 CTAs, 16 tiles each
    ([16000], 4, 1, 100, 64, 128, 48, 0, 0, True),           # 16
    ([4096, 70, 64, 3000], 32, 8, 64, 128, 64, 64, 0, 0, True),   # 2, lengths apart
    ([300, 200, 130], 9, 3, 130, 64, 64, 16, 90, 5, False),  # rows that no head fills, later tokens seen
    ([260], 200, 1, 3, 64, 64, 32, 0, 0, True),              # two chunks of heads
    ([40, 10], 6, 3, 130, 128, 128, 16, 0, 0, True),         # more queries than tokens
    ([8192 + 2048] * 2, 32, 8, 64, 128, 128, 16, 0, 0, True),     # one step more: equal shares
])
def test_more_rows_than_a_tile(lens, Hq, Hk, N, dk, dv, page, window, sinks, causal):
    test_cache(lens, Hq, Hk, N, dk, dv, page, window, sinks, causal, "bf16")


@pytest.mark.parametrize("B,Hq,Hk,N,M,dk,dv,window,sinks", [
    (3, 9, 3, 1500, 1700, 64, 64, 0, 0),      # heads that leave rows of a tile empty
    (3, 9, 3, 1501, 1501, 128, 64, 77, 5),
    (1, 200, 1, 203, 190, 64, 128, 33, 2),    # two chunks of heads, more queries than keys
    (7, 5, 5, 777, 901, 128, 128, 130, 1),
    (40, 4, 2, 300, 300, 64, 64, 0, 0),
])
def test_two_row_tiles(B, Hq, Hk, N, M, dk, dv, window, sinks):
    """Odd shapes with more work items than SMs, which take two row tiles each."""
    test_window("bf16", B, Hq, Hk, N, M, dk, dv, window, sinks)


@pytest.mark.parametrize("B,N", [(4, 1500), (1, 200)])
def test_hidden_values_that_are_not_numbers_without_pages(B, N):
    """Whole items of two row tiles and of one: a token's values that are not finite change only the rows that see it."""
    Hq, Hk, d, window = 8, 4, 64, 100
    g = torch.Generator(device="cuda").manual_seed(N)
    q, k, v = (rand(g, B, h, N, d, dtype="bf16", scale=1.5) for h in (Hq, Hk, Hk))
    clean = v.clone()
    t = N // 2
    v[-1, 1, t] = float("inf")
    o, lse = pkg.window_attn_lse(q, k, v, window=window)
    assert pkg.get_device_status() == _lib.MOA_OK
    assert bool(torch.isinf(o[-1, 2:4, t:t + window]).all()) and int(torch.isfinite(o).logical_not().sum()) == 2 * window * d
    see = seen(N, N, N, window, 0)
    for b, h in ((B - 1, 2), (B - 1, 3), (B - 1, 0), (0, 7)):
        ro, bound, _, _ = reference(q[b, h], k[b, h // 2], clean[b, h // 2], see, "bf16")
        ok = (o[b, h].double() - ro).abs() <= bound
        if b == B - 1 and h // 2 == 1:
            ok[t:t + window] = True
        assert bool(ok.all())
