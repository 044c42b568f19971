"""The paged 16- and 32-bit cache: appending with rotation (moa_kv_append) and attention over it
(moa_kv_attn) against plain implementations in 64 bits; the bounds are derived in window_reference.py."""
import math

import numpy as np
import pytest

import paper_2606_07713_gb300 as pkg
import window_reference as W
from ops_reference import bf16
from paper_2606_07713_gb300 import _lib
from test_kv4 import table_of

torch = pytest.importorskip("torch")

TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}


def cast(a, dtype):
    return bf16(a) if dtype == "bf16" else np.asarray(a, dtype=np.float32).astype(np.float64)


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
    return t if dtype is None else t.to(TORCH[dtype])


def host(t):
    return t.detach().double().cpu().numpy()


# -- append ---------------------------------------------------------------------------------------
APPENDS = [  # B, H_q, H_k, N, d_k, d_v, d_rot, page
    (1, 1, 1, 1, 64, 64, 64, 16),
    (2, 6, 3, 5, 128, 128, 128, 16),
    (3, 4, 2, 40, 128, 64, 32, 48),
    (2, 5, 1, 129, 64, 128, 16, 32),
    (1, 8, 4, 300, 128, 128, 96, 256),
    (33, 32, 8, 1, 128, 128, 128, 64),
]


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", APPENDS, ids=lambda s: "x".join(map(str, s)))
def test_append(shape, dtype, interleaved):
    B, Hq, Hk, N, dk, dv, rot, page = shape
    r = np.random.default_rng(sum(shape))
    q, k, v = (cast(r.normal(size=s), dtype) for s in ((B, Hq, N, dk), (B, Hk, N, dk), (B, Hk, N, dv)))
    L = N + 20
    table, n_pages = table_of(r, [L] * B, page)
    pos = np.stack([r.permutation(L)[:N] for _ in range(B)]).astype(np.int32)
    pos[r.random(size=pos.shape) < 0.1] = -1
    before = cast(r.normal(size=(n_pages, Hk, page, dk + dv)), dtype)
    cos, sin = pkg.rope_table(L, rot)
    pool = dev(before, dtype)
    # token-major views, as a projection leaves them
    view = lambda x: dev(x.transpose(0, 2, 1, 3), dtype).transpose(1, 2)  # noqa: E731
    got = pkg.kv_append(view(k), view(v), pool, dev(table), dev(pos), cos, sin, q=view(q), interleaved=interleaved)
    assert pkg.get_device_status() == _lib.MOA_OK
    c, s = host(cos), host(sin)
    live = (pos >= 0)[:, None, :, None]
    want_q = np.where(live, W.rotate(q, c, s, pos, interleaved), 0.0)
    assert np.all(np.abs(host(got) - want_q) <= W.rotate_bound(q, c, interleaved, dtype))
    want, slack = before.copy(), np.zeros_like(before)
    rk, bk = W.rotate(k, c, s, pos, interleaved), W.rotate_bound(k, c, interleaved, dtype)
    for b in range(B):
        for n in range(N):
            p = pos[b, n]
            if p < 0:
                continue
            at = (table[b, p // page], slice(None), p % page)
            want[at] = np.concatenate([rk[b, :, n], v[b, :, n]], -1)
            slack[at][:, :dk] = bk[b, :, n]
    assert np.all(np.abs(host(pool) - want) <= slack)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_without_rotation(dtype):
    B, H, N, dk, dv, page = 2, 3, 50, 128, 64, 32
    r = np.random.default_rng(4)
    k, v = (cast(r.normal(size=(B, H, N, d)), dtype) for d in (dk, dv))
    k[0, 0, 3, 7], v[1, 2, 4, 5] = np.nan, np.inf
    table, n_pages = table_of(r, [N] * B, page)
    pool = pkg.kv_pool(n_pages, H, page, dk, dv, dtype=TORCH[dtype])
    pos = np.tile(np.arange(N, dtype=np.int32), (B, 1))
    assert pkg.kv_append(dev(k, dtype), dev(v, dtype), pool, dev(table), dev(pos)) is None
    assert pkg.get_device_status() == _lib.MOA_OK
    got = host(pool)
    for b in range(B):
        rows = got[table[b, pos[b] // page], :, pos[b] % page]       # N, H, dk + dv
        assert np.array_equal(rows, np.concatenate([k[b], v[b]], -1).transpose(1, 0, 2), equal_nan=True)


@pytest.mark.gpu
def test_append_in_place_of_a_projection():
    """q, k and v as slices of one buffer, the rotated queries written over theirs."""
    B, Hq, Hk, N, d, page = 2, 4, 2, 33, 64, 16
    g = torch.Generator().manual_seed(0)
    qkv = torch.randn(B, N, Hq + 2 * Hk, d, generator=g).bfloat16().cuda().transpose(1, 2)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
    cos, sin = pkg.rope_table(64, d)
    table = torch.arange(B * 3, dtype=torch.int32, device="cuda").view(B, 3)
    pos = torch.arange(N, dtype=torch.int32, device="cuda").expand(B, N).contiguous()
    pools = [pkg.kv_pool(B * 3, Hk, page, d, d) for _ in range(2)]
    want = pkg.kv_append(k.contiguous(), v.contiguous(), pools[0], table, pos, cos, sin, q=q.contiguous())
    keep = qkv[:, Hq:].clone()
    got = pkg.kv_append(k, v, pools[1], table, pos, cos, sin, q=q, out=q)
    assert pkg.get_device_status() == _lib.MOA_OK
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want) and torch.equal(pools[0], pools[1])
    assert torch.equal(qkv[:, Hq:], keep)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_outside_the_tables(dtype):
    """Positions past the table of pages or of angles and pages outside the pool are not written, and
    are reported; the others are as ever."""
    B, Hq, Hk, N, d, page = 1, 2, 2, 6, 64, 16
    r = np.random.default_rng(5)
    q, k, v = (cast(r.normal(size=(B, h, N, d)), dtype) for h in (Hq, Hk, Hk))
    cos, sin = pkg.rope_table(40, d)
    table = np.array([[2, -1, 0, 99]], dtype=np.int32)
    pos = np.array([[5, 20, 70, 33, 39, 45]], dtype=np.int32)   # fine, no page, past all, fine, fine, no angles
    pool = dev(np.full((3, Hk, page, 2 * d), 3.0), dtype)
    got = host(pkg.kv_append(dev(k, dtype), dev(v, dtype), pool, dev(table), dev(pos), cos, sin, q=dev(q, dtype)))
    assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
    assert pkg.get_device_status() == _lib.MOA_OK
    assert np.array_equal(np.isnan(got[0, 0, :, 0]), [False, False, True, False, False, True])
    pool = host(pool)
    touched = np.zeros((3, page), dtype=bool)
    for n, (pg, at) in {0: (2, 5), 3: (0, 1), 4: (0, 7)}.items():
        touched[pg, at] = True
        assert np.array_equal(pool[pg, :, at, d:], v[0, :, n])
    assert np.all(pool.transpose(0, 2, 1, 3)[~touched] == 3.0)


# -- attention ------------------------------------------------------------------------------------
def cache_of(r, lens, Hk, page, dk, dv, dtype, width=None, junk=np.nan):
    """(pool, table, keys, values by sequence); what lies past a sequence's end is `junk`."""
    table, n_pages = table_of(r, lens, page, width=width)
    pool = np.full((n_pages, Hk, page, dk + dv), junk)
    keys, values = [], []
    scale = np.exp(0.3 * r.normal(size=(Hk, 1, dk)))
    for b, n in enumerate(lens):
        k, v = cast(r.normal(size=(Hk, n, dk)) * scale, dtype), cast(r.normal(size=(Hk, n, dv)), dtype)
        for t in range(n):
            pool[table[b, t // page], :, t % page] = np.concatenate([k[:, t], v[:, t]], -1)
        keys.append(k)
        values.append(v)
    return pool, table, keys, values


def check_attention(q, keys, values, lens, window, sinks, causal, dtype, o, lse, scale=None):
    dk = q.shape[3]
    scale = dk ** -0.5 if scale is None else scale
    for b, n in enumerate(lens):
        if n == 0:
            assert np.all(o[b] == 0) and np.all(lse[b] == -np.inf)
            continue
        ro, rl, av, size = W.attention(q[b], keys[b], values[b], n, window, sinks, scale, causal)
        bound = W.out_bound(ro, av, size, dk, dtype)
        err = np.abs(o[b] - ro)
        assert np.all(err <= bound), f"sequence {b}: {np.max(err / bound)} of the bound"
        assert np.array_equal(np.isfinite(lse[b]), np.isfinite(rl))
        with np.errstate(invalid="ignore"):
            diff = np.where(np.isfinite(rl), np.abs(lse[b] - rl), 0.0)
        assert np.all(diff <= W.lse_bound(rl, size, dk))


def run_attention(lens, Hq, Hk, N, dk, dv, page, window, sinks, causal, dtype, seed, released=False, max_len=None):
    r = np.random.default_rng(seed)
    pool, table, keys, values = cache_of(r, lens, Hk, page, dk, dv, dtype)
    if released:
        # pages before every window and behind the sinks were given back
        for b, n in enumerate(lens):
            for s in range(table.shape[1]):
                if s * page >= sinks and (s + 1) * page <= n - N - window + 1:
                    table[b, s] = -7
    q = cast(1.5 * r.normal(size=(len(lens), Hq, N, dk)), dtype)
    o, lse = pkg.kv_attn_lse(dev(q, dtype), dev(pool, dtype), dev(table), dev(np.array(lens, dtype=np.int32)),
                             max_len=max_len, window=window or None, sinks=sinks, causal=causal)
    assert pkg.get_device_status() == _lib.MOA_OK
    check_attention(q, keys, values, lens, window, sinks, causal, dtype, host(o), host(lse))


ATTENTIONS = [  # lens, H_q, H_k, N, d_k, d_v, page, window, sinks
    ([1], 1, 1, 1, 64, 64, 16, 0, 0),
    ([0, 1, 17], 4, 2, 1, 128, 128, 16, 0, 0),
    ([127, 128, 129, 0], 8, 1, 1, 128, 64, 32, 0, 0),
    ([300, 5, 1000], 6, 2, 1, 64, 128, 48, 0, 0),
    ([1000, 77, 3], 16, 2, 4, 128, 128, 64, 0, 0),      # drafts, rows before the sequence's start
    ([513], 40, 8, 3, 64, 64, 256, 0, 0),
    ([2000, 900], 4, 4, 1, 128, 128, 16, 100, 4),
    ([2000, 50], 12, 4, 5, 128, 64, 48, 333, 2),
    ([700, 333], 8, 2, 200, 128, 128, 64, 0, 0),        # chunks
    ([600], 8, 2, 200, 64, 64, 16, 64, 5),
    ([900, 100], 5, 1, 300, 128, 128, 96, 128, 130),
    ([450], 3, 1, 450, 64, 128, 112, 0, 0),             # a whole prompt
    ([260, 90], 2, 2, 129, 128, 64, 32, 1, 0),
    ([140], 130, 1, 2, 64, 64, 16, 20, 1),
]


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", ATTENTIONS, ids=lambda c: "x".join(map(str, c)).replace(" ", ""))
def test_attention(case, dtype, causal):
    lens, *rest = case
    run_attention(lens, *rest, causal, dtype, seed=sum(lens) + sum(rest), released=rest[6] > 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_contexts(dtype):
    """Many shares of one sequence, a close bound of the lengths and a wide one."""
    run_attention([6000, 3], 8, 2, 1, 128, 128, 32, 0, 0, True, dtype, 1, max_len=6000)
    run_attention([5000], 4, 1, 2, 64, 64, 16, 3000, 4, True, dtype, 2, released=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_lengths_and_pages_outside_their_range(dtype):
    """A length past max_len is clamped to it, one below zero to zero, tokens of pages outside the pool read
    as zeros; all are reported."""
    Hq, Hk, d, page = 4, 2, 64, 16
    r = np.random.default_rng(3)
    lens = [100, 60, 40]
    pool, table, keys, values = cache_of(r, lens, Hk, page, d, d, dtype, width=8)
    q = cast(r.normal(size=(3, Hq, 1, d)), dtype)
    args = dev(q, dtype), dev(pool, dtype)
    for told in ([2000, 60, 40], [100, -5, 40]):
        o, lse = pkg.kv_attn_lse(*args, dev(table), dev(np.array(told, dtype=np.int32)), max_len=100)
        assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
        clamped = [min(max(n, 0), 100) for n in told]
        check_attention(q, [k[:, :n] for k, n in zip(keys, clamped)], [v[:, :n] for v, n in zip(values, clamped)], clamped, 0, 0,
                        True, dtype, host(o), host(lse))
    for page_number in (-1, len(pool), 2 ** 31 - 1):
        other = table.copy()
        other[0, 2] = page_number
        o, lse = pkg.kv_attn_lse(*args, dev(other), dev(np.array(lens, dtype=np.int32)))
        assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
        zk, zv = keys[0].copy(), values[0].copy()
        zk[:, 32:48] = zv[:, 32:48] = 0
        check_attention(q, [zk, *keys[1:]], [zv, *values[1:]], lens, 0, 0, True, dtype, host(o), host(lse))


@pytest.mark.gpu
@pytest.mark.parametrize("N", [1, 3, 150])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_hidden_values_that_are_not_numbers(dtype, N):
    """Tokens before the window, or after a query of a chunk, may hold anything."""
    Hq, Hk, d, page, L, window = 4, 2, 64, 32, 400, 100
    r = np.random.default_rng(7)
    pool, table, keys, values = cache_of(r, [L], Hk, page, d, d, dtype)
    q = cast(r.normal(size=(1, Hq, N, d)), dtype)
    first = L - N - window + 1                            # the first token that any window reaches
    for t in [first - 1, first - 3] + ([L - 1] if N > 1 else []):
        pool[table[0, t // page], :, t % page] = np.nan
    o, lse = pkg.kv_attn_lse(dev(q, dtype), dev(pool, dtype), dev(table), dev(np.array([L], dtype=np.int32)), window=window,
                             sinks=2)
    assert pkg.get_device_status() == _lib.MOA_OK
    rows = N - 1 if N > 1 else N                          # the last query of a chunk sees token L - 1
    ro, rl, av, size = W.attention(q[0], keys[0], values[0], L, window, 2, d ** -0.5)
    assert np.all((np.abs(host(o)[0] - ro) <= W.out_bound(ro, av, size, d, dtype))[:, :rows])
    if N > 1:
        assert np.all(np.isnan(host(o)[0, :, -1]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["token major", "broadcast heads", "broadcast rows"])
def test_query_layouts(kind, dtype):
    B, Hq, Hk, N, d, page, lens = 2, 6, 2, 4, 64, 16, [90, 33]
    r = np.random.default_rng(11)
    pool, table, keys, values = cache_of(r, lens, Hk, page, d, d, dtype)
    q = cast(r.normal(size=(B, Hq, N, d)), dtype)
    big = torch.full((B, N + 1, Hq, d), 5.0, dtype=TORCH[dtype], device="cuda")
    out = big[:, :N].transpose(1, 2)
    if kind == "token major":
        t = dev(q.transpose(0, 2, 1, 3), dtype).transpose(1, 2)
    else:
        axis = 1 if kind == "broadcast heads" else 2
        q = np.broadcast_to(np.take(q, [0], axis), q.shape)
        t = dev(np.take(q, [0], axis), dtype).expand(*q.shape)
    o, lse = pkg.kv_attn_lse(t, dev(pool, dtype), dev(table), dev(np.array(lens, dtype=np.int32)), window=50, out=out)
    assert pkg.get_device_status() == _lib.MOA_OK and bool((big[:, N] == 5).all())
    check_attention(q, keys, values, lens, 50, 0, True, dtype, host(o), host(lse))


# -- together -------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_a_prompt_in_chunks_then_tokens(window, sinks, dtype):
    """A prompt appended and attended in chunks, then token by token, gives the rows of one windowed
    attention over the whole sequence: both sides against the same 64-bit rows, from the keys as the cache
    holds them."""
    B, Hq, Hk, L, d, page = 2, 8, 2, 331, 64, 16
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(B, h, L, d, generator=g).cuda().to(TORCH[dtype]) for h in (Hq, Hk, Hk))
    cos, sin = pkg.rope_table(L, d)
    pages = torch.randperm(B * 21, generator=g).to(torch.int32).view(B, 21).cuda()
    pool = pkg.kv_pool(B * 21, Hk, page, d, d, dtype=TORCH[dtype])
    outs, turned, at = [], [], 0
    for n in (200, 37, 90, 1, 1, 1, 1):
        pos = torch.arange(at, at + n, dtype=torch.int32, device="cuda").expand(B, n).contiguous()
        part = [x[:, :, at:at + n] for x in (q, k, v)]
        qr = pkg.kv_append(part[1], part[2], pool, pages, pos, cos, sin, q=part[0])
        at += n
        lens = torch.full((B,), at, dtype=torch.int32, device="cuda")
        outs.append(pkg.kv_attn(qr, pool, pages, lens, window=window or None, sinks=sinks))
        turned.append(qr)
    rows = pool[pages.long()].transpose(1, 2).flatten(2, 3)[:, :, :L]
    whole, lse = pkg.window_attn_lse(torch.cat(turned, 2), rows[..., :d].contiguous(), rows[..., d:].contiguous(),
                                     window=window or None, sinks=sinks)
    assert pkg.get_device_status() == _lib.MOA_OK
    qh, kh, vh = host(torch.cat(turned, 2)), host(rows[..., :d]), host(rows[..., d:])
    for o in (host(torch.cat(outs, 2)), host(whole)):
        check_attention(qh, kh, vh, [L] * B, window, sinks, True, dtype, o, host(lse))


def _step(t, stream=None):
    """Rotation and append, attention over the cache, windowed attention with its gradients."""
    s = dict(stream=stream)
    qr = pkg.kv_append(t["k"], t["v"], t["pool"], t["pages"], t["pos"], t["cos"], t["sin"], q=t["q"], **s)
    o, lse = pkg.kv_attn_lse(qr, t["pool"], t["pages"], t["lens"], window=t["window"], sinks=2, **s)
    one = pkg.kv_attn(qr[:, :, -1:], t["pool"], t["pages"], t["lens"], **s)
    w, wl = pkg.window_attn_lse(qr, t["k"], t["v"], window=t["window"], sinks=2, **s)
    return [qr, t["pool"], o, lse, one, w, wl, *pkg.window_attn_bwd(qr, t["k"], t["v"], w, wl, qr, window=t["window"], sinks=2, **s)]


def _inputs(dtype, seed):
    g = torch.Generator().manual_seed(seed)
    B, Hq, Hk, N, d, page = 3, 8, 2, 157, 64, 16
    r = lambda *s: torch.randn(*s, generator=g).to("cuda", dtype)  # noqa: E731
    cos, sin = pkg.rope_table(256, d)
    return dict(q=r(B, Hq, N, d), k=r(B, Hk, N, d), v=r(B, Hk, N, d), cos=cos, sin=sin, window=40,
                pos=torch.arange(N, dtype=torch.int32, device="cuda")[None].repeat(B, 1).contiguous(),
                pages=torch.randperm(B * 10, generator=g).to(torch.int32).reshape(B, 10).cuda(),
                pool=pkg.kv_pool(B * 10, Hk, page, d, d, dtype=dtype),
                lens=torch.tensor([N, N - 1, 5], dtype=torch.int32, device="cuda"))


def _same(got, want):
    for x, y in zip(got, want, strict=True):
        assert torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_stream_that_is_not_the_current_one(dtype):
    t = _inputs(dtype, 0)
    want = [x.clone() for x in _step(t)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = _step(t, side)
    noise = [torch.full((1 << 16,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    side.synchronize()
    torch.cuda.synchronize()
    _same(got, want)
    assert all(bool((n == 7).all()) for n in noise)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured_graphs_replay_on_new_inputs(dtype):
    """Two graphs of the same inputs, each with workspaces of its own pool, replayed in turn."""
    t = _inputs(dtype, 2)
    _step(t)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            outs.append(_step(t))
        graphs.append(graph)
    other = _inputs(dtype, 3)
    for name in ("q", "k", "v", "lens", "pages"):
        t[name].copy_(other[name])
    for graph in graphs:
        graph.replay()
    torch.cuda.synchronize()
    got = [[x.clone() for x in o] for o in outs]
    want = _step(t)
    _same(got[0], want)
    _same(got[1], want)


# -- refusals, without a GPU ------------------------------------------------------------------------
A = [0x10000000 * (i + 1) for i in range(12)]     # never dereferenced
APPEND = dict(Q=A[0], K=A[1], V=A[2], cos=A[3], sin=A[4], pool=A[5], pages=A[6], pos=A[7], Qo=A[8], B=1, H_q=4, H_k=2, N=8,
              d_k=64, d_v=64, d_rot=64, n_pos=100, n_pages=9, page_tokens=16, max_pages=4,
              strides=[4 * 512, 512, 64, 2 * 512, 512, 64, 2 * 512, 512, 64, 4 * 512, 512, 64], interleaved=0, dtype=1,
              stream=None)
ATTEND = dict(Q=A[0], pool=A[5], pages=A[6], lens=A[7], O=A[8], LSE=A[9], B=1, H_q=4, H_k=2, N=8, d_k=64, d_v=64, n_pages=9,
              page_tokens=16, max_pages=4, max_len=64, window=0, sinks=0, strides=[4 * 512, 512, 64, 4 * 512, 512, 64],
              scale=0.1, causal=1, dtype=1, workspace=A[10], workspace_bytes=1 << 30, stream=None)
INVALID, SHAPE, ALIGN, TYPE = (_lib.MOA_ERR_INVALID_ARG, _lib.MOA_ERR_UNSUPPORTED_SHAPE, _lib.MOA_ERR_MISALIGNED,
                               _lib.MOA_ERR_UNSUPPORTED_DTYPE)


@pytest.mark.parametrize("changes,status", [
    (dict(B=0), INVALID), (dict(N=0), INVALID), (dict(H_k=0), INVALID), (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID),
    (dict(K=None), INVALID), (dict(pool=None), INVALID), (dict(pos=None), INVALID), (dict(Qo=None), INVALID),
    (dict(cos=None), INVALID), (dict(cos=None, sin=None), INVALID), (dict(page_tokens=24), SHAPE), (dict(page_tokens=0), INVALID),
    (dict(d_k=96), SHAPE), (dict(d_v=32), SHAPE), (dict(d_rot=24), SHAPE), (dict(d_rot=80), SHAPE), (dict(n_pos=0), INVALID),
    (dict(dtype=3), TYPE), (dict(pool=A[5] + 8), ALIGN), (dict(pages=A[6] + 2), ALIGN), (dict(K=A[1] + 2), ALIGN),
    (dict(Qo=A[1]), INVALID), (dict(pool=A[1]), INVALID), (dict(pool=A[6]), INVALID), (dict(Qo=A[5]), INVALID),
    (dict(Qo=A[0] + 128), INVALID), (dict(pool=A[3]), INVALID), (dict(n_pages=2 ** 31), SHAPE), (dict(B=2 ** 40), SHAPE),
], ids=lambda x: str(x)[:40])
def test_append_refusals(changes, status):
    assert pkg.moa_kv_append(**dict(APPEND, **changes)) == status
    assert pkg.moa_last_error()


@pytest.mark.parametrize("changes,status", [
    (dict(B=0), INVALID), (dict(N=0), INVALID), (dict(H_q=0), INVALID), (dict(H_q=3), SHAPE), (dict(max_len=0), INVALID),
    (dict(max_len=65), INVALID), (dict(window=-1), INVALID), (dict(sinks=-2), INVALID), (dict(lens=None), INVALID),
    (dict(lens=A[7] + 1), ALIGN), (dict(pool=None), INVALID), (dict(page_tokens=20), SHAPE), (dict(d_k=32), SHAPE),
    (dict(O=A[0]), INVALID), (dict(O=A[5]), INVALID), (dict(LSE=A[8]), INVALID), (dict(LSE=A[9] + 2), ALIGN),
    (dict(scale=float("nan")), INVALID), (dict(dtype=9), TYPE), (dict(Q=A[0] + 4), ALIGN), (dict(n_pages=2 ** 31 - 1), SHAPE),
], ids=lambda x: str(x)[:40])
def test_attention_refusals(changes, status):
    assert pkg.moa_kv_attn(**dict(ATTEND, **changes)) == status
    assert pkg.moa_last_error()


def test_pool_sizes():
    assert pkg.moa_kv_pool_bytes(3, 2, 16, 64, 128, 1) == 3 * 2 * 16 * 192 * 2
    assert pkg.moa_kv_pool_bytes(3, 2, 16, 64, 128, 0) == 3 * 2 * 16 * 192 * 4
    for bad in ((0, 2, 16, 64, 64, 1), (3, 2, 8, 64, 64, 1), (3, 2, 16, 96, 64, 1), (3, 2, 16, 64, 64, 5),
                (2 ** 40, 2 ** 20, 16, 64, 64, 1)):
        assert pkg.moa_kv_pool_bytes(*bad) == 0
    with pytest.raises(ValueError):
        pkg.kv_pool(1, 1, 24, 64, 64, device="cpu")
    with pytest.raises(TypeError):
        pkg.kv_pool(1, 1, 16, 64, 64, dtype=torch.float16, device="cpu")
    pool = pkg.kv_pool(3, 2, 16, 64, 128, device="cpu")
    assert tuple(pool.shape) == (3, 2, 16, 192) and pool.dtype == torch.bfloat16


@pytest.mark.gpu
def test_binding_refusals():
    x = torch.zeros(1, 2, 8, 64, device="cuda")
    pool, pages = pkg.kv_pool(4, 2, 16, 64, 64, dtype=torch.float32), torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    pos, lens = torch.zeros(1, 8, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="cos and sin"):
        pkg.kv_append(x, x, pool, pages, pos, q=x)
    with pytest.raises(TypeError):
        pkg.kv_append(x.bfloat16(), x.bfloat16(), pool, pages, pos)
    with pytest.raises(ValueError):
        pkg.kv_append(x, x, pool, pages, pos, out=x)
    with pytest.raises(ValueError):
        pkg.kv_append(x, x, pool, pages, pos[:, :4])
    with pytest.raises(ValueError):
        pkg.kv_append(x[:, :1], x[:, :1], pool, pages, pos)
    with pytest.raises(TypeError):
        pkg.kv_attn(x.bfloat16(), pool, pages, lens)
    with pytest.raises(ValueError, match="window"):
        pkg.kv_attn(x, pool, pages, lens, window=0)
    with pytest.raises(pkg.MoaError):
        pkg.kv_attn(x, pool, pages, lens, max_len=17)
    with pytest.raises(pkg.MoaError):
        pkg.kv_attn(x[:, :1].expand(1, 3, 8, 64), pool, pages, lens)
    with pytest.raises(TypeError):
        pkg.kv_attn(x, pool, pages.long(), lens)


def test_attention_refuses_lengths_past_the_last_tile():
    """max_len 2^31 - 1024 of 2^17 pages of 2^14 tokens: one more than the kernels take."""
    a = dict(ATTEND, page_tokens=2 ** 14, max_pages=2 ** 17, max_len=2 ** 31 - 1024, window=0, sinks=0)
    assert pkg.moa_kv_attn(**a) == INVALID and "max_len" in pkg.moa_last_error()
