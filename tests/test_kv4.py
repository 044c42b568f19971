"""The paged 4-bit cache (moa_kv4_write, moa_kv4_read) and attention over it (moa_kv4_attn) against a
plain implementation in 64 bits.

Writing and reading are exact: codes and scales are those of the definition (s = bf16(max|x| / 7),
code = rint(x / s)), what is read is code * s rounded once, and no byte outside the named rows
changes.

Attention, element by element, with p the row's softmax weights:
  bf16  weights and values are rounded to bf16 (8 significant bits) at most once each
        (2 * 2^-8 sum p |v|), the output once (2^-8 |o|);
  fp32  products of 24 bits: 2^-23 of each instead.
  Both  scores accumulate in fp32 over d_k products: each within e = (d_k + 8) 2^-24 scale
        max_j sum_c |q_c k_jc| of its value, which moves every weight by at most 2 e relative; the
        exponentials and their differences from the maximum, at most 2^7 here, add 2^-17; sums of
        n weighted values in fp32 add n 2^-24, here at most 2^-13 in the longest rows and averaged
        over four warps and the ranges: 2^-15.
  LSE   e + 2^-17 + 2^-20 |lse|.
"""
import math

import numpy as np
import pytest

import ops_reference as R
import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib

torch = pytest.importorskip("torch")


def cast(a, dtype):
    return R.bf16(a) if dtype == "bf16" else np.asarray(a, dtype=np.float32).astype(np.float64)


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
    return t if dtype is None else t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def host(t):
    return t.detach().double().cpu().numpy()


def table_of(r, lens, page, spare=2, width=None):
    """Shuffled pages for sequences of these lengths: (table with -1 past the last page, n_pages)."""
    per = [-(-n // page) for n in lens]
    order = r.permutation(sum(per) + spare)
    table = np.full((len(lens), width or max(1, max(per))), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    return table, len(order)


# -- write and read -------------------------------------------------------------------------------
CACHES = [  # B, H, N, d_k, d_v, page
    (1, 1, 1, 64, 64, 16),
    (2, 3, 5, 128, 128, 16),
    (3, 2, 40, 128, 64, 48),
    (2, 1, 129, 64, 128, 32),
    (1, 4, 300, 128, 128, 256),
    (5, 8, 17, 64, 64, 64),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", CACHES, ids=lambda s: "x".join(map(str, s)))
def test_write_and_read_are_exact(shape, dtype):
    B, H, N, dk, dv, page = shape
    r = np.random.default_rng(sum(shape))
    k = cast(r.normal(size=(B, H, N, dk)) * np.exp(2 * r.normal(size=(B, H, N, 1))), dtype)
    v = cast(r.normal(size=(B, H, N, dv)), dtype)
    v[:, :, N // 2] = 0.0                                 # a row of zeros
    k[0, 0, 0, :32] = cast(np.arange(32) - 16.0, dtype)   # ties of the rounding among them
    table, n_pages = table_of(r, [N + 20] * B, page)
    # the tokens in any order of positions, some of them padding
    pos = np.stack([r.permutation(N + 20)[:N] for _ in range(B)]).astype(np.int32)
    pos[r.random(size=pos.shape) < 0.1] = -1
    before = r.integers(0, 256, size=(n_pages, H, page // 16, 9 * (dk + dv))).astype(np.uint8)
    pool = dev(before)
    pkg.kv4_write(dev(k, dtype), dev(v, dtype), pool, dev(table), dev(pos))
    got_k, got_v = pkg.kv4_read(pool, dev(table), dev(pos), dk, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    assert pkg.get_device_status() == _lib.MOA_OK
    (kc, ks), (vc, vs) = R.quantise(k), R.quantise(v)
    live = (pos >= 0)[:, None, :, None]
    assert np.array_equal(host(got_k), np.where(live, cast(R.values(kc, ks), dtype), 0.0))
    assert np.array_equal(host(got_v), np.where(live, cast(R.values(vc, vs), dtype), 0.0))
    # the bytes: what the rows' places held is replaced, everything else is as it was
    kc0, ks0, vc0, vs0 = R.unpack(before, dk, dv)
    for b in range(B):
        for n in range(N):
            p = pos[b, n]
            if p < 0:
                continue
            at = (table[b, p // page], slice(None), p % page // 16, p % 16)
            kc0[at], ks0[at], vc0[at], vs0[at] = kc[b, :, n], ks[b, :, n], vc[b, :, n], vs[b, :, n]
    after = pool.cpu().numpy()
    kc1, ks1, vc1, vs1 = R.unpack(after, dk, dv)
    assert np.array_equal(kc1, kc0) and np.array_equal(vc1, vc0)
    assert np.array_equal(ks1, ks0, equal_nan=True) and np.array_equal(vs1, vs0, equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_extreme_values(dtype):
    """Groups with NaN or infinities read as NaN, their neighbours as ever; the largest and the
    smallest magnitudes keep to the definition."""
    B, H, N, dk, dv, page = 1, 1, 16, 128, 64, 16
    k = np.ones((B, H, N, dk))
    v = np.ones((B, H, N, dv))
    k[0, 0, 1, 5], k[0, 0, 2, 40], v[0, 0, 3, 63] = np.nan, np.inf, -np.inf
    k[0, 0, 4] = cast(np.full(dk, 3.0e38), dtype)
    k[0, 0, 5, ::2] = -3.3e38
    k[0, 0, 6] = cast(np.linspace(-1e-38, 1e-38, dk), dtype)
    k[0, 0, 7], k[0, 0, 7, 3] = 0.0, 2.0 ** -133            # the smallest bf16: its scale is zero
    k = cast(k, dtype)
    pool = pkg.kv4_pool(1, H, page, dk, dv)
    table, pos = np.zeros((1, 1), np.int32), np.arange(16, dtype=np.int32)[None]
    pkg.kv4_write(dev(k, dtype), dev(v, dtype), pool, dev(table), dev(pos))
    got_k, got_v = pkg.kv4_read(pool, dev(table), dev(pos), dk, dtype=torch.float32)
    kc, ks = R.quantise(k)
    vc, vs = R.quantise(cast(v, dtype))
    with np.errstate(over="ignore"):
        assert np.array_equal(host(got_k), (R.values(kc, ks)).astype(np.float32).astype(np.float64), equal_nan=True)
        assert np.array_equal(host(got_v), (R.values(vc, vs)).astype(np.float32).astype(np.float64), equal_nan=True)
    assert np.isnan(host(got_k)[0, 0, 1, :32]).all() and np.isfinite(host(got_k)[0, 0, 1, 32:]).all()


@pytest.mark.gpu
def test_strided_tensors_and_places_outside_the_tables():
    B, H, N, dk, dv, page = 2, 4, 21, 128, 128, 16
    r = np.random.default_rng(4)
    table, n_pages = table_of(r, [N] * B, page)
    pos = np.tile(np.arange(N, dtype=np.int32), (B, 1))
    whole = torch.randn(B, N, 2 * H, dk, device="cuda:0").to(torch.bfloat16)
    k, v = whole[:, :, :H].transpose(1, 2), whole[:, :, H:].transpose(1, 2)
    a, b = (pkg.kv4_pool(n_pages, H, page, dk, dv) for _ in range(2))
    pkg.kv4_write(k, v, a, dev(table), dev(pos))
    pkg.kv4_write(k.contiguous(), v.contiguous(), b, dev(table), dev(pos))
    assert torch.equal(a, b)
    want = pkg.kv4_read(a, dev(table), dev(pos), dk)
    out = torch.zeros(B, N, 2 * H, dk, device="cuda:0", dtype=torch.bfloat16)
    ko, vo = out[:, :, :H].transpose(1, 2), out[:, :, H:].transpose(1, 2)
    pkg.kv4_read(a, dev(table), dev(pos), dk, out=(ko, vo))
    assert torch.equal(ko, want[0]) and torch.equal(vo, want[1])
    # a position past the table, a page outside the pool
    bad = pos.copy()
    bad[0, 4] = table.shape[1] * page
    wrong = table.copy()
    wrong[1, 1] = n_pages
    for tb, ps, rows in ((table, bad, (0, slice(4, 5))), (wrong, pos, (1, slice(16, N)))):
        c = a.clone()
        pkg.kv4_write(k * 2, v * 2, c, dev(tb), dev(ps))
        assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
        ck, _ = pkg.kv4_read(c, dev(table), dev(pos), dk)
        keep = ck[rows[0], :, rows[1]]
        assert torch.equal(keep, want[0][rows[0], :, rows[1]])       # not written
        rk, rv = pkg.kv4_read(c, dev(tb), dev(ps), dk)
        assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
        assert bool(torch.isnan(rk[rows[0], :, rows[1]]).all()) and bool(torch.isnan(rv[rows[0], :, rows[1]]).all())
        assert int(torch.isnan(rk).sum()) == rk[rows[0], :, rows[1]].numel()


# -- attention ------------------------------------------------------------------------------------
def problem(lens, Hq, Hk, N, dk, dv, page, dtype, seed, q_scale=1.0, garbage=True, width=None):
    r = np.random.default_rng(seed)
    table, n_pages = table_of(r, lens, page, width=width)
    k = r.normal(size=(n_pages, Hk, page // 16, 16, dk)) * np.exp(0.3 * r.normal(size=dk))
    v = r.normal(size=(n_pages, Hk, page // 16, 16, dv))
    (kc, ks), (vc, vs) = R.quantise(k), R.quantise(v)
    if garbage:     # what lies past a sequence's end, and in pages of nobody, is anything
        mine = np.zeros((n_pages, page), dtype=bool)
        for b, n in enumerate(lens):
            for p in range(n):
                mine[table[b, p // page], p % page] = True
        hidden = ~mine.reshape(n_pages, 1, page // 16, 16)
        for s in (ks, vs):
            bad = np.where(r.random(size=s.shape) < 0.5, np.nan, np.inf)
            s[:] = np.where(hidden[..., None], bad, s)
    pool = R.pack(kc, ks, vc, vs)
    q = cast(q_scale * r.normal(size=(len(lens), Hq, N, dk)), dtype)
    flat_k = R.values(kc, ks).transpose(0, 2, 3, 1, 4).reshape(n_pages, page, Hk, dk)
    flat_v = R.values(vc, vs).transpose(0, 2, 3, 1, 4).reshape(n_pages, page, Hk, dv)
    return q, pool, table, flat_k, flat_v


def reference(q, table, flat_k, flat_v, lens, scale, causal):
    out = []
    for b, n in enumerate(lens):
        pages = table[b, :max(1, -(-n // flat_k.shape[1]))]
        pages = pages if n else np.zeros(1, dtype=np.int64)
        k, v = (f[pages].reshape(-1, *f.shape[2:]).transpose(1, 0, 2)[:, :max(n, 1)] for f in (flat_k, flat_v))
        out.append(R.attention(q[b], k, v, n, scale, causal))
    return [np.stack(x) for x in zip(*out)]


def check(o, lse, ref, dk, dtype, what=""):
    want, want_lse, av, size = ref
    e = (dk + 8) * 2.0 ** -24 * size
    once = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    bound = (2 * once + 2 * e[..., None] + 2.0 ** -17 + 2.0 ** -15) * av + once * np.abs(want)
    err = np.abs(host(o) - want)
    assert np.all(err <= bound), (what, float(np.max(err / np.maximum(bound, 1e-300))))
    if lse is not None:
        got = host(lse)
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got), empty), what
        d = np.abs(got[~empty] - want_lse[~empty])
        assert np.all(d <= e[~empty] + 2.0 ** -17 + 2.0 ** -20 * np.abs(want_lse[~empty])), (what, float(d.max(initial=0)))


ATTN = [  # lens, Hq, Hk, N, d_k, d_v, page, causal
    ([1], 1, 1, 1, 64, 64, 16, True),
    ([0], 4, 2, 1, 128, 128, 16, True),
    ([0, 1, 15, 16, 17, 63, 64, 65, 200], 4, 4, 1, 64, 64, 16, True),
    ([5, 1000, 0, 333], 8, 2, 1, 128, 128, 32, True),
    ([700], 8, 1, 1, 128, 64, 48, True),
    ([300, 77], 12, 4, 3, 128, 64, 48, True),
    ([300, 2, 0], 10, 2, 4, 64, 128, 64, True),       # queries before a sequence's first token
    ([129, 64], 3, 3, 2, 128, 128, 256, False),
    ([40, 3], 14, 2, 9, 64, 64, 16, True),
    ([257, 31, 0, 100], 4, 4, 37, 128, 128, 32, True),
    ([150, 10], 6, 2, 70, 64, 64, 16, False),
    ([500], 4, 1, 130, 128, 64, 80, True),
    ([2100], 16, 16, 1, 64, 64, 128, True),
    ([640, 200], 2, 1, 129, 64, 128, 64, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", ATTN, ids=lambda c: "x".join(map(str, c)).replace(" ", ""))
def test_attention(case, dtype):
    lens, Hq, Hk, N, dk, dv, page, causal = case
    q, pool, table, fk, fv = problem(lens, Hq, Hk, N, dk, dv, page, dtype, seed=sum(lens) + N)
    scale = 1 / math.sqrt(dk)
    ref = reference(q, table, fk, fv, lens, scale, causal)
    t = [dev(q, dtype), dev(pool), dev(table), dev(np.array(lens, dtype=np.int32))]
    o, lse = pkg.kv4_attn_lse(*t, max_len=max(1, max(lens)), causal=causal)
    assert pkg.get_device_status() == _lib.MOA_OK
    check(o, lse, ref, dk, dtype)
    assert torch.equal(o, pkg.kv4_attn(*t, max_len=max(1, max(lens)), causal=causal))    # the same bits
    # a loose bound of the lengths divides the work otherwise; the answer is the same within bounds
    o, lse = pkg.kv4_attn_lse(*t, causal=causal)
    check(o, lse, ref, dk, dtype, "loose")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", [1, 40])
@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_attention_scales_and_peaks(scale, N, dtype):
    """Weights from uniform to one-hot, and a negative scale."""
    lens, Hq, Hk, dk, dv, page = [450, 60], 4, 2, 64, 64, 32
    q, pool, table, fk, fv = problem(lens, Hq, Hk, N, dk, dv, page, dtype, seed=8, q_scale=0.5)
    ref = reference(q, table, fk, fv, lens, scale, True)
    o, lse = pkg.kv4_attn_lse(dev(q, dtype), dev(pool), dev(table), dev(np.array(lens, dtype=np.int32)), scale=scale)
    check(o, lse, ref, dk, dtype, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("N", [1, 65])
def test_attention_long_context_and_large_pool(N):
    """Many ranges joined, and blocks past 2^31 bytes into the pool: the pages of the one sequence
    are spread over a pool of more than 4 GB."""
    dk = dv = 128
    page, Hk, G, n = 64, 1, 4, 9000
    n_pages = (5 << 30) // (4 * 9 * 256)
    r = np.random.default_rng(2)
    pool = torch.full((n_pages, Hk, page // 16, 9 * (dk + dv)), 255, dtype=torch.uint8, device="cuda:0")  # NaN scales
    table = np.sort(r.choice(n_pages, size=-(-n // page), replace=False)).astype(np.int32)[::-1].copy()[None]
    k = cast(r.normal(size=(1, Hk, n, dk)), "bf16")
    v = cast(r.normal(size=(1, Hk, n, dv)), "bf16")
    pos = np.arange(n, dtype=np.int32)[None]
    pkg.kv4_write(dev(k, "bf16"), dev(v, "bf16"), pool, dev(table), dev(pos))
    q = cast(r.normal(size=(1, Hk * G, N, dk)), "bf16")
    (kc, ks), (vc, vs) = R.quantise(k), R.quantise(v)
    got_k, _ = pkg.kv4_read(pool, dev(table), dev(pos), dk)
    assert np.array_equal(host(got_k), cast(R.values(kc, ks), "bf16"))
    ref = [x[None] for x in R.attention(q[0], R.values(kc, ks)[0], R.values(vc, vs)[0], n, dk ** -0.5, True)]
    o, lse = pkg.kv4_attn_lse(dev(q, "bf16"), pool, dev(table), dev(np.array([n], dtype=np.int32)), max_len=table.shape[1] * page)
    assert pkg.get_device_status() == _lib.MOA_OK
    check(o, lse, ref, dk, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_strided_queries_outputs_and_another_stream(dtype):
    lens, Hq, Hk, N, dk, dv, page = [100, 33], 6, 2, 5, 128, 64, 16
    q, pool, table, fk, fv = problem(lens, Hq, Hk, N, dk, dv, page, dtype, seed=6)
    t = [dev(pool), dev(table), dev(np.array(lens, dtype=np.int32))]
    want = pkg.kv4_attn(dev(q, dtype), *t)
    tokens = dev(q, dtype).transpose(1, 2).contiguous().transpose(1, 2)       # token-major storage
    out = torch.zeros(2, N, Hq + 1, dv, dtype=want.dtype, device="cuda:0")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    pkg.kv4_attn(tokens, *t, out=out[:, :, :Hq].transpose(1, 2), stream=s)
    s.synchronize()
    assert torch.equal(out[:, :, :Hq].transpose(1, 2), want) and bool((out[:, :, Hq] == 0).all())
    one = dev(q, dtype)[:, :1].expand(2, Hq, N, dk)                           # one head broadcast
    assert torch.equal(pkg.kv4_attn(one, *t), pkg.kv4_attn(one.contiguous(), *t))


@pytest.mark.gpu
@pytest.mark.parametrize("N", [1, 40])
def test_attention_lengths_and_pages_outside_their_tables(N):
    lens, Hq, Hk, dk, dv, page = [100, 64], 4, 2, 64, 64, 16
    q, pool, table, fk, fv = problem(lens, Hq, Hk, N, dk, dv, page, "bf16", seed=6)
    t = [dev(q, "bf16"), dev(pool)]
    good = pkg.kv4_attn(*t, dev(table), dev(np.array(lens, dtype=np.int32)))
    assert pkg.get_device_status() == _lib.MOA_OK
    o = pkg.kv4_attn(*t, dev(table), dev(np.array([100, -7], dtype=np.int32)))
    assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
    assert torch.equal(o[0], good[0]) and bool((o[1] == 0).all())
    o = pkg.kv4_attn(*t, dev(table), dev(np.array([100, 90], dtype=np.int32)), max_len=64)   # 90, 100 > max_len
    assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
    check(o[1:], None, [x[1:] for x in reference(q, table, fk, fv, lens, dk ** -0.5, True)], dk, "bf16")
    # tokens of a page that is not there are hidden, whether its number is too large or negative
    for wrong in (len(pool), -1):
        tb = table.copy()
        tb[0, 2] = wrong
        o = pkg.kv4_attn(*t, dev(tb), dev(np.array(lens, dtype=np.int32)), causal=False)
        assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
        rest = np.delete(table, 2, axis=1)
        ref = reference(q, rest, fk, fv, [84, 48], dk ** -0.5, False)
        check(o[:1], None, [x[:1] for x in ref], dk, "bf16")
    assert pkg.get_device_status() == _lib.MOA_OK


@pytest.mark.gpu
def test_tokens_past_the_end_have_no_influence():
    """The same lengths over pools that differ only in what nobody may see: the same bits."""
    lens, Hq, Hk, dk, dv, page = [37, 5, 90], 8, 4, 128, 128, 32
    for N in (1, 6, 50):
        outs = []
        q = problem(lens, Hq, Hk, N, dk, dv, page, "bf16", seed=3)[0]
        for garbage in (False, True):
            _, pool, table, _, _ = problem(lens, Hq, Hk, N, dk, dv, page, "bf16", seed=3, garbage=garbage)
            outs.append(pkg.kv4_attn(dev(q, "bf16"), dev(pool), dev(table), dev(np.array(lens, dtype=np.int32))))
        assert torch.equal(*outs)


@pytest.mark.gpu
@pytest.mark.parametrize("N", [1, 48])
def test_a_visible_nan_reaches_its_queries_only(N):
    lens, Hq, Hk, dk, dv, page = [80, 80], 4, 2, 64, 64, 16
    q, pool, table, fk, fv = problem(lens, Hq, Hk, N, dk, dv, page, "bf16", seed=13)
    good = pkg.kv4_attn(dev(q, "bf16"), dev(pool), dev(table), dev(np.array(lens, dtype=np.int32)))
    at = R.scale_place(dk, dv, 79 % 16, 0, False)
    pool = pool.copy()
    pool[table[0, 79 // page], 1, 79 % page // 16, at:at + 2] = 255            # the last key of one head: NaN
    o = pkg.kv4_attn(dev(q, "bf16"), dev(pool), dev(table), dev(np.array(lens, dtype=np.int32)))
    assert bool(torch.isnan(o[0, 2:, N - 1]).all())
    o[0, 2:, N - 1] = good[0, 2:, N - 1]
    assert torch.equal(o, good)


# -- refusals (host only: fake, never dereferenced addresses) -------------------------------------
P = [0x10000000000 * (i + 1) for i in range(8)]


@pytest.fixture(scope="module")
def L():
    from paper_2606_07713_gb300 import build
    build.build()
    return _lib.lib()


def contiguous(H, N, d):
    return (H * N * d, N * d, d)


def move(name="moa_kv4_write", ptrs=None, B=2, H=4, N=8, dk=128, dv=64, n_pages=10, page=32, max_pages=5,
         strides=None, dtype=1):
    p = list(P[:5]) if ptrs is None else ptrs
    return getattr(_lib, name)(*p, B, H, N, dk, dv, n_pages, page, max_pages,
                               strides or contiguous(H, N, dk) + contiguous(H, N, dv), dtype, None)


def attn(ptrs=None, lse=None, B=2, Hq=8, Hk=4, N=1, dk=128, dv=64, n_pages=10, page=32, max_pages=5, max_len=160,
         strides=None, scale=0.1, dtype=1):
    p = list(P[:5]) if ptrs is None else ptrs
    return _lib.moa_kv4_attn(*p, lse, B, Hq, Hk, N, dk, dv, n_pages, page, max_pages, max_len,
                             strides or contiguous(Hq, N, dk) + contiguous(Hq, N, dv), scale, 1, dtype, None, 0, None)


def put(i, v):
    p = list(P[:5])
    p[i] = v
    return p


MOVES = [
    *[(dict(ptrs=put(i, None)), _lib.MOA_ERR_INVALID_ARG) for i in range(5)],
    *[(dict(ptrs=put(i, P[i] + 2)), _lib.MOA_ERR_MISALIGNED) for i in range(5)],
    (dict(dtype=2), _lib.MOA_ERR_UNSUPPORTED_DTYPE),
    (dict(B=0), _lib.MOA_ERR_INVALID_ARG),
    (dict(N=0), _lib.MOA_ERR_INVALID_ARG),
    (dict(max_pages=0), _lib.MOA_ERR_INVALID_ARG),
    (dict(dk=96), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(dv=256), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(page=24), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(page=1 << 21), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(n_pages=2 ** 40), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(B=2 ** 40, N=2 ** 20), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(ptrs=put(2, P[0] + 16)), _lib.MOA_ERR_INVALID_ARG),          # the pool over the keys
    (dict(ptrs=put(2, P[3])), _lib.MOA_ERR_INVALID_ARG),               # the pool over the table
    (dict(strides=(4096, 1024, 124) + contiguous(4, 8, 64)), _lib.MOA_ERR_MISALIGNED),
]


@pytest.mark.parametrize("name", ["moa_kv4_write", "moa_kv4_read"])
@pytest.mark.parametrize("kwargs,code", MOVES)
def test_cache_refusals(L, name, kwargs, code):
    assert move(name, **kwargs) == code
    assert _lib.moa_last_error() != ""


def test_read_refuses_overlapping_outputs(L):
    assert move("moa_kv4_read", ptrs=put(1, P[0] + 64)) == _lib.MOA_ERR_INVALID_ARG      # V inside K
    assert move("moa_kv4_read", ptrs=put(4, P[0])) == _lib.MOA_ERR_INVALID_ARG           # pos under K
    st = (4096, 1024, 0) + contiguous(4, 8, 64)
    assert move("moa_kv4_read", strides=st) == _lib.MOA_ERR_INVALID_ARG                  # K's rows on one another


@pytest.mark.parametrize("kwargs,code", [
    *[(dict(ptrs=put(i, None)), _lib.MOA_ERR_INVALID_ARG) for i in range(5)],
    *[(dict(ptrs=put(i, P[i] + 2)), _lib.MOA_ERR_MISALIGNED) for i in range(5)],
    (dict(lse=P[5] + 2), _lib.MOA_ERR_MISALIGNED),
    (dict(lse=P[4]), _lib.MOA_ERR_INVALID_ARG),
    (dict(ptrs=put(4, P[0])), _lib.MOA_ERR_INVALID_ARG),               # O over Q
    (dict(ptrs=put(4, P[1] + 64)), _lib.MOA_ERR_INVALID_ARG),          # O inside the pool
    (dict(dtype=-1), _lib.MOA_ERR_UNSUPPORTED_DTYPE),
    (dict(Hq=6), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(Hk=0), _lib.MOA_ERR_INVALID_ARG),
    (dict(N=0), _lib.MOA_ERR_INVALID_ARG),
    (dict(max_len=0), _lib.MOA_ERR_INVALID_ARG),
    (dict(max_len=161), _lib.MOA_ERR_INVALID_ARG),
    (dict(max_pages=2 ** 30, max_len=2 ** 31 - 20), _lib.MOA_ERR_INVALID_ARG),
    (dict(scale=float("inf")), _lib.MOA_ERR_INVALID_ARG),
    (dict(dk=32), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(N=2 ** 31), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(strides=contiguous(8, 1, 128) + (0, 64, 64)), _lib.MOA_ERR_INVALID_ARG),   # two sequences in one place
])
def test_attention_refusals(L, kwargs, code):
    assert attn(**kwargs) == code
    assert _lib.moa_last_error() != ""


def test_pool_bytes(L):
    f = pkg.moa_kv4_pool_bytes
    assert f(3, 4, 48, 128, 64) == 3 * 4 * 3 * 9 * 192
    assert f(3, 4, 40, 128, 64) == f(0, 4, 48, 128, 64) == f(3, 4, 48, 96, 64) == 0
    assert f(2 ** 40, 2 ** 20, 48, 128, 64) == 0


def test_reference_packs_and_unpacks():
    r = np.random.default_rng(0)
    k, v = r.normal(size=(3, 16, 128)), r.normal(size=(3, 16, 64))
    q = R.quantise(k) + R.quantise(v)
    for a, b in zip(R.unpack(R.pack(*q), 128, 64), q):
        assert np.array_equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", [1, 5])
def test_attention_of_very_large_and_small_queries(N, dtype):
    """Rows of queries from 2^-100 to 2^100 against keys of the inverse size: scores of ordinary size."""
    Hq, Hk, dk, dv, page, n = 8, 4, 64, 64, 16, 200
    r = np.random.default_rng(17)
    table, n_pages = table_of(r, [n], page)
    for power in (-100, -60, 0, 60, 96):
        k = cast(r.normal(size=(1, Hk, n, dk)) * 2.0 ** -power, dtype)
        v = cast(r.normal(size=(1, Hk, n, dv)), dtype)
        q = cast(r.normal(size=(1, Hq, N, dk)) * 2.0 ** power, dtype)
        pool = pkg.kv4_pool(n_pages, Hk, page, dk, dv)
        pkg.kv4_write(dev(k, dtype), dev(v, dtype), pool, dev(table), dev(np.arange(n, dtype=np.int32)[None]))
        ref = [x[None] for x in R.attention(q[0], R.values(*R.quantise(k))[0], R.values(*R.quantise(v))[0], n, dk ** -0.5, True)]
        o, lse = pkg.kv4_attn_lse(dev(q, dtype), pool, dev(table), dev(np.array([n], dtype=np.int32)))
        check(o, lse, ref, dk, dtype, power)
