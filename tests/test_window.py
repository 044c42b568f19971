"""Attention with a sliding window and sinks (moa_window_attn) and its gradients (moa_window_attn_bwd)
against plain implementations in 64 bits; the bounds are derived in window_reference.py."""
import math

import numpy as np
import pytest

import paper_2606_07713_gb300 as pkg
import window_reference as W
from ops_reference import bf16
from paper_2606_07713_gb300 import _lib

torch = pytest.importorskip("torch")

TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}


def cast(a, dtype):
    return bf16(a) if dtype == "bf16" else np.asarray(a, dtype=np.float32).astype(np.float64)


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0", TORCH[dtype])


def host(t):
    return t.detach().double().cpu().numpy()


def inputs(shape, dtype, seed):
    B, Hq, Hk, N, M, dk, dv = shape
    r = np.random.default_rng(seed)
    q = cast(1.5 * r.normal(size=(B, Hq, N, dk)), dtype)
    k = cast(r.normal(size=(B, Hk, M, dk)) * np.exp(0.3 * r.normal(size=(1, Hk, 1, dk))), dtype)
    v = cast(r.normal(size=(B, Hk, M, dv)), dtype)
    do = cast(0.1 * r.normal(size=(B, Hq, N, dv)), dtype)
    return q, k, v, do


def check_forward(q, k, v, window, sinks, dtype, o, lse, scale=None):
    dk, M = q.shape[3], k.shape[2]
    scale = 1.0 / math.sqrt(dk) if scale is None else scale
    for b in range(q.shape[0]):
        ro, rl, av, size = W.attention(q[b], k[b], v[b], M, window, sinks, scale)
        bound = W.out_bound(ro, av, size, dk, dtype)
        err = np.abs(o[b] - ro)
        assert np.all(err <= bound), f"o: {np.max(err / bound)} of the bound"
        if lse is None:
            continue
        assert np.array_equal(np.isfinite(lse[b]), np.isfinite(rl))
        with np.errstate(invalid="ignore"):
            diff = np.where(np.isfinite(rl), np.abs(lse[b] - rl), 0.0)
        assert np.all(diff <= W.lse_bound(rl, size, dk))


def check_gradients(q, k, v, o, lse, do, window, sinks, dtype, got, scale=None):
    scale = 1.0 / math.sqrt(q.shape[3]) if scale is None else scale
    for b in range(q.shape[0]):
        want, bound = W.gradients(q[b], k[b], v[b], o[b], lse[b], do[b], window, sinks, scale, dtype)
        for name, g, x, e in zip(("dq", "dk", "dv"), got, want, bound):
            err = np.abs(g[b] - x)
            assert np.all(err <= e), f"{name}: {np.max(err / e)} of the bound"


def run_both(shape, window, sinks, dtype, seed, scale=None):
    q, k, v, do = inputs(shape, dtype, seed)
    t = [dev(x, dtype) for x in (q, k, v, do)]
    o, lse = pkg.window_attn_lse(*t[:3], window=window or None, sinks=sinks, scale=scale)
    grads = pkg.window_attn_bwd(*t[:3], o, lse, t[3], window=window or None, sinks=sinks, scale=scale)
    assert pkg.get_device_status() == _lib.MOA_OK
    check_forward(q, k, v, window, sinks, dtype, host(o), host(lse), scale)
    check_gradients(q, k, v, host(o), host(lse), do, window, sinks, dtype, [host(g) for g in grads], scale)


SHAPES = [  # B, H_q, H_k, N_q, N_k, d_k, d_v, window, sinks
    (1, 1, 1, 1, 1, 64, 64, 0, 0),
    (2, 2, 1, 1, 300, 128, 128, 0, 0),           # one query over many keys
    (1, 4, 4, 127, 127, 64, 64, 0, 0),
    (1, 2, 2, 128, 128, 128, 128, 0, 0),
    (2, 4, 2, 129, 129, 128, 64, 0, 0),
    (1, 6, 2, 260, 260, 64, 128, 0, 0),          # three heads a key head: 126 of 128 rows
    (1, 5, 1, 300, 411, 128, 128, 50, 0),        # five heads, more keys than queries
    (2, 8, 2, 333, 333, 64, 64, 64, 4),
    (1, 4, 1, 700, 700, 128, 128, 128, 1),
    (1, 2, 1, 515, 515, 128, 64, 1, 0),          # a window of the token itself
    (1, 2, 1, 515, 515, 64, 128, 1, 3),
    (1, 1, 1, 640, 640, 64, 64, 100, 130),       # sinks past a tile
    (1, 3, 3, 400, 400, 128, 128, 37, 399),      # all but one token a sink
    (2, 2, 2, 300, 100, 64, 64, 0, 0),           # rows that see nothing
    (1, 4, 2, 300, 100, 128, 128, 30, 2),
    (1, 8, 1, 17, 1000, 128, 128, 200, 4),
    (1, 2, 2, 513, 513, 64, 64, 5000, 4),        # a window past every token
    (1, 130, 1, 9, 40, 64, 64, 11, 2),           # more heads of a key head than rows of a tile
    (1, 128, 1, 5, 300, 128, 64, 0, 0),
    (3, 7, 7, 65, 65, 64, 128, 3, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward_and_gradients(shape, dtype):
    run_both(shape[:7], shape[7], shape[8], dtype, sum(shape))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [-0.1, 0.0, 0.5])
def test_scales(scale, dtype):
    run_both((1, 4, 2, 200, 200, 64, 64), 70, 3, dtype, 5, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long(dtype):
    """Several shares of a row's tokens, sinks' rows in many pieces."""
    run_both((1, 2, 1, 1900, 2100, 64, 64), 0, 0, dtype, 1)
    run_both((1, 2, 1, 2100, 2100, 128, 128), 200, 4, dtype, 2)


@pytest.mark.gpu
def test_largest_scores():
    """Scores in the thousands of both signs: maxima that rise from tile to tile."""
    q, k, v, do = inputs((1, 2, 2, 400, 400, 64, 64), "bf16", 9)
    k = k * np.exp2(np.floor(np.arange(400) / 50))[None, None, :, None]
    t = [dev(x, "bf16") for x in (q, k, v)]
    o, lse = pkg.window_attn_lse(*t, window=150, sinks=2)
    assert pkg.get_device_status() == _lib.MOA_OK
    check_forward(q, k, v, 150, 2, "bf16", host(o), host(lse))


# -- layouts ------------------------------------------------------------------------------------
def token_major(a, dtype):
    """[B, H, N, d] as a view of a [B, N, H, d] tensor."""
    return dev(a.transpose(0, 2, 1, 3), dtype).transpose(1, 2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["token major", "slices", "reversed", "broadcast batch", "broadcast heads", "broadcast rows"])
def test_layouts(kind, dtype):
    B, Hq, Hk, N, d, window, sinks = 2, 6, 3, 150, 64, 40, 2
    q, k, v, do = inputs((B, Hq, Hk, N, N, d, d), dtype, 3)
    if kind.startswith("broadcast"):
        axis = {"broadcast batch": 0, "broadcast heads": 1, "broadcast rows": 2}[kind]
        q, k, v, do = (np.broadcast_to(np.take(x, [0], axis), x.shape) for x in (q, k, v, do))
        t = [dev(np.take(x, [0], axis), dtype).expand(*x.shape) for x in (q, k, v, do)]
    elif kind == "token major":
        t = [token_major(x, dtype) for x in (q, k, v, do)]
    elif kind == "slices":      # of one projection's output [B, N, H_q + 2 H_k, d]
        qkv = token_major(np.concatenate([q, k, v], 1), dtype)
        t = [qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:], token_major(do, dtype)]
    else:                       # negative strides along the batch: torch has none, the C interface has
        t = [dev(x, dtype) for x in (q, k, v, do)]
    code = _lib.MOA_BF16 if dtype == "bf16" else _lib.MOA_FP32
    if kind == "reversed":
        flipped = [x.flip(0).contiguous() for x in t]
        ptr = [x.data_ptr() + x.stride(0) * x.element_size() for x in flipped]
        st = [s for x in flipped for s in (-x.stride(0), x.stride(1), x.stride(2))]
        o, lse = torch.empty_like(t[0]), torch.empty(B, Hq, N, dtype=torch.float32, device="cuda")
        ws = torch.empty(max(16, pkg.moa_window_attn_workspace_bytes(B, Hq, Hk, N, N, d, d, window, sinks, code)),
                         dtype=torch.uint8, device="cuda")
        pkg.check(pkg.moa_window_attn(*ptr[:3], o.data_ptr(), lse.data_ptr(), B, Hq, Hk, N, N, d, d, window, sinks,
                                      st[:9] + list(o.stride()[:3]), d ** -0.5, code, ws.data_ptr(), ws.numel(),
                                      torch.cuda.current_stream().cuda_stream))
        grads = [torch.empty_like(x) for x in t[:3]]
        ws = torch.empty(pkg.moa_window_attn_bwd_workspace_bytes(B, Hq, Hk, N, N, d, d, window, sinks, code),
                         dtype=torch.uint8, device="cuda")
        strides = st[:9] + list(o.stride()[:3]) + st[9:] + [s for g in grads for s in g.stride()[:3]]
        pkg.check(pkg.moa_window_attn_bwd(*ptr[:3], o.data_ptr(), ptr[3], lse.data_ptr(), *[g.data_ptr() for g in grads], B,
                                          Hq, Hk, N, N, d, d, window, sinks, strides, d ** -0.5, code, ws.data_ptr(),
                                          ws.numel(), torch.cuda.current_stream().cuda_stream))
    else:
        o, lse = pkg.window_attn_lse(*t[:3], window=window, sinks=sinks)
        grads = pkg.window_attn_bwd(*t[:3], o, lse, t[3], window=window, sinks=sinks)
    assert pkg.get_device_status() == _lib.MOA_OK
    check_forward(q, k, v, window, sinks, dtype, host(o), host(lse))
    check_gradients(q, k, v, host(o), host(lse), do, window, sinks, dtype, [host(g) for g in grads])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_outputs_given(dtype):
    """Outputs as views of larger buffers: what lies between their rows stays."""
    B, Hq, Hk, N, d = 2, 4, 2, 90, 64
    q, k, v, do = inputs((B, Hq, Hk, N, N, d, d), dtype, 8)
    t = [dev(x, dtype) for x in (q, k, v, do)]
    big = torch.full((B, N + 5, Hq + 1, d), 7.0, dtype=TORCH[dtype], device="cuda")
    out = big[:, :N, :Hq].transpose(1, 2)
    lse = torch.empty(B, Hq, N, dtype=torch.float32, device="cuda")
    o, l = pkg.window_attn_lse(*t[:3], window=33, sinks=1, out=out, lse=lse)
    assert o.data_ptr() == big.data_ptr() and l is lse
    grad = torch.full((B, N, Hq + 2 * Hk + 1, d), 9.0, dtype=TORCH[dtype], device="cuda").transpose(1, 2)
    parts = grad[:, :Hq], grad[:, Hq:Hq + Hk], grad[:, Hq + Hk:Hq + 2 * Hk]
    pkg.window_attn_bwd(*t[:3], o, l, t[3], window=33, sinks=1, out=parts)
    assert pkg.get_device_status() == _lib.MOA_OK
    assert bool((big[:, N:] == 7).all()) and bool((big[:, :, Hq] == 7).all()) and bool((grad[:, -1] == 9).all())
    check_forward(q, k, v, 33, 1, dtype, host(o), host(l))
    check_gradients(q, k, v, host(o), host(l), do, 33, 1, dtype, [host(g) for g in parts])
    assert torch.equal(pkg.window_attn(*t[:3], window=33, sinks=1), o)


# -- numbers that are none ------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_hidden_tokens_that_are_not_numbers(bad, dtype):
    """Keys and values of tokens that a row does not see have no influence on it; rows that see one
    of its values get what the formula gives in that feature, and their own elsewhere."""
    N, d, window, sinks, at = 300, 64, 40, 2, 137
    q, k, v, _ = inputs((1, 4, 2, N, N, d, d), dtype, 4)
    bad_k, bad_v = k.copy(), v.copy()
    bad_k[:, 0, at] = bad
    bad_v[:, :, at, 5] = bad
    o, lse = pkg.window_attn_lse(dev(q, dtype), dev(bad_k, dtype), dev(bad_v, dtype), window=window, sinks=sinks)
    assert pkg.get_device_status() == _lib.MOA_OK
    o, lse = host(o), host(lse)
    ro, rl, av, size = W.attention(q[0], k[0], v[0], N, window, sinks, d ** -0.5)
    bound = W.out_bound(ro, av, size, d, dtype)
    hit = np.zeros(N, dtype=bool)
    hit[at:at + window] = True
    assert np.all(np.abs(o[0] - ro)[:, ~hit] <= bound[:, ~hit])
    assert np.all(np.abs(lse[0] - rl)[:, ~hit] <= W.lse_bound(rl, size, d)[:, ~hit])
    # the second key head's rows: only feature 5 is touched
    other = np.arange(d) != 5
    assert np.all(np.abs(o[0] - ro)[2:][..., other] <= bound[2:][..., other])
    assert not np.any(np.isfinite(o[0, 2:, hit, 5]))
    if math.isinf(bad):
        assert np.all(o[0, 2:, hit, 5] == bad)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_query_that_is_not_a_number(dtype):
    N, d = 300, 64
    q, k, v, _ = inputs((1, 2, 1, N, N, d, d), dtype, 6)
    bad = q.copy()
    bad[0, 1, 7, 3] = np.nan
    o = host(pkg.window_attn(dev(bad, dtype), dev(k, dtype), dev(v, dtype), window=64))
    good = host(pkg.window_attn(dev(q, dtype), dev(k, dtype), dev(v, dtype), window=64))
    assert np.all(np.isnan(o[0, 1, 7]))
    o[0, 1, 7] = good[0, 1, 7] = 0
    assert np.array_equal(o, good)


@pytest.mark.gpu
def test_batch_padded_at_the_end():
    """Padding past a sequence's end, with zero gradients there, changes nothing before it."""
    B, Hq, Hk, N, L, d = 2, 4, 2, 320, 201, 128
    q, k, v, do = inputs((B, Hq, Hk, N, N, d, d), "bf16", 12)
    do[1, :, L:] = 0
    t = [dev(x, "bf16") for x in (q, k, v, do)]
    o, lse = pkg.window_attn_lse(*t[:3], window=77, sinks=3)
    grads = [host(g)[1, :, :L] for g in pkg.window_attn_bwd(*t[:3], o, lse, t[3], window=77, sinks=3)]
    cut = [x[1:, :, :L] for x in (q, k, v, do)]
    check_forward(*cut[:3], 77, 3, "bf16", host(o)[1:, :, :L], host(lse)[1:, :, :L])
    check_gradients(*cut[:3], host(o)[1:, :, :L], host(lse)[1:, :, :L], cut[3], 77, 3, "bf16", [g[None] for g in grads])


# -- gradients against differences ------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks,Nq,Nk", [(0, 0, 40, 40), (9, 2, 60, 60), (5, 0, 30, 70)])
def test_gradients_against_differences(window, sinks, Nq, Nk):
    """The fp32 gradients' product with a random direction against central differences, in 64 bits, of
    the loss sum(do * o).  With step h the differences are off by h^2 / 6 times the third derivative along
    the direction: of the order of the loss times (|direction| scale |q|)^3, here below 2^10; h = 2^-14 makes
    that 2^-20, and 64-bit cancellation adds 2^-50 / h.  The kernel's own error is that of its bounds: relative
    2^-15 of sums of magnitudes.  2^-10 of the sum of |gradient x direction| holds both."""
    Hq, Hk, d = 4, 2, 64
    q, k, v, do = inputs((1, Hq, Hk, Nq, Nk, d, d), "fp32", 21)
    t = [dev(x, "fp32") for x in (q, k, v, do)]
    o, lse = pkg.window_attn_lse(*t[:3], window=window or None, sinks=sinks)
    grads = [host(g) for g in pkg.window_attn_bwd(*t[:3], o, lse, t[3], window=window or None, sinks=sinks)]
    r = np.random.default_rng(2)
    loss = lambda a: float((W.attention(a[0][0], a[1][0], a[2][0], Nk, window, sinks, d ** -0.5)[0] * do[0]).sum())  # noqa: E731
    h = 2.0 ** -14
    for n in range(3):
        z = r.normal(size=grads[n].shape)
        up, down = [q, k, v], [q, k, v]
        up[n], down[n] = up[n] + h * z, down[n] - h * z
        diff = (loss(up) - loss(down)) / (2 * h)
        assert abs(diff - float((grads[n] * z).sum())) <= 2.0 ** -10 * float(np.abs(grads[n] * z).sum())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_same_bits_every_time(dtype):
    q, k, v, do = inputs((2, 8, 2, 777, 777, 128, 128), dtype, 31)
    t = [dev(x, dtype) for x in (q, k, v, do)]
    runs = []
    for _ in range(3):
        o, lse = pkg.window_attn_lse(*t[:3], window=100, sinks=5)
        runs.append([o, lse, *pkg.window_attn_bwd(*t[:3], o, lse, t[3], window=100, sinks=5)])
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


# -- refusals, without a GPU ------------------------------------------------------------------------
A = [0x10000000 * (i + 1) for i in range(12)]     # never dereferenced
FWD = dict(Q=A[0], K=A[1], V=A[2], O=A[3], LSE=A[4], B=1, H_q=4, H_k=2, N_q=8, N_k=8, d_k=64, d_v=64, window=4, sinks=1,
           strides=[4 * 512, 512, 64, 2 * 512, 512, 64, 2 * 512, 512, 64, 4 * 512, 512, 64], scale=0.1, dtype=1,
           workspace=A[5], workspace_bytes=1 << 30, stream=None)
BWD = dict(Q=A[0], K=A[1], V=A[2], O=A[3], dO=A[6], LSE=A[4], dQ=A[7], dK=A[8], dV=A[9], B=1, H_q=4, H_k=2, N_q=8, N_k=8,
           d_k=64, d_v=64, window=4, sinks=1,
           strides=[4 * 512, 512, 64, 2 * 512, 512, 64, 2 * 512, 512, 64, 4 * 512, 512, 64, 4 * 512, 512, 64, 4 * 512, 512, 64,
                    2 * 512, 512, 64, 2 * 512, 512, 64], scale=0.1, dtype=1, workspace=A[5], workspace_bytes=1 << 30,
           stream=None)
BAD = [
    (dict(B=0), _lib.MOA_ERR_INVALID_ARG), (dict(N_q=0), _lib.MOA_ERR_INVALID_ARG), (dict(N_k=0), _lib.MOA_ERR_INVALID_ARG),
    (dict(H_k=0), _lib.MOA_ERR_INVALID_ARG), (dict(H_k=3), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(d_k=96), _lib.MOA_ERR_UNSUPPORTED_SHAPE), (dict(d_v=32), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(window=-1), _lib.MOA_ERR_INVALID_ARG), (dict(sinks=-1), _lib.MOA_ERR_INVALID_ARG),
    (dict(scale=float("nan")), _lib.MOA_ERR_INVALID_ARG), (dict(scale=float("inf")), _lib.MOA_ERR_INVALID_ARG),
    (dict(dtype=5), _lib.MOA_ERR_UNSUPPORTED_DTYPE), (dict(Q=None), _lib.MOA_ERR_INVALID_ARG),
    (dict(K=A[1] + 8), _lib.MOA_ERR_MISALIGNED), (dict(LSE=A[4] + 2), _lib.MOA_ERR_MISALIGNED),
    (dict(N_q=2 ** 31), _lib.MOA_ERR_UNSUPPORTED_SHAPE), (dict(N_k=2 ** 31), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(B=2 ** 40, N_q=2 ** 20), _lib.MOA_ERR_UNSUPPORTED_SHAPE), (dict(strides=None), _lib.MOA_ERR_INVALID_ARG),
]


def forward(**changes):
    a = dict(FWD, **changes)
    if a["strides"] is None:
        return _lib.lib().moa_window_attn(*[a[n] for n in FWD if n not in ("strides", "scale", "dtype", "workspace",
                                                                           "workspace_bytes", "stream")],
                                          None, a["scale"], a["dtype"], None, 0, None)
    return pkg.moa_window_attn(**a)


def backward(**changes):
    a = dict(BWD, **changes)
    if a["strides"] is None:
        return _lib.lib().moa_window_attn_bwd(*[a[n] for n in BWD if n not in ("strides", "scale", "dtype", "workspace",
                                                                               "workspace_bytes", "stream")],
                                              None, a["scale"], a["dtype"], None, 0, None)
    return pkg.moa_window_attn_bwd(**a)


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("changes,status", BAD, ids=lambda x: str(x)[:40])
def test_refusals(call, changes, status):
    assert call(**changes) == status
    assert pkg.moa_last_error()


def test_refusals_of_outputs_on_inputs():
    for changes in (dict(O=A[0]), dict(O=A[2] + 16), dict(LSE=A[1]), dict(O=A[4])):
        assert forward(**changes) == _lib.MOA_ERR_INVALID_ARG, changes
    for changes in (dict(dQ=A[0]), dict(dK=A[1]), dict(dV=A[8]), dict(workspace=A[3]), dict(workspace=A[7]), dict(dQ=A[4]),
                    dict(workspace=None), dict(workspace_bytes=8)):
        assert backward(**changes) == _lib.MOA_ERR_INVALID_ARG, changes
    rows = list(FWD["strides"])
    rows[11] = 32                                        # an output's rows on one another
    assert forward(strides=rows) == _lib.MOA_ERR_INVALID_ARG
    rows = list(FWD["strides"])
    rows[5] = 60                                         # not a multiple of 16 bytes
    assert forward(strides=rows) == _lib.MOA_ERR_MISALIGNED


def test_workspace_sizes_of_invalid_calls():
    f = pkg.moa_window_attn_bwd_workspace_bytes
    assert f(1, 4, 2, 8, 8, 64, 64, 0, 0, 1) > 0
    for bad in ((0, 4, 2, 8, 8, 64, 64, 0, 0, 1), (1, 4, 3, 8, 8, 64, 64, 0, 0, 1), (1, 4, 2, 8, 8, 96, 64, 0, 0, 1),
                (1, 4, 2, 8, 8, 64, 64, -1, 0, 1), (1, 4, 2, 8, 8, 64, 64, 0, 0, 9), (1, 4, 2, 8, 2 ** 31, 64, 64, 0, 0, 1)):
        assert f(*bad) == 0
        assert pkg.moa_window_attn_workspace_bytes(*bad) == 0


def test_binding_refusals():
    x = torch.zeros(1, 2, 8, 64)
    for call in (lambda: pkg.window_attn(x, x, x), lambda: pkg.window_attn_bwd(x, x, x, x, x, x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(TypeError):
        pkg.window_attn(1, x, x)


@pytest.mark.gpu
def test_binding_refusals_on_the_device():
    x = torch.zeros(1, 2, 8, 64, device="cuda")
    with pytest.raises(ValueError, match="window"):
        pkg.window_attn(x, x, x, window=0)
    with pytest.raises(pkg.MoaError):
        pkg.window_attn(x, x, x, window=3, sinks=-1)
    with pytest.raises(TypeError):
        pkg.window_attn(x, x.bfloat16(), x)
    with pytest.raises(ValueError):
        pkg.window_attn(x, x[:, :, :5], x)
    with pytest.raises(TypeError):
        pkg.window_attn(x.half(), x.half(), x.half())
    o, lse = pkg.window_attn_lse(x, x, x)
    with pytest.raises(ValueError):
        pkg.window_attn_bwd(x, x, x, o, lse[..., :4], x)
    with pytest.raises(ValueError):
        pkg.window_attn_bwd(x, x, x, o, lse, x, out=(x, x))
    with pytest.raises(ValueError):
        pkg.window_attn(x.transpose(2, 3), x, x)


@pytest.mark.parametrize("call", [forward, backward], ids=["forward", "backward"])
@pytest.mark.parametrize("changes,status", [
    (dict(N_q=2 ** 29 - 256), _lib.MOA_ERR_UNSUPPORTED_SHAPE), (dict(N_k=2 ** 30 - 512), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(scale=2.5e38), _lib.MOA_ERR_INVALID_ARG), (dict(scale=-3.4e38), _lib.MOA_ERR_INVALID_ARG),
], ids=lambda x: str(x)[:40])
def test_refusals_at_the_ends_of_ranges(call, changes, status):
    """Rows and tokens one step past 2^31 - 1025 (4 and 2 heads), and scales that overflow times log2 e."""
    assert call(**changes) == status
    assert pkg.moa_last_error()
