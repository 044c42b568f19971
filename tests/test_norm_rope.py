"""moa_qk_norm_rope and its gradients against a plain implementation in 64 bits.

Bounds, with A the largest |w x r| of the row: the kernel works in fp32 with row sums of at most
eight terms a lane and five tree steps, so r is within 16 * 2^-24 relative, and a rotated value
within 2e-6 A of the formula on the same inputs; a bf16 output (8 significant bits) adds half a unit, 2^-8 |y|.
Backward, with S = r (max |w t| + max |x r| mean |w t x r|): dx within 6e-6 S, plus 2^-8 |dx| in
bf16; dw is a sum in fp32 of terms within 4e-6 relative along chains of at most 200 additions
(200 * 2^-24 = 1.2e-5), so within 2e-5 of sum |t x r|.
"""
import numpy as np
import pytest

import ops_reference as R
import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib

torch = pytest.importorskip("torch")
EPS = 1e-6

# B, Hq, Hk, N, d, d_rot, interleaved
SHAPES = [
    (1, 1, 1, 1, 64, 64, False),
    (1, 1, 1, 1, 8 * 3, 16, True),
    (2, 3, 1, 5, 64, 32, True),
    (2, 4, 4, 33, 128, 128, False),
    (1, 8, 2, 257, 96, 96, False),
    (3, 5, 5, 19, 80, 48, True),
    (1, 2, 1, 70, 256, 128, False),
    (1, 2, 3, 31, 200, 16, False),
    (64, 16, 16, 1, 128, 128, True),
    (2, 20, 4, 600, 128, 64, False),
]


def make(B, Hq, Hk, N, d, d_rot, dtype, seed, P=None):
    r = np.random.default_rng(seed)
    P = P or N + 37
    cast = R.bf16 if dtype == "bf16" else lambda a: np.asarray(a, dtype=np.float32).astype(np.float64)
    x = {"q": cast(r.normal(size=(B, Hq, N, d)) * np.exp(r.normal(size=(B, Hq, 1, 1)))),
         "k": cast(r.normal(size=(B, Hk, N, d)) * np.exp(r.normal(size=(B, Hk, 1, 1)))),
         "wq": cast(1 + 0.3 * r.normal(size=d)), "wk": cast(1 + 0.3 * r.normal(size=d)),
         "gq": cast(r.normal(size=(B, Hq, N, d))), "gk": cast(r.normal(size=(B, Hk, N, d)))}
    a = r.uniform(-np.pi, np.pi, size=(P, d_rot // 2))
    x["cos"], x["sin"] = (f(a).astype(np.float32).astype(np.float64) for f in (np.cos, np.sin))
    x["pos"] = r.integers(0, P, size=(B, N)).astype(np.int32)
    return x


def dev(a, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
    return t if a.dtype == np.int32 else t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def on_device(x, dtype):
    return {n: dev(a, "fp32" if n in ("cos", "sin") else dtype) for n, a in x.items()}


def host(t):
    return t.detach().double().cpu().numpy()


def check_fwd(y, x, w, c, s, pos, inter, dtype, what):
    ref = R.norm_rope(x, w, c, s, pos, EPS, inter)
    r = 1 / np.sqrt(np.mean(x * x, -1, keepdims=True) + EPS)
    bound = 2e-6 * np.max(np.abs(x * r * w), -1, keepdims=True) + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0)
    err = np.abs(host(y) - ref)
    assert np.all(err <= bound), (what, float(np.max(err / bound)))


def check_bwd(dx, dw, x, w, c, s, pos, g, inter, dtype, what):
    ref, dw_ref, dw_abs = R.norm_rope_bwd(x, w, c, s, pos, g, EPS, inter)
    live = (pos >= 0)[:, None, :, None]
    r = 1 / np.sqrt(np.mean(x * x, -1, keepdims=True) + EPS)
    t = np.where(live, np.abs(g) + np.max(np.abs(g), -1, keepdims=True), 0)   # |t| <= |a| + |b|
    n = np.abs(x * r)
    S = r * (np.max(np.abs(w) * t, -1, keepdims=True) + n.max(-1, keepdims=True) * np.mean(np.abs(w) * t * n, -1, keepdims=True))
    bound = 6e-6 * S + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0)
    err = np.abs(host(dx) - ref)
    assert np.all(err <= bound), (what, float(np.max(err / np.maximum(bound, 1e-300))))
    err = np.abs(host(dw) - dw_ref)
    assert np.all(err <= 2e-5 * dw_abs + 1e-30), (what, float(np.max(err / np.maximum(dw_abs, 1e-30))))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward_and_gradients(shape, dtype):
    *dims, inter = shape
    x = make(*dims, dtype, seed=sum(dims))
    t = on_device(x, dtype)
    q, k = pkg.qk_norm_rope(t["q"], t["k"], t["wq"], t["wk"], t["cos"], t["sin"], t["pos"], EPS, inter)
    dq, dk, dwq, dwk = pkg.qk_norm_rope_bwd(t["q"], t["k"], t["wq"], t["wk"], t["cos"], t["sin"], t["pos"],
                                            t["gq"], t["gk"], EPS, inter)
    assert pkg.get_device_status() == _lib.MOA_OK
    c, s, pos = x["cos"], x["sin"], x["pos"]
    for y, dy, dw, n in ((q, dq, dwq, "q"), (k, dk, dwk, "k")):
        check_fwd(y, x[n], x["w" + n], c, s, pos, inter, dtype, n)
        check_bwd(dy, dw, x[n], x["w" + n], c, s, pos, x["g" + n], inter, dtype, n)
    # the same bits again
    again = pkg.qk_norm_rope_bwd(t["q"], t["k"], t["wq"], t["wk"], t["cos"], t["sin"], t["pos"], t["gq"], t["gk"],
                                 EPS, inter)
    assert all(torch.equal(a, b) for a, b in zip(again, (dq, dk, dwq, dwk)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dims", [(1, 4, 4, 7501, 64, 64), (2, 5, 3, 2570, 64, 32), (1, 7, 2, 5003, 128, 128)],
                         ids=lambda s: "x".join(map(str, s)))
def test_gradients_of_more_tokens_than_one_round(dims, dtype):
    """More groups of tokens than CTAs: whole rounds, and a last one whose few groups' heads are shared
    by several CTAs (evenly, unevenly, or by more than there are heads).  The bounds are those above:
    a lane's chain of additions is its rounds' heads, far below 200."""
    x = make(*dims, dtype, seed=sum(dims))
    x["pos"][:, ::97] = -1
    t = on_device(x, dtype)
    dq, dk, dwq, dwk = pkg.qk_norm_rope_bwd(t["q"], t["k"], t["wq"], t["wk"], t["cos"], t["sin"], t["pos"],
                                            t["gq"], t["gk"], EPS, False)
    assert pkg.get_device_status() == _lib.MOA_OK
    for dy, dw, n in ((dq, dwq, "q"), (dk, dwk, "k")):
        check_bwd(dy, dw, x[n], x["w" + n], x["cos"], x["sin"], x["pos"], x["g" + n], False, dtype, n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_slices_of_one_buffer_in_place_and_transposed(dtype):
    """Token-major projections [B, N, (Hq + Hk + Hv) d]: q and k as strided views, written in place;
    the values between the tokens' heads stay untouched.  Outputs may be token-major too, and
    inputs broadcast."""
    B, Hq, Hk, N, d, rot = 2, 6, 2, 45, 64, 64
    x = make(B, Hq, Hk, N, d, rot, dtype, 5)
    t = on_device(x, dtype)
    want = pkg.qk_norm_rope(t["q"], t["k"], t["wq"], t["wk"], t["cos"], t["sin"], t["pos"])
    whole = torch.zeros(B, N, Hq + 2 * Hk, d, dtype=t["q"].dtype, device="cuda:0")
    q, k, v = (whole[:, :, a:b].transpose(1, 2) for a, b in ((0, Hq), (Hq, Hq + Hk), (Hq + Hk, Hq + 2 * Hk)))
    q.copy_(t["q"]), k.copy_(t["k"]), v.fill_(7.0)
    got = pkg.qk_norm_rope(q, k, t["wq"], t["wk"], t["cos"], t["sin"], t["pos"], out=(q, k))
    assert got[0].data_ptr() == q.data_ptr()
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and bool((v == 7.0).all())
    # one head's features and one token's row broadcast
    one = t["q"][:, :1, :1].expand(B, Hq, N, d)
    y, _ = pkg.qk_norm_rope(one, t["k"], t["wq"], t["wk"], t["cos"], t["sin"], t["pos"])
    z, _ = pkg.qk_norm_rope(one.contiguous(), t["k"], t["wq"], t["wk"], t["cos"], t["sin"], t["pos"])
    assert torch.equal(y, z)
    # gradients in place over the outputs' gradients
    ref = pkg.qk_norm_rope_bwd(t["q"], t["k"], t["wq"], t["wk"], t["cos"], t["sin"], t["pos"], t["gq"], t["gk"])
    gq, gk = t["gq"].clone(), t["gk"].clone()
    got = pkg.qk_norm_rope_bwd(t["q"], t["k"], t["wq"], t["wk"], t["cos"], t["sin"], t["pos"], gq, gk, out=(gq, gk))
    assert all(torch.equal(a, b) for a, b in zip(got, ref)) and got[0] is gq


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_padding_zero_rows_and_positions_outside_the_table(dtype):
    B, Hq, Hk, N, d, rot = 2, 3, 1, 40, 128, 64
    x = make(B, Hq, Hk, N, d, rot, dtype, 9)
    x["pos"][0, 30:] = -1
    x["pos"][1, 0] = -5
    x["q"][0, 0, 31] = np.nan          # what a padding row holds has no influence
    x["gq"][0, 1, 32] = np.inf
    x["q"][1, 2, 7] = 0.0              # a row of zeros: r = eps^(-1/2), finite
    t = on_device(x, dtype)
    args = [t[n] for n in ("q", "k", "wq", "wk", "cos", "sin", "pos")]
    q, k = pkg.qk_norm_rope(*args)
    dq, dk, dwq, dwk = pkg.qk_norm_rope_bwd(*args, t["gq"], t["gk"])
    assert pkg.get_device_status() == _lib.MOA_OK
    clean = {n: np.where(np.isfinite(a), a, 0.0) if a.dtype != np.int32 else a for n, a in x.items()}
    for y, dy, dw, n in ((q, dq, dwq, "q"), (k, dk, dwk, "k")):
        check_fwd(y, clean[n], clean["w" + n], x["cos"], x["sin"], x["pos"], False, dtype, n)
        check_bwd(dy, dw, clean[n], clean["w" + n], x["cos"], x["sin"], x["pos"], clean["g" + n], False, dtype, n)
    # a position past the table: its rows are NaN, the others unchanged, the status says so
    t["pos"][0, 3] = x["cos"].shape[0]
    q2, _ = pkg.qk_norm_rope(*args)
    assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
    assert pkg.get_device_status() == _lib.MOA_OK
    assert bool(torch.isnan(q2[0, :, 3]).all())
    q2[0, :, 3] = q[0, :, 3]
    assert torch.equal(q2, q)
    d2 = pkg.qk_norm_rope_bwd(*args, t["gq"], t["gk"])
    assert pkg.get_device_status() == _lib.MOA_ERR_DEVICE_INDEX
    assert bool(torch.isnan(d2[0][0, :, 3]).all()) and bool(torch.isfinite(d2[2]).all())


@pytest.mark.gpu
def test_gradient_against_differences_of_the_forward():
    """sum(g * y) along random directions of q, k and both weights: central differences of the fp32
    forward, step h = 2^-6 of inputs of size one.  The third derivatives of the normalised rows are
    of the order of the gradient, so the differences are within h^2 = 2.5e-4 of it relative to
    |gradient| |direction|; the forward's rounding adds 1e-7 |g| |y| / h = 1e-5 |g| |y|."""
    B, Hq, Hk, N, d, rot = 1, 2, 1, 6, 64, 32
    x = make(B, Hq, Hk, N, d, rot, "fp32", 21)
    r = np.random.default_rng(3)
    for n in ("q", "k"):
        x[n] = x[n] / np.sqrt(np.mean(x[n] ** 2, -1, keepdims=True))
    t = on_device(x, "fp32")
    names = ("q", "k", "wq", "wk")
    grads = pkg.qk_norm_rope_bwd(*[t[n] for n in names], t["cos"], t["sin"], t["pos"], t["gq"], t["gk"])

    def loss(moved):
        y = pkg.qk_norm_rope(*[moved[n] for n in names], t["cos"], t["sin"], t["pos"])
        return sum(float((host(a) * x[n]).sum()) for a, n in zip(y, ("gq", "gk")))

    y = pkg.qk_norm_rope(*[t[n] for n in names], t["cos"], t["sin"], t["pos"])
    noise = 1e-5 * sum(np.linalg.norm(host(a)) * np.linalg.norm(x[n]) for a, n in zip(y, ("gq", "gk")))
    h = 2.0 ** -6
    for name, grad in zip(names, grads):
        v = r.normal(size=x[name].shape)
        v /= np.sqrt(np.mean(v * v, -1, keepdims=True))
        step = dev(v.astype(np.float32).astype(np.float64) * h, "fp32")
        diff = (loss({**t, name: t[name] + step}) - loss({**t, name: t[name] - step})) / (2 * h)
        want = float((host(grad) * v).sum())
        bound = 4 * h * h * np.linalg.norm(host(grad)) * np.linalg.norm(v) + noise
        assert abs(diff - want) <= bound, (name, diff, want, bound)


def test_reference_gradient_is_the_derivative():
    """The 64-bit reference's gradient against its own differences (host only)."""
    r = np.random.default_rng(1)
    for inter in (False, True):
        x = make(1, 1, 1, 3, 24, 16, "fp32", 2)
        x["pos"][0, 1] = -1
        args = (x["cos"], x["sin"], x["pos"])
        dx, dw, _ = R.norm_rope_bwd(x["q"], x["wq"], *args, x["gq"], EPS, inter)
        f = lambda a, w: float((R.norm_rope(a, w, *args, EPS, inter) * x["gq"]).sum())
        for _ in range(5):
            v, u, h = r.normal(size=x["q"].shape), r.normal(size=24), 1e-5
            want = (f(x["q"] + h * v, x["wq"]) - f(x["q"] - h * v, x["wq"])) / (2 * h)
            assert abs(want - (dx * v).sum()) <= 1e-7 * (np.abs(dx * v).sum() + 1)
            want = (f(x["q"], x["wq"] + h * u) - f(x["q"], x["wq"] - h * u)) / (2 * h)
            assert abs(want - (dw * u).sum()) <= 1e-7 * (np.abs(dw * u).sum() + 1)


# -- refusals (host only: fake, never dereferenced addresses) -------------------------------------
P = [0x10000000 * (i + 1) for i in range(14)]


@pytest.fixture(scope="module")
def L():
    from paper_2606_07713_gb300 import build
    build.build()
    return _lib.lib()


def contiguous(H, N, d):
    return (H * N * d, N * d, d)


def fwd(ptrs=None, B=2, Hq=4, Hk=2, N=8, d=64, rot=64, n_pos=100, strides=None, eps=1e-6, inter=0, dtype=1):
    p = list(P[:9]) if ptrs is None else ptrs
    st = strides or (contiguous(Hq, N, d) + contiguous(Hk, N, d)) * 2
    return _lib.moa_qk_norm_rope(*p, B, Hq, Hk, N, d, rot, n_pos, st, eps, inter, dtype, None)


def bwd(ptrs=None, B=2, Hq=4, Hk=2, N=8, d=64, rot=64, n_pos=100, ws=P[13], ws_bytes=1 << 20, dtype=1):
    p = list(P[:13]) if ptrs is None else ptrs
    st = (contiguous(Hq, N, d) + contiguous(Hk, N, d)) * 3
    return _lib.moa_qk_norm_rope_bwd(*p, B, Hq, Hk, N, d, rot, n_pos, st, 1e-6, 0, dtype, ws, ws_bytes, None)


def put(n, i, v):
    p = list(P[:n])
    p[i] = v
    return p


@pytest.mark.parametrize("kwargs,code", [
    *[(dict(ptrs=put(9, i, None)), _lib.MOA_ERR_INVALID_ARG) for i in range(9)],
    *[(dict(ptrs=put(9, i, P[i] + 2)), _lib.MOA_ERR_MISALIGNED) for i in range(9)],
    (dict(dtype=3), _lib.MOA_ERR_UNSUPPORTED_DTYPE),
    (dict(B=0), _lib.MOA_ERR_INVALID_ARG),
    (dict(N=-1), _lib.MOA_ERR_INVALID_ARG),
    (dict(n_pos=0), _lib.MOA_ERR_INVALID_ARG),
    (dict(eps=0.0), _lib.MOA_ERR_INVALID_ARG),
    (dict(eps=float("nan")), _lib.MOA_ERR_INVALID_ARG),
    (dict(d=60, rot=32), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(d=264), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(rot=72), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(rot=24), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(rot=0), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(B=2 ** 40, N=2 ** 30), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(Hq=70000), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
    (dict(ptrs=put(9, 7, P[1])), _lib.MOA_ERR_INVALID_ARG),            # Qo over K
    (dict(ptrs=put(9, 7, P[0] + 16)), _lib.MOA_ERR_INVALID_ARG),       # Qo shifted over Q
    (dict(ptrs=put(9, 8, P[7] + 64)), _lib.MOA_ERR_INVALID_ARG),       # Ko inside Qo
    (dict(ptrs=put(9, 7, P[4])), _lib.MOA_ERR_INVALID_ARG),            # Qo over cos
    # rows of 60 elements apart: not whole 16-byte units
    (dict(strides=(2048, 512, 60) + contiguous(2, 8, 64) + contiguous(4, 8, 64) + contiguous(2, 8, 64)), _lib.MOA_ERR_MISALIGNED),
    # an output whose rows lie on one another
    (dict(strides=contiguous(4, 8, 64) + contiguous(2, 8, 64) + (2048, 512, 0) + contiguous(2, 8, 64)), _lib.MOA_ERR_INVALID_ARG),
    (dict(strides=contiguous(4, 8, 64) + contiguous(2, 8, 64) + (2048, 448, 64) + contiguous(2, 8, 64)), _lib.MOA_ERR_INVALID_ARG),
    (dict(strides=(2 ** 60, 512, 64) + contiguous(2, 8, 64) + contiguous(4, 8, 64) + contiguous(2, 8, 64)), _lib.MOA_ERR_MISALIGNED),
])
def test_forward_refusals(L, kwargs, code):
    assert fwd(**kwargs) == code
    assert _lib.moa_last_error() != ""


@pytest.mark.parametrize("kwargs,code", [
    *[(dict(ptrs=put(13, i, None)), _lib.MOA_ERR_INVALID_ARG) for i in range(13)],
    (dict(ws=None), _lib.MOA_ERR_INVALID_ARG),
    (dict(ws=P[13] + 8), _lib.MOA_ERR_MISALIGNED),
    (dict(ws=P[0]), _lib.MOA_ERR_INVALID_ARG),                         # workspace over Q
    (dict(ptrs=put(13, 11, P[2])), _lib.MOA_ERR_INVALID_ARG),          # dW_q over W_q
    (dict(ptrs=put(13, 12, P[11] + 4)), _lib.MOA_ERR_INVALID_ARG),     # dW_k over dW_q
    (dict(ptrs=put(13, 9, P[0])), _lib.MOA_ERR_INVALID_ARG),           # dQ over Q
    (dict(ptrs=put(13, 10, P[9])), _lib.MOA_ERR_INVALID_ARG),          # dK over dQ
    (dict(dtype=2), _lib.MOA_ERR_UNSUPPORTED_DTYPE),
    (dict(d=12), _lib.MOA_ERR_UNSUPPORTED_SHAPE),
])
def test_backward_refusals(L, kwargs, code):
    assert bwd(**kwargs) == code
    assert _lib.moa_last_error() != ""


def test_python_refusals_without_gpu():
    x = torch.zeros(1, 1, 1, 64)
    with pytest.raises(ValueError):
        pkg.qk_norm_rope(x, x, x, x, x, x, x)
    with pytest.raises(ValueError):
        pkg.kv4_write(x, x, x, x, x)


def test_rope_table_values():
    c, s = pkg.rope_table(50, 32, base=500.0, device="cpu")
    p, i = np.arange(50)[:, None], np.arange(16)
    a = p * 500.0 ** (-2 * i / 32)
    assert c.shape == (50, 16) and c.dtype == torch.float32
    assert np.abs(c.double().numpy() - np.cos(a)).max() <= 2.0 ** -24
    assert np.abs(s.double().numpy() - np.sin(a)).max() <= 2.0 ** -24
