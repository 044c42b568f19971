"""Calls whose work is divided between the CTAs of clusters, where the device has no room for clusters of that size (a context
with a part of the SMs): they take smaller ones, or none, and need the workspace that goes with it."""
import contextlib

import pytest

import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib

torch = pytest.importorskip("torch")


@contextlib.contextmanager
def room_for(most):
    assert pkg.moa_selftest_cluster_limit(most) == _lib.MOA_OK
    try:
        yield
    finally:
        assert pkg.moa_selftest_cluster_limit(0) == _lib.MOA_OK


@pytest.mark.parametrize("most", [-1, 3, 12, 17, 32, 2 ** 31 - 1])
def test_limits_that_are_none(most):
    assert pkg.moa_selftest_cluster_limit(most) == _lib.MOA_ERR_INVALID_ARG
    assert pkg.moa_last_error()


DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def rand(seed, dtype, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(DTYPES[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,Hq,Hk,N,dk,dv,window,sinks", [
    ([5000], 4, 1, 1, 128, 128, 1024, 4), ([8192], 16, 8, 1, 128, 64, 0, 0), ([2000, 900, 0], 8, 2, 5, 64, 64, 0, 0),
    ([300] * 3, 8, 4, 60, 64, 128, 0, 0), ([130], 2, 1, 1, 64, 64, 0, 0),
])
@pytest.mark.parametrize("most", [1, 2, 4, 8])
def test_smaller_clusters(lens, Hq, Hk, N, dk, dv, window, sinks, dtype, most):
    """The same rows, from other divisions: both within the roundings of the products' operands (bf16: the weights, 2^-8 of
    sum p |v|, and the output), of the scores (2 (d + 8) 2^-24 of their terms) and of the sums (2^-15)."""
    page, B = 32, len(lens)
    per = -(-max(lens) // page)
    pool = rand(1, dtype, B * per, Hk, page, dk + dv)
    pages = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per)
    q, ln = rand(2, dtype, B, Hq, N, dk), torch.tensor(lens, dtype=torch.int32, device="cuda")
    call = lambda **a: pkg.kv_attn_lse(q, pool, pages, ln, max_len=max(lens), window=window or None, sinks=sinks, **a)  # noqa: E731
    want, want_lse = call()
    with room_for(most):
        got, lse = call()
    again, again_lse = call()
    assert pkg.get_device_status() == _lib.MOA_OK
    assert torch.equal(again, want) and torch.equal(again_lse, want_lse)
    u = HALF[dtype]
    x = pool.view(B, per, Hk, page, dk + dv).transpose(1, 2).reshape(B, Hk, per * page, dk + dv).double()
    for b, n in enumerate(lens):
        for h in range(Hq):
            k, v = x[b, h // (Hq // Hk), :n, :dk], x[b, h // (Hq // Hk), :n, dk:]
            qq = q[b, h].double()
            p_, j = torch.arange(n - N, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
            see = (j <= p_) & ((j > p_ - window) | (j < sinks)) if window else j <= p_
            if n == 0:
                assert bool((got[b, h] == 0).all())
                continue
            p = torch.nan_to_num(torch.softmax((qq @ k.T * dk ** -0.5).masked_fill(~see, -torch.inf), 1), nan=0.0)
            size = (qq.abs() @ k.abs().T * dk ** -0.5).amax(1, keepdim=True)
            one = (2 * (dk + 8) * 2.0 ** -24 * size + 2.0 ** -18 + 2.0 ** -15 + (u if dtype == "bf16" else 0)) * (p @ v.abs())
            one = 1.02 * (one + u * (p @ v).abs()) + 1e-30
            for o in (got, want):
                assert bool(((o[b, h].double() - p @ v).abs() <= one).all()), (b, h)
    assert bool(((lse - want_lse).abs() <= 2.0 ** -15 + 2.0 ** -18 * want_lse.abs())[torch.isfinite(want_lse)].all())
    assert torch.equal(torch.isfinite(lse), torch.isfinite(want_lse))


@pytest.mark.gpu
def test_the_workspace_goes_with_the_division():
    """fp32: shares that no cluster joins lie in the workspace, one that is too small is refused."""
    size = lambda: pkg.moa_kv_attn_workspace_bytes(1, 4, 1, 1, 128, 128, 3000, 0, 0, _lib.MOA_FP32)  # noqa: E731
    assert size() == 0
    with room_for(1):
        need = size()
        assert need > 0
        q, pool = rand(1, "fp32", 1, 4, 1, 128), rand(2, "fp32", 100, 1, 32, 256)
        pages = torch.arange(100, dtype=torch.int32, device="cuda").view(1, 100)
        lens = torch.tensor([3000], dtype=torch.int32, device="cuda")
        with pytest.raises(pkg.MoaError):
            pkg.kv_attn(q, pool, pages, lens, max_len=3000, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))
        given = torch.empty(need, dtype=torch.uint8, device="cuda")
        got = pkg.kv_attn(q, pool, pages, lens, max_len=3000, workspace=given)
        assert torch.equal(got, pkg.kv_attn(q, pool, pages, lens, max_len=3000))
    assert size() == 0
    assert pkg.get_device_status() == _lib.MOA_OK
