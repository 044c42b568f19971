"""Workspaces of the caller's in the Python calls of windowed attention, its gradients and attention over the cache; the device
status after queries that are not numbers."""
import pytest

import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"bf16": (torch.bfloat16, _lib.MOA_BF16), "fp32": (torch.float32, _lib.MOA_FP32)}


def rand(seed, dtype, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def buffer(n, shift=0):
    """n bytes from a 16-byte boundary, or `shift` past one, with 256 bytes on either side that stay as they are."""
    whole = torch.full((n + 512 + 16,), 7, dtype=torch.uint8, device="cuda")
    at = 256 + -whole.data_ptr() % 16 + shift
    return whole, whole[at:at + n]


def untouched(whole, part):
    at = part.data_ptr() - whole.data_ptr()
    return bool((whole[:at] == 7).all()) and bool((whole[at + part.numel():] == 7).all())


def check(call, need, want):
    """The same results with a workspace of the size asked for; one that is smaller, not aligned, or on a tensor is refused."""
    whole, ws = buffer(max(need, 16))
    got = call(ws)
    torch.cuda.synchronize()
    assert pkg.get_device_status() == _lib.MOA_OK
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and untouched(whole, ws)
    if need == 0:
        return
    with pytest.raises(pkg.MoaError, match="too small"):
        call(ws[:need - 1])
    with pytest.raises(pkg.MoaError, match="aligned"):
        call(buffer(need, 8)[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,Hq,Hk,N,M,dk,dv,window,sinks", [
    (1, 4, 2, 1, 5000, 128, 128, 900, 4), (2, 8, 2, 900, 900, 64, 64, 100, 3), (1, 2, 2, 40, 6000, 128, 64, 0, 0),
    (3, 4, 4, 130, 130, 64, 128, 0, 0),
])
def test_dense(B, Hq, Hk, N, M, dk, dv, window, sinks, dtype):
    dt, code = DTYPES[dtype]
    q, k, v, do = rand(1, dt, B, Hq, N, dk), rand(2, dt, B, Hk, M, dk), rand(3, dt, B, Hk, M, dv), rand(4, dt, B, Hq, N, dv)
    sight = dict(window=window or None, sinks=sinks)
    o, lse = pkg.window_attn_lse(q, k, v, **sight)
    sizes = (B, Hq, Hk, N, M, dk, dv, window, sinks, code)
    need = pkg.moa_window_attn_workspace_bytes(*sizes)
    check(lambda ws: pkg.window_attn_lse(q, k, v, **sight, workspace=ws), need, (o, lse))
    check(lambda ws: (pkg.window_attn(q, k, v, **sight, workspace=ws),), need, (o,))
    check(lambda ws: pkg.window_attn_bwd(q, k, v, o, lse, do, **sight, workspace=ws), pkg.moa_window_attn_bwd_workspace_bytes(*sizes),
          pkg.window_attn_bwd(q, k, v, o, lse, do, **sight))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,Hq,Hk,N", [([5000], 8, 2, 1), ([900] * 40, 8, 4, 3), ([300, 2000], 4, 2, 200)])
def test_cache(lens, Hq, Hk, N, dtype):
    dt, code = DTYPES[dtype]
    page, d, B, L = 64, 128, len(lens), max(lens)
    per = -(-L // page)
    pool, q = rand(1, dt, B * per, Hk, page, 2 * d), rand(2, dt, B, Hq, N, d)
    pages = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    call = lambda ws=None: pkg.kv_attn_lse(q, pool, pages, ln, max_len=L, workspace=ws)  # noqa: E731
    check(call, pkg.moa_kv_attn_workspace_bytes(B, Hq, Hk, N, d, d, L, 0, 0, code), call())
    need = pkg.moa_kv_attn_workspace_bytes(B, Hq, Hk, N, d, d, L, 0, 0, code)
    if 0 < need <= pool.numel() * pool.element_size():
        with pytest.raises(pkg.MoaError, match="overlaps"):
            call(pool.view(-1).view(torch.uint8)[:need])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens", [[100], [1500, 40, 129], [200] * 20, [9000] * 2])
def test_queries_that_are_not_numbers_leave_no_status(lens, dtype):
    dt, _ = DTYPES[dtype]
    Hq, Hk, N, d, page, B = 8, 4, 3, 64, 32, len(lens)
    per = -(-max(lens) // page)
    pool, q = rand(1, dt, B * per, Hk, page, 2 * d), rand(2, dt, B, Hq, N, d)
    pages = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q[-1, 5, 1, 7] = float("nan")
    o, lse = pkg.kv_attn_lse(q, pool, pages, ln, window=50, sinks=2)
    assert pkg.get_device_status() == _lib.MOA_OK
    assert int(torch.isnan(o).sum()) == d and int(torch.isnan(lse).sum()) == 1 and bool(torch.isnan(o[-1, 5, 1]).all())
