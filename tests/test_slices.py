"""Outputs that are slices of one buffer with other tensors: a call takes them where no element is shared
and refuses them where one is, whatever the rows' lengths.  No GPU is needed: every call here is refused in the
end, for its tensors or, where those pass, for a fault that is looked at after them."""
import itertools

import numpy as np
import pytest

import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib

BASE = 0x10000000
UNIT = 8   # bf16 values of 16 bytes: pointers and strides are multiples


def units(at, strides, B, H, N, d):
    """The 16-byte pieces that a tensor's elements lie in (`at` and strides in elements)."""
    rows = [at + b * strides[0] + h * strides[1] + n * strides[2] for b, h, n in itertools.product(range(B), range(H), range(N))]
    return {(r + e) // UNIT for r in rows for e in range(0, d, UNIT)}


def append(q_at, k_at, v_at, sq, sk, sv, B, H_q, H_k, N, d_k, d_v):
    """moa_kv_append with the queries rotated in place; the pool lies on the angles, which is refused after the tensors."""
    far = BASE + (1 << 32)
    status = pkg.moa_kv_append(
        Q=BASE + 2 * q_at, K=BASE + 2 * k_at, V=BASE + 2 * v_at, cos=far, sin=far + (1 << 28), pool=far, pages=far + (2 << 28),
        pos=far + (3 << 28), Qo=BASE + 2 * q_at, B=B, H_q=H_q, H_k=H_k, N=N, d_k=d_k, d_v=d_v, d_rot=d_k, n_pos=64, n_pages=9,
        page_tokens=16, max_pages=4, strides=[*sq, *sk, *sv, *sq], interleaved=0, dtype=_lib.MOA_BF16, stream=None)
    assert status == _lib.MOA_ERR_INVALID_ARG
    return pkg.moa_last_error()


def read(k_at, v_at, sk, sv, B, H, N, d_k, d_v):
    """moa_kv4_read; pos lies on K, which is refused after K and V."""
    far = BASE + (1 << 32)
    status = pkg.moa_kv4_read(
        pool=far, pages=far + (1 << 28), pos=BASE + 2 * k_at, K=BASE + 2 * k_at, V=BASE + 2 * v_at, B=B, H=H, N=N, d_k=d_k, d_v=d_v,
        n_pages=9, page_tokens=16, max_pages=4, strides=[*sk, *sv], dtype=_lib.MOA_BF16, stream=None)
    assert status == _lib.MOA_ERR_INVALID_ARG
    return pkg.moa_last_error()


TENSORS_PASS = {append: "the pool overlaps", read: "an output overlaps pages or pos"}


@pytest.mark.parametrize("d_k,d_v", [(64, 64), (128, 128), (128, 64), (64, 128)])
@pytest.mark.parametrize("B,H_q,H_k,N", [(2, 4, 2, 33), (1, 6, 3, 1), (3, 2, 2, 5), (2, 1, 1, 7)])
def test_the_projection_of_a_layer(B, H_q, H_k, N, d_k, d_v):
    """[B, N, H_q d_k + H_k d_k + H_k d_v], and the same with the tokens inside the heads."""
    width = H_q * d_k + H_k * (d_k + d_v)
    s = lambda d: (N * width, d, width)  # noqa: E731
    assert TENSORS_PASS[append] in append(0, H_q * d_k, (H_q + H_k) * d_k, s(d_k), s(d_k), s(d_v), B, H_q, H_k, N, d_k, d_v)
    s = lambda d: (N * width, N * d, d)  # noqa: E731
    if N == 1 or d_k == d_v:   # (rows of one token's stride: another's where the rows differ in length)
        assert TENSORS_PASS[append] in append(0, H_q * d_k * N, (H_q + H_k) * d_k * N, s(d_k), s(d_k), s(d_v), B, H_q, H_k, N, d_k,
                                              d_v)
    both = H_k * (d_k + d_v)
    s = lambda d: (N * both, d, both)  # noqa: E731
    assert TENSORS_PASS[read] in read(0, H_k * d_k, s(d_k), s(d_v), B, H_k, N, d_k, d_v)
    # keys and values in turn, head after head
    s = (N * both, d_k + d_v, both)
    assert TENSORS_PASS[read] in read(0, d_k, s, s, B, H_k, N, d_k, d_v)


def test_values_that_reach_into_the_next_head():
    """Heads 128 apart, keys of 64 features at 0 and values of 128 at 64: a value ends in the next head's key."""
    s = (3 * 256, 128, 256)
    assert "K overlaps V" in read(0, 64, s, s, 2, 2, 3, 64, 128)
    assert "Qo overlaps V" in append(0, 4096, 64, s, (4096, 64, 256), s, 1, 2, 2, 3, 64, 128)
    # the last head's value would reach into the next token
    assert "K overlaps V" in read(0, 64, (4096, 64, 128), (4096, 64, 128), 1, 1, 3, 64, 128)


@pytest.mark.parametrize("call", [append, read], ids=["append", "read"])
def test_nothing_that_is_shared_is_taken(call):
    """Small random layouts: whatever passes shares no element."""
    r = np.random.default_rng(11)
    taken = shared = 0
    for _ in range(6000):
        B, N, H, Hk = (int(x) for x in r.integers(1, 4, size=4))
        d_k, d_v = (int(x) for x in r.choice([64, 128], size=2))
        sb, sn = (int(x) * 64 for x in r.integers(1, 13, size=2))
        heads = [int(x) * 64 for x in r.integers(1, 7, size=2)]
        at = int(r.integers(-12, 13)) * 64
        if call is append:
            a = (0, (sb, heads[0], sn), B, H, N, d_k)
            b = (at, (sb, heads[1], sn), B, Hk, N, d_v)
            msg = append(0, 1 << 24, at, a[1], (1 << 20, 1 << 16, 1 << 12), b[1], B, H, Hk, N, d_k, d_v)
        else:
            a = (0, (sb, heads[0], sn), B, H, N, d_k)
            b = (at, (sb, heads[1], sn), B, H, N, d_v)
            msg = read(0, at, a[1], b[1], B, H, N, d_k, d_v)
        if "rows overlap" in msg:
            continue
        both = units(*a) & units(*b)
        if TENSORS_PASS[call] in msg:
            taken += 1
            assert not both, (a, b)
        else:
            shared += bool(both)
            assert "overlaps V" in msg
    assert taken > 100 and shared > 100


torch = pytest.importorskip("torch")
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def pieces(B, N, heads, lengths, dtype, seed):
    """A layer's projection [B, N, sum of heads x lengths], and its slices [B, heads, N, length]."""
    g = torch.Generator().manual_seed(seed)
    whole = torch.randn(B, N, sum(h * d for h, d in zip(heads, lengths)), generator=g).to("cuda", dtype)
    out, at = [], 0
    for h, d in zip(heads, lengths):
        out.append(whole[..., at:at + h * d].unflatten(-1, (h, d)).transpose(1, 2))
        at += h * d
    return whole, out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d_k,d_v", [(128, 64), (64, 128)])
def test_append_in_place_of_rows_of_two_lengths(d_k, d_v, dtype):
    B, Hq, Hk, N, page = 2, 4, 2, 33, 16
    whole, (q, k, v) = pieces(B, N, (Hq, Hk, Hk), (d_k, d_k, d_v), DTYPES[dtype], 5)
    cos, sin = pkg.rope_table(64, d_k)
    table = torch.arange(B * 3, dtype=torch.int32, device="cuda").view(B, 3)
    pos = torch.arange(N, dtype=torch.int32, device="cuda").expand(B, N).contiguous()
    pools = [pkg.kv_pool(B * 3, Hk, page, d_k, d_v, dtype=DTYPES[dtype]) for _ in range(2)]
    want = pkg.kv_append(k.contiguous(), v.contiguous(), pools[0], table, pos, cos, sin, q=q.contiguous())
    keep = whole[..., Hq * d_k:].clone()
    got = pkg.kv_append(k, v, pools[1], table, pos, cos, sin, q=q, out=q)
    assert pkg.get_device_status() == _lib.MOA_OK
    assert got.data_ptr() == whole.data_ptr() and torch.equal(got, want) and torch.equal(pools[0], pools[1])
    assert torch.equal(whole[..., Hq * d_k:], keep)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d_k,d_v", [(128, 64), (64, 128)])
def test_gradients_into_the_gradient_of_a_projection(d_k, d_v, dtype):
    B, Hq, Hk, N = 2, 4, 2, 150
    _, (q, k, v) = pieces(B, N, (Hq, Hk, Hk), (d_k, d_k, d_v), DTYPES[dtype], 6)
    o, lse = pkg.window_attn_lse(q, k, v, window=40, sinks=3)
    do = torch.randn(B, Hq, N, d_v, generator=torch.Generator().manual_seed(7)).to("cuda", DTYPES[dtype])
    want = pkg.window_attn_bwd(q, k, v, o, lse, do, window=40, sinks=3)
    _, out = pieces(B, N, (Hq, Hk, Hk), (d_k, d_k, d_v), DTYPES[dtype], 8)
    got = pkg.window_attn_bwd(q, k, v, o, lse, do, window=40, sinks=3, out=out)
    assert pkg.get_device_status() == _lib.MOA_OK
    for x, y, z in zip(got, want, out):
        assert x.data_ptr() == z.data_ptr() and torch.equal(x, y)
