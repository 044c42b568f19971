"""Outputs of the operators around attention that are slices of one buffer: whatever the order of its
dimensions, slices that share no element are written, and slices that do are refused."""
import numpy as np
import pytest

import paper_2606_07713_gb300 as pkg
from paper_2606_07713_gb300 import _lib

torch = pytest.importorskip("torch")

B, H_Q, H_K, N, D = 3, 4, 2, 21, 64

# name: (whole, q, k), q [B, H_Q, N, D] and k [B, H_K, N, D] views of one new buffer
def token_major(heads=H_Q + H_K + 1):
    x = torch.zeros(B, N, heads, D, device="cuda:0", dtype=torch.bfloat16)
    return x, x[:, :, :H_Q].transpose(1, 2), x[:, :, H_Q:H_Q + H_K].transpose(1, 2)


def head_major():
    x = torch.zeros(B, H_Q + H_K + 1, N, D, device="cuda:0", dtype=torch.bfloat16)
    return x, x[:, :H_Q], x[:, H_Q:H_Q + H_K]


def keys_first():
    x = torch.zeros(B, H_Q + H_K, N, D, device="cuda:0", dtype=torch.bfloat16)
    return x, x[:, H_K:], x[:, :H_K]


def tokens_before_sequences():
    x = torch.zeros(N, B, H_Q + H_K, D, device="cuda:0", dtype=torch.bfloat16)
    return x, x[:, :, :H_Q].permute(1, 2, 0, 3), x[:, :, H_Q:].permute(1, 2, 0, 3)


def heads_before_all():
    x = torch.zeros(H_Q + H_K, N, B, D, device="cuda:0", dtype=torch.bfloat16)
    return x, x[:H_Q].permute(2, 0, 1, 3), x[H_Q:].permute(2, 0, 1, 3)


def features_beside_each_other():
    x = torch.zeros(B, N, H_Q, 2, D, device="cuda:0", dtype=torch.bfloat16)
    return x, x[:, :, :, 0].transpose(1, 2), x[:, :, :H_K, 1].transpose(1, 2)


LAYOUTS = [token_major, head_major, keys_first, tokens_before_sequences, heads_before_all, features_beside_each_other]


def operands():
    g = torch.Generator(device="cuda:0").manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda:0").bfloat16()  # noqa: E731
    cos, sin = pkg.rope_table(64, D, device="cuda:0")
    pos = torch.arange(N, dtype=torch.int32, device="cuda:0").repeat(B, 1)
    return rand(B, H_Q, N, D), rand(B, H_K, N, D), (rand(D), rand(D), cos, sin, pos)


def untouched(whole, views):
    """Whether the buffer holds zeros outside the views."""
    mine = torch.zeros_like(whole)
    for v in views:
        at = v.storage_offset()
        mine.as_strided(v.shape, v.stride(), at).fill_(1.0)
    return bool((whole[mine == 0] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda f: f.__name__)
def test_norm_in_place_and_gradients(layout):
    q, k, rest = operands()
    want = pkg.qk_norm_rope(q, k, *rest)
    whole, qs, ks = layout()
    qs.copy_(q), ks.copy_(k)
    pkg.qk_norm_rope(qs, ks, *rest, out=(qs, ks))
    assert torch.equal(qs, want[0]) and torch.equal(ks, want[1]) and untouched(whole, (qs, ks))
    grads = pkg.qk_norm_rope_bwd(q, k, *rest, *want)
    whole, qs, ks = layout()
    qs.copy_(want[0]), ks.copy_(want[1])
    got = pkg.qk_norm_rope_bwd(q, k, *rest, qs, ks, out=(qs, ks))
    assert all(torch.equal(a, b) for a, b in zip(got, grads)) and untouched(whole, (qs, ks))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda f: f.__name__)
def test_rows_read_into_slices(layout):
    _, _, rest = operands()
    whole, x, _ = layout()
    pool = pkg.kv4_pool(B * 2, H_K, 16, D, D)
    pages = torch.arange(2 * B, dtype=torch.int32, device="cuda:0").view(B, 2)
    k, v = torch.randn(2, B, H_K, N, D, device="cuda:0").bfloat16()
    pkg.kv4_write(k, v, pool, pages, rest[-1])
    want = pkg.kv4_read(pool, pages, rest[-1], D)
    whole, qs, ks = layout()
    vs = qs[:, :H_K]
    pkg.kv4_read(pool, pages, rest[-1], D, out=(ks, vs))
    assert torch.equal(ks, want[0]) and torch.equal(vs, want[1]) and untouched(whole, (ks, vs))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", LAYOUTS[:4], ids=lambda f: f.__name__)
def test_slices_that_share_elements_are_refused(layout):
    """The keys' slice moved by one head, one token or eight features into the queries'."""
    q, k, rest = operands()
    whole, qs, ks = layout()
    for step in (qs.stride(1), qs.stride(2), 8, qs.stride(0)):
        at = qs.storage_offset() + step
        if at + sum((s - 1) * st for s, st in zip(ks.shape, ks.stride())) >= whole.numel():
            continue
        moved = whole.view(-1).as_strided(ks.shape, ks.stride(), at)
        with pytest.raises(_lib.MoaError) as e:
            pkg.qk_norm_rope(q, k, *rest, out=(qs, moved))
        assert "overlaps" in str(e.value)
    torch.cuda.synchronize()
    assert bool((whole == 0).all())
