"""The operators around attention on streams other than torch's current one, and in captured graphs.

The outputs have to be bit for bit those of a plain call on the current stream: the same kernels run
on the same inputs, and none of them depends on the order in which CTAs finish.
"""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def _layer(dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    B, Hq, Hk, N, d, page = 3, 8, 2, 37, 64, 16
    r = lambda *s: torch.randn(*s, generator=g).to("cuda", dtype)  # noqa: E731
    import paper_2606_07713_gb300 as pkg
    cos, sin = pkg.rope_table(256, 64)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")[None].repeat(B, 1).contiguous()
    pages = torch.randperm(B * 8, generator=g)[:B * 8].to(torch.int32).reshape(B, 8).cuda()
    return dict(q=r(B, Hq, N, d), k=r(B, Hk, N, d), v=r(B, Hk, N, d), wq=r(d), wk=r(d), cos=cos, sin=sin,
                pos=pos, pages=pages, pool=pkg.kv4_pool(B * 8, Hk, page, d, d),
                lens=torch.tensor([N, N, 5], dtype=torch.int32, device="cuda"))


def _run(t, stream=None):
    """Every operator, each on the one before it; new outputs and workspaces."""
    import paper_2606_07713_gb300 as pkg
    a = (t["wq"], t["wk"], t["cos"], t["sin"], t["pos"])
    qr, kr = pkg.qk_norm_rope(t["q"], t["k"], *a, stream=stream)
    pkg.kv4_write(kr, t["v"], t["pool"], t["pages"], t["pos"], stream=stream)
    o, lse = pkg.kv4_attn_lse(qr, t["pool"], t["pages"], t["lens"], stream=stream)
    kb, vb = pkg.kv4_read(t["pool"], t["pages"], t["pos"], 64, dtype=t["q"].dtype, stream=stream)
    grads = pkg.qk_norm_rope_bwd(t["q"], t["k"], *a, qr, kr, stream=stream)
    return [qr, kr, o, lse, kb, vb, *grads]


def _same(got, want):
    for x, y in zip(got, want, strict=True):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_stream_that_is_not_the_current_one(dtype):
    t = _layer(dtype)
    want = _run(t)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = _run(t, side)
    # memory asked for meanwhile on the current stream is not that of the calls still under way
    noise = [torch.full((1 << 16,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    side.synchronize()
    torch.cuda.synchronize()
    _same(got, want)
    assert all(bool((n == 7).all()) for n in noise)


def test_the_default_stream_named_while_another_is_current():
    t = _layer(torch.bfloat16, 1)
    want = _run(t)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = _run(t, torch.cuda.default_stream())
    torch.cuda.synchronize()
    _same(got, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_captured_graph_replays_on_new_inputs(dtype):
    t = _layer(dtype, 2)
    _run(t)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = _run(t)
    other = _layer(dtype, 3)
    for name in ("q", "k", "v", "lens", "pages"):
        t[name].copy_(other[name])
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in got]
    _same(got, _run(t))
