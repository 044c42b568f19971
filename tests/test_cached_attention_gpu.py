"""The example layer (examples/cached_attention.py): what it generates from its 4-bit cache against a
plain fp32 layer that keeps every key and value, quantised the same way.

The plain layer follows the library's own outputs token by token, so its inputs are the same; what
differs is rounding: projections (bf16, 2^-8), the norm's output (2^-8), a code that falls the other
way for it (one step, a seventh of a group's largest value, for the few per cent of values within 2^-7
of a boundary: about 0.03 of a value's size on average), weights and output (2^-8 each).  Bound: 0.1 of
the largest output.
"""
import os
import sys

import numpy as np
import pytest

import ops_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import cached_attention as ex  # noqa: E402


def plain_step(layer, tokens):
    """Output [H, d] of the last of tokens [n, d_model], in 64 bits on the host."""
    h = lambda t: t.detach().double().cpu().numpy()
    n, H, d = tokens.shape[0], layer.heads, layer.d
    y = (h(tokens) @ h(layer.w)).reshape(n, 3, H, d).transpose(1, 2, 0, 3)[:, None]
    pos = np.arange(n, dtype=np.int32)[None]
    q, k = (R.bf16(R.norm_rope(R.bf16(x), h(w), h(layer.cos), h(layer.sin), pos, 1e-6, False))
            for x, w in ((y[0], layer.wq), (y[1], layer.wk)))
    kv = [R.values(*R.quantise(x))[0] for x in (k, R.bf16(y[2]))]
    return R.attention_dense(q[0, :, -1:], *kv, n, d ** -0.5, True)[0][:, 0]


def test_generation_follows_the_plain_layer():
    torch.manual_seed(3)
    layer = ex.Layer(d_model=512, heads=8, d=64, max_tokens=400)
    prompts = [torch.randn(n, 512, device="cuda").bfloat16() for n in (300, 131, 1)]
    steps = 4
    out, cache = ex.generate(layer, prompts, steps, chunk=128)
    assert cache.lens == [n + steps for n in (300, 131, 1)]
    for b, p in enumerate(prompts):
        # the first step's token is the prompt's last output: only later steps' tokens are known here
        tokens = [p] + [None] + [o[b].reshape(1, 512) for o in out[:-1]]
        first = plain_step(layer, p)
        tokens[1] = torch.from_numpy(first.reshape(1, 512)).cuda().bfloat16()
        for i in range(steps):
            want = plain_step(layer, torch.cat(tokens[:2 + i]))
            got = out[i, b].double().cpu().numpy()
            assert np.abs(got - want).max() <= 0.1 * np.abs(want).max(), (b, i)


def test_chunks_and_single_tokens_agree():
    """The same sequence in chunks of 128, of 37, and token by token: the same cache, bit for bit, and
    outputs that differ by the weights' rounding only (2 * 2^-8 of the values' size, plus the
    output's)."""
    torch.manual_seed(4)
    layer = ex.Layer(d_model=256, heads=4, d=64, max_tokens=300)
    x = torch.randn(1, 150, 256, device="cuda").bfloat16()
    results = []
    for chunk in (150, 37, 1):
        cache = ex.Cache(layer, 1, 150)
        o = [ex.extend(layer, cache, x[:, i:i + chunk].contiguous(), [min(chunk, 150 - i)]) for i in range(0, 150, chunk)]
        results.append((torch.cat(o, 2), cache.pool[cache.pages[0].long()]))
    for o, pool in results[1:]:
        assert torch.equal(pool, results[0][1])
        assert float((o - results[0][0]).abs().max()) <= 4 * 2.0 ** -8 * float(results[0][0].abs().max()) + 1e-3


def test_training_step_gradients():
    """dwq, dwk of the layer's loss by central differences in the weights (the loss is smooth in them;
    bf16 rounding of norms, weights and outputs leaves about a per cent)."""
    torch.manual_seed(5)
    layer = ex.Layer(d_model=256, heads=4, d=64, max_tokens=300)
    x = torch.randn(2, 256, 256, device="cuda").bfloat16()
    target = torch.randn(2, 4, 256, 64, device="cuda")
    loss, dq, dk, dv, dwq, dwk = layer.train_step(x, target)
    assert all(bool(torch.isfinite(t).all()) for t in (loss, dq, dk, dv, dwq, dwk))
    for name, grad in (("wq", dwq), ("wk", dwk)):
        v = torch.sign(grad)
        w, h = getattr(layer, name), 0.125
        moved = []
        for s in (h, -h):
            setattr(layer, name, (w.float() + s * v).bfloat16())
            moved.append(float(layer.train_step(x, target)[0]))
        setattr(layer, name, w)
        step = float(((w.float() + h * v).bfloat16().float() - (w.float() - h * v).bfloat16().float()).abs().mean())
        want = (moved[0] - moved[1]) / step
        got = float(grad.abs().sum())
        assert abs(got - want) <= 0.1 * abs(want), (name, got, want)
