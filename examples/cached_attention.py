"""One attention layer of a language model on this library, trained for a step and then generating.

    python examples/cached_attention.py [--tokens 256] [--steps 16]

The layer projects tokens to queries, keys and values (qkv_proj), norms each query and key head and
rotates it by its token's position (qk_norm_rope), and attends.  Training attends to the whole
sequence both ways (attn_fwd_lse; the gradients go back through attn_bwd and qk_norm_rope_bwd).
Generating, keys and values live in a paged 4-bit cache: a prompt is written (kv4_write) and attended
to in chunks, then every step appends one token to each sequence and attends with one query
(kv4_attn).  Sequences have prompts of different lengths; the cache's pages are handed out as they
grow.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_07713_gb300 as moa  # noqa: E402


class Layer:
    """Weights and shapes of the layer; tokens are rows of x [B, N, d_model] in bf16."""

    def __init__(self, d_model=512, heads=8, d=64, max_tokens=4096, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.d, self.device = heads, d, device
        self.w = (torch.randn(d_model, 3 * heads * d, generator=g, device=device) / d_model ** 0.5).bfloat16()
        self.wq = (1 + 0.1 * torch.randn(d, generator=g, device=device)).bfloat16()
        self.wk = (1 + 0.1 * torch.randn(d, generator=g, device=device)).bfloat16()
        self.cos, self.sin = moa.rope_table(max_tokens, d, device=device)

    def project(self, x, pos):
        """(q, k normed and rotated, v, and q, k before that) of tokens x at positions pos [B, N]."""
        q, k, v = moa.qkv_proj(x, self.w, self.heads, self.d, self.d)
        qn, kn = moa.qk_norm_rope(q, k, self.wq, self.wk, self.cos, self.sin, pos)
        return qn, kn, v, q, k

    def train_step(self, x, target):
        """Loss of the layer's output against target [B, H, N, d], and the gradients that reach the
        projections' outputs and the norms' weights: (loss, dq, dk, dv, dwq, dwk)."""
        B, N, _ = x.shape
        pos = torch.arange(N, dtype=torch.int32, device=x.device).expand(B, N).contiguous()
        qn, kn, v, q, k = self.project(x, pos)
        o, lse = moa.attn_fwd_lse(qn, kn, v)
        err = o.float() - target.float()
        do = (err * (2.0 / err.numel())).bfloat16()
        dqn, dkn, dv = moa.attn_bwd(qn, kn, v, o, lse, do)
        dq, dk, dwq, dwk = moa.qk_norm_rope_bwd(q, k, self.wq, self.wk, self.cos, self.sin, pos, dqn, dkn,
                                                out=(dqn, dkn))
        return (err * err).mean(), dq, dk, dv, dwq, dwk


class Cache:
    """Pages of the 4-bit cache for a batch of sequences, handed out as the sequences grow."""

    def __init__(self, layer: Layer, batch: int, max_tokens: int, page: int = 64):
        width = -(-max_tokens // page)
        self.page, self.device = page, layer.device
        self.pool = moa.kv4_pool(batch * width, layer.heads, page, layer.d, layer.d, device=layer.device)
        self.free = list(range(batch * width))
        self.pages = torch.full((batch, width), -1, dtype=torch.int32)   # on the host
        self.lens = [0] * batch

    def append(self, counts):
        """Room for counts[b] more tokens of each sequence: (their positions [B, max count] with -1 for
        padding, the table, the new lengths), on the device."""
        n = max(counts)
        pos = torch.full((len(counts), n), -1, dtype=torch.int32)
        for b, count in enumerate(counts):
            start = self.lens[b]
            # queries are the last of a call's n rows, so padding comes first
            pos[b, n - count:] = torch.arange(start, start + count, dtype=torch.int32)
            for slot in range(-(-start // self.page), -(-(start + count) // self.page)):
                self.pages[b, slot] = self.free.pop()
            self.lens[b] += count
        lens = torch.tensor(self.lens, dtype=torch.int32)
        return pos.to(self.device), self.pages.to(self.device), lens.to(self.device)


def extend(layer: Layer, cache: Cache, x, counts):
    """Attention output [B, H, N, d] of N new tokens a sequence (sequence b has counts[b] of them, the
    last rows of x[b]): they go into the cache and attend to all that it then holds before them."""
    pos, pages, lens = cache.append(counts)
    q, k, v, _, _ = layer.project(x, pos)
    moa.kv4_write(k, v, cache.pool, pages, pos)
    return moa.kv4_attn(q, cache.pool, pages, lens, max_len=max(cache.lens))


def generate(layer: Layer, prompts, steps: int, chunk: int = 128):
    """Runs prompts (a list of [n_b, d_model] tensors) in chunks and then `steps` single tokens a
    sequence, each next token being a fixed function of the last output (there is no vocabulary
    here).  Returns the outputs of the steps [steps, B, H, d] and the cache."""
    B, d_model = len(prompts), prompts[0].shape[1]
    cache = Cache(layer, B, max(p.shape[0] for p in prompts) + steps)
    done = [0] * B
    last = torch.zeros(B, layer.heads, layer.d, dtype=torch.bfloat16, device=layer.device)
    while any(done[b] < p.shape[0] for b, p in enumerate(prompts)):
        counts = [min(chunk, p.shape[0] - done[b]) for b, p in enumerate(prompts)]
        n = max(counts)
        x = torch.zeros(B, n, d_model, dtype=torch.bfloat16, device=layer.device)
        for b, p in enumerate(prompts):
            if counts[b]:
                x[b, n - counts[b]:] = p[done[b]:done[b] + counts[b]]
                done[b] += counts[b]
        o = extend(layer, cache, x, counts)
        for b in range(B):
            if counts[b]:
                last[b] = o[b, :, -1]
    outputs = []
    for _ in range(steps):
        x = torch.nn.functional.pad(last.reshape(B, 1, -1), (0, d_model - layer.heads * layer.d))
        last = extend(layer, cache, x.contiguous(), [1] * B)[:, :, 0]
        outputs.append(last)
    moa.check(moa.get_device_status())
    return torch.stack(outputs), cache


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=256, help="longest prompt")
    ap.add_argument("--steps", type=int, default=16, help="tokens to generate")
    a = ap.parse_args()
    layer = Layer(max_tokens=a.tokens + a.steps)
    x = torch.randn(2, a.tokens, 512, device="cuda").bfloat16()
    loss, *grads = layer.train_step(x, torch.zeros(2, layer.heads, a.tokens, layer.d, device="cuda"))
    print("one training step: loss %.4f, gradient sizes %s" % (loss, ["%.2e" % float(g.float().norm()) for g in grads]))
    prompts = [torch.randn(max(1, n), 512, device="cuda").bfloat16() for n in (a.tokens, a.tokens // 2, 3)]
    out, cache = generate(layer, prompts, a.steps)
    print("generated %d tokens for prompts of %s; the cache holds %s tokens in %.1f bits a value" % (
        a.steps, [p.shape[0] for p in prompts], cache.lens, 8 * cache.pool.shape[3] / (16 * 2 * layer.d)))
    print("size of the last outputs: %.3f" % float(out[-1].float().norm()))


if __name__ == "__main__":
    main()
