"""Operators around attention: per-head norms of queries and keys with the rotation of positions,
their gradients, and a paged 4-bit cache with the attention that reads it.

The same thin binding as the rest of the package: every step of the computation runs in
libmoa_attn.so, and argument checks and marshalling in moa_torch.so beside it (a decoding step makes
several of these calls, so they are kept to a few microseconds).  Tensors are [B, H, N, d] CUDA
tensors with unit stride along d and any other strides (a transposed view of a token-major
[B, N, H, d] tensor needs no copy).  Calls run asynchronously on `stream` (default: torch's current
stream of the device); outputs and workspaces that they make are memory of that stream, as if it were
the current one; inputs have to live until their call has run there.  Nothing is recorded for
automatic differentiation: results of tensors that require gradients carry none, as with the rest of
the package, and writing into `out` does not count as a change of it.  What lives on the device
(positions, lengths, page numbers) is checked there: check(get_device_status()) raises if one was
outside its table.
"""
from __future__ import annotations

import importlib.machinery
import importlib.util
import os
import threading

from ._lib import MOA_BF16, MOA_FP32, MoaError

BINDING_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_build", "moa_torch.so")
_lock = threading.Lock()


class _Unloaded:
    """Stands for moa_torch until its first use, which loads it or raises."""

    def __getattr__(self, name):
        return getattr(_load(), name)


_b = _Unloaded()


def _load():
    global _b
    with _lock:
        if isinstance(_b, _Unloaded):
            import torch  # noqa: F401  (the binding links against its libraries)
            if not os.path.exists(BINDING_PATH):
                raise RuntimeError(
                    f"{BINDING_PATH} is missing: build it with "
                    "`python -c 'import __graft_entry__ as g; g.build()'` (needs nvcc and g++)")
            loader = importlib.machinery.ExtensionFileLoader("moa_torch", BINDING_PATH)
            spec = importlib.util.spec_from_file_location("moa_torch", BINDING_PATH, loader=loader)
            module = importlib.util.module_from_spec(spec)
            loader.exec_module(module)
            module.set_error(MoaError)
            _b = module
    return _b


def rope_table(n_pos: int, d_rot: int, base: float = 10000.0, device="cuda"):
    """(cos, sin) float32 [n_pos, d_rot / 2] of the angles p * base^(-2 i / d_rot), computed in 64
    bits and rounded once: the tables qk_norm_rope reads.  A program builds them once."""
    import torch
    i = torch.arange(d_rot // 2, dtype=torch.float64, device=device)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * float(base) ** (-2.0 * i / d_rot)
    return a.cos().float(), a.sin().float()


def qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps: float = 1e-6, interleaved: bool = False,
                 out=None, stream=None):
    """(q', k'): each head of q [B, H_q, N, d] and k [B, H_k, N, d] divided by its root mean square
    (with eps), multiplied by the weight wq or wk [d], its first d_rot features rotated by the
    angles of its token's position.  One pass over q and k.

    cos, sin: float32 [n_pos, d_rot / 2] (rope_table); pos: int32 [B, N], negative for padding (its
    rows become zeros).  Pairs are (i, i + d_rot/2), or (2i, 2i + 1) with interleaved.  out: a pair
    of tensors; q and k themselves for in place."""
    return _b.qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps, interleaved, out, stream)


def qk_norm_rope_bwd(q, k, wq, wk, cos, sin, pos, dqo, dko, eps: float = 1e-6,
                     interleaved: bool = False, out=None, workspace=None, stream=None):
    """(dq, dk, dwq, dwk): the gradients of qk_norm_rope for the gradients dqo, dko of its outputs.
    dq and dk have q's dtype, dwq and dwk are float32 [d].  out: a pair of tensors for dq and dk
    (dqo and dko themselves for in place); workspace: a CUDA uint8 tensor, allocated when not given."""
    return _b.qk_norm_rope_bwd(q, k, wq, wk, cos, sin, pos, dqo, dko, eps, interleaved, out, workspace, stream)


def kv4_pool(n_pages: int, H: int, page_tokens: int, d_k: int, d_v: int, device="cuda"):
    """An empty pool of the 4-bit cache: uint8 [n_pages, H, page_tokens / 16, 9 (d_k + d_v)], 4.5
    bits a value.  The other kv4 functions read the sizes from its shape."""
    import torch
    if page_tokens % 16 or page_tokens < 16 or d_k not in (64, 128) or d_v not in (64, 128):
        raise ValueError("kv4_pool: page_tokens must be a multiple of 16, d_k and d_v 64 or 128")
    return torch.zeros((n_pages, H, page_tokens // 16, 9 * (d_k + d_v)), dtype=torch.uint8, device=device)


def kv4_write(k, v, pool, pages, pos, stream=None) -> None:
    """Quantises keys [B, H, N, d_k] and values [B, H, N, d_v] into the pool (kv4_pool): token n of
    sequence b goes to position pos[b, n], that is to page pages[b, pos // page_tokens], place
    pos % page_tokens.  pages: int32 [B, max_pages]; pos: int32 [B, N], negative: not written."""
    _b.kv4_write(k, v, pool, pages, pos, stream)


def kv4_read(pool, pages, pos, d_k: int, dtype=None, out=None, stream=None):
    """(k, v): the cached rows at positions pos [B, N], widened to dtype (torch.bfloat16 by default):
    [B, H, N, d_k] and [B, H, N, d_v].  Negative positions give zeros."""
    import torch
    if out is not None and dtype is not None and any(t.dtype != dtype for t in out):
        raise TypeError(f"kv4_read: out must be {dtype}")
    if dtype is not None and dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise TypeError(f"kv4_read: unsupported dtype {dtype}; use torch.bfloat16 or torch.float32")
    return _b.kv4_read(pool, pages, pos, d_k, MOA_FP32 if dtype is torch.float32 else MOA_BF16, out, stream)


def kv4_attn(q, pool, pages, lens, max_len: int | None = None, scale: float | None = None,
             causal: bool = True, out=None, workspace=None, stream=None):
    """Attention of q [B, H_q, N, d_k] over each sequence's cached tokens: [B, H_q, N, d_v].

    lens: int32 [B] on the device, the tokens that each sequence has in the cache, the N queries
    being its last N tokens: with causal, query i sees the first lens[b] - N + i + 1 of them, else
    all.  A query that sees nothing gives zeros.  Query head j reads key head j // (H_q / H_k).
    max_len: an upper bound of lens known to the host (default: what the page table holds); the
    work is divided by it, so a close bound is faster."""
    return _b.kv4_attn(q, pool, pages, lens, max_len, scale, causal, out, None, workspace, stream)


def kv4_attn_lse(q, pool, pages, lens, max_len: int | None = None, scale: float | None = None,
                 causal: bool = True, out=None, lse=None, workspace=None, stream=None):
    """(o, lse): kv4_attn's output and the float32 [B, H_q, N] natural logarithm of each row's sum of
    exponentials of scaled scores (-inf for a query that sees nothing)."""
    return _b.kv4_attn(q, pool, pages, lens, max_len, scale, causal, out, True if lse is None else lse, workspace,
                       stream)
