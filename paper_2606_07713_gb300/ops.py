"""Operators around attention: per-head norms of queries and keys with the rotation of positions,
their gradients, a paged 4-bit cache with the attention that reads it, attention with a sliding window
and its gradients, and a paged 16- or 32-bit cache with the attention that reads it.

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


def window_attn(q, k, v, window: int | None = None, sinks: int = 0, scale: float | None = None, out=None,
                workspace=None, stream=None):
    """Causal attention of q [B, H_q, N_q, d_k] over k [B, H_k, N_k, d_k] and v [B, H_k, N_k, d_v]:
    [B, H_q, N_q, d_v].

    The queries stand at the last N_q of the N_k positions.  A query at position p sees the tokens
    j <= p with j > p - window or j < sinks (window None: all j <= p); one that sees nothing gives
    zeros.  Query head h reads key head h // (H_q / H_k).  scale defaults to 1 / sqrt(d_k).
    A batch padded at the end needs no lengths; what a query does not see, not numbers included, has no
    influence on it."""
    return _b.window_attn(q, k, v, window, sinks, scale, out, None, workspace, stream)


def window_attn_lse(q, k, v, window: int | None = None, sinks: int = 0, scale: float | None = None, out=None,
                    lse=None, workspace=None, stream=None):
    """(o, lse): window_attn's output and the float32 [B, H_q, N_q] natural logarithm of each row's sum
    of exponentials of scaled scores (-inf for a query that sees nothing)."""
    return _b.window_attn(q, k, v, window, sinks, scale, out, True if lse is None else lse, workspace, stream)


def window_attn_bwd(q, k, v, o, lse, do, window: int | None = None, sinks: int = 0, scale: float | None = None,
                    out=None, workspace=None, stream=None):
    """(dq, dk, dv): the gradients of window_attn for the gradient do of its output, from the o and lse
    of window_attn_lse.  out: three tensors of the shapes of q, k and v.

    What a query does not see, not numbers included, has no influence on its gradient, nor it on a hidden
    token's.  A batch's padding is finite all the same: by the formula a query that is not a number reaches all tokens that it sees."""
    return _b.window_attn_bwd(q, k, v, o, lse, do, window, sinks, scale, out, workspace, stream)


def kv_pool(n_pages: int, H: int, page_tokens: int, d_k: int, d_v: int, dtype=None, device="cuda"):
    """An empty pool of the 16- or 32-bit cache: [n_pages, H, page_tokens, d_k + d_v] of dtype
    (torch.bfloat16 by default), a token's key and then its value."""
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    if page_tokens % 16 or page_tokens < 16 or d_k not in (64, 128) or d_v not in (64, 128):
        raise ValueError("kv_pool: page_tokens must be a multiple of 16, d_k and d_v 64 or 128")
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"kv_pool: unsupported dtype {dtype}; use torch.bfloat16 or torch.float32")
    return torch.zeros((n_pages, H, page_tokens, d_k + d_v), dtype=dtype, device=device)


def kv_append(k, v, pool, pages, pos, cos=None, sin=None, q=None, interleaved: bool = False, out=None, stream=None):
    """Writes keys [B, H_k, N, d_k] and values [B, H_k, N, d_v] into the pool (kv_pool): token n of
    sequence b goes to position pos[b, n], that is to page pages[b, pos // page_tokens], place
    pos % page_tokens.  pages: int32 [B, max_pages]; pos: int32 [B, N], negative: not written.

    With cos and sin (rope_table) the keys' first d_rot features are rotated by their positions' angles
    on the way (pairs as in qk_norm_rope), and so is q [B, H_q, N, d_k] if given: it is returned rotated
    (out: a tensor for it, q itself for in place), with zeros where the position is negative."""
    return _b.kv_append(k, v, pool, pages, pos, cos, sin, q, interleaved, out, stream)


def kv_attn(q, pool, pages, lens, max_len: int | None = None, window: int | None = None, sinks: int = 0,
            scale: float | None = None, causal: bool = True, out=None, workspace=None, stream=None):
    """Attention of q [B, H_q, N, d_k] over each sequence's tokens in the pool (kv_pool, kv_append):
    [B, H_q, N, d_v].

    lens: int32 [B] on the device, the tokens that each sequence has in the cache, the N queries being
    its last N: a query at position p sees the tokens j <= p (without causal: all) with j > p - window
    or j < sinks (window None: all of them).  A query that sees nothing gives zeros.  Query head h reads
    key head h // (H_q / H_k).  Pages that lie before every query's window are not looked at.
    max_len: an upper bound of lens known to the host (default: what the page table holds); the work is
    divided by it, so a close bound is faster."""
    return _b.kv_attn(q, pool, pages, lens, max_len, window, sinks, scale, causal, out, None, workspace, stream)


def kv_attn_lse(q, pool, pages, lens, max_len: int | None = None, window: int | None = None, sinks: int = 0,
                scale: float | None = None, causal: bool = True, out=None, lse=None, workspace=None, stream=None):
    """(o, lse): kv_attn's output and the float32 [B, H_q, N] natural logarithm of each row's sum of
    exponentials of scaled scores (-inf for a query that sees nothing)."""
    return _b.kv_attn(q, pool, pages, lens, max_len, window, sinks, scale, causal, out, True if lse is None else lse,
                      workspace, stream)
