"""Operators around attention: per-head norms of queries and keys with the rotation of positions,
their gradients, and a paged 4-bit cache with the attention that reads it.

The same thin binding as the rest of the package: argument checks and marshalling here, every step
of the computation in libmoa_attn.so.  Tensors are [B, H, N, d] CUDA tensors with unit stride along
d and any other strides (a transposed view of a token-major [B, N, H, d] tensor needs no copy).
Calls run asynchronously on `stream` (default: torch's current stream of the device).  What lives
on the device (positions, lengths, page numbers) is checked there: check(get_device_status())
raises if one was outside its table.
"""
from __future__ import annotations

import math

from ._lib import (MOA_BF16, MOA_FP32, check, moa_kv4_attn, moa_kv4_attn_workspace_bytes,
                   moa_kv4_read, moa_kv4_write, moa_qk_norm_rope, moa_qk_norm_rope_bwd,
                   moa_qk_norm_rope_bwd_workspace_bytes)


def _code(what, dtype) -> int:
    import torch
    if dtype is torch.bfloat16:
        return MOA_BF16
    if dtype is torch.float32:
        return MOA_FP32
    raise TypeError(f"{what}: unsupported dtype {dtype}; use torch.bfloat16 or torch.float32")


def _heads(what, name, t, like=None, shape=None):
    """Checks a [B, H, N, d] tensor; returns its (b, h, n) strides."""
    if not t.is_cuda:
        raise ValueError(f"{what} needs CUDA tensors ({name})")
    if t.dim() != 4 or t.stride(3) != 1 and t.shape[3] > 1:
        raise ValueError(f"{what}: {name} must be [B, H, N, d] with unit stride along d")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: {name} must be {tuple(shape)}, got {tuple(t.shape)}")
    if like is not None:
        if t.dtype != like.dtype:
            raise TypeError(f"{what}: {name} must be {like.dtype}, got {t.dtype}")
        if t.device != like.device:
            raise ValueError(f"{what}: tensors on different devices")
    return t.stride()[:3]


def _flat(what, name, t, dtype, shape, device):
    if t.dtype != dtype:
        raise TypeError(f"{what}: {name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{what}: {name} must be a contiguous {tuple(shape)} tensor, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{what}: {name} is on {t.device}, not on {device}")


def _run(device, stream, call):
    """Runs call(raw stream) with `device` current and raises its error."""
    import torch
    if stream is None:
        stream = torch.cuda.current_stream(device)
    if device.index is None or device.index == torch.cuda.current_device():
        check(call(stream.cuda_stream))
        return
    with torch.cuda.device(device):
        check(call(stream.cuda_stream))


def rope_table(n_pos: int, d_rot: int, base: float = 10000.0, device="cuda"):
    """(cos, sin) float32 [n_pos, d_rot / 2] of the angles p * base^(-2 i / d_rot), computed in 64
    bits and rounded once: the tables qk_norm_rope reads.  A program builds them once."""
    import torch
    i = torch.arange(d_rot // 2, dtype=torch.float64, device=device)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * float(base) ** (-2.0 * i / d_rot)
    return a.cos().float(), a.sin().float()


def _norm_args(what, q, k, wq, wk, cos, sin, pos):
    import torch
    sq = _heads(what, "q", q)
    sk = _heads(what, "k", k, like=q)
    B, Hq, N, d = q.shape
    if k.shape[0] != B or k.shape[2] != N or k.shape[3] != d:
        raise ValueError(f"{what}: q and k must share B, N and d, got {tuple(q.shape)} {tuple(k.shape)}")
    dev = q.device
    _flat(what, "wq", wq, q.dtype, (d,), dev)
    _flat(what, "wk", wk, q.dtype, (d,), dev)
    if cos.dim() != 2:
        raise ValueError(f"{what}: cos must be [n_pos, d_rot / 2]")
    _flat(what, "cos", cos, torch.float32, cos.shape, dev)
    _flat(what, "sin", sin, torch.float32, cos.shape, dev)
    _flat(what, "pos", pos, torch.int32, (B, N), dev)
    return (B, Hq, k.shape[1], N, d, 2 * cos.shape[1], cos.shape[0]), sq + sk


def qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps: float = 1e-6, interleaved: bool = False,
                 out=None, stream=None):
    """(q', k'): each head of q [B, H_q, N, d] and k [B, H_k, N, d] divided by its root mean square
    (with eps), multiplied by the weight wq or wk [d], its first d_rot features rotated by the
    angles of its token's position.  One pass over q and k.

    cos, sin: float32 [n_pos, d_rot / 2] (rope_table); pos: int32 [B, N], negative for padding (its
    rows become zeros).  Pairs are (i, i + d_rot/2), or (2i, 2i + 1) with interleaved.  out: a pair
    of tensors; q and k themselves for in place."""
    import torch
    dims, strides = _norm_args("qk_norm_rope", q, k, wq, wk, cos, sin, pos)
    if out is None:
        qo = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        ko = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    else:
        qo, ko = out
    strides += (_heads("qk_norm_rope", "out[0]", qo, q, q.shape) +
                _heads("qk_norm_rope", "out[1]", ko, q, k.shape))
    code = _code("qk_norm_rope", q.dtype)
    _run(q.device, stream, lambda s: moa_qk_norm_rope(
        q.data_ptr(), k.data_ptr(), wq.data_ptr(), wk.data_ptr(), cos.data_ptr(), sin.data_ptr(),
        pos.data_ptr(), qo.data_ptr(), ko.data_ptr(), *dims, strides, float(eps),
        int(interleaved), code, s))
    return qo, ko


def qk_norm_rope_bwd(q, k, wq, wk, cos, sin, pos, dqo, dko, eps: float = 1e-6,
                     interleaved: bool = False, out=None, workspace=None, stream=None):
    """(dq, dk, dwq, dwk): the gradients of qk_norm_rope for the gradients dqo, dko of its outputs.
    dq and dk have q's dtype, dwq and dwk are float32 [d].  out: a pair of tensors for dq and dk
    (dqo and dko themselves for in place); workspace: a CUDA uint8 tensor, allocated when not given."""
    import torch
    what = "qk_norm_rope_bwd"
    dims, strides = _norm_args(what, q, k, wq, wk, cos, sin, pos)
    strides += _heads(what, "dqo", dqo, q, q.shape) + _heads(what, "dko", dko, q, k.shape)
    dev = q.device
    if out is None:
        dq = torch.empty(q.shape, dtype=q.dtype, device=dev)
        dk = torch.empty(k.shape, dtype=k.dtype, device=dev)
    else:
        dq, dk = out
    strides += _heads(what, "out[0]", dq, q, q.shape) + _heads(what, "out[1]", dk, q, k.shape)
    dw = torch.empty((2, dims[4]), dtype=torch.float32, device=dev)
    code = _code(what, q.dtype)

    def call(s):
        ws = workspace
        if ws is None:
            need = moa_qk_norm_rope_bwd_workspace_bytes(*dims[:5])
            ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
        return moa_qk_norm_rope_bwd(
            q.data_ptr(), k.data_ptr(), wq.data_ptr(), wk.data_ptr(), cos.data_ptr(), sin.data_ptr(),
            pos.data_ptr(), dqo.data_ptr(), dko.data_ptr(), dq.data_ptr(), dk.data_ptr(),
            dw.data_ptr(), dw.data_ptr() + 4 * dims[4], *dims, strides, float(eps),
            int(interleaved), code, ws.data_ptr(), ws.numel(), s)

    _run(dev, stream, call)
    return dq, dk, dw[0], dw[1]


def kv4_pool(n_pages: int, H: int, page_tokens: int, d_k: int, d_v: int, device="cuda"):
    """An empty pool of the 4-bit cache: uint8 [n_pages, H, page_tokens / 16, 9 (d_k + d_v)], 4.5
    bits a value.  The other kv4 functions read the sizes from its shape."""
    import torch
    if page_tokens % 16 or page_tokens < 16 or d_k not in (64, 128) or d_v not in (64, 128):
        raise ValueError("kv4_pool: page_tokens must be a multiple of 16, d_k and d_v 64 or 128")
    return torch.zeros((n_pages, H, page_tokens // 16, 9 * (d_k + d_v)), dtype=torch.uint8, device=device)


def _cache(what, pool, pages, B, d_k, device):
    """(n_pages, H, page_tokens, max_pages, d_v) of a pool and a page table."""
    import torch
    if pool.dim() != 4 or pool.dtype != torch.uint8 or not pool.is_contiguous() or pool.shape[3] % 9:
        raise ValueError(f"{what}: pool must be a contiguous uint8 tensor as kv4_pool makes it")
    if pool.device != device:
        raise ValueError(f"{what}: pool is on {pool.device}, not on {device}")
    if pages.dim() != 2:
        raise ValueError(f"{what}: pages must be [B, max_pages]")
    _flat(what, "pages", pages, torch.int32, (B, pages.shape[1]), device)
    d_v = pool.shape[3] // 9 - d_k
    if d_k not in (64, 128) or d_v not in (64, 128):
        raise ValueError(f"{what}: the pool's rows do not fit d_k = {d_k}")
    return pool.shape[0], pool.shape[1], 16 * pool.shape[2], pages.shape[1], d_v


def kv4_write(k, v, pool, pages, pos, stream=None) -> None:
    """Quantises keys [B, H, N, d_k] and values [B, H, N, d_v] into the pool (kv4_pool): token n of
    sequence b goes to position pos[b, n], that is to page pages[b, pos // page_tokens], place
    pos % page_tokens.  pages: int32 [B, max_pages]; pos: int32 [B, N], negative: not written."""
    import torch
    what = "kv4_write"
    strides = _heads(what, "k", k)
    B, H, N, d_k = k.shape
    strides += _heads(what, "v", v, like=k)
    n_pages, Hp, page, max_pages, d_v = _cache(what, pool, pages, B, d_k, k.device)
    if Hp != H or tuple(v.shape) != (B, H, N, d_v):
        raise ValueError(f"{what}: k {tuple(k.shape)} and v {tuple(v.shape)} do not fit the pool "
                         f"({Hp} heads, d_v = {d_v})")
    _flat(what, "pos", pos, torch.int32, (B, N), k.device)
    code = _code(what, k.dtype)
    _run(k.device, stream, lambda s: moa_kv4_write(
        k.data_ptr(), v.data_ptr(), pool.data_ptr(), pages.data_ptr(), pos.data_ptr(), B, H, N, d_k,
        d_v, n_pages, page, max_pages, strides, code, s))


def kv4_read(pool, pages, pos, d_k: int, dtype=None, out=None, stream=None):
    """(k, v): the cached rows at positions pos [B, N], widened to dtype (torch.bfloat16 by default):
    [B, H, N, d_k] and [B, H, N, d_v].  Negative positions give zeros."""
    import torch
    what = "kv4_read"
    if pos.dim() != 2 or not pos.is_cuda:
        raise ValueError(f"{what}: pos must be a CUDA [B, N] tensor")
    B, N = pos.shape
    n_pages, H, page, max_pages, d_v = _cache(what, pool, pages, B, d_k, pos.device)
    _flat(what, "pos", pos, torch.int32, (B, N), pos.device)
    if out is None:
        dtype = torch.bfloat16 if dtype is None else dtype
        k = torch.empty((B, H, N, d_k), dtype=dtype, device=pos.device)
        v = torch.empty((B, H, N, d_v), dtype=dtype, device=pos.device)
    else:
        k, v = out
        if k.device != pos.device or dtype is not None and dtype != k.dtype:
            raise ValueError(f"{what}: out has another device or dtype")
    strides = _heads(what, "k", k, None, (B, H, N, d_k)) + _heads(what, "v", v, k, (B, H, N, d_v))
    code = _code(what, k.dtype)
    _run(pos.device, stream, lambda s: moa_kv4_read(
        k.data_ptr(), v.data_ptr(), pool.data_ptr(), pages.data_ptr(), pos.data_ptr(), B, H, N, d_k,
        d_v, n_pages, page, max_pages, strides, code, s))
    return k, v


def kv4_attn(q, pool, pages, lens, max_len: int | None = None, scale: float | None = None,
             causal: bool = True, out=None, workspace=None, stream=None):
    """Attention of q [B, H_q, N, d_k] over each sequence's cached tokens: [B, H_q, N, d_v].

    lens: int32 [B] on the device, the tokens that each sequence has in the cache, the N queries
    being its last N tokens: with causal, query i sees the first lens[b] - N + i + 1 of them, else
    all.  A query that sees nothing gives zeros.  Query head j reads key head j // (H_q / H_k).
    max_len: an upper bound of lens known to the host (default: what the page table holds); the
    work is divided by it, so a close bound is faster."""
    return _attn("kv4_attn", q, pool, pages, lens, max_len, scale, causal, out, None, workspace, stream)


def kv4_attn_lse(q, pool, pages, lens, max_len: int | None = None, scale: float | None = None,
                 causal: bool = True, out=None, lse=None, workspace=None, stream=None):
    """(o, lse): kv4_attn's output and the float32 [B, H_q, N] natural logarithm of each row's sum of
    exponentials of scaled scores (-inf for a query that sees nothing)."""
    import torch
    if lse is None:
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    else:
        _flat("kv4_attn_lse", "lse", lse, torch.float32, q.shape[:3], q.device)
    return _attn("kv4_attn_lse", q, pool, pages, lens, max_len, scale, causal, out, lse, workspace, stream), lse


def _attn(what, q, pool, pages, lens, max_len, scale, causal, out, lse, workspace, stream):
    import torch
    strides = _heads(what, "q", q)
    B, Hq, N, d_k = q.shape
    dev = q.device
    n_pages, Hk, page, max_pages, d_v = _cache(what, pool, pages, B, d_k, dev)
    _flat(what, "lens", lens, torch.int32, (B,), dev)
    if max_len is None:
        max_len = max_pages * page
    if scale is None:
        scale = 1.0 / math.sqrt(d_k)
    if out is None:
        out = torch.empty((B, Hq, N, d_v), dtype=q.dtype, device=dev)
    strides += _heads(what, "out", out, q, (B, Hq, N, d_v))
    code = _code(what, q.dtype)

    def call(s):
        ws = workspace
        if ws is None:
            need = moa_kv4_attn_workspace_bytes(B, Hq, Hk, N, d_k, d_v, max_len, code)
            if need:
                ws = torch.empty(need, dtype=torch.uint8, device=dev)
        return moa_kv4_attn(
            q.data_ptr(), pool.data_ptr(), pages.data_ptr(), lens.data_ptr(), out.data_ptr(),
            None if lse is None else lse.data_ptr(), B, Hq, Hk, N, d_k, d_v, n_pages, page,
            max_pages, max_len, strides, float(scale), int(causal), code,
            None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), s)

    _run(dev, stream, call)
    return out
