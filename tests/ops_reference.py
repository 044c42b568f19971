"""Plain 64-bit implementations (numpy) of the operators around attention, written from their
definitions feature by feature: the references of test_norm_rope.py and test_kv4.py."""
from __future__ import annotations

import math

import numpy as np

from paper_2606_07713_gb300 import inputs as I


def bf16(a):
    """float64 values rounded to bf16 (ties to even), as float64."""
    return I.bf16_bits_to_f32(I.f32_to_bf16_bits(np.asarray(a, dtype=np.float32))).astype(np.float64)


# -- norm and rotation ----------------------------------------------------------------------------
def _pairs(d_rot, interleaved):
    i = np.arange(d_rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + d_rot // 2)


def _rotate(u, c, s, interleaved):
    a, b = _pairs(2 * c.shape[-1], interleaved)
    y = u.copy()
    y[..., a] = u[..., a] * c - u[..., b] * s
    y[..., b] = u[..., b] * c + u[..., a] * s
    return y


def norm_rope(x, w, cos, sin, pos, eps, interleaved):
    """x [B, H, N, d], w [d], cos/sin [P, d_rot/2], pos [B, N] (negative: zeros)."""
    live = (pos >= 0)[:, None, :, None]
    at = np.maximum(pos, 0)
    c, s = cos[at][:, None], sin[at][:, None]
    r = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    return np.where(live, _rotate(x * r * w, c, s, interleaved), 0.0)


def norm_rope_bwd(x, w, cos, sin, pos, g, eps, interleaved):
    """(dx, dw, sum over rows of |t x r|)."""
    live = (pos >= 0)[:, None, :, None]
    at = np.maximum(pos, 0)
    c, s = cos[at][:, None], sin[at][:, None]
    r = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    t = np.where(live, _rotate(g, c, -s, interleaved), 0.0)
    n = x * r
    dx = r * (w * t - n * np.mean(w * t * n, axis=-1, keepdims=True))
    return dx, np.sum(t * n, axis=(0, 1, 2)), np.sum(np.abs(t * n), axis=(0, 1, 2))


# -- the 4-bit cache ------------------------------------------------------------------------------
def quantise(x):
    """(codes int [..., d], scales float64 [..., d/32]) of x, in the float32 operations that the
    definition rounds by: s = bf16(max|x| / 7), code = rint(x / s)."""
    x = np.asarray(x, dtype=np.float32)
    y = x.reshape(*x.shape[:-1], -1, 32)
    with np.errstate(all="ignore"):
        m = np.max(np.abs(y), axis=-1, keepdims=True)          # NaN if any is
        s = bf16(np.where(np.isfinite(m), m / np.float32(7.0), np.float32(0))).astype(np.float32)
        c = np.clip(np.rint(y / s), -7, 7)
    c = np.where(np.isfinite(m) & (s > 0), c, 0.0)
    s = np.where(np.isfinite(m), s, np.float32(np.nan))
    return c.reshape(x.shape).astype(np.int64), s[..., 0].astype(np.float64)


def values(codes, scales):
    return codes * np.repeat(scales, 32, axis=-1)


def code_place(d_k, d_v, token, feature, value):
    """(byte, high nibble) in a 16-token block of the code of one feature of one token."""
    g, e = feature // 32, feature % 32
    if value:
        word = ((token // 8 * 8 + e // 4) * 4 + token % 8 // 2) * (d_v // 32) + g
        nibble = 4 * (token % 2) + e % 4
        base = 8 * d_k
    else:
        word = (token * 4 + e // 8) * (d_k // 32) + g
        nibble = 4 * (e % 2) + e % 8 // 2
        base = 0
    return base + 4 * word + nibble // 2, nibble % 2


def scale_place(d_k, d_v, token, group, value):
    base = 8 * (d_k + d_v) + (d_k if value else 0)
    return base + 2 * (token * ((d_v if value else d_k) // 32) + group)


def unpack(block, d_k, d_v):
    """(k codes, k scales, v codes, v scales) of blocks [..., bytes]: codes [..., 16, d]."""
    out = []
    block = np.asarray(block)
    for d, value in ((d_k, False), (d_v, True)):
        codes = np.zeros(block.shape[:-1] + (16, d), dtype=np.int64)
        scales = np.zeros(block.shape[:-1] + (16, d // 32))
        for token in range(16):
            for f in range(d):
                byte, high = code_place(d_k, d_v, token, f, value)
                codes[..., token, f] = ((block[..., byte] >> (4 * high)) & 15).astype(np.int64) - 8
            for g in range(d // 32):
                at = scale_place(d_k, d_v, token, g, value)
                bits = block[..., at].astype(np.uint16) | block[..., at + 1].astype(np.uint16) << 8
                scales[..., token, g] = I.bf16_bits_to_f32(bits)
        out += [codes, scales]
    return out


def pack(kc, ks, vc, vs):
    """Blocks [..., bytes] (uint8) of codes [..., 16, d] and scales [..., 16, d/32]."""
    d_k, d_v = kc.shape[-1], vc.shape[-1]
    block = np.zeros(kc.shape[:-2] + (9 * (d_k + d_v),), dtype=np.uint8)
    for codes, scales, value in ((kc, ks, False), (vc, vs, True)):
        for token in range(16):
            for f in range(codes.shape[-1]):
                byte, high = code_place(d_k, d_v, token, f, value)
                block[..., byte] |= ((codes[..., token, f] + 8) << (4 * high)).astype(np.uint8)
            for g in range(scales.shape[-1]):
                at = scale_place(d_k, d_v, token, g, value)
                bits = I.f32_to_bf16_bits(scales[..., token, g].astype(np.float32))
                block[..., at], block[..., at + 1] = (bits & 255).astype(np.uint8), (bits >> 8).astype(np.uint8)
    return block


def attention(q, k, v, length, scale, causal):
    """One sequence.  q [H_q, N, d_k], k [H_k, T, d_k], v [H_k, T, d_v] (T >= length): (o, lse,
    sum_j p_j |v_j|, scale * max_j sum_c |q_c k_jc| over visible keys)."""
    Hq, N, _ = q.shape
    G = Hq // k.shape[0]
    o = np.zeros((Hq, N, v.shape[-1]))
    av, lse, size = np.zeros_like(o), np.full((Hq, N), -np.inf), np.zeros((Hq, N))
    for h in range(Hq):
        for i in range(N):
            n = length - N + i + 1 if causal else length
            if n <= 0:
                continue
            kk, vv = k[h // G, :n], v[h // G, :n]
            s = scale * (kk @ q[h, i])
            m = s.max()
            p = np.exp(s - m)
            lse[h, i] = m + math.log(p.sum())
            p /= p.sum()
            o[h, i], av[h, i] = p @ vv, p @ np.abs(vv)
            size[h, i] = abs(scale) * (np.abs(kk) @ np.abs(q[h, i])).max()
    return o, lse, av, size


def attention_dense(q, k, v, length, scale, causal):
    """attention() for many rows at once (one sequence, the same results)."""
    Hq, N, _ = q.shape
    G = Hq // k.shape[0]
    seen = np.arange(length)[None] < (length - N + 1 + np.arange(N)[:, None] if causal else np.full((N, 1), length))
    out = []
    for h in range(Hq):
        kk, vv = k[h // G, :length], v[h // G, :length]
        s = np.where(seen, scale * (q[h] @ kk.T), -np.inf)
        m = s.max(axis=1, initial=-np.inf, keepdims=True)
        p = np.where(seen, np.exp(s - np.where(np.isfinite(m), m, 0.0)), 0.0)
        total = p.sum(axis=1, keepdims=True)
        with np.errstate(divide="ignore"):
            lse = (m + np.log(total))[:, 0]
        p /= np.where(total == 0, 1.0, total)
        size = np.where(seen, abs(scale) * (np.abs(q[h]) @ np.abs(kk).T), 0.0).max(axis=1, initial=0.0)
        out.append((p @ vv, lse, p @ np.abs(vv), size))
    return [np.stack(x) for x in zip(*out)]
