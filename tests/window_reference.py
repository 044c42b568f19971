"""Plain 64-bit implementations (numpy) of attention with a sliding window and first tokens that stay
visible, its gradients, and the paged 16- and 32-bit cache, with the bounds that their tests compare by.

Bounds, element by element, with u the half step of the type (bf16 2^-8, fp32 2^-24) and p the row's
softmax weights:

  scores   accumulate in fp32 over d_k products: each within e = (d_k + 8) 2^-24 scale
           max_j sum_c |q_c k_jc| of its value.  The exponents c s - m are formed in fp32 and the
           exponential instruction adds 2^-22: every weight is within w = 2 e + 2^-18 of its value, relative.
  outputs  w sum p |v| + n 2^-24 sum p |v| for the sums (n tokens, averaged over tiles and shares: 2^-15 of
           sum p |v|), weights rounded to bf16 once (u sum p |v|), the output once (u |o|).
  LSE      e + 2^-17 + 2^-20 |lse|.
  dV       the weights, now exp(s - LSE): w sum p |dO|; bf16 u of it; sums 2^-15; the output u |dV|.
  dS       p (<dO, v> - D): p times the fp32 error of the two dot products, (d_v + 8) 2^-24
           (sum |dO v| + sum |dO O|), and w |dS|; bf16 rounds it once (u |dS|); then dQ and dK are sums of dS k
           and dS q: those errors summed with |k|, |q|, 2^-15 of sum |dS| |k|, and u of the result.
"""
from __future__ import annotations

import numpy as np

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
SUMS = 2.0 ** -15
WEIGHT = 2.0 ** -18


def seen(N, T, length, window, sinks, causal=True):
    """[N, T]: which of T places each of the last N of `length` tokens sees."""
    p = length - N + np.arange(N)[:, None]
    j = np.arange(T)[None]
    see = (j <= p) if causal else (j < length) & (p == p)
    if window:
        see = see & ((j > p - window) | (j < sinks))
    return see


def _weights(q, k, see, scale):
    """(p, lse, size) of one head: q [N, d], k [T, d]; what is hidden has no influence."""
    with np.errstate(invalid="ignore"):
        s = np.where(see, scale * (q @ k.T), -np.inf)
        size = np.where(see, abs(scale) * (np.abs(q) @ np.abs(k).T), 0.0)
        m = s.max(axis=1, initial=-np.inf, keepdims=True)
        p = np.where(see, np.exp(s - np.where(m == -np.inf, 0.0, m)), 0.0)
    total = p.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (m + np.log(total))[:, 0]
    return p / np.where(total == 0, 1.0, total), lse, size.max(axis=1, initial=0.0)


def attention(q, k, v, length, window, sinks, scale, causal=True):
    """One sequence: q [H_q, N, d_k], k [H_k, T, d_k], v [H_k, T, d_v].  (o, lse, sum p |v|, size)."""
    Hq, N, dk = q.shape
    Hk, T, dv = v.shape
    see = seen(N, T, length, window, sinks, causal)
    o, av = np.zeros((Hq, N, dv)), np.zeros((Hq, N, dv))
    lse, size = np.zeros((Hq, N)), np.zeros((Hq, N))
    used = see.any(axis=0)
    for h in range(Hq):
        kk, vv = k[h // (Hq // Hk)], v[h // (Hq // Hk)]
        # what no row sees may hold anything
        kk, vv = np.where(used[:, None], kk, 0.0), np.where(used[:, None], vv, 0.0)
        p, lse[h], size[h] = _weights(q[h], kk, see, scale)
        o[h], av[h] = p @ vv, p @ np.abs(vv)
    return o, lse, av, size


def out_bound(o, av, size, dk, dtype):
    e = (dk + 8) * 2.0 ** -24 * size[..., None]
    u = HALF[dtype]
    return (2 * e + WEIGHT + SUMS + (u if dtype == "bf16" else 0.0)) * av * 1.02 + u * np.abs(o) * 1.02 + 1e-30


def lse_bound(lse, size, dk):
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(lse), (dk + 8) * 2.0 ** -24 * size + 2.0 ** -17 + 2.0 ** -20 * np.abs(lse), 0.0)


def gradients(q, k, v, o, lse, do, window, sinks, scale, dtype):
    """One sequence, from the o and lse that are given: ((dq, dk, dv), their bounds)."""
    Hq, N, dk = q.shape
    Hk, T, dv = v.shape
    G, u = Hq // Hk, HALF[dtype]
    ub = u if dtype == "bf16" else 0.0
    see = seen(N, T, T, window, sinks)
    out = [np.zeros_like(x) for x in (q, k, v)]
    err = [np.zeros_like(x) for x in (q, k, v)]
    for h in range(Hq):
        kk, vv = k[h // G], v[h // G]
        base = np.where(np.isfinite(lse[h]), lse[h], 0.0)[:, None]
        p = np.where(see, np.exp(np.where(see, scale * (q[h] @ kk.T) - base, -np.inf)), 0.0)
        size = np.where(see, abs(scale) * (np.abs(q[h]) @ np.abs(kk).T), 0.0).max(axis=1, initial=0.0)
        w = (2 * (dk + 8) * 2.0 ** -24 * size + WEIGHT + 2.0 ** -22 * np.abs(base[:, 0]))[:, None]
        dp = do[h] @ vv.T
        delta = (do[h] * o[h]).sum(axis=1, keepdims=True)
        ds = p * (dp - delta)
        dot = (dv + 8) * 2.0 ** -24 * (np.abs(do[h]) @ np.abs(vv).T + (np.abs(do[h]) * np.abs(o[h])).sum(axis=1, keepdims=True))
        eds = (w + ub) * np.abs(ds) + p * dot * 1.02
        out[0][h] = scale * ds @ kk
        err[0][h] = abs(scale) * ((eds + SUMS * np.abs(ds)) @ np.abs(kk))
        out[1][h // G] += scale * ds.T @ q[h]
        err[1][h // G] += abs(scale) * ((eds + SUMS * np.abs(ds)).T @ np.abs(q[h]))
        out[2][h // G] += p.T @ do[h]
        err[2][h // G] += ((w + ub + SUMS) * p).T @ np.abs(do[h])
    return out, [1.02 * e + 1.02 * u * np.abs(x) + 1e-30 for e, x in zip(err, out)]


def rotate(x, cos, sin, pos, interleaved):
    """x [B, H, N, d], pos [B, N] (negative: unchanged), cos and sin [P, d_rot / 2]."""
    half = cos.shape[1]
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    c, s = cos[np.maximum(pos, 0)][:, None], sin[np.maximum(pos, 0)][:, None]
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return np.where((pos >= 0)[:, None, :, None], y, x)


def rotate_bound(x, cos, interleaved, dtype):
    """Two products and a sum in fp32, rounded once: of the pair's magnitudes."""
    half = cos.shape[1]
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    pair = np.abs(x[..., a]) + np.abs(x[..., b])
    e = np.zeros_like(x)
    e[..., a] = e[..., b] = pair * (4 * 2.0 ** -24 + HALF[dtype])
    return e * 1.02
