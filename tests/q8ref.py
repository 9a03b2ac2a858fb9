"""Plain 64-bit forms of the normed appends, the 8-bit caches and decode over them, on the CPU
with numpy, and the tolerances the GPU tests hold the kernels to.

Tolerances count roundings: half a step is finfo.eps / 2 relative to the value (bf16 2^-8, e4m3
2^-4, fp32 2^-24), in e4m3 half of the smallest step, 2^-10, below 2^-6.
"""
from __future__ import annotations

import math

import numpy as np
import torch

BF16_HALF, E4M3_HALF, E4M3_TINY = 2.0 ** -8, 2.0 ** -4, 2.0 ** -10
MIN_EXP, MAX_EXP = -60, 119


def f64(t):
    return t.detach().to("cpu").to(torch.float32).numpy().astype(np.float64)


# every finite e4m3 value by its byte's low 7 bits: 4 exponent bits (bias 7), 3 fraction bits
E4M3 = np.array([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** (max(e, 1) - 7)
                 for e in range(16) for m in range(8)][:127])


def e4m3_round(x):
    """The nearest e4m3 number of every |x| <= 448, ties to the even byte, by search."""
    a = np.abs(x)
    hi = np.searchsorted(E4M3, a).clip(max=126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.copysign(E4M3[pick], x)


def exponent(amax):
    """Smallest e in [-60, 119] with amax <= 448 * 2^e."""
    e = np.full(np.shape(amax), MIN_EXP)
    for k in range(MIN_EXP, MAX_EXP):
        e = np.where(np.asarray(amax) > 448.0 * 2.0 ** k, k + 1, e)
    return e


def quantise(x):
    """x [..., d] -> (numbers [..., d], NaN where x is not finite; exponents [...])."""
    fin = np.isfinite(x)
    e = exponent(np.where(fin, np.abs(x), 0.0).max(axis=-1))
    y = np.where(fin, x, 0.0) / 2.0 ** e[..., None].astype(np.float64)
    return np.where(fin, e4m3_round(np.clip(y, -448.0, 448.0)), np.nan), e


def norm_rotate(x, weight, eps, pos, theta):
    """(result, bound of its fp32 error) of x [n, h, d] at positions pos [n], 64 bits.

    The kernel's fp32: a sum of d squares (each step 2^-24 of a positive sum: (d + 2) 2^-24 of
    it, half of that in its root), the root's and its product's roundings, and per number two
    products of weight, cos or sin (2^-23 off themselves) and input: within 2^-17 of
    |x_own w_own| + |x_other w_other|, over the root."""
    d = x.shape[-1]
    w = np.ones(d) if weight is None else weight
    rs = 1.0 if weight is None else 1.0 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    y = x * w * rs
    a = pos.astype(np.float64)[:, None, None] * theta
    lo, hi = y[..., : d // 2], y[..., d // 2:]
    with np.errstate(invalid="ignore"):  # (an infinity times 0)
        r = np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], axis=-1)
    m = np.abs(lo) + np.abs(hi)
    return r, 2.0 ** -17 * np.concatenate([m, m], axis=-1)


# ---- layouts: caches <-> tokens [B, h, T, d]

def dims(d):
    """[d/16, 16]: the dims of a pair-chunk's 16 numbers."""
    return np.arange(d).reshape(2, d // 16, 8).transpose(1, 0, 2).reshape(d // 16, 16)


def k_tokens(k):
    """[.., d/16, T, 16] -> [.., T, d] (any array)."""
    nc = k.shape[-3]
    out = np.empty(k.shape[:-3] + (k.shape[-2], 16 * nc), k.dtype)
    for c in range(nc):
        out[..., dims(16 * nc)[c]] = k[..., c, :, :]
    return out


BF16_SLOT = np.array([8 * (t // 4 % 2) + 4 * (t // 8) + t % 4 for t in range(16)])


def v_tokens(v, bf16):
    """[.., nb, d, 16] -> [.., 16 nb, d]; a bf16 block's tokens are permuted, an 8-bit one's not."""
    v = v[..., BF16_SLOT] if bf16 else v
    v = np.swapaxes(v, -1, -2)
    return v.reshape(v.shape[:-3] + (-1, v.shape[-1]))


def paged(x, table, b, tokens, T):
    """Rows of a token-major page pool [pages, h, page_tokens, ..] that row b's table names."""
    got = x[table[b, : -(-T // tokens)]]
    return np.concatenate(list(got), axis=1)[:, :T]


# ---- decode

def decode(q, k, v, q_pos, W, scale):
    """One row: q [h_q, d], k and v [h_kv, T, d]; (o, lse, bound of o's error, of lse's).

    Scores are fp32 sums of exact products: d + 8 roundings of 2^-24 of sum |q k| (the 8 for the
    scale, the maximum and the exponential, whose argument's rounding is 2^-24 of a number below
    2^7).  The probabilities' error is that of the scores and 2^-16 (two bf16 numbers, the sums),
    and goes into o through sum p |v|, twice with the normaliser; o is then rounded to bf16."""
    h_q, d = q.shape
    h_kv, T = k.shape[:2]
    G = h_q // h_kv
    n = min(T, q_pos + 1)
    o, lse = np.zeros((h_q, d)), np.full(h_q, -np.inf)
    o_err, lse_err = np.zeros((h_q, d)), np.zeros(h_q)
    if n == 0:
        return o, lse, o_err, lse_err
    z = q_pos - np.arange(n)
    keep = z[:, None] <= np.concatenate([W, W])[None, :]
    for h in range(h_q):
        kk, vv = np.where(keep, k[h // G, :n], 0.0), v[h // G, :n]
        s = kk @ q[h] * scale
        size = np.abs(kk) @ np.abs(q[h]) * scale
        m = s.max()
        p = np.exp(s - m)
        delta = (2.0 ** -24 * (d + 8) * size.max() + 2.0 ** -24 * 128)
        o[h] = p @ vv / p.sum()
        lse[h] = m + math.log(p.sum())
        o_err[h] = BF16_HALF * np.abs(o[h]) + (2 * delta + 2.0 ** -15) * (p @ np.abs(vv)) / p.sum() + 2.0 ** -126
        lse_err[h] = delta + 2.0 ** -16 + 2.0 ** -22 * abs(lse[h])
    return o, lse, o_err, lse_err


def thresholds(head_dim, base, k, theta=None):
    th = base ** (-2.0 * np.arange(head_dim // 2) / head_dim) if theta is None else np.asarray(theta)
    if math.isinf(k):
        return np.full(head_dim // 2, 2 ** 31 - 1)
    with np.errstate(divide="ignore"):
        return np.minimum(np.floor(k * 2 * math.pi / th), 2 ** 31 - 1).astype(np.int64)


def theta(head_dim, base):
    return base ** (-2.0 * np.arange(head_dim // 2) / head_dim)
