"""Plain 64-bit forms of the prompt calls (rotary append, chunk attention,
sampling) and the tolerances of their tests, in numpy.

Tolerances (all derived from the arithmetic, before the first run):

* rotation: x c - y s with c, s correct to 2^-22 (a 32-bit angle of 2^-31
  half turns rounded to fp32, sincospi's 2 ulp, the magnitude's rounding) and
  three fp32 roundings: |g - r| <= 2^-20 mag (|x| + |y|), plus 2^-8 |r| where
  the result is rounded to bf16 (8 significant bits);
* attention: tests/_gpu.py's bound, (A + |r|) (u (1 + 2^-7) + e^(2 Delta) - 1
  + (tiles + 70) 2^-23) with A = sum p |v|, u = 2^-8 for bf16 and 0 for fp32
  (no rounding of P), Delta = scale |q| |k| 2^-16 + 2^-22 + 2^-24 ln 2 (2
  log2(e) scale |q| |k| + 8) bounding the error of a score; the fp32 kernel
  adds up N weights and products in fp32, 2^-23 (N + 70) in place of the tiles;
* log-sum-exp: Delta + 2^-21 (1 + |lse|) + (N + 70) 2^-24.
"""
import math

import numpy as np

U_BF16 = 2.0 ** -8


def frequencies(rot, theta, scaling="none", factor=1.0, context=0, beta_fast=32.0, beta_slow=1.0):
    i = np.arange(rot // 2)
    base = theta * factor ** (rot / (rot - 2)) if scaling == "ntk" else theta
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":
        rho = context * f / (2 * math.pi)
        g = np.clip((rho - beta_slow) / (beta_fast - beta_slow), 0, 1)
        return (1 - g) * f / factor + g * f, 0.1 * math.log(factor) + 1
    return f, 1.0


def rotate(x, pos, layout, rot, freq):
    """x [T][H][d] float64 (exact values), pos [T]; returns the rotated rows
    and |x| + |y| of each component's pair (0 where nothing turns)."""
    f, mag = freq
    # whole turns are taken off the integer position times the frequency in
    # extended precision, so that the reference is good at 2^30 too
    ang = np.asarray(pos, dtype=np.longdouble)[:, None] * np.asarray(f, dtype=np.longdouble)
    two_pi = np.longdouble("6.283185307179586476925286766559005768")
    ang = np.asarray(ang - two_pi * np.floor(ang / two_pi), dtype=np.float64)
    c, s = np.cos(ang)[:, None] * mag, np.sin(ang)[:, None] * mag
    y = np.array(x, dtype=np.float64)
    size = np.zeros_like(y)
    a, b = ((slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half"
            else (slice(0, rot, 2), slice(1, rot, 2)))
    u, v = x[..., a], x[..., b]
    y[..., a], y[..., b] = u * c - v * s, u * s + v * c
    size[..., a] = size[..., b] = (np.abs(u) + np.abs(v)) * mag
    return y, size


def rope_tolerance(r, size, bf16):
    return 2.0 ** -20 * size + (U_BF16 * np.abs(r) * (size > 0) if bf16 else 0.0) + 1e-30


def visible(n, C, i, block, window, start):
    """[lo, hi) of token i of a chunk of C after n cached rows."""
    N, p = n + C, n + i
    hi = min(N, (p // block + 1) * block) if block else N
    lo = max(0, start, p + 1 - window if window else 0)
    return lo, hi


def attention(q, k_rows, v_rows, n, C, scale, block=1, window=0, start=0):
    """One sequence: q [C][Hq][d], k_rows / v_rows [N][Hkv][d] float64 (rows
    that nobody sees may hold anything).  Returns out, lse, A."""
    Hq, d = q.shape[1:]
    g = Hq // k_rows.shape[1]
    out = np.zeros((C, Hq, d))
    absv = np.zeros((C, Hq, d))
    lse = np.full((C, Hq), -np.inf)
    for i in range(C):
        lo, hi = visible(n, C, i, block, window, start)
        if lo >= hi:
            continue
        for h in range(Hq):
            x = k_rows[lo:hi, h // g] @ q[i, h] * scale
            m = x.max()
            w = np.exp(x - m)
            z = w.sum()
            out[i, h] = w @ v_rows[lo:hi, h // g] / z
            absv[i, h] = w @ np.abs(v_rows[lo:hi, h // g]) / z
            lse[i, h] = m + math.log(z)
    return out, lse, absv


def attention_tolerance(out, absv, qk, N, bf16):
    delta = 2.0 ** -16 * qk + 2.0 ** -22 + 2.0 ** -24 * math.log(2) * (2 / math.log(2) * qk + 8)
    steps = (N // 128 + 2 + 70) if bf16 else (N + 70)
    u = U_BF16 * (1 + 2.0 ** -7) if bf16 else 0.0
    return (absv + np.abs(out)) * (u + math.expm1(2 * delta) + steps * 2.0 ** -23) + 1e-12


def lse_tolerance(lse, qk, N):
    delta = 2.0 ** -16 * qk + 2.0 ** -22 + 2.0 ** -24 * math.log(2) * (2 / math.log(2) * qk + 8)
    return delta + 2.0 ** -21 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0))) + (N + 70) * 2.0 ** -24


# ---------------------------------------------------------------- sampling
def order_of(x):
    """Indices by falling value, ties by rising index; -inf and NaN left out."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, dtype=np.float64))
    idx = np.lexsort((np.arange(len(x)), -x))
    return idx[np.isfinite(x[idx]) | (x[idx] > 0)], x


def sample_row(x, u, T=1.0, k=0, p=1.0, min_p=0.0):
    """token, kept indices (in the order), log-probabilities of the kept."""
    idx, x = order_of(x)
    if T == 0:
        k, T = 1, 1.0
    if k >= 1:
        idx = idx[:k]
    with np.errstate(invalid="ignore"):
        lw = np.where(x[idx] == x[idx[0]], 0.0, (x[idx] - x[idx[0]]) / T)
    w = np.exp(lw)
    if p < 1:
        c = np.cumsum(w)
        n = int((c < max(p, 0.0) * c[-1]).sum()) + 1
        idx, w, lw = idx[:n], w[:n], lw[:n]
    if min_p > 0:
        keep = w >= min(min_p, 1.0)
        idx, w, lw = idx[keep], w[keep], lw[keep]
    by = np.argsort(idx)
    c = np.cumsum(w[by])
    j = min(int((c <= u * c[-1]).sum()), len(c) - 1)
    return int(idx[by[j]]), idx, lw - math.log(w.sum())


def settle(x, u, T=1.0, k=0, p=1.0, min_p=0.0):
    """u, p and min_p moved to the middle of the intervals in which they give
    the same result, so that no test hangs on the last bit of a sum."""
    idx, xx = order_of(x)
    if T == 0:
        return u, p, min_p
    if k >= 1:
        idx = idx[:k]
    w = np.exp(np.where(xx[idx] == xx[idx[0]], 0.0, (xx[idx] - xx[idx[0]]) / T))
    if 0 < p < 1:
        c = np.cumsum(w)
        n = int((c < p * c[-1]).sum())
        p = float((c[n] - 0.5 * w[n]) / c[-1])
        idx, w = idx[:n + 1], w[:n + 1]
    if min_p > 0:
        n = int((w >= min(min_p, 1.0)).sum())
        if n < len(w) and w[n] > 0:
            min_p = math.sqrt(w[n - 1] * w[n])
        idx, w = idx[:n], w[:n]
    by = np.argsort(idx)
    c = np.cumsum(w[by])
    j = min(int((c <= u * c[-1]).sum()), len(c) - 1)
    u = float((c[j] - 0.5 * w[by[j]]) / c[-1])
    return min(u, 1 - 2.0 ** -24), p, min_p
