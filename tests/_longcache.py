"""Plain forms of the calls for long caches (4-bit cache, windows with visible
first rows, pages) and the tolerances of their tests, in numpy.

Tolerances (derived from the arithmetic, before the first run):

* a row in 4 bits: the rotated value y is good to t = 2^-20 mag (|x| + |y|)
  (tests/_prompt.py) and the division and the scale's quotient add 2^-23 of
  the value, so a scale is one whose distance from max|y| / 6 exceeds the
  nearest one's by at most twice that, and a code, given the scale, one whose
  distance from y does;  values that are not rotated and have 8 significant
  bits are exact, ties included;
* attention by codes: scores as in tests/_prompt.py (q in fp16 adds 2^-25 of
  its row's largest component to each, at most 2^-21 scale |q| |k| in a
  score, below the 2^-16 there); a probability is rounded to fp16: 2^-11 of
  it, or where it is below 2^-14 of the reference, of which the sum holds at
  least one, 2^-25: (A 2^-11 + |r| 2^-8) (1 + 2^-7) + (A + |r|) (e^(2 Delta) -
  1 + (tiles + 70) 2^-23) + N 2^-25 max|v|;
* attention through the image: its keys and values are exact in bf16, so the
  tolerance is that of the bf16 (fp32) call.
"""
import math

import numpy as np

from tests import _prompt

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# scale of byte i < 127: 3 bits of fraction below 4 of exponent
SCALES = np.array([(i & 7) * 2.0 ** -9 if i < 8 else (8 + (i & 7)) * 2.0 ** ((i >> 3) - 10) for i in range(127)])


def decode(codes, scales, unit=1.0):
    """codes [..][d/2], scales [..][d/16] uint8 -> values [..][d] float64."""
    both = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.where(both >= 8, -1.0, 1.0) * LEVELS[both & 7]
    s = np.where(scales < 127, SCALES[np.minimum(scales, 126)], np.nan)
    return (v.reshape(*v.shape[:-1], -1, 16) * s[..., None]).reshape(v.shape) * unit


def encode(y):
    """The nearest scales and codes of y [..][d] (ties to even), as values."""
    g = y.reshape(*y.shape[:-1], -1, 16)
    a = np.abs(g).max(-1) / 6
    i = np.clip(np.searchsorted(SCALES, a), 1, 126)
    lo, hi = a - SCALES[i - 1], SCALES[i] - a
    k = np.where((lo < hi) | ((lo == hi) & (i % 2 == 1)), i - 1, i)
    s = SCALES[np.maximum(k, 1)][..., None]
    q = np.abs(g) / s
    j = np.clip(np.searchsorted(LEVELS, q), 1, 7)
    lo, hi = q - LEVELS[j - 1], LEVELS[j] - q
    c = np.where((lo < hi) | ((lo == hi) & (j % 2 == 1)), j - 1, j)
    return (np.sign(g) * LEVELS[c] * s).reshape(y.shape)


def check_codes(codes, scales, y, t, unit=1.0):
    """Codes and scales are nearest to y / unit, whose entries are good to t."""
    g, t = (x.reshape(*x.shape[:-1], -1, 16) / unit for x in (y, t))
    t = t + 2.0 ** -23 * np.abs(g)
    assert (scales < 127).all() and (scales >= 1).all()
    s, a = SCALES[scales], np.abs(g).max(-1) / 6
    slack = 2 * t.max(-1) / 6 + 2.0 ** -22 * a
    best = np.abs(a[..., None] - SCALES[1:]).min(-1)
    assert np.all(np.abs(s - a) <= best + slack)
    v = decode(codes, scales).reshape(g.shape)
    q = np.abs(g)[..., None] - LEVELS * s[..., None, None]
    assert np.all(np.abs(v - g) <= np.abs(q).min(-1) + 2 * t)
    assert np.all((np.sign(v) == np.sign(g)) | (v == 0) | (np.abs(g) <= t))


def visible(n, C, i, block, window, start, sinks):
    """Row numbers that token i of a chunk of C after n cached rows sees."""
    lo, hi = _prompt.visible(n, C, i, block, window, start)
    first = max(0, start)
    seen = set(range(lo, hi)) | (set(range(first, min(first + sinks, hi))) if window else set())
    return np.array(sorted(seen), dtype=int)


def attention(q, k_rows, v_rows, n, C, scale, block=1, window=0, start=0, sinks=0):
    """One sequence, as tests/_prompt.py's attention."""
    Hq, d = q.shape[1:]
    g = Hq // k_rows.shape[1]
    out, absv = np.zeros((C, Hq, d)), np.zeros((C, Hq, d))
    lse = np.full((C, Hq), -np.inf)
    for i in range(C):
        rows = visible(n, C, i, block, window, start, sinks)
        if not len(rows):
            continue
        k, v = k_rows[rows], v_rows[rows]
        for h in range(Hq):
            x = k[:, h // g] @ q[i, h] * scale
            m = x.max()
            w = np.exp(x - m)
            z = w.sum()
            out[i, h], absv[i, h] = w @ v[:, h // g] / z, w @ np.abs(v[:, h // g]) / z
            lse[i, h] = m + math.log(z)
    return out, lse, absv


def q4_tolerance(out, absv, qk, N, vmax):
    delta = 2.0 ** -16 * qk + 2.0 ** -22 + 2.0 ** -24 * math.log(2) * (2 / math.log(2) * qk + 8)
    return ((absv * 2.0 ** -11 + np.abs(out) * 2.0 ** -8) * (1 + 2.0 ** -7)
            + (absv + np.abs(out)) * (math.expm1(2 * delta) + (N // 128 + 72) * 2.0 ** -23)
            + N * 2.0 ** -25 * vmax + 1e-12)


class Pool:
    """Tables, counts and contents of a pool, with the calls as their
    definitions have them.  Contents: one number a page."""

    def __init__(self, Bt, max_pages, num_pages, P):
        self.table = np.full((Bt, max_pages), -1, dtype=np.int64)
        self.refs = np.zeros(num_pages, dtype=np.int64)
        self.lens = np.zeros(Bt, dtype=np.int64)
        self.data = np.arange(num_pages, dtype=np.int64) * 7 + 3
        self.P = P

    def _free(self):
        return np.flatnonzero(self.refs == 0)

    def extend(self, add):
        want = [(b, k) for b in range(len(add)) if add[b] > 0
                for k in range(self.lens[b] // self.P, -(-(self.lens[b] + add[b]) // self.P)) if self.table[b, k] < 0]
        free = self._free()
        if len(free) < len(want):
            return False
        for (b, k), p in zip(want, free):
            self.table[b, k] = p
            self.refs[p] = 1
        return True

    def release(self, seq, first, last):
        for b, f, l in zip(seq, first, last):
            for k in range(self.table.shape[1]):
                if k * self.P >= f and (k + 1) * self.P <= l and self.table[b, k] >= 0:
                    self.refs[self.table[b, k]] -= 1
                    self.table[b, k] = -1

    def fork(self, src, dst):
        free, want = self._free(), 0
        pairs = [(s, d) for s, d in zip(src, dst)
                 if 0 <= min(s, d) and max(s, d) < len(self.lens) and list(dst).count(d) == 1 and d not in src]
        part = [self.lens[s] % self.P > 0 and self.table[s, self.lens[s] // self.P] >= 0 for s, d in pairs]
        if len(free) < sum(part):
            return False
        for (s, d), p in zip(pairs, part):
            n, whole = self.lens[s], self.lens[s] // self.P
            row = np.full(self.table.shape[1], -1)
            row[:whole] = self.table[s, :whole]
            if p:
                row[whole] = free[want]
                self.data[free[want]] = self.data[self.table[s, whole]]
                want += 1
            np.add.at(self.refs, row[row >= 0], 1)
            np.add.at(self.refs, self.table[d][self.table[d] >= 0], -1)
            self.table[d], self.lens[d] = row, n
        return True

    def compact(self):
        live = int((self.refs > 0).sum())
        holes, out = np.flatnonzero(self.refs[:live] == 0), live + np.flatnonzero(self.refs[live:] > 0)
        to = np.arange(len(self.refs))
        to[out] = holes
        self.data[holes] = self.data[out]
        self.refs[holes] = self.refs[out]
        self.refs[out] = 0
        self.table = np.where(self.table >= 0, to[self.table], -1)
        return live
