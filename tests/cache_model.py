"""Plain 64-bit model of the paged 8-bit cache, of attention over it and of rotary positions
(test infrastructure; shares nothing with the library)."""
import math

import numpy as np
import torch

E4M3 = np.array([(-1.0 if c & 128 else 1.0) * (
    ((8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10)) if c >> 3 & 15 else (c & 7) * 2.0 ** -9)
    for c in range(256)])
E4M3[[127, 255]] = np.nan


def round8(x):
    """Nearest e4m3 number, ties to even, saturating at 448."""
    x = np.clip(np.asarray(x, np.float64), -448.0, 448.0)
    _, e = np.frexp(x)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.rint(x / step) * step


def scale_of(amax):
    """Smallest power of two s with amax / s <= 448, its exponent within [-100, 120]."""
    e = -100
    if amax > 0:
        e = math.ceil(math.log2(amax / 448.0))
        e += amax > 448.0 * 2.0 ** e
        e -= amax <= 448.0 * 2.0 ** (e - 1)
    return 2.0 ** min(max(e, -100), 120)


class Sequence:
    """Keys or values of one sequence: values [n, Hkv, d] and one scale per (page, head)."""

    def __init__(self, page, Hkv, d):
        self.page, self.x, self.scale = page, np.zeros((0, Hkv, d)), np.zeros((0, Hkv))

    def copy(self):
        c = Sequence(self.page, 1, 1)
        c.x, c.scale = self.x.copy(), self.scale.copy()
        return c

    def append(self, new):
        new = np.asarray(new, np.float64)
        while len(new):
            n, G = len(self.x), self.page
            take = min(len(new), G - n % G)
            part, new = new[:take], new[take:]
            for h in range(part.shape[1]):
                s = scale_of(np.abs(part[:, h]).max())
                if n % G:
                    s = max(s, self.scale[-1, h])
                    old = self.x[n - n % G:, h]
                    old[:] = round8(old / s) * s
                    self.scale[-1, h] = s
                elif h == 0:
                    self.scale = np.concatenate([self.scale, np.zeros((1, part.shape[1]))])
                self.scale[-1, h] = s
            s = self.scale[-1][None, :, None]
            # Nothing rounds up past float32: 256 * 2^120 is the first number that would.
            most = np.where(s == 2.0 ** 120, 240.0, 448.0)
            self.x = np.concatenate([self.x, round8(np.clip(part / s, -most, most)) * s])

    def keep(self, start, span, kept):
        """Only the tokens outside the span and the listed ones of it."""
        kept = list(kept)
        if len(kept) == span:
            return
        first = next((i for i, v in enumerate(kept) if v != i), len(kept))
        G = self.page
        f = (start + first) // G
        src = list(range(start)) + [start + v for v in kept] + list(range(start + span, len(self.x)))
        x, scale = self.x[src], self.scale[:f]
        for p in range(f, -(-len(src) // G)):
            blk = x[p * G:(p + 1) * G]
            s = np.array([scale_of(np.abs(blk[:, h]).max()) for h in range(blk.shape[1])])
            blk[:] = round8(blk / s[None, :, None]) * s[None, :, None]
            scale = np.concatenate([scale, s[None]])
        self.x, self.scale = x, scale


def attention(q, k, v, causal, scale=None):
    """q [T, H, d], k and v [L, Hkv, d] in float64; rows are the last T of L tokens.
    Outputs, natural-log normalisers, and sum_j p_j |v_j| (what errors of p scale with)."""
    T, H, d = q.shape
    L, Hkv = k.shape[0], k.shape[1]
    scale = 1.0 / math.sqrt(d) if not scale else scale
    out, lse, mag = np.zeros((T, H, d)), np.full((T, H), -np.inf), np.zeros((T, H, d))
    for h in range(H):
        g = h // (H // Hkv)
        s = q[:, h] @ k[:, g].T * scale
        if causal:
            s[np.arange(L)[None, :] > (L - T + np.arange(T))[:, None]] = -np.inf
        for t in range(T):
            if L == 0 or np.isneginf(s[t].max()):
                continue
            m = s[t].max()
            p = np.exp(s[t] - m)
            lse[t, h] = m + math.log(p.sum())
            p /= p.sum()
            out[t, h], mag[t, h] = p @ v[:, g], p @ np.abs(v[:, g])
    return out, lse, mag


def check_attention(got, lse, q, k, v, causal, scale=None):
    """Outputs within: half a bf16 step of the value; 2^-12 (a probability rounded to f16)
    and the error of the logits (f32 sums of d exact products, twice: numerator and sum) of
    sum p |v|; and, for values far below the largest, half of f16's smallest step (2^-25)
    relative to twice the largest magnitude."""
    want, wl, mag = attention(q, k, v, causal, scale)
    d = q.shape[-1]
    if len(k):
        big = np.abs(q).sum(-1).max() * np.abs(k).max() * (scale or 1 / math.sqrt(d))
    else:
        big = 0.0
    delta = (d + 8) * 2.0 ** -24 * big
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -12 + 2 * delta + len(k) * 2.0 ** -24 + 2.0 ** -20) * mag
    tol += 2.0 ** -24 * (np.abs(v).max() if len(v) else 0.0) + 1e-38
    bad = np.abs(got - want) > tol
    assert not bad.any(), "out: worst %g of its bound" % (np.abs(got - want) / tol).max()
    if lse is not None:
        fin = np.isfinite(wl)
        assert np.array_equal(fin, np.isfinite(lse)) and np.all(lse[~fin] == -np.inf)
        tol = delta + 2.0 ** -22 * np.abs(wl[fin]) + len(k) * 2.0 ** -24 + 1e-6
        assert np.all(np.abs(lse[fin] - wl[fin]) <= tol), np.abs(lse[fin] - wl[fin]).max()


def turned(x, pos, axis, freq, adjacent, inverse):
    """x [rows, heads, d] float64, pos [rows, axes] ints; angles reduced in longdouble."""
    n = len(freq)
    a = np.asarray(pos, np.longdouble)[:, axis] * np.asarray(freq, np.longdouble)
    a = np.fmod(a, 2 * np.longdouble("3.14159265358979323846264338327950288"))
    c, s = np.cos(a).astype(np.float64)[:, None], np.sin(a).astype(np.float64)[:, None]
    s = -s if inverse else s
    i = np.arange(n)
    u, w = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
    y = x.copy()
    y[..., u], y[..., w] = x[..., u] * c - x[..., w] * s, x[..., u] * s + x[..., w] * c
    return y


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()
