"""A stricter comparison of attention over the 8-bit cache than cache_model's (test
infrastructure; shares nothing with the library): nothing that is not a number passes, and
what a row may be off by follows from the keys that this row sees."""
import math

import numpy as np


def attention(q, k, v, scales, causal, scale=None):
    """q [T, H, d], k and v [L, Hkv, d] in float64, scales [L, Hkv] the block scale of every
    key's values; rows are the last T of L tokens.  A dict of arrays: out [T, H, d], lse [T, H]
    (natural log), mag = sum_j p_j |v_j|, size = max_j |q| |k_j| scale (what errors of a logit
    scale with), top = max_j p_j scales_j (the row's largest weight), codes = sum_j |v_j| /
    scales_j; all over the keys that the row sees."""
    T, H, d = q.shape
    L, Hkv = k.shape[0], k.shape[1]
    scale = 1.0 / math.sqrt(d) if not scale else scale
    r = dict(out=np.zeros((T, H, d)), lse=np.full((T, H), -np.inf), mag=np.zeros((T, H, d)),
             size=np.zeros((T, H)), top=np.zeros((T, H)), codes=np.zeros((T, H, d)))
    if L == 0:
        return r
    seen = np.ones((T, L), bool)
    if causal:
        seen = np.arange(L)[None, :] <= (L - T + np.arange(T))[:, None]
    live = seen.any(1)
    for h in range(H):
        g = h // (H // Hkv)
        s = np.where(seen, q[:, h] @ k[:, g].T * scale, -np.inf)
        m = np.where(live, s.max(1), 0.0)
        p = np.exp(s - m[:, None])
        total = np.where(live, p.sum(1), 1.0)
        p /= total[:, None]
        r["lse"][:, h] = np.where(live, m + np.log(total), -np.inf)
        r["out"][:, h], r["mag"][:, h] = p @ v[:, g], p @ np.abs(v[:, g])
        r["size"][:, h] = np.where(seen, np.abs(q[:, h]) @ np.abs(k[:, g]).T * scale, 0.0).max(1)
        r["top"][:, h] = (p * scales[None, :, g]).max(1)
        r["codes"][:, h] = seen @ (np.abs(v[:, g]) / scales[:, g, None])
    return r


def bounds(r, d, L):
    """What outputs and normalisers may be off by.  The logits are float32 sums of d exact
    products, and the exponent is taken of them times the scale less the maximum: within
    delta of the exact one.  A probability is rounded to f16 (half a step, 2^-11 of it) once;
    the sums are float32, and the exponentials good to a few units.  A weight (a probability
    times its block's scale) far below the row's largest is held to 2^-26 of that, times the
    key's code.  The output is rounded to bf16 (half a step, 2^-8 of it)."""
    delta = (d + 8) * 2.0 ** -24 * r["size"]
    out = (2.0 ** -11 + 2 * delta[..., None] + L * 2.0 ** -24 + 2.0 ** -20) * r["mag"]
    out = out + 2.0 ** -26 * r["top"][..., None] * r["codes"]
    out = out + 2.0 ** -8 * (np.abs(r["out"]) + out) + 1e-38
    lse = delta + 2.0 ** -22 * np.where(np.isfinite(r["lse"]), np.abs(r["lse"]), 0.0) + L * 2.0 ** -24 + 1e-6
    return out, lse


def check(got, lse, q, k, v, scales, causal, scale=None):
    r = attention(q, k, v, scales, causal, scale)
    tol, tol_lse = bounds(r, q.shape[-1], len(k))
    with np.errstate(invalid="ignore"):
        off = np.abs(got - r["out"])
    assert np.all(off <= tol), "out: %d of %d not numbers, worst %g of its bound" % (
        np.isnan(got).sum(), got.size, np.nanmax(off / tol))
    if lse is not None:
        fin = np.isfinite(r["lse"])
        assert np.all(lse[~fin] == -np.inf)
        assert np.all(np.abs(lse[fin] - r["lse"][fin]) <= tol_lse[fin])


def per_token(sequence):
    """The block scale of every token of a cache_model.Sequence, [tokens, Hkv]."""
    return sequence.scale[np.arange(len(sequence.x)) // sequence.page]
