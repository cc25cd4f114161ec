"""How far attention in float may be off, as a standard deviation per output (numpy, 64 bits).

A rounding at magnitude M is off by at most u M, u = 2^-24, and by u M / sqrt(3) in the root mean square; different
roundings are taken as independent, so their variances add up.  In order, for one sequence and query head:

  query   scale log2(e) q is rounded twice: an error of the score of every key, through each of its products
  scores  a rounding at the magnitude of the partial sum after every product of the matrix cores, and one within it at
          that of its terms.  float32: one a dimension; bfloat16: three products a step of 32 dimensions; 4 bits:
          sums of (16 + code) q a group (the product of the largest part; the others are 2^-7 of it), the sum of
          (least - 16 step) times the sum of q, and an addition a group
  weights an exponential to one ulp of its argument's difference to the maximum, which is rounded; that of a block of
          32 keys is taken again when the maximum moves and when parts are joined
  sums    of a block's weighted values (4 bits: on 23.5 steps more than they are, and the middles apart), of the
          blocks, of the weights; the division

An error e_j of key j's score moves the output by p_j e_j (v_j - out).

An output's error over its deviation is z.  The model leaves open in which order the matrix cores add within a
product, and its roundings are not quite independent, so a root mean square of 2 and a largest value of 10 are allowed
(ten deviations: rounding errors are bounded, and of a normal distribution none of 10^6 values lies beyond 5).
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
BLOCK = 32
RMS, MOST = 2.0, 10.0


def fits(z):
    """Whether the errors z (in deviations) are those of float."""
    z = np.concatenate([np.ravel(x) for x in z])
    return bool(np.isfinite(z).all() and np.sqrt((z ** 2).mean()) <= RMS and np.abs(z).max() <= MOST)


def _blocks(x, axis=0):
    """Sums over blocks of 32 keys."""
    return np.add.reduceat(x, np.arange(0, x.shape[axis], BLOCK), axis)


def _steps(terms, width):
    """Variance (in units of u^2 / 3) of a sum of terms [n, dh] made `width` terms at a time."""
    t = terms.reshape(terms.shape[0], -1, width)
    return (np.cumsum(t.sum(-1), -1) ** 2).sum(-1) + (t ** 2).sum((-1, -2))


def attend(cache, q, k, v, scale, k_par=None, v_par=None):
    """One head: q [dh], k, v [n, dh] as the cache holds them; 4 bits: k_par, v_par = (codes [n, dh], steps, least
    [n, groups]).  Returns out [dh], its standard deviation [dh], and the weights [n]."""
    n, dh = k.shape
    terms = scale * q * k
    s = terms.sum(-1)
    p = np.exp(s - s.max())
    p /= p.sum()
    out = p @ v
    off = v - out

    # the query, common to the keys
    var = (((p[:, None] * terms).T @ off) ** 2).sum(0) + 2 * ((p * s) @ off) ** 2
    # each key's score, and its weight's exponential
    if cache == "f32":
        own = _steps(terms, 1)
    elif cache == "bf16":
        own = 3 * _steps(terms, min(dh, 32))
    else:
        code, step, least = k_par
        g = step.shape[1]
        t = scale * (16 + code) * q * np.repeat(step, dh // g, -1)
        t = t.reshape(n, g, -1)
        qs = scale * q.reshape(g, -1).sum(-1)
        d = (least - 16 * step) * qs
        own = (t.sum(-1) ** 2).sum(-1) + (t ** 2).sum((-1, -2)) + (1 + g) * d.sum(-1) ** 2 + (d ** 2).sum(-1)
    own = own + (s - s.max()) ** 2 + 3 * 4
    var = var + (p ** 2 * own) @ off ** 2
    # blocks: their weights, their sums, the sums of them
    P, O = _blocks(p), _blocks(p[:, None] * v)  # noqa: E741
    var = var + 3 * 12 * ((O - P[:, None] * out) ** 2).sum(0)
    var = var + 3 * (O ** 2).sum(0) + (np.cumsum(O, 0) ** 2).sum(0) + 3 * _blocks((p[:, None] * v) ** 2).sum(0)
    if cache == "int4":
        code, step, least = v_par
        rep = lambda x: np.repeat(x, dh // step.shape[1], -1)  # noqa: E731
        r, mid = _blocks(p[:, None] * 23.5 * step), p[:, None] * (least + 7.5 * step)
        var = var + rep(3 * (r ** 2).sum(0) + 3 * (_blocks(np.abs(mid)) ** 2).sum(0) + (np.cumsum(mid, 0)[::BLOCK] ** 2).sum(0))
    var = var + ((np.cumsum(P) ** 2).sum() + 3 * (P ** 2).sum() + 4 + 2) * out ** 2
    return out, U / np.sqrt(3) * np.sqrt(var), p
