"""What the bounds of tests/attend_error.py accept and refuse, on the CPU: plain float arithmetic passes; an output of
zeros, a dropped key (a missing appended token is one), a key too many, queries or weights of fewer bits do not."""
import numpy as np
import pytest
import torch

from tests import attend_error as E, operators_ref as R

CASES = [(c, dh, n) for c in ("f32", "bf16", "int4") for dh, n in ((16, 2), (16, 41), (32, 129), (64, 17), (64, 138), (64, 1000), (128, 132), (128, 9001))]


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).double().numpy()


def head(cache, dh, n, seed=0, size=0.5):
    """q, k, v of a head as the cache holds them, and the arguments of a cache in 4 bits."""
    g = np.random.default_rng(seed + dh + n)
    q = (size * g.normal(size=dh)).astype(np.float32).astype(np.float64)
    if cache != "int4":
        k, v = g.normal(size=(2, n, dh)).astype(np.float32).astype(np.float64)
        return (q, bf16(k), bf16(v), {}) if cache == "bf16" else (q, k, v, {})
    kw, kv = {}, []
    for name in ("k_par", "v_par"):
        step = bf16(0.1 + 0.3 * g.random((n, max(1, dh // 32))))
        least = bf16(-7.5 * step + 0.5 * g.normal(size=step.shape))
        kw[name] = g.integers(0, 16, (n, dh)), step, least
        kv.append(R.dequantise(*kw[name]))
    return q, *kv, kw


def plain(q, k, v, scale):
    """In float32, one key after the other."""
    f = np.float32
    q, k, v, m, l, o = f(f(scale) * q.astype(f)), k.astype(f), v.astype(f), f(-np.inf), f(0), np.zeros(len(q), f)
    for kj, vj in zip(k, v):
        s = f(0)
        for a, b in zip(kj, q):
            s = f(s + f(a * b))
        new = max(m, s)
        r, p = np.exp(f(m - new)), np.exp(f(s - new))
        l, o, m = f(l * r + p), o * r + p * vj, new
    return (o / l).astype(np.float64)


def attend(q, k, v, scale, keep=slice(None)):
    return R.attend(q[None], k[keep][:, None], v[keep][:, None], scale)[0][0]


@pytest.mark.parametrize("cache,dh,n", CASES)
def test_float_passes_and_mistakes_do_not(cache, dh, n):
    scale = dh ** -0.5
    g = np.random.default_rng(n)
    heads = [head(cache, dh, n, seed) for seed in range(2 if n > 2000 else 4)]
    exact = [E.attend(cache, q, k, v, scale, **kw) for q, k, v, kw in heads]
    for (q, k, v, _), (ref, *_) in zip(heads, exact):
        np.testing.assert_allclose(ref, attend(q, k, v, scale), atol=1e-13)
    z = lambda got: [(o - ref) / sd for o, (ref, sd, _) in zip(got, exact)]  # noqa: E731
    if n <= 1000:
        assert E.fits(z([plain(q, k, v, scale) for q, k, v, _ in heads]))
    assert E.fits(z([ref for ref, *_ in exact]))
    assert not E.fits(z([np.zeros(dh) for _ in heads]))
    assert not E.fits(z([np.full(dh, np.nan) for _ in heads]))
    for j in {0, n // 2, n - 1, int(g.integers(0, n))}:        # of one head only
        wrong = [ref for ref, *_ in exact]
        q, k, v, _ = heads[0]
        wrong[0] = attend(q, k, v, scale, np.arange(n) != j)
        assert not E.fits(z(wrong)), j
        wrong[0] = attend(q, k, v, scale, np.append(np.arange(n), j))
        assert not E.fits(z(wrong)), j
    assert not E.fits(z([attend(bf16(q), k, v, scale) for q, k, v, _ in heads]))
    short = []
    for q, k, v, _ in heads:                                   # weights of eight bits
        p = np.exp(scale * (k @ q))
        short.append(bf16(p) @ v / p.sum())
    assert not E.fits(z(short))


def test_two_parts_of_a_weight_are_too_few_for_a_float():
    """Weights of 16 bits over a short cache: beyond the bounds, which float's 24 are not."""
    heads = [head("bf16", 64, 17, seed) for seed in range(8)]
    zs = {16: [], 24: []}
    for q, k, v, kw in heads:
        ref, sd, _ = E.attend("bf16", q, k, v, 0.125, **kw)
        p = np.exp(0.125 * (k @ q))
        p /= p.max()
        for bits, out in zs.items():
            m, e = np.frexp(p)
            cut = np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)
            out.append((cut @ v / p.sum() - ref) / sd)
    assert E.fits(zs[24])
    assert not E.fits(zs[16])
