"""Pins of the beam-search oracle: greedy at one beam, brute force where the beam holds every sequence, scores that
add up, and the cache in 4 bits against the operators' reference."""
import dataclasses
import itertools
import math

import numpy as np
import pytest

import oracle
from oracle import beam as OB
from paper_2305_10427_amd import configs as C, synth
from tests import operators_ref as R


def _model(vocab=40, seed=3, eos_bias=0.0, **kw):
    cfg = dataclasses.replace(C.TINY, name="t", vocab=vocab, n_enc=1, n_dec=2, d_model=32, n_heads=2, d_ff=64, **kw)
    return oracle.Model(cfg, synth.make_weights(cfg, seed=seed, bias_std=0.3, ln_std=0.2, eos_bias=eos_bias).values)


@pytest.mark.parametrize("eos_bias", [0.0, 3.0])
def test_one_beam_is_greedy(eos_bias):
    M = _model(eos_bias=eos_bias)
    for seed in range(4):
        enc = M.encode(np.random.default_rng(seed).integers(4, 40, 7))
        want = oracle.decode(M, enc, 9, "ar", 1)
        got = OB.beam_search(M, enc, 9, 1, 0.6, C.BOS_ID, C.EOS_ID)
        assert got.hyps[0].tokens == list(want.out) and got.steps == len(want.out)


@pytest.mark.parametrize("alpha", [0.0, 1.0])
def test_a_beam_that_holds_everything_finds_the_best(alpha):
    M = _model(vocab=6, seed=5)
    enc = M.encode(np.array([4, 5, 4]))
    m = 3
    best = []
    for n in range(1, m + 1):
        for t in itertools.product(range(6), repeat=n):
            if C.EOS_ID in t[:-1] or (n < m and t[-1] != C.EOS_ID):
                continue
            s = OB.rescore(M, enc, list(t), C.BOS_ID)
            best.append((-s / n ** alpha, t, s))
    best.sort()
    r = OB.beam_search(M, enc, m, 6 ** m, alpha, C.BOS_ID, C.EOS_ID)
    assert len(r.hyps) == len(best)
    assert [tuple(h.tokens) for h in r.hyps[:20]] == [t for _, t, _ in best[:20]]
    np.testing.assert_allclose([h.score for h in r.hyps], [s for *_, s in best], atol=1e-9)
    assert abs(math.fsum(math.exp(h.score) for h in r.hyps) - 1) < 1e-9       # all sequences: their probabilities add to one


def test_scores_are_sums_of_log_probabilities_in_order():
    M = _model(eos_bias=2.0)
    enc = M.encode(np.arange(4, 12))
    for cache in ("native", "int4"):
        r = OB.beam_search(M, enc, 10, 5, 0.7, C.BOS_ID, C.EOS_ID, cache)
        keys = [h.score / len(h.tokens) ** 0.7 for h in r.hyps]
        assert keys == sorted(keys, reverse=True) and r.gap >= 0 and len(r.hyps) == 5
        assert len({tuple(h.tokens) for h in r.hyps}) == 5
        for h in r.hyps:
            assert h.done and (h.tokens[-1] == C.EOS_ID or len(h.tokens) == 10) and C.EOS_ID not in h.tokens[:-1]
            assert abs(OB.rescore(M, enc, h.tokens, C.BOS_ID, cache) - h.score) < 1e-9


def test_the_quantised_cache_is_the_operators():
    g = np.random.default_rng(1)
    for hd in (16, 32, 64):
        x = g.normal(size=(5, 4 * hd)) * 3 + g.normal(size=(5, 1))
        want = R.dequantise(*R.quantise(x.reshape(5, 4, hd))).reshape(5, -1)
        np.testing.assert_array_equal(OB.quantised(x, hd), want)
        assert (OB.quantised(np.full((1, hd), 0.5), hd) == 0.5).all()
