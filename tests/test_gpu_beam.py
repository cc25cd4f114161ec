"""Beam decoding (pd_decode_beam) on the GPU against the oracle's beam search.

Tolerance.  A logit is off by at most EPS[dtype] * max|logit| (tests/parity.py,
measured by tests/test_gpu_logits.py), so a log-probability by twice that and
the score of a hypothesis of n tokens by n times as much; scores are summed in
float, one rounding of at most half a step of 2^-23 of the sum a step.  Every
returned hypothesis has to have the oracle's score for its own tokens within
that.  The hypotheses themselves have to be the oracle's, unless the oracle met
two neighbouring keys closer than two such errors (a near tie, after which the
searches may part).

A cache in 4 bits rounds each key and value to a code: one that lies within the
GPU's rounding of a border takes the neighbouring code, a whole step away.  How
far such flips move a score is measured on the oracle itself: its keys and
values are shifted by random rounding-sized amounts (2^-20 of the largest of the
head vector, float32's error after a few products) before they are quantised,
and the largest change of the score over four such runs, doubled, is added.
"""
import ctypes
import dataclasses
import os

import numpy as np
import pytest
import torch

import oracle
from oracle import beam as OB
from paper_2305_10427_amd import configs as C, pdec, synth
from tests.parity import EPS, gpu_decode_batch

pytestmark = pytest.mark.gpu

SMALL_BF16 = dataclasses.replace(C.TINY, name="small_bf16", pre_ln=True, act_gelu=True, dtype=C.BF16)
WIDE_HEADS = dataclasses.replace(C.TINY, name="wide_heads", d_model=256, n_heads=2, d_ff=256, vocab=1111, pre_ln=True)
LONG_BF16 = dataclasses.replace(C.TINY, name="long", n_dec=3, d_model=128, n_heads=2, vocab=523, dtype=C.BF16)


def say(*a):
    print(*a, flush=True)


@dataclasses.dataclass
class Fixture:
    cfg: object
    ctx: object
    M: object


_made = {}


def fixture(cfg, eos_bias=0.0, batch=4, max_src=24, max_tgt=40, seed=11):
    key = (cfg.name, cfg.dtype, eos_bias, batch, max_tgt)
    if key not in _made:
        w = synth.make_weights(cfg, seed=seed, bias_std=0.3, ln_std=0.2, eos_bias=eos_bias)
        _made[key] = Fixture(cfg, pdec.Context(pdec.Model(cfg, w), batch, max_src, max_tgt), oracle.Model(cfg, w.values))
    return _made[key]


def sources(cfg, lens, seed):
    g = np.random.default_rng(seed)
    return [g.integers(4, cfg.vocab, n).astype(np.int32) for n in lens]


def encode(ctx, srcs):
    src = np.zeros((len(srcs), max(map(len, srcs))), np.int32)
    for r, s in enumerate(srcs):
        src[r, :len(s)] = s
    ctx.encode(torch.from_numpy(src).cuda(), [len(s) for s in srcs])


def run(f, srcs, ms, **kw):
    encode(f.ctx, srcs)
    return tuple(t.cpu().numpy() for t in f.ctx.decode_beam(ms, **kw))


def flip_tolerance(f, enc, tokens):
    """Twice the largest change of the score when keys and values are shifted by roundings before they are quantised."""
    base = OB.rescore(f.M, enc, tokens, C.BOS_ID, "int4")
    worst, plain = 0.0, OB.quantised
    for seed in range(4):
        g = np.random.default_rng(seed)

        def shifted(x, head_dim):
            big = np.abs(x.reshape(*x.shape[:-1], -1, head_dim)).max(-1, keepdims=True)
            return plain(x + (2.0 ** -20 * big * g.uniform(-1, 1, big.shape[:-1] + (head_dim,))).reshape(x.shape), head_dim)

        OB.quantised = shifted
        try:
            worst = max(worst, abs(OB.rescore(f.M, enc, tokens, C.BOS_ID, "int4") - base))
        finally:
            OB.quantised = plain
    return 2 * worst


def check(f, srcs, ms, out, beam, alpha, cache="native"):
    ids, lens, scores, k, flags = out
    exact = 0
    for b, (src, m) in enumerate(zip(srcs, ms)):
        enc = f.M.encode(src)
        want = OB.beam_search(f.M, enc, m, beam, alpha, C.BOS_ID, C.EOS_ID, cache)
        per_token = 2 * EPS[f.cfg.dtype] * want.linf
        hyps = [list(map(int, ids[b, j, :lens[b, j]])) for j in range(beam)]
        worst = 0.0
        for j, h in enumerate(hyps):
            assert 1 <= len(h) <= m and C.EOS_ID not in h[:-1] and (len(h) == m or h[-1] == C.EOS_ID), (b, j, h)
            assert (ids[b, j, lens[b, j]:] == C.PAD_ID).all()
            ref = OB.rescore(f.M, enc, h, C.BOS_ID, cache)
            tol = len(h) * (per_token + abs(ref) * 2.0 ** -24) + (flip_tolerance(f, enc, h) if cache == "int4" else 0.0)
            worst = max(worst, tol)
            assert abs(scores[b, j] - ref) <= tol, (b, j, scores[b, j], ref, tol)
        assert len({tuple(h) for h in hyps}) == beam
        keys = scores[b] / np.maximum(lens[b], 1) ** np.float64(alpha)
        assert (np.diff(keys) <= 1e-6 * np.abs(keys[1:])).all()
        assert flags[b] & 1 and bool(flags[b] & 2) == (hyps[0][-1] == C.EOS_ID) and not flags[b] & 8
        same = hyps == [h.tokens for h in want.hyps]
        say(f"  sentence {b}: m={m} k={k[b]} same={same} gap={want.gap:.2e} tol={worst:.2e}")
        if same:
            exact += 1
            assert k[b] == want.steps
        else:
            assert want.gap <= 2 * worst, (b, hyps, [h.tokens for h in want.hyps])
    return exact


@pytest.mark.parametrize("cfg,beam,alpha,cache", [
    (C.TINY, 4, 1.0, "native"), (C.TINY, 5, 0.6, "int4"), (C.TINY, 1, 0.0, "native"), (C.TINY, 16, 0.0, "native"),
    (SMALL_BF16, 5, 0.6, "native"), (SMALL_BF16, 4, 1.0, "int4"), (WIDE_HEADS, 3, 1.0, "native"),
    (WIDE_HEADS, 6, 0.6, "int4")], ids=lambda v: v.name if hasattr(v, "name") else str(v))
@pytest.mark.parametrize("eos_bias", [0.0, 4.0])
def test_beam_decoding_against_the_oracle(cfg, beam, alpha, cache, eos_bias):
    f = fixture(cfg, eos_bias)
    srcs, ms = sources(cfg, [16, 3, 24, 11], 5), [16, 9, 20, 1]
    say(f"beam {cfg.name} beam={beam} alpha={alpha} cache={cache} eos={eos_bias}")
    exact = check(f, srcs, ms, run(f, srcs, ms, beam=beam, alpha=alpha, cache=cache), beam, alpha, cache)
    if cfg.dtype == C.F32 and cache == "native":
        assert exact >= 2                      # the rule for near ties is not what passes


def test_one_beam_is_greedy_decoding():
    for cfg in (C.TINY, WIDE_HEADS):
        f = fixture(cfg, 4.0)
        srcs, ms = sources(cfg, [16, 9, 20], 8), [24, 40, 17]
        want = gpu_decode_batch(f.ctx, srcs, ms, "ar")
        ids, lens, _, k, _ = run(f, srcs, ms, beam=1, alpha=0.0)
        for b, w in enumerate(want):
            enc = f.M.encode(srcs[b])
            ref = OB.beam_search(f.M, enc, ms[b], 1, 0.0, C.BOS_ID, C.EOS_ID)
            if ref.gap > 4 * EPS[cfg.dtype] * ref.linf:
                assert list(ids[b, 0, :lens[b, 0]]) == list(w.ids) and k[b] == w.k


def test_a_long_search_over_many_pages():
    f = fixture(LONG_BF16, 0.0, batch=2, max_src=40, max_tgt=130)
    srcs, ms = sources(LONG_BF16, [33, 40], 9), [130, 77]
    out = run(f, srcs, ms, beam=5, alpha=1.0)
    check(f, srcs, ms, out, 5, 1.0)
    out4 = run(f, srcs, ms, beam=4, alpha=1.0, cache="int4")
    check(f, srcs, ms, out4, 4, 1.0, "int4")
    f = fixture(dataclasses.replace(LONG_BF16, name="long_f32", dtype=C.F32), 0.0, batch=2, max_src=40, max_tgt=130)
    check(f, srcs, ms, run(f, srcs, ms, beam=5, alpha=1.0), 5, 1.0)


def test_calls_are_repeatable_and_do_not_depend_on_what_ran_before():
    f = fixture(C.TINY, 4.0)
    g = fixture(C.TINY, 4.0, batch=5, seed=11)          # other limits, the same model
    srcs, ms = sources(C.TINY, [16, 3, 24], 15), [30, 12, 21]
    first = run(f, srcs, ms, beam=4)
    gpu_decode_batch(f.ctx, srcs[:2], ms[:2], "hybrid", 4)
    run(f, srcs[1:], ms[1:], beam=7, alpha=0.3, cache="int4")
    run(f, sources(C.TINY, [9], 1), [40], beam=4)
    for again in (run(f, srcs, ms, beam=4), run(g, srcs, ms, beam=4)):
        for a, b in zip(first, again):
            np.testing.assert_array_equal(a, b)
    # a decode after a beam search is what it was
    want = gpu_decode_batch(g.ctx, srcs, ms, "gs_jacobi", 4)
    got = gpu_decode_batch(f.ctx, srcs, ms, "gs_jacobi", 4)
    for a, b in zip(got, want):
        np.testing.assert_array_equal(a.ids, b.ids)
        assert (a.k, a.flags) == (b.k, b.flags)


def test_a_sentence_does_not_depend_on_its_batch():
    f = fixture(C.TINY, 4.0)
    srcs, ms = sources(C.TINY, [16, 3, 24, 11], 25), [30, 12, 21, 40]
    ids, lens, scores, k, fl = run(f, srcs, ms, beam=5)
    for b in range(4):
        one = run(f, [srcs[b]], [ms[b]], beam=5)
        ref = OB.beam_search(f.M, f.M.encode(srcs[b]), ms[b], 5, 1.0, C.BOS_ID, C.EOS_ID)
        if ref.gap > 8 * ms[b] * EPS[C.F32] * ref.linf:
            np.testing.assert_array_equal(one[0][0], ids[b, :, :ms[b]])
            np.testing.assert_array_equal(one[1][0], lens[b])
        np.testing.assert_allclose(one[2][0], scores[b], atol=4 * ms[b] * EPS[C.F32] * ref.linf)


def test_steps_launched_directly_equal_captured_ones(monkeypatch):
    f = fixture(SMALL_BF16, 2.0)
    srcs, ms = sources(SMALL_BF16, [16, 3, 24], 35), [30, 12, 21]
    want = run(f, srcs, ms, beam=5, cache="int4")
    monkeypatch.setenv("PDEC_GRAPHS", "0")
    ctx = pdec.Context(f.ctx.model, 4, 24, 40)
    got = run(Fixture(f.cfg, ctx, f.M), srcs, ms, beam=5, cache="int4")
    for a, b in zip(got, want):
        np.testing.assert_array_equal(a, b)


def test_many_settings_of_one_context():
    """More settings than captured steps are kept for."""
    f = fixture(C.TINY, 4.0)
    srcs, ms = sources(C.TINY, [16, 3], 65), [9, 6]
    alphas = [0.0] + [0.25 + 0.01 * i for i in range(40)]
    first = run(f, srcs, ms, beam=3, alpha=alphas[0])
    for a in alphas[1:]:
        run(f, srcs, ms, beam=3, alpha=a)
    for a, b in zip(run(f, srcs, ms, beam=3, alpha=alphas[0]), first):
        np.testing.assert_array_equal(a, b)


def test_many_sentences_on_another_stream():
    f = fixture(C.TINY, 4.0, batch=70, max_src=8, max_tgt=12)
    srcs, ms = sources(C.TINY, [3 + i % 6 for i in range(70)], 45), [1 + i % 12 for i in range(70)]
    want = run(f, srcs, ms, beam=4)
    check(f, srcs[60:64], ms[60:64], tuple(x[60:64] for x in want), 4, 1.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        encode(f.ctx, srcs)
    out = f.ctx.decode_beam(ms, beam=4, stream=s)
    s.synchronize()
    for a, b in zip(out, want):
        np.testing.assert_array_equal(a.cpu().numpy(), b)


def test_the_widest_beam():
    f = fixture(C.TINY, 4.0)
    srcs, ms = sources(C.TINY, [16, 3], 55), [20, 6]
    check(f, srcs, ms, run(f, srcs, ms, beam=64, alpha=0.6), 64, 0.6)


def test_a_vocabulary_smaller_than_the_beam_and_logits_that_are_not_finite():
    cfg = dataclasses.replace(C.TINY, name="few_words", vocab=7)
    f = fixture(cfg, 0.0, batch=2)
    srcs = sources(cfg, [5, 9], 2)
    ids, lens, scores, k, fl = run(f, srcs, [1, 3], beam=20)
    assert (lens[0, :7] == 1).all() and (lens[0, 7:] == 0).all() and (scores[0, 7:] == -np.inf).all()
    assert sorted(ids[0, :7, 0]) == list(range(7)) and abs(np.exp(scores[0, :7].astype(np.float64)).sum() - 1) < 1e-4
    assert (lens[1] >= 1).all() and fl[0] & 1
    # a NaN in the output bias: that word is never taken, and the flag is set
    w = synth.make_weights(cfg, seed=11, bias_std=0.3, ln_std=0.2)
    w.values["out_bias"][5] = np.nan
    ctx = pdec.Context(pdec.Model(cfg, w), 2, 24, 40)
    ids, lens, scores, k, fl = run(Fixture(cfg, ctx, None), srcs, [6, 6], beam=4)
    assert (fl & 8).all() and not (ids == 5).any() and np.isfinite(scores).all()


def test_refusals():
    f = fixture(C.TINY, 0.0, batch=2)
    L = pdec.load_library()
    fresh = pdec.Context(f.ctx.model, 2, 24, 40)
    with pytest.raises(pdec.PdError):
        fresh.decode_beam([4])                              # nothing encoded
    encode(f.ctx, sources(C.TINY, [4, 5], 1))
    for kw, status in ((dict(beam=0), 1), (dict(beam=65), 2), (dict(alpha=-1.0), 1), (dict(alpha=float("nan")), 1),
                       (dict(cache="bf16"), 1), (dict(tgt_m=[4]), 1), (dict(tgt_m=[4, 41]), 2), (dict(tgt_m=[0, 4]), 2)):
        with pytest.raises(pdec.PdError) as e:
            f.ctx.decode_beam(kw.pop("tgt_m", [4, 4]), **kw)
        assert e.value.status == status, kw
    n = ctypes.c_size_t()
    assert L.pd_decode_beam_bytes(f.ctx.handle, 4, 1, ctypes.byref(n)) == 1      # a bf16 cache under a float32 model
    assert L.pd_decode_beam_bytes(f.ctx.handle, 4, 0, ctypes.byref(n)) == 0
    buf = torch.empty(n.value + 256, dtype=torch.uint8, device="cuda")
    out = torch.empty(4096, dtype=torch.int32, device="cuda")
    o = out.data_ptr()
    at = (buf.data_ptr() + 255) // 256 * 256
    m = (ctypes.c_int32 * 2)(4, 4)
    call = lambda **k: L.pd_decode_beam(f.ctx.handle, 4, 1.0, 0, k.get("m", m), k.get("ids", o), k.get("ld", 4), o,  # noqa: E731
                                        k.get("scores", o), o, o, k.get("ws", at), k.get("bytes", n.value), None)
    for kw, status in ((dict(m=None), 1), (dict(ids=None), 1), (dict(scores=None), 1), (dict(ld=3), 1), (dict(ws=None), 3),
                       (dict(ws=at + 128), 3), (dict(bytes=n.value - 1), 3)):
        assert call(**kw) == status, kw
    with pytest.raises(pdec.PdError) as e:
        fresh.decode_beam([])
    assert e.value.status == 6


def test_null_contexts_are_refused():
    L = pdec.load_library()
    n = ctypes.c_size_t()
    assert L.pd_decode_beam_bytes(None, 4, 0, ctypes.byref(n)) == 1
    assert L.pd_decode_beam(None, 4, 1.0, 0, None, None, 4, None, None, None, None, None, 0, None) == 1
