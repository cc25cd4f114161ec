"""CPU oracle, part 3: beam search as the plain procedure, one sentence at a time.

TEST INFRASTRUCTURE ONLY (see oracle/model.py).

Hypotheses start as one empty one.  A step extends every unfinished hypothesis
by every word (score: sum of log-probabilities), keeps finished ones as they
are, and takes the `beam` best by score / length**alpha, equal ones in the order
(hypothesis, word).  A hypothesis is finished by [EOS] or at m tokens; the
search ends when all are.

A cache in 4 bits holds, per group of min(head_dim, 32) dimensions of a token's
head vector, least (the minimum rounded down to bfloat16), step (the smallest
bfloat16 with 15 step >= range) and the nearest codes 0 .. 15.
"""
from __future__ import annotations

import dataclasses
import math
from typing import List

import numpy as np


def _bf16_down(x):
    m, e = np.frexp(x)
    return np.ldexp(np.floor(m * 256.0), e - 8)


def quantised(x, head_dim):
    """Rows [.., d] as a cache in 4 bits holds them."""
    g = x.reshape(*x.shape[:-1], -1, min(head_dim, 32))
    least = _bf16_down(g.min(-1, keepdims=True))
    step = -_bf16_down(-(g.max(-1, keepdims=True) - least) / 15)
    code = np.clip(np.rint((g - least) / np.where(step > 0, step, 1)), 0, 15)
    return (least + code * step).reshape(x.shape)


class _Rows:
    """Cache rows that are quantised as they are written."""

    def __init__(self, a, head_dim):
        self.a, self.head_dim = a, head_dim

    def __setitem__(self, i, x):
        self.a[i] = quantised(x, self.head_dim)

    def __getitem__(self, i):
        return self.a[i]

    def copy(self):
        return _Rows(self.a.copy(), self.head_dim)


@dataclasses.dataclass
class Hypothesis:
    tokens: List[int]
    score: float
    done: bool = False


@dataclasses.dataclass
class BeamResult:
    hyps: List[Hypothesis]     # best first
    steps: int                 # decoder forwards
    gap: float                 # least distance of two neighbouring keys among the beam + 1 best of any step
    linf: float                # largest |logit| seen


def _key(score, n, alpha):
    return score / max(n, 1) ** alpha


def _log_softmax(x):
    m = x.max()
    return x - (m + math.log(np.exp(x - m).sum()))


def beam_search(model, enc, m, beam, alpha, bos, eos, cache="native") -> BeamResult:
    hd = model.cfg.head_dim

    def new_cache():
        c = model.new_cache(m)
        if cache == "int4":
            c.k, c.v = ([_Rows(a, hd) for a in t] for t in (c.k, c.v))
        return c

    def copy(c):
        return dataclasses.replace(c, k=[a.copy() for a in c.k], v=[a.copy() for a in c.v])

    beams = [(Hypothesis([], 0.0), new_cache())]
    steps, gap, linf = 0, math.inf, 0.0
    while any(not h.done for h, _ in beams):
        cands = []
        for i, (h, c) in enumerate(beams):
            if h.done:
                cands.append((-_key(h.score, len(h.tokens), alpha), i, -1, h.score))
                continue
            p = len(h.tokens)
            x = model.logits(model.decode_rows(enc, c, [h.tokens[-1] if p else bos], p))[0]
            linf = max(linf, float(np.abs(x).max()))
            lp = h.score + _log_softmax(x)
            for v in np.argsort(-lp, kind="stable")[:beam + 1]:
                cands.append((-_key(lp[v], p + 1, alpha), i, int(v), float(lp[v])))
        steps += 1
        cands.sort(key=lambda t: t[:3])
        keys = [-t[0] for t in cands[:beam + 1]]
        gap = min([gap] + [a - b for a, b in zip(keys, keys[1:])])
        new = []
        for _, i, v, s in cands[:beam]:
            h, c = beams[i]
            if v < 0:
                new.append((h, c))
            else:
                t = h.tokens + [v]
                new.append((Hypothesis(t, s, v == eos or len(t) >= m), copy(c)))
        beams = new
    return BeamResult([h for h, _ in beams], steps, gap, linf)


def rescore(model, enc, tokens, bos, cache="native") -> float:
    """Sum of log-probabilities of a hypothesis, token by token."""
    c = model.new_cache(len(tokens))
    if cache == "int4":
        c.k, c.v = ([_Rows(a, model.cfg.head_dim) for a in t] for t in (c.k, c.v))
    s, prev = 0.0, bos
    for p, t in enumerate(tokens):
        s += float(_log_softmax(model.logits(model.decode_rows(enc, c, [prev], p))[0])[t])
        prev = t
    return s
