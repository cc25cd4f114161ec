"""Plain 64-bit implementations of the beam-search operators, for the tests (numpy, one element or sequence at a time)."""
from __future__ import annotations

import math

import numpy as np

NONFINITE = 8


# --- selection -------------------------------------------------------------------


def candidates(logits, scores, lens, done, pad, alpha):
    """A sentence's candidates (-key, beam, rank, score, token, length, finished), best first, and its flags."""
    K, V = logits.shape
    cands, flags = [], 0
    for k in range(K):
        s = float(scores[k])
        if not math.isfinite(s):
            continue
        if done[k]:
            cands.append((-s / max(int(lens[k]), 1) ** float(alpha), k, 0, s, pad, int(lens[k]), 1))
            continue
        x = np.array(logits[k], np.float64)
        bad = np.isnan(x) | (x == np.inf)
        flags |= NONFINITE * bool(bad.any())
        x[bad] = -np.inf
        words = np.nonzero(x > -np.inf)[0]
        if not len(words):
            continue
        m = x.max()
        lse = m + math.log(math.fsum(np.exp(x[words] - m)))
        for r, v in enumerate(words[np.lexsort((words, -x[words]))][:K]):
            c = s + (x[v] - lse)
            n = int(lens[k]) + 1
            cands.append((-c / max(n, 1) ** float(alpha), k, r, c, int(v), n, 0))
    return sorted(cands, key=lambda c: c[:3]), flags


def select(logits, scores, lens, done, eos, pad, alpha, max_len=None):
    """logits [B, K, V] float64; returns (scores f64, parents, tokens, lens, done, src, flags)."""
    B, K, V = logits.shape
    S = np.full((B, K), -np.inf)
    par, tok, ln, dn, src = (np.zeros((B, K), np.int32) for _ in range(5))
    par[:], tok[:], dn[:], src[:] = -1, pad, 1, -1
    flags = np.zeros(B, np.int32)
    for b in range(B):
        cands, flags[b] = candidates(logits[b], scores[b], lens[b], done[b], pad, alpha)
        for j, (_, k, _, c, v, n, fin) in enumerate(cands[:K]):
            S[b, j], par[b, j], tok[b, j], ln[b, j] = c, k, v, n
            dn[b, j] = int(fin or v == eos or (max_len is not None and n >= max_len[b]))
            src[b, j] = -1 if dn[b, j] else b * K + k
    return S, par, tok, ln, dn, src, flags


# --- the cache in 4 bits -----------------------------------------------------------


def bf16_down(x):
    """The largest bfloat16 up to x (float64 in, float64 out)."""
    m, e = np.frexp(np.asarray(x, np.float64))
    return np.ldexp(np.floor(m * 256.0), e - 8)


def bf16_up(x):
    return -bf16_down(-np.asarray(x, np.float64))


def quantise(x):
    """[..., dh] float64 -> codes, step, least [..., groups] by the definition."""
    dh = x.shape[-1]
    g = x.reshape(*x.shape[:-1], max(1, dh // 32), -1)
    least = bf16_down(g.min(-1))
    step = bf16_up((g.max(-1) - least) / 15)
    with np.errstate(invalid="ignore", divide="ignore"):
        code = np.where(step[..., None] > 0, np.clip(np.rint((g - least[..., None]) / step[..., None]), 0, 15), 0)
    return code.reshape(x.shape), step, least


def dequantise(code, step, least):
    per = code.shape[-1] // step.shape[-1]
    return code * np.repeat(step, per, -1) + np.repeat(least, per, -1)


def nibble(e):
    return e // 2 + 4 * (e % 2)


def pack(code):
    """Codes along the last axis to bytes, eight to a little-endian word."""
    c = np.asarray(code, np.uint32).reshape(*code.shape[:-1], -1, 8)
    w = np.zeros(c.shape[:-1], np.uint32)
    for e in range(8):
        w |= c[..., e] << np.uint32(4 * nibble(e))
    return np.ascontiguousarray(w).view(np.uint8).reshape(*code.shape[:-1], -1)


def unpack(b):
    w = np.ascontiguousarray(b).view(np.uint32)
    c = np.stack([(w >> np.uint32(4 * nibble(e))) & 15 for e in range(8)], -1)
    return c.reshape(*b.shape[:-1], -1).astype(np.float64)


# --- attention -----------------------------------------------------------------------


def attend(q, keys, values, scale):
    """q [H, dh], keys and values [n, kv heads, dh] float64 of one sequence -> out [H, dh], weights [H, n]."""
    H, dh = q.shape
    out = np.zeros((H, dh))
    n, kv = keys.shape[0], keys.shape[1]
    w = np.zeros((H, n))
    if n == 0:
        return out, w
    for h in range(H):
        s = scale * (keys[:, h // (H // kv)] @ q[h])
        p = np.exp(s - s.max())
        w[h] = p / p.sum()
        out[h] = w[h] @ values[:, h // (H // kv)]
    return out, w


# --- pages ---------------------------------------------------------------------------


def _pages(n, ps):
    return -(-n // ps)


def fork(table, lens, parents, pages, ps, grow):
    """Returns (table, lens, refs, status, [(from, to)])."""
    n_in, ld = table.shape
    n_out = len(parents)
    new = np.full((n_out, ld), -1, np.int64)
    ln = np.zeros(n_out, np.int64)
    for s, p in enumerate(parents):
        if 0 <= p < n_in:
            ln[s] = min(max(int(lens[p]), 0), ld * ps)
            for j in range(_pages(ln[s], ps)):
                new[s, j] = table[p, j] if 0 <= table[p, j] < pages else -1
    refs = np.bincount(new[new >= 0], minlength=pages)
    status = [0, 0]
    copies = []
    if grow:
        alive = [s for s in range(n_out) if 0 <= parents[s] < n_in]
        full = [s for s in alive if ln[s] == ld * ps]
        writers = {}
        for s in alive:
            if ln[s] % ps and new[s, ln[s] // ps] >= 0:
                writers.setdefault(new[s, ln[s] // ps], []).append(s)
        need = []
        for s in alive:
            if s in full:
                continue
            p = new[s, ln[s] // ps] if ln[s] % ps else -1
            if p < 0:
                need.append((s, None))
            elif not (refs[p] == len(writers[p]) and writers[p][0] == s):
                need.append((s, p))
        free = [p for p in range(pages) if refs[p] == 0]
        status[0] = max(0, len(need) - len(free)) + len(full)
        if status[0]:
            return np.full((n_out, ld), -1, np.int64), np.zeros(n_out, np.int64), np.zeros(pages, np.int64), status, []
        for (s, p), to in zip(need, free):
            new[s, ln[s] // ps] = to
            if p is not None:
                copies.append((p, to))
        for s in alive:
            ln[s] += 1
    refs = np.bincount(new[new >= 0], minlength=pages)
    status[1] = int((refs > 0).sum())
    return new, ln, refs, status, copies


def compact(table, lens, pages, ps):
    """Returns (table, remap, status, [(from, to)])."""
    S, ld = table.shape
    at = [(s, j) for s in range(S) for j in range(min(_pages(max(int(lens[s]), 0), ps), ld)) if 0 <= table[s, j] < pages]
    used = sorted({int(table[i]) for i in at})
    n = len(used)
    remap = np.full(pages, -1, np.int64)
    remap[used] = used
    moves = list(zip([p for p in used if p >= n], [p for p in range(n) if p not in set(used)]))
    for a, b in moves:
        remap[a] = b
    new = np.full((S, ld), -1, np.int64)
    for i in at:
        new[i] = remap[table[i]]
    return new, remap, [len(moves), n], moves
