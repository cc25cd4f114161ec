"""The beam-search operators' host side, without a GPU: refusals of the C entry points and of the Python wrappers, and
the plain references the GPU tests compare with."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from paper_2305_10427_amd import pdec
from tests import operators_ref as R

ARG, SHAPE, WORKSPACE, UNSUPPORTED = 1, 2, 3, 5
P = ctypes.c_void_p


def _lib():
    if not os.path.exists(pdec.LIB_PATH):
        pytest.skip("libpdec.so not built (run __graft_entry__.build())")
    return pdec.load_library()


def _size(fn, *a):
    n = ctypes.c_size_t()
    assert fn(*a, ctypes.byref(n)) == 0
    return n.value


FAKE = 1 << 20          # aligned addresses, never read on the host


def _select(L, **kw):
    a = dict(logits=FAKE, dtype=0, ld=1000, B=2, K=4, V=1000, scores=FAKE, lens=FAKE, done=FAKE, max_len=None, eos=2,
             pad=0, alpha=1.0, outs=[FAKE] * 7, ws=FAKE, bytes=1 << 30)
    a.update(kw)
    return L.pd_beam_select(a["logits"], a["dtype"], a["ld"], a["B"], a["K"], a["V"], a["scores"], a["lens"], a["done"],
                            a["max_len"], a["eos"], a["pad"], a["alpha"], *a["outs"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), ARG), (dict(scores=None), ARG), (dict(lens=None), ARG), (dict(done=None), ARG),
    (dict(outs=[FAKE] * 6 + [None]), ARG), (dict(outs=[None] + [FAKE] * 6), ARG), (dict(dtype=2), ARG), (dict(B=0), ARG),
    (dict(K=0), ARG), (dict(V=0), ARG), (dict(K=65), SHAPE), (dict(V=(1 << 24) + 1, ld=1 << 25), SHAPE),
    (dict(B=1 << 20, K=8), SHAPE), (dict(ld=999), ARG), (dict(alpha=-0.5), ARG), (dict(alpha=math.nan), ARG),
    (dict(alpha=math.inf), ARG), (dict(logits=FAKE + 2), ARG), (dict(logits=FAKE + 1, dtype=1), ARG),
    (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 128), WORKSPACE), (dict(bytes=0), WORKSPACE)])
def test_selection_refuses(kw, status):
    assert _select(_lib(), **kw) == status
    assert pdec.load_library().pd_last_error()


def _cache(dtype=1, layers=2, pages=10, ps=16, kv=4, dh=32, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE):
    return pdec.pd_cache(dtype, layers, pages, ps, kv, dh, k, v, ks, vs)


BAD_CACHES = [(dict(dtype=3), ARG), (dict(dtype=-1), ARG), (dict(layers=0), ARG), (dict(pages=0), ARG), (dict(kv=0), ARG),
              (dict(ps=8), UNSUPPORTED), (dict(ps=48), UNSUPPORTED), (dict(dh=48), UNSUPPORTED),
              (dict(dh=256), UNSUPPORTED), (dict(pages=(1 << 24) + 1), SHAPE), (dict(layers=5000), SHAPE),
              (dict(kv=1025), SHAPE)]
BAD_BUFFERS = [(dict(k=None), ARG), (dict(v=None), ARG), (dict(k=FAKE + 8), ARG), (dict(dtype=2, ks=None), ARG),
               (dict(dtype=2, vs=FAKE + 4), ARG)]


def _attend(L, c, **kw):
    a = dict(layer=0, q=FAKE, qdt=0, qld=128, heads=4, nk=FAKE, nv=FAKE, ndt=1, nld=128, table=FAKE, ld=8, lens=FAKE, S=6,
             group=3, top=128, scale=0.2, out=FAKE, odt=0, old=128, ws=FAKE, bytes=1 << 40)
    a.update(kw)
    return L.pd_cache_attend(ctypes.byref(c), a["layer"], a["q"], a["qdt"], a["qld"], a["heads"], a["nk"], a["nv"],
                             a["ndt"], a["nld"], a["table"], a["ld"], a["lens"], a["S"], a["group"], a["top"], a["scale"],
                             a["out"], a["odt"], a["old"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw,status", BAD_CACHES + BAD_BUFFERS)
def test_every_call_checks_the_cache(kw, status):
    L = _lib()
    c = _cache(**kw)
    n = ctypes.c_size_t()
    assert _attend(L, c) == status
    assert L.pd_cache_read(ctypes.byref(c), 0, FAKE, 8, FAKE, 6, FAKE, 1, FAKE, FAKE, None) == status
    assert L.pd_pages_fork(ctypes.byref(c), FAKE, 8, FAKE, 6, FAKE, 6, 1, 2 * FAKE, 2 * FAKE, FAKE, FAKE, FAKE, 1 << 40,
                           None) == status
    assert L.pd_pages_compact(ctypes.byref(c), FAKE, 8, FAKE, 6, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == status
    if (kw, status) in BAD_CACHES:
        assert L.pd_cache_bytes(ctypes.byref(c), ctypes.byref(n), ctypes.byref(n)) == status
        assert L.pd_cache_attend_bytes(ctypes.byref(c), 4, 6, 3, 128, ctypes.byref(n)) == status
        assert L.pd_pages_bytes(ctypes.byref(c), 6, ctypes.byref(n)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(layer=-1), ARG), (dict(layer=2), ARG), (dict(q=None), ARG), (dict(out=None), ARG), (dict(qdt=2), ARG),
    (dict(odt=2), ARG), (dict(heads=6), ARG), (dict(heads=0), ARG), (dict(heads=68, qld=4096, old=4096), UNSUPPORTED),
    (dict(S=0), ARG), (dict(group=0), ARG), (dict(group=4), ARG), (dict(top=0), ARG), (dict(top=(1 << 30) + 1), SHAPE),
    (dict(S=3 << 20), SHAPE), (dict(table=None), ARG), (dict(lens=None), ARG), (dict(ld=0), ARG),
    (dict(ld=1 << 27), SHAPE), (dict(qld=120), ARG), (dict(old=127), ARG), (dict(qld=132), ARG), (dict(q=FAKE + 4), ARG),
    (dict(out=FAKE + 8), ARG), (dict(nk=None), ARG), (dict(nv=None), ARG), (dict(ndt=2), ARG), (dict(nld=64), ARG),
    (dict(nld=130), ARG), (dict(nk=FAKE + 2), ARG), (dict(scale=math.inf), ARG), (dict(scale=math.nan), ARG)])
def test_attention_refuses(kw, status):
    assert _attend(_lib(), _cache(), **kw) == status


def test_page_calls_refuse():
    L = _lib()
    c = _cache()
    B = ctypes.byref(c)

    def fork(table=FAKE, ld=8, lens=FAKE, n=6, par=FAKE, n_out=6, ot=2 * FAKE, ol=2 * FAKE, refs=FAKE, st=FAKE, ws=FAKE,
             size=1 << 40):
        return L.pd_pages_fork(B, table, ld, lens, n, par, n_out, 1, ot, ol, refs, st, ws, size, None)

    for kw, status in [(dict(table=None), ARG), (dict(lens=None), ARG), (dict(par=None), ARG), (dict(ot=None), ARG),
                       (dict(ol=None), ARG), (dict(refs=None), ARG), (dict(st=None), ARG), (dict(ld=0), ARG),
                       (dict(n=0), ARG), (dict(n_out=0), ARG), (dict(n_out=(1 << 22) + 1), SHAPE), (dict(ot=FAKE), ARG),
                       (dict(ot=FAKE + 4 * 8 * 6 - 4), ARG), (dict(ol=FAKE + 4), ARG), (dict(ws=None), WORKSPACE),
                       (dict(size=8), WORKSPACE)]:
        assert fork(**kw) == status, kw

    def compact(table=FAKE, ld=8, lens=FAKE, n=6, ot=2 * FAKE, remap=FAKE, st=FAKE, ws=FAKE, size=1 << 40):
        return L.pd_pages_compact(B, table, ld, lens, n, ot, remap, st, ws, size, None)

    for kw, status in [(dict(table=None), ARG), (dict(lens=None), ARG), (dict(ot=None), ARG), (dict(remap=None), ARG),
                       (dict(st=None), ARG), (dict(n=0), ARG), (dict(ot=FAKE + 4), ARG), (dict(ws=None), WORKSPACE),
                       (dict(size=8), WORKSPACE)]:
        assert compact(**kw) == status, kw
    read = lambda **k: L.pd_cache_read(B, k.get("layer", 0), FAKE, 8, FAKE, 6, k.get("first", FAKE),  # noqa: E731
                                       k.get("count", 1), k.get("k", FAKE), FAKE, None)
    for kw in (dict(layer=2), dict(first=None), dict(count=0), dict(k=None)):
        assert read(**kw) == ARG, kw


def test_sizes_of_a_cache():
    L = _lib()
    kv, sc = ctypes.c_size_t(), ctypes.c_size_t()
    n = 2 * 10 * 4
    for dtype, dh, page, scale in ((0, 32, 16 * 32 * 4, 0), (1, 16, 16 * 16 * 2, 0), (2, 16, 16 * 8, 16 * 4),
                                   (2, 64, 16 * 32, 16 * 2 * 4), (2, 128, 16 * 64, 16 * 4 * 4)):
        assert L.pd_cache_bytes(ctypes.byref(_cache(dtype=dtype, dh=dh, k=None, v=None)), ctypes.byref(kv),
                                ctypes.byref(sc)) == 0
        assert (kv.value, sc.value) == (n * page, n * scale)


def test_wrappers_refuse_what_is_not_on_a_gpu_or_of_another_type():
    _lib()
    x, s = torch.zeros(2, 4, 100), torch.zeros(2, 4)
    i = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(pdec.PdError):
        pdec.beam_select(x, s, i, i)                       # CPU tensors
    with pytest.raises(pdec.PdError):
        pdec.beam_select(x.double(), s, i, i)
    with pytest.raises(pdec.PdError):
        pdec.PagedCache("fp8", 1, 4, 16, 4, 32, device="cpu")
    with pytest.raises(pdec.PdError) as e:
        pdec.PagedCache("bf16", 1, 4, 17, 4, 32, device="cpu")
    assert e.value.status == UNSUPPORTED
    with pytest.raises(pdec.PdError):
        pdec.PagedCache("bf16", 1, 4, 16, 4, 32, k=torch.zeros(1, 4, 4, 16, 32))


# --- the references ---------------------------------------------------------------


def test_reference_packing_and_quantisation():
    g = np.random.default_rng(3)
    code = g.integers(0, 16, (5, 64))
    np.testing.assert_array_equal(R.unpack(R.pack(code)), code)
    w = R.pack(np.arange(8)[None]).view(np.uint32)[0, 0]          # two neighbours of a word in its two halves
    for j in range(4):
        assert ((w >> (4 * j)) & 0x000F000F) == (2 * j) | ((2 * j + 1) << 16)
    x = g.normal(size=(50, 128)) * np.exp(g.normal(size=(50, 1)) * 3) + g.normal(size=(50, 1)) * 10
    code, step, least = R.quantise(x)
    assert (np.abs(R.dequantise(code, step, least) - x) <= np.repeat(step, 32, -1) / 2 * (1 + 1e-12)).all()
    for y in (step, least):                                        # bfloat16 values
        t = torch.from_numpy(y)
        assert torch.equal(t.to(torch.bfloat16).double(), t)
    c, s, l = R.quantise(np.full((1, 32), 0.375))
    assert s[0, 0] == 0 and (R.dequantise(c, s, l) == 0.375).all()


def test_reference_selection_by_hand():
    no = -np.inf
    logits = np.array([[[no, 0.0, 0.0], [0.0, 0.0, no]]])          # four continuations of probability 1/2
    S, par, tok, ln, dn, src, fl = R.select(logits, np.array([[-1.0, -1.0]]), np.array([[3, 3]]), np.zeros((1, 2), int), 1,
                                            0, 0.0)
    np.testing.assert_allclose(S, [[-1 - math.log(2)] * 2])        # ties to the lower beam, then the lower word
    assert par.tolist() == [[0, 0]] and tok.tolist() == [[1, 2]] and dn.tolist() == [[1, 0]] and src.tolist() == [[-1, 0]]
    S, par, tok, ln, dn, src, fl = R.select(logits, np.array([[-1.0, -9.0]]), np.array([[2, 3]]), np.array([[1, 0]]), 1, 0,
                                            1.0)
    assert par.tolist() == [[0, 1]] and tok.tolist() == [[0, 0]] and ln.tolist() == [[2, 4]] and dn.tolist() == [[1, 0]]
    S, par, *_ = R.select(logits[:, :, 1:2], np.array([[0.0, no]]), np.zeros((1, 2), int), np.zeros((1, 2), int), 1, 0, 1.0)
    assert S.tolist() == [[0.0, no]] and par.tolist() == [[0, -1]]
    assert R.select(np.array([[[math.nan, 1.0]]]), np.zeros((1, 1)), np.zeros((1, 1)), np.zeros((1, 1), int), 5, 0, 1.0)[6] == [8]


def test_reference_fork_by_hand():
    t = np.array([[5, 2, -1], [5, 3, -1]])
    # both children of row 0, 20 tokens in pages of 16: the first keeps page 2, the second copies it to page 0
    new, ln, refs, st, cp = R.fork(t, [20, 20], [0, 0], 6, 16, True)
    assert new.tolist() == [[5, 2, -1], [5, 0, -1]] and ln.tolist() == [21, 21] and cp == [(2, 0)]
    assert refs.tolist() == [1, 0, 1, 0, 0, 2] and st == [0, 3]
    new, ln, refs, st, cp = R.fork(t, [32, 20], [0, -1], 6, 16, True)
    assert new.tolist() == [[5, 2, 0], [-1, -1, -1]] and ln.tolist() == [33, 0] and cp == []
    assert R.fork(t, [32, 32], [0, 1], 6, 16, True)[3] == [0, 5]
    assert R.fork(t, [32, 32], [0, 1], 4, 16, True)[3] == [0, 4]            # page 5 is outside a pool of four: left out
    new, _, _, st, _ = R.fork(np.array([[1, 2], [0, 3]]), [32, 31], [0, 1], 4, 16, True)
    assert st == [1, 0] and (new == -1).all()


def test_reference_compaction_by_hand():
    new, remap, st, mv = R.compact(np.array([[7, 1, 4], [7, 6, 2]]), [33, 30], 8, 16)
    assert mv == [(4, 0), (6, 2), (7, 3)] and st == [3, 4]          # page 2 is behind its sequence's end: a hole
    assert new.tolist() == [[3, 1, 0], [3, 2, -1]] and remap.tolist() == [-1, 1, -1, -1, 0, -1, 2, 3]
