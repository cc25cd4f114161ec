"""Memory of beam decoding's Python call (Context.decode_beam)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2305_10427_amd import configs as C, pdec
from tests.test_gpu_beam import Fixture, encode, fixture, run, sources

pytestmark = pytest.mark.gpu


def test_what_a_call_uses_is_allocated_on_its_stream(monkeypatch):
    """The allocator orders a block's next use after its last one on the same stream only: a workspace allocated on
    another stream than the call's could be written while that stream still reads what lay there."""
    f = fixture(C.TINY, 4.0)
    ctx = pdec.Context(f.ctx.model, 4, 24, 40)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        encode(ctx, sources(C.TINY, [16, 3], 65))
    made, real = [], torch.empty

    def empty(*a, **k):
        made.append((k.get("dtype"), torch.cuda.current_stream().cuda_stream))
        return real(*a, **k)

    monkeypatch.setattr(torch, "empty", empty)
    ctx.decode_beam([9, 6], beam=3, stream=s)
    s.synchronize()
    assert torch.uint8 in [d for d, _ in made]
    assert {at for _, at in made} == {s.cuda_stream}


def test_a_context_keeps_one_workspace():
    """Whatever widths and cache types it has decoded with: the largest one's, which serves the others too."""
    f = fixture(C.TINY, 4.0)
    ctx = pdec.Context(f.ctx.model, 4, 24, 40)
    g = Fixture(f.cfg, ctx, f.M)
    srcs, ms = sources(C.TINY, [16, 3, 24], 15), [12, 9, 6]
    n, most = ctypes.c_size_t(), 0
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    first = {}
    for beam, cache in ((2, "native"), (9, "int4"), (3, "int4"), (12, "native"), (5, "native"), (2, "native"), (9, "int4"), (12, "native")):
        out = run(g, srcs, ms, beam=beam, cache=cache)
        assert pdec.load_library().pd_decode_beam_bytes(ctx.handle, beam, pdec.CACHE_TYPES["f32" if cache == "native" else cache],
                                                        ctypes.byref(n)) == 0
        most = max(most, n.value)
        torch.cuda.synchronize()
        assert torch.cuda.memory_allocated() - before <= most + (64 << 10)       # the sources and rounding besides
        for a, b in zip(first.setdefault((beam, cache), out), out):
            np.testing.assert_array_equal(a, b)
    for (beam, cache), want in first.items():                  # as a workspace of a call's own gives
        for a, b in zip(run(f, srcs, ms, beam=beam, cache=cache), want):
            np.testing.assert_array_equal(a, b)
