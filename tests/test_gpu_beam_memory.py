"""Memory of beam decoding's Python call (Context.decode_beam)."""
import numpy as np
import pytest
import torch

from paper_2305_10427_amd import configs as C, pdec
from tests.test_gpu_beam import encode, fixture, sources

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
