"""The beam-search operators at the edges of their ranges, on the GPU."""
import numpy as np
import pytest
import torch

from tests.test_gpu_operators import Pool, gpu, i32, say, tree_tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache,kv,dh,ps,group,lens", [
    ("bf16", 8, 64, 16, 5, [138, 40, 17, 90, 138]), ("bf16", 2, 128, 32, 1, [4001, 2999]), ("bf16", 4, 32, 16, 2, [33, 64]),
    ("bf16", 1, 16, 64, 1, [700]), ("int4", 8, 64, 16, 5, [200, 250, 31, 256, 1]), ("int4", 2, 128, 64, 2, [5001, 4000]),
    ("int4", 4, 32, 16, 1, [77]), ("int4", 2, 16, 16, 1, [300, 5]), ("f32", 2, 64, 16, 1, [50, 1000])])
def test_bfloat16_outputs_are_the_float_ones_rounded_once(cache, kv, dh, ps, group, lens):
    """The sums are held in float whatever the output's type: one rounding at the end, no other difference."""
    g = np.random.default_rng(dh + len(lens))
    ld = -(-max(lens) // ps)
    pages = sum(-(-n // ps) for n in lens)
    pool = Pool(g, cache, 1, pages, ps, kv, dh)
    table = tree_tables(g, lens, group, ps, pages, True, ld)
    q = gpu(2 * g.normal(size=(len(lens), 2 * kv, dh)), torch.float32)
    run = lambda t: pool.cache.attend(q, i32(table), i32(lens), group=group, out_dtype=t)  # noqa: E731
    say("rounded once", cache, dh, lens)
    assert int((run(torch.bfloat16) != run(torch.float32).to(torch.bfloat16)).sum()) == 0
