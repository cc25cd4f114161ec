"""The beam-search operators at the edges of their ranges, on the GPU."""
import numpy as np
import pytest
import torch

from tests import attend_error as E, operators_ref as R
from tests.test_gpu_operators import Pool, gpu, host, i32, say, tree_tables

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


def codes(pool, name):
    """(codes, steps, least) of the keys or values of layer 0 of a pool in 4 bits, [pages][kv][ps][dh or groups]."""
    c = R.unpack(getattr(pool.cache, name)[0].cpu().numpy())
    par = getattr(pool.cache, name + "_scale")[0].double().cpu().numpy()
    return (c.swapaxes(-1, -2) if name == "v" else c), par[..., 0], par[..., 1]


def deviations(pool, q, out, table, lens, scale=None):
    """(out - exact) / deviation of every sequence and head (layer 0)."""
    scale = pool.dh ** -0.5 if scale is None else scale
    got, qh, z = host(out), host(q), []
    H = qh.shape[1]
    par = {n: codes(pool, n) for n in "kv"} if pool.dtype == "int4" else {}
    for s, n in enumerate(lens):
        row, slot = [table[s, j // pool.ps] for j in range(n)], [j % pool.ps for j in range(n)]
        for h in range(H if n else 0):
            kh = h // (H // pool.kv)
            of = lambda x: x[row, kh, slot]  # noqa: B023, E731
            kw = {a + "_par": tuple(of(x) for x in t) for a, t in par.items()}
            ref, sd, _ = E.attend(pool.dtype, qh[s, h], of(pool.k[0]), of(pool.v[0]), scale, **kw)
            z.append((got[s, h] - ref) / sd)
    return z


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_scores_in_4_bits_take_a_querys_whole_sum(dh):
    """Queries whose sum over a group needs more bits than a float has: 1 and values of a little less than half its
    last place, which a float sum of them drops.  The keys' steps differ, so what is dropped moves the weights."""
    g = np.random.default_rng(dh)
    n, ps, kv = 96, 32, 2
    pool = Pool(g, "int4", 1, 3, ps, kv, dh)
    step = torch.from_numpy(np.where(g.random(pool.cache.k_scale.shape[:-1]) < 0.5, 2.0 ** -6, 1.0)).cuda()
    pool.cache.k_scale[..., 0] = step
    pool.cache.k_scale[..., 1] = -7.5 * step
    c, st, least = codes(pool, "k")
    c[..., ::8] = 7 + g.integers(0, 2, c[..., ::8].shape)        # scores of little spread: every key has a weight
    pool.cache.k[0].copy_(torch.from_numpy(R.pack(c)))
    pool.k = R.dequantise(c, st, least)[None]
    q = np.full((2, kv, dh), 1.9 * 2.0 ** -25)
    q[..., ::8] = 1.0
    q[1] *= -1
    q = gpu(q, torch.float32)
    table, lens, scale = np.tile(np.arange(3), (2, 1)), [n, n - 5], 0.6932 * 32 / dh      # scale log2(e) just above a power of two
    z = deviations(pool, q, pool.cache.attend(q, i32(table), i32(lens), scale=scale), table, lens, scale)
    say("deviations", dh, float(np.sqrt((np.array(z) ** 2).mean())), float(np.abs(z).max()))
    assert E.fits(z)
