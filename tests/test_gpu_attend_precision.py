"""Attention over the paged cache on the GPU within the errors of float arithmetic (tests/attend_error.py): every shape
of the comparison with 64 bits, at bounds that a dropped key or a query of fewer bits does not meet
(tests/test_attend_error.py)."""
import numpy as np
import pytest
import torch

from tests import attend_error as E, operators_ref as R
from tests.test_gpu_operators import ATTEND, TYPES, Pool, gpu, host, i32, say, tree_tables
from tests.test_gpu_operators_edges import codes, deviations

pytestmark = pytest.mark.gpu

MORE = [
    ("int4", 8, 8, 64, 16, 5, [200, 250, 31, 256, 1], True, "f32", "f32"),
    ("int4", 16, 4, 128, 64, 1, [4001, 20011], False, "f32", "f32"),
    ("bf16", 16, 16, 64, 32, 1, [16381], False, "f32", "f32"),
    ("bf16", 8, 2, 128, 16, 2, [5000, 4999], True, "f32", "f32"),
    ("f32", 4, 2, 128, 64, 1, [9001], False, "f32", "f32"),
    ("f32", 8, 8, 64, 16, 4, [4000] * 4, True, "f32", "f32"),
]


def made(case, layers=1):
    cache, H, kv, dh, ps, group, lens, share, qt, _ = case
    g = np.random.default_rng(1000 + dh + sum(lens))
    ld = -(-max(max(lens), 1) // ps) + 1
    pages = sum(-(-n // ps) for n in lens) + 3
    return g, Pool(g, cache, layers, pages, ps, kv, dh), tree_tables(g, lens, group, ps, pages, share, ld)


def report(z):
    z = np.concatenate([np.ravel(x) for x in z])
    say(f"  deviations: rms {np.sqrt((z ** 2).mean()):.2f}, most {np.abs(z).max():.2f}")


@pytest.mark.parametrize("case", ATTEND + MORE, ids=lambda c: f"{c[0]}-h{c[1]}:{c[2]}x{c[3]}-p{c[4]}-g{c[5]}-{max(c[6])}")
def test_attention_is_as_exact_as_float(case):
    cache, H, kv, dh, ps, group, lens, share, qt, _ = case
    g, pool, table = made(case)
    for size in (0.5, 2.0):                                    # weights of like size, and few large ones
        q = gpu(size * g.normal(size=(len(lens), H, dh)), TYPES[qt])
        say("attend", case, size)
        out = pool.cache.attend(q, i32(table), i32(lens), group=group, out_dtype=torch.float32)
        z = deviations(pool, q, out, table, lens)
        report(z)
        assert E.fits(z)
        for s, n in enumerate(lens):
            assert n > 0 or not out[s].any()
        half = pool.cache.attend(q, i32(table), i32(lens), group=group, out_dtype=torch.bfloat16)
        assert int((half != out.to(torch.bfloat16)).sum()) == 0


@pytest.mark.parametrize("cache,kv,H,dh,ps", [("f32", 3, 6, 64, 16), ("bf16", 2, 8, 16, 32), ("bf16", 3, 3, 64, 16), ("bf16", 1, 4, 128, 64),
                                              ("int4", 3, 6, 16, 16), ("int4", 2, 2, 32, 32), ("int4", 3, 6, 64, 64), ("int4", 2, 8, 128, 16)])
def test_an_appended_token_has_its_weight(cache, kv, H, dh, ps):
    """The new key and value count as the cache holds them, also where a part of a long cache ends with them."""
    for lens in ([1, ps, ps + 1, 2 * ps - 1, 33, 64, 65, 7], [3001, 2049, 127, 128]):
        case = (cache, H, kv, dh, ps, 1, lens, False, "f32", "f32")
        g, pool, table = made(case)
        q, nk, nv = (gpu(0.5 * g.normal(size=(len(lens), h, dh)), torch.float32) for h in (H, kv, kv))
        say("append", case)
        out = pool.cache.attend(q, i32(table), i32(lens), new_k=nk, new_v=nv, out_dtype=torch.float32)
        for n in "kv":                                         # what the cache holds now
            if cache == "int4":
                setattr(pool, n, R.dequantise(*codes(pool, n))[None])
            else:
                t = getattr(pool.cache, n).double().cpu().numpy()
                setattr(pool, n, t.swapaxes(-1, -2) if n == "v" else t)
        for x, n in ((nk, "k"), (nv, "v")):
            x = host(x)
            for s, m in enumerate(lens):
                held = getattr(pool, n)[0, table[s, (m - 1) // ps], :, (m - 1) % ps]
                if cache == "int4":
                    code, step, least = R.quantise(x[s])
                    np.testing.assert_array_equal(held, R.dequantise(code, step, least))
                else:
                    np.testing.assert_array_equal(held, torch.from_numpy(x[s]).to(TYPES[cache]).double().numpy())
        z = deviations(pool, q, out, table, lens)
        report(z)
        assert E.fits(z)
