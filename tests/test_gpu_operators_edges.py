"""The beam-search operators at the edges of their ranges, on the GPU."""
import numpy as np
import pytest
import torch

from paper_2305_10427_amd import pdec
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


@pytest.mark.parametrize("cache", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [16, 32, 64, 128])
def test_infinite_keys_and_values(cache, dh):
    """A value of inf with a weight is inf, inf and -inf together NaN; a key whose score is -inf has no weight, whether
    the key is infinite or the finite product overflows however far; a score of inf makes the row NaN."""
    g = np.random.default_rng(dh)
    ps, kv, pages = 16, 2, 40
    top = float(torch.finfo(torch.bfloat16).max)
    for q_in in (1.0, -0.3, 2.0 ** 30):
        pool = Pool(g, cache, 1, pages, ps, kv, dh)
        if abs(q_in) > 1:                                      # scores of the usual keys stay small
            pool.cache.k.mul_(1 / q_in)
        lens = [1, 37, 37, 20, 64, 64, 5, 3]
        table = np.arange(pages).reshape(8, 5)
        kc, vc = pool.cache.k[0], pool.cache.v[0]              # [pages][kv][ps][dh], [pages][kv][dh][ps]
        at = lambda s, j: (table[s, j // ps], j % ps)  # noqa: E731
        for s, j, d, x in ((0, 0, 3, np.inf), (1, 5, 0, -np.inf), (1, 36, 1, np.inf), (2, 3, 2, np.inf), (2, 20, 2, -np.inf)):
            p, t = at(s, j)
            vc[p, :, d, t] = x
        for s, j, x in ((3, 4, -np.inf), (4, 0, -2.0 ** 120), (4, 1, -top), (4, 40, -2.0 ** 100), (6, 2, np.inf)):
            p, t = at(s, j)
            kc[p, :, t] = x * np.sign(q_in)
        for j in range(64):                                    # no key with a weight: the row is zero
            p, t = at(5, j)
            kc[p, :, t] = (-np.inf if j % 3 else -top if abs(q_in) > 1 else -np.inf) * np.sign(q_in)
        for j in range(3):
            p, t = at(7, j)
            kc[p, :, t] = -np.inf * np.sign(q_in)
        q = gpu(np.full((8, 4, dh), q_in), torch.float32)
        say("infinite", cache, dh, q_in)
        for group in (1, 4):
            out = host(pool.cache.attend(q, i32(table), i32(lens), group=group))
            z = []
            for s, n in enumerate(lens):
                row, slot = [at(s, j)[0] for j in range(n)], [j % ps for j in range(n)]
                for h in range(4):
                    k, v = host(kc)[row, h // 2, slot], host(vc)[row, h // 2, :, slot]
                    sc = dh ** -0.5 * (k @ np.full(dh, float(np.float32(q_in))))
                    sc[sc < -np.finfo(np.float32).max] = -np.inf
                    if (sc == np.inf).any():
                        assert np.isnan(out[s, h]).all()
                        continue
                    keep = sc > -np.inf
                    if not keep.any():
                        assert (out[s, h] == 0).all()
                        continue
                    w = np.exp(sc - sc.max()) / np.exp(sc - sc.max()).sum()
                    assert (w[~np.isfinite(v).all(-1)] > 1e-20).all()      # an infinite value with no weight is not asked
                    with np.errstate(invalid="ignore"):
                        want = w[keep] @ v[keep]
                    usual = np.isfinite(want)
                    np.testing.assert_array_equal(out[s, h][~usual], want[~usual])
                    v = np.where(np.isfinite(v), v, 0.0)
                    ref, sd, _ = E.attend(cache, np.full(dh, float(np.float32(q_in))), k[keep], v[keep], dh ** -0.5)
                    z.append(((out[s, h] - ref) / sd)[usual])
            assert E.fits(z)


@pytest.mark.parametrize("pages", [40, 9000])
def test_compaction_of_lengths_beyond_the_table(pages):
    """A length names at most the table's row, however large it is, and none if it is negative."""
    g = np.random.default_rng(pages)
    ps, ld = 16, 3
    lens = [2 ** 31 - 1, 2 ** 31 - ps, -2 ** 31, ld * ps + 1, 2 ** 30, 0, -1, ld * ps, 17]
    table = g.permutation(pages)[:len(lens) * ld].reshape(len(lens), ld)
    pool = Pool(g, "bf16", 2, pages, ps, 1, 16)
    before = {n: t.clone() for n, t in pool.tensors().items()}
    r = pool.cache.compact(i32(table), i32(lens))
    new, remap, st, mv = R.compact(table, np.clip(lens, 0, ld * ps), pages, ps)
    np.testing.assert_array_equal(host(r.table), new)
    np.testing.assert_array_equal(host(r.remap), remap)
    assert r.status.tolist() == st and st[1] == 5 * ld + 2
    for n, t in before.items():
        for a, b in mv:
            t[:, b] = t[:, a]
        assert torch.equal(t, pool.tensors()[n])


@pytest.mark.parametrize("dh", [16, 32, 128])
def test_append_in_4_bits_over_floats_whole_range(dh):
    """Every finite value is held within half a step of its group, also where the range or fifteen steps are beyond
    float's largest value; values below bfloat16's lowest count as that."""
    top, low = float(torch.finfo(torch.float32).max), -float(torch.finfo(torch.bfloat16).max)
    tiny = 2.0 ** -149
    w = min(dh, 32)
    line = lambda a, b: np.linspace(a, b, w)  # noqa: E731
    rows = [line(-3e38, 3e38), line(-top, top), line(0, top), line(-top, 0), np.full(w, -top), np.full(w, top), line(low, 1e38),
            np.where(np.arange(w) % 2, 1.0, top), np.where(np.arange(w) % 3, -1.0, -top), line(0, 9 * tiny), line(-5 * tiny, 0),
            line(2.0 ** -126, 2.0 ** -120), line(-1e-40, 3e-39), np.array([-3e38, 1e38, 3e38, 0.0] * (w // 4)), line(1e38, 1.1e38)]
    x = np.stack([np.roll(np.tile(r, (2, dh // w)), i, 1) for i, r in enumerate(rows)]).astype(np.float32)    # [S][kv 2][dh]
    S = len(rows)
    pool = Pool(np.random.default_rng(dh), "int4", 1, S, 16, 2, dh)
    t, n = i32(np.arange(S)[:, None]), i32([1 + i for i in range(S)])
    pool.cache.attend(torch.zeros(S, 2, dh, device="cuda"), t, n, new_k=gpu(x), new_v=gpu(-x))
    for name, want, got in zip("kv", (x, -x), pool.cache.read(t, n, n - 1)):
        want, got = np.maximum(want.astype(np.float64), low).reshape(S, 2, -1, w), host(got)[:, 0].reshape(S, 2, -1, w)
        # bfloat16 below 2^-126: the multiples of 2^-133 (exponent -126, seven places), coarser than eight places of the value
        small = 2.0 ** -133
        least = np.minimum(np.maximum(R.bf16_down(want.min(-1)), low), np.floor(want.min(-1) / small) * small)
        step = np.maximum(R.bf16_up((want.max(-1) - least) / 15), np.ceil((want.max(-1) - least) / 15 / small) * small)
        # half a step; a difference, its quotient and the value read are rounded (u of the range each, or to a multiple of tiny)
        tol = (step / 2 + 2.0 ** -24 * (2 * 15 * step + np.abs(want).max(-1)) + tiny)[..., None]
        err = np.abs(got - want)
        say(name, dh, float((err / tol).max()))
        assert np.isfinite(got).all() and (err <= tol).all(), np.argwhere(~(err <= tol))[:5]


@pytest.mark.parametrize("call", ["attend", "append", "read", "fork", "compact", "select"])
def test_inputs_of_a_call_on_another_stream_may_be_dropped_at_once(call):
    """The call waits on its stream; meanwhile its inputs go, and what the current stream allocates next is overwritten."""
    g = np.random.default_rng(7)
    S, H, dh, ps, ld = 6, 4, 64, 16, 8
    table = g.permutation(S * ld + 20)[:S * ld].reshape(S, ld)
    lens = [100, 64, 1, 127, 33, 90]

    def inputs():
        r = np.random.default_rng(8)
        pool = Pool(r, "bf16", 1, S * ld + 20, ps, H, dh).cache
        q, k, v = (gpu(r.normal(size=(S, H, dh)), torch.float32) for _ in range(3))
        t, n, par = i32(table), i32(lens), i32([0, 0, 3, 5, -1, 1])
        x, z, i = gpu(r.normal(size=(2, 3, 5000)), torch.float32), torch.zeros(2, 3, device="cuda"), i32(np.zeros((2, 3)))
        return {"attend": lambda **o: pool.attend(q, t, n, **o), "append": lambda **o: pool.attend(q, t, n, new_k=k, new_v=v, **o),
                "read": lambda **o: pool.read(t, n, n - 1 if not o else first, **o), "fork": lambda **o: pool.fork(t, n, par, **o),
                "compact": lambda **o: pool.compact(t, n, **o), "select": lambda **o: pdec.beam_select(x, z, i, i, **o)}[call]

    first = i32(lens) - 1
    whole = lambda out: [out] if torch.is_tensor(out) else list(out)  # noqa: E731
    want = [t.clone() for t in whole(inputs()())]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    f = inputs()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)                         # about a tenth of a second
    out = whole(f(stream=s))
    del f
    junk = [torch.full((n,), 113, dtype=torch.uint8, device="cuda") for n in [1 << 9] * 40 + [1 << 14] * 40 + [1 << 17] * 20 + [1 << 19] * 20]
    torch.cuda.synchronize()
    del junk
    for a, b in zip(out, want):
        assert torch.equal(a, b)


def test_calls_on_a_given_stream_can_be_captured():
    """Captured on a stream that the calls are given too; every replay equals the eager calls made between them."""
    g = np.random.default_rng(51)
    pool = Pool(g, "int4", 1, 64, 16, 4, 64).cache
    t, n = i32(np.arange(60).reshape(4, 15)), i32([200, 100, 50, 180])
    q = gpu(g.normal(size=(4, 8, 64)), torch.float32)
    x, z, i = gpu(3 * g.normal(size=(4, 1, 40001)), torch.float32), torch.zeros(4, 1, device="cuda"), i32(np.zeros((4, 1)))
    s = torch.cuda.Stream()

    def run(**o):
        return (pool.attend(q * 0.5, t, n, **o), *pdec.beam_select(x, z, i, i, **o), *pool.fork(t, n, i[:, 0] + 1, grow=False, **o),
                *pool.read(t, n, n - 1, **o))

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = run(stream=s)
    for k in range(4):
        q.copy_(gpu(g.normal(size=(4, 8, 64)), torch.float32))
        x.mul_(-0.9)
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k


@pytest.mark.parametrize("cache,n_in,pages", [("f32", 12, 90), ("bf16", 30, 200), ("int4", 12, 90), ("int4", 40, 8500), ("bf16", 2100, 9000)])
def test_fork_at_page_borders_and_full_rows(cache, n_in, pages):
    """Lengths that end a page (a fresh page), lie inside one (kept or copied), are none, or fill the table's row (refused)."""
    g = np.random.default_rng(n_in + pages)
    seen = {"border": 0, "inside": 0, "none": 0, "full": 0, "copied": 0, "kept": 0, "refused": 0, "grown": 0}
    for trial in range(12 if n_in < 100 else 3):
        ps, ld = int(g.choice([16, 64])), 4
        lens = g.integers(0, ld, n_in) * ps
        inside = g.random(n_in) < 0.4
        lens[inside] = g.integers(0, ld, inside.sum()) * ps + g.integers(1, ps, inside.sum())
        if trial % 3 == 2:
            lens[int(g.integers(0, n_in))] = ld * ps
        table, ids = np.full((n_in, ld), -1, np.int64), iter(g.permutation(pages))
        for s in range(n_in):
            for j in range(-(-int(lens[s]) // ps)):
                share = s and g.random() < 0.5 and table[s - 1, j] >= 0 and (j < lens[s] // ps) == (j < lens[s - 1] // ps)
                table[s, j] = table[s - 1, j] if share else next(ids, -1)
        parents = g.integers(0, n_in, n_in)
        parents[:n_in // 4] = -1                               # finished hypotheses
        if trial % 3 == 2:
            parents[-1] = int(np.argmax(lens))
        pool = Pool(g, cache, 2, pages, ps, 1, 16)
        before = {n: t.clone() for n, t in pool.tensors().items()}
        r = pool.cache.fork(i32(table), i32(lens), i32(parents))
        new, ln, refs, st, cp = R.fork(table, lens, parents, pages, ps, True)
        for got, want in ((r.table, new), (r.lens, ln), (r.refs, refs)):
            np.testing.assert_array_equal(host(got), want)
        assert r.status.tolist() == st
        for n, t in before.items():
            for a, b in cp:
                t[:, b] = t[:, a]
            assert torch.equal(t, pool.tensors()[n])
        n = lens[parents[parents >= 0]]
        seen["full"] += int((n == ld * ps).sum())
        seen["none"] += int((n == 0).sum())
        seen["border"] += int(((n % ps == 0) & (n > 0) & (n < ld * ps)).sum())
        seen["inside"] += int((n % ps > 0).sum())
        seen["refused"] += st[0] > 0
        seen["grown"] += st[0] == 0
        seen["copied"] += len(cp)
        seen["kept"] += int((n % ps > 0).sum()) - len(cp) if st[0] == 0 else 0
    say(cache, n_in, pages, seen)
    assert min(seen.values()) > 0


def test_tensors_that_require_a_gradient_are_refused():
    """The operators have no backward pass: a graph is never cut silently."""
    c = pdec.PagedCache("f32", 1, 4, 16, 2, 16)
    t, n, i = i32([[0], [1]]), i32([3, 4]), i32([[0], [0]])
    q, k, x, z = (torch.ones(*shape, device="cuda") for shape in ((2, 4, 16), (2, 2, 16), (2, 1, 50), (2, 1)))
    grad = lambda a: a.clone().requires_grad_()  # noqa: E731
    calls = [lambda f: c.attend(f(q), t, n), lambda f: c.attend(q, t, n, new_k=f(k), new_v=k), lambda f: c.attend(q, t, n, new_k=k, new_v=f(k)),
             lambda f: pdec.beam_select(f(x), z, i, i).scores, lambda f: pdec.beam_select(x, f(z), i, i).scores,
             lambda f: pdec.PagedCache("f32", 1, 4, 16, 2, 16, k=f(c.k)).attend(q, t, n),
             lambda f: pdec.PagedCache("f32", 1, 4, 16, 2, 16, v=f(c.v)).attend(q, t, n)]
    for call in calls:
        with pytest.raises(pdec.PdError) as e:
            call(grad)
        assert e.value.status == 5
        with torch.no_grad():
            a = call(grad)
        assert torch.equal(a, call(lambda x: grad(x).detach())) and not a.requires_grad


def test_arguments_that_are_no_tensors_are_refused():
    c = pdec.PagedCache("bf16", 1, 4, 16, 2, 16)
    t, n, q, k = i32([[0], [1]]), i32([3, 4]), torch.ones(2, 4, 16, device="cuda"), torch.ones(2, 2, 16, device="cuda")
    x, z, i = torch.ones(2, 1, 50, device="cuda"), torch.ones(2, 1, device="cuda"), i32([[0], [0]])
    for bad in (None, [[0], [1]], np.zeros((2, 1), np.int32), 3.0):
        for call in (lambda: c.attend(bad, t, n), lambda: c.attend(q, bad, n), lambda: c.attend(q, t, bad), lambda: c.fork(t, n, bad),
                     lambda: c.fork(bad, n, n), lambda: c.compact(bad, n), lambda: c.compact(t, bad), lambda: c.read(t, n, bad),
                     lambda: c.read(bad, n, n), lambda: pdec.beam_select(bad, z, i, i), lambda: pdec.beam_select(x, bad, i, i),
                     lambda: pdec.beam_select(x, z, bad, i), lambda: pdec.beam_select(x, z, i, bad), lambda: c.attend(q, t, n, new_k=k, new_v=[1])):
            with pytest.raises(pdec.PdError):
                call()
