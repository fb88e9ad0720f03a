"""Eviction by mass (viscache_mass_evict) against the selection written out in numpy: kept
rows, masses, indices and lengths are equal bit for bit, and nothing else changes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2608_24063_amd as vc
    vc.lib()
    return torch.device("cuda:0")


def kept_rows(mass, k, sinks, recent):
    """The rows of a unit that stay, ascending."""
    n = len(mass)
    k = max(min(k, n), 0)
    a = min(sinks, k)
    z = min(recent, k - a)
    m = mass[a:n - z].astype(np.float64)
    m = np.where(np.isnan(m), -np.inf, np.where(np.isneginf(m), -1e300, m))  # NaN behind -inf
    order = np.argsort(-m, kind="stable")  # ties to the lower index
    return np.sort(np.concatenate((np.arange(a), a + order[:k - a - z], np.arange(n - z, n)))).astype(np.int64)


def _masses(rng, n, kind):
    m = np.exp(2 * rng.standard_normal(n))
    if kind == "ties":
        m = np.round(m * 2) / 2
    elif kind == "equal":
        m = np.full(n, 0.25)
    elif kind == "odd":  # zeros of both signs, negative values, infinities, NaN, subnormals
        m = rng.choice(np.array([0.0, -0.0, -1.0, np.inf, -np.inf, np.nan, 1e-42, 3.0]), n)
    elif kind == "near":  # values that differ in their last bits
        m = np.float32(1.0) + np.float32(2.0 ** -23) * rng.integers(0, 40, n)
    return m.astype(np.float32)


def _cache(rng, dev, L, B, Hkv, d, lens, caps, kind="plain"):
    from paper_2608_24063_amd.tensors import MassCache
    c = MassCache(L, B, Hkv, Hkv, d, caps, dev)
    g = torch.Generator(device=dev)
    g.manual_seed(int(rng.integers(0, 1 << 30)))
    for x in (c.k_pool, c.v_pool):
        x.view(torch.int16).random_(generator=g)
    mass = np.concatenate([_masses(rng, cap, kind) for cap in caps] + [np.zeros(0 if sum(caps) else 1, np.float32)])
    c.mass.copy_(torch.from_numpy(mass))
    c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    return c


def _state(c):
    return [x.view(torch.int16 if x.dtype is torch.bfloat16 else torch.int32).cpu().numpy().copy()
            for x in (c.k_pool, c.v_pool, c.mass)] + [c.len.cpu().numpy().copy()]


def _run(c, keep, sinks, recent, to=None, wide=None, max_rows=None):
    before, target = _state(c), _state(to if to is not None else c)
    lens, offs, caps = before[3].tolist(), c.row_off.tolist(), c.cap.tolist()
    t_off, t_cap = (to.row_off.tolist(), to.cap.tolist()) if to is not None else (offs, [1 << 31] * len(offs))
    index = None if wide is None else torch.full((len(lens), wide), -7, dtype=torch.int32, device=c.device)
    c.evict(torch.tensor(keep, dtype=torch.int32, device=c.device), sinks, recent, to=to, index=index, max_rows=max_rows)
    torch.cuda.synchronize()
    after, got = _state(c), _state(to if to is not None else c)
    if to is not None:
        assert all(np.array_equal(x, y) for x, y in zip(before, after))
    free = [np.ones(len(x), bool) for x in got[:3]]
    for u, n in enumerate(lens):
        n = max(min(n, caps[u], n if max_rows is None else max_rows), 0)
        o, t = offs[u], t_off[u]
        rows = kept_rows(before[2][o:o + n].view(np.float32), min(keep[u], t_cap[u]), sinks, recent)
        k = len(rows)
        for i, name in enumerate(("keys", "values", "masses")):
            assert np.array_equal(got[i][t:t + k], before[i][o + rows]), (u, n, k, name)
            free[i][t:t + (n if to is None else k)] = False
        assert got[3][u] == k, u
        if index is not None:
            row = index[u].tolist()
            m = min(k, wide)
            assert row[:m] == rows[:m].tolist() and row[m:] == [-7] * (wide - m), u
    for i in range(3):  # no row of another unit, or past this one's, was touched
        assert np.array_equal(got[i][free[i]], target[i][free[i]])


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "odd", "near"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inplace", [True, False])
def test_odd_sizes(dev, kind, d, inplace):
    rng = np.random.default_rng(3)
    lens = [0, 1, 2, 31, 64, 65, 127, 128, 129, 200, 257, 511, 700, 1023, 1025, 1500]
    caps = [x + int(rng.integers(0, 4)) for x in lens]
    for sinks, recent in ((0, 0), (4, 32), (3, 1000), (2000, 7)):
        for share in (0.0, 0.01, 0.5, 0.97, 1.0, 2.0):
            keep = [int(share * x + rng.integers(0, 2)) for x in lens]
            keep[5], keep[9] = -3, 2 ** 31 - 1
            c = _cache(rng, dev, 2, 2, 4, d, lens, caps, kind)
            to = None
            if not inplace:  # some of the other cache's units have too little room
                room = [max(min(k, x), 0) + int(rng.integers(-1, 3)) for k, x in zip(keep, lens)]
                to = _cache(rng, dev, 2, 2, 4, d, [0] * 16, [max(r, 0) for r in room])
            _run(c, keep, sinks, recent, to, wide=int(rng.choice([1, 40, 1500])))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inplace", [True, False])
def test_long_units(dev, d, inplace):
    """Many chunks a unit, from none moving to all, masses that keep the far end, a row bound."""
    rng = np.random.default_rng(5)
    for lens, share in (([40000, 3], 0.5), ([33000, 2500, 9000, 1], 0.9), ([2300] * 40, 0.03), ([8000] * 24, 0.6)):
        c = _cache(rng, dev, 1, 1, len(lens), d, lens, [x + 5 for x in lens], "ties")
        for bound in (None, 2100):
            if bound:
                c.len.copy_(torch.tensor(lens, dtype=torch.int32))
            keep = [int(share * x) for x in lens]
            to = None if inplace else _cache(rng, dev, 1, 1, len(lens), d, [0] * len(lens), [k + 1 for k in keep])
            _run(c, keep, 4, 32, to, wide=max(keep), max_rows=bound)
        # every row moves by one, and only the last ones stay
        c.len.copy_(torch.tensor(lens, dtype=torch.int32))
        off = c.row_off.long()
        c.mass.fill_(1.0)
        c.mass[off] = 0.0
        _run(c, [x - 1 for x in lens], 0, 0)
        _run(c, [x // 3 for x in lens], 0, max(lens))


def test_again_and_again(dev):
    """The cut repeated in place, until nothing is left."""
    rng = np.random.default_rng(7)
    lens = [5000, 700, 64, 3001]
    c = _cache(rng, dev, 1, 2, 2, 128, lens, lens, "ties")
    for share in (0.9, 0.9, 0.5, 0.5, 0.1, 0.0):
        _run(c, [int(share * x) for x in c.len.tolist()], 4, 32)
    assert c.len.tolist() == [0] * 4


def test_streams_and_graphs(dev):
    """Captured once, replayed over new masses and lengths, against eager calls on another stream."""
    rng = np.random.default_rng(9)
    lens = [3000, 500, 64, 1200]
    a, b = (_cache(np.random.default_rng(1), dev, 1, 2, 2, 64, lens, lens, "ties") for _ in range(2))
    keep = torch.tensor([1500, 100, 64, 1000], dtype=torch.int32, device=dev)
    index = [torch.full((4, 1500), -1, dtype=torch.int32, device=dev) for _ in range(2)]
    a.evict(keep, 4, 32, index=index[0])
    b.evict(keep, 4, 32, index=index[1])
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.evict(keep, 4, 32, index=index[1])
    for i in range(4):
        now = torch.tensor([int(x) for x in rng.integers(0, 3000, 4)], dtype=torch.int32).clamp(max=torch.tensor(lens)).int()
        fresh = torch.from_numpy(_masses(rng, sum(lens), "ties"))
        for c in (a, b):
            c.len.copy_(now)
            c.mass.copy_(fresh)
        graph.replay()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            a.evict(keep, 4, 32, index=index[0])
        torch.cuda.synchronize()
        for x, y in zip(_state(a), _state(b)):
            assert np.array_equal(x, y)
        assert torch.equal(*index)


def test_refusals(dev):
    rng = np.random.default_rng(11)
    c = _cache(rng, dev, 1, 2, 2, 64, [10] * 4, [20] * 4)
    other = _cache(rng, dev, 1, 2, 2, 128, [0] * 4, [20] * 4)
    before = _state(c)
    keep = torch.full((4,), 5, dtype=torch.int32, device=dev)
    idx = torch.zeros((4, 6), dtype=torch.int32, device=dev)
    from paper_2608_24063_amd import VisCacheError
    for f in (lambda: c.evict(None), lambda: c.evict(keep.long()), lambda: c.evict(keep[:3]), lambda: c.evict(keep.cpu()),
              lambda: c.evict(keep, index=idx.long()), lambda: c.evict(keep, index=idx[:3]), lambda: c.evict(keep, index=idx[:, ::2]),
              lambda: c.evict(keep, index=idx[0]), lambda: c.evict(keep, to=other)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: c.evict(keep, sinks=-1), lambda: c.evict(keep, recent=-1), lambda: c.evict(keep, to=c),
              lambda: c.evict(keep, max_rows=-1)):
        with pytest.raises(VisCacheError):
            f()
    assert all(np.array_equal(x, y) for x, y in zip(before, _state(c)))
