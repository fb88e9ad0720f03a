"""Infinities and NaN in the 8-bit cache: they make their block meaningless, and
nothing else.  Queries that see no row of the block give the same bits as over a
cache without them."""
import numpy as np
import pytest

from tests.test_gpu_q8 import FMTS, _filled, _make, _t, _values, dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d,G,n,lens", [(64, 1, 16, [64 * 3 + 5, 64 * 40 + 15]), (128, 2, 8, [64 * 90 + 3, 64 + 7]),
                                        (64, 4, 40, [64 * 3 + 9, 64 * 30 + 39]), (128, 7, 60, [64 * 90 + 25, 64 * 2 + 1]),
                                        (128, 8, 70, [64 * 4 + 63, 64 * 9 + 30])])
@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("bad", [float("nan"), -float("inf")])
@pytest.mark.parametrize("whole", [False, True])
def test_open_block(dev, fmt, d, G, n, lens, fp32, bad, whole):  # noqa: F811
    """One value of one open row, of keys and values, of units cut along their rows
    and (batched until they fill the card) whole ones."""
    B = 150 if whole else 1
    if whole:
        lens = [min(x, 64 * 9 + x % 64) for x in lens] * B
    a, b = (_make(1, B, 2 * G, 2, d, lens, dev, fmt) for _ in range(2))
    g = torch.Generator(device=dev)
    g.manual_seed(61)
    k, v = (torch.randn((1, B, max(lens), 2, d), generator=g, device=dev).to(torch.bfloat16) for _ in "kv")
    for c in (a, b):
        c.append(k, v)  # as far as each unit has room
        assert c.len.tolist() == lens
    q = _t(_values(np.random.default_rng(62), (1, B, n, 2 * G, d)), dev)
    for side in "kv":
        getattr(b, side + "_tail")[:, 0, 3] = bad  # the first open row of every unit
    typ = torch.float32 if fp32 else torch.bfloat16
    oa, ob = (torch.full((1, B, n, 2 * G, d), 7.0, dtype=typ, device=dev) for _ in range(2))
    a.attend(q, oa, 0.1)
    b.attend(q, ob, 0.1)
    torch.cuda.synchronize()
    checked = 0
    for g in range(2):
        clean = max(0, n - lens[g] % 64)  # queries before the open block
        mine = slice(g * G, g * G + G)
        assert torch.equal(oa[:, :, :clean, mine], ob[:, :, :clean, mine]), g
        checked += clean
    assert checked > 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n", [3, 40])
def test_appended_rows(dev, fmt, n):  # noqa: F811
    """The same through append: the blocks before the row's, sealed or not, are clean."""
    lens = [64 * 5, 64 * 60]
    a, b = (_filled(np.random.default_rng(63), dev, 1, 1, 8, 2, 64, lens, fmt, extra=200)[0] for _ in range(2))
    rng = np.random.default_rng(64)
    k, v = (_values(rng, (1, 1, 100, 2, 64)) for _ in "kv")
    a.append(_t(k, dev), _t(v, dev))
    k[:, :, 70, :, 9], v[:, :, 90, :, 3] = np.nan, np.inf  # open rows 6 and 26
    b.append(_t(k, dev), _t(v, dev))
    q = _t(_values(rng, (1, 1, n, 8, 64)), dev)
    oa, ob = (torch.zeros((1, 1, n, 8, 64), dtype=torch.float32, device=dev) for _ in range(2))
    a.attend(q, oa, 0.1)
    b.attend(q, ob, 0.1)
    clean = max(0, n - 36)
    assert torch.equal(oa[:, :, :clean], ob[:, :, :clean])
    for c, o in ((a, oa), (b, ob)):
        c.attend(q, o, 0.1, causal=False, max_rows=64 * 6)  # up to the open block of the first, past none of the second
    assert torch.equal(oa, ob)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d,G,n,lens", [(64, 4, 1, [200, 90]), (128, 7, 1, [64 * 90 + 3, 64 * 40]), (64, 8, 2, [64 * 90, 5]),
                                        (64, 4, 9, [64 * 3, 64 * 30 + 9]), (128, 8, 70, [64 * 60, 64 * 9 + 30])])
@pytest.mark.parametrize("fp32", [True, False])
def test_query_with_a_nan(dev, fmt, d, G, n, lens, fp32):  # noqa: F811
    """NaN for the query's head and no other, of units that are cut along their rows and
    whole ones; zeros still for one that sees no row."""
    c = _filled(np.random.default_rng(65), dev, 1, 1, 2 * G, 2, d, lens, fmt)[0]
    x = _values(np.random.default_rng(66), (1, 1, n, 2 * G, d))
    typ = torch.float32 if fp32 else torch.bfloat16
    clean, out = (torch.full((1, 1, n, 2 * G, d), 7.0, dtype=typ, device=dev) for _ in range(2))
    c.attend(_t(x, dev), clean, 0.1)
    x[0, 0, n - 1, ::2, 5] = np.nan
    c.attend(_t(x, dev), out, 0.1)
    torch.cuda.synchronize()
    assert out[0, 0, n - 1, ::2].isnan().all()
    same = torch.ones(out.shape, dtype=torch.bool, device=dev)
    same[0, 0, n - 1, ::2] = False
    if fp32 or n * G <= 16:
        assert torch.equal(out[same], clean[same])
    else:  # a wave's columns may be rescaled together, which moves roundings
        a, b = out[same].float(), clean[same].float()
        assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 2.0 ** -10 * b.abs().max()).all()
    c.len.zero_()
    c.attend(_t(x, dev), out, 0.1)
    assert (out == 0).all()
