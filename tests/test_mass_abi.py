"""The cache with masses on the host: every refusal of its entry points (no GPU: the checks
run before any device call), workspaces, and the handling of the Python class."""
import math

import pytest

from tests.test_q8_abi import BAD_SHAPES, P16, _rows, _shape, _status, vc  # noqa: F401


def _cache(vc, at=P16, **kw):  # noqa: F811
    c = vc.vc_mass_cache(*[at] * 6, None)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _attend(vc, shape=None, cache=None, k=1, v=1, q=None, out=None, n=4, fp32=0, scale=0.1, decay=1.0, rows=1000,  # noqa: F811
            ws=1 << 20, bytes_=1 << 40):
    r = _rows(vc)
    pick = lambda x: r if x == 1 else x  # noqa: E731
    return _status(vc, vc.viscache_mass_attend, shape or _shape(vc), cache or _cache(vc), pick(k), pick(v), q or r, out or r,
                   n, 0, fp32, scale, decay, rows, ws, bytes_, 0)


def _evict(vc, shape=None, cache=None, to=None, keep=P16, sinks=4, recent=4, rows=1000, index=0, wide=0, ws=1 << 20,  # noqa: F811
           bytes_=1 << 40):
    return _status(vc, vc.viscache_mass_evict, shape or _shape(vc), cache or _cache(vc), to, keep, sinks, recent, rows,
                   index, wide, ws, bytes_, 0)


FIELDS = ("k_pool", "v_pool", "mass", "row_off", "cap", "len")


def test_shapes_and_caches(vc):  # noqa: F811
    for kw, err in BAD_SHAPES:
        s, want = _shape(vc, **kw), getattr(vc, "VC_ERR_" + err)
        assert _attend(vc, s) == _attend(vc, s, n=0) == _evict(vc, s) == want, kw
        assert vc.viscache_mass_attend_workspace_bytes(s, 4, 100) == vc.viscache_mass_evict_workspace_bytes(s, 100) == 0
    bad = [_cache(vc, **{f: None}) for f in FIELDS] + [_cache(vc, k_pool=P16 + 8), _cache(vc, v_pool=P16 + 2),
                                                       _cache(vc, mass=P16 + 2)]
    for c in bad:
        assert _attend(vc, cache=c) == _attend(vc, cache=c, n=0) == _evict(vc, cache=c) == vc.VC_ERR_ARG
        assert _evict(vc, cache=_cache(vc, at=2 * P16), to=c) == vc.VC_ERR_ARG


def test_attention_arguments(vc):  # noqa: F811
    A = vc.VC_ERR_ARG
    for kw in (dict(n=-1), dict(rows=-1), dict(fp32=2), dict(fp32=-1), dict(k=None), dict(v=None), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(decay=-0.5), dict(decay=math.nan),
               dict(decay=math.inf)):
        assert _attend(vc, **kw) == A, kw
    for bad in (_rows(vc, data=P16 + 8), _rows(vc, data=None), _rows(vc, head=-8), _rows(vc, token=1028), _rows(vc, layer=-16)):
        for name in ("k", "v", "q", "out"):
            assert _attend(vc, **{name: bad}) == A, name
    assert _attend(vc, out=_rows(vc, head=64)) == A  # rows on each other
    assert _attend(vc, q=_rows(vc, head=0), ws=0) == vc.VC_ERR_WORKSPACE  # an input may repeat
    assert _attend(vc, k=None, v=None, ws=0) == vc.VC_ERR_WORKSPACE
    assert _attend(vc, n=0) == vc.VC_OK
    assert _attend(vc, decay=0.0, ws=0) == vc.VC_ERR_WORKSPACE


@pytest.mark.parametrize("n", [1, 4, 5, 64, 3000])
@pytest.mark.parametrize("rows", [0, 1, 1000, 40000])
def test_attention_workspace(vc, n, rows):  # noqa: F811
    s, W = _shape(vc), vc.VC_ERR_WORKSPACE
    need = vc.viscache_mass_attend_workspace_bytes(s, n, rows)
    assert need > 0
    assert _attend(vc, n=n, rows=rows, bytes_=need - 1) == _attend(vc, n=n, rows=rows, ws=(1 << 20) + 128) == W
    assert _attend(vc, n=n, rows=rows, ws=0, scale=0.0) == vc.VC_ERR_ARG  # checked last
    if n * 4 <= 16:
        assert need >= 16 * 12  # the units' states
    else:
        assert need >= 8 * 12 * 4 * n
    assert vc.viscache_mass_attend_workspace_bytes(s, n, rows + 1) >= need


def test_limits(vc):  # noqa: F811
    U, s = vc.VC_ERR_UNSUPPORTED, _shape(vc)
    assert _attend(vc, n=1 << 23) == U and vc.viscache_mass_attend_workspace_bytes(s, 1 << 23, 100) == 0
    big, row = _shape(vc, B=1 << 20, L=8, Hq=1, Hkv=1), _rows(vc, 1 << 20, 1 << 38, 1 << 18, 128, 128)
    for n in (1, 17, 40):
        assert _attend(vc, big, k=row, v=row, q=row, out=row, n=n) == U
        assert vc.viscache_mass_attend_workspace_bytes(big, n, 100) == 0
    assert _evict(vc, big) == U and vc.viscache_mass_evict_workspace_bytes(big, 100) == 0
    # a row bound past what a unit may hold: 2^23 workgroups add up a prompt's masses, single tokens take fewer
    one = _shape(vc, B=1, L=1, Hq=1, Hkv=1)
    assert vc.viscache_mass_attend_workspace_bytes(one, 40, 2 ** 31 - 1) > 0
    assert vc.viscache_mass_attend_workspace_bytes(_shape(vc, B=1, L=1), 40, 2 ** 31 - 1) == 0
    assert vc.viscache_mass_attend_workspace_bytes(_shape(vc, B=1, L=1), 1, 2 ** 31 - 1) > 0
    assert vc.viscache_mass_attend_workspace_bytes(s, -1, 100) == vc.viscache_mass_attend_workspace_bytes(s, 1, -1) == 0


@pytest.mark.parametrize("high", [2 ** 32, 2 ** 40, -2 ** 32, 2 ** 63], ids=hex)
def test_arguments_past_32_bits(vc, high):  # noqa: F811
    x, far = high + 4, high > 0
    s = _shape(vc, B=1, L=1)
    A, U, W = vc.VC_ERR_ARG, vc.VC_ERR_UNSUPPORTED, vc.VC_ERR_WORKSPACE
    assert _attend(vc, n=x) == (U if far else A)
    assert _attend(vc, s, n=1, rows=x, ws=0) == (W if far else A)
    assert _evict(vc, sinks=x, ws=0) == _evict(vc, recent=x, ws=0) == (W if far else A)
    assert _evict(vc, index=P16, wide=x, ws=0) == (W if far else A)


def test_eviction_arguments(vc):  # noqa: F811
    A, W = vc.VC_ERR_ARG, vc.VC_ERR_WORKSPACE
    for kw in (dict(keep=0), dict(sinks=-1), dict(recent=-1), dict(rows=-1), dict(index=P16, wide=-1), dict(wide=5)):
        assert _evict(vc, **kw) == A, kw
    for f in ("k_pool", "v_pool", "mass", "len"):  # the other cache's arrays have to be its own
        assert _evict(vc, to=_cache(vc, at=2 * P16, **{f: P16})) == A, f
    assert _evict(vc, to=_cache(vc, at=2 * P16), ws=0) == W
    for rows in (0, 1, 128, 129, 40000):
        need = vc.viscache_mass_evict_workspace_bytes(_shape(vc), rows)
        assert need >= 4 * 12 * rows
        assert _evict(vc, rows=rows, bytes_=need - 1) == _evict(vc, rows=rows, ws=0) == W
        assert _evict(vc, rows=rows, ws=(1 << 20) + 64) == W


def test_class_on_the_host():
    import torch
    from paper_2608_24063_amd.tensors import MassCache
    c = MassCache(1, 2, 4, 2, 64, [5, 0, 7, 3], "cpu")
    assert c.row_off.tolist() == [0, 5, 5, 12] and c.cap.tolist() == [5, 0, 7, 3] and c.k_pool.shape == (15, 64)
    assert [c._bound(x) for x in (None, 0, 6, 2 ** 40)] == [7, 0, 6, 7]
    assert MassCache(1, 1, 2, 1, 64, [0], "cpu").k_pool.shape == (1, 64)
    for caps in ([1, 2, 3], [1, 2, 3, -1]):
        with pytest.raises(ValueError):
            MassCache(1, 2, 4, 2, 64, caps, "cpu")
    good = dict(k_pool=c.k_pool, v_pool=c.v_pool, mass=c.mass, row_off=c.row_off, cap=c.cap, len=c.len)
    MassCache(1, 2, 4, 2, 64, [5, 0, 7, 3], "cpu", buffers=good)
    for name, x in (("k_pool", c.k_pool[:14]), ("v_pool", c.v_pool.float()), ("mass", c.mass.double()),
                    ("row_off", c.row_off.int()), ("cap", c.cap[:3]), ("len", c.len.long()),
                    ("mass", torch.zeros(30)[::2])):
        with pytest.raises(ValueError, match=name):
            MassCache(1, 2, 4, 2, 64, [5, 0, 7, 3], "cpu", buffers=dict(good, **{name: x}))
