"""The 8-bit cache and the rotary positions on the host: every refusal of their
entry points (no GPU: the checks run before any device call), workspace
sizes, and the plain forms the GPU tests compare with against closed forms."""
import ctypes
import os

import numpy as np
import pytest

from tests import q8_ref as ref

P16 = 0x10000  # an address that is never read: every call here is refused or does nothing


@pytest.fixture(scope="module")
def vc():
    import paper_2608_24063_amd as vc
    if not os.path.exists(vc.LIB_PATH):
        from paper_2608_24063_amd import build
        build.build()
    vc.lib()
    return vc


def _shape(vc, B=2, L=3, Hq=8, Hkv=2, d=128):
    return vc.vc_decode_shape(B, L, Hq, Hkv, d)


def _cache(vc, **kw):
    c = vc.vc_q8cache(kw.pop("format", vc.VC_Q8_INT8), *[P16] * 9, None)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _rows(vc, data=P16, layer=1 << 20, seq=1 << 16, token=1024, head=128):
    return vc.vc_rows(data, layer, seq, token, head)


def _status(vc, fn, *a):
    try:
        fn(*a)
    except vc.VisCacheError as e:
        return e.status
    return vc.VC_OK


BAD_SHAPES = [(dict(B=0), "SHAPE"), (dict(L=0), "SHAPE"), (dict(Hq=0), "SHAPE"), (dict(Hkv=0), "SHAPE"),
              (dict(Hq=7), "SHAPE"), (dict(Hq=34, Hkv=2), "UNSUPPORTED"), (dict(d=96), "UNSUPPORTED"),
              (dict(d=256), "UNSUPPORTED"), (dict(L=1 << 20, B=1 << 20), "SHAPE"),
              (dict(L=2 ** 31 - 1, B=2 ** 31 - 1, Hq=16, Hkv=16), "SHAPE")]


def _append(vc, shape=None, cache=None, k=None, v=None, n=4):
    return _status(vc, vc.viscache_q8_append, shape or _shape(vc), cache or _cache(vc), k or _rows(vc), v or _rows(vc),
                   n, 0, 0, 0)


def _read(vc, shape=None, cache=None, k=None, v=None, rows=4, fp32=0):
    return _status(vc, vc.viscache_q8_read, shape or _shape(vc), cache or _cache(vc), rows, k or _rows(vc),
                   v or _rows(vc), 0, fp32, 0)


def _attend(vc, shape=None, cache=None, q=None, out=None, n=1, causal=1, fp32=0, scale=0.1, rows=100, ws=P16,
            bytes_=1 << 40):
    return _status(vc, vc.viscache_q8_attend, shape or _shape(vc), cache or _cache(vc), q or _rows(vc),
                   out or _rows(vc), n, 0, causal, fp32, scale, rows, ws, bytes_, 0)


def _step(vc, shape=None, cache=None, rope=None, pos=0, q=None, k=None, v=None, out=None, fp32=0, scale=0.1, rows=100,
          ws=P16, bytes_=1 << 40):
    r = [x or _rows(vc) for x in (q, k, v, out)]
    return _status(vc, vc.viscache_q8_step, shape or _shape(vc), cache or _cache(vc), rope, pos, *r, fp32, scale, rows,
                   ws, bytes_, 0)


def _rope_args(vc, **kw):
    a = dict(rot=128, s=(16, 24, 24), layout=0, pairing=0, fp32=0, inverse=0, scale=1.0, theta=1e4, inv_freq=None)
    a.update(kw)
    return vc.vc_rope(a["rot"], (ctypes.c_int32 * 3)(*a["s"]), a["layout"], a["pairing"], a["fp32"], a["inverse"],
                      a["scale"], a["theta"], a["inv_freq"])


def _rope(vc, shape=None, n=4, pos=P16, q=(1, 1), k=(1, 1), rows=None, **kw):
    r = [(rows or _rows(vc)) if x else None for x in q + k]
    return _status(vc, vc.viscache_rope, shape or _shape(vc), _rope_args(vc, **kw), n, pos, 0, *r, 0)


@pytest.mark.parametrize("kw,want", BAD_SHAPES)
def test_bad_shapes(vc, kw, want):
    s, want = _shape(vc, **kw), getattr(vc, "VC_ERR_" + want)
    assert _append(vc, s) == _read(vc, s) == _attend(vc, s) == _rope(vc, s) == _step(vc, s) == want
    assert vc.viscache_q8_attend_workspace_bytes(s, 1, 100) == 0


@pytest.mark.parametrize("name", ["k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "row_off", "cap", "len"])
def test_null_cache_members(vc, name):
    c = _cache(vc, **{name: None})
    assert _append(vc, cache=c) == _read(vc, cache=c) == _attend(vc, cache=c) == _step(vc, cache=c) == vc.VC_ERR_ARG


@pytest.mark.parametrize("kw", [dict(format=2), dict(format=-1), dict(k_codes=P16 + 8), dict(v_codes=P16 + 4),
                                dict(k_tail=P16 + 2), dict(v_tail=P16 + 8)])
def test_bad_cache(vc, kw):
    c = _cache(vc, **kw)
    assert _append(vc, cache=c) == _read(vc, cache=c) == _attend(vc, cache=c) == _step(vc, cache=c) == vc.VC_ERR_ARG


@pytest.mark.parametrize("kw", [dict(data=None), dict(data=P16 + 8), dict(layer=-8), dict(seq=4), dict(token=1001),
                                dict(head=-128), dict(token=1 << 62)])
def test_bad_rows(vc, kw):
    r, A = _rows(vc, **kw), vc.VC_ERR_ARG
    assert _append(vc, k=r) == _append(vc, v=r) == _read(vc, k=r) == _read(vc, v=r) == A
    assert _attend(vc, q=r, n=2) == _attend(vc, out=r, n=2) == A
    assert _rope(vc, rows=r) == A


@pytest.mark.parametrize("kw", [dict(layer=0), dict(seq=0), dict(token=64), dict(head=0)])
def test_outputs_on_themselves(vc, kw):
    """Strides under d (0 among them) repeat rows: refused for outputs."""
    r, A = _rows(vc, **kw), vc.VC_ERR_ARG
    assert _read(vc, k=r) == _read(vc, v=r) == _attend(vc, out=r, n=2) == _rope(vc, rows=r) == A


def test_step_refusals(vc):
    A, W = vc.VC_ERR_ARG, vc.VC_ERR_WORKSPACE
    for kw in (dict(data=None), dict(data=P16 + 8), dict(layer=-8), dict(seq=4), dict(head=-128)):
        r = _rows(vc, **kw)
        assert _step(vc, q=r) == _step(vc, k=r) == _step(vc, v=r) == _step(vc, out=r) == A
    assert _step(vc, out=_rows(vc, head=64)) == _step(vc, rows=-1) == _step(vc, fp32=2) == _step(vc, scale=0.0) == A
    assert _step(vc, ws=0) == _step(vc, ws=P16 + 128) == W
    assert _step(vc, bytes_=vc.viscache_q8_attend_workspace_bytes(_shape(vc), 1, 100) - 1) == W
    assert _step(vc, rope=_rope_args(vc), pos=0) == _step(vc, rope=_rope_args(vc, fp32=1), pos=P16) == A
    assert _step(vc, rope=_rope_args(vc, rot=144), pos=P16) == _step(vc, rope=_rope_args(vc, theta=0.0), pos=P16) == A


def test_scalars(vc):
    A = vc.VC_ERR_ARG
    assert _append(vc, n=-1) == _read(vc, rows=-1) == _read(vc, fp32=2) == _read(vc, fp32=-1) == A
    assert _attend(vc, n=-1) == _attend(vc, rows=-1) == _attend(vc, causal=2) == _attend(vc, fp32=2) == A
    for s in (0.0, -1.0, float("inf"), float("nan")):
        assert _attend(vc, scale=s) == A
    assert _rope(vc, n=-1) == _rope(vc, pos=0) == A


def test_nothing_to_do(vc):
    assert _append(vc, n=0) == _read(vc, rows=0) == _attend(vc, n=0) == _rope(vc, n=0) == vc.VC_OK


def test_workspace(vc):
    W = vc.VC_ERR_WORKSPACE
    for n in (1, 5):
        need = vc.viscache_q8_attend_workspace_bytes(_shape(vc), n, 5000)
        assert need > 0
        assert _attend(vc, n=n, rows=5000, ws=0) == _attend(vc, n=n, rows=5000, ws=P16 + 16) == W
        assert _attend(vc, n=n, rows=5000, bytes_=need - 1) == W
    for d in (64, 128):
        for n in (0, 1, 2, 4, 33, 1000):
            for rows in (0, 1, 64, 4096, 2 ** 31 - 1):
                assert 256 <= vc.viscache_q8_attend_workspace_bytes(_shape(vc, d=d), n, rows) < 1 << 30


def test_too_large(vc):
    U = vc.VC_ERR_UNSUPPORTED
    big = _shape(vc, B=1 << 20, L=8, Hq=1, Hkv=1)
    row = _rows(vc, layer=1 << 38, seq=1 << 18, token=128)
    assert _append(vc, big, n=1, k=row, v=row) == _append(vc, n=2 ** 31 - 1) == U
    assert _read(vc, big, k=row, v=row, rows=1) == _read(vc, rows=2 ** 31 - 1) == U
    assert _attend(vc, big, q=row, out=row) == _attend(vc, n=1 << 23) == U
    assert vc.viscache_q8_attend_workspace_bytes(_shape(vc), 1 << 23, 10) == 0
    assert _rope(vc, n=1 << 22) == U


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=8), dict(rot=120), dict(rot=144), dict(s=(64, 1, 0)),
                                dict(s=(-1, 33, 32)), dict(s=(65, 0, -1)), dict(s=(2 ** 31 - 1, 2 ** 31 - 1, 66)),
                                dict(layout=2), dict(layout=-1), dict(pairing=2), dict(fp32=2), dict(inverse=-1),
                                dict(scale=float("nan")), dict(scale=float("inf")), dict(theta=0.0),
                                dict(theta=-2.0), dict(theta=float("inf")), dict(q=(1, 0)), dict(k=(0, 1)),
                                dict(q=(0, 0), k=(0, 0))])
def test_rope_refusals(vc, kw):
    assert _rope(vc, **kw) == vc.VC_ERR_ARG


def test_rope_frequencies_are_checked(vc):
    f = (ctypes.c_double * 64)(*[1.0] * 64)
    assert _rope(vc, n=0, theta=0.0, inv_freq=f) == vc.VC_OK  # theta is not read
    f[63] = float("nan")
    assert _rope(vc, n=0, inv_freq=f) == vc.VC_ERR_ARG


def test_python_checks():
    """Shapes, types and devices are checked before any pointer is taken."""
    import torch
    from paper_2608_24063_amd.tensors import Q8Cache, Rope
    with pytest.raises(ValueError):
        Rope(64).apply(None)
    with pytest.raises(ValueError):
        Rope(64).apply(torch.zeros(3, 1, 2, dtype=torch.int32), torch.zeros(1, 1, 2, 4, 64))  # not on a GPU
    with pytest.raises(ValueError):
        Rope(64, inv_freq=[1.0] * 31)
    with pytest.raises(ValueError):
        Q8Cache(1, 1, 2, 2, 64, [5], "cpu")
    c = Q8Cache(1, 1, 4, 2, 64, [5, 70], "cpu")
    assert c.k_codes.shape == (3, 64, 64) and c.row_off.tolist() == [0, 64]
    x = torch.zeros(1, 1, 2, 2, 64, dtype=torch.bfloat16)
    for bad in (x.float(), x[..., :32], x[:, :, :, :1]):
        with pytest.raises(ValueError):
            c.append(bad, x)
        with pytest.raises(ValueError):
            c.append(x, bad)
    with pytest.raises(ValueError):
        c.append(x, x, count=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        c.attend(x, x, 1.0)
    with pytest.raises(ValueError):  # the right shapes, but nothing of it on a GPU
        c.append(x, x)
    with pytest.raises(ValueError):
        c.read(x, x)
    q = torch.zeros(1, 1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        c.attend(q, q, 1.0)
    buf = {n: getattr(c, n) for n in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "row_off", "cap", "len")}
    Q8Cache(1, 1, 4, 2, 64, [5, 70], "cpu", buffers=buf)
    with pytest.raises(ValueError):
        Q8Cache(1, 1, 4, 2, 64, [5, 70], "cpu", format="int8", buffers=buf)


# ---- the plain forms themselves ------------------------------------------------

def test_plain_quantiser():
    import torch
    rng = np.random.default_rng(0)
    x = ref.bf16(rng.standard_normal((64, 64)) * np.exp(rng.standard_normal((64, 64))))
    for fmt in ("int8", "e4m3"):
        c, s = ref.quantise(x, fmt)
        Q = ref.TOP[fmt]
        assert np.abs(c).max() == Q and abs(float(s) * Q / np.abs(x).max() - 1) <= 2.0 ** -23
        step = float(s) if fmt == "int8" else None
        if step:
            assert np.abs(c * np.float64(s) - x).max() <= step * 0.5000001
        else:  # half a step of 2^-4 relative, or half of the smallest step
            assert (np.abs(c * np.float64(s) - x) <= np.abs(x) * 2.0 ** -4 * 1.0001 + float(s) * 2.0 ** -10).all()
    y = np.linspace(-448, 448, 4001)
    assert np.array_equal(ref.round_e4m3(y), torch.from_numpy(y).to(torch.float8_e4m3fn).double().numpy())
    mid = np.array([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 432.0])  # midpoints go to even
    assert np.array_equal(ref.round_e4m3(mid), [16.0, 20.0, 0.0, 2.0 ** -8, 448.0])
    z, s = ref.quantise(np.zeros((64, 64)), "int8")
    assert not z.any() and s == np.float32(2.0 ** -60)
    assert ref.open_scale(np.array([[1.0, -3.0]])) == 2.0 ** -13 and ref.open_scale(np.zeros((0, 4))) == 2.0 ** -60


def test_plain_rope_turns_and_turns_back():
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((7, 64)), rng.integers(0, 1000, (3, 7))
    f = 1e4 ** (-2.0 * np.arange(16) / 32)
    for inter in (False, True):
        ax = ref.rope_axes(32, (6, 5, 5), inter)
        assert [ax.count(a) for a in (0, 1, 2)] == [6, 5, 5]
        for adj in (False, True):
            y = ref.rope(x, pos, 32, f, ax, adj, False, 1.0)
            assert np.allclose(np.linalg.norm(y, axis=1), np.linalg.norm(x, axis=1))
            assert np.allclose(ref.rope(y, pos, 32, f, ax, adj, True, 1.0), x)
            assert np.array_equal(y[:, 32:], x[:, 32:])


def test_plain_attention_over_nothing():
    o, r = ref.attend(np.ones(4), np.ones((3, 4)), np.ones((3, 4)), 1.0, 0)
    assert not o.any() and r == 0.0
