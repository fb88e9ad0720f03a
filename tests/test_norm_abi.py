"""The normed rotations on the host: every refusal of their entry points (no GPU: the
checks run before any device call) and the gradient's workspace."""
import ctypes
import math

import pytest

from tests.test_q8_abi import BAD_SHAPES, P16, _rows, _shape, _status, vc  # noqa: F401


def _rope(vc, **kw):  # noqa: F811
    r = vc.vc_rope(128, (ctypes.c_int32 * 3)(64, 0, 0), 0, 0, 0, 0, 1.0, 1e6, None)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _norm(vc, **kw):  # noqa: F811
    n = vc.vc_norm(1e-6, 0, P16, P16)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def _fwd(vc, shape=None, rope=None, norm=None, n=4, pos=P16, q=True, k=True, q_in=None, q_out=None):  # noqa: F811
    r = _rows(vc)
    qi, qo = (q_in or r, q_out or r) if q else (q_in, q_out)
    ki = r if k else None
    return _status(vc, vc.viscache_norm_rope, shape or _shape(vc), rope or _rope(vc), norm or _norm(vc), n, pos, 0, qi,
                   qo, ki, ki, 0)


def _grad(vc, shape=None, rope=None, norm=None, n=4, pos=P16, q=(1, 1, 1, 1), k=(1, 1, 1, 1), ws=1 << 20, bytes_=1 << 40,  # noqa: F811
          rows=None):
    r = rows or _rows(vc)
    side = lambda s: [r if s[0] else None, r if s[1] else None, r if s[2] else None, P16 if s[3] else 0]  # noqa: E731
    return _status(vc, vc.viscache_norm_rope_grad, shape or _shape(vc), rope or _rope(vc), norm or _norm(vc), n, pos, 0,
                   *side(q), *side(k), ws, bytes_, 0)


def test_shapes(vc):  # noqa: F811
    for kw, err in BAD_SHAPES:
        want = getattr(vc, "VC_ERR_" + err)
        assert _fwd(vc, _shape(vc, **kw)) == _grad(vc, _shape(vc, **kw)) == want, kw
        assert vc.viscache_norm_rope_grad_workspace_bytes(_shape(vc, **kw), 4) == 0


def test_arguments(vc):  # noqa: F811
    A = vc.VC_ERR_ARG
    for f in (_fwd, _grad):
        for kw in (dict(eps=0.0), dict(eps=-1e-6), dict(eps=math.inf), dict(eps=math.nan), dict(eps=1e-39),
                   dict(weight_fp32=2), dict(q_weight=None), dict(q_weight=P16 + 8), dict(k_weight=None),
                   dict(k_weight=P16 + 2)):
            assert f(vc, norm=_norm(vc, **kw)) == A, kw
        for kw in (dict(rot=24), dict(rot=144), dict(layout=2), dict(pairing=2), dict(fp32=2), dict(inverse=2),
                   dict(scale=math.nan), dict(theta=-1.0)):
            assert f(vc, rope=_rope(vc, **kw)) == A, kw
        assert f(vc, n=-1) == f(vc, pos=0) == A
        assert f(vc, n=1 << 23, shape=_shape(vc, B=1, L=2)) == vc.VC_ERR_UNSUPPORTED
    assert _fwd(vc, q=False, k=False) == _fwd(vc, q=False, q_in=_rows(vc)) == _fwd(vc, q=False, q_out=_rows(vc)) == A
    assert _fwd(vc, q_in=_rows(vc, data=P16 + 8)) == _fwd(vc, q_out=_rows(vc, head=64)) == A
    assert _fwd(vc, q_in=_rows(vc, head=132)) == A  # not a multiple of 16 bytes
    assert _fwd(vc, n=0) == vc.VC_OK
    for s in ((1, 1, 1, 0), (1, 1, 0, 1), (1, 0, 1, 1), (0, 1, 1, 1), (0, 0, 0, 1)):
        assert _grad(vc, q=s) == _grad(vc, k=s) == A, s
    assert _grad(vc, q=(0,) * 4, k=(0,) * 4) == _grad(vc, rows=_rows(vc, data=P16 + 4)) == _grad(vc, rows=_rows(vc, head=-128)) == A


def test_gradient_workspace(vc):  # noqa: F811
    need, s = vc.viscache_norm_rope_grad_workspace_bytes, _shape(vc)
    W = vc.VC_ERR_WORKSPACE
    for n in (0, 1, 4, 5000):
        b = need(s, n)
        groups = max(1, min(-(-2 * n // 4), 1024 // 3))
        assert b >= 4 * 2 * 128 * 3 * groups and b % 256 == 0
        assert _grad(vc, n=n, bytes_=b - 1) == _grad(vc, n=n, ws=0) == _grad(vc, n=n, ws=(1 << 20) + 128) == W
    # checked last, and the limits
    assert _grad(vc, ws=0, norm=_norm(vc, eps=0.0)) == vc.VC_ERR_ARG
    assert need(s, -1) == 0 and need(s, 1 << 22) == 0
    assert need(_shape(vc, B=1, L=1 << 17, Hq=1, Hkv=1), 1) == 0
    one = _rows(vc, layer=128, seq=128, token=128, head=128)
    assert _grad(vc, _shape(vc, B=1, L=1 << 17, Hq=1, Hkv=1), rows=one, n=1) == vc.VC_ERR_UNSUPPORTED
    assert _grad(vc, _shape(vc, B=1, L=1 << 17, Hq=1, Hkv=1), rows=one, n=0) == vc.VC_ERR_UNSUPPORTED


@pytest.mark.parametrize("x", [2 ** 32 + 4, 2 ** 40, 2 ** 63, -2 ** 32 + 4])
def test_arguments_past_32_bits(vc, x):  # noqa: F811
    far = x > 0
    assert _fwd(vc, n=x) == _grad(vc, n=x) == (vc.VC_ERR_UNSUPPORTED if far else vc.VC_ERR_ARG)
    assert vc.viscache_norm_rope_grad_workspace_bytes(_shape(vc), x) == 0
