"""The angle's bits past fp32.  A rotation reduces its angle to a number of turns a in
64 bits, rounds that to fp32 (h), and turns the result by what the rounding left,
e = 2 pi (a - h).  Rows (1, 0) come back as (cos, sin), whose angle is off by delta =
sin cos* - cos sin*.  Against e over many angles delta has the slope 0 if e was taken
account of, -1 if it was dropped, -2 if it went in with the wrong sign.

Tolerances.  Sine and cosine are taken to be off by two steps of fp32 (2^-23) at most,
their correction rounds once more (2^-25).  e is spread over at least 4e-8; with delta
at most 2^-23 + 2^-25 the slope of N angles is off by less than 4 / sqrt(N) a standard
deviation, 0.018 at 51200, so 0.1 holds it and tells the three apart.  A rotated row is off by
(|x1| + |x2|) (2^-23 + 2^-25 + 2 2^-24), the product's and the sum's roundings last:
under 5 steps of 2^-24."""
import numpy as np
import pytest

N, HALF = 800, 64
F32 = np.float32


def _angles():
    rng = np.random.default_rng(101)
    freq = rng.uniform(0.3, 1.0, HALF)
    pos = rng.integers(2 ** 20 - 50000, 2 ** 20, (3, 1, N)).astype(np.int32)
    a = pos[0, 0][:, None].astype(np.float64) * (freq / (2 * np.pi))
    a -= np.rint(a)
    return freq, pos, a, 2 * np.pi * (a - a.astype(F32).astype(np.float64))


def _slope(c, s, a, e):
    d = s * np.cos(2 * np.pi * a) - c * np.sin(2 * np.pi * a)
    return float((d * e).sum() / (e * e).sum())


def _model(a, sign):
    """The rotation's sine and cosine in fp32 steps, e times `sign`."""
    h = a.astype(F32)
    e = F32(6.2831853) * (a - h.astype(np.float64)).astype(F32) * F32(sign)
    c, s = (f(2 * np.pi * h.astype(np.float64)).astype(F32) for f in (np.cos, np.sin))
    fma = lambda x, y, z: (x.astype(np.float64) * y + z).astype(F32)  # noqa: E731
    return fma(-s, e, c).astype(np.float64), fma(c, e, s).astype(np.float64)


def test_the_slope_tells_the_forms_apart():
    _, _, a, e = _angles()
    assert np.sqrt((e * e).mean()) > 4e-8
    for sign, want in ((1, 0.0), (0, -1.0), (-1, -2.0)):
        assert abs(_slope(*_model(a, sign), a, e) - want) < 0.1


@pytest.mark.gpu
@pytest.mark.parametrize("adjacent", [False, True])
def test_the_angles_last_bits(adjacent):
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_24063_amd.tensors import Rope
    freq, pos, a, e = _angles()
    x = np.zeros((1, 1, N, 2, 2 * HALF), dtype=np.float32)
    one, two = (slice(0, None, 2), slice(1, None, 2)) if adjacent else (slice(0, HALF), slice(HALF, None))
    x[..., 0, one] = 1
    x[..., 1, :] = np.random.default_rng(102).standard_normal((1, 1, N, 2 * HALF))
    t = torch.from_numpy(x).cuda()
    Rope(2 * HALF, inv_freq=freq, pairing=int(adjacent)).apply(torch.from_numpy(pos).cuda(), q=t)
    got = t.cpu().numpy().astype(np.float64)[0, 0]
    assert abs(_slope(got[:, 0, one], got[:, 0, two], a, e)) < 0.1
    c, s = np.cos(2 * np.pi * a), np.sin(2 * np.pi * a)
    for h in range(2):
        p, q = x[0, 0, :, h, one].astype(np.float64), x[0, 0, :, h, two].astype(np.float64)
        tol = (np.abs(p) + np.abs(q)) * 5 * 2.0 ** -24
        assert (np.abs(got[:, h, one] - (p * c - q * s)) <= tol).all()
        assert (np.abs(got[:, h, two] - (q * c + p * s)) <= tol).all()
