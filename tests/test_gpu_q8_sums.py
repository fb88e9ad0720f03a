"""What attention over the 8-bit cache holds on its way to bf16 outputs: weights
of single tokens in as many bits as for fp32 ones, and the partial sums of units
and tiles that are cut along their rows in 32 bits."""
import numpy as np
import pytest

from tests import q8_ref as ref
from tests.test_gpu_q8 import FMTS, _filled, _run_attend, _t, _values, dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d,G,n", [(64, 4, 1), (128, 7, 1), (128, 7, 2), (64, 1, 16)])
def test_bf16_outputs_are_fp32_outputs_rounded(dev, fmt, d, G, n):  # noqa: F811
    """Up to 16 columns: nothing but the last rounding differs, whole units and cut ones."""
    rng = np.random.default_rng(31 + d + G)
    for lens in ([5, 64, 100, 700], [64 * 90 + 3, 64 * 40, 1, 6000]):
        c, _, _ = _filled(rng, dev, 1, 2, 2 * G, 2, d, lens, fmt)
        q = ref.bf16(rng.standard_normal((1, 2, n, 2 * G, d)))
        full, short = (np.asarray(_run_attend(c, q, dev, fp32, d ** -0.5)) for fp32 in (True, False))
        assert np.array_equal(short, ref.bf16(full))


@pytest.mark.parametrize("fmt", FMTS)
def test_bf16_step_is_the_fp32_step_rounded(dev, fmt):  # noqa: F811
    lens = [63, 64, 700, 6398]
    a, b = (_filled(np.random.default_rng(32), dev, 1, 2, 14, 2, 128, lens, fmt, extra=2)[0] for _ in range(2))
    rng = np.random.default_rng(33)
    q, k, v = (_t(_values(rng, (1, 2, 1, h, 128)), dev) for h in (14, 2, 2))
    oa, ob = (torch.zeros((1, 2, 1, 14, 128), dtype=t, device=dev) for t in (torch.float32, torch.bfloat16))
    a.step(q, k, v, oa, 0.09)
    b.step(q, k, v, ob, 0.09)
    assert torch.equal(oa.to(torch.bfloat16), ob)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d,G,n", [(64, 4, 20), (128, 8, 40), (128, 7, 3)])
def test_partial_sums_of_prompts(dev, fmt, d, G, n):  # noqa: F811
    """Equal weights over whole-number values, blocks of either sign, whose scales are all
    1: every weight is a power of two, every sum exact in 32 bits, the division and the
    parts' join take a few roundings of 2^-24, and so the output is the mean rounded to
    bf16 wherever the mean is not within 2^-20 of itself of a tie."""
    rng = np.random.default_rng(34 + d)
    rows = 64 * 150
    top = ref.TOP[fmt]
    v = 8.0 * rng.integers(8, 16, (1, 1, rows, 1, d)).astype(np.float32)
    v *= np.repeat(rng.choice([-1.0, 1.0], rows // 64), 64)[None, None, :, None, None]
    v[0, 0, ::64, 0, 5] = top  # the largest of every block: scale 1
    k = _values(rng, (1, 1, rows, 1, d))
    from paper_2608_24063_amd.tensors import Q8Cache
    c = Q8Cache(1, 1, G, 1, d, [rows], dev, format=fmt)
    c.append(_t(k, dev), _t(v, dev))
    assert (c.v_scale == 1).all()
    out = np.asarray(_run_attend(c, np.zeros((1, 1, n, G, d), dtype=np.float32), dev, False, 0.1, None, False))
    v = ref.read_back(v[0, 0, :, 0], fmt)
    assert (v == np.rint(v)).all()
    mean = v.sum(axis=0) / rows
    want, lo, hi = (ref.bf16((mean * f).astype(np.float32)) for f in (1, 1 - 2.0 ** -20, 1 + 2.0 ** -20))
    sure = lo == hi
    assert sure.mean() > 0.95 and (out[..., sure] == want[sure]).all()
