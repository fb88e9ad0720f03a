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
