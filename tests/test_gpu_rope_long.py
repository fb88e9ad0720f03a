"""Rotations that the shapes of attention do not cover, and long ones with counts and
strides (four tokens a workgroup from 8192 tokens over all layers on)."""
import numpy as np
import pytest

from tests import q8_ref as ref
from tests.test_gpu_rope import _check, dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_heads_that_attention_does_not_take(dev):  # noqa: F811
    """Together refused, each with a call of its own rotated."""
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(91)
    rope = Rope(64, sections=(8, 12, 12), theta=1e4)
    pos = rng.integers(0, 9000, (3, 2, 5)).astype(np.int32)
    tp = torch.from_numpy(pos).to(dev)
    freq, ax = [1e4 ** (-2.0 * i / 64) for i in range(32)], ref.rope_axes(64, (8, 12, 12), False)
    for Hq, Hkv, status in ((34, 2, vc.VC_ERR_UNSUPPORTED), (5, 2, vc.VC_ERR_SHAPE), (2, 4, vc.VC_ERR_SHAPE)):
        q, k = (rng.standard_normal((1, 2, 5, h, 64)).astype(np.float32) for h in (Hq, Hkv))
        tq, tk = torch.from_numpy(q).to(dev), torch.from_numpy(k).to(dev)
        with pytest.raises(vc.VisCacheError) as e:
            rope.apply(tp, tq, tk)
        assert e.value.status == status
        rope.apply(tp, q=tq)
        rope.apply(tp, k=tk)
        for t, x in ((tq, q), (tk, k)):
            _check(t.cpu().numpy(), x, pos, 64, freq, ax, False, False, 1.0, True)
