"""Rotations that the shapes of attention do not cover, and long ones with counts and
strides (of few heads four tokens a workgroup, of many one)."""
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


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("L,B,n,d,rot,Hq,Hkv", [(1, 3, 2731, 128, 96, 3, 1), (4, 3, 701, 64, 64, 3, 1),
                                                (2, 5, 843, 128, 128, 3, 1), (1, 3, 2731, 64, 48, 34, 17),
                                                (1, 3, 683, 128, 64, 2, 1)])
def test_long_with_counts_and_strides(dev, fp32, adjacent, L, B, n, d, rot, Hq, Hkv):  # noqa: F811
    """Ragged counts that end inside a group of four tokens, heads of a wider projection
    laid out head by head, in place and beside; what is behind a count, and the
    projection's other heads, as they were."""
    from paper_2608_24063_amd.tensors import Rope
    assert L * B * n > 2048 and B * n % 4
    rng = np.random.default_rng(d + rot + n)
    typ = torch.float32 if fp32 else torch.bfloat16
    wide = rng.standard_normal((L, B, Hq + 2 * Hkv, n, d)).astype(np.float32)
    wide = wide if fp32 else ref.bf16(wide)
    pos = rng.integers(-50, 20000, (3, B, n)).astype(np.int32)
    counts = [n, 0, n - 1, n + 9, 5][:B]
    sections = (rot // 2 - 2 * (rot // 8), rot // 8, rot // 8)
    rope = Rope(d, rot=rot, theta=1e5, sections=sections, pairing=int(adjacent), scale=0.75)
    freq, ax = [1e5 ** (-2.0 * i / rot) for i in range(rot // 2)], ref.rope_axes(rot, sections, False)
    tp, cnt = torch.from_numpy(pos).to(dev), torch.tensor(counts, dtype=torch.int32, device=dev)
    for inverse in (False, True):
        w = torch.from_numpy(wide).to(dev).to(typ)
        t = w.transpose(2, 3)
        beside = [torch.full((L, B, n, h, d), 7.0, dtype=typ, device=dev) for h in (Hq, Hkv)]
        rope.apply(tp, t[:, :, :, :Hq], t[:, :, :, Hq:Hq + Hkv], q_out=beside[0], k_out=beside[1], count=cnt, inverse=inverse)
        torch.cuda.synchronize()
        assert np.array_equal(w.float().cpu().numpy(), wide)
        rope.apply(tp, t[:, :, :, :Hq], t[:, :, :, Hq:Hq + Hkv], count=cnt, inverse=inverse)
        got, was = t.float().cpu().numpy(), wide.transpose(0, 1, 3, 2, 4)
        assert np.array_equal(got[:, :, :, Hq + Hkv:], was[:, :, :, Hq + Hkv:])
        out = torch.cat(beside, dim=3).float().cpu().numpy()
        for b, c in enumerate(min(max(x, 0), n) for x in counts):
            assert np.array_equal(got[:, b, c:], was[:, b, c:]) and (out[:, b, c:] == 7.0).all()
            assert np.array_equal(got[:, b, :c, :Hq + Hkv], out[:, b, :c])
            m = min(c, 40)
            for sl in (slice(0, m), slice(c - m, c)) if c else ():
                _check(got[:, b:b + 1, sl, :Hq + Hkv], was[:, b:b + 1, sl, :Hq + Hkv], pos[:, b:b + 1, sl], rot, freq, ax,
                       adjacent, inverse, 0.75, fp32)
