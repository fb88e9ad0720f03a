"""The gradient of the normed rotation's weights over very many tokens: sums in parts of at
most 256 additions or one token's heads, and rows past 2^31 values."""
import numpy as np
import pytest

from tests.test_gpu_norm_rope import dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_many_equal_terms(dev):  # noqa: F811
    """16000 tokens alike in each of 1024 layers, whose workgroup's waves take 4000 each: x = 1
    throughout, so n = (1 + eps)^-1/2, positions of zero, so g = dout, a number of its own for
    each channel.  Added one after another the terms of a channel would all be rounded to the
    same side: of 64 channels the worst is off by 4000 / 2 half steps' mean, about 1e-4.
    Tolerance, of the sum: n 2^-20 (tests/norm_ref.py), a term's product and sum 256 roundings,
    the waves and groups 40 more."""
    from paper_2608_24063_amd.tensors import NormRope, Rope
    L, n, d = 1024, 16000, 64
    rope = NormRope(Rope(d), eps=1e-6)
    g = torch.from_numpy((1 + np.random.default_rng(3).random(d)).astype(np.float32)).to(dev)
    x = torch.ones((d,), device=dev)
    big = lambda t: t.expand(L, 1, n, 1, d)  # noqa: E731  (an input's rows may repeat)
    w = torch.ones((L, d), device=dev)
    pos = torch.zeros((3, 1, n), dtype=torch.int32, device=dev)
    din = torch.empty((L, 1, n, 1, d), device=dev)
    want = n * g.double() * (1 + float(np.float32(1e-6))) ** -0.5
    tol = want * (2.0 ** -20 + 296 * 2.0 ** -24)
    _, _, dw, _ = rope.grad(pos, q=big(x), q_weight=w, q_dout=big(g), q_din=din)
    assert ((dw.double() - want).abs() <= tol).all()
    _, _, _, dw2 = rope.grad(pos, k=big(x), k_weight=w, k_dout=big(g), k_din=din)
    assert torch.equal(dw, dw2)


def test_weights_past_32_bits(dev):  # noqa: F811
    """Rows past 2^31 values whose gradients are not zero in the first and last tokens alone,
    where every term of dw is a whole number: no sum rounds, so a head counted twice or left
    out is one too many or too few.  (x is +1 or -1, so n = x (1 + eps)^-1/2 with eps 2^-126 is
    x; positions of zero turn nothing.)"""
    from paper_2608_24063_amd.tensors import NormRope, Rope
    n, Hq, Hkv, d, m = 140_000, 128, 8, 128, 9
    rope = NormRope(Rope(d), eps=2.0 ** -126)
    g = torch.Generator(device=dev)
    g.manual_seed(5)
    pos = torch.zeros((3, 1, n), dtype=torch.int32, device=dev)
    w = torch.ones((2, 1, d), device=dev)

    def side(H):
        x = torch.empty((1, 1, n, H, d), dtype=torch.bfloat16, device=dev)
        x.random_(0, 2, generator=g).mul_(2).sub_(1)
        dout = torch.zeros_like(x)
        dout[:, :, :m].random_(1, 100, generator=g)
        dout[:, :, n - m:].random_(1, 100, generator=g)
        ends = torch.cat((torch.arange(m), torch.arange(n - m, n))).to(dev)
        want = (x[0, 0, ends].double() * dout[0, 0, ends].double()).sum(dim=(0, 1))
        return x, dout, want
    q, dq, wq = side(Hq)
    k, dk, wk = side(Hkv)
    assert q.numel() > 2 ** 31
    _, _, gq, gk = rope.grad(pos, q, k, w[0], w[1], dq, dk, q_din=dq, k_din=dk)
    assert torch.equal(gq[0].double(), wq) and torch.equal(gk[0].double(), wk)
