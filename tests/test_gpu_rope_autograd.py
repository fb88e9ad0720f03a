"""The rotation and autograd: it writes through addresses, so what autograd would
record without it is refused, and what it writes counts as changed."""
import numpy as np
import pytest

from tests.test_gpu_rope import dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture()
def call(dev):  # noqa: F811
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(81)
    x = [torch.from_numpy(rng.standard_normal((1, 2, 9, h, 64)).astype(np.float32)).to(dev) for h in (4, 2)]
    pos = torch.from_numpy(rng.integers(0, 9000, (3, 2, 9)).astype(np.int32)).to(dev)
    return Rope(64, sections=(8, 12, 12)), pos, x[0], x[1]


def test_what_requires_grad_is_refused(call):
    rope, pos, q, k = call
    was = q.clone()
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    for args in (dict(q=leaf(q)), dict(q=leaf(q) * 1, k=k), dict(q=q, k=leaf(k)), dict(k=leaf(k)),
                 dict(q=leaf(q), q_out=torch.empty_like(q)), dict(q=q, q_out=leaf(q)), dict(q=q, k=k, k_out=leaf(k) * 1)):
        with pytest.raises(ValueError, match="requires grad"):
            rope.apply(pos, **args)
    torch.cuda.synchronize()
    assert torch.equal(q, was)
    # where nothing is recorded they are ordinary tensors
    want = rope.apply(pos, q=q.clone())[0]
    with torch.no_grad():
        assert torch.equal(rope.apply(pos, q=leaf(q))[0], want)
    with torch.inference_mode():
        assert torch.equal(rope.apply(pos, q=q.clone())[0], want)


def test_outputs_count_as_changed(call):
    rope, pos, q, k = call
    w = torch.ones((64,), device=q.device, requires_grad=True)
    for rotate in (lambda: rope.apply(pos, q=q), lambda: rope.apply(pos, k=k, k_out=q[:, :, :, :2]),
                   lambda: rope.apply(pos, q, k), lambda: rope.apply(pos, q=q, inverse=True)):
        loss = (q * w).sum()  # keeps q for the gradient of w
        rotate()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    v = q._version
    rope.apply(pos, q=q, q_out=torch.empty_like(q))
    assert q._version == v  # an input is not


def test_step_turns_rows_that_require_grad(call):
    """A serving step records nothing, with one token or several, and leaves its rows alone."""
    from paper_2608_24063_amd.tensors import Q8Cache, Rope
    rope, _, q, _ = call
    rope = Rope(64)
    outs = []
    for grad in (False, True):
        c = Q8Cache(1, 1, 4, 2, 64, [40, 40], q.device)
        for n in (3, 1):
            g = torch.Generator(device=q.device)
            g.manual_seed(n)
            x = [torch.randn((1, 1, n, h, 64), generator=g, device=q.device).to(torch.bfloat16).requires_grad_(grad) for h in (4, 2, 2)]
            out = torch.zeros((1, 1, n, 4, 64), dtype=torch.float32, device=q.device)
            c.step(*x, out, 0.125, rope=rope, pos=torch.full((3, 1, n), 7, dtype=torch.int32, device=q.device))
            outs.append(out)
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


def test_inside_an_autograd_function(call):
    """The pair as a program wraps it: the gradient through the function is the rotation
    by the negative angle, against autograd of a plain rotation in 64 bits."""
    rope, pos, q, _ = call

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return rope.apply(pos, q=x, q_out=torch.empty_like(x))[0]

        @staticmethod
        def backward(ctx, g):
            g = g.contiguous()
            return rope.apply(pos, q=g, q_out=torch.empty_like(g), inverse=True)[0]

    leaf, weight = q.clone().requires_grad_(), torch.randn_like(q)
    (Turn.apply(leaf) * weight).sum().backward()
    freq = 1e6 ** (-2.0 * torch.arange(32, dtype=torch.float64) / 64)
    axis = torch.tensor([0] * 8 + [1] * 12 + [2] * 12)
    a = pos.cpu()[axis].permute(1, 2, 0).double() * freq
    c, s = torch.cos(a)[None, :, :, None], torch.sin(a)[None, :, :, None]
    x = q.cpu().double().requires_grad_()
    y = torch.cat((x[..., :32] * c - x[..., 32:] * s, x[..., 32:] * c + x[..., :32] * s), dim=-1)
    (y * weight.cpu().double()).sum().backward()
    tol = 2 * weight.abs().max().item() * 2.0 ** -20
    assert (leaf.grad.cpu().double() - x.grad).abs().max() <= tol
