"""Attention with masses and eviction record nothing for autograd: tensors that require grad
are ordinary ones, and outputs have no history."""
import pytest

from tests.test_gpu_mass_attend import Pair, _bf16, dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("n", [1, 20])
def test_tensors_that_require_grad(dev, n):  # noqa: F811
    a, b = (Pair(61, dev, 1, 2, 8, 2, 64, [70, 5, 300, 0], [400] * 4) for _ in range(2))
    q, k, v = (_bf16(x, dev) for x in a.inputs(n))
    outs = [torch.zeros(q.shape, device=dev) for _ in range(2)]
    a.c.attend(q, outs[0], 0.125, k=k, v=v)
    q, k, v = (x.clone().requires_grad_() * 1 for x in (q, k, v))
    b.c.attend(q, outs[1], 0.125, k=k, v=v)
    assert torch.equal(*outs) and torch.equal(a.c.mass, b.c.mass)
    assert not outs[1].requires_grad and not b.c.mass.requires_grad and not b.c.k_pool.requires_grad
