"""Forward-mode autograd and the rotations, on the host (what they refuse is looked at before
the device is): a tensor's tangent would stay what it was while its rows are turned."""
import pytest

torch = pytest.importorskip("torch")
forward = torch.autograd.forward_ad


@pytest.fixture(scope="module")
def calls():
    from paper_2608_24063_amd.tensors import NormRope, Rope
    rope = Rope(64)
    return rope, NormRope(rope)


def test_tensors_with_a_tangent_are_refused(calls):
    rope, normed = calls
    pos = torch.zeros((3, 1, 2), dtype=torch.int32)
    x, w = torch.ones((1, 1, 2, 2, 64)), torch.ones((1, 64))
    with forward.dual_level():
        d, dw = forward.make_dual(x, x), forward.make_dual(w, w)
        for f in (lambda: rope.apply(pos, q=d), lambda: rope.apply(pos, k=d), lambda: rope.apply(pos, q=x, q_out=d),
                  lambda: rope.apply(pos, q=x, k=x, k_out=d), lambda: normed.apply(pos, q=d, q_weight=w),
                  lambda: normed.apply(pos, q=x, q_weight=dw), lambda: normed.apply(pos, k=x, k_weight=w, k_out=d),
                  lambda: normed.grad(pos, q=x, q_weight=w, q_dout=d), lambda: normed.grad(pos, q=d, q_weight=w, q_dout=x),
                  lambda: normed.grad(pos, q=x, q_weight=w, q_dout=x, q_din=d)):
            with pytest.raises(ValueError, match="tangent"):
                f()
            with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
                f()
        # others are not, in the same place (they go on to the check of their device)
        for f in (lambda: rope.apply(pos, q=x), lambda: normed.apply(pos, q=x, q_weight=w)):
            with pytest.raises(ValueError, match="on GPU|need"):
                f()


def test_a_function_of_the_programs_own(calls):
    """Inside the forward of an autograd function the tensors carry none."""
    rope, _ = calls
    pos = torch.zeros((3, 1, 2), dtype=torch.int32)

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(x):
            return rope.apply(pos, q=x, q_out=torch.empty_like(x))[0]

        @staticmethod
        def setup_context(ctx, inputs, output):
            pass

        @staticmethod
        def jvp(ctx, t):
            return t
    with forward.dual_level():
        x = forward.make_dual(torch.ones((1, 1, 2, 2, 64)), torch.ones((1, 1, 2, 2, 64)))
        with pytest.raises(ValueError, match="on GPU|need"):  # (its device)
            Turn.apply(x)
