"""A step of several tokens that its attention would refuse appends nothing."""
import numpy as np
import pytest

from tests.test_gpu_q8 import _filled, _t, _values, dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _args(dev, n=3):  # noqa: F811
    rng = np.random.default_rng(71)
    q, k, v = (_t(_values(rng, (1, 2, n, h, 64)), dev) for h in (8, 2, 2))
    return dict(q=q, k=k, v=v, out=torch.zeros_like(q), scale=0.125)


@pytest.mark.parametrize("turned", [False, True])
def test_refusals_of_the_attention_come_first(dev, turned):  # noqa: F811
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import Rope
    a = _filled(np.random.default_rng(72), dev, 1, 2, 8, 2, 64, [100, 63, 64, 0], "int8", extra=70)[0]
    args = _args(dev)
    if turned:
        args.update(rope=Rope(64), pos=torch.zeros((3, 2, 3), dtype=torch.int32, device=dev))
    before, tail = a.len.clone(), a.k_tail.clone()
    room = torch.zeros(args["q"].numel() + 4, dtype=torch.bfloat16, device=dev)
    off = room[4:].view(args["q"].shape)  # 8 bytes past a multiple of 16
    bad = [dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(out=off),
           dict(out=args["out"][:, :, :1].expand_as(args["out"]))]
    bad.append(dict(q_out=off) if turned else dict(q=off))
    for x in bad:
        with pytest.raises(vc.VisCacheError) as e:
            a.step(**{**args, **x})
        assert e.value.status == vc.VC_ERR_ARG
        torch.cuda.synchronize()
        assert torch.equal(a.len, before) and torch.equal(a.k_tail.view(torch.uint8), tail.view(torch.uint8))
    a.step(**args)
    assert torch.equal(a.len, before + 3)


def test_more_queries_than_attention_takes(dev):  # noqa: F811
    """n * Hq/Hkv past 2^24, which an append of as many rows is not."""
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import Q8Cache
    n = (1 << 22) + 1
    c = Q8Cache(1, 1, 4, 1, 64, [10], dev)
    one = torch.zeros((1, 1, 1, 4, 64), dtype=torch.bfloat16, device=dev)
    out = torch.empty((1, 1, n, 4, 64), dtype=torch.bfloat16, device=dev)
    kv = one[:, :, :, :1].expand(1, 1, n, 1, 64)
    with pytest.raises(vc.VisCacheError) as e:
        c.step(one.expand(1, 1, n, 4, 64), kv, kv, out, 0.1)
    assert e.value.status == vc.VC_ERR_UNSUPPORTED
    assert c.len.tolist() == [0]
