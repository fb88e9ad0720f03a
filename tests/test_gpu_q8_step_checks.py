"""A step of several tokens that its attention would refuse appends nothing."""
import numpy as np
import pytest

from tests.test_gpu_q8 import _filled, _same_caches, _t, _values, dev  # noqa: F401

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


@pytest.mark.parametrize("n", [1, 3, 20])
def test_rotated_rows_are_left_where_asked(dev, n):  # noqa: F811
    """q_out and k_out, either or both, whatever the number of tokens; refused before
    anything is appended where they do not fit."""
    from paper_2608_24063_amd.tensors import Rope
    a = _filled(np.random.default_rng(73), dev, 1, 2, 8, 2, 64, [100, 63, 64, 0], "e4m3", extra=90)[0]
    args, rope = _args(dev, n), Rope(64, sections=(8, 12, 12))
    pos = torch.from_numpy(np.random.default_rng(74).integers(0, 9000, (3, 2, n)).astype(np.int32)).to(dev)
    q, k = args["q"].clone(), args["k"].clone()
    wq, wk = rope.apply(pos, q, k)
    for names in (("q_out",), ("k_out",), ("q_out", "k_out")):
        given = {x: torch.full_like(wq if x == "q_out" else wk, 7.0) for x in names}
        a.step(**args, rope=rope, pos=pos, **given)
        assert all(torch.equal(t, wq if x == "q_out" else wk) for x, t in given.items())
    # in place, and the same results as a step that is not asked for them
    b = _filled(np.random.default_rng(73), dev, 1, 2, 8, 2, 64, [100, 63, 64, 0], "e4m3", extra=90)[0]
    c = _filled(np.random.default_rng(73), dev, 1, 2, 8, 2, 64, [100, 63, 64, 0], "e4m3", extra=90)[0]
    ob = torch.zeros_like(args["out"])
    b.step(args["q"], args["k"], args["v"], ob, 0.125, rope=rope, pos=pos)
    q, k = args["q"].clone(), args["k"].clone()
    c.step(q, k, args["v"], args["out"], 0.125, rope=rope, pos=pos, q_out=q, k_out=k)
    assert torch.equal(q, wq) and torch.equal(k, wk) and torch.equal(ob, args["out"])
    _same_caches(b, c)
    before = a.len.clone()
    for bad in (dict(q_out=wk), dict(k_out=wq), dict(q_out=wq.float()), dict(k_out=wk.cpu())):
        with pytest.raises(ValueError):
            a.step(**args, rope=rope, pos=pos, **bad)
    assert torch.equal(a.len, before)


@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("most", [0, 64, 150, 2 ** 40])
def test_row_bound_of_a_step(dev, n, most):  # noqa: F811
    """max_rows bounds what a step attends, and nothing else."""
    a, b = (_filled(np.random.default_rng(75), dev, 1, 2, 8, 2, 64, [100, 63, 64, 300], "int8", extra=90)[0]
            for _ in range(2))
    args = _args(dev, n)
    want = torch.zeros_like(args["out"])
    a.step(**args, max_rows=most)
    b.append(args["k"], args["v"])
    b.attend(args["q"], want, 0.125, max_rows=most)
    assert torch.equal(args["out"], want)
    _same_caches(a, b)
    with pytest.raises(Exception):
        a.step(**args, max_rows=-1)
    _same_caches(a, b)
