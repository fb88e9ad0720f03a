"""A step, a question and an eviction of one cache, captured into graphs of their own that
share its workspace, replayed after one another with eager calls between them that make the
workspace grow; every state against the same calls made eagerly on a cache of its own."""
import pytest

from tests.test_gpu_mass_attend import Pair, _bf16, dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fp32", [True, False])
def test_graphs_that_share_a_workspace(dev, fp32):  # noqa: F811
    lens = [1500, 40, 0, 700, 64, 1, 900, 333]
    a, b = (Pair(67, dev, 2, 2, 8, 2, 64, lens, [2600] * 8) for _ in range(2))
    typ = torch.float32 if fp32 else torch.bfloat16
    step, ask = [[_bf16(x, dev) for x in a.inputs(n)] for n in (1, 40)]
    outs = {c: [torch.zeros(x[0].shape, dtype=typ, device=dev) for x in (step, ask)] for c in (a, b)}
    keep = torch.tensor([600, 40, 0, 500, 10, 1, 900, 100], dtype=torch.int32, device=dev)
    index = {c: torch.full((8, 900), -1, dtype=torch.int32, device=dev) for c in (a, b)}

    def calls(c):
        return (lambda: c.c.attend(step[0], outs[c][0], 0.125, k=step[1], v=step[2], decay=0.9),
                lambda: c.c.attend(ask[0], outs[c][1], 0.125, k=ask[1], v=ask[2]),
                lambda: c.c.evict(keep, sinks=4, recent=16, index=index[c]))
    for c in (a, b):
        for f in calls(c):  # (a call that is captured has run once)
            f()
    torch.cuda.synchronize()
    side, graphs = torch.cuda.Stream(), []
    for f in calls(b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            f()
    before = b.c._ws.numel()
    for turn, which in enumerate((0, 1, 2, 0, 0, 1, 2, 2, 1, 0, 2)):
        graphs[which].replay()
        calls(a)[which]()
        if turn in (2, 6):  # eager calls of other sizes, the first of which needs more room
            n = (90, 3)[turn > 2]
            q, k, v = (_bf16(x, dev) for x in a.inputs(n))
            o = [torch.zeros(q.shape, dtype=typ, device=dev) for _ in range(2)]
            a.c.attend(q, o[0], 0.125, k=k, v=v)
            b.c.attend(q, o[1], 0.125, k=k, v=v)
            assert torch.equal(*o)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs[a], outs[b]))
        assert torch.equal(a.c.len, b.c.len) and torch.equal(index[a], index[b])
        for u, o in enumerate(a.off):
            r = slice(o, o + int(a.c.len[u]))
            assert torch.equal(a.c.mass[r], b.c.mass[r]), (turn, u)
            for x, y in ((a.c.k_pool, b.c.k_pool), (a.c.v_pool, b.c.v_pool)):
                assert torch.equal(x[r].view(torch.int16), y[r].view(torch.int16)), (turn, u)
    assert b.c._ws.numel() > before
