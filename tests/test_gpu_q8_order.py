"""The order in which single-token calls over the 8-bit cache start on its units:
any permutation gives the same results, and a unit that it leaves out is left
alone, whether units are cut in pieces that a second launch joins or not, and
whatever the workspace holds."""
import numpy as np
import pytest

from tests.test_gpu_q8 import _filled, _t, _values, dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("lens", [[6398, 6399, 12, 8063], [63, 64, 12, 200]], ids=["cut", "whole"])
@pytest.mark.parametrize("order", [[3, 1, 0, 2], [2, 0, -1, 99], [-1, -1, 1, 2 ** 31 - 1], [-2 ** 31, 4, -1, 5]], ids=str)
@pytest.mark.parametrize("form", ["step", "attend", "draft"])
def test_order(dev, lens, order, form):  # noqa: F811
    L, B, Hq, Hkv, d = 1, 2, 14, 2, 128
    a, b = (_filled(np.random.default_rng(41), dev, L, B, Hq, Hkv, d, lens, "e4m3", extra=5)[0] for _ in range(2))
    a.order = torch.tensor(order, dtype=torch.int32, device=dev)
    a.c.order = a.order.data_ptr()
    b.c.order = None
    rng = np.random.default_rng(42)
    n = 2 if form == "draft" else 1
    taken = [u for u in range(4) if u in order]
    for t in range(3):
        q, k, v = (_t(_values(rng, (L, B, n, h, d)), dev) for h in (Hq, Hkv, Hkv))
        oa, ob = (torch.full((L, B, n, Hq, d), 7.0, dtype=torch.float32, device=dev) for _ in range(2))
        before = {x: getattr(a, x).view(torch.uint8).clone() for x in ("k_codes", "v_codes", "k_scale", "v_scale")}
        tails, len0 = (a.k_tail.clone(), a.v_tail.clone()), a.len.clone()
        a._workspace(n, a.max_cap)
        a._ws.fill_(0xFF)  # what no launch has written is no part
        if form == "step":
            a.step(q, k, v, oa, 0.09)
            b.step(q, k, v, ob, 0.09)
        else:
            a.attend(q, oa, 0.09)
            b.attend(q, ob, 0.09)
        torch.cuda.synchronize()
        for u in range(4):
            mine = slice(u % 2 * 7, u % 2 * 7 + 7)
            blocks = slice(int(a.row_off[u]) // 64, (int(a.row_off[u]) + int(a.cap[u]) + 63) // 64)
            if u in taken:
                assert torch.equal(oa[0, u // 2, :, mine], ob[0, u // 2, :, mine]), u
                assert torch.equal(a.len[u], b.len[u])
                assert torch.equal(a.k_tail[u].view(torch.uint8), b.k_tail[u].view(torch.uint8))
                assert torch.equal(a.v_tail[u].view(torch.uint8), b.v_tail[u].view(torch.uint8))
            else:
                assert (oa[0, u // 2, :, mine] == 7.0).all(), u
                assert torch.equal(a.len[u], len0[u])
                assert torch.equal(a.k_tail[u].view(torch.uint8), tails[0][u].view(torch.uint8))
                assert torch.equal(a.v_tail[u].view(torch.uint8), tails[1][u].view(torch.uint8))
                for x, was in before.items():
                    now = getattr(a, x).view(torch.uint8)
                    assert torch.equal(now.reshape(len(a.k_scale), -1)[blocks], was.reshape(len(a.k_scale), -1)[blocks]), x
