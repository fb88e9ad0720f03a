"""A serving run as a program makes it: rows are normed and turned, appended and attended,
their weights added up, and the cache cut back by them when it is over its budget; every
step against the same run in 64 bits, which goes on from the library's rows where its
rounding of them and its choice between near masses enter."""
import numpy as np
import pytest

from tests import mass_ref, q8_ref as ref
from tests.norm_ref import Norm
from tests.test_gpu_mass_attend import dev  # noqa: F401
from tests.test_gpu_mass_evict import kept_rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fp32", [False, True])
def test_answers_under_a_budget(dev, fp32):  # noqa: F811
    from paper_2608_24063_amd.tensors import MassCache, NormRope, Rope
    L, B, Hq, Hkv, d, budget, cap = 2, 2, 8, 2, 64, 96, 200
    G, scale, rng = Hq // Hkv, d ** -0.5, np.random.default_rng(3)
    units = L * B * Hkv
    sections = (12, 10, 10)
    rope = NormRope(Rope(d, theta=1e4, sections=sections), eps=1e-5)
    args = (d, [1e4 ** (-2.0 * i / d) for i in range(d // 2)], ref.rope_axes(d, sections, False), False)
    c = MassCache(L, B, Hq, Hkv, d, [cap] * units, dev)
    spare = MassCache(L, B, Hq, Hkv, d, [budget] * units, dev)
    keep = torch.full((units,), budget, dtype=torch.int32, device=dev)
    host = [mass_ref.Unit(np.zeros((0, d), np.float32), np.zeros((0, d), np.float32), np.zeros(0), cap) for _ in range(units)]
    put = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev).to(torch.bfloat16)  # noqa: E731
    out_np = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    w = {s: 1 + 0.2 * rng.standard_normal((L, d)).astype(np.float32) for s in "qk"}
    tw = {s: torch.from_numpy(x).to(dev) for s, x in w.items()}
    at, cuts = 0, 0
    for n in (130, 1, 1, 1, 40, 3, 1, 70, 1, 1):
        x = {s: ref.bf16(rng.standard_normal((L, B, n, H, d))) for s, H in (("q", Hq), ("k", Hkv), ("v", Hkv))}
        pos = np.broadcast_to(at + np.arange(n, dtype=np.int32), (3, B, n)).copy()
        t = {s: put(y) for s, y in x.items()}
        rope.apply(torch.from_numpy(pos).to(dev), t["q"], t["k"], tw["q"], tw["k"])
        turned = {}
        for s in "qk":
            nr = Norm(x[s], w[s], pos, *args, eps=1e-5)
            turned[s] = out_np(t[s])
            assert (np.abs(turned[s] - nr.forward()) <= nr.forward_tol(False)).all()
        out = torch.zeros((L, B, n, Hq, d), dtype=torch.float32 if fp32 else torch.bfloat16, device=dev)
        c.attend(t["q"], out, scale, k=t["k"], v=t["v"], decay=0.9)
        mass, lens = c.mass.cpu().numpy(), c.len.tolist()
        for u, unit in enumerate(host):
            l, b, g = u // (B * Hkv), u // Hkv % B, u % Hkv
            heads = slice(g * G, (g + 1) * G)
            want, tol, size = unit.attend(turned["q"][l, b, :, heads], scale, turned["k"][l, b, :, g].astype(np.float32),
                                          x["v"][l, b, :, g], 0.9)
            got = out_np(out[l, b, :, heads])
            assert (np.abs(got - want) <= mass_ref.out_tol(want, tol, size, fp32, n * G > 16)).all(), (n, u)
            assert lens[u] == len(unit.K)
            m = mass[cap * u:cap * u + lens[u]]
            assert (np.abs(m - unit.mass) <= unit.mass_tol).all(), (n, u)
        at += n
        if max(lens) > budget:  # over the budget: cut back, in place and through the other cache in turn
            cuts += 1
            rows = [kept_rows(mass[int(o):][:r], budget, 4, 16) for o, r in zip(c.row_off.tolist(), lens)]
            if cuts % 2:
                c.evict(keep, sinks=4, recent=16)
            else:
                c.evict(keep, sinks=4, recent=16, to=spare)
                big = MassCache(L, B, Hq, Hkv, d, [cap] * units, dev)
                spare.evict(keep, to=big)
                c = big
            for unit, r in zip(host, rows):
                unit.K, unit.V, unit.mass, unit.mass_tol = unit.K[r], unit.V[r], unit.mass[r], unit.mass_tol[r]
            K, V, lens = out_np(c.k_pool), out_np(c.v_pool), c.len.tolist()
            for unit, o, r in zip(host, c.row_off.tolist(), lens):
                assert r == len(unit.K) and np.array_equal(K[o:o + r], unit.K) and np.array_equal(V[o:o + r], unit.V)
    assert cuts >= 3
