"""Loading a pruned cache into an 8-bit one: all of its rows, or none."""
import pytest

from tests.test_gpu_q8 import dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_rows_are_not_dropped(dev, sg):  # noqa: F811
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import PruneCall, Q8Cache
    from synthgen.device import upload_layers
    w = sg.TINY
    dv, _ = upload_layers(w, range(w.L), dev, keep_host=True)
    pc = PruneCall(w.B, w.L, w.Hq, w.Hkv, w.d, w.W, [int(x) for x in w.n_vis()], vc.make_params(w.retention),
                   [dv["K"][l] for l in range(w.L)], [dv["V"][l] for l in range(w.L)], [dv["Q"][l] for l in range(w.L)])
    pc.run()
    units = w.L * w.B * w.Hkv
    kept = [pc.k[u // w.Hkv % w.B * w.L + u // (w.B * w.Hkv)] for u in range(units)]
    assert min(kept) == 0 < max(kept)
    exact = Q8Cache(w.L, w.B, w.Hq, w.Hkv, w.d, kept, dev)
    exact.load_pruned(pc)
    assert exact.len.tolist() == kept
    for short in (kept.index(max(kept)), max(u for u in range(units) if kept[u])):
        caps = [n + 3 * (u != short) - (u == short) for u, n in enumerate(kept)]
        c = Q8Cache(w.L, w.B, w.Hq, w.Hkv, w.d, caps, dev)
        with pytest.raises(ValueError, match=f"unit {short} "):
            c.load_pruned(pc)
        assert c.len.tolist() == [0] * units
    # rows that are there already take their room; units that get none need none
    c = Q8Cache(w.L, w.B, w.Hq, w.Hkv, w.d, [n + 3 for n in kept], dev)
    c.len.copy_(torch.tensor([3 if n else 1000 for n in kept], dtype=torch.int32))
    before = c.len.tolist()
    c.load_pruned(pc)
    assert c.len.tolist() == [n + 3 if n else 1000 for n in kept]
    with pytest.raises(ValueError):
        c.load_pruned(pc)
    assert c.len.tolist() != before
