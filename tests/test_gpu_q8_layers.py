"""One layer of an 8-bit cache at a time, through the entry points with the cache's
descriptors cut at the layer: the same cache and outputs as all layers in one call."""
import numpy as np
import pytest

from tests.test_gpu_q8 import FMTS, _check_attend, _filled, _same_caches, _t, _values, dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _layer(vc, c, l):
    per = c.B * c.Hkv
    at = slice(l * per, None)
    return vc.vc_q8cache(c.c.format, c.c.k_codes, c.c.v_codes, c.c.k_scale, c.c.v_scale, c.k_tail[at].data_ptr(),
                         c.v_tail[at].data_ptr(), c.row_off[at].data_ptr(), c.cap[at].data_ptr(), c.len[at].data_ptr(), None)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("lens", [[61, 62, 63, 64, 0, 1, 127, 700, 300, 63, 500, 64], [6398, 63, 4000, 12] * 3],
                         ids=["whole", "cut"])
def test_layer_by_layer(dev, fmt, lens):  # noqa: F811
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import Rope
    L, B, Hq, Hkv, d, extra = 3, 2, 8, 2, 64, 40
    a, b = (_filled(np.random.default_rng(111), dev, L, B, Hq, Hkv, d, lens, fmt, extra=extra)[0] for _ in range(2))
    one = vc.vc_decode_shape(B, 1, Hq, Hkv, d)
    rng = np.random.default_rng(112)
    rope, stream = Rope(d, sections=(8, 12, 12)), torch.cuda.current_stream().cuda_stream
    rows = lambda t: vc.vc_rows(t.data_ptr(), *t.stride()[:4])  # noqa: E731
    need = max(vc.viscache_q8_attend_workspace_bytes(one, n, a.max_cap) for n in (1, 9))
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    keep = [[] for _ in lens]
    for n in (1, 1, 9, 1):
        q, k, v = (_t(_values(rng, (L, B, n, h, d)), dev) for h in (Hq, Hkv, Hkv))
        pos = torch.from_numpy(rng.integers(0, 9000, (3, B, n)).astype(np.int32)).to(dev)
        oa, ob = (torch.full((L, B, n, Hq, d), 7.0, dtype=torch.float32, device=dev) for _ in range(2))
        a.step(q, k, v, oa, 0.125, rope=rope, pos=pos)
        tq, tk = rope.apply(pos, q.clone(), k.clone())
        for l in range(L):
            c, o = _layer(vc, b, l), ob[l:l + 1]
            if n == 1:
                vc.viscache_q8_step(one, c, rope._params[0][0], pos.data_ptr(), rows(q[l:l + 1]), rows(k[l:l + 1]),
                                    rows(v[l:l + 1]), rows(o), 1, 0.125, b.max_cap, ws.data_ptr(), need, stream)
            else:
                vc.viscache_q8_append(one, c, rows(tk[l:l + 1]), rows(v[l:l + 1]), n, 0, 0, stream)
                vc.viscache_q8_attend(one, c, rows(tq[l:l + 1]), rows(o), n, 0, 1, 1, 0.125, b.max_cap, ws.data_ptr(), need,
                                      stream)
        _same_caches(a, b)
        if max(lens) <= 12 * 64:  # never cut, so the sums are the same ones
            assert torch.equal(oa, ob)
        for u in range(len(lens)):
            l, s, g = u // (B * Hkv), u // Hkv % B, u % Hkv
            keep[u].append((tk[l, s, :, g].float().cpu().numpy(), v[l, s, :, g].float().cpu().numpy()))
    ko, vo = (torch.zeros((L, B, a.max_cap, Hkv, d), dtype=torch.float32, device=dev) for _ in "kv")
    b.read(ko, vo)
    at = lambda t, u: t[u // (B * Hkv), u // Hkv % B, :, u % Hkv].cpu().numpy().astype(np.float64)  # noqa: E731
    now = [n + 12 for n in lens]
    for u, n in enumerate(now):  # what is open still is the rows that came last
        for side, t in enumerate((ko, vo)):
            came = np.concatenate([x[side] for x in keep[u]])
            m = min(n % 64, len(came))
            assert np.array_equal(at(t, u)[n - m:n], came[len(came) - m:])
    K, V = ([at(t, u)[:n] for u, n in enumerate(now)] for t in (ko, vo))
    for out in (oa, ob):
        _check_attend(out.cpu().numpy(), tq.float().cpu().numpy(), K, V, now, L, B, Hq, Hkv, 0.125, [1] * B, True)
