"""GPU parity of the rotary positions with several axes (viscache_rope) against
the 64-bit form of tests/q8_ref.py, its gradient against the formula and against
differences.

Tolerances: the angle is reduced in 64 bits, so sine and cosine come from a
reduced angle rounded to fp32 (2^-25 of a turn, 2 pi 2^-25 < 2^-22 in the angle) and
are themselves off by a few steps of fp32: 2^-21 together; the rotation takes three
roundings of 2^-24, each relative to |x1| + |x2|.  So (|x1| + |x2|) scale 2^-20, plus
half a step of bf16 (2^-8 of the value) where the output is bf16."""
import numpy as np
import pytest

from tests import q8_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2608_24063_amd as vc
    vc.lib()
    return torch.device("cuda:0")


def _check(got, x, pos, rot, freq, ax, adjacent, inverse, scale, fp32):
    """got, x [L, B, n, H, d]; pos [3, B, n]."""
    for l in range(x.shape[0]):
        for b in range(x.shape[1]):
            for h in range(x.shape[3]):
                want = ref.rope(x[l, b, :, h], pos[:, b], rot, freq, ax, adjacent, inverse, scale)
                size = np.zeros_like(want)
                for i in range(rot // 2):
                    p, q = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
                    size[:, p] = size[:, q] = np.abs(x[l, b, :, h, p]) + np.abs(x[l, b, :, h, q])
                tol = size * abs(scale) * 2.0 ** -20 + (0 if fp32 else np.abs(want) * 2.0 ** -8)
                tol[:, rot:] = 0  # copied
                assert (np.abs(got[l, b, :, h] - want) <= tol).all(), (l, b, h)


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("d,rot,sections,inter", [(128, 128, (16, 24, 24), False), (128, 128, (24, 20, 20), True),
                                                  (64, 64, (32, 0, 0), False), (128, 64, (10, 11, 11), True),
                                                  (64, 16, (0, 4, 4), False), (64, 32, (0, 0, 16), True)])
@pytest.mark.parametrize("L,B,n,Hq,Hkv", [(3, 2, 1, 14, 2), (1, 3, 67, 5, 5), (1, 1, 8300, 2, 1)])
def test_rotation(dev, fp32, adjacent, d, rot, sections, inter, L, B, n, Hq, Hkv):
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(d + rot + n)
    typ = torch.float32 if fp32 else torch.bfloat16
    q, k = rng.standard_normal((L, B, n, Hq, d)), 3 * rng.standard_normal((L, B, n, Hkv, d))
    q, k = (x.astype(np.float32) if fp32 else ref.bf16(x) for x in (q, k))
    pos = rng.integers(-100, 20000, (3, B, n)).astype(np.int32)
    for inverse, scale in ((False, 1.0), (True, 0.75)):
        r = Rope(d, rot=rot, theta=1e5, sections=sections, layout=int(inter), pairing=int(adjacent), scale=scale)
        tq, tk = torch.from_numpy(q).to(dev).to(typ), torch.from_numpy(k).to(dev).to(typ)
        tp = torch.from_numpy(pos).to(dev)
        oq, ok = r.apply(tp, tq, tk, q_out=torch.empty_like(tq), k_out=torch.empty_like(tk), inverse=inverse)
        torch.cuda.synchronize()
        assert np.array_equal(tq.float().cpu().numpy(), q)
        freq, ax = [1e5 ** (-2.0 * i / rot) for i in range(rot // 2)], ref.rope_axes(rot, sections, inter)
        m = min(n, 64)  # the plain form of the long case: its first and last tokens
        for sl in (slice(0, m), slice(n - m, n)):
            _check(oq.float().cpu().numpy()[:, :, sl], q[:, :, sl], pos[:, :, sl], rot, freq, ax, adjacent, inverse, scale, fp32)
            _check(ok.float().cpu().numpy()[:, :, sl], k[:, :, sl], pos[:, :, sl], rot, freq, ax, adjacent, inverse, scale, fp32)
        # in place, and each alone, give the same bits
        r.apply(tp, tq, tk, inverse=inverse)
        assert torch.equal(tq, oq) and torch.equal(tk, ok)
        tq2 = torch.from_numpy(q).to(dev).to(typ)
        r.apply(tp, q=tq2, inverse=inverse)
        tk2 = torch.from_numpy(k).to(dev).to(typ)
        r.apply(tp, k=tk2, inverse=inverse)
        assert torch.equal(tq2, oq) and torch.equal(tk2, ok)


def test_far_positions_and_own_frequencies(dev):
    """Positions up to 2^31 - 1 and below zero, with frequencies of the caller's."""
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(2)
    d, n = 64, 33
    freq = rng.uniform(0, 1, d // 2)
    freq[0], freq[1] = 1.0, 0.0
    pos = rng.integers(-2 ** 31, 2 ** 31, (3, 1, n)).astype(np.int32)
    pos[0, 0, :3] = [2 ** 31 - 1, -2 ** 31, 0]
    x = rng.standard_normal((1, 1, n, 2, d)).astype(np.float32)
    t = torch.from_numpy(x).to(dev)
    Rope(d, sections=(20, 6, 6), inv_freq=freq).apply(torch.from_numpy(pos).to(dev), q=t)
    got = t.cpu().numpy()
    ax = ref.rope_axes(d, (20, 6, 6), False)
    for h in range(2):
        want = ref.rope(x[0, 0, :, h], pos[:, 0], d, freq, ax, False, False, 1.0)
        # Both sides round pos * f (over 2 pi or not) to 53 bits at 2^31: 2^-21 each.
        tol = np.abs(x[0, 0, :, h]).max(axis=1, keepdims=True) * 2 * (2.0 ** -20 + 2 * 2.0 ** -21 * 6.3)
        assert (np.abs(got[0, 0, :, h] - want) <= tol).all()


@pytest.mark.parametrize("adjacent", [False, True])
def test_gradient(dev, adjacent):
    """The inverse is the gradient: the formula's, through autograd in 64 bits, and
    differences: for a linear map <g, f(x + e) - f(x)> = <grad, e> for every e."""
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(3)
    L, B, n, H, d, rot = 2, 2, 19, 3, 64, 32
    sections = (6, 5, 5)
    x, g, e = (rng.standard_normal((L, B, n, H, d)).astype(np.float32) for _ in range(3))
    pos = rng.integers(0, 9000, (3, B, n)).astype(np.int32)
    r = Rope(d, rot=rot, theta=1e4, sections=sections, pairing=int(adjacent), scale=1.25)
    tp = torch.from_numpy(pos).to(dev)
    grad = torch.from_numpy(g).to(dev)
    r.apply(tp, q=grad, inverse=True)
    # the formula, by autograd over the plain form
    f = torch.tensor([1e4 ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64)
    ax = torch.tensor(ref.rope_axes(rot, sections, False))
    a = torch.from_numpy(pos)[ax].permute(1, 2, 0).double() * f
    c, s = torch.cos(a)[None, :, :, None], torch.sin(a)[None, :, :, None]
    leaf = torch.from_numpy(x).double().requires_grad_()
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if adjacent else (slice(0, rot // 2), slice(rot // 2, rot))
    y = leaf.clone()
    y[..., lo] = 1.25 * (leaf[..., lo] * c - leaf[..., hi] * s)
    y[..., hi] = 1.25 * (leaf[..., hi] * c + leaf[..., lo] * s)
    y.backward(torch.from_numpy(g).double())
    assert (grad.cpu().double() - leaf.grad).abs().max() <= 2 * np.abs(g).max() * 1.25 * 2.0 ** -20
    t0, t1 = torch.from_numpy(x).to(dev), torch.from_numpy(x + e).to(dev)
    r.apply(tp, q=t0)
    r.apply(tp, q=t1)
    torch.cuda.synchronize()
    left = (torch.from_numpy(g).double() * (t1 - t0).cpu().double()).sum()
    right = (grad.cpu().double() * (torch.from_numpy(x + e).double() - torch.from_numpy(x).double())).sum()
    terms = np.abs(g).sum() * np.abs(x).max() * 4 * 2.0 ** -19
    assert abs(float(left - right)) <= terms


def test_counts_strides_and_streams(dev):
    """Tokens behind a sequence's count stay as they were; heads of one wider
    projection, in place, on another stream."""
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(4)
    L, B, n, Hq, Hkv, d = 1, 4, 21, 6, 2, 64
    wide = ref.bf16(rng.standard_normal((L, B, n, Hq + 2 * Hkv, d)))
    pos = rng.integers(0, 500, (3, B, n)).astype(np.int32)
    w, tp = torch.from_numpy(wide).to(dev).to(torch.bfloat16), torch.from_numpy(pos).to(dev)
    count = torch.tensor([n, 0, 5, -1], dtype=torch.int32, device=dev)
    r = Rope(d, sections=(8, 12, 12), theta=1e4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        r.apply(tp, w[:, :, :, :Hq], w[:, :, :, Hq:Hq + Hkv], count=count)
    torch.cuda.synchronize()
    got = w.float().cpu().numpy()
    freq, ax = [1e4 ** (-2.0 * i / d) for i in range(d // 2)], ref.rope_axes(d, (8, 12, 12), False)
    for b, c in enumerate([n, 0, 5, 0]):
        assert np.array_equal(got[:, b, c:], wide[:, b, c:])
        assert np.array_equal(got[:, b, :, Hq + Hkv:], wide[:, b, :, Hq + Hkv:])
        if c:
            _check(got[:, b:b + 1, :c, :Hq + Hkv], wide[:, b:b + 1, :c, :Hq + Hkv], pos[:, b:b + 1, :c], d, freq, ax,
                   False, False, 1.0, False)


def test_graph_replays(dev):
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(5)
    r = Rope(128, sections=(16, 24, 24))
    x = torch.from_numpy(rng.standard_normal((2, 1, 40, 4, 128)).astype(np.float32)).to(dev)
    pos = torch.zeros((3, 1, 40), dtype=torch.int32, device=dev)
    out, want = torch.empty_like(x), torch.empty_like(x)
    r.apply(pos, q=x, q_out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.apply(pos, q=x, q_out=out)
    for t in range(4):
        pos.copy_(torch.from_numpy(rng.integers(0, 10000, (3, 1, 40)).astype(np.int32)))
        g.replay()
        r.apply(pos, q=x, q_out=want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), t


def test_refusals_and_empty(dev):
    """Tensors that do not belong together are refused before a launch; no tokens
    are nothing to do, no heads an error."""
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import Rope
    rope = Rope(64)
    z = lambda *s, t=torch.bfloat16: torch.ones(s, dtype=t, device=dev)  # noqa: E731
    pos = torch.ones((3, 2, 5), dtype=torch.int32, device=dev)
    q, k = z(1, 2, 5, 4, 64), z(1, 2, 5, 2, 64)
    for bad in (dict(k=z(1, 2, 4, 2, 64)), dict(k=z(2, 5, 2, 64)), dict(k=z(1, 2, 5, 2, 128)),
                dict(k=z(1, 2, 5, 2, 64, t=torch.float32)), dict(q_out=z(1, 2, 5, 2, 64)), dict(k_out=z(1, 2, 5, 4, 64)),
                dict(q=z(1, 2, 5, 4, 128)), dict(q=z(1, 2, 5, 4, 64, t=torch.float16)), dict(k=k.cpu()),
                dict(q=z(1, 2, 5, 64, 4).transpose(3, 4)), dict(pos=pos[:, :, :4]), dict(pos=pos.long()),
                dict(count=torch.ones(3, dtype=torch.int32, device=dev))):
        args = dict(pos=pos, q=q, k=k)
        args.update(bad)
        with pytest.raises(ValueError):
            rope.apply(**args)
    with pytest.raises(vc.VisCacheError):
        rope.apply(pos, q, z(1, 2, 5, 0, 64))
    with pytest.raises(vc.VisCacheError):
        rope.apply(None, q, k)
    torch.cuda.synchronize()
    assert (q == 1).all() and (k == 1).all()
    rope.apply(pos[:, :, :0].contiguous(), z(1, 2, 0, 4, 64), z(1, 2, 0, 2, 64))
