"""GPU parity of the normed rotation and its gradient (viscache_norm_rope,
viscache_norm_rope_grad) against 64 bits; tolerances are derived in tests/norm_ref.py."""
import numpy as np
import pytest

from tests import q8_ref as ref
from tests.norm_ref import Norm

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2608_24063_amd as vc
    vc.lib()
    return torch.device("cuda:0")


def _values(rng, shape, fp32, loud=3.0):
    x = loud * rng.standard_normal(shape)
    return x.astype(np.float32) if fp32 else ref.bf16(x)


def _put(x, dev, fp32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dev).to(torch.float32 if fp32 else torch.bfloat16)


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _problem(seed, dev, L, B, n, Hq, Hkv, d, rot, sections, inter, adjacent, fp32, w_fp32, scale=1.0, eps=1e-6):
    """A NormRope with its rows, weights and gradients on the GPU, and their values."""
    from paper_2608_24063_amd.tensors import NormRope, Rope
    rng = np.random.default_rng(seed)
    v = {"pos": rng.integers(-100, 200000, (3, B, n)).astype(np.int32), "n": n}
    for side, H in (("q", Hq), ("k", Hkv)):
        v[side] = _values(rng, (L, B, n, H, d), fp32)
        v[side + "_dout"] = _values(rng, (L, B, n, H, d), fp32, 0.01)
        v[side + "_weight"] = _values(rng, (L, d), w_fp32, 1.0)
    t = {k: _put(x, dev, w_fp32 if "weight" in k else fp32) for k, x in v.items() if k not in ("pos", "n")}
    t["pos"] = torch.from_numpy(v["pos"]).to(dev)
    rope = NormRope(Rope(d, rot=rot, theta=1e5, sections=sections, layout=int(inter), pairing=int(adjacent), scale=scale),
                    eps=eps)
    args = (rot, [1e5 ** (-2.0 * i / rot) for i in range(rot // 2)], ref.rope_axes(rot, sections, inter), adjacent)
    return rope, v, t, args


def _fwd(t):
    return t["pos"], t["q"], t["k"], t["q_weight"], t["k_weight"]


def _cut(v, side, sl):
    return v[side][:, :, sl]


@pytest.mark.parametrize("fp32,w_fp32", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("d,rot,sections,inter", [(128, 128, (16, 24, 24), False), (128, 64, (10, 11, 11), True),
                                                  (64, 64, (12, 10, 10), True), (64, 16, (0, 4, 4), False)])
@pytest.mark.parametrize("L,B,n,Hq,Hkv", [(3, 2, 1, 14, 2), (1, 3, 67, 5, 5), (2, 1, 33, 28, 4), (1, 1, 5000, 2, 1)])
def test_forward_and_gradient(dev, fp32, w_fp32, adjacent, d, rot, sections, inter, L, B, n, Hq, Hkv):
    for inverse, scale, eps in ((False, 1.0, 1e-6), (True, 0.75, 0.3)):
        rope, v, t, args = _problem(d + rot + n, dev, L, B, n, Hq, Hkv, d, rot, sections, inter, adjacent, fp32, w_fp32,
                                    scale, eps)
        oq, ok = rope.apply(*_fwd(t), q_out=torch.empty_like(t["q"]), k_out=torch.empty_like(t["k"]), inverse=inverse)
        gq, gk, wq, wk = rope.grad(*_fwd(t), t["q_dout"], t["k_dout"], inverse=inverse)
        torch.cuda.synchronize()
        toks = B * n
        groups = max(1, min(-(-toks // 4), 1024 // L))
        for side, H, out, dx, dw in (("q", Hq, oq, gq, wq), ("k", Hkv, ok, gk, wk)):
            assert np.array_equal(_np(t[side]), v[side])  # an input is left alone
            m = min(n, 40)  # a long case: its first and last tokens; its sums over all of them
            for sl in (slice(0, m), slice(n - m, n)) if n > 40 else (slice(0, n),):
                nr = Norm(_cut(v, side, sl), v[side + "_weight"], v["pos"][:, :, sl], *args, inverse, scale, eps)
                assert (np.abs(_np(out)[:, :, sl] - nr.forward()) <= nr.forward_tol(fp32)).all(), side
                want, _, tol, _ = nr.grad(_cut(v, side + "_dout", sl))
                assert (np.abs(_np(dx)[:, :, sl] - want) <= tol + (0 if fp32 else np.abs(want) * 2.0 ** -8)).all(), side
            nr = Norm(v[side], v[side + "_weight"], v["pos"], *args, inverse, scale, eps)
            _, want, _, size = nr.grad(v[side + "_dout"])
            roundings = -(-toks // (4 * groups)) * H + 40
            assert dw.dtype is torch.float32
            assert (np.abs(_np(dw) - want) <= size * (2.0 ** -18 + roundings * 2.0 ** -24)).all(), side
        # the same bits in place, each side alone, and again
        a, b = t["q"].clone(), t["k"].clone()
        rope.apply(t["pos"], a, b, t["q_weight"], t["k_weight"], inverse=inverse)
        assert torch.equal(a, oq) and torch.equal(b, ok)
        a, b = t["q"].clone(), t["k"].clone()
        assert rope.apply(t["pos"], q=a, q_weight=t["q_weight"], inverse=inverse)[1] is None
        rope.apply(t["pos"], k=b, k_weight=t["k_weight"], inverse=inverse)
        assert torch.equal(a, oq) and torch.equal(b, ok)
        a, b = t["q_dout"].clone(), t["k"].clone()  # over the outputs' gradients, over the rows
        _, _, w1, w2 = rope.grad(t["pos"], t["q"], b, t["q_weight"], t["k_weight"], a, t["k_dout"], q_din=a, k_din=b,
                                 inverse=inverse)
        assert torch.equal(a, gq) and torch.equal(b, gk) and torch.equal(w1, wq) and torch.equal(w2, wk)
        a, none, w1, none2 = rope.grad(t["pos"], q=t["q"], q_weight=t["q_weight"], q_dout=t["q_dout"], inverse=inverse)
        assert torch.equal(a, gq) and torch.equal(w1, wq) and none is None and none2 is None
        none, b, none2, w2 = rope.grad(t["pos"], k=t["k"], k_weight=t["k_weight"], k_dout=t["k_dout"], inverse=inverse)
        assert torch.equal(b, gk) and torch.equal(w2, wk) and none is None and none2 is None


@pytest.mark.parametrize("fp32", [False, True])
def test_counts_and_strides(dev, fp32):
    """Padded batches: rows past a sequence's tokens stay as they are and count for nothing, NaN
    among them; head-major tensors; inputs whose rows repeat."""
    L, B, n, Hq, Hkv, d = 2, 4, 9, 6, 3, 64
    count = [9, 0, 4, 1]
    rope, v, t, args = _problem(5, dev, L, B, n, Hq, Hkv, d, 64, (12, 10, 10), False, False, fp32, True)
    cnt = torch.tensor(count, dtype=torch.int32, device=dev)
    for side in "qk":
        for b in range(B):
            t[side][:, b, count[b]:] = float("nan")
            t[side + "_dout"][:, b, count[b]:] = float("nan")
    hm = lambda x: x.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)  # noqa: E731
    marks = {s: hm(torch.full_like(t[s], 7.0)) for s in "qk"}
    rope.apply(t["pos"], hm(t["q"]), hm(t["k"]), t["q_weight"], t["k_weight"], q_out=marks["q"], k_out=marks["k"], count=cnt)
    dins = {s: hm(torch.full_like(t[s], 5.0)) for s in "qk"}
    _, _, wq, wk = rope.grad(*_fwd(t), hm(t["q_dout"]), hm(t["k_dout"]), q_din=dins["q"], k_din=dins["k"], count=cnt)
    new = rope.grad(*_fwd(t), t["q_dout"], t["k_dout"], count=cnt)
    for i, (side, H, dw) in enumerate((("q", Hq, wq), ("k", Hkv, wk))):
        nr = Norm(v[side], v[side + "_weight"], v["pos"], *args, count=count)
        dx, want, tol, size = nr.grad(v[side + "_dout"])
        out, din, live = _np(marks[side]), _np(dins[side]), nr.live
        assert (out[~live] == 7).all() and (din[~live] == 5).all()
        assert (np.abs(out - nr.forward()) <= nr.forward_tol(fp32))[live].all()
        assert (np.abs(din - dx) <= tol + (0 if fp32 else np.abs(dx) * 2.0 ** -8))[live].all()
        assert (np.abs(_np(dw) - want) <= size * (2.0 ** -18 + (H + 40) * 2.0 ** -24)).all()
        assert (_np(new[i])[~live] == 0).all() and (_np(new[i])[live] == din[live]).all()
    # one head's gradient for all of them, one layer's rows for both
    one = t["q_dout"][:, :, :, :1].expand(-1, -1, -1, Hq, -1)
    row = t["q"][:1].expand(L, -1, -1, -1, -1)
    a = rope.grad(t["pos"], q=row, q_weight=t["q_weight"], q_dout=one, count=cnt)
    b = rope.grad(t["pos"], q=row.contiguous(), q_weight=t["q_weight"], q_dout=one.contiguous(), count=cnt)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


def test_gradient_against_differences(dev):
    """The gradient of sum(dout out) is the slope of the 64-bit forward pass."""
    L, B, n, Hq, Hkv, d = 1, 1, 5, 2, 1, 64
    rope, v, t, args = _problem(9, dev, L, B, n, Hq, Hkv, d, 32, (6, 5, 5), False, True, True, True)
    dx, _, dw, _ = rope.grad(t["pos"], q=t["q"], q_weight=t["q_weight"], q_dout=t["q_dout"])
    rng = np.random.default_rng(1)
    loss = lambda x, w: (Norm(x, w, v["pos"], *args).forward() * v["q_dout"].astype(np.float64)).sum()  # noqa: E731
    x, w, h = v["q"].astype(np.float64), v["q_weight"].astype(np.float64), 1e-5
    _, _, tol, size = Norm(x, w, v["pos"], *args).grad(v["q_dout"])
    for _ in range(40):
        at = tuple(int(rng.integers(0, s)) for s in x.shape)
        e = np.zeros_like(x)
        e[at] = h
        slope = (loss(x + e, w) - loss(x - e, w)) / (2 * h)
        assert abs(slope - float(dx[at])) <= tol[at] + 1e-8  # (differences: h^2 and 2^-52 / h of the loss)
        c = int(rng.integers(0, d))
        e = np.zeros_like(w)
        e[0, c] = h
        slope = (loss(x, w + e) - loss(x, w - e)) / (2 * h)
        assert abs(slope - float(dw[0, c])) <= size[0, c] * (2.0 ** -18 + 60 * 2.0 ** -24) + 1e-8


def test_rows_at_the_border(dev):
    """Rows of zeros, tiny and large rows, infinities and NaN, each a row's own affair."""
    d = 128
    rope, v, t, args = _problem(3, dev, 1, 1, 8, 2, 1, d, 128, (16, 24, 24), False, False, True, True, eps=1e-6)
    clean = rope.apply(t["pos"], q=t["q"].clone(), q_weight=t["q_weight"])[0]
    gclean = rope.grad(t["pos"], q=t["q"], q_weight=t["q_weight"], q_dout=t["q_dout"])[0]
    x = v["q"].copy()
    x[0, 0, 0] = 0
    x[0, 0, 1] *= 1e-30
    x[0, 0, 2] *= 1e15
    x[0, 0, 3, 0, 5] = np.inf
    x[0, 0, 4, 1, 7] = np.nan
    q = _put(x, dev, True)
    out = rope.apply(t["pos"], q=q, q_weight=t["q_weight"], q_out=torch.empty_like(q))[0]
    g = rope.grad(t["pos"], q=q, q_weight=t["q_weight"], q_dout=t["q_dout"])[0]
    nr = Norm(x[:, :, :3], v["q_weight"], v["pos"][:, :, :3], *args)
    assert (np.abs(_np(out)[:, :, :3] - nr.forward()) <= nr.forward_tol(True)).all()
    dx, _, tol, _ = nr.grad(v["q_dout"][:, :, :3])
    assert (np.abs(_np(g)[:, :, :3] - dx) <= tol).all()
    assert torch.isnan(out[0, 0, 3, 0]).any() and torch.isnan(out[0, 0, 4, 1]).all()
    assert torch.equal(out[0, 0, 3, 1], clean[0, 0, 3, 1]) and torch.equal(out[0, 0, 4, 0], clean[0, 0, 4, 0])
    assert torch.equal(out[0, 0, 5:], clean[0, 0, 5:]) and torch.equal(g[0, 0, 5:], gclean[0, 0, 5:])


def test_nothing_to_do(dev):
    from paper_2608_24063_amd.tensors import NormRope, Rope
    rope = NormRope(Rope(64))
    w = torch.ones((2, 64), device=dev)
    for B, n in ((0, 3), (2, 0)):
        q = torch.zeros((2, B, n, 4, 64), device=dev)
        pos = torch.zeros((3, B, n), dtype=torch.int32, device=dev)
        assert rope.apply(pos, q=q, q_weight=w)[0] is q
        dx, _, dw, _ = rope.grad(pos, q=q, q_weight=w, q_dout=q)
        assert dx.shape == q.shape and dw.shape == (2, 64) and not dw.any()


def test_streams_and_graphs(dev):
    """Both directions on another stream, and captured and replayed with new inputs between."""
    rope, v, t, args = _problem(21, dev, 2, 2, 50, 8, 2, 64, 64, (12, 10, 10), False, False, False, False)
    out = {s: torch.empty_like(t[s]) for s in "qk"}
    din = {s: torch.empty_like(t[s]) for s in "qk"}

    def both():
        rope.apply(*_fwd(t), q_out=out["q"], k_out=out["k"])
        return rope.grad(*_fwd(t), t["q_dout"], t["k_dout"], q_din=din["q"], k_din=din["k"])[2:]
    both()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        wq, wk = both()
    for seed in range(3):
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        for name in ("q", "k", "q_dout", "k_dout"):
            t[name].copy_(torch.randn(t[name].shape, generator=g, device=dev))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out["q"], out["k"], din["q"], din["k"], wq, wk)]
        with torch.cuda.stream(s):
            eager = both()
        s.synchronize()
        for a, b in zip(got, (out["q"], out["k"], din["q"], din["k"], *eager)):
            assert torch.equal(a, b)


def test_autograd(dev):
    """The pair as a program wraps it, against autograd of the plain form in 64 bits; what
    requires grad is refused outside of such a function."""
    rope, v, t, args = _problem(31, dev, 1, 2, 9, 4, 2, 64, 64, (8, 12, 12), False, False, True, True)

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            ctx.save_for_backward(x, w)
            return rope.apply(t["pos"], q=x, q_weight=w, q_out=torch.empty_like(x))[0]

        @staticmethod
        def backward(ctx, g):
            x, w = ctx.saved_tensors
            dx, _, dw, _ = rope.grad(t["pos"], q=x, q_weight=w, q_dout=g.contiguous())
            return dx, dw

    x, w = t["q"].clone().requires_grad_(), t["q_weight"].clone().requires_grad_()
    (Turn.apply(x, w) * t["q_dout"]).sum().backward()
    freq = torch.tensor(args[1], dtype=torch.float64)
    a = torch.from_numpy(v["pos"])[torch.tensor(args[2])].permute(1, 2, 0).double() * freq
    c, s = torch.cos(a)[None, :, :, None], torch.sin(a)[None, :, :, None]
    X, W = (torch.from_numpy(v[k]).double().requires_grad_() for k in ("q", "q_weight"))
    y = X * torch.rsqrt((X * X).mean(-1, keepdim=True) + float(np.float32(1e-6))) * W[:, None, None, None]
    y = torch.cat((y[..., :32] * c - y[..., 32:] * s, y[..., 32:] * c + y[..., :32] * s), dim=-1)
    (y * torch.from_numpy(v["q_dout"]).double()).sum().backward()
    _, _, tol, size = Norm(v["q"], v["q_weight"], v["pos"], *args).grad(v["q_dout"])
    assert (np.abs(_np(x.grad) - X.grad.numpy()) <= tol).all()
    assert (np.abs(_np(w.grad) - W.grad.numpy()) <= size * (2.0 ** -18 + 60 * 2.0 ** -24)).all()
    for kw in (dict(q=x, q_weight=t["q_weight"]), dict(q=t["q"], q_weight=w)):
        with pytest.raises(ValueError, match="requires grad"):
            rope.apply(t["pos"], **kw)
        with pytest.raises(ValueError, match="requires grad"):
            rope.grad(t["pos"], **kw, q_dout=t["q_dout"])
    with torch.no_grad():
        rope.apply(t["pos"], q=x, q_weight=w, q_out=torch.empty_like(x))


def test_refusals(dev):
    rope, v, t, _ = _problem(41, dev, 1, 2, 3, 4, 2, 64, 64, (8, 12, 12), False, False, False, False)
    q, k, qw, kw, pos = t["q"], t["k"], t["q_weight"], t["k_weight"], t["pos"]
    bad = [lambda: rope.apply(pos), lambda: rope.apply(pos, q=q), lambda: rope.apply(pos, q_weight=qw),
           lambda: rope.apply(pos, q=q, q_weight=qw.float()[:, :32]), lambda: rope.apply(pos, q, k, qw, kw.float()),
           lambda: rope.apply(pos, q=q.half(), q_weight=qw), lambda: rope.apply(pos, q, k[:, :1], qw, kw),
           lambda: rope.apply(pos.long(), q=q, q_weight=qw), lambda: rope.apply(pos[:, :1], q=q, q_weight=qw),
           lambda: rope.apply(pos, q=q, q_weight=qw.cpu()), lambda: rope.apply(pos, q=q.cpu(), q_weight=qw.cpu()),
           lambda: rope.apply(pos, q=q, q_weight=qw, q_out=q.float()),
           lambda: rope.apply(pos, q=q.transpose(3, 4), q_weight=qw),
           lambda: rope.grad(pos, q=q, q_weight=qw), lambda: rope.grad(pos, q=q, q_weight=qw, k_dout=k),
           lambda: rope.grad(pos, q=q, q_weight=qw, q_dout=q.float()),
           lambda: rope.grad(pos, q=q, q_weight=qw, q_dout=q[:, :, :2])]
    for f in bad:
        with pytest.raises(ValueError):
            f()


def test_rows_past_32_bits(dev):
    """More than 2^31 values of queries: the first and last tokens have the bits of a call of their own."""
    from paper_2608_24063_amd.tensors import NormRope, Rope
    n, Hq, Hkv, d, m = 140_000, 128, 8, 128, 9
    rope = NormRope(Rope(d, theta=1e4))
    g = torch.Generator(device=dev)
    g.manual_seed(3)
    rows = lambda H: torch.randn((1, 1, n, H, d), generator=g, device=dev, dtype=torch.bfloat16)  # noqa: E731
    q, k, dq, dk = rows(Hq), rows(Hkv), rows(Hq), rows(Hkv)
    w = torch.randn((2, 1, d), generator=g, device=dev)
    pos = torch.arange(n, dtype=torch.int32, device=dev).expand(3, 1, n).contiguous()
    dq[:, :, m:-m] = 0  # (the weights' gradients are those tokens' alone)
    dk[:, :, m:-m] = 0
    oq, ok = rope.apply(pos, q, k, w[0], w[1], q_out=torch.empty_like(q), k_out=torch.empty_like(k))
    gq, gk, wq, wk = rope.grad(pos, q, k, w[0], w[1], dq, dk)
    sums = [0, 0]
    for sl in (slice(0, m), slice(n - m, n)):
        cut = lambda x: x[:, :, sl].clone()  # noqa: E731  (turned in place)
        p = pos[:, :, sl].contiguous()
        a, b = rope.apply(p, cut(q), cut(k), w[0], w[1])
        assert torch.equal(a, oq[:, :, sl]) and torch.equal(b, ok[:, :, sl])
        a, b, wa, wb = rope.grad(p, cut(q), cut(k), w[0], w[1], cut(dq), cut(dk))
        assert torch.equal(a, gq[:, :, sl]) and torch.equal(b, gk[:, :, sl])
        sums = [sums[0] + wa.double(), sums[1] + wb.double()]
    assert not gq[:, :, m:-m].any() and not gk[:, :, m:-m].any()
    # Two sums of the same terms in other orders: at most 2 m H + 1024 roundings of the sum of the
    # terms' magnitudes, which are normal values' products: well below 8 sqrt 2 on average.
    for got, want, H in ((wq, sums[0], Hq), (wk, sums[1], Hkv)):
        terms = 2 * m * H
        assert (got.double() - want).abs().max() <= 2 * (terms + 1024) * 2.0 ** -24 * terms * 8 * 2 ** 0.5
