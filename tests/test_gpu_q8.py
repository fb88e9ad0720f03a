"""GPU parity of the 8-bit cache (viscache_q8_append, viscache_q8_read) and of
attention over it (viscache_q8_attend) against the 64-bit forms of
tests/q8_ref.py.  Codes, scales and tails are whole results of exact or
correctly rounded steps and must agree bit for bit; attention is held to the
tolerance derived in q8_ref.tolerance."""
import ctypes

import numpy as np
import pytest

from tests import q8_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
FMTS = ("int8", "e4m3")


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2608_24063_amd as vc
    vc.lib()
    return torch.device("cuda:0")


def _values(rng, shape):
    """bf16 rows (as fp32): a few loud channels and tokens, as a model leaves them."""
    x = rng.standard_normal(shape) * np.exp(0.5 * rng.standard_normal(shape[-1:]))
    x *= np.where(rng.random(shape[:-1]) < 0.05, 6.0, 1.0)[..., None]
    return ref.bf16(x)


def _t(x, dev, typ=torch.bfloat16):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dev).to(typ)


def _foul(c):
    """Whatever a pool may hold where nothing was written: NaN codes, scales and tails."""
    for side in "kv":
        getattr(c, side + "_codes").view(torch.uint8).fill_(0x7F)
        getattr(c, side + "_scale").fill_(float("nan"))
        getattr(c, side + "_tail").fill_(float("nan"))


def _make(L, B, Hq, Hkv, d, caps, dev, fmt, foul=True):
    from paper_2608_24063_amd.tensors import Q8Cache
    c = Q8Cache(L, B, Hq, Hkv, d, caps, dev, format=fmt)
    if foul:
        _foul(c)
    return c


def _host(c):
    """The cache's buffers on the host; codes as the values they stand for."""
    torch.cuda.synchronize()
    h = {"len": c.len.cpu().numpy(), "first": c.row_off.cpu().numpy() // 64}
    for side in "kv":
        h[side + "_codes"] = getattr(c, side + "_codes").cpu().float().numpy()
        h[side + "_raw"] = getattr(c, side + "_codes").view(torch.uint8).cpu().numpy()
        h[side + "_scale"] = getattr(c, side + "_scale").cpu().numpy()
        h[side + "_tail"] = getattr(c, side + "_tail").cpu().float().numpy()
    return h


def _check_cache(c, rows, fmt):
    """The cache against the rows appended to each unit: [(k, v)] per unit.  What
    no row reached still holds what _foul left."""
    h = _host(c)
    used = np.zeros(len(h["k_scale"]), dtype=bool)
    for u, kv in enumerate(rows):
        n = len(kv[0])
        assert h["len"][u] == n, f"unit {u}"
        b0 = h["first"][u]
        for side, x in zip("kv", kv):
            for j in range(n // 64):
                code, s = ref.quantise(x[64 * j:64 * j + 64], fmt)
                got = h[side + "_codes"][b0 + j]
                got = got if side == "k" else got.T
                assert np.array_equal(got, code), f"unit {u} block {j} {side}: codes"
                assert h[side + "_scale"][b0 + j] == s, f"unit {u} block {j} {side}: scale"
                used[b0 + j] = True
            r = n % 64
            tail = h[side + "_tail"][u]
            assert np.array_equal(tail[:r], x[n - r:]), f"unit {u} {side}: tail"
            if r:
                assert h[side + "_scale"][b0 + n // 64] == ref.open_scale(x[n - r:]), f"unit {u} {side}: open scale"
                used[b0 + n // 64] = True
    for side in "kv":
        assert np.isnan(h[side + "_scale"][~used]).all(), "scales of unused blocks"
        assert (h[side + "_raw"][~used] == 0x7F).all(), "codes of unused blocks"
    return h


# ---- writing -------------------------------------------------------------------

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("calls", [[1] * 3, [64], [63, 1], [1, 63], [63, 2], [64, 64], [65, 1, 62], [130, 3, 200],
                                   [40, 64, 64], [5, 300], [0, 7, 0]], ids=str)
def test_append_in_steps(dev, fmt, d, calls):
    """However the rows come, the cache is the one their order gives."""
    rng = np.random.default_rng(sum(calls) + d)
    L, B, Hkv, n = 2, 2, 2, sum(calls)
    c = _make(L, B, 4, Hkv, d, [n + 3] * (L * B * Hkv), dev, fmt)
    k, v = _values(rng, (L, B, n, Hkv, d)), _values(rng, (L, B, n, Hkv, d))
    at = 0
    for m in calls:
        c.append(_t(k[:, :, at:at + m], dev), _t(v[:, :, at:at + m], dev))
        at += m
    rows = [(k[l, b, :, g], v[l, b, :, g]) for l in range(L) for b in range(B) for g in range(Hkv)]
    _check_cache(c, rows, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_append_counts_and_room(dev, fmt):
    """Counts per layer and sequence (clamped to 0 .. n), units with too little
    room or none, a length beyond the capacity, and the rows behind a
    tail's open rows, which stay as they were."""
    rng = np.random.default_rng(3)
    L, B, Hkv, d, n = 2, 3, 2, 64, 150
    caps = [200, 10, 64, 65, 0, 149, 150, 128, 63, 1, 200, 200]
    c = _make(L, B, 2, Hkv, d, caps, dev, fmt)
    k, v = _values(rng, (L, B, Hkv, n, d)), _values(rng, (L, B, Hkv, n, d))
    count = [150, 90, -5, 1000, 64, 0]
    c.append(_t(k, dev), _t(v, dev), count=torch.tensor(count, dtype=torch.int32, device=dev), head_major=True)
    rows = []
    for u, cap in enumerate(caps):
        l, b, g = u // (B * Hkv), u // Hkv % B, u % Hkv
        m = min(max(min(count[l * B + b], n), 0), cap)
        rows.append((k[l, b, g, :m], v[l, b, g, :m]))
    h = _check_cache(c, rows, fmt)
    for u, (x, _) in enumerate(rows):
        assert np.isnan(h["k_tail"][u][len(x) % 64:]).all() and np.isnan(h["v_tail"][u][len(x) % 64:]).all()
    # full units take nothing more
    before = _host(c)
    full = torch.tensor([len(r[0]) >= cap for r, cap in zip(rows, caps)])
    c.append(_t(k[:, :, :, :1], dev), _t(v[:, :, :, :1], dev), head_major=True)
    assert torch.equal(c.len.cpu()[full], torch.from_numpy(before["len"])[full])
    # a length past the capacity is left alone
    c.len.fill_(500)
    c.append(_t(k, dev), _t(v, dev), head_major=True)
    assert (c.len.cpu() == 500).all()


def test_append_strides_and_offsets(dev):
    """Keys and values inside one wider projection, heads shared by a stride of
    0, and packed rows through unit_off."""
    import paper_2608_24063_amd as vc
    rng = np.random.default_rng(4)
    L, B, Hkv, d, n = 1, 2, 3, 64, 77
    wide = _values(rng, (L, B, n, 4 + 2 * Hkv, d))
    w = _t(wide, dev)
    c = _make(L, B, 6, Hkv, d, [n] * 6, dev, "int8")
    c.append(w[:, :, :, 4:4 + Hkv], w[:, :, :, 4 + Hkv:])
    _check_cache(c, [(wide[0, b, :, 4 + g], wide[0, b, :, 4 + Hkv + g]) for b in range(B) for g in range(Hkv)], "int8")
    c = _make(L, B, 6, Hkv, d, [n] * 6, dev, "e4m3")
    one = w[:, :, :, :1].expand(L, B, n, Hkv, d)
    c.append(one, one)
    _check_cache(c, [(wide[0, b, :, 0], wide[0, b, :, 0]) for b in range(B) for g in range(Hkv)], "e4m3")
    # packed: unit u's rows start at off[u]
    lens = [5, 64, 70, 0, 1, 63]
    off = np.concatenate(([0], np.cumsum(lens)[:-1]))
    pk, pv = _values(rng, (sum(lens), d)), _values(rng, (sum(lens), d))
    shape = vc.vc_decode_shape(6, 1, 2, 1, d)  # counts are per sequence: a unit a sequence
    c = _make(1, 6, 2, 1, d, [80] * 6, dev, "int8")
    tk, tv = _t(pk, dev), _t(pv, dev)
    cnt = torch.tensor(lens, dtype=torch.int32, device=dev)
    o = torch.from_numpy(off * d).to(dev)
    vc.viscache_q8_append(shape, c.c, vc.vc_rows(tk.data_ptr(), -1, -1, d, -1), vc.vc_rows(tv.data_ptr(), 0, 0, d, 0), 70,
                          cnt.data_ptr(), o.data_ptr(), torch.cuda.current_stream().cuda_stream)
    _check_cache(c, [(pk[o0:o0 + m], pv[o0:o0 + m]) for o0, m in zip(off, lens)], "int8")


def _special_blocks(d):
    b = []
    b.append(np.zeros((64, d)))
    z = np.zeros((64, d))
    z[::3] = -0.0
    z[5, 7] = 2.0 ** -126
    b.append(z)                                                    # a normal below the smallest scale
    b.append(np.full((64, d), -1.5))                               # one magnitude
    b.append(np.where(np.arange(64 * d) % 5 == 0, 3e38, -1e38).reshape(64, d))  # past the largest scale
    b.append((np.arange(64 * d) % 255 - 127).reshape(64, d) / 2.0)  # int8 ties at every half
    t = (np.arange(64 * d) % 449).reshape(64, d) * 1.0
    t[0, 0] = 448.0
    b.append(t)                                                    # e4m3 midpoints at every spacing
    b.append(2.0 ** -(np.arange(64 * d) % 30).reshape(64, d) * 1.0)  # down through the subnormals
    b.append(((np.arange(64 * d) % 251) * 2.0 ** -70).reshape(64, d))
    return np.stack([ref.bf16(x) for x in b])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d", [64, 128])
def test_quantiser_at_its_edges(dev, fmt, d):
    """Zeros of both signs, one magnitude, magnitudes past both ends of the
    scales, ties: bit for bit, also where all pairs (x, largest) of a binade meet."""
    x = _special_blocks(d)
    grid = np.empty((128, 64, d), dtype=np.float32)
    vals = (np.arange(64 * d) % 512 + 1).reshape(64, d)
    for a in range(128):  # every mantissa as the largest value
        top = (128 + a) * 4.0
        grid[a] = ref.bf16(np.minimum(vals, top))
        grid[a, 0, 0] = top
        grid[a, :, 1::2] *= -2.0 ** -(a % 9)
    x = np.concatenate((x, grid)).reshape(-1, d)
    c = _make(1, 1, 1, 1, d, [len(x)], dev, fmt)
    t = _t(x, dev)[None, None, :, None]
    c.append(t, -t)
    _check_cache(c, [(x, -x)], fmt)


# ---- reading back ----------------------------------------------------------------

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_read(dev, fmt, fp32, d):
    """Rows below the length (and the row bound) equal code * scale, rounded once;
    the others stay as they were."""
    rng = np.random.default_rng(5)
    L, B, Hkv = 1, 7, 2
    lens = [0, 1, 63, 64, 65, 129, 200]
    typ = torch.float32 if fp32 else torch.bfloat16
    k, v = _values(rng, (L, B, Hkv, 200, d)), _values(rng, (L, B, Hkv, 200, d))
    c = _make(L, B, 2, Hkv, d, [200] * (B * Hkv), dev, fmt)
    c.append(_t(k, dev), _t(v, dev), count=torch.tensor(lens, dtype=torch.int32, device=dev), head_major=True)
    for hm, most in ((True, None), (False, None), (True, 100)):
        shape = (L, B, Hkv, 203, d) if hm else (L, B, 203, Hkv, d)
        ko = torch.full(shape, 7.0, dtype=typ, device=dev)
        vo = torch.full(shape, 7.0, dtype=typ, device=dev)
        c.read(ko, vo, max_rows=most, head_major=hm)
        for out, x in ((ko, k), (vo, v)):
            got = out.float().cpu().numpy() if hm else out.float().transpose(2, 3).cpu().numpy()
            for b in range(B):
                for g in range(Hkv):
                    n = lens[b] if most is None else min(lens[b], most)
                    want = ref.read_back(x[0, b, g, :lens[b]], fmt).astype(np.float32)[:n]
                    want = want if fp32 else ref.bf16(want)
                    assert np.array_equal(got[0, b, g, :n], want), (b, g)
                    assert (got[0, b, g, n:] == 7.0).all(), (b, g)


def test_read_into_decode_pools(dev):
    """A parked cache goes back into the pools of a DecodeCache by unit_off."""
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import DecodeCache
    rng = np.random.default_rng(6)
    L, B, Hkv, d = 2, 1, 2, 128
    n = 100
    k, v = _values(rng, (L, B, n, Hkv, d)), _values(rng, (L, B, n, Hkv, d))
    c = _make(L, B, 4, Hkv, d, [n] * 4, dev, "int8")
    c.append(_t(k, dev), _t(v, dev))
    dc = DecodeCache(L, B, 4, Hkv, d, [n + 1] * 4, dev)
    off = dc.row_off * d
    vc.viscache_q8_read(c.shape, c.c, n, vc.vc_rows(dc.k_pool.data_ptr(), 0, 0, d, 0),
                        vc.vc_rows(dc.v_pool.data_ptr(), 0, 0, d, 0), off.data_ptr(), 0,
                        torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for u in range(4):
        l, g = u // 2, u % 2
        r0 = dc.offs_host[u]
        assert np.array_equal(dc.k_pool[r0:r0 + n].float().cpu().numpy(), ref.bf16(ref.read_back(k[l, 0, :, g], "int8")))
        assert np.array_equal(dc.v_pool[r0:r0 + n].float().cpu().numpy(), ref.bf16(ref.read_back(v[l, 0, :, g], "int8")))


# ---- attention ---------------------------------------------------------------------

def _filled(rng, dev, L, B, Hq, Hkv, d, lens, fmt, extra=0, gain=1.0):
    """A cache of these lengths per unit (through append, a length at a time) and its
    rows as they read back."""
    units = L * B * Hkv
    c = _make(L, B, Hq, Hkv, d, [n + extra for n in lens], dev, fmt)
    K = [_values(rng, (n, d)) * np.float32(gain) for n in lens]
    V = [_values(rng, (n, d)) for n in lens]
    import paper_2608_24063_amd as vc
    off = np.concatenate(([0], np.cumsum(lens)[:-1])).astype(np.int64) * d
    if max(lens):
        tk, tv = _t(np.concatenate(K), dev), _t(np.concatenate(V), dev)
        one = vc.vc_decode_shape(units, 1, 1, 1, d)  # a unit a sequence: counts of their own
        cnt = torch.tensor(lens, dtype=torch.int32, device=dev)
        o = torch.from_numpy(off).to(dev)
        vc.viscache_q8_append(one, c.c, vc.vc_rows(tk.data_ptr(), 0, 0, d, 0), vc.vc_rows(tv.data_ptr(), 0, 0, d, 0),
                              max(lens), cnt.data_ptr(), o.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
    return c, [ref.read_back(x, fmt) for x in K], [ref.read_back(x, fmt) for x in V]


def _check_attend(out, q, K, V, lens, L, B, Hq, Hkv, scale, counts, causal, max_rows=1 << 30, left=7.0, sample=None):
    """out [L, B, n, Hq, d] (numpy) against the plain form, row by row; `sample`: only
    these query indices."""
    n, d = out.shape[2], out.shape[4]
    G = Hq // Hkv
    fp32 = out.dtype == np.float32 and getattr(out, "_fp32", True)
    worst = 0.0
    for u, ln in enumerate(lens):
        l, b, g = u // (B * Hkv), u // Hkv % B, u % Hkv
        c = min(max(counts[b], 0), n)
        vmax = float(np.abs(V[u]).max()) if ln else 0.0
        for i in range(n) if sample is None else sample:
            for h in range(g * G, (g + 1) * G):
                got = out[l, b, i, h]
                if i >= c:
                    assert (got == left).all(), f"row {(l, b, i, h)} was written"
                    continue
                end = min(ln - c + i + 1 if causal else ln, max_rows)
                want, reach = ref.attend(q[l, b, i, h], K[u], V[u], scale, end)
                tol = ref.tolerance(max(end, 0), d, reach, vmax, fp32)
                err = float(np.abs(got - want).max())
                assert err <= tol, f"row {(l, b, i, h)}, {end} rows seen: {err} > {tol}"
                worst = max(worst, err / tol)
    return worst


class _Out(np.ndarray):
    pass


def _run_attend(c, q, dev, fp32, scale, counts=None, causal=True, max_rows=None):
    out = torch.full(q.shape, 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device=dev)
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=dev)
    c.attend(_t(q, dev), out, scale, count=cnt, causal=causal, max_rows=max_rows)
    torch.cuda.synchronize()
    a = out.float().cpu().numpy().view(_Out)
    a._fp32 = fp32
    return a


LENS = [0, 1, 2, 63, 64, 65, 127, 128, 300, 511, 512, 700]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d,G", [(64, 4), (128, 7), (128, 1), (64, 16)])
@pytest.mark.parametrize("fp32", [True, False])
def test_decode(dev, fmt, d, G, fp32):
    """One token over caches of every awkward length, in several pieces a unit or one."""
    rng = np.random.default_rng(d + G)
    L, B, Hkv = 2, 3, 2
    c, K, V = _filled(rng, dev, L, B, G * Hkv, Hkv, d, LENS, fmt)
    q = ref.bf16(rng.standard_normal((L, B, 1, G * Hkv, d)))
    out = _run_attend(c, q, dev, fp32, d ** -0.5)
    _check_attend(out, q, K, V, LENS, L, B, G * Hkv, Hkv, d ** -0.5, [1] * B, True)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d,G,n", [(64, 4, 4), (128, 7, 2), (128, 1, 16), (128, 7, 3), (64, 4, 5), (64, 4, 33),
                                   (128, 8, 17), (128, 7, 40), (64, 16, 20)])
@pytest.mark.parametrize("causal", [True, False])
def test_several_queries(dev, fmt, d, G, n, causal):
    """Short drafts and prompts, ragged counts (none, too many), queries that see
    nothing, rows behind a sequence's queries left alone."""
    rng = np.random.default_rng(d * 100 + G * 10 + n)
    L, B, Hkv = 1, 6, 2
    counts = [n, 0, 1, n + 5, max(1, n - 1), -3]
    lens = LENS
    c, K, V = _filled(rng, dev, L, B, G * Hkv, Hkv, d, lens, fmt)
    q = ref.bf16(rng.standard_normal((L, B, n, G * Hkv, d)))
    for fp32 in (True, False):
        out = _run_attend(c, q, dev, fp32, d ** -0.5, counts, causal)
        _check_attend(out, q, K, V, lens, L, B, G * Hkv, Hkv, d ** -0.5, counts, causal,
                      sample=sorted({0, 1, n // 2, n - 1}))


@pytest.mark.parametrize("n", [1, 4, 150])
@pytest.mark.parametrize("most", [0, 1, 64, 100, 256])
def test_row_bound(dev, n, most):
    """Rows past max_rows are not attended, whatever the lengths."""
    rng = np.random.default_rng(n + most)
    lens = [300, 90, 64, 200]
    c, K, V = _filled(rng, dev, 1, 2, 8, 2, 64, lens, "int8")
    q = ref.bf16(rng.standard_normal((1, 2, n, 8, 64)))
    for causal in (True, False):
        out = _run_attend(c, q, dev, True, 0.125, None, causal, max_rows=most)
        _check_attend(out, q, K, V, lens, 1, 2, 8, 2, 0.125, [n] * 2, causal, max_rows=most,
                      sample=sorted({0, n // 2, n - 1}))


@pytest.mark.parametrize("n", [1, 9])
def test_long_units_in_many_pieces(dev, n):
    """Few units, many rows: the pieces' join, and again on the same workspace."""
    rng = np.random.default_rng(n)
    lens = [20011, 13, 6400, 9999]
    c, K, V = _filled(rng, dev, 1, 2, 14, 2, 128, lens, "e4m3")
    q = ref.bf16(rng.standard_normal((1, 2, n, 14, 128)))
    first = _run_attend(c, q, dev, True, 0.1)
    _check_attend(first, q, K, V, lens, 1, 2, 14, 2, 0.1, [n] * 2, True, sample=[0, n - 1])
    for _ in range(3):
        assert np.array_equal(first, _run_attend(c, q, dev, True, 0.1))


@pytest.mark.parametrize("n", [1, 20])
@pytest.mark.parametrize("fp32", [True, False])
def test_values_of_unlike_blocks(dev, n, fp32):
    """Blocks whose scales differ by many powers of two, an all-zero block, large
    logits: the block that carries the weight decides, however small its values."""
    rng = np.random.default_rng(11)
    d, lens = 64, [64 * 9 + 20]
    gains = [1.0, 1e-4, 0.0, 1e4, 1.0, 2e-9, 3.0, 0.0, 1.0, 1e-3]
    k = _values(rng, (1, 1, lens[0], 1, d))
    v = _values(rng, (1, 1, lens[0], 1, d))
    for j, gv in enumerate(gains):
        v[0, 0, 64 * j:64 * j + 64] = ref.bf16(v[0, 0, 64 * j:64 * j + 64] * gv)
    c = _make(1, 1, 4, 1, d, lens, dev, "int8")
    c.append(_t(k, dev), _t(v, dev))
    K, V = ref.read_back(k[0, 0, :, 0], "int8"), ref.read_back(v[0, 0, :, 0], "int8")
    # Queries that pick one row of each block with almost all the weight.
    for j in range(10):
        q = np.zeros((1, 1, n, 4, d), dtype=np.float32)
        row = min(64 * j + 11, lens[0] - 1)
        q[:] = ref.bf16(K[row] * 60.0 / (K[row] @ K[row]))
        out = _run_attend(c, q, dev, fp32, 1.0, None, False)
        for h in range(4):
            want, reach = ref.attend(q[0, 0, n - 1, h], K, V, 1.0, lens[0])
            tol = ref.tolerance(lens[0], d, reach, float(np.abs(V).max()), fp32)
            s = K @ q[0, 0, 0, 0].astype(np.float64)
            p = np.exp(s - s.max())
            p /= p.sum()
            # the average of |V| under the weights bounds every term of the output
            tol = tol / np.abs(V).max() * float((p @ np.abs(V)).max()) * 4 + 1e-30
            assert np.abs(out[0, 0, n - 1, h] - want).max() <= tol, (j, h)


@pytest.mark.parametrize("B,Hkv,G,n,rows", [(130, 1, 4, 8, 700), (70, 2, 7, 40, 600), (3, 1, 16, 20, 9000)])
@pytest.mark.parametrize("fp32", [True, False])
def test_ragged_batches_cut_along_their_rows(dev, B, Hkv, G, n, rows, fp32):
    """Counts of many sequences, some without queries, whose tiles' workgroups go
    to the others as further splits."""
    rng = np.random.default_rng(B)
    L = 2 if B == 70 else 1
    counts = [int(x) for x in rng.integers(0, n + 1, B)]
    counts[0], counts[-1], counts[B // 2] = n, n, 0
    lens = [int(x) for x in rng.integers(rows // 2, rows, L * B * Hkv)]
    c, K, V = _filled(rng, dev, L, B, G * Hkv, Hkv, 64, lens, "int8")
    q = ref.bf16(rng.standard_normal((L, B, n, G * Hkv, 64)))
    out = _run_attend(c, q, dev, fp32, 0.125, counts)
    _check_attend(out, q, K, V, lens, L, B, G * Hkv, Hkv, 0.125, counts, True, sample=[0, n - 1])
    none = _run_attend(c, q, dev, fp32, 0.125, [0] * B)
    assert (none == 7.0).all()


@pytest.mark.parametrize("L,B,Hkv,G,n,d", [(1, 40, 2, 4, 20, 64), (1, 3, 2, 8, 70, 128), (2, 25, 5, 16, 2, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_unlike_lengths_cut_along_their_rows(dev, L, B, Hkv, G, n, d, causal):
    """Units of no row to thousands whose rows are shared out, with one tile or
    several a unit, with and without counts, and with a bound below the longest."""
    rng = np.random.default_rng(B + causal)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(4000), L * B * Hkv))]
    lens[0], lens[1], lens[-1], lens[-2] = 4000, 0, 1, 64
    c, K, V = _filled(rng, dev, L, B, G * Hkv, Hkv, d, lens, "e4m3")
    q = ref.bf16(rng.standard_normal((L, B, n, G * Hkv, d)))
    for counts, most in ((None, 4000), (None, 1500), ([int(x) for x in rng.integers(0, n + 1, B)], 4000)):
        out = _run_attend(c, q, dev, False, d ** -0.5, counts, causal, max_rows=most)
        _check_attend(out, q, K, V, lens, L, B, G * Hkv, Hkv, d ** -0.5, counts or [n] * B, causal, most,
                      sample=[0, n - 1])


def test_parts_of_almost_nothing(dev):
    """A split whose values are zero but for rows of almost no weight: its part is
    tiny, not lost and not infinite."""
    rng = np.random.default_rng(24)
    d, rows, n = 64, 64 * 40, 20
    k, v = _values(rng, (1, 1, rows, 1, d)), np.zeros((1, 1, rows, 1, d), dtype=np.float32)
    k[0, 0, :, 0] = 0
    k[0, 0, ::2, 0, 0] = 1.0
    v[0, 0, 1::128, 0] = 1.0  # on rows of the small weight alone
    c = _make(1, 1, 4, 1, d, [rows], dev, "e4m3")
    c.append(_t(k, dev), _t(v, dev))
    K, V = ref.read_back(k[0, 0, :, 0], "e4m3"), ref.read_back(v[0, 0, :, 0], "e4m3")
    for pull in (1.0, 20.0, 60.0, 80.0):  # weights of e^-pull
        q = np.zeros((1, 1, n, 4, d), dtype=np.float32)
        q[..., 0] = pull
        for fp32 in (True, False):
            out = _run_attend(c, q, dev, fp32, 1.0, None, False)
            want, reach = ref.attend(q[0, 0, 0, 0], K, V, 1.0, rows)
            # Every term is positive, so the roundings are relative to the sum; but
            # weights are held in fp16, whose smallest step is 2^-24: half of it where
            # the largest weight is 2^14 (fp32 outputs) or at least 2^8, for each of
            # the 20 rows with values (the sum of the weights is at least 1).
            tol = ref.tolerance(rows, d, reach, 1.0, fp32) * np.abs(want).max() * 4
            tol += 20 * 2.0 ** -25 / (2.0 ** 14 if fp32 else 2.0 ** 8)
            assert np.isfinite(out).all() and float(np.abs(np.asarray(out[0, 0]) - want).max()) <= tol


def test_shared_and_strided_rows(dev):
    """Queries repeated by a stride of 0, outputs inside a wider tensor."""
    import paper_2608_24063_amd as vc
    rng = np.random.default_rng(12)
    lens = [200, 90]
    c, K, V = _filled(rng, dev, 1, 1, 8, 2, 128, lens, "int8")
    for n in (1, 30):
        q1 = ref.bf16(rng.standard_normal((1, 1, 1, 8, 128)))
        q = _t(q1, dev).expand(1, 1, n, 8, 128)
        wide = torch.full((1, 1, n, 12, 128), 7.0, dtype=torch.float32, device=dev)
        c.attend(q, wide[:, :, :, 2:10], 0.09)
        torch.cuda.synchronize()
        w = wide.cpu().numpy()
        assert (w[..., :2, :] == 7.0).all() and (w[..., 10:, :] == 7.0).all()
        _check_attend(w[..., 2:10, :], np.broadcast_to(q1, (1, 1, n, 8, 128)), K, V, lens, 1, 1, 8, 2, 0.09, [n], True,
                      sample=[0, n - 1])


def test_far_offsets(dev):
    """Rows whose codes lie more than 2^32 bytes into the pools."""
    from paper_2608_24063_amd.tensors import Q8Cache
    rng = np.random.default_rng(13)
    d, n = 128, 200
    far = (1 << 25) + 640  # rows; times d: past 2^32
    c = Q8Cache(1, 2, 2, 1, d, [far, n + 1], dev, format="int8")
    assert int(c.row_off[1]) * d > 1 << 32
    k, v = _values(rng, (1, 2, n, 1, d)), _values(rng, (1, 2, n, 1, d))
    c.append(_t(k, dev), _t(v, dev))
    K, V = [ref.read_back(k[0, b, :, 0], "int8") for b in range(2)], [ref.read_back(v[0, b, :, 0], "int8") for b in range(2)]
    for m in (1, 20):
        q = ref.bf16(rng.standard_normal((1, 2, m, 2, d)))
        out = _run_attend(c, q, dev, True, 0.1, max_rows=n)
        _check_attend(out, q, K, V, [n, n], 1, 2, 2, 1, 0.1, [m] * 2, True, sample=[0, m - 1])
    ko = torch.zeros((1, 2, n, 1, d), dtype=torch.float32, device=dev)
    vo = torch.zeros_like(ko)
    c.read(ko, vo)
    assert np.array_equal(ko[0, 1, :, 0].cpu().numpy(), K[1].astype(np.float32))
    assert np.array_equal(vo[0, 1, :, 0].cpu().numpy(), V[1].astype(np.float32))


# ---- a step in one call -------------------------------------------------------------

def _twins(rng_seed, dev, *a, **kw):
    return [_filled(np.random.default_rng(rng_seed), dev, *a, **kw)[0] for _ in range(2)]


def _same_caches(a, b):
    torch.cuda.synchronize()
    for n in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "len"):
        assert torch.equal(getattr(a, n).view(torch.uint8), getattr(b, n).view(torch.uint8)), n


ROPES = [None, dict(), dict(pairing=1), dict(rot=32, sections=(6, 5, 5), layout=1),
         dict(rot=48, sections=(0, 12, 12), pairing=1, scale=0.5)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d,G", [(64, 4), (128, 7), (128, 16), (64, 1)])
@pytest.mark.parametrize("turn", range(len(ROPES)))
@pytest.mark.parametrize("fp32", [True, False])
def test_step_is_its_three_calls(dev, fmt, d, G, turn, fp32):
    """viscache_q8_step against viscache_rope, _append and _attend: every buffer and
    output bit for bit, over units that are empty, full, about to be sealed."""
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(d + G + turn)
    L, B, Hkv = 2, 2, 3
    Hq = G * Hkv
    lens = [0, 1, 61, 62, 63, 64, 126, 127, 128, 500, 63, 64]
    a, b = _twins(turn, dev, L, B, Hq, Hkv, d, lens, fmt, extra=2)
    for c in (a, b):
        c.cap[10:] = torch.tensor([63, 64], dtype=torch.int32, device=dev)  # full ones
    rope = None if ROPES[turn] is None else Rope(d, theta=1e4, **ROPES[turn])
    for t in range(4):
        q, k, v = (_t(_values(rng, (L, B, 1, h, d)), dev) for h in (Hq, Hkv, Hkv))
        pos = torch.from_numpy(rng.integers(0, 9000, (3, B, 1)).astype(np.int32)).to(dev)
        typ = torch.float32 if fp32 else torch.bfloat16
        oa, ob = (torch.full((L, B, 1, Hq, d), 7.0, dtype=typ, device=dev) for _ in range(2))
        keep = [x.clone() for x in (q, k, v)]
        a.step(q, k, v, oa, 0.11, rope=rope, pos=pos)
        assert all(torch.equal(x, y) for x, y in zip((q, k, v), keep))
        if rope is not None:
            rope.apply(pos, q, k)
        b.append(k, v)
        b.attend(q, ob, 0.11)
        assert torch.equal(oa, ob), t
        _same_caches(a, b)
    assert a.len.cpu().tolist() == [min(n + 4, n + 2) if i < 10 else n for i, n in enumerate(lens)]


@pytest.mark.parametrize("fmt", FMTS)
def test_step_over_cut_units(dev, fmt):
    """Few long units, whose rows go to several workgroups: the last one appends,
    the join advances the lengths; across a sealing, on strided inputs."""
    rng = np.random.default_rng(21)
    L, B, Hq, Hkv, d = 1, 2, 14, 2, 128
    lens = [6398, 6399, 12, 8063]
    a, b = _twins(3, dev, L, B, Hq, Hkv, d, lens, fmt, extra=5)
    for t in range(4):
        wide = _t(_values(rng, (L, B, 1, Hq + 2 * Hkv, d)), dev)
        q, k, v = wide[:, :, :, :Hq], wide[:, :, :, Hq:Hq + Hkv], wide[:, :, :, Hq + Hkv:]
        oa, ob = (torch.zeros((L, B, 1, Hq, d), dtype=torch.float32, device=dev) for _ in range(2))
        a.step(q, k, v, oa, 0.09)
        b.append(k, v)
        b.attend(q, ob, 0.09)
        assert torch.equal(oa, ob), t
        _same_caches(a, b)
    assert a.len.cpu().tolist() == [n + 4 for n in lens]


def test_step_past_its_row_bound(dev):
    """A row bound below the lengths bounds what is attended, not what is appended."""
    import paper_2608_24063_amd as vc
    rng = np.random.default_rng(22)
    lens = [100, 63, 64, 200]
    a, b = _twins(4, dev, 1, 2, 8, 2, 64, lens, "int8", extra=3)
    q, k, v = (_t(_values(rng, (1, 2, 1, h, 64)), dev) for h in (8, 2, 2))
    oa, ob = (torch.zeros((1, 2, 1, 8, 64), dtype=torch.float32, device=dev) for _ in range(2))
    ws, nbytes = a._workspace(1, 64)
    r = lambda t: vc.vc_rows(t.data_ptr(), *t.stride()[:4])  # noqa: E731
    vc.viscache_q8_step(a.shape, a.c, None, 0, r(q), r(k), r(v), r(oa), 1, 0.125, 64, ws, nbytes,
                        torch.cuda.current_stream().cuda_stream)
    b.append(k, v)
    b.attend(q, ob, 0.125, max_rows=64)
    assert torch.equal(oa, ob)
    _same_caches(a, b)


def test_step_of_several_tokens(dev):
    """Prompts and drafts through step(): three calls, the inputs left alone."""
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(23)
    a, b = _twins(5, dev, 1, 2, 8, 2, 64, [100, 63, 64, 0], "e4m3", extra=70)
    rope = Rope(64, sections=(8, 12, 12))
    for n in (2, 66):
        q, k, v = (_t(_values(rng, (1, 2, n, h, 64)), dev) for h in (8, 2, 2))
        pos = torch.from_numpy(rng.integers(0, 9000, (3, 2, n)).astype(np.int32)).to(dev)
        oa, ob = (torch.zeros((1, 2, n, 8, 64), dtype=torch.bfloat16, device=dev) for _ in range(2))
        keep = q.clone()
        a.step(q, k, v, oa, 0.125, rope=rope, pos=pos)
        assert torch.equal(q, keep)
        rope.apply(pos, q, k)
        b.append(k, v)
        b.attend(q, ob, 0.125)
        assert torch.equal(oa, ob)
        _same_caches(a, b)


# ---- streams, graphs, runs of them together ------------------------------------------

def test_refused_step_appends_nothing(dev):
    """A step of several tokens looks at all of its tensors before the first launch."""
    rng = np.random.default_rng(24)
    a, _ = _twins(6, dev, 1, 2, 8, 2, 64, [100, 63, 64, 0], "int8", extra=70)
    before = a.len.clone()
    q, k, v = (_t(_values(rng, (1, 2, 3, h, 64)), dev) for h in (8, 2, 2))
    out = torch.zeros((1, 2, 3, 8, 64), dtype=torch.bfloat16, device=dev)
    for bad in (dict(out=out[:, :, :2]), dict(out=out.half()), dict(q=q[:, :, :, :6]), dict(v=v[:, :, :2]),
                dict(k=k[:, :, :2], v=v[:, :, :2]), dict(k=k.float())):
        args = dict(q=q, k=k, v=v, out=out, scale=0.125)
        args.update(bad)
        with pytest.raises(ValueError):
            a.step(**args)
        assert torch.equal(a.len, before)


def test_other_stream(dev):
    rng = np.random.default_rng(14)
    lens = [300, 70]
    c, K, V = _filled(rng, dev, 1, 1, 8, 2, 64, lens, "e4m3", extra=40)
    q = ref.bf16(rng.standard_normal((1, 1, 1, 8, 64)))
    tq, out = _t(q, dev), torch.zeros((1, 1, 1, 8, 64), dtype=torch.float32, device=dev)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.attend(tq, out, 0.125)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    _check_attend(out.cpu().numpy(), q, K, V, lens, 1, 1, 8, 2, 0.125, [1], True)


@pytest.mark.parametrize("fmt", FMTS)
def test_graph_of_steps(dev, fmt):
    """A captured serving step, replayed across a block's sealing with eager work
    between the replays, and a second graph on the same workspace, equals eager
    steps on a second cache bit for bit."""
    from paper_2608_24063_amd.tensors import Rope
    rng = np.random.default_rng(15)
    L, B, Hq, Hkv, d, steps = 2, 2, 8, 2, 64, 7
    lens = [60, 61, 62, 63, 64, 0, 640, 1000]
    a, _, _ = _filled(np.random.default_rng(1), dev, L, B, Hq, Hkv, d, lens, fmt, extra=40)
    b, _, _ = _filled(np.random.default_rng(1), dev, L, B, Hq, Hkv, d, lens, fmt, extra=40)
    rope = Rope(d, sections=(8, 12, 12))
    xs = {n: _t(_values(rng, (steps, L, B, 1, h, d)), dev) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
    ps = torch.from_numpy(rng.integers(0, 5000, (steps, 3, B, 1)).astype(np.int32)).to(dev)
    buf = {n: torch.zeros_like(x[0]) for n, x in xs.items()}
    pos = torch.zeros_like(ps[0])
    oa = torch.zeros((L, B, 1, Hq, d), dtype=torch.float32, device=dev)
    ob, oc = torch.zeros_like(oa), torch.zeros_like(oa)
    qr = torch.zeros_like(buf["q"])
    pq = _t(_values(rng, (L, B, 9, Hq, d)), dev)
    po, pe = torch.zeros((L, B, 9, Hq, d), dtype=torch.bfloat16, device=dev), torch.zeros((L, B, 9, Hq, d), dtype=torch.bfloat16, device=dev)
    a._workspace(9, a.max_cap), a._workspace(1, a.max_cap)
    keep = {n: getattr(a, n).view(torch.uint8).clone() for n in ("k_codes", "v_codes", "k_tail", "v_tail", "k_scale", "v_scale", "len")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # once before the capture
        a.step(buf["q"], buf["k"], buf["v"], oa, 0.125, rope=rope, pos=pos)
        a.attend(pq, po, 0.125)
    torch.cuda.current_stream().wait_stream(side)
    for n, x in keep.items():
        getattr(a, n).view(torch.uint8).copy_(x)
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        a.step(buf["q"], buf["k"], buf["v"], oa, 0.125, rope=rope, pos=pos)
    with torch.cuda.graph(g2):
        a.attend(pq, po, 0.125)
    torch.cuda.synchronize()
    for t in range(steps):
        for n in buf:
            buf[n].copy_(xs[n][t])
        pos.copy_(ps[t])
        g1.replay()
        g2.replay()
        torch.cuda.synchronize()
        b.step(xs["q"][t], xs["k"][t], xs["v"][t], ob, 0.125, rope=rope, pos=ps[t].contiguous())
        rope.apply(pos, buf["q"], q_out=qr)
        b.attend(pq, pe, 0.125)
        a.attend(qr, oc, 0.125)  # eager, on the graphs' workspace
        torch.cuda.synchronize()
        assert torch.equal(oa, ob) and torch.equal(po, pe) and torch.equal(oc, oa), f"step {t}"
    assert torch.equal(a.len, b.len)
    for n in ("k_codes", "v_codes"):
        assert torch.equal(getattr(a, n).view(torch.uint8), getattr(b, n).view(torch.uint8))
    # a larger call grows the workspace; the graphs keep the one they know
    before = po.clone()
    big = _t(_values(rng, (L, B, 300, Hq, d)), dev)
    a.attend(big, torch.zeros_like(big), 0.125)
    g2.replay()
    torch.cuda.synchronize()
    assert torch.equal(po, before)


def test_pruned_cache_to_decode(dev, sg):
    """The whole run: prune a cache, load its kept rows in 8 bits, answer a few
    tokens and a second prompt over it, each against the plain form."""
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import PruneCall, Q8Cache, Rope
    from synthgen.device import upload_layers
    w = sg.TINY
    n = [int(x) for x in w.n_vis()]
    dv, _ = upload_layers(w, range(w.L), dev, keep_host=True)
    pc = PruneCall(w.B, w.L, w.Hq, w.Hkv, w.d, w.W, n, vc.make_params(w.retention), [dv["K"][l] for l in range(w.L)],
                   [dv["V"][l] for l in range(w.L)], [dv["Q"][l] for l in range(w.L)])
    pc.run()
    units = w.L * w.B * w.Hkv
    kept = [pc.k[u // w.Hkv % w.B * w.L + u // (w.B * w.Hkv)] for u in range(units)]
    steps, m = 3, 11
    c = Q8Cache(w.L, w.B, w.Hq, w.Hkv, w.d, [x + steps + m for x in kept], dev, format="e4m3")
    _foul(c)
    c.load_pruned(pc)
    rows = []
    for u in range(units):
        l, b, g = u // (w.B * w.Hkv), u // w.Hkv % w.B, u % w.Hkv
        r0, r1 = pc.unit_rows(l, b, g)
        rows.append([pc.k_out[l][r0:r1].float().cpu().numpy(), pc.v_out[l][r0:r1].float().cpu().numpy()])
    assert [len(r[0]) for r in rows] == kept and min(kept) == 0 < max(kept)
    _check_cache(c, rows, "e4m3")
    rng = np.random.default_rng(16)
    rope = Rope(w.d, sections=(8, 12, 12), theta=1e6)
    freq = [1e6 ** (-2.0 * i / w.d) for i in range(w.d // 2)]
    ax = ref.rope_axes(w.d, (8, 12, 12), False)
    for t, cnt in enumerate([1] * steps + [m]):
        q, k, v = (_values(rng, (w.L, w.B, cnt, h, w.d)) for h in (w.Hq, w.Hkv, w.Hkv))
        pos = np.broadcast_to(max(n) + 20 * t + np.arange(cnt), (3, w.B, cnt)).astype(np.int32)
        tq, tk = _t(q, dev), _t(k, dev)
        out = torch.full((w.L, w.B, cnt, w.Hq, w.d), 7.0, dtype=torch.float32, device=dev)
        tp = _t(pos, dev, torch.int32)
        c.step(tq, tk, _t(v, dev), out, w.d ** -0.5, rope=rope, pos=tp)
        assert np.array_equal(tq.float().cpu().numpy(), q) and np.array_equal(tk.float().cpu().numpy(), k)
        rope.apply(tp, tq, tk)  # the rows as the step turned them
        torch.cuda.synchronize()
        # the rotation, to half a step of bf16 (2^-8) and the roundings of an fp32 rotation
        gq, gk = tq.float().cpu().numpy(), tk.float().cpu().numpy()
        for x, got in ((q, gq), (k, gk)):
            for l in range(w.L):
                for b in range(w.B):
                    for h in range(x.shape[3]):
                        want = ref.rope(x[l, b, :, h], pos[:, b], w.d, freq, ax, False, False, 1.0)
                        assert (np.abs(got[l, b, :, h] - want) <= np.abs(want) * 2.0 ** -8 + 1e-6 * np.abs(x).max()).all()
        for u in range(units):  # the cache holds the rotated rows as the device rounded them
            l, b, g = u // (w.B * w.Hkv), u // w.Hkv % w.B, u % w.Hkv
            rows[u][0] = np.concatenate((rows[u][0], gk[l, b, :, g]))
            rows[u][1] = np.concatenate((rows[u][1], v[l, b, :, g]))
        _check_cache(c, rows, "e4m3")
        K = [ref.read_back(r[0], "e4m3") for r in rows]
        V = [ref.read_back(r[1], "e4m3") for r in rows]
        _check_attend(out.cpu().numpy(), gq, K, V, [len(x) for x in K], w.L, w.B, w.Hq, w.Hkv, w.d ** -0.5, [cnt] * w.B,
                      True, sample=[0, cnt - 1])


def test_workspace_growth_is_refused_in_a_capture(dev):
    c = _make(1, 1, 4, 2, 64, [300, 300], dev, "int8", foul=False)
    q = torch.zeros((1, 1, 9, 4, 64), dtype=torch.bfloat16, device=dev)
    g = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError):
        with torch.cuda.graph(g):
            c.attend(q, torch.empty_like(q), 0.125)
    torch.cuda.synchronize()
    c.attend(q, torch.empty_like(q), 0.125)
    torch.cuda.synchronize()
