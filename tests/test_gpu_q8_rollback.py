"""Rows taken back from an 8-bit cache by lowering its lengths: to a multiple of the
block or within the open block, as the library documents.  What is appended then
makes the cache that its rows alone make."""
import numpy as np
import pytest

from tests import q8_ref as ref
from tests.test_gpu_q8 import FMTS, _check_attend, _make, _run_attend, _t, _values, dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("first,back,then", [(66, 64, 3), (66, 65, 63), (190, 128, 0), (190, 128, 5), (190, 190, 2),
                                             (190, 64, 64), (127, 100, 30), (128, 128, 1), (130, 0, 70), (40, 1, 0)])
@pytest.mark.parametrize("single", [True, False])
def test_rows_taken_back(dev, fmt, first, back, then, single):  # noqa: F811
    """first rows, the length lowered to `back`, then other rows, one call or a row a call."""
    rng = np.random.default_rng(first + back + then)
    B, Hkv, d = 2, 2, 64
    c = _make(1, B, 4, Hkv, d, [300] * (B * Hkv), dev, fmt)
    k, v = (_values(rng, (1, B, first, Hkv, d)) for _ in "kv")
    k[:, :, back:] *= 8  # louder than what stays
    c.append(_t(k, dev), _t(v, dev))
    c.len.fill_(back)
    k2, v2 = (_values(rng, (1, B, then, Hkv, d)) for _ in "kv")
    for i in range(then) if single or then == 0 else [slice(0, then)]:
        i = slice(i, i + 1) if single else i
        c.append(_t(k2[:, :, i], dev), _t(v2[:, :, i], dev))
    k, v = (np.concatenate((a[:, :, :back], b), axis=2) for a, b in ((k, k2), (v, v2)))
    n = back + then
    rows = [(k[0, b, :, g], v[0, b, :, g]) for b in range(B) for g in range(Hkv)]
    if n % 64 == 0 or then > n % 64 or back % 64 == 0:  # no open block that was lowered into
        c2 = _make(1, B, 4, Hkv, d, [300] * (B * Hkv), dev, fmt)
        c2.append(_t(k, dev), _t(v, dev))
        torch.cuda.synchronize()
        for u in range(B * Hkv):
            b0, nb = int(c.row_off[u]) // 64, (n + 63) // 64
            for x in ("k_scale", "v_scale"):
                assert torch.equal(getattr(c, x)[b0:b0 + nb], getattr(c2, x)[b0:b0 + nb])
            for x in ("k_codes", "v_codes"):
                x, y = (getattr(z, x)[b0:b0 + n // 64].view(torch.uint8) for z in (c, c2))
                assert torch.equal(x, y)
    ko = torch.zeros((1, B, 300, Hkv, d), dtype=torch.float32, device=dev)
    vo = torch.zeros_like(ko)
    c.read(ko, vo)
    for u, (x, y) in enumerate(rows):
        for out, want in ((ko, x), (vo, y)):
            assert np.array_equal(out[0, u // Hkv, :n, u % Hkv].cpu().numpy(), ref.read_back(want, fmt).astype(np.float32))
    K, V = ([ref.read_back(r[i], fmt) for r in rows] for i in (0, 1))
    for m in (1, 9):
        q = ref.bf16(rng.standard_normal((1, B, m, 4, d)))
        out = _run_attend(c, q, dev, True, 0.1)
        _check_attend(out, q, K, V, [n] * len(rows), 1, B, 4, Hkv, 0.1, [m] * B, True)
