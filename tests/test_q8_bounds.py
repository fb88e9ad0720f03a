"""Row bounds and lengths that do not fit 32 bits: an argument keeps its meaning or
is refused, and never comes to the library as its low 32 bits."""
import pytest

from tests.test_q8_abi import _append, _attend, _read, _rope, _shape, _step, vc  # noqa: F401


@pytest.mark.parametrize("high", [2 ** 32, 2 ** 40, -2 ** 32, 2 ** 63], ids=hex)
@pytest.mark.parametrize("low", [0, 4, 64])
def test_arguments_past_32_bits(vc, high, low):  # noqa: F811
    x, s = high + low, _shape(vc)
    A, U, W = vc.VC_ERR_ARG, vc.VC_ERR_UNSUPPORTED, vc.VC_ERR_WORKSPACE
    far = x > 0
    # as a count of rows, queries or tokens: more than any call takes
    assert _append(vc, n=x) == _read(vc, rows=x) == _attend(vc, n=x) == _rope(vc, n=x) == (U if far else A)
    assert vc.viscache_q8_attend_workspace_bytes(s, x, 100) == 0
    # as a row bound: no bound
    need = vc.viscache_q8_attend_workspace_bytes(s, 1, 2 ** 31 - 1)
    assert vc.viscache_q8_attend_workspace_bytes(s, 1, x) == (need if far else 0)
    assert _attend(vc, rows=x, bytes_=need - 1) == _step(vc, rows=x, bytes_=need - 1) == (W if far else A)


def test_workspace_is_checked_last(vc):  # noqa: F811
    """A call without a workspace asks for the other checks."""
    big, none = _shape(vc, B=1 << 20, L=8, Hq=1, Hkv=1), dict(ws=0, bytes_=0)
    row = vc.vc_rows(0x10000, 1 << 38, 1 << 18, 128, 128)
    for n in (1, 3, 40):
        assert _attend(vc, n=n, **none) == vc.VC_ERR_WORKSPACE
        assert _attend(vc, n=n, scale=0.0, **none) == _attend(vc, n=n, q=vc.vc_rows(8), **none) == vc.VC_ERR_ARG
    assert _attend(vc, n=1 << 23, **none) == _attend(vc, big, q=row, out=row, **none) == vc.VC_ERR_UNSUPPORTED


def test_bound_of_a_cache():
    from paper_2608_24063_amd.tensors import Q8Cache
    c = Q8Cache(1, 1, 4, 2, 64, [5, 70], "cpu")
    assert [c._bound(x) for x in (None, 0, 64, 70, 71, 2 ** 31, 2 ** 32, 2 ** 32 + 64, 2 ** 40)] == [70, 0, 64] + [70] * 6
    assert c._bound(-1) < 0 and c._bound(-2 ** 32) < 0 and c._bound(-2 ** 32 + 64) < 0


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 9])
def test_no_bound_attends_every_row(n):
    import numpy as np
    torch = pytest.importorskip("torch")
    from tests.test_gpu_q8 import _filled, _t
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    rng = np.random.default_rng(51)
    c, _, _ = _filled(rng, dev, 1, 2, 8, 2, 64, [300, 90, 64, 200], "int8")
    q = _t(rng.standard_normal((1, 2, n, 8, 64)), dev)
    want = torch.empty(q.shape, dtype=torch.float32, device=dev)
    c.attend(q, want, 0.125)
    for most in (2 ** 31, 2 ** 32, 2 ** 32 + 64, 2 ** 40):
        out = torch.zeros_like(want)
        c.attend(q, out, 0.125, max_rows=most)
        assert torch.equal(out, want), most
    k = torch.zeros((1, 2, 300, 2, 64), dtype=torch.bfloat16, device=dev)
    with pytest.raises(ValueError):
        c.read(k, k.clone(), max_rows=2 ** 32 + 5)
