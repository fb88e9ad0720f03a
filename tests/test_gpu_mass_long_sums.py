"""Masses of prompts with very many columns: a row's sum over all of them is formed in parts
of at most 64 blocks of 64 columns."""
import pytest

from tests.test_gpu_mass_attend import dev  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_many_equal_weights(dev):  # noqa: F811
    """2^18 columns that all see the same 524163 rows of equal keys, so that each gives a row w
    = 1 / 524163.  Added one after another, a lane's 2^13 weights would each be rounded to the
    same side once their sum is large: the last 4096 steps lose 0.29 of half a step each on
    average, 1.2e-4 of the whole.  Tolerance: w is off by 2^-23 (the quotient's rounding and
    a step), a part's sum by 128 additions in a lane and 4 over the lanes, and the whole, in
    64 bits, is rounded once: 133 2^-24 and 2^-23, 8.1e-6."""
    from paper_2608_24063_amd.tensors import MassCache
    rows, n, Hq, d = 524163, 1 << 14, 16, 64
    c = MassCache(1, 1, Hq, 1, d, [rows + n], dev)
    c.k_pool.zero_()
    c.v_pool.fill_(1.0)
    c.len.fill_(rows + n)  # query 0 sees rows + 1 of them
    q = torch.ones((1, 1, n, Hq, d), dtype=torch.bfloat16, device=dev)
    out = torch.zeros_like(q)
    c.attend(q, out, 1.0, decay=0.0, max_rows=rows)
    want = n * Hq / rows
    got = c.mass[:rows].double()
    assert (got - want).abs().max() <= want * (133 * 2.0 ** -24 + 2.0 ** -23)
    assert not c.mass[rows:].any() and (out == 1).all()
