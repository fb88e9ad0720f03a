"""A decay of zero leaves the last call's weights alone, whatever the masses were before: never
written, infinite or spoilt by a query with a NaN."""
import numpy as np
import pytest

from tests import mass_paths as mp
from tests.test_gpu_mass_attend import dev  # noqa: F401
from tests.test_gpu_mass_finite import Finite

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

CUT = mp.Path("cut", 1, 2, 8, 2, 1, 5000, {})            # single tokens in pieces
SPLIT = mp.Path("split", 1, 2, 8, 2, 300, 900, {})       # a prompt's tiles and masses in parts
SPILLED, WHOLE = mp.TOKENS[4], mp.PROMPTS[1]
SMALL = mp.Path("small", 1, 3, 28, 4, 2, 200, {})


@pytest.mark.parametrize("p", [SMALL, CUT, SPILLED, SPLIT, WHOLE], ids=lambda p: p.name)
@pytest.mark.parametrize("was", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("append", [True, False])
def test_nothing_is_left(dev, p, was, append):  # noqa: F811
    lens, caps = mp.sizes(p)
    x = Finite(47, dev, p.L, p.B, p.Hq, p.Hkv, 64, lens, caps)
    for unit, o in zip(x.units, x.off):
        x.c.mass[o:o + len(unit.K)] = was
        unit.mass[:] = 0.0  # (the reference multiplies)
    q, k, v = x.inputs(p.n)
    x.attend(q, *((k, v) if append else ()), decay=0.0)
    x.attend(*x.inputs(p.n), decay=1.0)  # and adds to numbers again


def test_a_decay_keeps_what_is_infinite(dev):  # noqa: F811
    """Any other decay multiplies: an infinite mass stays infinite, none becomes a number again."""
    lens, caps = mp.sizes(SMALL)
    x = Finite(53, dev, 1, 3, 28, 4, 64, lens, caps)
    o, n = x.off[1], lens[1]
    x.c.mass[o], x.c.mass[o + 1] = float("inf"), float("nan")
    q, k, v = (torch.from_numpy(np.ascontiguousarray(t)).to(dev).to(torch.bfloat16) for t in x.inputs(2))
    x.c.attend(q, torch.zeros(q.shape, device=dev), 0.1, k=k, v=v, decay=0.5)
    got = x.c.mass[o:o + n]
    assert torch.isposinf(got[0]) and torch.isnan(got[1]) and torch.isfinite(got[2:]).all()
