"""The parity tests of attention with masses once more, with every output and mass held to
be a number: a NaN is no further from a value than a tolerance allows (no comparison with it
holds), so a test that looks for values past theirs takes it for right."""
import numpy as np
import pytest

from tests import test_gpu_mass_attend as base
from tests.test_gpu_mass_attend import (Pair, dev, test_calls_after_one_another, test_long_units_in_pieces,  # noqa: F401
                                        test_many_long_units_in_pieces, test_masses_of_many_calls, test_row_bound,
                                        test_strides)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


class Finite(Pair):
    """A Pair whose outputs, rows and masses are finite throughout."""

    def attend(self, *args, **kw):
        out = super().attend(*args, **kw)
        assert torch.isfinite(out).all()
        return out

    def check_cache(self):
        super().check_cache()
        mass = self.c.mass.cpu().numpy()
        for u, (unit, o) in enumerate(zip(self.units, self.off)):
            assert np.isfinite(mass[o:o + unit.cap]).all(), u


@pytest.fixture(autouse=True)
def finite(monkeypatch):
    monkeypatch.setattr(base, "Pair", Finite)
