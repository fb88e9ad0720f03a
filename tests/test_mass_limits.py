"""Row bounds up to the largest: single tokens over units that are cut are refused where a
launch would hold 2^32 threads, and nowhere before (the header's limits)."""
import pytest

from tests.test_q8_abi import _shape, vc  # noqa: F401


@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("units", [1, 2, 3, 4, 7, 8, 9, 64])
def test_second_launch_of_single_tokens(vc, units, n):  # noqa: F811
    """1024 threads join 4096 rows: 2^19 workgroups a unit of 2^31 - 1025 rows, 2^22 in all are
    one too many."""
    s = _shape(vc, B=1, L=units, Hq=4, Hkv=1)
    for rows in (1 << 20, 1 << 27, 2 ** 31 - 1025, 2 ** 31 - 1):
        tiles = -(-min(rows, 2 ** 31 - 1025) // 4096)
        fits = units * tiles < 1 << 22
        assert (vc.viscache_mass_attend_workspace_bytes(s, n, rows) > 0) == fits, (units, rows)


def test_short_bounds_are_as_before(vc):  # noqa: F811
    for units, rows in ((1, 600), (96, 40000), (128, 23000), (4, 5000)):
        assert vc.viscache_mass_attend_workspace_bytes(_shape(vc, B=1, L=units, Hq=4, Hkv=1), 1, rows) > 0
