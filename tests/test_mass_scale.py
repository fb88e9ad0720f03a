"""The scale of attention with masses times log2(e), which the kernels take, is finite."""
from tests.test_mass_abi import _attend, vc  # noqa: F401


def test_scales_at_the_upper_end(vc):  # noqa: F811
    for scale in (2.4e38, 3.4e38):
        assert _attend(vc, scale=scale) == _attend(vc, scale=scale, n=1) == vc.VC_ERR_ARG
    for scale in (1e-38, 2.3e38):
        assert _attend(vc, scale=scale, ws=0) == vc.VC_ERR_WORKSPACE
