"""Scales past the range that the sums are held in are refused (CPU only: no rows, so that no pointer is looked at)."""
import pytest

from test_router_embed_mx4_validation import ROWS, dpc  # noqa: F401


@pytest.mark.parametrize("x", ROWS)
def test_scale_past_the_sums_range(dpc, x):  # noqa: F811
    lib = dpc._lib
    most = 1.7976931348623157e308 if x == "f64" else 3.4028234663852886e38

    def calls(scale):
        return [getattr(lib, f"dp_route_topk_{x}")(None, None, 0, 8, 2, 0, 1, 1, 1, 1, scale, None, None, None),
                getattr(lib, f"dp_route_topk_grad_{x}")(None, None, None, 0, 8, 2, 0, 1, scale, None, None),
                getattr(lib, f"dp_embed_fwd_{x}")(None, None, 0, 8, 100, scale, None, None, None)]

    for scale in (most, -most, 0.0, 1e-300):
        assert calls(scale) == [dpc.DP_OK] * 3
    for scale in ((float("inf"),) if x == "f64" else (most * 1.0001, -1e39, 1e300, float("-inf"))):
        assert calls(scale) == [dpc.DP_ERR_SHAPE] * 3, scale
        assert getattr(lib, f"dp_embed_grad_{x}")(None, None, None, None, 0, 8, 100, scale, 0, None, None, 0, None) == dpc.DP_ERR_SHAPE
