"""Scales whose product with log2 e is not finite in 32 bits are refused: scores are scaled by that product, and 0 times it would be NaN.
Host code, no GPU needed: what passes the check of the scale is refused for its workspace."""
import pytest

from test_draft_refusals import _attn, ngc     # noqa: F401 (a fixture)


@pytest.mark.parametrize("paged", [False, True])
def test_scales_at_the_end_of_the_range(ngc, paged):     # noqa: F811
    for scale in (2.4e38, 2.5e38, 2.9e38, 3.0e38, 3.4e38):
        assert _attn(ngc, paged, scale=scale, ws_bytes=64) == ngc.NGC_EINVAL, scale
    for scale in (2.35e38, 1e38, 1.0, 1e-38, 1e-45):
        assert _attn(ngc, paged, scale=scale, ws_bytes=64) == ngc.NGC_ENOSPC, scale
