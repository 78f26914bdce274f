"""slicer_kv_*, calls that need no GPU: refusals of scales that fp32 does not hold."""
import pytest

from tests.test_kv_cpu import attend, handle, lib  # noqa: F401 (a fixture)


@pytest.mark.parametrize("scale", [3e38, -3e38, 1e39, 1e300, -1e300])
def test_scales_beyond_fp32_are_refused(lib, scale):  # noqa: F811
    """3e38 is finite in fp32, and times log2(e) it is not."""
    assert attend(lib, handle(), scale=scale) == -1
