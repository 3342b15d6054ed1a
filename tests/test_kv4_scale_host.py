"""The largest scale of the attention: the kernels take it times log2(e) * 2^16, which
has to be finite in float32."""
import pytest

from tests.test_kv4_host import _attend, lib  # noqa: F401


@pytest.mark.parametrize("scale", [2.0 ** 110 * 1.001, 1e34, 3.4e38])
def test_scales_beyond_the_range_are_refused(lib, scale):  # noqa: F811
    assert _attend(lib, scale=scale) == 1
