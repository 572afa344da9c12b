"""Arguments at the ends of what the paged-cache calls take.  No device work: every call here is refused."""
import ctypes

import pytest

from paper_2603_28768_amd import binding

import test_kv_cache_host as host


@pytest.mark.parametrize("scale", [3.0e38, -3.0e38, 2.4e38])
def test_a_scale_that_overflows_as_a_power_of_two_is_refused(scale):
    # the kernels multiply scores by scale * log2(e): an infinity would make every weight a NaN
    a = host.attention(scale=scale, workspace_bytes=1 << 40)
    assert binding.lib().craft_decode_attention(ctypes.byref(host.cache()), ctypes.byref(a), None) == host.EINVAL
