"""What the example asks of the paged cache, without a GPU."""
import pytest

from examples import decode_steps
from paper_2603_28768_amd import binding

import test_kv_cache_host as host


@pytest.mark.parametrize("cache", ["latent", "latent_e4m3"])
def test_latent_rows_of_the_example_go_through_their_own_kernel(cache):
    """It serves latent rows of more than 256 elements.  Its parts are whole workgroups' of 64 heads, and it has records
    of the cuts beside them, so the workspace it asks for tells it from the kernel of ordinary rows."""
    heads, dk, dv = decode_steps.cache_rows(cache)
    assert heads == 1 and 256 < dk <= 576 and dv <= dk

    def size(dk, dv):
        c = host.cache(v=None, heads=heads, dk=dk, dv=dv, k_page=16 * dk, k_head=16 * dk, k_token=dk, k_scale=host.ADDR,
                       format=binding.CRAFT_KV_E4M3 if cache.endswith("e4m3") else binding.CRAFT_KV_BF16)
        rc, n = host.size_of(c, host.attention(Hq=decode_steps.HEADS))
        assert rc == host.OK
        return n
    part = (16 * 512 + 128) * 4                       # 16 heads' sums
    a_worker = 16 + 2 * 4 * part                      # its cut, and its two parts of 64 heads
    assert (size(dk, dv) - (48 << 10)) % a_worker == 0 and (size(256, 256) - (48 << 10)) % a_worker != 0
