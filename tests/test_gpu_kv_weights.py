"""How exactly the weights of decode attention enter the sum of values: few tokens and columns whose values nearly cancel,
where a rounding of the weights is large beside the result's own."""
import pytest
import torch

import kv_reference as ref
from test_gpu_kv_cache import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,P", [(64, 16), (128, 16), (128, 4), (256, 64), (80, 1)])
def test_weights_count_with_16_bits(torch_cuda, fmt, d, P):
    """kv_reference's bound allows 2^-8 of A, the sum of weights times absolute values, for the rounding of the weights to
    bf16.  Rounded to the nearest bf16 number and to the nearest to the rest they are off by 2^-8 * 2^-8."""
    print("weights", fmt, d, P, flush=True)
    s = Setup(torch_cuda, [2, 3, 4, 5, 7, 9, 33, 100, 400] * 4, 32, 4, d, d, P, fmt, seed=d + P, peak=0.5)
    s.call()
    c = s.cache
    args = (s.q, c.k, c.v, c.k_scale, c.v_scale, s.lens, s.d_table, s.scale)
    want, _, bound, _ = ref.attention(*args)
    absolute = c.v.float().abs().to(c.v.dtype)
    A = ref.attention(s.q, c.k, absolute, *args[3:])[0]
    bound = bound - (2.0 ** -8 - 2.0 ** -16) * A
    err = (s.attn.out.double().cpu() - want).abs()
    small = want.abs() < A / 16
    assert int(small.sum()) > 1000
    assert bool((err <= bound).all()), f"over the bound by {(err / bound).max():.2f}, where values cancel by {(err / bound)[small].max():.2f}"
