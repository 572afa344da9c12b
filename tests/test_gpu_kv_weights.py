"""How exactly the weights of decode attention enter the sum of values: few tokens and columns whose values nearly cancel,
where a rounding of the weights is large beside the result's own."""
import pytest
import torch

import kv_reference as ref
from test_gpu_kv_cache import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,P", [(64, 16), (128, 16), (128, 4), (256, 64), (80, 1)])
def test_weights_count_with_15_bits(torch_cuda, fmt, d, P):
    """kv_reference's bound allows 2^-8 of A, the sum of weights times absolute values, for the rounding of the weights to
    bf16.  As an upper half and the nearest bf16 number to the rest, which is below 2^-7 of the weight (and taken as 2^-20 of
    it where it is less), they are off by 2^-7 * 2^-8 + 2^-20."""
    print("weights", fmt, d, P, flush=True)
    s = Setup(torch_cuda, [2, 3, 4, 5, 7, 9, 33, 100, 400] * 4, 32, 4, d, d, P, fmt, seed=d + P, peak=0.5)
    s.call()
    c = s.cache
    args = (s.q, c.k, c.v, c.k_scale, c.v_scale, s.lens, s.d_table, s.scale)
    want, _, bound, _ = ref.attention(*args)
    absolute = c.v.float().abs().to(c.v.dtype)
    A = ref.attention(s.q, c.k, absolute, *args[3:])[0]
    bound = bound - (2.0 ** -8 - 2.0 ** -15 - 2.0 ** -20) * A
    err = (s.attn.out.double().cpu() - want).abs()
    small = want.abs() < A / 16
    assert int(small.sum()) > 1000
    assert bool((err <= bound).all()), f"over the bound by {(err / bound).max():.2f}, where values cancel by {(err / bound)[small].max():.2f}"


@pytest.mark.parametrize("fmt", ["f32", "bf16"])
@pytest.mark.parametrize("P", [4, 64])
def test_infinite_values_of_visible_tokens(torch_cuda, fmt, P):
    """A visible token's infinity makes its column infinite, whatever the token's weight (all of its bits in one bf16 number,
    the largest, a small one), and no other column."""
    print("infinite values", fmt, P, flush=True)
    lens, d = [1, 2, 40, 300], 64
    s = Setup(torch_cuda, lens, 8, 2, d, d, P, fmt, seed=P, peak=1.0)
    s.q[:, ::2] = 0                                       # weights of exactly one
    c = s.cache
    signs = {}
    for r, n in enumerate(lens):
        for j, i in enumerate((0, n // 2, n - 1)):
            page, place = int(s.table[r, i // P]), i % P
            for h in range(2):
                column = 3 + 16 * j + h
                sign = -1.0 if (r + h) % 2 else 1.0
                c.v[page, h, place, column] = sign * float("inf")
                signs[r, h, column] = sign
    out = s.call().float().cpu()
    finite = c.v.clone()
    finite[torch.isinf(finite)] = 0
    want, _, bound, _ = ref.attention(s.q, c.k, finite, None, None, s.lens, s.d_table, s.scale)
    for (r, h, column), sign in signs.items():
        assert bool((out[r, 4 * h:4 * h + 4, column] == sign * float("inf")).all()), (r, h, column)
        want[r, 4 * h:4 * h + 4, column] = bound[r, 4 * h:4 * h + 4, column] = out[r, 4 * h:4 * h + 4, column] = 0
    assert bool(((out.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("P", [4, 64])
def test_an_infinite_scale_of_a_visible_token(torch_cuda, P):
    """A row of codes whose scale is infinite has infinities of its codes' signs, and NaN where the code is zero."""
    lens, d = [1, 33, 300], 64
    s = Setup(torch_cuda, lens, 8, 2, d, d, P, "e4m3", seed=P, peak=1.0)
    c = s.cache
    for r, n in enumerate(lens):
        i = n // 2
        page, place = int(s.table[r, i // P]), i % P
        c.v_scale[page, 0, place] = float("inf")
        codes = torch.full((d,), 1.0, device=c.v.device)
        codes[1::3], codes[2::3] = -2.0, 0.0
        c.v.view(torch.uint8)[page, 0, place] = codes.to(c.v.dtype).view(torch.uint8)
    out = s.call().float().cpu()
    assert bool((out[:, :4, 0::3] == float("inf")).all()) and bool((out[:, :4, 1::3] == float("-inf")).all()) and bool(torch.isnan(out[:, :4, 2::3]).all())
    assert bool(torch.isfinite(out[:, 4:]).all())
