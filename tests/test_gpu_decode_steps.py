"""Tables, cache writes, attention and experts together, as the example serves requests with them."""
import pytest

from examples import decode_steps

import kv_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "latent", "latent_e4m3"])
def test_requests_served_by_a_recorded_step_and_by_eager_ones(torch_cuda, cache):
    torch = torch_cuda
    print("decode steps", cache, flush=True)
    server, answers = decode_steps.serve(R=6, steps=40, page_size=16, cache=cache)
    eager, same = decode_steps.serve(R=6, steps=40, page_size=16, cache=cache, eager=True)
    assert answers == same and len(answers) > 6 and sum(map(len, answers)) == 6 * 40
    t = server.tables
    # every page is either a request's or free, and each of them once
    have = (t.lens.cpu() + 15) // 16
    take, back = t.pool.tolist()
    N = len(t.ring)
    ring = t.ring.tolist()
    held = [p for r in range(6) for p in t.table[r, :have[r]].tolist()] + [ring[i % N] for i in range(take, back)]
    assert sorted(held) == list(range(N))
    # the last step's attention in every layer against 64 bits over what the cache holds
    for layer in server.layers:
        c = layer.cache
        out, _, bound, _ = ref.attention(layer.q, c.k, c.v, c.k_scale, c.v_scale, t.lens.cpu(), t.table, c.dk ** -0.5, dv=c.dv)
        assert bool(((layer.attention.out.cpu().double() - out).abs() <= bound).all())


def test_requests_served_over_pages_of_another_size(torch_cuda):
    # where the rows lie is no part of the result; runs of units do not depend on the size of pages either
    answers = [decode_steps.serve(R=4, steps=20, page_size=P)[1] for P in (16, 64)]
    assert answers[0] == answers[1]
