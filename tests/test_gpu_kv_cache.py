"""The paged cache on the GPU: tables against a request-by-request walk (equal), writes (equal; 8 bits against the CPU
oracle's codes and scales), attention against 64 bits within the bound that kv_reference.attention derives."""
import numpy as np
import pytest

import oracle
from paper_2603_28768_amd import binding

import kv_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
COUNTERS = 48 << 10         # bytes of an attention workspace that are zero between calls


# ------------------------------------------------------------------------ tables

def _tables_state(g, R, M, P, spare, longest, ended, idle, most_new):
    cap = M * P
    lens = np.minimum(g.integers(0, longest + 1, R), cap).astype(np.int32)
    add = g.integers(1, most_new + 1, R).astype(np.int32)
    add[g.random(R) < ended] = -1
    add[g.random(R) < idle] = 0
    have = -(-lens // P)
    N = max(int(have.sum()) + spare, 1)
    order = g.permutation(N).astype(np.int32)
    table = np.full((R, M), -7, np.int32)
    at = 0
    for r in range(R):
        table[r, :have[r]] = order[at:at + have[r]]
        at += have[r]
    taken = int(g.integers(0, 3 * N))
    ring = np.full(N, -9, np.int32)
    ring[(taken + np.arange(N - at)) % N] = order[at:]
    return lens, add, table, ring, np.array([taken, taken + N - at], np.int64)


def _run_tables(torch, lens, add, table, ring, pool, P, max_new, in_place=True, pad=0):
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    R, M = table.shape
    wide = torch.full((R, M + pad), -77, dtype=torch.int32, device=DEV)
    wide[:, :M] = d(table)
    t = binding.KvTables(R, M, len(ring), P, max_new, lens=d(lens), table=wide[:, :M], ring=d(ring), pool=d(pool))
    t.slots.fill_(-5)
    t.positions.fill_(-5)
    lo, po = (None, None) if in_place else (torch.empty_like(t.lens), torch.empty_like(t.pool))
    t.step(d(add), lens_out=lo, pool_out=po)
    torch.cuda.synchronize()
    if pad:
        assert bool((wide[:, M:] == -77).all())
    n = lambda x: x.cpu().numpy()  # noqa: E731
    if not in_place:
        assert np.array_equal(n(t.lens), lens) and np.array_equal(n(t.pool), pool)
    return dict(slots=n(t.slots), positions=n(t.positions), token_off=n(t.token_off), lens=n(t.lens if in_place else lo), table=n(t.table),
                ring=n(t.ring), pool=n(t.pool if in_place else po))


def _same(got, want):
    for name in want:
        assert np.array_equal(got[name], want[name]), name


@pytest.mark.parametrize("R,M,P,spare,longest,most_new,short", [
    (1, 1, 1, 1, 0, 1, 0), (1, 9, 16, 9, 100, 40, 0), (7, 40, 1, 200, 30, 5, 0), (64, 20, 16, 500, 300, 1, 0), (256, 64, 64, 2000, 4000, 1, 0),
    (300, 33, 8, 3000, 250, 60, 0), (1024, 8, 16, 5000, 100, 3, 0), (1025, 8, 16, 5000, 100, 3, 0), (1500, 64, 16, 30000, 900, 100, 0),
    (9001, 4, 32, 20000, 100, 20, 0), (20, 500, 65536, 100, 1 << 20, 70000, 0),
    # places or pages run out, rows are full
    (200, 16, 16, 50, 200, 60, 0), (200, 16, 16, 4000, 200, 60, 1500), (2000, 16, 16, 700, 200, 60, 0), (2000, 16, 16, 9000, 200, 60, 9000),
    (50, 4, 16, 0, 64, 30, 0)])
def test_tables_match_the_walk(torch_cuda, R, M, P, spare, longest, most_new, short):
    torch = torch_cuda
    print(f"tables R={R} M={M} P={P} spare={spare} longest={longest} most_new={most_new} short={short}", flush=True)
    g = np.random.default_rng(R * 7 + M)
    state = _tables_state(g, R, M, P, spare, longest, 0.1, 0.1, most_new)
    max_new = short or int(np.maximum(state[1], 0).sum()) + 3
    want = ref.tables(state[0], state[1], *state[2:], P, max_new)
    _same(_run_tables(torch, *state, P, max_new), want)
    _same(_run_tables(torch, *state, P, max_new, in_place=False, pad=3), want)


def test_tables_with_nothing_to_do(torch_cuda):
    torch = torch_cuda
    t = binding.KvTables(0, 4, 10, 16, 5)
    t.slots.fill_(3)
    t.step(torch.empty(0, dtype=torch.int32, device=DEV))
    assert t.slots.tolist() == [-1] * 5 and t.positions.tolist() == [-1] * 5 and t.token_off.tolist() == [0] and t.pool.tolist() == [0, 10]
    t = binding.KvTables(3, 4, 10, 16, 0)
    t.step(torch.tensor([1, 0, -1], dtype=torch.int32, device=DEV))       # no place for any token
    assert t.token_off.tolist() == [0, 0, 0, 0] and t.lens.tolist() == [0, 0, 0] and t.pool.tolist() == [0, 10]


@pytest.mark.parametrize("R", [40, 1100])
def test_tables_with_lengths_and_entries_nobody_wrote(torch_cuda, R):
    # lengths past either end count as the nearer end; entries that are no page give slot -1
    torch = torch_cuda
    g = np.random.default_rng(R)
    lens, add, table, ring, pool = _tables_state(g, R, 8, 16, 3000, 100, 0.0, 0.2, 9)
    lens[::7], lens[3::11] = -2 ** 31, 2 ** 31 - 1
    table[g.random(table.shape) < 0.2] = 2 ** 31 - 1
    table[g.random(table.shape) < 0.2] = -2 ** 31
    max_new = int(np.maximum(add, 0).sum())
    _same(_run_tables(torch, lens, add, table, ring, pool, 16, max_new), ref.tables(lens, add, table, ring, pool, 16, max_new))


@pytest.mark.parametrize("max_new", [64, 5000])
def test_tables_step_after_step(torch_cuda, max_new):
    # requests come and go over a pool that the pages go round many times; both ways of launching
    torch = torch_cuda
    g = np.random.default_rng(max_new)
    R, M, P, N = 24, 10, 8, 120
    t = binding.KvTables(R, M, N, P, max_new)
    state = dict(lens=np.zeros(R, np.int32), table=np.full((R, M), -1, np.int32), ring=np.arange(N, dtype=np.int32), pool=np.array([0, N], np.int64))
    for step in range(50):
        add = np.where(g.random(R) < 0.1, -1, g.integers(0, 12, R)).astype(np.int32)
        t.step(torch.from_numpy(add).to(DEV))
        want = ref.tables(state["lens"], add, state["table"], state["ring"], state["pool"], P, max_new)
        got = dict(slots=t.slots, positions=t.positions, token_off=t.token_off, lens=t.lens, table=t.table, ring=t.ring, pool=t.pool)
        _same({n: x.cpu().numpy() for n, x in got.items()}, want)
        state = {n: want[n] for n in state}


# ------------------------------------------------------------------------ writes

def _cache(torch, g, pages, H, P, dk, dv, fmt, latent=False, token_major=False, fill=float("nan")):
    td = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[fmt]

    def rows(d):
        shape = (pages, P, H, d) if token_major else (pages, H, P, d)
        x = torch.full(shape, fill, device=DEV).to(td)
        return x.transpose(1, 2) if token_major else x
    scales = lambda: torch.full((pages, H, P), fill, device=DEV) if fmt == "e4m3" else None  # noqa: E731
    return binding.KvCache(rows(dk), None if latent else rows(dv), scales(), None if latent else scales(), dv=dv)


def _bits(t):
    import torch
    return t.contiguous().view({4: torch.int32, 2: torch.int16, 1: torch.uint8}[t.element_size()])


@pytest.mark.parametrize("T,H,P,dk,dv,fmt,latent,token_major,fused", [
    (1, 1, 1, 8, 8, "bf16", False, False, False), (250, 8, 64, 128, 128, "bf16", False, False, True), (77, 3, 16, 80, 48, "bf16", False, True, True),
    (33, 1, 8, 576, 512, "bf16", True, False, False), (64, 2, 32, 64, 68, "f32", False, False, True), (1000, 4, 16, 128, 128, "e4m3", False, False, True),
    (9, 1, 16, 16, 64, "e4m3", False, False, False), (130, 2, 16, 96, 256, "e4m3", False, True, True), (50, 1, 64, 576, 512, "e4m3", True, False, False),
    (3, 5, 2, 256, 32, "e4m3", False, False, False)])
def test_append(torch_cuda, T, H, P, dk, dv, fmt, latent, token_major, fused):
    torch = torch_cuda
    print(f"append T={T} H={H} P={P} dk={dk} dv={dv} {fmt} latent={latent}", flush=True)
    g = np.random.default_rng(T + dk)
    pages = -(-2 * T // P) + 1
    c = _cache(torch, g, pages, H, P, dk, dv, fmt, latent, token_major)
    td = c.dtype
    new = lambda d: torch.from_numpy((g.standard_normal((T, H, d)) * np.exp(g.uniform(-8, 8, (T, H, 1)))).astype(np.float32)).to(DEV).to(td)  # noqa: E731
    k, v = new(dk), None if latent else new(dv)
    k[0, 0] = 0                                                    # a row of zeros
    if fused and not latent:
        both = torch.cat([k.reshape(T, -1), v.reshape(T, -1)], dim=1)
        both = torch.cat([both, torch.zeros((T, 8), dtype=td, device=DEV)], dim=1)
        k, v = both[:, :H * dk].view(T, H, dk), both[:, H * dk:H * (dk + dv)].view(T, H, dv)
    slots = g.permutation(pages * P)[:T].astype(np.int32)
    if T > 4:
        slots[1], slots[2], slots[3] = -1, pages * P, -2 ** 31      # skipped
    before = [None if x is None else x.clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]
    c.append(k, v, torch.from_numpy(slots).to(DEV))
    torch.cuda.synchronize()
    live = (slots >= 0) & (slots < pages * P)
    page, at = torch.from_numpy(slots[live] // P).to(DEV).long(), torch.from_numpy(slots[live] % P).to(DEV).long()
    for x, scale, rows, old, old_scale in ((c.k, c.k_scale, k, before[0], before[2]), (c.v, c.v_scale, v, before[1], before[3])):
        if x is None:
            continue
        want = _bits(old).clone()
        rows = rows[torch.from_numpy(live).to(DEV)]
        if fmt != "e4m3":
            want[page, :, at] = _bits(rows)
        else:
            codes, sc = oracle.quantize_e4m3(rows.float().cpu().numpy().reshape(-1, rows.shape[2]))
            want[page, :, at] = torch.from_numpy(codes).to(DEV).view(rows.shape)
            old_scale[page, :, at] = torch.from_numpy(sc).to(DEV).view(rows.shape[:2])
            assert torch.equal(_bits(scale), _bits(old_scale))
        assert torch.equal(_bits(x), want)


def test_append_of_nothing_and_of_padding_only(torch_cuda):
    torch = torch_cuda
    c = _cache(torch, None, 2, 1, 16, 64, 64, "bf16", fill=1.0)
    e = torch.empty((0, 1, 64), dtype=torch.bfloat16, device=DEV)
    c.append(e, e, torch.empty(0, dtype=torch.int32, device=DEV))
    x = torch.full((5, 1, 64), 2.0, dtype=torch.bfloat16, device=DEV)
    c.append(x, x, torch.full((5,), -1, dtype=torch.int32, device=DEV))
    assert bool((c.k == 1).all()) and bool((c.v == 1).all())


# --------------------------------------------------------------------- attention

class Setup:
    """A filled cache whose unused places hold NaN, lengths, tables and queries."""

    def __init__(self, torch, lens, Hq, H, dk, dv, P, fmt, latent=False, token_major=False, seed=0, peak=2.0, spare_columns=2):
        g = np.random.default_rng(seed)
        self.lens = np.asarray(lens, np.int64)
        R = len(self.lens)
        n_pages = -(-np.maximum(self.lens, 0) // P)
        M = int(n_pages.max()) + spare_columns if R else 1
        pages = int(n_pages.sum()) + 2
        order = g.permutation(pages)
        self.table = np.full((R, M), -1, np.int32)
        slots, at = [], 0
        for r in range(R):
            self.table[r, :n_pages[r]] = order[at:at + n_pages[r]]
            at += n_pages[r]
            i = np.arange(max(0, self.lens[r]))
            slots.append(self.table[r, i // P].astype(np.int64) * P + i % P)
        slots = np.concatenate(slots) if slots else np.zeros(0, np.int64)
        self.cache = _cache(torch, g, pages, H, P, dk, dv, fmt, latent, token_major)
        td = self.cache.dtype
        gen = torch.Generator(device=DEV).manual_seed(seed)
        new = lambda d: torch.randn((len(slots), H, d), generator=gen, device=DEV).to(td)  # noqa: E731
        self.cache.append(new(dk), None if latent else new(dv), torch.from_numpy(slots.astype(np.int32)).to(DEV))
        self.q = (torch.randn((R, Hq, dk), generator=gen, device=DEV) * peak).to(td)
        self.scale = dk ** -0.5
        self.d_lens = torch.from_numpy(self.lens.astype(np.int32)).to(DEV)
        self.d_table = torch.from_numpy(self.table).to(DEV)

    def call(self, window=0, want_lse=True, q=None):
        c = self.cache
        q = self.q if q is None else q
        self.attn = binding.DecodeAttention(c, q.shape[0], q.shape[1], self.table.shape[1], scale=self.scale, window=window, want_lse=want_lse)
        self.attn.workspace[COUNTERS:] = 0xff           # whatever was left there
        self.attn.out.fill_(float("nan"))
        return self.attn(q, self.d_lens, self.d_table)

    def want(self, window=0):
        c = self.cache
        return ref.attention(self.q, c.k, c.v, c.k_scale, c.v_scale, self.lens, self.d_table, self.scale, window, c.dv)


def _check(torch, s, window=0):
    out = s.call(window)
    torch.cuda.synchronize()
    assert not bool(s.attn.workspace[:COUNTERS].any())
    want, lse, bound, lse_bound = s.want(window)
    err = (out.double().cpu() - want).abs()
    assert torch.isfinite(out.float()).all()
    assert bool((err <= bound).all()), f"largest error {err.max():.3e}, over its bound by {(err / bound.clamp(min=1e-300)).max():.3f}"
    got = s.attn.lse.double().cpu()
    empty = torch.isneginf(lse)
    assert torch.equal(torch.isneginf(got), empty)
    assert bool(((got - lse).abs()[~empty] <= lse_bound[~empty]).all())


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, -5]


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("P", [1, 2, 8, 16, 32, 64, 512])
def test_attention_lengths_at_the_edges(torch_cuda, fmt, P):
    print(f"attention edges {fmt} P={P}", flush=True)
    _check(torch_cuda, Setup(torch_cuda, EDGES, 8, 2, 64, 64, P, fmt, seed=P))


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("dk,dv", [(16, 16), (32, 64), (64, 32), (80, 80), (96, 96), (112, 48), (128, 128), (192, 128), (128, 192), (256, 256), (208, 16)])
def test_attention_row_sizes(torch_cuda, fmt, dk, dv):
    print(f"attention rows {fmt} {dk} {dv}", flush=True)
    for P in (4, 16):
        _check(torch_cuda, Setup(torch_cuda, [0, 5, 100, 333], 6, 3, dk, dv, P, fmt, seed=dk))


@pytest.mark.parametrize("fmt,dk,dv", [("f32", 4, 8), ("f32", 60, 100), ("bf16", 8, 8), ("bf16", 72, 24), ("bf16", 8, 256)])
def test_attention_smallest_row_units(torch_cuda, fmt, dk, dv):
    _check(torch_cuda, Setup(torch_cuda, [1, 50, 200], 4, 2, dk, dv, 16, fmt, seed=dk))


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("group", [1, 2, 3, 7, 8, 15, 16, 17, 31, 33, 71])
def test_attention_heads_that_share_a_key(torch_cuda, fmt, group):
    print(f"attention group {fmt} {group}", flush=True)
    _check(torch_cuda, Setup(torch_cuda, [0, 70, 1000], 2 * group, 2, 128, 128, 32, fmt, seed=group))


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("Hq,dk,dv", [(1, 576, 512), (5, 576, 512), (16, 576, 512), (40, 576, 512), (128, 576, 512), (64, 320, 256), (16, 64, 32), (130, 272, 272)])
def test_attention_latent_rows(torch_cuda, fmt, Hq, dk, dv):
    for P in (8, 16, 64):
        print(f"attention latent {fmt} Hq={Hq} {dk} {dv} P={P}", flush=True)
        _check(torch_cuda, Setup(torch_cuda, [0, 1, 33, 64, 65, 500, 1111], Hq, 1, dk, dv, P, fmt, latent=True, seed=Hq + P))


def test_attention_latent_rows_of_several_heads(torch_cuda):
    for fmt in ("f32", "bf16", "e4m3"):
        _check(torch_cuda, Setup(torch_cuda, [3, 200, 97], 60, 3, 576, 512, 16, fmt, latent=True, token_major=True))


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("window", [1, 5, 16, 31, 32, 33, 100, 4096])
def test_attention_window(torch_cuda, fmt, window):
    print(f"attention window {fmt} {window}", flush=True)
    for P in (4, 16, 64):
        _check(torch_cuda, Setup(torch_cuda, [0, 1, 31, 33, 100, 333, 1000], 8, 2, 64, 64, P, fmt, seed=window), window)
    _check(torch_cuda, Setup(torch_cuda, [0, 1, 31, 33, 100, 333, 1000], 20, 1, 576, 512, 16, fmt, latent=True, seed=window), window)


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("R,lens,H,Hq,dk,latent", [
    (1, 40000, 1, 4, 128, False), (3, 9000, 2, 8, 64, False), (2, 17000, 1, 4, 256, False), (1, 20000, 1, 20, 576, True),
    (700, 60, 2, 4, 64, False), (1300, 3, 1, 2, 128, False), (300, 40, 1, 3, 576, True)])
def test_attention_long_and_many(torch_cuda, fmt, R, lens, H, Hq, dk, latent):
    print(f"attention R={R} lens={lens} {fmt} dk={dk}", flush=True)
    g = np.random.default_rng(R)
    ls = np.maximum(0, lens - g.integers(0, max(2, lens // 2), R))
    _check(torch_cuda, Setup(torch_cuda, ls, Hq, H, dk, 512 if latent else dk, 16, fmt, latent=latent, seed=R))


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
def test_attention_of_a_ragged_batch(torch_cuda, fmt):
    ls = [0] * 20 + [1] * 50 + [12000, 1, 0, 300, 7000] + [40] * 30
    _check(torch_cuda, Setup(torch_cuda, ls, 12, 2, 128, 128, 16, fmt, token_major=True))


@pytest.mark.parametrize("P", [4, 16, 64])
@pytest.mark.parametrize("latent", [False, True])
def test_attention_leaves_out_what_has_no_page(torch_cuda, P, latent):
    torch = torch_cuda
    for fmt in ("f32", "bf16", "e4m3"):
        print(f"attention bad pages P={P} latent={latent} {fmt}", flush=True)
        s = Setup(torch, [40, 64, 300, 64, 3], 4, 1, 576 if latent else 64, 512 if latent else 64, P, fmt, latent=latent)
        g = np.random.default_rng(P)
        bad = g.choice(np.array([-1, -2 ** 31, 2 ** 31 - 1, s.cache.pages], dtype=np.int64), s.table.shape)
        s.table = np.where(g.random(s.table.shape) < 0.3, bad, s.table).astype(np.int32)
        s.table[3] = -1                                             # nothing left of this one
        s.d_table = torch.from_numpy(s.table).to(DEV)
        _check(torch, s)


def test_attention_length_past_the_table(torch_cuda):
    torch = torch_cuda
    s = Setup(torch, [64, 100, 128], 4, 2, 64, 64, 16, "bf16", spare_columns=0)
    s.lens[2] = 2 ** 31 - 1
    s.d_lens = torch.from_numpy(s.lens.astype(np.int32)).to(DEV)
    _check(torch, s)


def test_attention_large_scores_and_far_apart(torch_cuda):
    # a maximum that grows at the very end of each request, scores hundreds apart
    torch = torch_cuda
    for fmt in ("f32", "bf16", "e4m3"):
        s = Setup(torch, [500, 1000, 3000], 4, 1, 64, 64, 16, fmt, peak=60.0)
        _check(torch, s)


def test_attention_infinities_in_masked_places(torch_cuda):
    # rows behind the last token: the type's lowest value, infinities, NaN
    torch = torch_cuda
    for fill in (float("inf"), float("-inf"), -3.0e38):
        s = Setup(torch, [5, 40, 129], 4, 2, 64, 64, 64, "bf16")
        used = torch.zeros((s.cache.pages, s.cache.page_size), dtype=torch.bool, device=DEV)
        for r, n in enumerate(s.lens):
            i = np.arange(n)
            used[torch.from_numpy(s.table[r, i // 64]).long().to(DEV), torch.from_numpy(i % 64).to(DEV)] = True
        for x in (s.cache.k, s.cache.v):
            x.copy_(torch.where(used[:, None, :, None], x, torch.full_like(x, fill)))
        _check(torch, s)


def test_attention_query_strides_and_other_outputs(torch_cuda):
    torch = torch_cuda
    s = Setup(torch, [100, 5, 0, 700], 8, 2, 64, 64, 16, "bf16")
    base = s.call().clone()
    wide = torch.full((4, 8 * 64 + 72), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 8:8 + 512] = s.q.reshape(4, 512)
    assert torch.equal(s.call(q=wide[:, 8:8 + 512].view(4, 8, 64)), base)
    heads = torch.full((8, 4, 80), float("nan"), dtype=torch.bfloat16, device=DEV)
    heads[:, :, :64] = s.q.transpose(0, 1)
    assert torch.equal(s.call(q=heads.transpose(0, 1)[:, :, :64]), base)
    assert torch.equal(s.call(want_lse=False), base)


def test_attention_is_the_same_every_time(torch_cuda):
    torch = torch_cuda
    for latent in (False, True):
        s = Setup(torch, [30000, 1, 500, 0, 9000], 16, 1, 576 if latent else 128, 512 if latent else 128, 16, "bf16", latent=latent)
        first = s.call().clone()
        for _ in range(5):
            assert torch.equal(s.attn(s.q, s.d_lens, s.d_table), first)


def test_attention_rows_that_overlap(torch_cuda):
    # a row starts inside the one before: the last rows of a page end behind 16 (or page_size) strides
    torch = torch_cuda
    pages, P, d, step = 3, 16, 64, 24
    g = torch.Generator(device=DEV).manual_seed(9)
    store = torch.randn(pages * 500, generator=g, device=DEV).bfloat16()
    k = torch.as_strided(store, (pages, 1, P, d), (496, 496, step, 1))
    table = torch.tensor([[1, 0, 2]], dtype=torch.int32, device=DEV)
    q = torch.randn((1, 4, d), generator=g, device=DEV).bfloat16()
    out = binding.DecodeAttention(binding.KvCache(k, k), 1, 4, 3)(q, torch.tensor([47], dtype=torch.int32, device=DEV), table)
    want, _, bound, _ = ref.attention(q, k, k, None, None, [47], table, d ** -0.5)
    assert bool(((out.double().cpu() - want).abs() <= bound).all())


def test_attention_places_beyond_4_gib(torch_cuda):
    # pages farther apart than 32-bit offsets reach; the rows in use are at both ends
    torch = torch_cuda
    pages, H, P, d = 3, 1, 16, 64
    gap = (3 << 30) // 2                                             # elements between pages: 3 GiB
    store = torch.zeros(2 * gap + H * P * d, dtype=torch.bfloat16, device=DEV)
    k = torch.as_strided(store, (pages, H, P, d), (gap, P * d, d, 1))
    c = binding.KvCache(k, k)
    g = torch.Generator(device=DEV).manual_seed(1)
    rows = torch.randn((40, 1, 64), generator=g, device=DEV).bfloat16()
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV)
    i = torch.arange(40, device=DEV)
    c.append(rows, rows, (table[0].long()[i // P] * P + i % P).to(torch.int32))
    q = torch.randn((1, 4, 64), generator=g, device=DEV).bfloat16()
    out = binding.DecodeAttention(c, 1, 4, 3)(q, torch.tensor([40], dtype=torch.int32, device=DEV), table)
    near = torch.stack([k[p].cpu() for p in range(3)])
    want, _, bound, _ = ref.attention(q, near, near, None, None, [40], table, 64 ** -0.5)
    assert bool(((out.double().cpu() - want).abs() <= bound).all())


def test_attention_no_requests(torch_cuda):
    torch = torch_cuda
    c = _cache(torch, None, 2, 1, 16, 64, 64, "bf16")
    out = binding.DecodeAttention(c, 0, 4, 3)(torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV),
                                              torch.empty(0, dtype=torch.int32, device=DEV), torch.empty((0, 3), dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert out.shape == (0, 4, 64)


# -------------------------------------------------------------- graphs and streams

def test_a_step_in_a_graph_and_on_another_stream(torch_cuda):
    """Tables, writes and attention of a growing batch, recorded once and replayed, against eager steps."""
    torch = torch_cuda
    R, Hq, H, d, P, M, steps = 5, 8, 2, 64, 16, 8, 7
    g = torch.Generator(device=DEV).manual_seed(11)
    add = torch.tensor([1, 1, 0, 1, 1], dtype=torch.int32, device=DEV)
    inputs = [tuple(torch.randn((R, n, d), generator=g, device=DEV).bfloat16() for n in (Hq, H, H)) for _ in range(steps)]

    def make():
        cache = binding.KvCache.allocate(R * M, P, H, d)
        tables = binding.KvTables(R, M, R * M, P, R)
        attn = binding.DecodeAttention(cache, R, Hq, M)
        first = binding.KvTables(R, M, R * M, P, 64, lens=tables.lens, table=tables.table, ring=tables.ring, pool=tables.pool)
        # prompts of 15 tokens: the first step is the last place of a page, the second needs a new one
        first.step(torch.full((R,), 12, dtype=torch.int32, device=DEV))
        gg = torch.Generator(device=DEV).manual_seed(12)
        rows = torch.randn((64, H, d), generator=gg, device=DEV).bfloat16()
        cache.append(rows, rows, first.slots)
        return cache, tables, attn

    def step(cache, tables, attn, q, k, v):
        tables.step(add)
        cache.append(k, v, tables.slots)
        return attn(q, tables.lens, tables.table)

    eager = make()
    want = [step(*eager, *x).clone() for x in inputs]
    torch.cuda.synchronize()
    # another stream than the one the tensors were made on
    side = torch.cuda.Stream()
    other = make()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [step(*other, *x).clone() for x in inputs]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # a graph, replayed with eager work and synchronisation in between
    c, t, a = make()
    q, k, v = (x.clone() for x in inputs[0])
    keep = t.lens.clone(), t.table.clone(), t.ring.clone(), t.pool.clone(), c.k.clone(), c.v.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(c, t, a, q, k, v)
    for dst, src in zip((t.lens, t.table, t.ring, t.pool, c.k, c.v), keep):
        dst.copy_(src)
    for i, x in enumerate(inputs):
        for dst, src in zip((q, k, v), x):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i]), i
        assert step(*make(), *inputs[0]).equal(want[0])
    assert torch.equal(t.lens, eager[1].lens) and torch.equal(t.table, eager[1].table)
