"""Decode attention where its work is cut: contexts so long that items are cut among many workgroups, runs so long that
table entries are renewed on the way, both ways in which the parts of latent rows are joined.  Caches and bounds of
unit_marks: a unit that is lost, doubled or read from another page shows in full."""
import numpy as np
import pytest

from paper_2603_28768_amd import binding

import unit_marks as marks

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
COUNTERS = 48 << 10


class Marked:
    """A cache of unit_marks' rows; unused places hold NaN.  bad: share of table entries that are no page."""

    def __init__(self, torch, lens, H, group, dk, dv, P, fmt, latent=False, seed=0, bad=0.0, token_major=False):
        g = np.random.default_rng(seed)
        self.lens, self.H, self.group, self.dk, self.dv, self.P, self.fmt = [int(n) for n in lens], H, group, dk, dv, P, fmt
        R = len(lens)
        have = [-(-max(0, n) // P) for n in self.lens]
        M, pages = max(have) + 1, sum(have) + 2
        order = g.permutation(pages)
        table = np.full((R, M), -1, np.int32)
        at = 0
        for r in range(R):
            table[r, :have[r]] = order[at:at + have[r]]
            at += have[r]
        td = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[fmt]
        raw = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.uint8}[fmt]      # what is written by index
        code = lambda x: x.to(td).view(raw)  # noqa: E731

        def rows(d):
            shape = (pages, P, H, d) if token_major else (pages, H, P, d)
            x = code(torch.full((1,), float("nan"), device=DEV)).expand(shape).contiguous()
            return x.transpose(1, 2) if token_major else x
        k = rows(dk)
        v = None if latent else rows(dv)
        for r, n in enumerate(self.lens):
            if n <= 0:
                continue
            i = torch.arange(n, device=DEV)
            page, place = torch.from_numpy(table[r]).to(DEV).long()[i // P], i % P
            u = i // marks.UNIT
            k[page, :, place] = 0
            if v is not None:
                v[page, :, place] = 0
            for h in range(H):
                c = marks.column(u, r, h, dv)
                (k if latent else v)[page, h, place, c] = code(marks.value(u, dv).float())
                k[page, h, place, dk - 1] = code(marks.score(c).float())
        ones = lambda: torch.ones((pages, H, P), device=DEV) if fmt == "e4m3" else None  # noqa: E731
        self.cache = binding.KvCache(k.view(td), None if v is None else v.view(td), ones(), None if latent else ones(), dv=dv)
        if bad:
            no_page = g.choice(np.array([-1, -2 ** 31, 2 ** 31 - 1, pages], dtype=np.int64), table.shape)
            table = np.where(g.random(table.shape) < bad, no_page, table).astype(np.int32)
        self.there = [((0 <= table[r]) & (table[r] < pages))[np.arange(max(0, n)) // P] for r, n in enumerate(self.lens)]
        self.table = torch.from_numpy(table).to(DEV)
        self.d_lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.q = torch.zeros((R, H * group, dk), dtype=self.cache.dtype, device=DEV)
        self.q[:, 1::2, dk - 1] = 1
        self.handle = None

    def call(self, window=0):
        if self.handle is None:
            self.handle = binding.DecodeAttention(self.cache, len(self.lens), self.H * self.group, self.table.shape[1], scale=marks.SCALE,
                                                  window=window, want_lse=True)
            self.handle.workspace[COUNTERS:] = 0xff
        self.handle.out.fill_(float("nan"))
        return self.handle(self.q, self.d_lens, self.table)

    def check(self, units, window=0):
        out, lse = self.handle.out.double().cpu().numpy(), self.handle.lse.double().cpu().numpy()
        want, want_lse = marks.expected(self.lens, self.H, self.group, self.dv, window, self.there)
        wrong = marks.rejected(out, lse, want, want_lse, self.cache.dtype, units)
        assert not wrong, wrong
        assert not bool(self.handle.workspace[:COUNTERS].any())


def _cus(torch):
    return torch.cuda.get_device_properties(0).multi_processor_count


def _ordinary(torch, lens, H, group, d, P, fmt, window=0, at_least_groups=0, at_least_pages=0, **kw):
    print(f"ordinary rows: {len(lens)} requests up to {max(lens)}, {H} x {group} heads of {d}, pages of {P}, {fmt}, window {window}", flush=True)
    runs = marks.ordinary_runs(lens, fmt, H, group, d, d, P, _cus(torch), window)
    assert marks.most_workgroups(runs, 4) >= at_least_groups and marks.most_pages(runs, lens, P, window) >= at_least_pages
    s = Marked(torch, lens, H, group, d, d, P, fmt, seed=len(lens) + P, **kw)
    s.call(window)
    s.check(marks.most_units(runs), window)


def _latent(torch, lens, H, group, P, fmt, dk=576, dv=512, at_least_pages=0, places=None, window=0, **kw):
    """places: "item" or "run", which has a place among the cuts."""
    print(f"latent rows: {len(lens)} requests up to {max(lens)}, {H} x {group} heads, {dk} and {dv}, pages of {P}, {fmt}", flush=True)
    runs, workers = marks.latent_runs(lens, H, group, _cus(torch), window)
    assert marks.most_pages(runs, lens, P, window) >= at_least_pages
    assert places is None or (len(lens) * H <= workers) == (places == "item")
    s = Marked(torch, lens, H, group, dk, dv, P, fmt, latent=True, seed=len(lens) + P, **kw)
    s.call(window)
    s.check(marks.most_units(runs), window)
    return runs


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("lens,H,group,d,P,groups", [
    ([30537], 1, 4, 128, 16, 100), ([131071], 1, 2, 128, 64, 200), ([40000], 1, 16, 64, 16, 100), ([17000, 9001], 1, 4, 256, 16, 60),
    ([9000, 1, 8000, 0, 12345], 2, 3, 128, 32, 17), ([20000, 33], 1, 40, 128, 4, 17), ([50001], 1, 2, 80, 1, 100), ([100, 70000, 3], 1, 17, 192, 64, 17)])
def test_items_cut_among_many_workgroups(torch_cuda, fmt, lens, H, group, d, P, groups):
    _ordinary(torch_cuda, lens, H, group, d, P, fmt, at_least_groups=groups)


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("window", [20000, 33000])
def test_long_windows(torch_cuda, fmt, window):
    _ordinary(torch_cuda, [50000, 20000, 20001, 7], 1, 4, 128, 16, fmt, window, at_least_groups=17)


def test_a_ragged_batch_of_long_and_short(torch_cuda):
    g = np.random.default_rng(4)
    lens = np.r_[np.zeros(20), np.ones(40), [60000, 12000], g.integers(1, 4000, 200)].astype(int)
    for fmt in ("f32", "bf16", "e4m3"):
        _ordinary(torch_cuda, g.permutation(lens).tolist(), 2, 5, 64, 16, fmt)


@pytest.mark.parametrize("bad", [0.0, 0.2])
@pytest.mark.parametrize("R,lens,H,d,P,fmt,pages", [(16, 14000, 8, 128, 16, "bf16", 100), (12, 30000, 8, 128, 32, "bf16", 80), (16, 14000, 8, 256, 16, "e4m3", 100),
                                                    (9, 20000, 8, 128, 16, "f32", 80), (3, 90000, 8, 256, 16, "bf16", 120), (2, 1100000, 1, 128, 16, "bf16", 130)])
def test_runs_over_more_pages_than_are_held(torch_cuda, R, lens, H, d, P, fmt, pages, bad):
    # a wave holds 64 entries of a table and the 64 behind them
    _ordinary(torch_cuda, [lens - 37 * r for r in range(R)], H, 2, d, P, fmt, at_least_pages=pages, bad=bad)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("bad", [0.0, 0.2])
@pytest.mark.parametrize("lens,group,P,pages", [([70001], 5, 1, 200), ([90000, 100, 45000], 16, 2, 200), ([200000], 3, 4, 190), ([60000] * 5 + [33, 0], 2, 16, 65),
                                                ([280000, 290001], 66, 16, 200), ([330000], 2, 8, 140)])
def test_latent_runs_over_more_pages_than_are_held(torch_cuda, fmt, lens, group, P, pages, bad):
    _latent(torch_cuda, lens, 1, group, P, fmt, at_least_pages=pages, places="item", bad=bad)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("R,longest,H,group,P,places", [
    (150, 3000, 1, 128, 16, "run"), (300, 1500, 1, 130, 64, "run"), (200, 2500, 1, 100, 16, "run"), (60, 4000, 3, 128, 16, "run"), (130, 2500, 2, 67, 4, "run"),
    (300, 2000, 1, 16, 32, "run"), (70, 3000, 1, 130, 16, "item"), (20, 5000, 3, 128, 16, "item"), (128, 2500, 1, 128, 64, "item"), (256, 900, 1, 64, 16, "item")])
def test_latent_parts_with_a_place_for_every_item_or_run(torch_cuda, fmt, R, longest, H, group, P, places):
    g = np.random.default_rng(R + group)
    lens = g.integers(1, longest + 1, R)
    lens[::17] = 0
    lens[5::31] = 1
    lens[R // 2] = 12 * longest
    runs = _latent(torch_cuda, lens.tolist(), H, group, P, fmt, places=places)
    # many items are cut, and some of them more than once
    assert marks.most_workgroups(runs, 1) >= 3
    cut = {}
    for run in runs:
        for r, item, _, _ in run:
            cut[r, item] = cut.get((r, item), 0) + 1
    assert sum(n > 1 for n in cut.values()) >= 20


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("dk,dv", [(272, 256), (320, 64), (576, 16), (400, 384)])
def test_latent_rows_of_other_lengths(torch_cuda, fmt, dk, dv):
    _latent(torch_cuda, [30000, 1, 0, 800], 1, 7, 16, fmt, dk, dv)
    _latent(torch_cuda, [30000, 1, 0, 800], 1, 7, 4, fmt, dk, dv, window=9000)


@pytest.mark.parametrize("latent", [False, True])
@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3"])
def test_where_the_rows_lie_does_not_change_the_result(torch_cuda, fmt, latent):
    """The same rows over pages of other sizes and in another order: the same bits, among pages of 16 tokens and more and
    among smaller ones (which may have other runs).  Scores that round, so that the order of the sums shows."""
    torch = torch_cuda
    lens, H, group = [700, 1, 0, 5000, 12001], 1, 6
    dk, dv = (576, 512) if latent else (128, 128)
    td = torch.float32 if fmt == "f32" else torch.bfloat16
    gen = torch.Generator(device=DEV).manual_seed(5)
    k, v, q = (torch.randn((n, h, d), generator=gen, device=DEV).to(td) for n, h, d in
               ((sum(lens), H, dk), (sum(lens), H, dv), (len(lens), H * group, dk)))

    def run(P, seed, token_major):
        have = [-(-n // P) for n in lens]
        pages, M = sum(have) + 3, max(have)
        order = torch.from_numpy(np.random.default_rng(seed).permutation(pages))
        table = torch.full((len(lens), M), -1, dtype=torch.int64)
        at, slots = 0, []
        for r, n in enumerate(lens):
            table[r, :have[r]] = order[at:at + have[r]]
            at += have[r]
            i = torch.arange(n)
            slots.append(table[r, i // P] * P + i % P)
        code = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[fmt]

        def rows(d):
            x = torch.zeros((pages, P, H, d) if token_major else (pages, H, P, d), device=DEV).to(code)
            return x.transpose(1, 2) if token_major else x
        ones = lambda: torch.ones((pages, H, P), device=DEV) if fmt == "e4m3" else None  # noqa: E731
        c = binding.KvCache(rows(dk), None if latent else rows(dv), ones(), None if latent else ones(), dv=dv)
        c.append(k, None if latent else v, torch.cat(slots).to(DEV, torch.int32))
        a = binding.DecodeAttention(c, len(lens), H * group, M, want_lse=True)
        a(q, torch.tensor(lens, dtype=torch.int32, device=DEV), table.to(DEV, torch.int32))
        return a.out.clone(), a.lse.clone()
    for sizes in ((16, 32, 64, 1024), (8, 1, 4)):
        first = run(sizes[0], 0, False)
        for i, P in enumerate(sizes):
            again = run(P, i + 1, i % 2 == 1)
            assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1]), P


def test_calls_of_all_shapes_share_a_workspace(torch_cuda):
    torch = torch_cuda
    shapes = [([30537], 1, 4, 128, 128, 16, "bf16", False), ([5000, 300, 0, 7], 1, 70, 576, 512, 16, "e4m3", True), ([3, 40, 200], 2, 2, 64, 64, 4, "f32", False),
              ([20000, 900], 1, 3, 576, 512, 64, "bf16", True), ([700] * 300, 1, 130, 576, 512, 32, "bf16", True), ([9000, 100], 2, 33, 256, 256, 16, "e4m3", False),
              ([2000, 9000], 1, 3, 576, 512, 16, "f32", True), ([1], 1, 1, 80, 80, 64, "bf16", False)]
    all_of = []
    for i, (lens, H, group, dk, dv, P, fmt, latent) in enumerate(shapes):
        s = Marked(torch, lens, H, group, dk, dv, P, fmt, latent=latent, seed=i)
        s.call()
        all_of.append((s, s.handle.out.clone(), s.handle.lse.clone()))
    shared = torch.full((max(s.handle.workspace.numel() for s, _, _ in all_of),), 0xff, dtype=torch.uint8, device=DEV)
    shared[:COUNTERS] = 0
    for s, _, _ in all_of:
        s.handle.args.workspace, s.handle.args.workspace_bytes, s.handle.workspace = shared.data_ptr(), shared.numel(), shared
    g = np.random.default_rng(1)
    for _ in range(3):
        for i in g.permutation(len(all_of)):
            s, out, lse = all_of[i]
            print("shared workspace, shape", i, flush=True)
            s.handle.lse.fill_(float("nan"))
            s.call()
            assert torch.equal(s.handle.out, out) and torch.equal(s.handle.lse, lse)
            assert not bool(shared[:COUNTERS].any())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("R,longest,group", [(6, 9000, 20), (150, 1500, 128)])
def test_latent_steps_in_a_graph_and_on_another_stream(torch_cuda, fmt, R, longest, group):
    """Both launches of latent rows recorded once and replayed over other lengths and pages, with eager calls in between; and
    on another stream."""
    torch = torch_cuda
    g = np.random.default_rng(R)
    s = Marked(torch, g.integers(0, longest + 1, R).tolist(), 1, group, 576, 512, 16, fmt, latent=True, seed=R)
    most = [int(x) for x in s.lens]
    steps = [most, [x // 3 for x in most], [0 if i % 2 else x for i, x in enumerate(most)], [min(x, 1) for x in most], most]
    units = marks.most_units(marks.latent_runs(most, 1, group, _cus(torch))[0])
    s.call()
    other = binding.DecodeAttention(s.cache, R, group, s.table.shape[1], scale=marks.SCALE, want_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other(s.q, s.d_lens, s.table)                                # also the warm-up of the recording
    torch.cuda.synchronize()
    assert torch.equal(other.out, s.handle.out) and torch.equal(other.lse, s.handle.lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other(s.q, s.d_lens, s.table)
    for i, lens in enumerate(steps):
        print("replay", i, flush=True)
        s.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        s.lens = lens
        s.there = [np.ones(n, bool) for n in lens]
        other.out.fill_(float("nan"))
        other.lse.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        s.call()                                                      # eager work between the replays
        torch.cuda.synchronize()
        assert torch.equal(other.out, s.handle.out) and torch.equal(other.lse, s.handle.lse), i
        s.check(units)
        if i == 0:
            continue
        graph.replay()                                                # and a replay right behind another
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(other.out, s.handle.out), i
