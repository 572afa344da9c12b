"""Products of 8-bit integers, their quantisation and products grouped by expert, on the GPU against plain forms on the host
(product_reference.py says what is compared bit for bit and what within which bound)."""
import numpy as np
import pytest

import oracle
from paper_2603_28768_amd import binding, synth

from cases import Case
import product_reference as ref
import product_shapes as shapes

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


# ---------------------------------------------------------------------- quantize

def _hard_rows(g, rows, K):
    """Rows of every size a float has: ties, powers of two, zeros, rows near both ends of the range."""
    x = g.standard_normal((rows, K)).astype(np.float32)
    kind = np.arange(rows) % 8
    x[kind == 1] *= np.float32(1e-38)
    x[kind == 2] *= np.float32(1e37)
    x[kind == 3] = 0.0
    # whole and half multiples of the scale: ties of the rounding
    x[kind == 4] = np.rint(x[kind == 4] * 60).clip(-127, 127) * np.float32(0.5)
    x[kind == 4, 0] = 127.0
    x[kind == 5] *= np.float32(2.0 ** -140)
    x[kind == 6, 1:] = 0.0
    x[kind == 7] = np.ldexp(np.float32(1.0), g.integers(-120, 100, (int((kind == 7).sum()), 1))).astype(np.float32) * x[kind == 7]
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,K,pad", [(1, 16, 0), (17, 48, 16), (40, 256, 0), (33, 272, 0), (9, 1040, 8), (250, 4096, 4096), (16, 6160, 0),
                                        (8, 7168, 0), (16, 8192, 32), (24, 8208, 0), (8, 40000, 0), (3001, 64, 0)])
def test_quantize_is_the_definition(torch_cuda, dtype, rows, K, pad):
    torch = torch_cuda
    print(f"quantize {dtype} {rows}x{K}+{pad}", flush=True)
    x = _dev(_hard_rows(np.random.default_rng(rows + K), rows, K + pad)).to(binding._torch_dtype(dtype))[:, :K]
    codes, scale = binding.quantize_i8(x)
    want_codes, want_scale = ref.quantize(x.float().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), want_scale)
    assert np.array_equal(codes.cpu().numpy(), want_codes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [16, 512, 7168, 16384])
def test_quantize_marks_rows_that_are_not_finite(torch_cuda, dtype, K):
    torch = torch_cuda
    x = torch.randn((7, K), device=DEV).to(binding._torch_dtype(dtype))
    x[1, 3], x[2, K - 1], x[3, 0], x[5, K // 2] = float("inf"), float("nan"), float("-inf"), float("-nan")
    codes, scale = binding.quantize_i8(x)
    want_codes, want_scale = ref.quantize(x.float().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), want_scale, equal_nan=True) and np.isnan(want_scale).sum() == 4
    assert np.array_equal(codes.cpu().numpy(), want_codes)


# ------------------------------------------------------------------------ matmul

def _codes(g, rows, K, most=127):
    return g.integers(-most, most + 1, (rows, K)).astype(np.int8), np.exp(g.uniform(-9, 3, rows)).astype(np.float32)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 16), (1, 64, 64), (1, 7168, 4096), (2, 17, 144), (16, 16, 128), (17, 33, 2064), (31, 5, 48), (61, 4099, 272), (64, 257, 1040), (65, 200, 512),
    (128, 130, 8192), (129, 512, 112), (250, 1000, 640), (256, 256, 256), (257, 511, 400), (777, 300, 1552), (1025, 1537, 2048), (3000, 70, 96), (40, 40, 131056)])
def test_matmul_is_exact(torch_cuda, out, M, N, K):
    torch = torch_cuda
    print(f"matmul {M}x{N}x{K} {out}", flush=True)
    g = np.random.default_rng(M * 31 + N)
    (x, xs), (w, ws) = _codes(g, M, K), _codes(g, N, K)
    got = binding.matmul_i8(_dev(x), _dev(xs), _dev(w), _dev(ws), dtype=out)
    want = _dev(ref.product(x, w, xs, ws)[0]).to(got.dtype)
    assert torch.equal(got, want)


def test_matmul_at_the_ends_of_the_integers(torch_cuda):
    # the longest contraction of the largest codes stays inside 32 bits, with either sign
    torch = torch_cuda
    K = 131056
    x = np.full((20, K), -128, np.int8)
    x[1::2] = 127
    w = np.full((18, K), -128, np.int8)
    w[::3] = 127
    one = np.ones(20, np.float32)
    got = binding.matmul_i8(_dev(x), _dev(one), _dev(w), _dev(one[:18]), dtype="f32")
    assert torch.equal(got.cpu(), torch.from_numpy(ref.product(x, w, one, one[:18])[0]))


@pytest.mark.parametrize("M,N,K,pad,out_pad,out", [(37, 70, 208, 48, 1, "bf16"), (300, 257, 512, 16, 3, "f32"), (600, 96, 1024, 512, 32, "bf16"), (1, 50, 64, 0, 7, "f32")])
def test_matmul_of_views(torch_cuda, M, N, K, pad, out_pad, out):
    torch = torch_cuda
    g = np.random.default_rng(M)
    (x, xs), (w, ws) = _codes(g, M, K), _codes(g, N, K)
    wide = torch.full((M, K + pad), 99, dtype=torch.int8, device=DEV)
    wide[:, :K] = _dev(x)
    room = torch.full((M + 2, N + out_pad), -7.0, dtype=binding._torch_dtype(out), device=DEV)
    view = room[1:M + 1, :N]
    assert binding.matmul_i8(wide[:, :K], _dev(xs), _dev(w), _dev(ws), out=view) is view
    assert torch.equal(view, _dev(ref.product(x, w, xs, ws)[0]).to(view.dtype))
    room[1:M + 1, :N] = -7.0
    assert bool((room == -7.0).all())


def test_matmul_shows_a_row_that_was_not_finite(torch_cuda):
    torch = torch_cuda
    x = torch.randn((70, 512), device=DEV)
    x[3, 5], x[66, 0] = float("inf"), float("nan")
    got = binding.matmul_i8(*binding.quantize_i8(x), *binding.quantize_i8(torch.randn((300, 512), device=DEV)))
    bad = got.isnan().all(dim=1)
    assert bad.nonzero().flatten().tolist() == [3, 66] and not bool(got[~bad].isnan().any())


def test_no_rows_is_no_work(torch_cuda):
    torch = torch_cuda
    w, ws = torch.zeros((4, 32), dtype=torch.int8, device=DEV), torch.ones(4, device=DEV)
    assert binding.matmul_i8(torch.zeros((0, 32), dtype=torch.int8, device=DEV), ws[:0], w, ws).shape == (0, 4)
    assert binding.quantize_i8(torch.zeros((0, 32), device=DEV))[0].shape == (0, 32)
    off = torch.zeros(2, dtype=torch.int32, device=DEV)
    assert binding.GroupedMatmul(torch.zeros((1, 4, 32), device=DEV))(torch.zeros((0, 32), device=DEV), off).shape == (0, 4)


# ----------------------------------------------------------------------- grouped

class Problem:
    """Operands of a grouped product on the host and on the GPU."""

    def __init__(self, seed, fmt, sizes, N, K, is_gated, out="bf16", k=0, front=0, spare=0, whole=False, pad=0, out_pad=0):
        import torch
        g = np.random.default_rng(seed)
        self.fmt, self.N, self.K, self.k, self.gated = fmt, N, K, k, is_gated
        self.off = np.concatenate([[front], front + np.cumsum(sizes)]).astype(np.int32)
        self.M = int(self.off[-1]) + spare
        self.G = len(sizes)
        rows = self.M if k == 0 else max(1, self.M // 2)
        self.src = g.integers(0, rows * k, self.M).astype(np.int32) if k else None
        self.xs = self.ws = self.us = None
        self.out_dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[out if fmt == "i8" else fmt]
        if fmt == "i8":
            self.x, self.xs = _codes(g, rows, K)
            self.xs *= np.float32(K ** -0.5 / 2000)
            mats = [_codes(g, N, K) for _ in range(2 * self.G)]
            self.w, self.ws = np.stack([m[0] for m in mats[:self.G]]), np.stack([m[1] for m in mats[:self.G]])
            self.u, self.us = np.stack([m[0] for m in mats[self.G:]]), np.stack([m[1] for m in mats[self.G:]])
        else:
            # small whole numbers: sums of up to 2^14 products of at most 2^6 are exact in fp32
            make = (lambda *s: g.integers(-8, 9, s).astype(np.float32)) if whole else lambda *s: g.standard_normal(s).astype(np.float32)
            kind = binding._torch_dtype(fmt)
            stored = lambda a: torch.from_numpy(a).to(kind).float().numpy()  # noqa: E731
            scale = np.float32(1.0 if whole else K ** -0.5)
            self.x, self.w, self.u = stored(make(rows, K)), stored(make(self.G, N, K) * scale), stored(make(self.G, N, K) * scale)
        t = (lambda a: _dev(a)) if fmt == "i8" else (lambda a: _dev(a).to(binding._torch_dtype(fmt)))  # noqa: E731
        wide = torch.zeros((rows, K + pad), dtype=torch.int8 if fmt == "i8" else binding._torch_dtype(fmt), device=DEV)
        wide[:, :K] = t(self.x)
        self.d_x = wide[:, :K]
        self.d_w, self.d_u = t(self.w), t(self.u) if is_gated else None
        self.d_xs = None if self.xs is None else _dev(self.xs)
        self.d_off, self.d_src = _dev(self.off), None if self.src is None else _dev(self.src)
        s = lambda a: None if a is None else _dev(a)  # noqa: E731
        self.handle = binding.GroupedMatmul(self.d_w, scales=s(self.ws), up=self.d_u, up_scales=s(self.us) if is_gated else None,
                                            dtype=out if fmt == "i8" else None)
        self.room = torch.full((self.M, N + out_pad), -7.0, dtype=self.out_dtype, device=DEV)
        self.out = self.room[:, :N]

    def run(self, **kw):
        args = dict(x_scale=self.d_xs, src=self.d_src, k=max(self.k, 1), out=self.out)
        args.update(kw)
        return self.handle(self.d_x, self.d_off, **args)

    def check(self, got, off=None):
        """Rows of groups within their bounds (equal where nothing is gated and sums are exact), others untouched."""
        import torch
        got = got.cpu()
        off = self.off if off is None else off
        seen = np.zeros(self.M, bool)
        rows = self.x.shape[0]
        for g, lo, hi in ref.rows_of(None, off, self.M):
            seen[lo:hi] = True
            token = np.arange(lo, hi) if self.src is None else np.where(self.src[lo:hi] >= 0, self.src[lo:hi] // max(self.k, 1), -1)
            live = (token >= 0) & (token < rows)
            at = np.where(live, token, 0)
            xs = None if self.xs is None else self.xs[at]
            a, ea = ref.product(self.x[at], self.w[g], xs, None if self.ws is None else self.ws[g])
            mine = got[lo:hi]
            assert bool((mine[torch.from_numpy(~live)] == 0).all())
            if self.gated:
                b, eb = ref.product(self.x[at], self.u[g], xs, None if self.us is None else self.us[g])
                a, bound = ref.gated(a, ea, b, eb, self.out_dtype)
            elif ea is not None:
                bound = ea + np.abs(a) * ref.U[self.out_dtype]
            if not self.gated and (ea is None or self.exact):
                want = torch.from_numpy(np.ascontiguousarray(a)).float().to(self.out_dtype)
                assert torch.equal(mine[torch.from_numpy(live)], want[torch.from_numpy(live)]), g
            else:
                off_by = np.abs(mine.double().numpy() - a)[live]
                assert bool((off_by <= bound[live]).all()), (g, float((off_by / bound[live]).max()))
        rest = torch.from_numpy(~seen)
        assert bool((got[rest] == -7.0).all())
        assert bool((self.room[:, self.N:] == -7.0).all())

    exact = False


SIZES = [[1], [0, 1, 0], [3, 0, 16, 17, 1], [64, 65, 0, 31], [255, 0, 256, 257, 1], [700, 5, 90], [0] * 40 + [33] + [0] * 25 + [2], [2] * 130]


@pytest.mark.parametrize("fmt,out", [("i8", "bf16"), ("i8", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("is_gated", [False, True])
@pytest.mark.parametrize("which", range(len(SIZES)))
def test_grouped_rows(torch_cuda, fmt, out, is_gated, which):
    sizes = SIZES[which]
    for N, K, k in ((48, 128, 0), (131, 272, 2), (300, 1040 if fmt != "f32" else 100, 8)):
        print(f"grouped {fmt} {out} gated={is_gated} sizes={sizes[:6]} N={N} K={K} k={k}", flush=True)
        p = Problem(which * 7 + N, fmt, sizes, N, K, is_gated, out=out, k=k, front=which % 3, spare=which % 4, whole=not is_gated)
        p.exact = True
        p.check(p.run())


@pytest.mark.parametrize("fmt,out", [("i8", "bf16"), ("i8", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("is_gated", [False, True])
@pytest.mark.parametrize("sizes,N,K,pad,out_pad", [([300, 17, 0, 520], 520, 1168, 32, 5), ([40, 1000], 257, 2000, 16, 0), ([5, 9, 2, 30], 1000, 4112, 0, 8)])
def test_grouped_drawn_values(torch_cuda, fmt, out, is_gated, sizes, N, K, pad, out_pad):
    if fmt == "f32":
        K = K // 4 // 4 * 4
    print(f"grouped drawn {fmt} {out} gated={is_gated} {sizes} N={N} K={K}", flush=True)
    p = Problem(N, fmt, sizes, N, K, is_gated, out=out, k=3, spare=2, pad=pad, out_pad=out_pad)
    p.check(p.run())


# a tile of every height, the lowest ones of groups with few rows among them; the sum is about one round of tiles
HEIGHTS = [256, 200, 180, 150, 100, 70, 64, 33, 20, 5, 0, 512, 700, 900, 110]


@pytest.mark.parametrize("fmt,out", [("i8", "bf16"), ("i8", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("is_gated,N", [(False, 4096 + 5), (True, 2048 - 3)])
@pytest.mark.parametrize("K", [128, 592])
def test_tiles_of_every_height(torch_cuda, fmt, out, is_gated, N, K):
    print(f"heights {fmt} {out} gated={is_gated} N={N} K={K}", flush=True)
    p = Problem(N + K, fmt, HEIGHTS, N, K, is_gated, out=out, k=2, front=3, spare=7, whole=not is_gated, pad=16, out_pad=3)
    p.exact = True
    p.src[5::37] = -1
    p.src[6::41] = p.x.shape[0] * 2
    p.d_src = _dev(p.src)
    p.check(p.run())


@pytest.mark.parametrize("M,N,K", [(5121, 2048, 256), (2689, 4000, 144), (777, 4096, 1040), (1345, 1100, 2048), (641, 8192, 400), (400, 2500, 3000 // 16 * 16)])
def test_matmul_in_tiles(torch_cuda, M, N, K):
    # last tiles of one row, of half a fragment; rows that end inside a slab
    torch = torch_cuda
    print(f"matmul tiles {M}x{N}x{K}", flush=True)
    g = np.random.default_rng(M)
    (x, xs), (w, ws) = _codes(g, M, K), _codes(g, N, K)
    got = binding.matmul_i8(_dev(x), _dev(xs), _dev(w), _dev(ws), dtype="bf16")
    assert torch.equal(got, _dev(ref.product(x, w, xs, ws)[0]).bfloat16())


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("G,most", [(70, 90), (200, 30), (1024, 9), (130, 300)])
def test_many_groups(torch_cuda, fmt, G, most):
    # more groups than a wave has lanes, in tiles and in units
    g = np.random.default_rng(G)
    sizes = g.integers(0, most, G).tolist()
    K = 64 if fmt == "f32" else 128
    for N in (40, 520 if G < 1000 else 72):
        print(f"many groups {fmt} G={G} most={most} N={N}", flush=True)
        p = Problem(G, fmt, sizes, N, K, False, out="bf16", whole=True, spare=1)
        p.exact = True
        p.check(p.run())


@pytest.mark.parametrize("fmt", ["i8", "bf16"])
def test_rows_behind_an_offset_of_32_bits(torch_cuda, fmt):
    """Rows of x further from its start than 32 bits of bytes, in order and through a permutation: strides far beyond the rows."""
    torch = torch_cuda
    K, rows, N = 256, 300, 48
    kind = torch.int8 if fmt == "i8" else torch.bfloat16
    stride = (16 << 20) + 256 if fmt == "i8" else (8 << 20) + 128          # elements: a row every 16 MiB
    room = torch.empty(rows * stride, dtype=kind, device=DEV)
    x = room.as_strided((rows, K), (stride, 1))
    g = np.random.default_rng(1)
    x.copy_(_dev(g.integers(-8, 9, (rows, K)).astype(np.float32)).to(kind))
    w = _dev(g.integers(-8, 9, (2, N, K)).astype(np.float32)).to(kind)
    one = lambda *s: torch.ones(s, device=DEV) if fmt == "i8" else None  # noqa: E731
    op = binding.GroupedMatmul(w, scales=one(2, N))
    off = torch.tensor([0, 200, 300], dtype=torch.int32, device=DEV)
    want = torch.cat([x[:200].float() @ w[0].float().T, x[200:].float() @ w[1].float().T]).bfloat16()
    assert torch.equal(op(x, off, x_scale=one(rows)), want)
    src = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device=DEV)
    back = x.flip(0).float()
    want = torch.cat([back[:200] @ w[0].float().T, back[200:] @ w[1].float().T]).bfloat16()
    assert torch.equal(op(x, off, x_scale=one(rows), src=src), want)


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("off", [[5, 2, 9, 9], [-4, 30, 20, 1000], [40, 60, 80, 33], [90, 95, 95, 2000000000], [-2000000000, 0, 0, 0]])
def test_offsets_that_are_none_stay_inside(torch_cuda, fmt, off):
    torch = torch_cuda
    print(f"offsets {fmt} {off}", flush=True)
    p = Problem(3, fmt, [20, 30, 27], 72, 320, False, out="bf16", whole=True, spare=3)
    p.exact = True
    off = np.asarray(off, np.int32)
    got = p.handle(p.d_x, _dev(off), x_scale=p.d_xs, out=p.out)
    covered = [r for g, lo, hi in ref.rows_of(None, off, p.M) for r in range(lo, hi)]
    if len(set(covered)) == len(covered):
        p.check(got, off)


# (rows, columns, offsets): far more rows in all the groups than there are places, tall tiles, few rows and more groups than a
# wave has lanes among them; every last group has rows of its own
FALLING = [(8192, 2048, [0, 4096] * 7 + [0, 8192]), (5000, 2050, [500, 4900] * 4 + [0, 40]), (9000, 1030, [300, 8800] * 50 + [0, 9000])]


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("is_gated", [False, True])
@pytest.mark.parametrize("which", range(len(FALLING)))
def test_groups_that_overlap_lose_no_rows(torch_cuda, fmt, is_gated, which):
    """Rows that several groups have get any of their results, rows of one group its own."""
    torch = torch_cuda
    M, N, off = FALLING[which]
    G = len(off) - 1
    print(f"overlap {fmt} gated={is_gated} M={M} N={N} G={G}", flush=True)
    p = Problem(31, fmt, [0] * (G - 1) + [M], N, 64 if fmt == "f32" else 256, is_gated, whole=True, out="bf16")
    p.exact = True
    off = np.asarray(off, np.int32)
    got = p.handle(p.d_x, _dev(off), x_scale=p.d_xs, out=p.out).clone()
    fits = torch.zeros((M, N), dtype=torch.bool, device=DEV)
    covered = np.zeros(M, bool)
    for g, lo, hi in ref.rows_of(None, off, M):
        covered[lo:hi] = True
        alone = np.asarray([lo] * (g + 1) + [hi] * (G - g), np.int32)
        one = p.handle(p.d_x, _dev(alone), x_scale=p.d_xs, out=p.out.fill_(-7.0))
        fits[lo:hi] |= one[lo:hi] == got[lo:hi]
    p.check(one, alone)                            # the last group
    rows = torch.from_numpy(covered).to(DEV)
    lost = (rows & ~fits.all(dim=1)).nonzero().flatten().tolist()
    assert not lost, (len(lost), lost[0], lost[-1])
    assert bool((got[~rows] == -7.0).all())


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("is_gated", [False, True])
@pytest.mark.parametrize("rows", [20, 300])
def test_places_that_name_no_row_are_zeros(torch_cuda, fmt, is_gated, rows):
    p = Problem(5, fmt, [rows, 7, rows], 100, 144, is_gated, k=4, whole=True, out="f32")
    p.exact = True
    p.src[::3] = -1
    p.src[1::5] = p.x.shape[0] * 4
    p.src[2::7] = 2 ** 31 - 1
    p.d_src = _dev(p.src)
    p.check(p.run())


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,N", [(9, 90), (300, 90), (1500, 2100)])
def test_infinities_and_nan_stay_in_their_rows(torch_cuda, fmt, rows, N):
    # the last pieces of rows that end inside a slab: what is read in place of the rest may hold anything
    torch = torch_cuda
    K = 208 if fmt == "bf16" else 100
    p = Problem(11, fmt, [rows, 40 + rows // 2], N, K, False, whole=True)
    x = p.d_x.clone().abs() + 1
    w = p.d_w.clone().abs() + 1
    x[2, K - 1], x[rows + 5, K - 8], x[4, 0] = float("inf"), float("nan"), float("-inf")
    w[1, 7, K - 1] = float("inf")
    got = binding.GroupedMatmul(w)(x, p.d_off).float().cpu()
    want = torch.full((p.M, N), 0.0)
    want[2], want[4], want[rows + 5] = float("inf"), float("-inf"), float("nan")
    want[rows:, 7] = float("inf")
    want[rows + 5] = float("nan")
    odd = ~torch.isfinite(got)
    assert torch.equal(odd, ~torch.isfinite(want))
    assert torch.equal(got[odd].nan_to_num(7.0, 8.0, 9.0), want[odd].nan_to_num(7.0, 8.0, 9.0))


def test_one_matrix_in_several_places(torch_cuda):
    # copies of an expert share its weights
    torch = torch_cuda
    p = Problem(8, "i8", [30, 70, 5], 64, 256, False, out="f32")
    one = binding.GroupedMatmul([p.d_w[0], p.d_w[0], p.d_w[2]], scales=[_dev(p.ws[0]), _dev(p.ws[0]), _dev(p.ws[2])], dtype="f32")
    p.w[1], p.ws[1] = p.w[0], p.ws[0]
    p.check(one(p.d_x, p.d_off, x_scale=p.d_xs, out=p.out))


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("is_gated", [False, True])
def test_recorded_calls_follow_their_inputs(torch_cuda, fmt, is_gated):
    # offsets, rows and activations change between replays; eager calls of the same handle in between
    torch = torch_cuda
    p = Problem(21, fmt, [200, 3, 0, 300, 40], 136, 528, is_gated, k=2, spare=9, out="bf16")
    other = torch.empty_like(p.out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    g = np.random.default_rng(5)
    for sizes in ([1, 1, 1, 1, 1], [0, 0, 543, 0, 0], [100, 100, 100, 100, 100], [200, 3, 0, 300, 40]):
        p.off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        p.src = g.integers(0, p.x.shape[0] * 2, p.M).astype(np.int32)
        p.d_off.copy_(_dev(p.off))
        p.d_src.copy_(_dev(p.src))
        p.out.fill_(-7.0)
        graph.replay()
        p.check(p.out)
        again = p.run(out=other.fill_(-7.0))
        torch.cuda.synchronize()
        assert torch.equal(again, p.out)


def test_calls_on_a_stream_of_their_own(torch_cuda):
    torch = torch_cuda
    p = Problem(2, "i8", [90, 400, 11], 200, 512, True, out="bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = p.run(stream=side)
    x, xs = binding.quantize_i8(torch.ones((5, 64), device=DEV), stream=side)
    y = binding.matmul_i8(x, xs, x, xs, dtype="f32", stream=side)
    side.synchronize()
    p.check(got)
    assert torch.equal(x, torch.full_like(x, 127)) and bool((y - 64.0).abs().max() <= 64 * 6 * 2.0 ** -24)


@pytest.mark.parametrize("T,H,I,E,k", [(40, 256, 208, 6, 2), (700, 512, 400, 5, 3)])
def test_expert_layer_in_8_bits(torch_cuda, T, H, I, E, k):
    """A run of the operators together: quantize, gate and up by expert, quantize, down by expert; against the same steps in
    64 bits on the codes' values.  What separates the two: the gated product's rounding to bf16 and its own bound carry over
    into codes, off by at most one and then by one scale."""
    torch = torch_cuda
    g = np.random.default_rng(T)
    x = _dev(g.standard_normal((T, H)).astype(np.float32)).bfloat16()
    weights = {n: binding.quantize_i8(_dev((g.standard_normal((E * r, c)) * c ** -0.5).astype(np.float32)))
               for n, r, c in (("gate", I, H), ("up", I, H), ("down", H, I))}
    shaped = {n: (c.view(E, -1, c.shape[1]), s.view(E, -1)) for n, (c, s) in weights.items()}
    ids = np.stack([g.choice(E, k, replace=False) for _ in range(T)]).reshape(-1)
    src = np.argsort(ids, kind="stable").astype(np.int32)
    off = np.concatenate([[0], np.cumsum(np.bincount(ids, minlength=E))]).astype(np.int32)
    first = binding.GroupedMatmul(shaped["gate"][0], scales=shaped["gate"][1], up=shaped["up"][0], up_scales=shaped["up"][1])
    second = binding.GroupedMatmul(shaped["down"][0], scales=shaped["down"][1], dtype="f32")
    xq, xs = binding.quantize_i8(x)
    h = first(xq, _dev(off), x_scale=xs, src=_dev(src), k=k)
    hq, hs = binding.quantize_i8(h)
    y = second(hq, _dev(off), x_scale=hs).cpu().double().numpy()
    val = {n: (c.double() * s.double()[..., None]).cpu().numpy() for n, (c, s) in shaped.items()}
    xv = (xq.double() * xs.double()[:, None]).cpu().numpy()[src // k]
    scale = hs.cpu().double().numpy()
    for e in range(E):
        r = slice(off[e], off[e + 1])
        a, b = xv[r] @ val["gate"][e].T, xv[r] @ val["up"][e].T
        hv = a / (1 + np.exp(-a)) * b
        # codes: half a scale from h, h a bf16 rounding (2^-8) from hv
        bound = (0.5 + 2.0 ** -7) * scale[r, None] + np.abs(hv) * 2.0 ** -7
        off_by = np.abs(y[r] - hv @ val["down"][e].T)
        assert (off_by <= bound @ np.abs(val["down"][e]).T + 1e-5 * np.abs(y[r])).all()


# ------------------------------------------------------- products in tiles (test_product_choice.py: that they are)

@pytest.mark.parametrize("fmt,out", [("i8", "bf16"), ("i8", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("is_gated,which", [(gated, i) for gated in (False, True) for i in range(len(shapes.SHAPES[gated]))])
def test_every_tile(torch_cuda, fmt, out, is_gated, which):
    s = shapes.SHAPES[is_gated][which]
    K = shapes.elements(fmt, s.row_bytes)
    print(f"tiles {fmt} {out} gated={is_gated} {s.width}x{s.height} N={s.N} K={K}", flush=True)
    p = Problem(which + K, fmt, s.sizes, s.N, K, is_gated, out=out, k=2, front=shapes.FRONT, spare=shapes.SPARE, whole=not is_gated,
                pad=shapes.elements(fmt, 32), out_pad=which % 2)
    p.exact = True
    p.check(p.run())


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("is_gated", [False, True])
def test_recorded_calls_in_tiles(torch_cuda, fmt, is_gated):
    # what a replay has to find by itself: rows of each group, other rows of x, groups that overlap and do not any more
    torch = torch_cuda
    G, M, N, row_bytes = shapes.CHANGING
    p = Problem(23, fmt, [700, 3, 0, 1300, 190], N, shapes.elements(fmt, row_bytes), is_gated, k=2, spare=M - 2193, out="bf16", whole=not is_gated)
    assert p.M == M and p.G == G
    p.exact = True
    other = torch.empty_like(p.out)
    p.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    g = np.random.default_rng(6)
    for off in ([0, 1, 2, 3, 4, 5], [0, 0, 0, 2193, 2193, 2200], [300, 300, 740, 1180, 1620, 2060], [0, 2200, 0, 2200, 0, 2200], [0, 700, 703, 703, 2003, 2193]):
        p.off = np.asarray(off, np.int32)
        p.src = g.integers(0, p.x.shape[0] * 2, M).astype(np.int32)
        p.src[::50] = -1
        p.d_off.copy_(_dev(p.off))
        p.d_src.copy_(_dev(p.src))
        fill = -7.0 if off[2] >= off[1] else float("nan")
        p.out.fill_(fill)
        graph.replay()
        again = p.run(out=other.fill_(fill))
        torch.cuda.synchronize()
        if off[2] >= off[1]:
            p.check(p.out)
            assert torch.equal(again, p.out)
        else:
            # every place is in three groups
            assert not bool(p.out.isnan().any()) and not bool(again.isnan().any())


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("is_gated", [False, True])
@pytest.mark.parametrize("off", [[5, 2, 1500, 1500, 2150, 2150], [-4, 700, 700, 1500, 2000, 2 ** 31 - 1], [1500, 1900, 20, 800, 800, 33],
                                 [2190, 2195, 2195, 2 ** 31 - 1, 2 ** 31 - 1, 0], [-2 ** 31, 0, 0, 0, -1, 0], [-2 ** 31, 2 ** 31 - 1, 2 ** 31 - 1, -2 ** 31, -5, -5]])
def test_offsets_that_are_none_in_tiles(torch_cuda, fmt, is_gated, off):
    G, M, N, row_bytes = shapes.CHANGING
    print(f"offsets in tiles {fmt} gated={is_gated} {off}", flush=True)
    p = Problem(9, fmt, [0] * (G - 1) + [M], N, shapes.elements(fmt, row_bytes), is_gated, out="bf16", whole=not is_gated)
    p.exact = True
    off = np.asarray(off, np.int32)
    p.check(p.handle(p.d_x, _dev(off), x_scale=p.d_xs, out=p.out), off)


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("gathered", [False, True])
def test_tiles_of_rows_up_to_32_bits_apart(torch_cuda, fmt, gathered):
    """Offsets of rows, from the start of x or of a tile, between 2^31 and 2^32."""
    torch = torch_cuda
    rows, stride, places, N = shapes.FAR_GATHERED if gathered else shapes.FAR_IN_ORDER
    K, step = shapes.elements(fmt, shapes.FAR_BYTES), shapes.elements(fmt, stride)
    print(f"far rows {fmt} gathered={gathered} {rows} x {stride}", flush=True)
    kind = {"i8": torch.int8, "bf16": torch.bfloat16, "f32": torch.float32}[fmt]
    x = torch.empty((rows - 1) * step + K, dtype=kind, device=DEV).as_strided((rows, K), (step, 1))
    g = np.random.default_rng(12)
    x.copy_(_dev(g.integers(-8, 9, (rows, K)).astype(np.float32)).to(kind))
    G = 2 if gathered else 1
    w = _dev(g.integers(-8, 9, (G, N, K)).astype(np.float32)).to(kind)
    one = lambda *s: torch.ones(s, device=DEV) if fmt == "i8" else None  # noqa: E731
    cuts = [0, 301, places] if gathered else [0, places]
    at = np.concatenate([g.integers(0, rows, places - 2), [rows - 1, rows - 2]]).astype(np.int64) if gathered else np.arange(places)
    got = binding.GroupedMatmul(w, scales=one(G, N), dtype="f32" if fmt == "i8" else None)(
        x, _dev(np.asarray(cuts, np.int32)), x_scale=one(rows), src=_dev(at.astype(np.int32)) if gathered else None)
    near = x[_dev(at)].float()
    for e, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
        # sums of 256 products of at most 64: exact in fp32
        assert torch.equal(got[lo:hi], (near[lo:hi] @ w[e].float().T).to(got.dtype)), e


# ------------------------------------------------------- quantisation: a width for every number of units and lanes a row

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,K,pad", [(8200, 272, 16), (8200, 512, 0), (8195, 528, 0), (8193, 768, 0), (8193, 1040, 32), (8193, 1536, 0), (9000, 800, 0), (9, 1552, 0),
                                        (9, 2560, 0), (9, 5120, 64), (9, 6144, 0), (9, 12288, 0), (9, 20000, 0), (9, 32768, 0), (9, 32784, 0)])
def test_quantize_rows_of_every_width(torch_cuda, dtype, rows, K, pad):
    torch = torch_cuda
    print(f"quantize width {dtype} {rows}x{K}+{pad}", flush=True)
    x = _dev(_hard_rows(np.random.default_rng(rows + K), rows, K + pad)).to(binding._torch_dtype(dtype))[:, :K]
    # the largest element of one row and one that is not finite in another, both in the last unit
    x[1] = 0.25
    x[1, K - 1] = -3.0
    x[rows - 1, K - 2] = float("nan")
    x[rows - 2, K - 16] = float("-inf")
    room = torch.full((rows + 2, K), 77, dtype=torch.int8, device=DEV)
    scale_room = torch.full((rows + 2,), 77.0, device=DEV)
    codes, scale = binding.quantize_i8(x, codes=room[1:rows + 1], scale=scale_room[1:rows + 1])
    want_codes, want_scale = ref.quantize(x.float().cpu().numpy())
    assert np.isnan(want_scale).sum() == 2 and want_codes[1, K - 1] == -127
    assert np.array_equal(scale.cpu().numpy(), want_scale, equal_nan=True)
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    assert bool((room[::rows + 1] == 77).all()) and bool((scale_room[::rows + 1] == 77.0).all())


# ------------------------------------------------------- behind the framework's own dispatch

@pytest.mark.parametrize("T", [48, 1500])
def test_layers_on_the_dispatch_of_the_forward(torch_cuda, T):
    """src and slot_off as the rank forward leaves them: T k places, of which one rank's are somewhere in the middle.  In bf16 the
    layer is the forward's own, held to the oracle's as that is; in 8 bits it equals the one on the rank's rows alone.  Then both
    recorded behind the forward, replayed on other scores."""
    torch = torch_cuda
    cfg = synth.scaled(synth.CONFIGS["qwen3"], T=T, H=512, I=384, E=32, k=4, D=4, replica_slots=3, zipf_s=1.2, profile_batches=2)
    case = Case(cfg)
    rank = max(range(1, 3), key=lambda r: case.rows[r])            # places in front of its own and behind
    fwd, x, logits = case.gpu_rank(rank)
    first_slot, end_slot = (int(v) for v in case.rank_slot_off[rank:rank + 2])
    src, off = fwd.debug["src"], fwd.debug["slot_off"][first_slot:end_slot + 1]
    wg, wu, wd = fwd._weights
    q = [[binding.quantize_i8(w) for w in ws] for ws in (wg, wu, wd)]
    codes, scales = [[c for c, _ in m] for m in q], [[s for _, s in m] for m in q]
    first, second = binding.GroupedMatmul(wg, up=wu), binding.GroupedMatmul(wd)
    first8 = binding.GroupedMatmul(codes[0], scales=scales[0], up=codes[1], up_scales=scales[1])
    second8 = binding.GroupedMatmul(codes[2], scales=scales[2], dtype="f32")
    places = T * cfg.k
    make = lambda n, kind: torch.full((places, n), -7.0, dtype=kind, device=DEV)  # noqa: E731
    h, y, h8, y8 = make(cfg.I, torch.bfloat16), make(cfg.H, torch.bfloat16), make(cfg.I, torch.bfloat16), make(cfg.H, torch.float32)

    def step():
        fwd(x, logits)
        first(x, off, src=src, k=cfg.k, out=h)
        second(h, off, out=y)
        xq, xs = binding.quantize_i8(x)
        first8(xq, off, x_scale=xs, src=src, k=cfg.k, out=h8)
        hq, hs = binding.quantize_i8(h8)
        second8(hq, off, x_scale=hs, out=y8)

    def check():
        torch.cuda.synchronize()
        bounds = off.cpu().numpy()
        lo, hi = int(bounds[0]), int(bounds[-1])
        assert 0 < lo < hi < places
        mine = np.zeros(places, bool)
        mine[lo:hi] = True
        for t in (h, y, h8, y8):
            assert bool((t[_dev(~mine)] == -7.0).all()) and not bool((t[lo:hi] == -7.0).all(dim=1).any())
        ref_out = oracle.rank_forward(case.x, logits.cpu().numpy(), cfg.k, case.slot_expert, case.rank_slot_off, rank, case.weights_of, True, None)["out"]
        dest, weight = fwd.debug["dest"].cpu().numpy().reshape(T, cfg.k), fwd.debug["topk_w"].cpu().double().numpy()
        here = (dest >= lo) & (dest < hi)
        values = y.double().cpu().numpy()[np.where(here, dest, 0)]
        out = (values * np.where(here, weight, 0.0)[:, :, None]).sum(axis=1)
        assert np.abs(out - ref_out).max() <= 1e-2 * np.abs(ref_out).max()
        xq, xs = binding.quantize_i8(x)
        near = (off - lo).contiguous()
        one = first8(xq, near, x_scale=xs, src=src[lo:hi].contiguous(), k=cfg.k)
        hq, hs = binding.quantize_i8(one)
        assert torch.equal(one, h8[lo:hi]) and torch.equal(second8(hq, near, x_scale=hs), y8[lo:hi])

    step()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for shift in (1, 5):
        logits.copy_(logits.roll(shift, dims=1))
        for t in (h, y, h8, y8):
            t.fill_(-7.0)
        graph.replay()
        check()
