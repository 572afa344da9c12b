"""Which kernel and which tiles products take (csrc/product_choice.h), compiled for the host: the products that the GPU tests send
through tiles get there, and between them reach every tile that there is."""
import os
import subprocess

import pytest

import product_shapes as shapes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_28768_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

DRIVER = r"""
#include <cstdio>
#include "product_choice.h"
int main() {
    int format, G, N, row_bytes, gated, src;
    long long M, x_rows, x_stride;
    static const unsigned char *none = nullptr;
    static const int32_t place = 0;
    while (std::scanf("%d %d %lld %d %d %d %d %lld %lld", &format, &G, &M, &N, &row_bytes, &gated, &src, &x_rows, &x_stride) == 9) {
        craft::ProductArgs a{};
        a.format = format;
        a.G = G;
        a.M = M;
        a.N = N;
        a.row_bytes = row_bytes;
        a.up = gated ? &none : nullptr;
        a.src = src ? &place : nullptr;
        a.x_rows = x_rows;
        a.x_stride = x_stride;
        a.num_cu = 256;
        const craft::ProductChoice c = craft::product_choice(a);
        std::printf("%d %d\n", c.width, c.height);
    }
    return 0;
}
"""
FORMATS = {"f32": 0, "bf16": 1, "i8": 2}


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    at = tmp_path_factory.mktemp("choice")
    (at / "driver.cpp").write_text(DRIVER)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"),
                           "-I", CSRC, str(at / "driver.cpp"), "-o", str(at / "driver")])

    def choose(fmt, G, M, N, row_bytes, is_gated, src=False, x_rows=None, x_stride=None):
        line = f"{FORMATS[fmt]} {G} {M} {N} {row_bytes} {int(is_gated)} {int(src)} {x_rows or M} {x_stride or row_bytes}\n"
        out = subprocess.run([str(at / "driver")], input=line, capture_output=True, text=True, check=True).stdout
        return tuple(int(v) for v in out.split())
    return choose


def _of_shape(choose, fmt, is_gated, s):
    M = shapes.FRONT + sum(s.sizes) + shapes.SPARE
    return choose(fmt, len(s.sizes), M, s.N, s.row_bytes, is_gated, src=True, x_rows=M // 2, x_stride=s.row_bytes + 32)


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("is_gated", [False, True])
def test_shapes_reach_every_tile(choose, fmt, is_gated):
    reached = {}
    for s in shapes.SHAPES[is_gated]:
        got = _of_shape(choose, fmt, is_gated, s)
        if fmt != "f32":
            assert got == (s.width, s.height), s
        assert got[0], s
        for tile in shapes.tiles_of(s.sizes, *got):
            reached.setdefault(tile, set()).add(s.row_bytes)
    every = {(8, 8), (8, 7), (8, 6), (8, 5), (8, 4), (8, 2), (4, 4), (4, 2), (4, 1)}
    assert set(reached) == every
    if fmt != "f32":
        assert all(at == set(shapes.ROW_BYTES) for at in reached.values()), reached


@pytest.mark.parametrize("fmt", ["i8", "bf16", "f32"])
def test_changing_and_far_rows_go_through_tiles(choose, fmt):
    G, M, N, row_bytes = shapes.CHANGING
    for is_gated in (False, True):
        for src in (False, True):
            assert choose(fmt, G, M, N, row_bytes, is_gated, src=src, x_rows=M)[0]
    far = shapes.FAR_BYTES
    rows, stride, places, N = shapes.FAR_GATHERED
    assert 1 << 31 < (rows - 1) * stride < rows * stride < 1 << 32
    assert choose(fmt, 2, places, N, far, False, src=True, x_rows=rows, x_stride=stride)[0]
    # a row more, or a longer stride: units, whose addresses are of 64 bits
    assert choose(fmt, 2, places, N, far, False, src=True, x_rows=rows + 1, x_stride=stride) == (0, 0)
    rows, stride, places, N = shapes.FAR_IN_ORDER
    assert choose(fmt, 1, places, N, far, False, x_stride=stride) == (256, 256) and 255 * stride > 1 << 31
    assert choose(fmt, 1, places, N, far, False, x_stride=stride + 16) == (0, 0)
