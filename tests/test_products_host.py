"""What the products refuse, without a GPU: every call here ends in the argument checks."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_28768_amd import binding

import product_reference as ref

EINVAL = -1
AT = 1 << 40              # stands in for a device address; nothing is launched


def _quantize(**kw):
    a = dict(dtype=1, x=AT, x_stride=64, rows=4, K=64, codes=AT, scale=AT)
    a.update(kw)
    return binding.lib().craft_quantize_i8(a["dtype"], a["x"], a["x_stride"], a["rows"], a["K"], a["codes"], a["scale"], None)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 40), dict(K=0), dict(K=-16), dict(K=24), dict(x_stride=63), dict(x_stride=48), dict(x_stride=0),
    dict(x_stride=-64), dict(x_stride=68), dict(x_stride=1 << 62), dict(rows=1 << 39, x_stride=1 << 20), dict(x=0), dict(x=AT + 8), dict(codes=0),
    dict(codes=AT + 4), dict(scale=0), dict(scale=AT + 2)])
def test_quantize_refuses(bad):
    assert _quantize(**bad) == EINVAL


def _matmul(**kw):
    a = dict(M=4, N=8, K=64, x=AT, x_stride=64, x_scale=AT, w=AT, w_scale=AT, out_dtype=1, out=AT, out_stride=8)
    a.update(kw)
    return binding.lib().craft_matmul_i8(a["M"], a["N"], a["K"], a["x"], a["x_stride"], a["x_scale"], a["w"], a["w_scale"], a["out_dtype"], a["out"],
                                         a["out_stride"], None)


@pytest.mark.parametrize("bad", [
    dict(M=-1), dict(M=1 << 31), dict(N=0), dict(N=-3), dict(N=(1 << 30) + 1, out_stride=1 << 31), dict(K=0), dict(K=8), dict(K=72), dict(K=131072, x_stride=131072),
    dict(x=0), dict(x=AT + 8), dict(x_stride=48), dict(x_stride=72), dict(x_stride=-64), dict(x_stride=1 << 50), dict(M=1 << 30, x_stride=1 << 20), dict(x_scale=0),
    dict(x_scale=AT + 1), dict(w=0), dict(w=AT + 8), dict(w_scale=0), dict(w_scale=AT + 2), dict(out_dtype=2), dict(out_dtype=-1), dict(out=0), dict(out=AT + 1),
    dict(out_dtype=0, out=AT + 2), dict(out_stride=7), dict(out_stride=1 << 50)])
def test_matmul_refuses(bad):
    assert _matmul(**bad) == EINVAL


def _grouped(**kw):
    a = binding.GroupedMatmulArgs()
    plain = dict(format=2, out_dtype=1, G=3, N=8, K=64, k=2, M=4, x_rows=4, x=AT, x_stride=64, x_scale=AT, src=AT, off=AT, w=AT, w_up=AT, w_scale=AT, up_scale=AT,
                 out=AT, out_stride=8)
    plain.update(kw)
    for n, v in plain.items():
        setattr(a, n, v or None if n in ("x", "x_scale", "src", "off", "w", "w_up", "w_scale", "up_scale", "out") else v)
    return binding.lib().craft_grouped_matmul(ctypes.byref(a), None)


@pytest.mark.parametrize("bad", [
    dict(format=3), dict(format=-1), dict(out_dtype=2), dict(format=0, out_dtype=1), dict(format=1, out_dtype=0), dict(G=0), dict(G=-1), dict(G=1025), dict(N=0),
    dict(N=-1), dict(K=0), dict(K=56), dict(format=1, K=60), dict(format=0, out_dtype=0, K=62), dict(K=131072, x_stride=131072),
    dict(format=1, K=1 << 22, x_stride=1 << 22), dict(k=0), dict(k=-2), dict(M=-1), dict(M=1 << 31), dict(M=(1 << 26) + 1), dict(x_rows=-1), dict(x_rows=0), dict(x_rows=1 << 31),
    dict(x=0), dict(x=AT + 4), dict(x_stride=60), dict(x_stride=72), dict(x_stride=1 << 60), dict(x_scale=0), dict(x_scale=AT + 1), dict(src=AT + 1), dict(off=0),
    dict(off=AT + 2), dict(w=0), dict(w=AT + 4), dict(w_up=AT + 4), dict(w_scale=0), dict(w_scale=AT + 4), dict(up_scale=0), dict(up_scale=AT + 4), dict(out=0),
    dict(out=AT + 1), dict(out_stride=7), dict(out_stride=1 << 60)])
def test_grouped_refuses(bad):
    assert _grouped(**bad) == EINVAL


def test_no_rows_is_no_launch():
    assert _quantize(rows=0) == 0 and _matmul(M=0) == 0 and _grouped(M=0) == 0
    assert binding.lib().craft_grouped_matmul(None, None) == EINVAL


def test_plain_forms():
    """The reference itself: hand-made rows, a hand-made product."""
    x = np.array([[127.0, 0.5, 1.5, -2.5] + [0.0] * 12, [0.0] * 16, [np.inf] + [1.0] * 15], np.float32)
    codes, scale = ref.quantize(x)
    assert scale[0] == 1.0 and codes[0, :4].tolist() == [127, 0, 2, -2]
    assert scale[1] == 1.0 and not codes[1].any() and np.isnan(scale[2]) and not codes[2].any()
    got, _ = ref.product(np.array([[1, -2]], np.int8), np.array([[3, 4], [5, 6]], np.int8), np.array([2.0], np.float32), np.array([1.0, 0.5], np.float32))
    assert got.tolist() == [[-10.0, -7.0]]
    assert [r for r in ref.rows_of(None, [2, 5, 4, 99], 8)] == [(0, 2, 5), (2, 4, 8)]


class Placed:
    """What the binding asks of a tensor that is said to be on a GPU."""

    def __init__(self, shape, dtype, gpu=0):
        self.shape, self.dtype, self.gpu, self.is_cuda = torch.Size(shape), dtype, gpu, True

    def stride(self, dim=None):
        st = [1]
        for n in reversed(self.shape[1:]):
            st.insert(0, st[0] * n)
        return tuple(st) if dim is None else st[dim]

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return self.gpu

    def data_ptr(self):
        return AT

    def is_contiguous(self):
        return True


@pytest.mark.parametrize("which", ["x_scale", "w", "w_scale", "out"])
def test_matmul_refuses_tensors_of_another_gpu(which):
    t = dict(x=Placed((4, 64), torch.int8), x_scale=Placed((4,), torch.float32), w=Placed((8, 64), torch.int8), w_scale=Placed((8,), torch.float32),
             out=Placed((4, 8), torch.bfloat16))
    t[which].gpu = 1
    with pytest.raises(AssertionError):
        binding.matmul_i8(**t)


@pytest.mark.parametrize("codes,scale", [(Placed((4, 64), torch.int8, 1), None), (None, Placed((4,), torch.float32, 1)), (Placed((4, 63), torch.int8), None),
                                         (Placed((4, 64), torch.uint8), None), (None, Placed((5,), torch.float32))])
def test_quantize_refuses_other_outputs(codes, scale):
    own = dict(codes=codes or Placed((4, 64), torch.int8), scale=scale or Placed((4,), torch.float32))
    with pytest.raises(AssertionError):
        binding.quantize_i8(Placed((4, 64), torch.float32), **own)


class Wide(Placed):
    device = torch.device("cpu")


def _beyond_32_bits():
    i8, f32, bf16 = torch.int8, torch.float32, torch.bfloat16
    far = (1 << 32) + 64                           # 64 in the lower half
    s = Wide((4,), f32)
    yield "quantize K", lambda: binding.quantize_i8(Wide((4, far), f32), codes=Wide((4, far), i8), scale=s)
    yield "matmul K", lambda: binding.matmul_i8(Wide((4, far), i8), s, Wide((4, far), i8), s, out=Wide((4, 4), bf16))
    yield "matmul N", lambda: binding.matmul_i8(Wide((4, 64), i8), s, Wide((far, 64), i8), Wide((far,), f32), out=Wide((4, far), bf16))
    yield "grouped K", lambda: binding.GroupedMatmul([Wide((8, far), bf16)])
    yield "grouped N", lambda: binding.GroupedMatmul([Wide((far, 64), bf16)])
    one = binding.GroupedMatmul([Wide((8, 64), bf16)])
    for k in ((1 << 32) + 2, (1 << 31), -(1 << 32) + 2):
        yield f"grouped k {k}", lambda k=k: one(Wide((4, 64), bf16), Wide((2,), torch.int32), src=Wide((4,), torch.int32), k=k, out=Wide((4, 8), bf16))


@pytest.mark.parametrize("which", range(8))
def test_sizes_beyond_32_bits_are_refused(which):
    # the library's sizes are 32-bit integers: a larger one would arrive as its lower half
    name, call = list(_beyond_32_bits())[which]
    with pytest.raises(AssertionError, match="32 bits"):
        call()
