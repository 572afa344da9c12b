"""The paged-cache calls refuse tensors that are not on the cache's (or the tables') GPU, and launch nothing: a kernel
of one GPU would be given addresses of another.  No GPU here: tensors are stood in for by objects that say where they
are, and the library's calls by recorders."""
import pytest
import torch

from paper_2603_28768_amd import binding


class Placed:
    """What the binding asks of a tensor, and the GPU it is said to be on (-1: host memory)."""

    def __init__(self, shape, dtype, gpu=0):
        self.shape, self.dtype, self.gpu = torch.Size(shape), dtype, gpu
        self.device, self.is_cuda = torch.device("cuda", gpu) if gpu >= 0 else torch.device("cpu"), gpu >= 0

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
        return 0x10000

    def is_contiguous(self):
        return True


class Recorder:
    """Stands in for a call of the library."""

    def __init__(self):
        self.calls = 0

    def __call__(self, *args):
        self.calls += 1
        return 0


@pytest.fixture(autouse=True)
def gpu(monkeypatch):
    """The current GPU and the number of every GPU's current stream, as torch would tell them."""
    now = dict(current=0, stream=0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now["current"], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda gpu: now["stream"], raising=False)
    return now


def make_cache(fmt=torch.bfloat16, latent=False, v=0, k_scale=0, v_scale=0):
    eight = fmt == torch.float8_e4m3fn
    c = binding.KvCache(Placed((9, 2, 16, 64), fmt), None if latent else Placed((9, 2, 16, 64), fmt, v),
                        Placed((9, 2, 16), torch.float32, k_scale) if eight else None,
                        Placed((9, 2, 16), torch.float32, v_scale) if eight and not latent else None, dv=64)
    c._append = Recorder()
    return c


@pytest.mark.parametrize("at", [1, -1])
def test_a_cache_lies_on_one_gpu(at):
    make_cache(torch.float8_e4m3fn)
    for other in (dict(v=at), dict(fmt=torch.float8_e4m3fn, k_scale=at), dict(fmt=torch.float8_e4m3fn, v_scale=at)):
        with pytest.raises(AssertionError):
            make_cache(**other)


def append(c, k=0, v=0, slots=0, **kw):
    rows = lambda gpu: Placed((5, 2, 64), torch.bfloat16, gpu)  # noqa: E731
    c.append(rows(k), None if c.v is None else rows(v), Placed((5,), torch.int32, slots), **kw)


@pytest.mark.parametrize("latent", [False, True])
@pytest.mark.parametrize("at", [1, -1])
def test_new_rows_from_elsewhere(at, latent):
    c = make_cache(latent=latent)
    for other in (dict(k=at), dict(slots=at)) + (() if latent else (dict(v=at),)):
        with pytest.raises(AssertionError):
            append(c, **other)
    assert c._append.calls == 0
    append(c)
    assert c._append.calls == 1


def make_attention(monkeypatch, c):
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: Placed(shape, dtype, device.index))
    monkeypatch.setattr(torch, "zeros", lambda shape, dtype, device: Placed((shape,), dtype, device.index))
    a = binding.DecodeAttention(c, 3, 4, 7)
    a._call = Recorder()
    return a


def attend(a, q=0, lens=0, table=0, **kw):
    return a(Placed((3, 4, 64), torch.bfloat16, q), Placed((3,), torch.int32, lens), Placed((3, 7), torch.int32, table), **kw)


@pytest.mark.parametrize("at", [1, -1])
def test_queries_lengths_and_tables_from_elsewhere(at, monkeypatch):
    a = make_attention(monkeypatch, make_cache())
    for other in (dict(q=at), dict(lens=at), dict(table=at)):
        with pytest.raises(AssertionError):
            attend(a, **other)
    assert a._call.calls == 0
    assert attend(a) is a.out and a._call.calls == 1


def make_tables(monkeypatch, lens=0, table=0, ring=0, pool=0):
    made = lambda *shape, dtype, device: Placed(shape, dtype, torch.device(device).index)  # noqa: E731
    monkeypatch.setattr(torch, "full", lambda shape, x, dtype, device: made(*shape, dtype=dtype, device=device))
    monkeypatch.setattr(torch, "zeros", made)
    monkeypatch.setattr(torch, "empty", made)
    i32 = torch.int32
    t = binding.KvTables(3, 7, 9, 16, 20, Placed((3,), i32, lens), Placed((3, 7), i32, table), Placed((9,), i32, ring), Placed((2,), torch.int64, pool))
    t._step = Recorder()
    return t


@pytest.mark.parametrize("at", [1, -1])
def test_tables_lie_on_one_gpu(at, monkeypatch):
    for other in (dict(lens=at), dict(table=at), dict(ring=at), dict(pool=at)):
        with pytest.raises(AssertionError):
            make_tables(monkeypatch, **other)
    t = make_tables(monkeypatch)
    i32 = torch.int32
    for add, lens_out, pool_out in ((at, 0, 0), (0, at, 0), (0, 0, at)):
        with pytest.raises(AssertionError):
            t.step(Placed((3,), i32, add), Placed((3,), i32, lens_out), Placed((2,), torch.int64, pool_out))
    assert t._step.calls == 0
    t.step(Placed((3,), i32))
    assert t._step.calls == 1


def test_another_gpu_is_the_current_one(gpu, monkeypatch):
    """Stream number 0 is the default one of whichever GPU is current; other numbers are streams of one GPU."""
    c = make_cache()
    with pytest.MonkeyPatch.context() as m:
        a = make_attention(m, c)
    t = make_tables(monkeypatch)

    class Stream:
        cuda_stream = 0
    calls = [lambda **kw: append(c, **kw), lambda **kw: attend(a, **kw), lambda **kw: t.step(Placed((3,), torch.int32), **kw)]
    gpu["current"] = 1
    for call in calls:
        for kw in (dict(), dict(stream=Stream())):
            with pytest.raises(AssertionError):
                call(**kw)
    assert c._append.calls == a._call.calls == t._step.calls == 0
    gpu["stream"] = Stream.cuda_stream = 77
    for call in calls:
        call()
        call(stream=Stream())
    assert c._append.calls == a._call.calls == t._step.calls == 2
