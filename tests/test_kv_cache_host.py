"""Argument checks of the paged-cache entry points, and the plain forms the GPU tests compare with.  No device work:
every call here is refused before anything is launched, or asks for a size."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_28768_amd import binding
from paper_2603_28768_amd.binding import AttentionArgs, KvCacheDesc, KvTablesArgs

import kv_reference as ref

OK, EINVAL, EWORKSPACE = 0, -1, -4
ADDR = 0x10000          # stands for an aligned device pointer; no call below gets as far as using it


def cache(**kw):
    d = KvCacheDesc()
    d.format, d.page_size, d.pages, d.heads, d.dk, d.dv = binding.CRAFT_KV_BF16, 16, 100, 4, 128, 128
    d.k = d.v = ADDR
    d.k_page = d.v_page = 4 * 16 * 128
    d.k_head = d.v_head = 16 * 128
    d.k_token = d.v_token = 128
    for n, x in kw.items():
        setattr(d, n, x)
    return d


def attention(**kw):
    a = AttentionArgs()
    a.R, a.Hq, a.max_pages, a.scale = 3, 16, 10, 0.1
    a.q, a.q_stride, a.q_head_stride = ADDR, 16 * 128, 128
    a.lens = a.table = a.out = a.workspace = ADDR
    a.table_stride = 10
    for n, x in kw.items():
        setattr(a, n, x)
    return a


def size_of(c, a):
    n = ctypes.c_size_t(123)
    rc = binding.lib().craft_decode_attention_workspace(ctypes.byref(c), ctypes.byref(a), ctypes.byref(n))
    return rc, n.value


BAD_CACHES = [dict(format=3), dict(format=-1), dict(page_size=0), dict(page_size=-16), dict(page_size=24), dict(page_size=131072),
              dict(pages=0), dict(pages=-1), dict(pages=1 << 31), dict(pages=1 << 27), dict(heads=0), dict(heads=-4), dict(dk=0), dict(dv=0),
              dict(dk=-8), dict(dk=124), dict(dv=4), dict(dk=264), dict(dv=264), dict(k=None), dict(k=ADDR + 8), dict(v=ADDR + 2),
              dict(k_page=0), dict(k_head=-1), dict(k_token=0), dict(k_token=129), dict(v_token=132), dict(v_page=7),
              dict(k_token=1 << 25), dict(v_token=1 << 25), dict(k_page=1 << 62), dict(v=None, dv=256), dict(v=None, dk=584),
              dict(v=None, dk=576, dv=520), dict(format=binding.CRAFT_KV_E4M3),
              dict(format=binding.CRAFT_KV_E4M3, k_scale=ADDR), dict(format=binding.CRAFT_KV_E4M3, k_scale=ADDR + 4, v_scale=ADDR),
              dict(format=binding.CRAFT_KV_E4M3, k_scale=ADDR, v_scale=ADDR, dk=120), dict(format=binding.CRAFT_KV_F32, dk=126)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches_are_refused_by_every_call(bad):
    lib = binding.lib()
    c, a = cache(**bad), attention(q_head_stride=1024, q_stride=16384)
    assert size_of(c, a)[0] == EINVAL
    a.workspace_bytes = 1 << 40
    assert lib.craft_decode_attention(ctypes.byref(c), ctypes.byref(a), None) == EINVAL
    assert lib.craft_kv_append(ctypes.byref(c), 5, ADDR, 65536, ADDR, 65536, ADDR, None) == EINVAL


@pytest.mark.parametrize("good", [dict(), dict(format=binding.CRAFT_KV_F32, dk=64, dv=68), dict(page_size=1), dict(page_size=65536),
                                  dict(v=None, dk=576, dv=512, heads=1, k_token=576), dict(dk=80, dv=8), dict(dk=256, dv=256),
                                  dict(format=binding.CRAFT_KV_E4M3, k_scale=ADDR, v_scale=ADDR)], ids=str)
def test_sizes_of_good_caches(good):
    rc, n = size_of(cache(**good), attention())
    assert rc == OK and 0 < n < 1 << 28


BAD_CALLS = [dict(R=-1), dict(Hq=0), dict(Hq=18), dict(Hq=-4), dict(R=1 << 28), dict(max_pages=0), dict(max_pages=1 << 27), dict(window=-1),
             dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(q=ADDR + 8), dict(q_stride=0), dict(q_stride=-2048),
             dict(q_stride=2044), dict(q_head_stride=120), dict(q_head_stride=132), dict(lens=None), dict(lens=ADDR + 2), dict(table=None),
             dict(table=ADDR + 1), dict(table_stride=9), dict(out=None), dict(out=ADDR + 8), dict(lse=ADDR + 2), dict(workspace=None),
             dict(workspace=ADDR + 8)]


@pytest.mark.parametrize("bad", BAD_CALLS, ids=str)
def test_bad_attention_calls_are_refused(bad):
    a = attention(workspace_bytes=1 << 40, **bad)
    assert binding.lib().craft_decode_attention(ctypes.byref(cache()), ctypes.byref(a), None) == EINVAL


def test_heads_that_share_a_key_are_limited():
    c = cache(heads=1, v=None, dk=576, dv=512, k_token=576)
    for Hq, rc in ((65536, OK), (65537, EINVAL), (1 << 27, EINVAL)):
        assert size_of(c, attention(Hq=Hq))[0] == rc
        if rc != OK:
            a = attention(Hq=Hq, q_stride=1 << 40, q_head_stride=576, workspace_bytes=1 << 40)
            assert binding.lib().craft_decode_attention(ctypes.byref(c), ctypes.byref(a), None) == rc


def test_null_structs_and_small_workspaces():
    lib = binding.lib()
    c, a = cache(), attention()
    assert lib.craft_decode_attention(None, ctypes.byref(a), None) == EINVAL
    assert lib.craft_decode_attention(ctypes.byref(c), None, None) == EINVAL
    assert lib.craft_decode_attention_workspace(ctypes.byref(c), ctypes.byref(a), None) == EINVAL
    rc, n = size_of(c, a)
    a.workspace_bytes = n - 1
    assert lib.craft_decode_attention(ctypes.byref(c), ctypes.byref(a), None) == EWORKSPACE
    # no requests: nothing to do, whatever the pointers
    z = attention(R=0, q=None, lens=None, table=None, out=None, workspace=None)
    assert lib.craft_decode_attention(ctypes.byref(c), ctypes.byref(z), None) == OK


def test_append_checks():
    lib = binding.lib()
    row = 4 * 128
    def call(c=None, T=5, k=ADDR, ks=row, v=ADDR, vs=row, slots=ADDR):
        return lib.craft_kv_append(ctypes.byref(c or cache()), T, k, ks, v, vs, slots, None)
    assert call(T=-1) == EINVAL and call(T=1 << 41) == EINVAL
    assert call(T=0, k=None, v=None, slots=None) == OK
    assert call(k=None) == EINVAL and call(v=None) == EINVAL and call(slots=None) == EINVAL
    assert call(k=ADDR + 8) == EINVAL and call(v=ADDR + 8) == EINVAL and call(slots=ADDR + 2) == EINVAL
    assert call(ks=row - 8) == EINVAL and call(vs=row - 8) == EINVAL and call(ks=row + 4) == EINVAL and call(vs=1 << 50) == EINVAL
    assert lib.craft_kv_append(None, 5, ADDR, row, ADDR, row, ADDR, None) == EINVAL


def tables(**kw):
    a = KvTablesArgs()
    a.R, a.max_pages, a.page_size, a.max_new, a.pages, a.table_stride = 5, 10, 16, 100, 50, 10
    for n in ("add", "lens", "table", "ring", "pool", "lens_out", "pool_out", "token_off", "slots", "positions", "workspace"):
        setattr(a, n, ADDR)
    a.workspace_bytes = 1 << 30
    for n, x in kw.items():
        setattr(a, n, x)
    return a


@pytest.mark.parametrize("bad", [dict(R=-1), dict(max_pages=0), dict(max_pages=1 << 27), dict(page_size=12), dict(page_size=0), dict(max_new=-1),
                                 dict(pages=0), dict(pages=1 << 27), dict(table_stride=9), dict(add=None), dict(lens=None), dict(table=None),
                                 dict(ring=None), dict(pool=None), dict(pool=ADDR + 4), dict(lens_out=None), dict(pool_out=None),
                                 dict(pool_out=ADDR + 4), dict(token_off=None), dict(slots=None), dict(slots=ADDR + 2),
                                 dict(positions=ADDR + 1), dict(workspace=None), dict(workspace=ADDR + 4)], ids=str)
def test_bad_table_steps_are_refused(bad):
    assert binding.lib().craft_kv_tables(ctypes.byref(tables(**bad)), None) == EINVAL


def test_table_workspace():
    lib = binding.lib()
    n = ctypes.c_size_t()
    a = tables()
    assert lib.craft_kv_tables_workspace(ctypes.byref(a), ctypes.byref(n)) == OK and n.value > 0
    a.workspace_bytes = n.value - 1
    assert lib.craft_kv_tables(ctypes.byref(a), None) == EWORKSPACE
    assert lib.craft_kv_tables_workspace(ctypes.byref(a), None) == EINVAL
    assert lib.craft_kv_tables_workspace(None, ctypes.byref(n)) == EINVAL
    assert lib.craft_kv_tables(None, None) == EINVAL


def test_binding_refuses_what_the_descriptor_cannot_say():
    t = torch.zeros(2, 1, 16, 64)
    with pytest.raises(AssertionError):
        binding.KvCache(t, t)                                        # not on a GPU
    with pytest.raises(AssertionError):
        binding.KvCache(t.half(), t.half())


# ---- the plain forms themselves

def test_plain_tables_keep_every_page_in_one_place():
    g = np.random.default_rng(5)
    R, M, P, N = 6, 8, 4, 30
    state = dict(lens=np.zeros(R, np.int32), table=np.full((R, M), -1, np.int32), ring=np.arange(N, dtype=np.int32),
                 pool=np.array([0, N], np.int64))
    for step in range(60):
        add = g.integers(-1, 7, R).astype(np.int32)
        out = ref.tables(state["lens"], add, state["table"], state["ring"], state["pool"], P, 20)
        state = {n: out[n] for n in state}
        held = [int(state["table"][r, c]) for r in range(R) for c in range(-(-int(state["lens"][r]) // P))]
        free = [int(state["ring"][i % N]) for i in range(*state["pool"])]
        assert sorted(held + free) == list(range(N))
        live = out["slots"][out["slots"] >= 0]
        assert len(set(live.tolist())) == len(live) == out["token_off"][-1]


def test_plain_attention_is_the_definition():
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn(4, 2, 4, 8, generator=g), torch.randn(4, 2, 4, 12, generator=g)
    q = torch.randn(1, 4, 8, generator=g)
    table = torch.tensor([[2, 0, -1]])
    out, lse, bound, _ = ref.attention(q, k, v, None, None, [7], table, 0.5, window=5)
    for h in range(4):
        s, vals = [], []
        for i in range(2, 7):
            page = [2, 0][i // 4]
            s.append(0.5 * float(q[0, h].double() @ k[page, h // 2, i % 4].double()))
            vals.append(v[page, h // 2, i % 4].double())
        w = np.exp(np.array(s))
        assert np.allclose(sum(a * b for a, b in zip(w / w.sum(), vals)), out[0, h])
        assert np.isclose(np.log(w.sum()), lse[0, h])
    assert (bound > 0).all()
