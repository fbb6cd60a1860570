"""Refusals of the paged-cache calls: argument errors are status codes found on the host before anything is launched."""
import ctypes

import pytest
import torch

from paper_2609_00891_b200 import binding as cb
from paper_2609_00891_b200 import build as cb_build

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up pointers: host-only")
OK, BAD, UNS, WS, CUDA = cb.CB_OK, cb.CB_ERR_INVALID_ARG, cb.CB_ERR_UNSUPPORTED, cb.CB_ERR_WORKSPACE, cb.CB_ERR_CUDA
P, I64, I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32


@pytest.fixture(scope="module", autouse=True)
def _built():
    cb_build.build()


def _pool(k=0x1000, v=0x2000, L=2, H=4, d=128, ps=16, n=10, sl=None, sp=None, ss=None, sh=None):
    ss = H * d if ss is None else ss
    sh = d if sh is None else sh
    sp = ps * H * d if sp is None else sp
    sl = n * ps * H * d if sl is None else sl
    return cb._PagePool(k, v, L, H, d, ps, n, sl, sp, ss, sh)


BAD_POOLS = [(dict(k=0), BAD), (dict(v=0x2004), BAD), (dict(L=0), BAD), (dict(H=0), BAD), (dict(ps=0), BAD), (dict(n=0), BAD), (dict(ss=516), BAD),
             (dict(sp=-8), BAD), (dict(d=96, sh=96), UNS), (dict(ps=24), UNS), (dict(ps=4), UNS), (dict(ps=512), UNS), (dict(n=1 << 31, sl=0, L=1), UNS),
             (dict(sl=0), UNS), (dict(sp=0), UNS), (dict(ss=0), UNS), (dict(sh=0), UNS), (dict(sp=1 << 40), UNS)]


def _tables(cached=0x100, new=0x200, B=3, ps=16, free=0x300, n_free=5, table=0x400, stride=8, cols=8, cu=0x500, total=0x600, pos=0x700,
            slot=0x800, rows=4, used=0x900):
    return cb.lib().cb_page_tables(P(cached), P(new), I32(B), I32(ps), P(free), I64(n_free), P(table), I64(stride), I32(cols), P(cu), P(total),
                                   P(pos), P(slot), I64(rows), P(used), P(0))


@pytest.mark.parametrize("change,want", [
    ({}, CUDA), (dict(used=0), CUDA), (dict(free=0, n_free=0), CUDA), (dict(pos=0, slot=0, rows=0), CUDA), (dict(B=1, stride=0), CUDA),
    (dict(B=0, cached=0, new=0, table=0, total=0), CUDA), (dict(B=-1), BAD), (dict(cached=0), BAD), (dict(new=0), BAD), (dict(table=0), BAD),
    (dict(total=0), BAD), (dict(cu=0), BAD), (dict(free=0), BAD), (dict(pos=0), BAD), (dict(slot=0), BAD), (dict(slot=0x804), BAD), (dict(pos=0x702), BAD),
    (dict(n_free=-1), BAD), (dict(rows=-1), BAD), (dict(cols=0), BAD), (dict(stride=7), BAD), (dict(ps=24), UNS), (dict(ps=0), UNS),
    (dict(rows=1 << 31), UNS), (dict(total=0x100), BAD), (dict(total=0x200), BAD), (dict(cu=0x100), BAD), (dict(cu=0x600), BAD)])
def test_page_tables(change, want):
    assert _tables(**change) == want


def _store(pool=None, k=0x1000, v=0x2000, dt=cb.CB_DTYPE_BF16, rows=5, sl=5 * 512, st=512, sh=128, slot=0x100):
    pool = _pool() if pool is None else pool
    return cb.lib().cb_paged_store(ctypes.byref(pool), P(k), P(v), I32(dt), I64(rows), I64(sl), I64(st), I64(sh), P(slot), P(0))


@pytest.mark.parametrize("change,want", [
    ({}, CUDA), (dict(rows=0), OK), (dict(dt=cb.CB_DTYPE_F32), CUDA), (dict(dt=2), BAD), (dict(k=0), BAD), (dict(v=0x2008), BAD), (dict(rows=-1), BAD),
    (dict(slot=0), BAD), (dict(slot=0x104), BAD), (dict(st=516), BAD), (dict(sh=-8), BAD), (dict(rows=1 << 31), UNS)])
def test_store(change, want):
    assert _store(**change) == want


@pytest.mark.parametrize("change,want", BAD_POOLS)
def test_pools(change, want):
    assert _store(pool=_pool(**change)) == want
    assert _attention(pool=_pool(**change)) == want
    assert cb.lib().cb_paged_store(None, P(1), P(1), I32(0), I64(1), I64(8), I64(8), I64(8), P(8), P(0)) == BAD


def _rope(x=0x1000, out=0x9000, L=2, H=4, d=128, T=5, xs=(2560, 512, 128), os=(2560, 512, 128), pos=0x100, ast=5, sections=(24, 20, 20), inter=0,
          base=1e6, null_sections=False):
    sec = (ctypes.c_int32 * len(sections))(*sections)
    return cb.lib().cb_rope_axes(P(x), P(out), I32(L), I32(H), I32(d), I64(T), I64(xs[0]), I64(xs[1]), I64(xs[2]), I64(os[0]), I64(os[1]), I64(os[2]),
                                 P(pos), I64(ast), I32(len(sections)), None if null_sections else sec, I32(inter), ctypes.c_double(base), I32(0), P(0))


@pytest.mark.parametrize("change,want", [
    ({}, CUDA), (dict(T=0), OK), (dict(inter=1), CUDA), (dict(sections=(64,)), CUDA), (dict(sections=(0, 64)), CUDA), (dict(sections=(24, 20)), BAD),
    (dict(sections=(70, -6)), BAD), (dict(null_sections=True), BAD), (dict(sections=()), BAD), (dict(sections=(8,) * 7 + (4, 4)), UNS), (dict(d=96), UNS),
    (dict(x=0), BAD), (dict(out=0x9008), BAD), (dict(pos=0), BAD), (dict(pos=0x102), BAD), (dict(base=1.0), BAD), (dict(base=float("nan")), BAD),
    (dict(base=1e13), BAD), (dict(xs=(2560, 516, 128)), BAD), (dict(os=(2560, 0, 128)), UNS), (dict(xs=(0, 512, 128)), CUDA), (dict(L=0), BAD),
    (dict(out=0x1000, os=(2560, 128, 640)), BAD), (dict(out=0x1000), CUDA), (dict(T=1 << 31), UNS), (dict(ast=-1), BAD), (dict(T=-1), BAD)])
def test_rope_axes(change, want):
    assert _rope(**change) == want


def _attention(pool=None, layer=1, q=0x1000, qs=(2048, 128), out=0x2000, os=(2048, 128), rows=5, heads=16, table=0x100, stride=8, cols=8, cu=0x200,
               total=0x300, B=2, max_new=1, scale=0.1, window=0, sinks=0, ws=0x10000, ws_bytes=1 << 30):
    pool = _pool() if pool is None else pool
    return cb.lib().cb_paged_attention(ctypes.byref(pool), I32(layer), P(q), I64(qs[0]), I64(qs[1]), P(out), I64(os[0]), I64(os[1]), I64(rows), I32(heads),
                                       P(table), I64(stride), I32(cols), P(cu), P(total), I32(B), I32(max_new), ctypes.c_float(scale), I32(window),
                                       I32(sinks), P(ws), ctypes.c_size_t(ws_bytes), P(0))


@pytest.mark.parametrize("change,want", [
    ({}, CUDA), (dict(rows=0), OK), (dict(B=0), OK), (dict(max_new=0), CUDA), (dict(window=5, sinks=3), CUDA), (dict(layer=2), BAD), (dict(layer=-1), BAD),
    (dict(heads=15), BAD), (dict(heads=0), BAD), (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD), (dict(scale=float("inf")), BAD),
    (dict(scale=float("nan")), BAD), (dict(window=-1), BAD), (dict(sinks=-1), BAD), (dict(max_new=-1), BAD), (dict(rows=-1), BAD), (dict(B=-1), BAD),
    (dict(cols=0), BAD), (dict(stride=4), BAD), (dict(q=0), BAD), (dict(q=0x1008), BAD), (dict(out=0), BAD), (dict(table=0), BAD), (dict(cu=0), BAD),
    (dict(total=0x302), BAD), (dict(qs=(2047, 128)), BAD), (dict(os=(0, 128)), UNS), (dict(os=(2048, 0)), UNS), (dict(qs=(0, 128)), UNS), (dict(qs=(2048, 0)), UNS), (dict(rows=1, qs=(0, 128), os=(0, 128)), CUDA),
    (dict(rows=1 << 28), UNS), (dict(ws=0), WS), (dict(ws=0x10010), WS), (dict(ws_bytes=1000), WS)])
def test_attention(change, want):
    assert _attention(**change) == want


def test_workspace_and_tensors_of_the_wrong_place():
    assert cb.cb_paged_attention_workspace_bytes(128) > cb.cb_paged_attention_workspace_bytes(64) > 0
    with pytest.raises(cb.CbError):
        cb.cb_paged_attention_workspace_bytes(96)
    pool = torch.zeros(1, 4, 8, 2, 64, dtype=torch.bfloat16)
    rows = torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):                                   # tensors of the host
        cb.cb_paged_store(cb.PagePool(pool, pool), rows, rows, torch.zeros(3, dtype=torch.int64))
    assert cb.cb_launch_count() == 0


@pytest.mark.parametrize("B,want", [((1 << 28) - 1, CUDA), (1 << 28, UNS), ((1 << 31) - 1, UNS)])
def test_request_counts(B, want):
    """Requests and what is counted from them stay far inside 32 bits."""
    assert _tables(B=B, cached=1 << 40, new=2 << 40, table=3 << 40, cu=4 << 40, total=5 << 40) == want
    assert _attention(B=B, rows=1) == want


@pytest.mark.parametrize("scale,want", [(2.3e38, CUDA), (2.4e38, BAD), (3.4e38, BAD), (1e-45, CUDA)])
def test_scales(scale, want):
    """The kernels scale scores by scale * log2(e): that product is finite too."""
    assert _attention(scale=scale) == want


@pytest.mark.parametrize("change,want", [
    (dict(pos=0x500), BAD), (dict(pos=0x104), BAD), (dict(pos=0x10c), CUDA), (dict(slot=0x700), BAD), (dict(used=0x508), BAD), (dict(used=0x510), CUDA),
    (dict(total=0x310), BAD), (dict(total=0x314), CUDA), (dict(cu=0x45c), BAD), (dict(cu=0x460), CUDA), (dict(total=0x20, stride=9, table=0x24), CUDA),
    (dict(free=0x400, n_free=1), BAD), (dict(pos=0x100, slot=0x200, rows=0), CUDA)])
def test_page_tables_outputs_in_the_place_of_other_arrays(change, want):
    assert _tables(**change) == want


def test_attention_in_place():
    assert _attention(out=0x1000) == BAD
