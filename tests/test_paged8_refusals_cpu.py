"""Refusals of the calls of a cache held in 8 bits: argument errors are status codes found on the host before anything is launched."""
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


def _pool(k=0x1000, v=0x2000, ke=0x31, ve=0x41, L=2, H=4, d=128, ps=16, fmt=cb.CB_CACHE_E4M3, block=8, n=10, sl=None, sp=None, ss=None, sh=None,
          el=None, ep=None, eb=None, eh=1):
    ss = H * d if ss is None else ss
    sh = d if sh is None else sh
    sp = ps * H * d if sp is None else sp
    sl = n * ps * H * d if sl is None else sl
    per = max(1, ps // max(block, 1))
    eb = H if eb is None else eb
    ep = per * H if ep is None else ep
    el = n * per * H if el is None else el
    return cb._PagePool8(k, v, ke, ve, L, H, d, ps, fmt, block, n, sl, sp, ss, sh, el, ep, eb, eh)


POOLS = [(dict(k=0), BAD), (dict(v=0x2008), BAD), (dict(ke=0), BAD), (dict(ve=0), BAD), (dict(L=0), BAD), (dict(H=0), BAD), (dict(ps=0), BAD), (dict(n=0), BAD),
         (dict(block=0), BAD), (dict(block=-8), BAD), (dict(fmt=2), BAD), (dict(fmt=-1), BAD), (dict(ss=520), BAD), (dict(sp=-16), BAD), (dict(ep=-1), BAD),
         (dict(d=96, sh=96), UNS), (dict(ps=24), UNS), (dict(ps=4, block=4), UNS), (dict(ps=512), UNS), (dict(block=4), UNS), (dict(block=12), UNS),
         (dict(block=32), UNS), (dict(n=1 << 31, sl=0, L=1), UNS), (dict(sl=0), UNS), (dict(sp=0), UNS), (dict(ss=0), UNS), (dict(sh=0), UNS),
         (dict(el=0), UNS), (dict(ep=0), UNS), (dict(eb=0), UNS), (dict(eh=0), UNS), (dict(sp=1 << 40), UNS), (dict(ep=1 << 40), UNS),
         (dict(sp=1 << 32), UNS), (dict(ss=1 << 32), UNS), (dict(ep=1 << 32), UNS), (dict(eb=1 << 32), UNS), (dict(sl=1 << 40), UNS), (dict(sh=1 << 40), UNS),
         (dict(el=1 << 40), UNS), (dict(eh=1 << 40), UNS), (dict(sp=(1 << 32) - 16, ss=(1 << 32) - 16, ep=(1 << 32) - 1, eb=(1 << 32) - 1), CUDA),
         (dict(block=16, eb=0), CUDA), (dict(L=1, sl=0, el=0), CUDA), (dict(H=1, sh=0, eh=0, ss=128), CUDA), (dict(fmt=cb.CB_CACHE_INT8), CUDA)]


def _rows(call, pool=None, k=0x10000, v=0x20000, dt=cb.CB_DTYPE_BF16, rows=5, sl=5 * 512, st=512, sh=128, slot=0x100):
    pool = _pool() if pool is None else pool
    return call(ctypes.byref(pool), k, v, dt, rows, sl, st, sh, slot, 0)


@pytest.mark.parametrize("change,want", [
    ({}, CUDA), (dict(rows=0), OK), (dict(rows=0, k=0, v=0, slot=0), OK), (dict(dt=cb.CB_DTYPE_F32), CUDA), (dict(dt=2), BAD), (dict(k=0), BAD),
    (dict(v=0x20008), BAD), (dict(rows=-1), BAD), (dict(slot=0), BAD), (dict(slot=0x104), BAD), (dict(st=516), BAD), (dict(sh=-8), BAD),
    (dict(rows=1 << 31), UNS), (dict(pool=_pool(H=1 << 17)), UNS), (dict(rows=1 << 30, pool=_pool(H=16)), UNS), (dict(rows=(1 << 30) - 1, pool=_pool(H=16)), CUDA), (dict(pool=_pool(L=1 << 16)), UNS)])
def test_rows(change, want):
    assert _rows(cb.lib().cb_paged_store8, **change) == want
    assert _rows(cb.lib().cb_paged_load8, **change) == want


@pytest.mark.parametrize("change,store,load", [
    (dict(sl=0), CUDA, UNS), (dict(st=0), CUDA, UNS), (dict(sh=0), CUDA, UNS), (dict(rows=1, st=0), CUDA, CUDA), (dict(v=0x10000), CUDA, BAD)])
def test_a_source_may_repeat_rows_and_a_result_may_not(change, store, load):
    assert _rows(cb.lib().cb_paged_store8, **change) == store
    assert _rows(cb.lib().cb_paged_load8, **change) == load


@pytest.mark.parametrize("change,want", POOLS)
def test_pools(change, want):
    assert _rows(cb.lib().cb_paged_store8, pool=_pool(**change)) == want
    assert _rows(cb.lib().cb_paged_load8, pool=_pool(**change)) == want
    if change.get("H") != 1:
        assert _attention(pool=_pool(**change)) == want
    assert cb.lib().cb_paged_store8(None, 16, 16, 0, 1, 8, 8, 8, 8, 0) == BAD


def _attention(pool=None, layer=1, q=0x1000, qs=(2048, 128), out=0x2000, os=(2048, 128), rows=5, heads=16, table=0x100, stride=8, cols=8, cu=0x200,
               total=0x300, B=2, max_new=1, scale=0.1, window=0, sinks=0, ws=0x10000, ws_bytes=1 << 30):
    pool = _pool() if pool is None else pool
    layer = min(layer, pool.n_layers - 1) if layer == 1 else layer
    return cb.lib().cb_paged_attention8(ctypes.byref(pool), layer, q, qs[0], qs[1], out, os[0], os[1], rows, heads, table, stride, cols, cu, total, B,
                                        max_new, scale, window, sinks, ws, ws_bytes, 0)


@pytest.mark.parametrize("change,want", [
    ({}, CUDA), (dict(rows=0), OK), (dict(B=0), OK), (dict(max_new=0), CUDA), (dict(max_new=5), CUDA), (dict(window=5, sinks=3), CUDA), (dict(layer=2), BAD),
    (dict(layer=-1), BAD), (dict(heads=15), BAD), (dict(heads=0), BAD), (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD), (dict(scale=float("inf")), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=2.4e38), BAD), (dict(window=-1), BAD), (dict(sinks=-1), BAD), (dict(max_new=-1), BAD), (dict(rows=-1), BAD),
    (dict(B=-1), BAD), (dict(cols=0), BAD), (dict(stride=4), BAD), (dict(q=0), BAD), (dict(q=0x1008), BAD), (dict(out=0), BAD), (dict(out=0x1000), BAD),
    (dict(table=0), BAD), (dict(cu=0), BAD), (dict(total=0x302), BAD), (dict(qs=(2047, 128)), BAD), (dict(os=(0, 128)), UNS), (dict(os=(2048, 0)), UNS),
    (dict(qs=(0, 128)), UNS), (dict(qs=(2048, 0)), UNS), (dict(rows=1, qs=(0, 128), os=(0, 128)), CUDA), (dict(rows=1 << 28), UNS), (dict(ws=0), WS),
    (dict(ws=0x10010), WS), (dict(ws_bytes=1000), WS), (dict(B=1 << 28, rows=1), UNS)])
def test_attention(change, want):
    assert _attention(**change) == want


def test_workspace_and_tensors_of_the_wrong_kind_or_place():
    assert cb.cb_paged_attention8_workspace_bytes(128) > cb.cb_paged_attention8_workspace_bytes(64) > 0
    with pytest.raises(cb.CbError):
        cb.cb_paged_attention8_workspace_bytes(96)
    assert cb.lib().cb_paged_attention8_workspace_bytes(128, None) == BAD
    code, e = torch.zeros(1, 4, 16, 2, 64, dtype=torch.int8), torch.zeros(1, 4, 2, 2, dtype=torch.int8)
    pool = cb.PagePool8(code, code, e, e)
    assert pool.block == 8 and len(pool.c) == ctypes.sizeof(cb._PagePool8)
    rows = torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16)
    for call in (cb.cb_paged_store8, cb.cb_paged_load8):
        with pytest.raises(ValueError):                                # tensors of the host
            call(pool, rows, rows, torch.zeros(3, dtype=torch.int64))
    for bad in ((code.to(torch.uint8), code.to(torch.uint8), e, e), (code, code.view(torch.float8_e4m3fn), e, e), (code, code, e[:, :3], e[:, :3]),
                (code, code, e, e.float()), (code, code, torch.zeros(1, 4, 3, 2, dtype=torch.int8), torch.zeros(1, 4, 3, 2, dtype=torch.int8)),
                (code[..., ::2], code[..., ::2], e, e)):
        with pytest.raises(AssertionError):
            cb.PagePool8(*bad)
    with pytest.raises(AssertionError):
        cb.cb_paged_store8(pool, rows[:, :, :1], rows[:, :, :1], torch.zeros(3, dtype=torch.int64))
    assert cb.cb_launch_count() == 0
