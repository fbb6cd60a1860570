"""The paged cache held in 8 bits on the GPU: store, read-back and attention, each against a plain 64-bit form, then a run of them."""
import numpy as np
import pytest
import torch

import paged8_ref as ref
import paged_ref
from paper_2609_00891_b200 import binding as cb

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3, INT8 = torch.float8_e4m3fn, torch.int8
KINDS = pytest.mark.parametrize("kind", [E4M3, INT8], ids=["e4m3", "int8"])


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _pool(kind, L, pages, page, block, H, d, hnd=False, seed=0, wild=True):
    """Codes and exponents of any bytes (NaN among the e4m3 codes), slots or heads outermost in a page; a wider exponent tensor."""
    g = _gen(seed)
    out = []
    for _ in range(2):
        shape = (L, pages, H, page, d) if hnd else (L, pages, page, H, d)
        x = torch.randint(-128 if wild else 0, 128 if wild else 1, shape, generator=g, device=DEV, dtype=torch.int32).to(torch.int8)
        out.append((x.transpose(2, 3) if hnd else x).view(kind))
        e = torch.randint(-128 if wild else 0, 128 if wild else 1, (L, pages, page // block, H + 3), generator=g, device=DEV, dtype=torch.int32).to(torch.int8)
        out.append(e[..., :H])
    return cb.PagePool8(out[0], out[2], out[1], out[3])


def _two(e):
    """2^e in 64 bits, exactly (a power function on the GPU is off by a step here and there)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _state(pool):
    """(codes, exponents) of K and of V as float64 and int64 numpy."""
    return [(ref.numbers(c), np.ascontiguousarray(e.cpu().numpy().astype(np.int64))) for c, e in ((pool.k, pool.k_exp), (pool.v, pool.v_exp))]


def _same(pool, state):
    for (c, e), (wc, we) in zip(_state(pool), state):
        assert np.array_equal(e, we), np.argwhere(e != we)[:5]
        bad = ~((c == wc) | (np.isnan(c) & np.isnan(wc)))
        assert not bad.any(), (bad.sum(), np.argwhere(bad)[:5], c[bad][:5], wc[bad][:5])


def _store(pool, state, x, slot):
    """One call, and the same in 64 bits."""
    cb.cb_paged_store8(pool, x[0], x[1], torch.tensor(slot, dtype=torch.int64, device=DEV))
    for (c, e), y in zip(state, x):
        ref.store(c, e, y.double().cpu().numpy(), slot, pool.k.dtype, pool.page_size, pool.block)
    _same(pool, state)


def _rows(L, T, H, d, dtype, seed, spread=1.0):
    """K and V rows of magnitudes that vary from row to row, head-major in a wider tensor."""
    g = _gen(seed)
    out = []
    for _ in range(2):
        x = torch.randn(L, H, T + 2, d, generator=g, device=DEV) * torch.exp2(torch.round(spread * torch.randn(L, H, T + 2, 1, generator=g, device=DEV)))
        out.append(x.to(dtype).transpose(1, 2)[:, :T])
    return out


# ---------------------------------------------------------------------------------------------------- store
@KINDS
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("L,T,H,d,page,block,hnd", [(1, 1, 1, 64, 8, 8, False), (3, 37, 2, 128, 16, 8, True), (2, 200, 5, 64, 256, 256, False),
                                                    (5, 33, 8, 128, 64, 32, False), (1, 300, 3, 128, 128, 64, True), (40, 70, 2, 64, 32, 16, False)])
def test_store(kind, dtype, L, T, H, d, page, block, hnd):
    """Rows of one request in three calls that end inside blocks, then its last rows once more, larger."""
    pages = -(-T // page) + 2
    pool = _pool(kind, L, pages, page, block, H, d, hnd)
    state = _state(pool)
    order = np.random.default_rng(1).permutation(pages)
    slot = [int(order[t // page]) * page + t % page for t in range(T)]
    x = _rows(L, T, H, d, dtype, 2, spread=2.0)
    cuts = sorted({0, T // 3, T // 2 + 1, T})
    for a, b in zip(cuts, cuts[1:]):
        _store(pool, state, [y[:, a:b] for y in x], slot[a:b])
    a = max(0, T - 5)
    _store(pool, state, [(8 * y[:, a:]).to(dtype) for y in x], slot[a:])


@KINDS
def test_store_token_by_token_is_what_one_call_writes_where_magnitudes_fall(kind):
    """The first row is the block's largest: later ones change no exponent, and the calls' number does not matter."""
    L, T, H, d, page, block = 2, 50, 3, 128, 16, 16
    x = _rows(L, T, H, d, torch.bfloat16, 3)
    x = [y * torch.tensor([16.0 if t % block == 0 else 0.0625 for t in range(T)], device=DEV)[None, :, None, None].bfloat16() for y in x]
    a, b = (_pool(kind, L, 5, page, block, H, d) for _ in range(2))
    slot = torch.arange(T, device=DEV) + page
    cb.cb_paged_store8(a, x[0], x[1], slot)
    for t in range(T):
        cb.cb_paged_store8(b, x[0][:, t:t + 1], x[1][:, t:t + 1], slot[t:t + 1])
    for p, q in ((a.k, b.k), (a.v, b.v)):
        assert torch.equal(p.view(torch.int8)[:, 1:4], q.view(torch.int8)[:, 1:4])
    assert torch.equal(a.k_exp, b.k_exp) and torch.equal(a.v_exp, b.v_exp)


@KINDS
def test_store_growing_exponents_keep_their_error_bound(kind):
    """Rows that double again and again: a held value is off by half a step of e4m3 (2^-4 of it) and half a subnormal step for each
    time it was rounded, below one step of the last in all; int8 by below one step of the last exponent."""
    L, T, H, d, page, block = 1, 16, 2, 64, 16, 16
    pool = _pool(kind, L, 2, page, block, H, d)
    state = _state(pool)
    x = [torch.randn(L, T, H, d, generator=_gen(5), device=DEV).bfloat16() * torch.exp2(torch.arange(T, device=DEV) * 1.0)[None, :, None, None].bfloat16() for _ in range(2)]
    for t in range(T):
        _store(pool, state, [y[:, t:t + 1] for y in x], [t])
    out = [torch.empty(L, T, H, d, device=DEV) for _ in range(2)]
    cb.cb_paged_load8(pool, out[0], out[1], torch.arange(T, device=DEV))
    for o, y, e in zip(out, x, (pool.k_exp, pool.v_exp)):
        step = _two(e[0, 0, 0])[None, None, :, None] * (2.0 ** -9 if kind is E4M3 else 1.0)
        assert ((o.double() - y.double()).abs() <= step + (y.double().abs() * 2.0 ** -4 if kind is E4M3 else 0)).all()


@KINDS
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_store_of_the_ends_of_the_range(kind, dtype):
    """Zeros, numbers under the least exponent, the largest finite ones, infinities, NaN, signed zeros: a block of each."""
    L, H, d, page, block = 1, 1, 64, 8, 8
    big = torch.finfo(dtype).max
    rows = [0.0, -0.0, 2.0 ** -126, -(2.0 ** -109), 1.5 * 2.0 ** -101, 448.0, 449.0, 464.0, 127.0, 127.5, 128.0, 2.0 ** 126, -(2.0 ** 127), big, float("inf"), float("nan"), 57344.0]
    x = torch.zeros(L, len(rows) * block, H, d, dtype=dtype)
    for i, v in enumerate(rows):
        x[0, i * block:(i + 1) * block] = (torch.linspace(-1, 1, block * d).reshape(block, 1, d) * (v if np.isfinite(v) else 1.0)).to(dtype)
        x[0, i * block + 3, 0, 5] = v
    x = x.to(DEV)
    pool = _pool(kind, L, len(rows) + 1, page, block, H, d)
    _store(pool, _state(pool), [x, -x], list(range(x.shape[1])))


@KINDS
@pytest.mark.parametrize("slot", [
    [-1] * 5, [-1, 3, -1, 4, 5, 1 << 40, 6, -7, 16, 17, -1], list(range(7, 300)),                           # skipped rows inside a block
    [8] + [-1] * 31 + [9] + [-1] * 70 + [40, 41], [-1] * 40 + [0, 1] + [-1] * 31 + [2], [5, 3, 1, 7, 2], [32 + (7 * i) % 32 for i in range(32)]])
def test_store_of_rows_between_skipped_ones_and_in_any_order_within_a_block(kind, slot):
    L, H, d, page, block = 2, 2, 64, 32, 32
    pool = _pool(kind, L, 10, page, block, H, d)
    _store(pool, _state(pool), _rows(L, len(slot), H, d, torch.bfloat16, 7), slot)


@KINDS
@pytest.mark.parametrize("n,L,H", [(1, 64, 8), (37, 3, 1), (500, 2, 9), (2500, 1, 2)])
def test_store_of_many_requests(kind, n, L, H):
    """One new row each, at any place of its block; in a batch with rows behind the last one."""
    d, page, block = 128, 16, 16
    rng = np.random.default_rng(n)
    pool = _pool(kind, L, n, page, block, H, d)
    slot = [int(p) * page + int(o) for p, o in zip(rng.permutation(n), rng.integers(0, page, n))] + [-1] * 9
    _store(pool, _state(pool), _rows(L, n + 9, H, d, torch.bfloat16, 8, spread=3.0), slot)


@KINDS
@pytest.mark.parametrize("block,dtype,d,H,L", [(16, torch.bfloat16, 128, 5, 20), (32, torch.bfloat16, 128, 3, 20), (16, torch.float32, 128, 8, 20),
                                               (8, torch.float32, 64, 2, 24), (32, torch.float32, 64, 9, 8), (64, torch.bfloat16, 64, 1, 24)])
def test_store_of_short_runs_in_many_layers(kind, block, dtype, d, H, L):
    """One to four rows of each of 400 requests, some of them twice: enough work that a thread block has 32 rows of the slot map."""
    page, n = 64, 400
    rng = np.random.default_rng(block + d)
    pool = _pool(kind, L, n, page, block, H, d)
    slot, row = [], []
    for p in rng.permutation(n):
        first = int(rng.integers(0, page - 4))
        for o in range(first, first + int(rng.integers(1, 5))):
            again = 1 + int(rng.integers(0, 8) == 0)
            row += [len(set(row))] * again
            slot += [int(p) * page + o] * again
    x = [y[:, row] for y in _rows(L, len(set(row)), H, d, dtype, 9, spread=3.0)]
    _store(pool, _state(pool), x, slot)


@KINDS
def test_store_and_load_nothing(kind):
    pool = _pool(kind, 2, 3, 8, 8, 2, 64)
    state = _state(pool)
    e, s = torch.empty(2, 0, 2, 64, dtype=torch.bfloat16, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    cb.cb_paged_store8(pool, e, e, s)
    cb.cb_paged_load8(pool, e, e.clone(), s)
    _same(pool, state)


# ---------------------------------------------------------------------------------------------------- load
@KINDS
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_load_of_every_code_and_exponent(kind, dtype):
    """256 codes under exponents -128 .. 127 (those outside the range count as its ends), exactly."""
    H, d = 2, 128
    code = torch.arange(-128, 128, device=DEV).to(torch.int8)
    k = code.view(1, 1, 1, 2, 128).expand(1, 256, 8, 2, 128).contiguous().view(kind)
    e = torch.arange(-128, 128, device=DEV).to(torch.int8).view(1, 256, 1, 1).expand(1, 256, 1, H).contiguous()
    pool = cb.PagePool8(k, k, e, e)
    slot = torch.randperm(256 * 8, generator=_gen(0), device=DEV)
    room = [torch.full((1, H, slot.numel() + 3, d + 8), 7.0, dtype=dtype, device=DEV) for _ in range(2)]
    out = [r[..., :d].transpose(1, 2)[:, :slot.numel()] for r in room]
    cb.cb_paged_load8(pool, out[0], out[1], slot)
    want = (k.double()[0] * _two(e[0].clamp(*ref.EXPS[kind]))[..., None])[slot // 8, slot % 8]
    used = ~(want.abs() >= 2.0 ** 128)                            # code -128, which the store does not write, is past fp32 at the last exponent
    assert (want[~used] == -2.0 ** 128).all()
    for o in out:
        got = o[0].double()
        assert (got[~used] == -torch.inf).all()
        assert ((got == want) | (got.isnan() & want.isnan()) | ~used).all()
    assert all((r[..., d:] == 7).all() and (r[:, :, slot.numel():] == 7).all() for r in room)


@KINDS
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("L,T,H,d,page,block,hnd", [(1, 1, 1, 64, 8, 8, False), (3, 65, 2, 128, 16, 8, True), (36, 130, 5, 64, 64, 64, False), (2, 1000, 8, 128, 32, 16, False)])
def test_load(kind, dtype, L, T, H, d, page, block, hnd):
    """Slots in any order, some twice, some skipped: those rows stay."""
    pool = _pool(kind, L, 9, page, block, H, d, hnd)
    pool.k_exp.clamp_(-99, 99), pool.v_exp.clamp_(-99, 99)
    rng = np.random.default_rng(T)
    slot = rng.integers(0, 9 * page, T)
    slot[1::4] = -1
    slot[3::16] = 9 * page
    out = [torch.full((L, T, H, d), 5.0, dtype=dtype, device=DEV) for _ in range(2)]
    cb.cb_paged_load8(pool, out[0], out[1], torch.tensor(slot, device=DEV))
    live = (slot >= 0) & (slot < 9 * page)
    for o, (c, e) in zip(out, _state(pool)):
        want = np.full((L, T, H, d), 5.0)
        want[:, live] = ref.values(c, e, block)[:, slot[live] // page, slot[live] % page]
        got = o.double().cpu().numpy()
        assert ((got == want) | (np.isnan(got) & np.isnan(want))).all()


@KINDS
def test_a_pool_past_32_bit_offsets(kind):
    pages, page, H, d = 70000, 64, 8, 128                     # 4.6e9 codes
    k = torch.zeros(1, pages, page, H, d, dtype=torch.int8, device=DEV).view(kind)
    e = torch.zeros(1, pages, 2, H, dtype=torch.int8, device=DEV)
    pool = cb.PagePool8(k, k, e, e)                           # K and V alike: written twice with the same values
    rows = torch.randn(1, 5, H, d, generator=_gen(1), device=DEV).bfloat16()
    slot = torch.tensor([0, (pages - 1) * page, 35000 * page, (pages - 1) * page + 32, 64], device=DEV)
    cb.cb_paged_store8(pool, rows, rows, slot)
    out = [torch.empty(1, 5, H, d, device=DEV) for _ in range(2)]
    cb.cb_paged_load8(pool, out[0], out[1], slot)
    bound = rows.float().abs().amax(-1, keepdim=True) / 127 + 1e-9 if kind is INT8 else rows.float().abs() / 16 + 1e-3
    assert torch.equal(out[0], out[1]) and ((out[0] - rows.float()).abs() <= bound).all()
    q = torch.randn(1, 8, d, generator=_gen(2), device=DEV).bfloat16()
    got = torch.empty_like(q)
    cb.cb_paged_attention8(q, got, pool, 0, _i32([[pages - 1]]), _i32([0, 1]), _i32([1]), 0.1, _workspace(d))
    assert torch.equal(got[0], out[0][0, 1].bfloat16())


# ---------------------------------------------------------------------------------------------------- attention
_ws = {}


def _workspace(d):
    if d not in _ws:
        _ws[d] = torch.zeros(cb.cb_paged_attention8_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    return _ws[d]


def _batch(kind, new, total, H, group, d, page, block, hnd=False, pad_rows=0, seed=0, layers=1, layer=0, grow=1.0):
    """A pool of any bytes in which the requests' rows are stored, and the batch's queries in a wider tensor."""
    g = _gen(seed)
    need = [-(-t // page) for t in total]
    pages = sum(need) + 2
    pool = _pool(kind, layers, pages, page, block, H, d, hnd, seed)
    cols = max(need + [1]) + 2
    table = torch.full((len(new), cols), -1, dtype=torch.int32, device=DEV)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    at, slot = 0, []
    for b, t in enumerate(total):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        j = torch.arange(t, device=DEV)
        slot.append(table[b, j // page].long() * page + j % page)
    slot = torch.cat(slot) if slot else torch.empty(0, dtype=torch.int64, device=DEV)
    n = slot.numel()
    scale = torch.exp(0.5 * torch.randn(H, d, generator=g, device=DEV))
    size = torch.exp2(torch.round(grow * torch.randn(n, 1, 1, generator=g, device=DEV)).clamp(-3, 1))      # rows of unlike size: exponents that differ
    k = (torch.randn(n, H, d, generator=g, device=DEV) * scale).bfloat16()
    v = ((torch.randn(n, H, d, generator=g, device=DEV) + 0.25) * size).bfloat16()
    one = cb.PagePool8(*(x[layer:layer + 1] for x in (pool.k, pool.v, pool.k_exp, pool.v_exp)))
    cb.cb_paged_store8(one, k[None], v[None], slot)
    q = torch.randn(sum(new) + pad_rows, H * group, d + 8, generator=g, device=DEV).bfloat16()[..., :d]
    if pad_rows:
        q[sum(new):] = float("nan")
    cu = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
    return q, pool, table, cu, total


def _attend(q, pool, table, cu, total, window=0, n_sink=0, max_new=None, layer=0, scale=None, out=None, stream=None):
    T, Hq, d = q.shape
    if out is None:
        out = torch.full((Hq, T, d), 5.0, dtype=torch.bfloat16, device=DEV).transpose(0, 1)   # head-major
    scale = d ** -0.5 if scale is None else scale
    most = max([b - a for a, b in zip(cu, cu[1:])] + [0]) if max_new is None else max_new
    cb.cb_paged_attention8(q, out, pool, layer, table, _i32(cu), _i32(total), scale, _workspace(d), max_new=most, window=window, n_sink=n_sink,
                           stream=stream)
    return out


def _plain(pool, layer):
    """The layer's values in float64, whatever is there."""
    out = []
    for c, e in ((pool.k, pool.k_exp), (pool.v, pool.v_exp)):
        f = _two(e[layer].clamp(*ref.EXPS[c.dtype])).repeat_interleave(pool.block, 1)
        out.append(c[layer].double() * f[..., None])
    return out


def _compare(q, pool, table, cu, total, window=0, n_sink=0, max_new=None, layer=0, scale=None, weight=2.0 ** -8):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out = _attend(q, pool, table, cu, total, window, n_sink, max_new, layer, scale)
    k, v = _plain(pool, layer)
    want, tol = ref.attention(q, k, v, table, cu, total, scale, window, n_sink, weight)
    n = cu[-1]
    err = (out[:n].double() - want[:n]).abs()
    bad = ~(err <= tol[:n])
    assert not bad.any(), (int(bad.sum()), err.max().item(), bad.nonzero()[:4].tolist())
    assert (out[n:] == 5).all()
    cb.cb_last_device_status()
    assert int(_workspace(q.shape[2])[:8192].sum()) == 0            # the join counters are ready for the next call
    return out


DECODE = [1, 2, 7, 8, 15, 16, 17, 63, 64, 65, 127, 128, 129, 1000]


@KINDS
@pytest.mark.parametrize("H,group,d,page,block,hnd", [(1, 1, 64, 8, 8, False), (2, 5, 128, 16, 16, True), (8, 8, 128, 16, 8, False), (3, 2, 64, 64, 32, False),
                                                      (2, 16, 128, 32, 32, False), (1, 17, 128, 128, 8, True), (2, 40, 64, 256, 256, False),
                                                      (1, 70, 128, 16, 16, False), (2, 9, 64, 16, 8, False)])
def test_attention_single_tokens(kind, H, group, d, page, block, hnd):
    b = _batch(kind, [1] * len(DECODE), DECODE, H, group, d, page, block, hnd, pad_rows=3)
    _compare(*b, weight=2.0 ** -11 if group <= 16 else 2.0 ** -8)


@KINDS
@pytest.mark.parametrize("new,total", [
    ([5], [5]), ([1, 0, 33, 64, 65, 130], [1, 0, 40, 64, 300, 131]), ([128, 129, 1, 256, 257], [128, 500, 700, 256, 258]),
    ([700], [1500]), ([0, 0, 3], [0, 10, 3]), ([4, 4, 4, 4], [4, 100, 1000, 77])])
@pytest.mark.parametrize("H,group,d,page,block,hnd", [(2, 5, 128, 16, 16, False), (1, 8, 64, 32, 8, True), (3, 1, 128, 128, 64, False)])
def test_attention_chunks(kind, new, total, H, group, d, page, block, hnd):
    b = _batch(kind, new, total, H, group, d, page, block, hnd, pad_rows=2)
    one = _compare(*b)
    _compare(*b, max_new=1)                              # the bound on new rows chooses a kernel, not the rows
    _compare(*b, max_new=0)
    assert torch.equal(one, _attend(*b))


@KINDS
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (16, 4), (63, 0), (64, 64), (65, 130), (100, 3), (4096, 4), (2**31 - 1, 2**31 - 1)])
@pytest.mark.parametrize("new,total", [([1, 1, 1, 1], [1, 65, 400, 2000]), ([130, 1, 300], [130, 777, 1000]), ([5, 9], [600, 601])])
def test_attention_window_and_sinks(kind, window, n_sink, new, total):
    page = 16
    q, pool, table, cu, total = _batch(kind, new, total, 2, 4, 128, page, 8)
    # keys between the sinks and the window of the request's first new row are gone: any code there, any exponent of blocks that hold
    # only such keys, and pages of only such keys are given back (their table entries point outside the pool)
    for b, t in enumerate(total):
        lo = max(0, t - new[b] - window + 1)
        j = torch.arange(min(n_sink, lo), lo, device=DEV)
        if j.numel():
            for c in (pool.k, pool.v):
                c.view(torch.int8)[0, table[b, j // page].long(), j % page] = 127        # e4m3's NaN
            whole = j[(j // 8 * 8 >= min(n_sink, lo)) & (j // 8 * 8 + 8 <= lo)]
            for i, e in enumerate((pool.k_exp, pool.v_exp)):
                e[0, table[b, whole // page].long(), whole % page // 8] = 127 if i else -128
        for p in range(-(-min(n_sink, lo) // page), lo // page):
            table[b, p] = 10**6 + p
    _compare(q, pool, table, cu, total, window, n_sink)
    _compare(q, pool, table, cu, total, window, n_sink, max_new=1)


@KINDS
@pytest.mark.parametrize("group,d", [(65, 128), (128, 128), (130, 64), (200, 128)])
def test_attention_of_many_query_heads(kind, group, d):
    b = _batch(kind, [1, 3, 40], [1, 500, 40], 2, group, d, 32, 16)
    _compare(*b)


@KINDS
@pytest.mark.parametrize("new", [[1] * 4, [20, 3, 1, 7]])
def test_attention_layers_missing_pages_and_room(kind, new):
    """The second of three layers; pages that are missing read as zeros; a batch larger than the room in q drops its last rows."""
    q, pool, table, cu, total = _batch(kind, new, [100, 37, 300, 64], 2, 4, 128, 16, 16, layers=3, layer=1)
    _compare(q, pool, table, cu, total, layer=1)
    table[0, 2], table[2, 0], table[2, 5] = -5, pool.n_pages, 2**31 - 1
    _compare(q, pool, table, cu, total, layer=1)
    full = _attend(q, pool, table, cu, total, layer=1)
    room = cu[-1] - 2
    part = _attend(q[:room], pool, table, cu, total, layer=1)
    assert ((part.float() - full[:room].float()).abs() <= 2.0 ** -7 * full[:room].float().abs() + 2.0 ** -8).all()
    short = _attend(q, pool, table[:, :4].contiguous(), cu, [min(t, 64) for t in total], layer=1)      # a table that ends at its last page
    assert short.isfinite().all()


@KINDS
def test_attention_of_a_long_request_and_of_many(kind):
    _compare(*_batch(kind, [1], [40000], 1, 8, 128, 64, 64, seed=3), weight=2.0 ** -11)
    _compare(*_batch(kind, [2, 300], [20000, 9000], 1, 4, 64, 16, 8, seed=4))
    rng = np.random.default_rng(0)
    total = rng.integers(1, 200, 600).tolist()
    _compare(*_batch(kind, [1] * 600, total, 2, 2, 64, 16, 16, seed=5), weight=2.0 ** -11)


@KINDS
@pytest.mark.parametrize("new", [1, 40])
def test_attention_with_exponents_far_apart(kind, new):
    """Blocks of values 2^-40 .. 2^40 apart in V and scores near zero: every block counts by what it holds."""
    H, group, d, page, block, n = 1, 4, 128, 16, 8, 200
    q, pool, table, cu, total = _batch(kind, [new], [n], H, group, d, page, block)
    e = torch.randint(-40, 41, pool.v_exp.shape, generator=_gen(9), device=DEV).to(torch.int8)
    pool.v_exp.copy_(e)
    pool.k_exp.copy_(pool.k_exp.clamp(-20, 0) - (e.abs() // 4))
    _compare(q, pool, table, cu, total)


@KINDS
@pytest.mark.parametrize("new", [1, 6, 40])
@pytest.mark.parametrize("low,high", [(-100, 60), (-100, -70), (-61, 80), (19, 80), (-100, 80)])
def test_attention_with_exponents_at_the_ends_of_what_is_allowed(kind, new, low, high):
    """Blocks of V at both ends, the large ones in turn of zeros only and seen: what the small ones give is not lost, whichever come first."""
    H, group, d, page, block, n = 2, 4, 128, 16, 8, 300
    for large_first in (False, True):
        for zeros in (False, True):
            q, pool, table, cu, total = _batch(kind, [new], [n], H, group, d, page, block)
            e = torch.full_like(pool.v_exp, low)
            late = torch.zeros(pool.v.shape[1], dtype=torch.bool, device=DEV)
            late[table[0, 4:11].long()] = True
            large = ~late if large_first else late
            e[:, large] = high
            pool.v_exp.copy_(e)
            if zeros:
                pool.v.view(torch.uint8)[:, large] = 0
            _compare(q, pool, table, cu, total)


@KINDS
@pytest.mark.parametrize("new", [1, 30])
def test_attention_of_queries_of_any_size(kind, new):
    """Rows of q from 2^-60 to 2^10, one of zeros, with channels 2^-20 of its largest: the same weights as in 64 bits."""
    q, pool, table, cu, total = _batch(kind, [new] * 3, [77, 300, 64], 2, 4, 128, 16, 16)
    for i, f in enumerate((2.0 ** -60, 1.0, 4.0)):
        q[cu[i]:cu[i + 1]] *= f
    q[cu[1]:cu[2], :, ::2] *= 2.0 ** -20
    q[cu[2]] = 0
    _compare(q, pool, table, cu, total)


@KINDS
def test_attention_a_flat_tail_behind_one_large_key(kind):
    """One key takes 2/3 of the weight and 30,000 keys of 2^-16 each share the rest: their weights are not lost."""
    H, group, d, page, n = 1, 8, 64, 64, 30001
    for new in (1, 4):
        q, pool, table, cu, total = _batch(kind, [new], [n + new - 1], H, group, d, page, 64)
        q.zero_()
        q[..., 0] = 1
        k = torch.zeros(1, n + new - 1, H, d, device=DEV)
        k[0, 0, 0, 0] = 10.75
        v = torch.full((1, n + new - 1, H, d), 1.0, device=DEV)
        v[0, 0] = -1.0
        j = torch.arange(n + new - 1, device=DEV)
        cb.cb_paged_store8(pool, k, v, table[0, j // page].long() * page + j % page)
        _compare(q, pool, table, cu, total, scale=1.0)


@KINDS
@pytest.mark.parametrize("new", [[1] * 20, [50, 1, 200]])
def test_attention_repeats_its_bits_on_streams_and_in_graphs(kind, new):
    """Two streams with a workspace each at once, and a captured call replayed while lengths grow."""
    total = [n + 40 * i for i, n in enumerate(new)]
    q, pool, table, cu, total = _batch(kind, new, [t + 30 for t in total], 2, 4, 128, 16, 16)
    want = _attend(q, pool, table, cu, total)
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.zeros_like(_workspace(128)) for _ in range(2)]
    outs = [[torch.empty_like(want) for _ in range(5)] for _ in range(2)]
    cu_t, total_t = _i32(cu), _i32(total)
    torch.cuda.synchronize()
    for i in range(5):
        for s, w, o in zip(streams, spaces, outs):
            cb.cb_paged_attention8(q, o[i], pool, 0, table, cu_t, total_t, 128 ** -0.5, w, max_new=max(new), stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for two in outs for o in two)
    out, graph = torch.empty_like(want), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cb.cb_paged_attention8(q, out, pool, 0, table, cu_t, total_t, 128 ** -0.5, spaces[0], max_new=max(new))
    for shrink in (0, 7, 30):
        total_t.copy_(_i32([t - shrink for t in total]))
        graph.replay()
        assert torch.equal(out, _attend(q, pool, table, cu, [t - shrink for t in total]))


# ---------------------------------------------------------------------------------------------------- sizes, batches, waits
@KINDS
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,block", [(8, 8), (16, 8), (32, 32), (64, 16), (128, 8), (128, 128), (256, 64), (256, 256)])
def test_attention_over_every_page_size(kind, d, page, block):
    """Decode and chunks, with and without a window, one slot of the last page used and all of them."""
    for new, total in (([1, 1, 2], [page, page + 1, 5 * page - 1]), ([70, 33], [3 * page + 70, 300])):
        b = _batch(kind, new, total, 2, 4, d, page, block, hnd=page >= 64, pad_rows=1, seed=page + block)
        _compare(*b)
        _compare(*b, window=page + 3, n_sink=5)


@KINDS
@pytest.mark.parametrize("new", [[1] * 6, [40, 1, 7, 100, 2, 33]])
def test_attention_of_the_later_requests_of_a_batch_by_themselves(kind, new):
    """Slices of a batch's tables: rows are counted from the batch's first, so q and out are the whole batch's."""
    total = [n + 50 * i for i, n in enumerate(new)]
    q, pool, table, cu, total = _batch(kind, new, total, 2, 4, 128, 16, 16)
    want = _attend(q, pool, table, cu, total)
    k, v = _plain(pool, 0)
    ref_out, tol = ref.attention(q, k, v, table, cu, total, 128 ** -0.5, weight=2.0 ** -8)
    for first in (2, 5):
        out = torch.full_like(want, 5.0)
        cb.cb_paged_attention8(q, out, pool, 0, table[first:], _i32(cu)[first:].contiguous(), _i32(total)[first:], 128 ** -0.5, _workspace(128),
                               max_new=max(new[first:]))
        assert (out[:cu[first]] == 5).all()
        assert ((out[cu[first]:].double() - ref_out[cu[first]:]).abs() <= tol[cu[first]:]).all()


@KINDS
@pytest.mark.parametrize("seed", range(12))
def test_attention_of_random_shapes(kind, seed):
    rng = np.random.default_rng(seed)
    page = int(rng.choice([8, 16, 32, 64, 128, 256]))
    block = int(rng.choice([b for b in (8, 16, 32, 64, 128, 256) if b <= page]))
    n = int(rng.integers(1, 9))
    new = rng.integers(0, rng.choice([2, 5, 40, 300]), n).tolist()
    total = [x + int(rng.integers(0, 700)) for x in new]
    window, n_sink = (0, 0) if rng.random() < 0.5 else (int(rng.integers(1, 400)), int(rng.integers(0, 140)))
    b = _batch(kind, new, total, int(rng.integers(1, 5)), int(rng.choice([1, 2, 3, 5, 8, 12])), int(rng.choice([64, 128])), page, block,
               hnd=bool(rng.random() < 0.5), pad_rows=int(rng.integers(0, 4)), seed=seed, grow=2.0)
    if b[0].shape[0]:
        _compare(*b, window=window, n_sink=n_sink, max_new=int(rng.choice([0, max(new + [1])])))


@KINDS
@pytest.mark.parametrize("seed", range(12))
def test_store_of_random_shapes(kind, seed):
    """Several calls of a ragged batch: some requests go on inside a block, some begin, some write their last rows again."""
    rng = np.random.default_rng(seed)
    page = int(rng.choice([8, 16, 32, 64, 128, 256]))
    block = int(rng.choice([b for b in (8, 16, 32, 64, 128, 256) if b <= page]))
    n, L, H, d = int(rng.integers(1, 6)), int(rng.integers(1, 4)), int(rng.integers(1, 11)), int(rng.choice([64, 128]))
    dtype = [torch.bfloat16, torch.float32][seed % 2]
    length = rng.integers(1, 300, n)
    pages = [-(-int(x) // page) for x in length]
    order = rng.permutation(sum(pages) + 2)
    own = np.split(order[:sum(pages)], np.cumsum(pages)[:-1])
    pool = _pool(kind, L, sum(pages) + 2, page, block, H, d, hnd=bool(rng.random() < 0.5), seed=seed)
    state = _state(pool)
    at = [0] * n
    for call in range(4):
        slot = []
        for b in range(n):
            first = max(0, at[b] - int(rng.integers(0, 3))) if call else 0
            last = int(length[b]) if call == 3 else min(int(length[b]), at[b] + int(rng.integers(0, 120)))
            slot += [int(own[b][t // page]) * page + t % page for t in range(first, last)] + [-1] * int(rng.integers(0, 3))
            at[b] = max(at[b], last)
        if slot:
            _store(pool, state, _rows(L, len(slot), H, d, dtype, 100 * seed + call, spread=2.0), slot)


@KINDS
@pytest.mark.parametrize("new,total,d,page,window", [([70, 9], [3000, 700], 128, 16, 0), ([300], [9000], 128, 128, 0), ([300, 40], [5000, 40], 64, 8, 1000)])
def test_attention_waits_that_run_out(kind, new, total, d, page, window):
    """Nothing copied, or consumers that give up while copies are in flight: the status says so, and the next call is right."""
    b = _batch(kind, new, total, 2, 8, d, page, 8)
    want = _compare(*b, window=window, n_sink=2)
    try:
        for hook in (dict(starve_producer=True), dict(consumers_give_up=True)):
            cb.cb_test_hooks(poll_limit=2000, **hook)
            _attend(*b, window=window, n_sink=2)
            with pytest.raises(cb.CbError) as e:
                cb.cb_last_device_status()
            assert e.value.status == cb.CB_ERR_TIMEOUT
            cb.cb_test_hooks()
            assert torch.equal(_compare(*b, window=window, n_sink=2), want)
    finally:
        cb.cb_test_hooks()


# ---------------------------------------------------------------------------------------------------- together
@KINDS
def test_a_served_target_cache(kind):
    """Mapped prompts of two requests enter the pages quantised, twelve tokens follow (tables, rotation, store, attention over
    captured steps), then the cache is read back and put into a bf16 pool, where the ordinary attention says the same."""
    L, H, group, d, page, block = 3, 2, 4, 128, 16, 16
    lens, steps = [37, 64], 12
    B, cols = len(lens), 8
    g = _gen(11)
    pool = _pool(kind, L, 16, page, block, H, d)
    free = torch.randperm(16, generator=g, device=DEV).to(torch.int32)
    table = torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
    room = sum(lens) + 3
    cached, new = _i32([0] * B), _i32(lens)
    cu, total, used = _i32([0] * (B + 1)), _i32([0] * B), _i32([0])
    pos, slot = _i32([0] * room), torch.zeros(room, dtype=torch.int64, device=DEV)
    cb.cb_page_tables(cached, new, page, free, table, cu, total, pos, slot, used)
    mapped = [torch.randn(L, room, H, d, generator=g, device=DEV) for _ in range(2)]               # as cb_apply's fp32 output
    cb.cb_paged_store8(pool, mapped[0], mapped[1], slot)
    taken = int(used[0])
    ws = torch.zeros(cb.cb_paged_attention8_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    pos1, slot1 = _i32([0] * B), torch.zeros(B, dtype=torch.int64, device=DEV)
    free1 = free[taken:].clone()
    cached.copy_(_i32(lens))
    new.fill_(1)
    kv = [torch.empty(L, B, H, d, dtype=torch.bfloat16, device=DEV) for _ in range(3)]             # keys, rotated keys, values
    qs, outs = (torch.empty(L, B, H * group, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    layers = [cb.PagePool8(*(x[l:l + 1] for x in (pool.k, pool.v, pool.k_exp, pool.v_exp))) for l in range(L)]

    def step():
        cb.cb_page_tables(cached, new, page, free1, table, cu, total, pos1, slot1, used)
        cb.cb_rope_axes(kv[0], kv[1], pos1[None], [64], 1e6)
        for l in range(L):
            cb.cb_paged_store8(layers[l], kv[1][l:l + 1], kv[2][l:l + 1], slot1)
            cb.cb_paged_attention8(qs[l], outs[l], pool, l, table, cu, total, d ** -0.5, ws, max_new=1)

    for x in (*kv, qs):
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
    keep = [x.clone() for x in (pool.k, pool.v, pool.k_exp, pool.v_exp)], table.clone()
    step()                                                                                          # loads the kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((pool.k, pool.v, pool.k_exp, pool.v_exp), keep[0]):
        x.copy_(y)
    table.copy_(keep[1])
    at = 0
    for i in range(steps):
        for x in (*kv, qs):
            x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        graph.replay()
        n = int(used[0])
        free1[:free1.numel() - n] = free1[n:].clone()
        at += n
        now = total.tolist()
        for l in range(L):
            k, v = _plain(pool, l)
            want, tol = ref.attention(qs[l], k, v, table, [0, 1, 2], now, d ** -0.5)
            assert ((outs[l].double() - want).abs() <= tol).all(), (i, l)
        cached.copy_(total)
    # the cache back in bf16, in pages of its own
    back = torch.cat([table[b, torch.arange(n, device=DEV) // page].long() * page + torch.arange(n, device=DEV) % page for b, n in enumerate(now)])
    rows = [torch.empty(L, back.numel(), H, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cb.cb_paged_load8(pool, rows[0], rows[1], back)
    wide = [torch.zeros(L, 16, page, H, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cb.cb_paged_store(cb.PagePool(*wide), rows[0], rows[1], back)
    big = torch.zeros(cb.cb_paged_attention_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(outs[0])
    for l in range(L):
        cb.cb_paged_attention(qs[l], out, cb.PagePool(*wide), l, table, cu, total, d ** -0.5, big, max_new=1)
        want, tol = paged_ref.attention(qs[l], wide[0][l], wide[1][l], table, [0, 1, 2], now, d ** -0.5)
        assert ((out.double() - want).abs() <= tol).all()
        assert ((out.double() - outs[l].double()).abs() <= 2 * tol).all()


@KINDS
def test_calls_refuse_another_device_and_a_wrong_stream(kind):
    pool = _pool(kind, 1, 3, 8, 8, 2, 64)
    x = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        cb.cb_paged_store8(pool, x, x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(cb.CbError):
        cb.cb_paged_load8(pool, x, x, torch.zeros(2, dtype=torch.int64, device=DEV))
