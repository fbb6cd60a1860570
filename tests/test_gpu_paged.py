"""Paged target cache on the GPU: page tables, store, rotary positions with several axes and attention over the pages,
each against a plain 64-bit form, then a run of them together behind the mapping calls."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2609_00891_b200 import binding as cb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------------------------------- page tables
def _tables(cached, new, page, n_free=None, cols=None, pad=0, seed=0, stride_pad=0):
    rng = np.random.default_rng(seed)
    B = len(cached)
    held = [-(-max(c, 0) // page) for c in cached]
    need = [-(-(max(c, 0) + max(n, 0)) // page) for c, n in zip(cached, new)]
    cols = max(need + [1]) + 1 if cols is None else cols
    ids = rng.permutation(sum(need) + 40).astype(np.int32)
    table = np.full((B, cols), -77, np.int32)
    at = 0
    for b in range(B):
        k = min(held[b], cols)
        table[b, :k] = ids[at:at + k]
        at += held[b]
    fresh = sum(need) - sum(held)
    free = ids[at:at + (fresh + 3 if n_free is None else n_free)]
    n_rows = sum(max(n, 0) for n in new) + pad
    want = ref.tables(cached, new, page, free.tolist(), table, n_rows)
    wide = torch.full((max(B, 1), cols + stride_pad), -77, dtype=torch.int32, device=DEV)[:B]
    wide[:, :cols] = torch.from_numpy(table).to(DEV)
    bt = wide[:, :cols]
    out = {"cu": _i32([-9] * (B + 1)), "total": _i32([-9] * B), "pos": _i32([-9] * n_rows),
           "slot": torch.full((n_rows,), -9, dtype=torch.int64, device=DEV), "used": _i32([-9])}
    args = (_i32(cached), _i32(new), page, torch.from_numpy(free.copy()).to(DEV), bt, out["cu"], out["total"], out["pos"], out["slot"], out["used"])
    return want, out, bt, wide, args


def _check_tables(want, out, bt):
    assert np.array_equal(bt.cpu().numpy(), want["table"])
    for k in ("cu", "total", "pos", "slot"):
        assert np.array_equal(out[k].cpu().numpy(), want[k]), k
    assert int(out["used"][0]) == want["used"]


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("cached,new,pad", [
    ([0], [1], 0), ([0], [0], 3), ([15, 16, 17, 0, 255, 256], [1, 1, 1, 1, 1, 1], 5), ([0, 0, 0], [300, 0, 7], 0),
    ([5, 0, 1000], [2049, 4096, 1], 100), ([-3, 4], [2, -1], 1)])
def test_tables(page, cached, new, pad):
    want, out, bt, wide, args = _tables(cached, new, page, pad=pad, stride_pad=3)
    for _ in range(2):                                     # the same call again writes the same
        cb.cb_page_tables(*args)
        _check_tables(want, out, bt)
    assert (wide[:, bt.shape[1]:] == -77).all()


@pytest.mark.parametrize("B", [1023, 1024, 1025, 2500])
def test_tables_many_requests(B):
    rng = np.random.default_rng(B)
    want, out, bt, _, args = _tables(rng.integers(0, 90, B).tolist(), rng.integers(0, 9, B).tolist(), 16, pad=11)
    cb.cb_page_tables(*args)
    _check_tables(want, out, bt)


def test_tables_short_of_pages_and_of_columns():
    want, out, bt, _, args = _tables([0, 30, 0], [40, 10, 40], 8, n_free=6)
    cb.cb_page_tables(*args)
    _check_tables(want, out, bt)
    assert int(out["used"][0]) > 6 and (out["slot"] == -1).any()
    want, out, bt, _, args = _tables([0, 30, 0], [40, 10, 40], 8, cols=3)
    cb.cb_page_tables(*args)
    _check_tables(want, out, bt)


def test_tables_room_for_fewer_rows_and_no_requests():
    want, out, bt, _, args = _tables([3, 4], [20, 30], 16)
    args = list(args)
    args[7], args[8] = out["pos"][:25], out["slot"][:25]
    out["pos"][25:], out["slot"][25:] = -9, -9
    cb.cb_page_tables(*args)
    assert np.array_equal(out["pos"][:25].cpu().numpy(), want["pos"][:25]) and (out["pos"][25:] == -9).all()
    assert np.array_equal(out["slot"][:25].cpu().numpy(), want["slot"][:25]) and (out["slot"][25:] == -9).all()
    want, out, bt, _, args = _tables([], [], 16, pad=4)
    cb.cb_page_tables(*args)
    _check_tables(want, out, bt)


@pytest.mark.parametrize("at", [1, 2, 3])
def test_tables_into_rows_that_are_not_16_byte_aligned(at):
    want, out, bt, _, args = _tables([5, 0, 1000, 30], [2049, 7, 1, 600], 16, pad=9)
    n = out["pos"].numel()
    pos, slot = torch.full((n + at + 2,), -9, dtype=torch.int32, device=DEV), torch.full((n + at + 2,), -9, dtype=torch.int64, device=DEV)
    out["pos"], out["slot"] = pos[at:at + n], slot[at:at + n]
    cb.cb_page_tables(*args[:7], out["pos"], out["slot"], out["used"])
    _check_tables(want, out, bt)
    for x in (pos, slot):
        assert (x[:at] == -9).all() and (x[at + n:] == -9).all()


# ---------------------------------------------------------------------------------------------------- store
def _pool(L, pages, page, H, d, hnd, fill=None, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    shape = (L, pages, H, page, d) if hnd else (L, pages, page, H, d)
    both = []
    for _ in range(2):
        x = torch.randn(shape, generator=g, device=DEV).bfloat16() if fill is None else torch.full(shape, fill, dtype=torch.bfloat16, device=DEV)
        both.append(x.transpose(2, 3) if hnd else x)
    return both


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("L,T,H,d,page,hnd", [(1, 1, 1, 64, 8, False), (3, 37, 2, 128, 16, True), (2, 200, 5, 64, 256, False), (64, 33, 8, 128, 64, False)])
def test_store(dtype, L, T, H, d, page, hnd):
    pages = T // page + 3
    k, v = _pool(L, pages, page, H, d, hnd)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    # source rows of a wider tensor, head-major: the strides are not the dense ones
    src = [torch.randn(L, H, T + 2, d, generator=g, device=DEV).to(dtype).transpose(1, 2)[:, :T] for _ in range(2)]
    slot = torch.randperm(pages * page, generator=g, device=DEV)[:T]
    slot[::5] = -1
    if T > 8:
        slot[3], slot[7] = pages * page, 1 << 40           # past the pool: skipped
    want = [k.clone(), v.clone()]
    live = (slot >= 0) & (slot < pages * page)
    for w, s in zip(want, src):
        w[:, slot[live] // page, slot[live] % page] = s[:, live].bfloat16()
    cb.cb_paged_store(cb.PagePool(k, v), src[0], src[1], slot)
    assert torch.equal(k.view(torch.int16), want[0].view(torch.int16)) and torch.equal(v.view(torch.int16), want[1].view(torch.int16))


def test_store_nothing():
    k, v = _pool(2, 3, 8, 2, 64, False)
    before = k.clone()
    e = torch.empty(2, 0, 2, 64, dtype=torch.bfloat16, device=DEV)
    cb.cb_paged_store(cb.PagePool(k, v), e, e, torch.empty(0, dtype=torch.int64, device=DEV))
    assert torch.equal(k, before)


def test_store_into_a_pool_past_32_bit_offsets():
    L, pages, page, H, d = 1, 66000, 64, 8, 128            # 4.3e9 elements
    k = torch.empty(L, pages, page, H, d, dtype=torch.bfloat16, device=DEV)
    pool = cb.PagePool(k, k)
    rows = torch.randn(L, 5, H, d, device=DEV).bfloat16()
    slot = torch.tensor([0, pages * page - 1, 33000 * page, (pages - 1) * page, 17], device=DEV)
    cb.cb_paged_store(pool, rows, rows, slot)
    assert torch.equal(k[0, slot // page, slot % page], rows[0])
    # and attention reads them there
    q = torch.randn(1, 8, d, device=DEV).bfloat16()
    out = torch.empty_like(q)
    table, cu, total = _i32([[pages - 1]]), _i32([0, 1]), _i32([1])
    cb.cb_paged_attention(q, out, pool, 0, table, cu, total, 0.1, _workspace(d))
    assert torch.equal(out[0], k[0, pages - 1, 0])


# ---------------------------------------------------------------------------------------------------- rotary positions
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("L,T,H,d,sections,far", [
    (1, 1, 1, 64, [32], 10), (2, 33, 3, 64, [12, 10, 10], 5000), (3, 70, 5, 128, [16, 24, 24], 1 << 20), (1, 257, 64, 128, [20, 20, 24], 2**31 - 1),
    (40, 9, 8, 128, [0, 30, 34, 0], 100000)])
def test_rope_axes(L, T, H, d, sections, far, interleaved, inverse):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn(L, T, H, d, generator=g, device=DEV).bfloat16()
    pos = torch.randint(0, far, (len(sections), T), generator=g, device=DEV, dtype=torch.int32)
    if far > 1 << 20:
        pos[:, ::3] *= -1
    base = 1e6
    want = ref.rope(x, pos, sections, base, interleaved, inverse)
    # rounding to bf16 (2^-8 of the value), the angle's 2^-22 turns and the polynomials' 2^-22 on the pair's length, and the
    # frequency's rounding from double: position times 2^-53 times the angle's rate, twice (library and reference)
    size = torch.sqrt(x[..., :d // 2].double() ** 2 + x[..., d // 2:].double() ** 2).repeat(1, 1, 1, 2)
    tol = want.abs() * 2.0 ** -8 + size * (2 * 3.1416 * 2.0 ** -22 + 2.0 ** -21 + 4 * far * 2.0 ** -53)
    # a head-major output with room behind every row, then in place
    room = torch.full((L, H, T, d + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    out = room[..., :d].transpose(1, 2)
    cb.cb_rope_axes(x, out, pos, sections, base, interleaved=interleaved, inverse=inverse)
    assert ((out.double() - want).abs() <= tol).all()
    assert (room[..., d:] == 7).all()
    y = x.clone()
    cb.cb_rope_axes(y, y, pos, sections, base, interleaved=interleaved, inverse=inverse)
    assert torch.equal(y, out)


def test_rope_one_axis_agrees_with_the_ordinary_embedding():
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    x = torch.randn(2, 50, 4, 128, generator=g, device=DEV).bfloat16()
    pos = torch.arange(50, dtype=torch.int32, device=DEV) * 3
    y = x.clone()
    cb.cb_rope_rotate(y, pos, 1e6, False)
    out = torch.empty_like(x)
    cb.cb_rope_axes(x, out, pos[None], [64], 1e6)
    # Before rounding each is off by its angle's 2^-22 turns and the polynomials' 2^-22, on the pair's length (positions up
    # to 150 leave the 0.32 fixed-point frequency's 2^-33 turns a step out of it); both then round to bf16: at most one step,
    # 2^-7 of the value, apart.  Where the two products cancel, the value is small and the first term is what counts.
    size = torch.sqrt(x[..., :64].double() ** 2 + x[..., 64:].double() ** 2).repeat(1, 1, 1, 2)
    tol = 2.0 ** -7 * y.double().abs() + 2 * size * (2 * 3.1416 * 2.0 ** -22 + 2.0 ** -21)
    assert ((out.double() - y.double()).abs() <= tol).all()


def test_rope_adjoint_is_the_inverse_form():
    """<y, R x> = <R' y, x>: the inverse form gives the gradient of the forward one."""
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    x, y = (torch.randn(1, 40, 3, 64, generator=g, device=DEV).bfloat16() for _ in range(2))
    pos = torch.randint(0, 9000, (3, 40), generator=g, device=DEV, dtype=torch.int32)
    rx, ry = torch.empty_like(x), torch.empty_like(y)
    cb.cb_rope_axes(x, rx, pos, [12, 10, 10], 1e4)
    cb.cb_rope_axes(y, ry, pos, [12, 10, 10], 1e4, inverse=True)
    a, b = (y.double() * rx.double()).sum(-1), (ry.double() * x.double()).sum(-1)
    size = (y.double().abs() * rx.double().abs()).sum(-1) + (ry.double().abs() * x.double().abs()).sum(-1)
    assert ((a - b).abs() <= 2.0 ** -8 * size + 1e-4).all()


# ---------------------------------------------------------------------------------------------------- attention
_ws = {}


def _workspace(d):
    if d not in _ws:
        _ws[d] = torch.zeros(cb.cb_paged_attention_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    return _ws[d]


def _batch(new, total, H, group, d, page, hnd=False, pad_rows=0, seed=0, wild=True, layers=1, layer=0):
    """A pool whose unused rows and pages are NaN, and the batch's queries in a wider tensor."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    need = [-(-t // page) for t in total]
    pages = sum(need) + 2
    k, v = _pool(layers, pages, page, H, d, hnd, fill=float("nan") if wild else 0.0)
    cols = max(need + [1]) + 2
    table = torch.full((len(new), cols), -1, dtype=torch.int32, device=DEV)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    at = 0
    scale = torch.exp(0.5 * torch.randn(H, d, generator=g, device=DEV))
    for b, t in enumerate(total):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        j = torch.arange(t, device=DEV)
        if t:
            k[layer, table[b, j // page].long(), j % page] = (torch.randn(t, H, d, generator=g, device=DEV) * scale).bfloat16()
            v[layer, table[b, j // page].long(), j % page] = (torch.randn(t, H, d, generator=g, device=DEV) + 0.25).bfloat16()
    T = sum(new)
    q = torch.randn(T + pad_rows, H * group, d + 8, generator=g, device=DEV).bfloat16()[..., :d]
    if pad_rows:
        q[T:] = float("nan")
    cu = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
    return q, k, v, table, cu, total


def _attend(q, k, v, table, cu, total, window=0, n_sink=0, max_new=None, layer=0, scale=None, out=None):
    T, Hq, d = q.shape
    if out is None:
        out = torch.full((Hq, T, d), 5.0, dtype=torch.bfloat16, device=DEV).transpose(0, 1)   # head-major
    scale = d ** -0.5 if scale is None else scale
    most = max([b - a for a, b in zip(cu, cu[1:])] + [0]) if max_new is None else max_new
    cb.cb_paged_attention(q, out, cb.PagePool(k, v), layer, table, _i32(cu), _i32(total), scale, _workspace(d), max_new=most,
                          window=window, n_sink=n_sink)
    return out


def _compare(q, k, v, table, cu, total, window=0, n_sink=0, max_new=None, layer=0, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    out = _attend(q, k, v, table, cu, total, window, n_sink, max_new, layer, scale)
    want, tol = ref.attention(q, k[layer], v[layer], table, cu, total, scale, window, n_sink)
    n = cu[-1]
    err = (out[:n].double() - want[:n]).abs()
    bad = ~(err <= tol[:n])
    assert not bad.any(), (int(bad.sum()), err.max().item(), bad.nonzero()[:4].tolist())
    assert (out[n:] == 5).all()
    cb.cb_last_device_status()
    assert int(_workspace(q.shape[2])[:8192].sum()) == 0            # the join counters are ready for the next call
    return out


DECODE = [1, 2, 7, 8, 15, 16, 17, 63, 64, 65, 127, 128, 129, 1000]


@pytest.mark.parametrize("H,group,d,page,hnd", [(1, 1, 64, 8, False), (2, 5, 128, 16, True), (8, 8, 128, 16, False), (3, 2, 64, 64, False),
                                                (2, 16, 128, 32, False), (1, 17, 128, 128, True), (2, 40, 64, 256, False), (1, 70, 128, 16, False)])
def test_attention_single_tokens(H, group, d, page, hnd):
    b = _batch([1] * len(DECODE), DECODE, H, group, d, page, hnd, pad_rows=3)
    _compare(*b)


@pytest.mark.parametrize("new,total", [
    ([5], [5]), ([1, 0, 33, 64, 65, 130], [1, 0, 40, 64, 300, 131]), ([128, 129, 1, 256, 257], [128, 500, 700, 256, 258]),
    ([700], [1500]), ([0, 0, 3], [0, 10, 3]), ([4, 4, 4, 4], [4, 100, 1000, 77])])
@pytest.mark.parametrize("H,group,d,page,hnd", [(2, 5, 128, 16, False), (1, 8, 64, 32, True), (3, 1, 128, 128, False)])
def test_attention_chunks(new, total, H, group, d, page, hnd):
    b = _batch(new, total, H, group, d, page, hnd, pad_rows=2)
    one = _compare(*b)
    # the bound on new rows chooses a kernel, not the rows
    _compare(*b, max_new=1)
    _compare(*b, max_new=0)
    assert torch.equal(one, _attend(*b))


@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (16, 4), (63, 0), (64, 64), (65, 130), (100, 3), (4096, 4), (2**31 - 1, 2**31 - 1)])
@pytest.mark.parametrize("new,total", [([1, 1, 1, 1], [1, 65, 400, 2000]), ([130, 1, 300], [130, 777, 1000]), ([5, 9], [600, 601])])
def test_attention_window_and_sinks(window, n_sink, new, total):
    q, k, v, table, cu, total = _batch(new, total, 2, 4, 128, 16)
    # keys between the sinks and the window of the request's first new row are gone: NaN there, and pages that hold only
    # such keys are given back (their table entries point outside the pool)
    for b, t in enumerate(total):
        lo = max(0, t - new[b] - window + 1)
        j = torch.arange(min(n_sink, lo), lo, device=DEV)
        if j.numel():
            k[0, table[b, j // 16].long(), j % 16] = float("nan")
            v[0, table[b, j // 16].long(), j % 16] = float("nan")
    for b, t in enumerate(total):
        lo = max(0, t - new[b] - window + 1)
        for p in range(-(-min(n_sink, lo) // 16), lo // 16):
            table[b, p] = 10**6 + p
    _compare(q, k, v, table, cu, total, window, n_sink)
    _compare(q, k, v, table, cu, total, window, n_sink, max_new=1)


@pytest.mark.parametrize("group,d", [(65, 128), (100, 64), (128, 128), (130, 64), (200, 128)])
def test_attention_many_query_heads_per_kv_head(group, d):
    """Up to 128 a tile holds whole tokens (one or two of them here); above that the warp-level kernel takes 64 rows a unit."""
    b = _batch([1, 1, 1], [1, 90, 700], 2, group, d, 16, pad_rows=1)
    _compare(*b)
    b = _batch([3, 0, 9], [3, 0, 400], 1, group, d, 32, hnd=True)
    _compare(*b)
    _compare(*b, window=50, n_sink=2)


@pytest.mark.parametrize("max_new", [1, 0])
def test_attention_more_requests_than_fit_shared_memory(max_new):
    """13,000 and 30,000 requests of one row each: the row's output is its own value."""
    for B in (13000, 30000):
        d = 64
        k, v = _pool(1, B, 8, 1, d, False, seed=1)
        q = torch.randn(B, 1, d, device=DEV).bfloat16()
        out = torch.zeros_like(q)
        table = torch.randperm(B, device=DEV).int()[:, None]
        cu = torch.arange(B + 1, dtype=torch.int32, device=DEV)
        cb.cb_paged_attention(q, out, cb.PagePool(k, v), 0, table, cu, torch.ones(B, dtype=torch.int32, device=DEV), 0.1, _workspace(d), max_new=max_new)
        assert torch.equal(out, v[0, table[:, 0].long(), 0])


def test_attention_no_rows_in_a_padded_batch():
    q, k, v, table, cu, total = _batch([0, 0], [20, 0], 2, 4, 128, 16)
    q = torch.full((5, 8, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    for max_new in (1, 0):
        out = torch.full_like(q, 5.0)
        _attend(q, k, v, table, cu, total, max_new=max_new, out=out)
        assert (out == 5).all()


@pytest.mark.parametrize("new,total", [([1, 1, 1], [40, 300, 90]), ([70, 1, 90], [100, 300, 90])])
def test_attention_strides_and_pages_outside_the_pool(new, total):
    q, k, v, table, cu, total = _batch(new, total, 2, 5, 128, 16, wild=False)
    k.nan_to_num_()
    v.nan_to_num_()
    wide = torch.full((len(new), table.shape[1] + 5), 3, dtype=torch.int32, device=DEV)
    wide[:, : table.shape[1]] = table
    table = wide[:, : table.shape[1]]                       # rows of a wider table
    table[0, 1], table[1, 3], table[2, 0] = -5, k.shape[1], 2**31 - 1
    heads = torch.randn(10, cu[-1], 128, device=DEV).bfloat16().transpose(0, 1)      # head-major queries
    _compare(heads, k, v, table, cu, total)


def test_attention_rows_that_see_nothing():
    # a cache shorter than the chunk: the first rows have negative positions
    q, k, v, table, cu, _ = _batch([6, 80, 3], [6, 80, 3], 2, 4, 128, 16)
    for total in ([2, 10, 0], [0, 0, 0], [1, 64, 2]):
        out = _compare(q, k, v, table, cu, total)
        assert (out[: 6 - total[0]] == 0).all()


@pytest.mark.parametrize("H,group,d", [(1, 8, 128), (2, 1, 64), (1, 33, 128)])
def test_attention_long_caches_are_split_and_joined(H, group, d):
    b = _batch([1, 1, 2], [30011, 64, 5000], H, group, d, 16)
    one = _compare(*b)
    for _ in range(3):
        assert torch.equal(one, _attend(*b))              # joined in a fixed order
    b = _batch([40, 3], [20011, 9000], H, group, d, 64)
    one = _compare(*b)
    assert torch.equal(one, _attend(*b))


def test_attention_many_requests():
    rng = np.random.default_rng(0)
    total = rng.integers(1, 60, 1500).tolist()
    new = [int(rng.integers(0, t + 1)) if i % 3 == 0 else 1 for i, t in enumerate(total)]
    b = _batch(new, total, 1, 4, 64, 16)
    _compare(*b, max_new=1)
    _compare(*b)


@pytest.mark.parametrize("new,total", [([1, 0, 33, 64, 65, 130], [1, 0, 40, 64, 300, 131]), ([700], [1500]), ([1, 2, 1], [255, 257, 900])])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (100, 3), (1, 0), (300, 130)])
@pytest.mark.parametrize("d,page,hnd", [(128, 8, False), (128, 256, True), (64, 8, True), (64, 256, False)])
def test_attention_smallest_and_largest_pages(d, page, hnd, window, n_sink, new, total):
    """Both kernels with sixteen boxes a tile and with boxes that start inside a page, windows and sinks over 64-channel heads."""
    b = _batch(new, total, 2, 8, d, page, hnd, pad_rows=1)
    one = _compare(*b, window=window, n_sink=n_sink, max_new=0)
    assert torch.equal(one, _attend(*b, window=window, n_sink=n_sink, max_new=0))
    _compare(*b, window=window, n_sink=n_sink, max_new=2)


@pytest.mark.parametrize("new", [[3, 9, 4], [2, 300, 1], [3, 1 << 28, 1 << 28]])
@pytest.mark.parametrize("H,group,d", [(2, 8, 128), (1, 16, 64), (2, 5, 64)])
def test_attention_rows_past_the_room_are_dropped(new, H, group, d):
    """A batch with more rows than q has room for, as the tables of a captured step describe it."""
    room, before = 7, [10, 20, 30]                          # rows of q; keys in the cache before the step
    kept = [min(n, room - at) for n, at in zip(new, (0, new[0], room))]
    q, k, v, table, cu, total = _batch(kept[:2] + [0], [b + n for b, n in zip(before, kept)], H, group, d, 16)
    assert cu[-1] == room
    want, tol = ref.attention(q, k[0], v[0], table, cu, total, d ** -0.5)
    all_cu = np.concatenate([[0], np.cumsum(new)]).tolist()
    for max_new in (1, 0, 1 << 30):
        out = _attend(q, k, v, table, all_cu, [b + n for b, n in zip(before, new)], max_new=max_new)
        assert ((out.double() - want).abs() <= tol).all()
        assert int(_workspace(d)[:8192].sum()) == 0


@pytest.mark.parametrize("heads,group,new,total", [(1, 1, 150 * 256, 2_000_003), (2, 1, 40_100, 2_000_003), (1, 8, 12_000, 1_500_001)])
def test_attention_pieces_longer_than_any_wait_within_a_tile(heads, group, new, total):
    """Blocks with one or several pieces of 20 ms and more: the warps that wait from piece to piece outlast them."""
    d, page = 64, 256
    pages = -(-total // page)
    k, v = _pool(1, pages, page, heads, d, False, seed=2)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    q = torch.randn(new, heads * group, d, generator=g, device=DEV).bfloat16()
    table = torch.randperm(pages, generator=g, device=DEV).int()[None]
    out = _attend(q, k, v, table, [0, new], [total], max_new=0)
    cb.cb_last_device_status()
    assert int(_workspace(d)[:8192].sum()) == 0
    rows = torch.tensor([0, 1, 255, 256, new // 2, new - 1], device=DEV)
    for h in range(heads):
        kd, vd = (x[0][table[0].long()].flatten(0, 1)[:total, h].double() for x in (k, v))
        for r in rows.tolist():
            n = total - new + r + 1
            qr = q[r, h * group:(h + 1) * group].double()
            s = qr @ kd[:n].T * d ** -0.5
            w = torch.softmax(s, -1)
            want, size = w @ vd[:n], w @ vd[:n].abs()
            # as in the plain form's tolerance, and the fp32 sums of n weights and products (in tiles of 128, then one tile after
            # the other): n / 128 + 128 roundings of 2^-24, of the sum and of the weighted values
            worst = float((qr.abs() @ kd[:n].abs().T).max()) * d ** -0.5
            tol = want.abs() * 2.0 ** -8 + size * (2.0 ** -8 + 2 * (2 * d * 2.0 ** -24 * worst + 2.0 ** -20) + 2 * (n / 128 + 128) * 2.0 ** -24)
            assert ((out[r, h * group:(h + 1) * group].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("new", [[5, 70, 1, 1, 33], [1, 1, 1, 1, 1, 1], [600, 3, 0, 2], [0, 0, 20, 300]])
@pytest.mark.parametrize("H,group,d", [(2, 1, 128), (1, 5, 64), (2, 8, 128), (1, 130, 64)])
def test_attention_later_requests_of_a_batch_by_themselves(H, group, d, new):
    """Slices of the tables of a batch, with all of its queries: the first row is not row 0, and rows before it stay as they are."""
    q, k, v, table, cu, total = _batch(new, [n + 40 * b for b, n in enumerate(new)], H, group, d, 16)
    whole, tol = ref.attention(q, k[0], v[0], table, cu, total, d ** -0.5)
    for first, last in ((1, len(new)), (2, len(new)), (len(new) - 1, len(new)), (1, 3)):
        for max_new in (1, 0):
            out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device=DEV)
            _attend(q, k, v, table[first:last], cu[first:last + 1], total[first:last], max_new=max_new, out=out)
            a, b = cu[first], cu[last]
            assert ((out[a:b].double() - whole[a:b]).abs() <= tol[a:b]).all()
            assert (out[:a] == 5).all() and (out[b:] == 5).all()
            assert int(_workspace(d)[:8192].sum()) == 0


def test_attention_large_scores_and_layers():
    q, k, v, table, cu, total = _batch([1, 3], [200, 100], 2, 4, 128, 16, layers=3, layer=2)
    _compare(q * 30, k, v, table, cu, total, layer=2)


def test_attention_nan_and_infinity_reach_only_their_rows():
    q, k, v, table, cu, total = _batch([1, 1], [100, 100], 1, 2, 64, 16)
    want = _attend(q, k, v, table, cu, total).clone()
    q2 = q.clone()
    q2[0, 1, 3] = float("nan")
    out = _attend(q2, k, v, table, cu, total)
    assert out[0, 1].isnan().all() and torch.equal(out[0, 0], want[0, 0]) and torch.equal(out[1], want[1])
    v[0, table[1, 2].long(), 5, 0, 7] = float("inf")
    out = _attend(q, k, v, table, cu, total)
    assert torch.isinf(out[1, :, 7]).all() and torch.isfinite(out[0]).all() and torch.isfinite(out[1, :, :7]).all()


def test_attention_on_another_stream_and_in_a_graph_whose_lengths_grow():
    page, H, group, d = 16, 2, 4, 128
    q, k, v, table, cu, total = _batch([1, 1], [150, 333], H, group, d, page)
    out = torch.full((2, H * group, d), 5.0, dtype=torch.bfloat16, device=DEV)
    ws, cu_d, total_d, pool = _workspace(d), _i32(cu), _i32([100, 200]), cb.PagePool(k, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cb.cb_paged_attention(q, out, pool, 0, table, cu_d, total_d, 0.1, ws, max_new=1)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cb.cb_paged_attention(q, out, pool, 0, table, cu_d, total_d, 0.1, ws, max_new=1)
    for lens in ([100, 200], [150, 333], [1, 17]):
        total_d.copy_(_i32(lens))
        g.replay()
        want, tol = ref.attention(q, k[0], v[0], table, cu, lens, 0.1)
        assert ((out.double() - want).abs() <= tol).all()


def test_attention_two_calls_at_once():
    """Two streams with a workspace each, both kernels in flight together, against the same calls one after the other."""
    one = _batch([1, 1, 1], [9000, 700, 50], 2, 8, 128, 16, seed=1)
    two = _batch([200, 90], [5000, 90], 2, 4, 128, 32, seed=2)
    calls = []
    for q, k, v, table, cu, total in (one, two):
        ws = torch.zeros(cb.cb_paged_attention_workspace_bytes(128), dtype=torch.uint8, device=DEV)
        args = (cb.PagePool(k, v), 0, table, _i32(cu), _i32(total), 128 ** -0.5, ws)
        want = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
        cb.cb_paged_attention(q, want, *args, max_new=cu[1])
        calls.append((q, args, want, cu[1], torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[torch.empty_like(c[2]) for _ in range(20)] for c in calls]
    for i in range(20):
        for c, out in zip(calls, outs):
            cb.cb_paged_attention(c[0], out[i], *c[1], max_new=c[3], stream=c[4])
    torch.cuda.synchronize()
    for c, out in zip(calls, outs):
        assert all(torch.equal(o, c[2]) for o in out)
    cb.cb_last_device_status()


def test_attention_time_out_is_reported_and_leaves_the_workspace_usable():
    b = _batch([1, 1, 70], [3000, 100, 70], 1, 4, 128, 16)
    want = _compare(*b)
    cb.cb_last_device_status()
    try:
        for max_new in (1, 70):
            cb.cb_test_hooks(poll_limit=2000, starve_producer=True)
            _attend(*b, max_new=max_new)
            with pytest.raises(cb.CbError) as e:
                cb.cb_last_device_status()
            assert e.value.status == cb.CB_ERR_TIMEOUT
            cb.cb_test_hooks()
            assert torch.equal(_compare(*b), want)
    finally:
        cb.cb_test_hooks()


@pytest.mark.parametrize("new,total,d,page,window", [
    ([1, 1, 70], [3000, 100, 70], 128, 16, 0), ([300, 1], [9000, 700], 128, 64, 0), ([300, 7], [20000, 40], 64, 8, 1000), ([1] * 9, [5000] * 9, 64, 16, 70)])
def test_attention_consumers_that_give_up_while_copies_are_in_flight(new, total, d, page, window):
    """Some warps take their first wait as run out while the copies go on: the block issues no more of them, lets those in
    flight land, reports, and leaves the workspace as a good run does."""
    b = _batch(new, total, 2, 4, d, page)
    want = _compare(*b, window=window, n_sink=2)
    try:
        for max_new in (1, 0, 1, 0):
            cb.cb_test_hooks(poll_limit=2000, consumers_give_up=True)
            _attend(*b, window=window, n_sink=2, max_new=max_new)
            with pytest.raises(cb.CbError) as e:
                cb.cb_last_device_status()
            assert e.value.status == cb.CB_ERR_TIMEOUT
            cb.cb_test_hooks()
            assert torch.equal(_compare(*b, window=window, n_sink=2), want)
    finally:
        cb.cb_test_hooks()


# ---------------------------------------------------------------------------------------------------- together
def test_a_decode_step_captured_once_and_replayed_as_requests_grow():
    """Tables, rotation, store and attention in one graph; the host only rotates the free list between replays."""
    g = torch.Generator(device=DEV)
    g.manual_seed(21)
    B, H, group, d, page, L = 3, 2, 8, 128, 8, 2
    pages, cols, steps = 64, 12, 20
    k, v = _pool(L, pages, page, H, d, False, fill=float("nan"))
    pool = cb.PagePool(k, v)
    lens = [5, 8, 15]
    ids = torch.randperm(pages, generator=g, device=DEV).int()
    table = torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
    table[0, :1], table[1, :1], table[2, :2] = ids[:1], ids[1:2], ids[2:4]
    free = ids[4:].clone()
    dense_k, dense_v = (torch.zeros(L, B, 15 + steps, H, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for b, n in enumerate(lens):
        j = torch.arange(n, device=DEV)
        for x, y in ((k, dense_k), (v, dense_v)):
            rows = torch.randn(L, n, H, d, generator=g, device=DEV).bfloat16()
            x[:, table[b, j // page].long(), j % page] = rows
            y[:, b, :n] = rows
    room = B + 2                                            # two padded rows behind the batch
    nk, nv = (torch.zeros(L, room, H, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rk = torch.zeros_like(nk)
    q = torch.zeros(1, room, H * group, d, dtype=torch.bfloat16, device=DEV)
    rq, out = torch.zeros_like(q), torch.full((L, room, H * group, d), 5.0, dtype=torch.bfloat16, device=DEV)
    cached, new = _i32(lens), _i32([1] * B)
    cu, total, used = _i32([0] * (B + 1)), _i32([0] * B), _i32([0])
    pos, slot = torch.zeros(1, room, dtype=torch.int32, device=DEV), torch.zeros(room, dtype=torch.int64, device=DEV)
    ws = _workspace(d)

    def step():
        cb.cb_page_tables(cached, new, page, free, table, cu, total, pos[0], slot, used)
        cb.cb_rope_axes(nk, rk, pos, [64], 1e6)
        cb.cb_rope_axes(q, rq, pos, [64], 1e6)
        cb.cb_paged_store(pool, rk, nv, slot)
        for layer in range(L):
            cb.cb_paged_attention(rq[0], out[layer], pool, layer, table, cu, total, d ** -0.5, ws, max_new=1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        keep = table.clone()
        step()                                              # warm-up; what it stored is stored again by the first replay
        table.copy_(keep)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        for x in (nk, nv, q):
            x.copy_(torch.randn(x.shape, generator=g, device=DEV).bfloat16())
        graph.replay()
        at = [n + i for n in lens]
        assert pos[0].tolist() == at + [0, 0] and slot[B:].tolist() == [-1, -1]
        for b in range(B):
            dense_k[:, b, at[b]], dense_v[:, b, at[b]] = rk[:, b], nv[:, b]
        for layer in range(L):
            want, tol = ref.attention(rq[0], dense_k[layer], dense_v[layer], torch.arange(B, device=DEV)[:, None], cu.tolist(), total.tolist(), d ** -0.5)
            assert ((out[layer, :B].double() - want[:B]).abs() <= tol[:B]).all()
            assert (out[layer, B:] == 5).all()
        free.copy_(free.roll(-int(used[0])))
        cached.copy_(total)
    cb.cb_last_device_status()


def test_a_step_layer_by_layer_through_views_of_one_layer():
    """A layer's queries, keys and values follow from the attention of the layer before it, so that its rows are stored just
    before its attention reads them; the whole step is captured and replayed as requests grow."""
    g = torch.Generator(device=DEV)
    g.manual_seed(31)
    B, H, group, d, page, L, base = 3, 2, 4, 64, 16, 3, 1e4
    pages, cols, Hq = 40, 6, 8
    k, v = _pool(L, pages, page, H, d, True, fill=float("nan"))
    pools = [cb.PagePool(k[l:l + 1], v[l:l + 1]) for l in range(L)]
    lens = [3, 16, 40]
    ids = torch.randperm(pages, generator=g, device=DEV).int()
    table, at = torch.full((B, cols), -1, dtype=torch.int32, device=DEV), 0
    old = []                                                # [request][layer] -> keys, values so far, as stored
    for b, n in enumerate(lens):
        held = -(-n // page)
        table[b, :held], at = ids[at:at + held], at + held
        j, rows = torch.arange(n, device=DEV), [torch.randn(L, n, H, d, generator=g, device=DEV).bfloat16() for _ in range(2)]
        k[:, table[b, j // page].long(), j % page], v[:, table[b, j // page].long(), j % page] = rows
        old.append(rows)
    free = ids[at:].clone()
    wq, wk, wv = (torch.randn(L, Hq * d, n * d, generator=g, device=DEV) * (Hq * d) ** -0.5 for n in (Hq, H, H))
    x0, cached, new = torch.randn(B, Hq * d, generator=g, device=DEV), _i32(lens), _i32([1] * B)
    cu, total, used, pos = _i32([0] * (B + 1)), _i32([0] * B), _i32([0]), torch.zeros(1, B, dtype=torch.int32, device=DEV)
    slot, o = torch.zeros(B, dtype=torch.int64, device=DEV), torch.zeros(L, B, Hq, d, dtype=torch.bfloat16, device=DEV)
    got = [[torch.zeros(B, n, d, dtype=torch.bfloat16, device=DEV) for n in (Hq, H, H)] for _ in range(L)]
    ws = _workspace(d)

    def step():
        x = x0
        cb.cb_page_tables(cached, new, page, free, table, cu, total, pos[0], slot, used)
        for l in range(L):
            q, kn, vn = ((x @ w[l]).bfloat16().view(1, B, -1, d) for w in (wq, wk, wv))
            cb.cb_rope_axes(q, q, pos, [d // 2], base)
            cb.cb_rope_axes(kn, kn, pos, [d // 2], base)
            cb.cb_paged_store(pools[l], kn, vn, slot)
            cb.cb_paged_attention(q[0], o[l], pools[l], 0, table, cu, total, d ** -0.5, ws, max_new=1)
            for t, s in zip(got[l], (q, kn, vn)):
                t.copy_(s[0])
            x = x + o[l].reshape(B, Hq * d).float()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        keep = table.clone()
        step()
        table.copy_(keep)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(20):
        x0.copy_(torch.randn(B, Hq * d, generator=g, device=DEV))
        graph.replay()
        assert pos[0].tolist() == [n + i for n in lens]
        x = x0
        for l in range(L):
            q, kn, vn = got[l]
            # The layer's rows follow from the attention of the layer before.  The fp32 product over 512 terms is off by up to
            # 2 * 512 * 2^-24 of the sum of sizes, a rounding to bf16 by 2^-8 of the value; queries and keys are then turned
            # (each part of the pair carries its error into both, the angle and polynomials add 2^-20 of the pair's length)
            # and rounded once more.
            for have, w, turn in ((q, wq, True), (kn, wk, True), (vn, wv, False)):
                row = (x.double() @ w[l].double()).view(B, -1, d)
                off = row.abs() * 2.0 ** -8 + 2 * 512 * 2.0 ** -24 * (x.abs().double() @ w[l].abs().double()).view(B, -1, d)
                if turn:
                    off = (off[..., :d // 2] + off[..., d // 2:] + 2.0 ** -20 * torch.sqrt(row[..., :d // 2] ** 2 + row[..., d // 2:] ** 2)).repeat(1, 1, 2)
                    row = ref.rope(row[None], pos, [d // 2], base, False, False)[0]
                    off = off + (row.abs() + off) * 2.0 ** -8
                assert ((have.double() - row).abs() <= off).all()
            n = max(lens) + i + 1
            kd, vd = (torch.zeros(B, n, H, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            for b in range(B):
                have = old[b][0].shape[1]
                kd[b, :have], vd[b, :have] = old[b][0][l], old[b][1][l]
                kd[b, have], vd[b, have] = kn[b], vn[b]
            want, tol = ref.attention(q, kd, vd, torch.arange(B, device=DEV)[:, None], list(range(B + 1)), total.tolist(), d ** -0.5)
            assert ((o[l].double() - want).abs() <= tol).all()
            x = x + o[l].reshape(B, Hq * d).float()
        for b in range(B):
            for c in range(2):
                old[b][c] = torch.cat([old[b][c], torch.stack([got[l][1 + c][b] for l in range(L)])[:, None]], 1)
        free.copy_(free.roll(-int(used[0])))
        cached.copy_(total)
    cb.cb_last_device_status()


def test_mapped_cache_into_pages_and_attention_over_it():
    """A fitted map's target cache is stored into pages, a chunk of new rows and then single tokens join it, and attention
    over the pages agrees with attention over the dense tensors."""
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    Ls, Hs, Lt, Ht, d, group, page = 3, 2, 4, 2, 128, 4, 16
    sl, sh = cb.cb_head_map_nearest(Ls, Hs, Lt, Ht)
    prob = cb.Problem(Ls, Hs, d, Lt, Ht, d, sl, sh)
    prompt = [70, 41]
    P = sum(prompt)
    src_k, src_v = (torch.randn(Ls, P, Hs, d, generator=g, device=DEV).bfloat16() for _ in range(2))
    Wb = torch.randn(prob.n_maps, d + 1, d, generator=g, device=DEV) * d ** -0.5
    positions = torch.cat([torch.arange(n, device=DEV) for n in prompt]).int()
    map_k, map_v = (torch.empty(Lt, P, Ht, d, dtype=torch.float32, device=DEV) for _ in range(2))
    cb.cb_apply_rope(prob, Wb, src_k, src_v, map_k, map_v, positions, 1e6, 1e6)
    pages, cols = 40, 12
    k, v = _pool(Lt, pages, page, Ht, d, False, fill=float("nan"))
    pool = cb.PagePool(k, v)
    free = torch.randperm(pages, generator=g, device=DEV).int()
    table = torch.full((2, cols), -1, dtype=torch.int32, device=DEV)
    dense = [[map_k[:, :70].bfloat16(), map_k[:, 70:].bfloat16()], [map_v[:, :70].bfloat16(), map_v[:, 70:].bfloat16()]]
    cached, used_pages = _i32([0, 0]), 0
    cu, total, used = _i32([0] * 3), _i32([0] * 2), _i32([0])
    for step, new in enumerate(([70, 41], [9, 30], [1, 1], [1, 0])):
        T = sum(new)
        pos, slot = torch.empty(T, dtype=torch.int32, device=DEV), torch.empty(T, dtype=torch.int64, device=DEV)
        cb.cb_page_tables(cached, _i32(new), page, free[used_pages:], table, cu, total, pos, slot, used)
        used_pages += int(used[0])
        if step == 0:
            assert torch.equal(pos, positions)
            cb.cb_paged_store(pool, map_k, map_v, slot)
        else:
            nk, nv = (torch.randn(Lt, T, Ht, d, generator=g, device=DEV).bfloat16() for _ in range(2))
            q = torch.randn(1, T, Ht * group, d, generator=g, device=DEV).bfloat16()
            three = pos[None].expand(3, T).contiguous()          # text: the same position on every axis
            cb.cb_rope_axes(nk, nk, three, [24, 20, 20], 1e6)
            cb.cb_rope_axes(q, q, three, [24, 20, 20], 1e6)
            cb.cb_paged_store(pool, nk, nv, slot)
            at = cu.tolist()
            for b in range(2):
                dense[0][b] = torch.cat([dense[0][b], nk[:, at[b]:at[b + 1]]], 1)
                dense[1][b] = torch.cat([dense[1][b], nv[:, at[b]:at[b + 1]]], 1)
            for layer in range(Lt):
                out = torch.full((T, Ht * group, d), 5.0, dtype=torch.bfloat16, device=DEV)
                cb.cb_paged_attention(q[0], out, pool, layer, table, cu, total, d ** -0.5, _workspace(d), max_new=max(new))
                # the dense caches as pools of one page each
                n = max(x.shape[1] for x in dense[0])
                kd, vd = (torch.stack([torch.nn.functional.pad(x[layer], (0, 0, 0, 0, 0, n - x.shape[1])) for x in y]) for y in dense)
                want, tol = ref.attention(q[0], kd, vd, torch.arange(2, device=DEV)[:, None], at, total.tolist(), d ** -0.5)
                assert ((out.double() - want).abs() <= tol).all()
        cached.copy_(total)
    cb.cb_last_device_status()
