// Host side of the paged target cache: argument checks and launches (page tables, store, rotary positions with several
// axes, attention).
#include <algorithm>
#include <cmath>
#include <cstring>
#include <iterator>

#include "cb_paged.cuh"
#include "cb_rope.cuh"

using namespace cb;

namespace {

constexpr int32_t MAX_REQUESTS = 1 << 28;      // the kernels count requests, and twice as many, in 32 bits

// log2 of a page size the kernels take (8 .. 256), or -1
int page_log2_of(int32_t ps)
{
    for (int l = 3; l <= 8; ++l)
        if (ps == (1 << l)) return l;
    return -1;
}

cb_status check_pool(const cb_page_pool *p)
{
    if (!p || p->n_layers <= 0 || p->n_heads <= 0 || p->head_dim <= 0 || p->page_size <= 0 || p->n_pages <= 0) return CB_ERR_INVALID_ARG;
    if (!p->k || !p->v || (((uintptr_t)p->k | (uintptr_t)p->v) & 15)) return CB_ERR_INVALID_ARG;
    if (p->stride_layer < 0 || p->stride_page < 0 || p->stride_slot < 0 || p->stride_head < 0) return CB_ERR_INVALID_ARG;
    if ((p->stride_layer | p->stride_page | p->stride_slot | p->stride_head) & 7) return CB_ERR_INVALID_ARG;
    if (p->head_dim != 64 && p->head_dim != 128) return CB_ERR_UNSUPPORTED;
    if (page_log2_of(p->page_size) < 0 || p->n_pages >= (1ll << 31)) return CB_ERR_UNSUPPORTED;
    // a broadcast over more than one layer, page, row or head: pieces of the cache would share memory
    if ((p->n_layers > 1 && p->stride_layer == 0) || (p->n_pages > 1 && p->stride_page == 0) || p->stride_slot == 0 ||
        (p->n_heads > 1 && p->stride_head == 0))
        return CB_ERR_UNSUPPORTED;
    // byte strides of a tensor map are below 2^40
    if (p->stride_page >= (1ll << 39) || p->stride_slot >= (1ll << 39) || p->stride_head >= (1ll << 39)) return CB_ERR_UNSUPPORTED;
    return CB_OK;
}

struct Range { const void *p; int64_t bytes; };
bool overlap(const Range &a, const Range &b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.bytes > 0 && b.bytes > 0 && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

template <class Args>
cb_status launch_state(Args &a)
{
    a.status = library_status_word();
    if (!a.status) return cuda_failed(cudaErrorNoDevice);
    const TestHooks h = test_hooks();
    a.poll_limit = h.poll_limit;
    a.starve = h.starve;
    a.give_up = h.give_up;
    return CB_OK;
}

}  // namespace

extern "C" {

cb_status cb_page_tables(const int32_t *cached_len, const int32_t *new_len, int32_t n_requests, int32_t page_size,
                         const int32_t *free_pages, int64_t n_free, int32_t *block_table, int64_t table_stride, int32_t max_pages,
                         int32_t *cu_new, int32_t *total_len, int32_t *positions, int64_t *slot_map, int64_t n_rows,
                         int32_t *pages_used, void *stream)
{
    if (n_requests < 0 || n_free < 0 || n_rows < 0 || max_pages <= 0 || table_stride < 0) return CB_ERR_INVALID_ARG;
    if (n_requests > 0 && (!cached_len || !new_len || !block_table || !total_len)) return CB_ERR_INVALID_ARG;
    if (n_requests > 1 && table_stride < max_pages) return CB_ERR_INVALID_ARG;
    if (!cu_new || (n_free > 0 && !free_pages) || (n_rows > 0 && (!positions || !slot_map))) return CB_ERR_INVALID_ARG;
    if ((((uintptr_t)cached_len | (uintptr_t)new_len | (uintptr_t)free_pages | (uintptr_t)block_table | (uintptr_t)cu_new |
          (uintptr_t)total_len | (uintptr_t)positions | (uintptr_t)pages_used) & 3) || ((uintptr_t)slot_map & 7))
        return CB_ERR_INVALID_ARG;
    const int lg = page_log2_of(page_size);
    if (lg < 0 || n_rows >= (1ll << 31) || n_requests >= MAX_REQUESTS) return CB_ERR_UNSUPPORTED;
    // Every block reads the inputs while others write their results.  (A table whose rows have room behind them may have
    // something else there, so its rows are not looked at then.)
    const int64_t B = n_requests;
    const bool dense = B <= 1 || table_stride == max_pages;
    const Range in[] = {{cached_len, B * 4}, {new_len, B * 4}, {free_pages, n_free * 4}},
                out[] = {{cu_new, (B + 1) * 4}, {total_len, B * 4}, {positions, n_rows * 4}, {slot_map, n_rows * 8},
                         {pages_used, pages_used ? 4 : 0}, {block_table, dense ? B * max_pages * 4 : 0}};
    for (size_t i = 0; i < std::size(out); ++i) {
        for (const Range &r : in)
            if (overlap(out[i], r)) return CB_ERR_INVALID_ARG;
        for (size_t j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return CB_ERR_INVALID_ARG;
    }
    if (const cudaError_t e = launch_page_tables(cached_len, new_len, n_requests, lg, free_pages, n_free, block_table, table_stride, max_pages,
                                                 cu_new, total_len, positions, reinterpret_cast<long long *>(slot_map), n_rows,
                                                 pages_used, static_cast<cudaStream_t>(stream)); e != cudaSuccess) return cuda_failed(e);
    return CB_OK;
}

cb_status cb_paged_store(const cb_page_pool *pool, const void *src_k, const void *src_v, int32_t src_dtype, int64_t n_rows,
                         int64_t stride_layer, int64_t stride_token, int64_t stride_head, const int64_t *slot_map, void *stream)
{
    cb_status s = check_pool(pool);
    if (s != CB_OK) return s;
    if (src_dtype != CB_DTYPE_BF16 && src_dtype != CB_DTYPE_F32) return CB_ERR_INVALID_ARG;
    if (n_rows < 0 || stride_layer < 0 || stride_token < 0 || stride_head < 0) return CB_ERR_INVALID_ARG;
    if ((stride_layer | stride_token | stride_head) & 7) return CB_ERR_INVALID_ARG;
    if (n_rows >= (1ll << 31) || pool->n_layers > 65535) return CB_ERR_UNSUPPORTED;
    if (n_rows * pool->n_heads >= (1ll << 35)) return CB_ERR_UNSUPPORTED;      // blocks of one launch
    if (n_rows == 0) return CB_OK;
    if (!src_k || !src_v || !slot_map || (((uintptr_t)src_k | (uintptr_t)src_v) & 15) || ((uintptr_t)slot_map & 7)) return CB_ERR_INVALID_ARG;
    StoreArgs a;
    a.src_k = src_k; a.src_v = src_v; a.src_f32 = src_dtype == CB_DTYPE_F32;
    a.s_sl = stride_layer; a.s_st = stride_token; a.s_sh = stride_head;
    a.k = static_cast<__nv_bfloat16 *>(pool->k); a.v = static_cast<__nv_bfloat16 *>(pool->v);
    a.d_sl = pool->stride_layer; a.d_sp = pool->stride_page; a.d_ss = pool->stride_slot; a.d_sh = pool->stride_head;
    a.slot_map = reinterpret_cast<const long long *>(slot_map);
    a.page_log2 = page_log2_of(pool->page_size);
    a.n_slots = pool->n_pages << a.page_log2;
    a.n_rows = n_rows;
    a.L = pool->n_layers; a.H = pool->n_heads; a.d = pool->head_dim;
    if (const cudaError_t e = launch_paged_store(a, static_cast<cudaStream_t>(stream)); e != cudaSuccess) return cuda_failed(e);
    return CB_OK;
}

cb_status cb_rope_axes(const void *x, void *out, int32_t n_layers, int32_t n_heads, int32_t head_dim, int64_t n_tokens,
                       int64_t x_stride_layer, int64_t x_stride_token, int64_t x_stride_head,
                       int64_t o_stride_layer, int64_t o_stride_token, int64_t o_stride_head,
                       const int32_t *positions, int64_t axis_stride, int32_t n_axes, const int32_t *sections,
                       int32_t interleaved, double rope_base, int32_t inverse, void *stream)
{
    if (n_layers <= 0 || n_heads <= 0 || n_tokens < 0 || n_axes <= 0 || !sections) return CB_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return CB_ERR_UNSUPPORTED;
    if (n_tokens >= (1ll << 31) || (int64_t)n_layers * n_heads > (1 << 18) || n_axes > 8) return CB_ERR_UNSUPPORTED;
    if (!(rope_base > 1.0) || !(rope_base <= 1e12)) return CB_ERR_INVALID_ARG;
    int64_t sum = 0;
    for (int i = 0; i < n_axes; ++i) {
        if (sections[i] < 0) return CB_ERR_INVALID_ARG;
        sum += sections[i];
    }
    if (sum != head_dim / 2) return CB_ERR_INVALID_ARG;
    const int64_t all[6] = {x_stride_layer, x_stride_token, x_stride_head, o_stride_layer, o_stride_token, o_stride_head};
    for (int i = 0; i < 6; ++i)
        if (all[i] < 0 || (all[i] & 7)) return CB_ERR_INVALID_ARG;
    // an input may repeat rows (stride 0); an output may not
    if ((n_layers > 1 && o_stride_layer == 0) || (n_tokens > 1 && o_stride_token == 0) || (n_heads > 1 && o_stride_head == 0)) return CB_ERR_UNSUPPORTED;
    if (n_tokens == 0) return CB_OK;
    if (!x || !out || !positions || (((uintptr_t)x | (uintptr_t)out) & 15) || ((uintptr_t)positions & 3) || axis_stride < 0) return CB_ERR_INVALID_ARG;
    if (x == out && (x_stride_layer != o_stride_layer || x_stride_token != o_stride_token || x_stride_head != o_stride_head)) return CB_ERR_INVALID_ARG;
    unsigned char axis[ROPE_MAX_FREQ] = {};
    for (int i = 0, a = 0, left = sections[0]; i < head_dim / 2; ++i) {
        if (interleaved) {
            axis[i] = (unsigned char)(i < n_axes * sections[i % n_axes] ? i % n_axes : 0);
        } else {
            while (left == 0) left = sections[++a];
            axis[i] = (unsigned char)a;
            --left;
        }
    }
    const long long xs[3] = {x_stride_layer, x_stride_token, x_stride_head}, os[3] = {o_stride_layer, o_stride_token, o_stride_head};
    if (const cudaError_t e = launch_rope_axes(x, out, n_layers, n_heads, head_dim, n_tokens, xs, os, positions, axis_stride, axis,
                                               rope_base, inverse ? 1 : 0, static_cast<cudaStream_t>(stream)); e != cudaSuccess) return cuda_failed(e);
    return CB_OK;
}

cb_status cb_paged_attention_workspace_bytes(int32_t head_dim, size_t *bytes)
{
    if (!bytes) return CB_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return CB_ERR_UNSUPPORTED;
    *bytes = PA_COUNTER_BYTES + std::max(paged_attn_few_workspace(head_dim), paged_attn_tc_workspace(head_dim));
    return CB_OK;
}

cb_status cb_paged_attention(const cb_page_pool *pool, int32_t layer, const void *q, int64_t q_stride_token, int64_t q_stride_head,
                             void *out, int64_t o_stride_token, int64_t o_stride_head, int64_t n_rows, int32_t n_q_heads,
                             const int32_t *block_table, int64_t table_stride, int32_t max_pages,
                             const int32_t *cu_new, const int32_t *total_len, int32_t n_requests, int32_t max_new,
                             float scale, int32_t window, int32_t n_sink, void *workspace, size_t workspace_bytes, void *stream)
{
    cb_status s = check_pool(pool);
    if (s != CB_OK) return s;
    if (layer < 0 || layer >= pool->n_layers || n_rows < 0 || n_q_heads <= 0 || n_requests < 0 || max_pages <= 0 || max_new < 0 ||
        table_stride < 0 || window < 0 || n_sink < 0)
        return CB_ERR_INVALID_ARG;
    const float scale_log2 = (float)(scale * 1.4426950408889634074);
    if (n_q_heads % pool->n_heads || !(scale > 0.f) || !std::isfinite(scale_log2)) return CB_ERR_INVALID_ARG;
    if (q_stride_token < 0 || q_stride_head < 0 || o_stride_token < 0 || o_stride_head < 0) return CB_ERR_INVALID_ARG;
    if ((q_stride_token | q_stride_head | o_stride_token | o_stride_head) & 7) return CB_ERR_INVALID_ARG;
    if ((n_rows > 1 && (o_stride_token == 0 || q_stride_token == 0)) || (n_q_heads > 1 && (o_stride_head == 0 || q_stride_head == 0))) return CB_ERR_UNSUPPORTED;
    if (q_stride_token >= (1ll << 39) || q_stride_head >= (1ll << 39)) return CB_ERR_UNSUPPORTED;
    // flattened rows and units are counted in 32 bits
    if (n_rows >= (1ll << 31) || n_rows * n_q_heads + n_requests >= (1ll << 31) || n_requests >= MAX_REQUESTS) return CB_ERR_UNSUPPORTED;
    if (n_requests > 1 && table_stride < max_pages) return CB_ERR_INVALID_ARG;
    if (n_rows == 0 || n_requests == 0) return CB_OK;
    if (q == out) return CB_ERR_INVALID_ARG;         // rows are written while other blocks still read theirs
    if (!q || !out || !block_table || !cu_new || !total_len) return CB_ERR_INVALID_ARG;
    if ((((uintptr_t)q | (uintptr_t)out) & 15) || (((uintptr_t)block_table | (uintptr_t)cu_new | (uintptr_t)total_len) & 3)) return CB_ERR_INVALID_ARG;
    size_t need = 0;
    cb_paged_attention_workspace_bytes(pool->head_dim, &need);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need) return CB_ERR_WORKSPACE;
    PagedArgs a;
    a.q = static_cast<const __nv_bfloat16 *>(q);
    a.out = static_cast<__nv_bfloat16 *>(out);
    a.q_st = q_stride_token; a.q_sh = q_stride_head; a.o_st = o_stride_token; a.o_sh = o_stride_head;
    a.table = block_table; a.table_stride = table_stride; a.table_cols = max_pages;
    a.cu = cu_new; a.total = total_len; a.n_requests = n_requests; a.n_rows = (int)n_rows;
    a.Hkv = pool->n_heads; a.group = n_q_heads / pool->n_heads;
    // n / d == mulhi(n, ceil(2^32 / d)) as long as n (d - 1) < 2^32
    auto reciprocal = [](int64_t d, int64_t most) {
        return d > 1 && (unsigned __int128)most * d < ((unsigned __int128)1 << 32) ? (unsigned)(((1ull << 32) + d - 1) / d) : 0u;
    };
    a.group_mul = reciprocal(a.group, n_rows * a.group);
    // tensor-core kernel: a tile of 128 rows holds whole tokens, so that one copy brings it
    a.unit_tokens = a.group <= 128 ? 2 * (128 / a.group) : 1;
    a.unit_rows = a.unit_tokens * a.group;
    a.unit_mul = reciprocal(a.unit_tokens, n_rows + a.unit_tokens);
    a.page_log2 = page_log2_of(pool->page_size);
    a.n_pages = (int)pool->n_pages;
    a.window = window; a.n_sink = window > 0 ? n_sink : 0;
    a.scale_log2 = scale_log2;
    a.q_min = 2;
    a.counters = static_cast<int *>(workspace);
    a.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + PA_COUNTER_BYTES);
    s = launch_state(a);
    if (s != CB_OK) return s;
    if (device_sm_count() * 8 > PA_COUNTERS) return CB_ERR_UNSUPPORTED;
    if (max_new == 0 || max_new > n_rows) max_new = (int32_t)n_rows;
    const __nv_bfloat16 *k = static_cast<const __nv_bfloat16 *>(pool->k) + layer * pool->stride_layer;
    const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(pool->v) + layer * pool->stride_layer;
    // Up to 16 flattened rows per request and KV head: the warp-level kernel, which has no rows to pad.  Measured on 16
    // requests of 8,192 keys, 8 KV heads (537 MB), pages of 16 and 64, warp-level against tensor-memory kernel: 8 rows 94 - 97
    // / 109 - 125 us, 16 rows 98 - 102 / 109 - 121 us, 32 rows 176 / 117 - 125 us, 64 rows 335 / 125 - 135 us.  (And more than
    // 128 query heads per KV head, which do not fit a tile.)
    const bool few = (long long)max_new * a.group <= 16 || a.group > 128;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = few ? launch_paged_attn_few(a, pool->head_dim, k, v, pool->page_size, pool->stride_page, pool->stride_slot, pool->stride_head, max_new, st)
                              : launch_paged_attn_tc(a, pool->head_dim, k, v, pool->page_size, pool->stride_page, pool->stride_slot, pool->stride_head, st);
    if (e != cudaSuccess) return cuda_failed(e);
    return CB_OK;
}

}  // extern "C"
