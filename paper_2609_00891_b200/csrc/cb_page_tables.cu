// Page tables, slots and positions of a batch from its request lengths.
//
// Request b keeps its ceil(cached/ps) pages and takes ceil((cached + new)/ps) minus that many from the free list, in
// request order; row t of the batch belongs to the request b with cu[b] <= t < cu[b + 1] and goes to position
// cached[b] + t - cu[b].  Everything follows from two prefix sums over the requests, which every block takes for itself
// (8 bytes a request, from L2) instead of waiting for another one: one launch, no workspace, no order between blocks.
// Bound by the launch for decode steps and by the 12 bytes written per row for whole prompts.
#include "cb_paged.cuh"

namespace cb {

static constexpr int PT_THREADS = 1024;
static constexpr int PT_SPAN = 2048;        // rows that are worth a block of their own

struct TablesArgs {
    const int *cached, *fresh;
    int B, page_log2;
    const int *free_pages;
    long long n_free;
    int *table;
    long long table_stride;
    int cols;
    int *cu, *total, *positions;
    long long *slot_map;
    long long n_rows;
    int *pages_used;
    int vector;               // positions and slot_map allow 16-byte stores
};

// The last i with at[i] <= e, for lanes whose e ascend (all 32 lanes): the first and last lane's by two votes each, on every
// 32nd entry and on the 32 behind it, the others' by a search between those two, which are mostly the same request.
__device__ __forceinline__ int locate(const unsigned *every32, const unsigned *at, unsigned e, int lane)
{
    auto vote = [&](unsigned x) {
        const int g = __popc(__ballot_sync(0xffffffffu, every32[lane] <= x)) - 1;
        return g * 32 + __popc(__ballot_sync(0xffffffffu, at[g * 32 + lane] <= x)) - 1;
    };
    int lo = vote(__shfl_sync(0xffffffffu, e, 0)), hi = vote(__shfl_sync(0xffffffffu, e, 31));
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (at[mid] <= e) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__global__ void __launch_bounds__(PT_THREADS) k_page_tables(const TablesArgs a)
{
    __shared__ unsigned long long warp_sums[32];
    __shared__ unsigned row_at[PT_THREADS + 1], page_at[PT_THREADS + 1];   // within the group of requests
    __shared__ int s_cached[PT_THREADS], s_held[PT_THREADS];
    __shared__ unsigned row_of_warp[32], page_of_warp[32];                // row_at and page_at of every 32nd request
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps1 = (1 << a.page_log2) - 1;
    const long long stride = (long long)gridDim.x * PT_THREADS, mine = (long long)blockIdx.x * PT_THREADS + tid;
    long long rows0 = 0, pages0 = 0;          // before this group of requests
    for (int b0 = 0; b0 < a.B; b0 += PT_THREADS) {
        const int b = b0 + tid;
        int cached = 0, fresh = 0;
        if (b < a.B) { cached = max(a.cached[b], 0); fresh = max(a.fresh[b], 0); }
        const long long sum = (long long)cached + fresh;
        const int held = (int)(((long long)cached + ps1) >> a.page_log2), need = (int)((sum + ps1) >> a.page_log2);
        // rows in the low half, pages in the high half: neither passes 2^32 in 1,024 requests that fit a pool
        unsigned long long incl = (unsigned long long)(unsigned)fresh | ((unsigned long long)(unsigned)(need - held) << 32);
        const unsigned long long own = incl;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 31) warp_sums[warp] = incl;
        __syncthreads();
        unsigned long long before = lane < warp ? warp_sums[lane] : 0ull;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
        const unsigned long long excl = before + incl - own;
        row_at[tid] = (unsigned)excl;
        page_at[tid] = (unsigned)(excl >> 32);
        if (lane == 0) { row_of_warp[warp] = (unsigned)excl; page_of_warp[warp] = (unsigned)(excl >> 32); }
        s_cached[tid] = cached;
        s_held[tid] = held;
        if (tid == PT_THREADS - 1) { row_at[PT_THREADS] = (unsigned)(excl + own); page_at[PT_THREADS] = (unsigned)((excl + own) >> 32); }
        if (blockIdx.x == 0 && b < a.B) {
            a.cu[b] = (int)(rows0 + (unsigned)excl);
            a.total[b] = (int)sum;
        }
        __syncthreads();
        const unsigned n_rows = row_at[PT_THREADS], n_pages = page_at[PT_THREADS];
        // new pages: the e-th of the group belongs to the last request whose pages start at or before e
        for (long long w0 = mine - lane; w0 < n_pages; w0 += stride) {
            const unsigned e = min((unsigned)w0 + lane, n_pages - 1);
            const int lo = locate(page_of_warp, page_at, e, lane);
            if (w0 + lane < n_pages) {
                const int col = s_held[lo] + (int)(e - page_at[lo]);
                const long long f = pages0 + e;
                if ((unsigned)col < (unsigned)a.cols) a.table[(long long)(b0 + lo) * a.table_stride + col] = f < a.n_free ? a.free_pages[f] : -1;
            }
        }
        // rows, four neighbours a thread: one search for the four
        const long long end = min(rows0 + (long long)n_rows, a.n_rows);
        for (long long w0 = rows0 / 4 * 4 + (mine - lane) * 4; w0 < end && rows0 < end; w0 += stride * 4) {
            const long long t0 = w0 + lane * 4;
            unsigned e = (unsigned)(min(max(t0, rows0), end - 1) - rows0);
            int lo = locate(row_of_warp, row_at, e, lane);
            if (t0 >= end) continue;
            int pos[4], page[4];
            // where the page id of a request's position stands: its table for the pages it held, else the free list
            auto source = [&](int request, int p) -> const int * {
                const int col = p >> a.page_log2;
                if ((unsigned)col >= (unsigned)a.cols) return nullptr;
                if (col < s_held[request]) return a.table + (long long)(b0 + request) * a.table_stride + col;
                const long long f = pages0 + page_at[request] + (col - s_held[request]);
                return f < a.n_free ? a.free_pages + f : nullptr;
            };
            if (t0 >= rows0 && t0 + 4 <= end && row_at[lo + 1] - e >= 4) {
                // four rows of one request: on one page or on two neighbours (a page has 8 rows or more)
                const int p = s_cached[lo] + (int)(e - row_at[lo]);
                const int *one = source(lo, p), *two = source(lo, p + 3);
                const int id1 = one ? *one : -1, id2 = two ? *two : -1;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    pos[k] = p + k;
                    page[k] = ((p + k) >> a.page_log2) == (p >> a.page_log2) ? id1 : id2;
                }
            } else {
                const int *from[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    pos[k] = 0;
                    from[k] = nullptr;
                    if (t0 + k < rows0 || t0 + k >= end) continue;
                    while (lo < PT_THREADS - 1 && row_at[lo + 1] <= e) ++lo;
                    pos[k] = s_cached[lo] + (int)(e - row_at[lo]);
                    from[k] = source(lo, pos[k]);
                    ++e;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) page[k] = from[k] ? *from[k] : -1;
            }
            long long slot[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) slot[k] = page[k] < 0 ? -1ll : ((long long)page[k] << a.page_log2) + (pos[k] & ps1);
            if (a.vector && t0 >= rows0 && t0 + 4 <= end) {
                *reinterpret_cast<int4 *>(a.positions + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
                *reinterpret_cast<longlong2 *>(a.slot_map + t0) = make_longlong2(slot[0], slot[1]);
                *reinterpret_cast<longlong2 *>(a.slot_map + t0 + 2) = make_longlong2(slot[2], slot[3]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (t0 + k >= rows0 && t0 + k < end) {
                        a.positions[t0 + k] = pos[k];
                        a.slot_map[t0 + k] = slot[k];
                    }
            }
        }
        rows0 += n_rows;
        pages0 += n_pages;
        __syncthreads();
    }
    for (long long e = rows0 + mine; e < a.n_rows; e += stride) {       // behind the last request
        a.positions[e] = 0;
        a.slot_map[e] = -1;
    }
    if (blockIdx.x == 0 && tid == 0) {
        a.cu[a.B] = (int)rows0;
        if (a.pages_used) a.pages_used[0] = (int)pages0;
    }
}

cudaError_t launch_page_tables(const int *cached, const int *fresh, int n_requests, int page_log2, const int *free_pages,
                               long long n_free, int *table, long long table_stride, int table_cols, int *cu, int *total,
                               int *positions, long long *slot_map, long long n_rows, int *pages_used, cudaStream_t st)
{
    TablesArgs a{cached, fresh, n_requests, page_log2, free_pages, n_free, table, table_stride, table_cols,
                 cu, total, positions, slot_map, n_rows, pages_used,
                 (((uintptr_t)positions | (uintptr_t)slot_map) & 15) == 0};
    long long grid = (n_rows + PT_SPAN - 1) / PT_SPAN;
    const int sms = device_sm_count();
    if (grid < 1) grid = 1;
    if (grid > sms) grid = sms;
    k_page_tables<<<(unsigned)grid, PT_THREADS, 0, st>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace cb
