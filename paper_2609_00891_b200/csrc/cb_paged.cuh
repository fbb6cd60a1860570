// Paged target cache: declarations shared by the attention kernels and their host side (not part of the C ABI).
//
// Attention work is cut into units (request, block of ROWS flattened query rows); a flattened row is token * group + g,
// so that every query head which shares a KV head sits in one block and the keys are read once for all of them.  A unit
// and a KV head together own n key tiles; all tiles of all (unit, KV head) pairs are laid out on one line, in unit
// order, and block c of the grid takes the tiles [c Q, (c + 1) Q): every block has the same number of tiles whatever the
// lengths are.  A pair whose tiles fall to several blocks is joined by the block that finishes last, in block order.
#pragma once

#include "cb_internal.cuh"

namespace cb {

constexpr int PA_COUNTERS = 2048;            // one per block (warp-level kernel), eight per block (two tiles of four warps)
constexpr size_t PA_COUNTER_BYTES = PA_COUNTERS * sizeof(int);

struct PagedArgs {
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    long long q_st, q_sh, o_st, o_sh;        // element strides of a token and of a head
    const int *table;                        // device [n_requests][table_cols]
    long long table_stride;
    int table_cols;
    const int *cu;                           // device [n_requests + 1]: first row of every request
    const int *total;                        // device [n_requests]: rows in the cache, the new ones included
    int n_requests, n_rows;                  // n_rows: rows of q and out
    int Hkv, group;
    unsigned group_mul;                      // ceil(2^32 / group) where that divides every row index exactly, else 0
    int unit_tokens, unit_rows;              // tensor-core kernel: new rows of a unit, and flattened
    unsigned unit_mul;                       // as group_mul, for unit_tokens
    int page_log2;
    int n_pages;
    int window, n_sink;                      // window 0: none
    float scale_log2;                        // softmax scale times log2(e)
    int q_min;                               // least tiles a block takes
    float *part;                             // partial results of split pairs, two records per block
    int *counters;                           // [PA_COUNTERS], zero between calls
    int *status;
    unsigned poll_limit;
    int starve, give_up;
};

cudaError_t launch_paged_attn_few(const PagedArgs &a, int d, const void *k, const void *v, int page_size, long long s_page,
                                  long long s_slot, long long s_head, int max_new, cudaStream_t st);
size_t paged_attn_few_workspace(int d);
cudaError_t launch_paged_attn_tc(const PagedArgs &a, int d, const void *k, const void *v, int page_size, long long s_page,
                                 long long s_slot, long long s_head, cudaStream_t st);
size_t paged_attn_tc_workspace(int d);

cudaError_t launch_page_tables(const int *cached, const int *fresh, int n_requests, int page_log2, const int *free_pages,
                               long long n_free, int *table, long long table_stride, int table_cols, int *cu, int *total,
                               int *positions, long long *slot_map, long long n_rows, int *pages_used, cudaStream_t st);

struct StoreArgs {
    const void *src_k, *src_v;
    int src_f32;
    long long s_sl, s_st, s_sh;              // source strides (elements): layer, token, head
    __nv_bfloat16 *k, *v;
    long long d_sl, d_sp, d_ss, d_sh;        // pool strides (elements): layer, page, slot, head
    const long long *slot_map;
    long long n_slots, n_rows;               // n_slots = pages * page size
    int page_log2, L, H, d;
};
cudaError_t launch_paged_store(const StoreArgs &a, cudaStream_t st);

cudaError_t launch_rope_axes(const void *x, void *out, int L, int H, int d, long long T, const long long xs[3],
                             const long long os[3], const int *positions, long long axis_stride, const unsigned char *axis_of_pair,
                             double base, int inverse, cudaStream_t st);

#ifdef __CUDACC__
// Flattened row -> row of the request (n / group): an integer division is ~30 dependent instructions, and several of them
// stand between the launch and the first copy.
__device__ __forceinline__ int pa_token(const PagedArgs &a, int n)
{
    return a.group_mul ? (int)__umulhi((unsigned)n, a.group_mul) : a.group == 1 ? n : n / a.group;
}
// Quotient of two non-negative numbers, in 32 bits where both fit.
__device__ __forceinline__ long long pa_div(long long n, long long d)
{
    return ((n | d) >> 32) == 0 ? (long long)((unsigned)n / (unsigned)d) : n / d;
}

// The unit at or before request row n, of units counted from row 0; ROWS flattened rows a unit, or a.unit_tokens rows (0).
template <int ROWS>
__device__ __forceinline__ int pa_unit_of(const PagedArgs &a, int n)
{
    if (ROWS) return (int)((unsigned)n * (unsigned)a.group / (ROWS ? ROWS : 1));
    return a.unit_mul ? (int)__umulhi((unsigned)n, a.unit_mul) : n / a.unit_tokens;
}

// One unit's place in the batch and its key tiles of KT keys.
struct PaUnit {
    int b, qt, nq;          // request, row block, row blocks of the request
    int row0, rows;         // first flattened row, rows in the block (those that q has)
    int tok0;               // first row of the request in q
    int base;               // position of the request's first new row (negative if the cache is shorter than the chunk)
    int p0, p1;             // positions of the block's first and last row
    int hi_key;             // keys [0, hi_key) can be seen by some row
    int lo_key;             // without the sinks, keys from lo_key on
    int ns, lo_tile, n;     // tiles that hold sinks, first tile of the window, number of tiles (at least 1)
};

template <int ROWS, int KT>
__device__ __forceinline__ bool pa_unit(const PagedArgs &a, const int *cu, const int *total, int b, int qt, PaUnit &u)
{
    const int c0 = cu[b], fresh = cu[b + 1] - c0;
    const int here = max(0, min(cu[b + 1], a.n_rows) - c0);       // rows past the room of q are dropped
    const int all = here * a.group;
    u.b = b;
    u.qt = qt;
    const int per = ROWS ? ROWS : a.unit_rows;
    u.nq = ROWS ? (all + ROWS - 1) / (ROWS ? ROWS : 1) : pa_unit_of<0>(a, here + a.unit_tokens - 1);
    if (qt >= u.nq) { u.n = 0; return false; }
    u.tok0 = c0;
    u.row0 = qt * per;
    u.rows = min(per, all - u.row0);
    const int len = max(total[b], 0);
    u.base = len - fresh;
    u.p0 = u.base + pa_token(a, u.row0);
    u.p1 = u.base + pa_token(a, u.row0 + u.rows - 1);
    u.hi_key = max(0, u.p1 + 1);
    const int hi_tile = (u.hi_key + KT - 1) / KT;
    u.lo_key = 0;
    u.ns = 0;
    u.lo_tile = 0;
    if (a.window > 0) {
        const long long lo = (long long)u.p0 - a.window + 1;
        u.lo_key = lo > 0 ? (int)lo : 0;
        u.ns = (min(a.n_sink, u.hi_key) + KT - 1) / KT;
        u.lo_tile = max(u.lo_key / KT, u.ns);
    }
    u.n = max(1, u.ns + max(0, hi_tile - u.lo_tile));
    return true;
}
__device__ __forceinline__ int pa_tile(const PaUnit &u, int t) { return t < u.ns ? t : u.lo_tile + (t - u.ns); }

// The tiles [t0, t1) of the unit of which every key is seen by every row (tiles of the sinks are not counted as such).
template <int KT>
__device__ __forceinline__ void pa_full_tiles(const PagedArgs &a, const PaUnit &u, int &t0, int &t1)
{
    int k0 = 0;
    const int k1 = u.p0 < 0 ? 0 : (u.p0 + 1) / KT;
    if (a.window > 0) {
        const long long lo = (long long)u.p1 - a.window + 1;      // first key that the last row sees
        k0 = lo > 0 ? (int)((lo + KT - 1) / KT) : 0;
    }
    t0 = max(u.ns, k0 - u.lo_tile + u.ns);
    t1 = k1 - u.lo_tile + u.ns;
}

// Some key in [key, key + n) is seen by some row of the unit.
__device__ __forceinline__ bool pa_wanted(const PagedArgs &a, const PaUnit &u, int key, int n)
{
    return key < u.hi_key && (key + n > u.lo_key || key < a.n_sink);
}
// Some key of the tile at j0 is seen by no row of the unit.
template <int KT>
__device__ __forceinline__ bool pa_clears(const PagedArgs &a, const PaUnit &u, int j0)
{
    return j0 + KT > u.hi_key || (j0 < u.lo_key && j0 + KT > a.n_sink);
}
__device__ __forceinline__ bool pa_sees(const PagedArgs &a, int p, int j)
{
    return j <= p && (a.window <= 0 || p - j < a.window || j < a.n_sink);
}

// The block's share of the line of tiles, left in shared memory by pa_schedule.
struct PaShare {
    long long begin, end;    // tiles of this block
    long long q;             // tiles per block
    long long unit_begin;    // where the first unit's tiles begin
    PaUnit u;                // the first unit
    int even;                // > 0: every pair takes this many places on the line, and no pair is split
};

struct alignas(16) PaSum { long long tiles; int units, most; };

// All threads of the block.  `staged`: shared memory for the lengths (cap ints), free until the first tile is copied.
// `sums`: one per warp.  Each thread counts the tiles of a run of consecutive units; one scan gives the line, one thread
// finds the block's start.
// Where there are no more pairs than blocks and the longest one is at most EVEN tiles above an equal share, every pair goes
// to a block of its own: joining two parts costs about that much (32 requests with a window of 1,024 keys, 256 pairs of 17
// or 18 tiles of 64 keys: 38 us split, see k_paged_attn_few; for the tensor-memory kernel the number was taken over, not
// measured).  A block takes at least q_min tiles, and the root of (tiles of the longest pair / JOINS), where its tiles and the
// join of its pair's parts take equally long (0: q_min alone).
template <int ROWS, int KT, int THREADS, int EVEN = 4, int JOINS = 0>
__device__ __forceinline__ void pa_schedule(const PagedArgs &a, int *staged, int cap, PaShare *share, PaSum *sums)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int NWARP = THREADS / 32;
    const int *cu = a.cu, *total = a.total;
    const int B = a.n_requests;
    if (2 * B + 1 <= cap) {
        for (int i = tid; i <= B; i += THREADS) staged[i] = a.cu[i];
        for (int i = tid; i < B; i += THREADS) staged[B + 1 + i] = a.total[i];
        cu = staged;
        total = staged + B + 1;
    }
    if (tid == 0) { share->begin = 0; share->end = 0; }
    __syncthreads();
    // unit index u: the last request b with floor((cu[b] - cu[0]) group / ROWS) + b <= u (some indices are no unit); 32 bits
    // hold rows * query heads, checked by the host
    const int cu0 = cu[0];                       // not 0 for the later requests of a batch, called by themselves
    auto first_unit = [&](int b) { return pa_unit_of<ROWS>(a, min(max(cu[b] - cu0, 0), a.n_rows)) + b; };
    const int n_units = pa_unit_of<ROWS>(a, a.n_rows) + B;
    const int per = (n_units + THREADS - 1) / THREADS;
    const int u0 = min(n_units, tid * per), u1 = min(n_units, u0 + per);
    int b0 = 0;
    if (u0 < u1) {
        int lo = 0, hi = B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (first_unit(mid) <= u0) lo = mid; else hi = mid - 1;
        }
        b0 = lo;
    }
    PaUnit un;
    long long mine = 0;
    int count = 0, most = 0;                     // units of this thread, tiles of the longest
    {
        int b = b0;
        for (int u = u0; u < u1; ++u) {
            while (b + 1 < B && first_unit(b + 1) <= u) ++b;
            if (pa_unit<ROWS, KT>(a, cu, total, b, u - first_unit(b), un)) { mine += un.n; ++count; most = max(most, un.n); }
        }
    }
    long long incl = mine;
    int incl_units = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, incl, o);
        const int upu = __shfl_up_sync(0xffffffffu, incl_units, o);
        if (lane >= o) { incl += up; incl_units += upu; }
        most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    }
    if (lane == 31) sums[warp] = PaSum{incl, incl_units, most};
    __syncthreads();
    long long before = 0, all = 0;
    int before_units = 0, all_units = 0;
    most = 0;
#pragma unroll
    for (int w = 0; w < NWARP; ++w) {
        const PaSum s = sums[w];
        if (w < warp) { before += s.tiles; before_units += s.units; }
        all += s.tiles;
        all_units += s.units;
        most = max(most, s.most);
    }
    long long line = all * a.Hkv;
    long long q = pa_div(line + gridDim.x - 1, gridDim.x);
    q = max(q, (long long)max(a.q_min, JOINS ? 1 + (int)sqrtf((float)max(most - 1, 0) / (JOINS ? JOINS : 1)) : 0));
    long long pre = (before + incl - mine) * a.Hkv;
    int even = 0;
    if ((long long)all_units * a.Hkv <= gridDim.x && most <= q + EVEN && most > 0) {
        even = most;
        q = most;
        line = (long long)all_units * a.Hkv * q;
        pre = (long long)(before_units + incl_units - count) * a.Hkv * q;
        mine = (long long)count * even;
    }
    const long long begin = (long long)blockIdx.x * q;
    if (begin < line && begin >= pre && begin < pre + mine * a.Hkv) {
        auto found = [&]() {
            share->u = un;
            share->unit_begin = pre;
            share->q = q;
            share->begin = begin;
            share->end = begin + q < line ? begin + q : line;
            share->even = even;
        };
        if (per == 1) {                          // the thread's one unit is still at hand
            found();
        } else {
            int b = b0;
            for (int u = u0; u < u1; ++u) {
                while (b + 1 < B && first_unit(b + 1) <= u) ++b;
                if (!pa_unit<ROWS, KT>(a, cu, total, b, u - first_unit(b), un)) continue;
                const long long len = (long long)(even ? even : un.n) * a.Hkv;
                if (begin < pre + len) {
                    found();
                    break;
                }
                pre += len;
            }
        }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the staged lengths' memory goes to the copies next
    __syncthreads();
}

// Walks the pieces of a block's share: a piece is a run of tiles of one (unit, KV head).
template <int ROWS, int KT>
struct PaWalk {
    PaUnit u;
    int h, t, t1;            // KV head, tiles [t, t1) of the unit
    int len, even;           // places of the pair on the line
    long long at, end, q;    // position on the line
    long long pair_begin;    // where the places of (unit, h) begin
    __device__ __forceinline__ bool open(const PagedArgs &a, const PaShare &s)
    {
        at = s.begin;
        end = s.end;
        q = s.q;
        even = s.even;
        if (at >= end) return false;
        u = s.u;
        len = even ? even : u.n;
        h = (int)pa_div(at - s.unit_begin, len);
        pair_begin = s.unit_begin + (long long)h * len;
        piece();
        return true;
    }
    __device__ __forceinline__ void piece()
    {
        t = (int)(at - pair_begin);
        t1 = (int)min((long long)u.n, end - pair_begin);
    }
    __device__ __forceinline__ bool next(const PagedArgs &a)
    {
        at = pair_begin + len;
        if (at >= end) return false;
        pair_begin += len;
        if (++h == a.Hkv) {
            h = 0;
            int b = u.b, qt = u.qt + 1;
            if (qt >= u.nq) {
                qt = 0;
                do { ++b; } while (b < a.n_requests && min(a.cu[b + 1], a.n_rows) <= a.cu[b]);
                if (b >= a.n_requests) return false;
            }
            pa_unit<ROWS, KT>(a, a.cu, a.total, b, qt, u);
            len = even ? even : u.n;
        }
        piece();
        return true;
    }
    __device__ __forceinline__ bool whole() const { return t == 0 && t1 == u.n; }
    __device__ __forceinline__ int first_block() const { return (int)pa_div(pair_begin, q); }
    __device__ __forceinline__ int last_block() const { return (int)pa_div(pair_begin + len - 1, q); }
    // Record of block c's part of this pair: a block has at most one part that began before it and one that ends after it.
    __device__ __forceinline__ int record(int c) const { return 2 * c + (pair_begin <= (long long)c * q ? 0 : 1); }
};

// One more part of a pair is in memory (the writes of the threads that met this one before count as its own); how many
// there were before, whose writes are visible from here on.
__device__ __forceinline__ int pa_arrive(int *counter)
{
    int n;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(n) : "l"(counter) : "memory");
    return n;
}
__device__ __forceinline__ float pa_exp2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Largest of three (one instruction on sm_100).
__device__ __forceinline__ float max3(float x, float y, float z)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}
#endif

}  // namespace cb
