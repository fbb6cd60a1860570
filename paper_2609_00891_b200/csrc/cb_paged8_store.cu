// Rows into the pages of a cache held in 8 bits, and back.  Both are bound by HBM: every row is read once and written once,
// in 3 bytes a value (bf16) or 5 (fp32).
#include "cb_paged8.cuh"
#include "cb_math.cuh"

namespace cb {

// A run is the rows of one block that stand together in slot_map (up to 31 skipped rows between two of them); a warp does
// one run of one head, K or V: largest magnitude, exponent, codes.  The first 16 rows stay in registers in between, so that
// a row is read once; those of a longer run come from L2 the second time.
// grid (row tiles, layers, groups of wpr of the 2 H heads of K and V); a block's 8 / wpr warp groups take its runs in turn.
template <bool F32, int FMT, int D>
__global__ void __launch_bounds__(256) k_paged8_store(const Store8Args a)
{
    constexpr int LPR = D / 8;                   // lanes of a row, 8 channels each
    constexpr int RPI = 32 / LPR;                // rows of one load of the warp
    constexpr int KEEP = 16;                     // rows of a chunk
    constexpr int ITER = KEEP / RPI;
    constexpr int W = F32 ? 2 : 1;               // 16-byte pieces of 8 channels
    const Pool8 &p = a.pool;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int pair = blockIdx.z * a.wpr + warp % a.wpr;
    if (pair >= 2 * p.H) return;
    const int h = pair >> 1, comp = pair & 1;
    const long long r0 = (long long)blockIdx.x * a.tile;
    const int layer = blockIdx.y;

    auto slot_of = [&](long long row) { return row >= 0 && row < a.n_rows ? __ldg(a.slot_map + row) : -1ll; };
    auto fits = [&](long long slot) { return slot >= 0 && slot < p.n_slots; };
    // runs that begin in this tile: valid rows whose nearest valid row of the 32 before them is of another block, or missing
    const long long mine = lane < a.tile ? slot_of(r0 + lane) : -1;
    const long long my_block = mine >> p.block_log2;
    const bool ok = fits(mine);
    const unsigned valid = __ballot_sync(0xffffffffu, ok);
    if (!valid) return;
    const long long back = slot_of(r0 - 32 + lane);
    const unsigned valid_back = __ballot_sync(0xffffffffu, fits(back));
    const unsigned here = valid & ((1u << lane) - 1u);
    const int from = here ? 31 - __clz(here) : valid_back ? 31 - __clz(valid_back) : 0;
    const long long prev_here = __shfl_sync(0xffffffffu, mine, from), prev_back = __shfl_sync(0xffffffffu, back, from);
    const bool near = here || (valid_back && lane <= from);                // at most 32 rows back
    const bool head = ok && !(near && ((here ? prev_here : prev_back) >> p.block_log2) == my_block);
    const unsigned heads = __ballot_sync(0xffffffffu, head);
    const int rank = __popc(heads & ((1u << lane) - 1u));

    const int sub = lane / LPR, c8 = (lane % LPR) * 8;                     // row of a load, first channel
    const char *src = static_cast<const char *>(comp ? a.src_v : a.src_k) + ((long long)layer * a.s_sl + (long long)h * a.s_sh + c8) * (F32 ? 4 : 2);
    uint8_t *codes = (comp ? p.v : p.k) + (long long)layer * p.sl + (long long)h * p.sh;
    int8_t *exps = (comp ? p.ve : p.ke) + (long long)layer * p.el + (long long)h * p.eh;
    const int slot_mask = (1 << p.page_log2) - 1, n_groups = 8 / a.wpr;

    for (int run = warp / a.wpr; run < __popc(heads); run += n_groups) {
        const int at = __ffs(__ballot_sync(0xffffffffu, head && rank == run)) - 1;
        const long long begin = r0 + at;
        const long long block = __shfl_sync(0xffffffffu, my_block, at);
        // rows of the run among the 32 from `row`, as bits; `last`: the latest one found so far, -1 at the end of the run
        long long slot;                                                    // this lane's
        auto members = [&](long long row, long long &last) -> unsigned {
            slot = slot_of(row + lane);
            const bool v = fits(slot), same = v && (slot >> p.block_log2) == block;
            unsigned m = __ballot_sync(0xffffffffu, same);
            const unsigned other = __ballot_sync(0xffffffffu, v && !same);
            if (other) m &= (other & -other) - 1u;                         // up to the next block's first row
            if (!m || row + __ffs(m) - 1 - last > 32) { last = -1; return 0u; }
            last = other ? -1 : row + 31 - __clz(m);
            return m;
        };
        uint4 keep[ITER][W];
        float most = 0.f;
        unsigned m0 = 0;                                                   // the first window's rows
        long long slot0 = -1;
        bool begun = false;
        auto load = [&](long long row, unsigned m, int first, uint4 (&x)[ITER][W]) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int k = first + i * RPI + sub;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    x[i][w] = make_uint4(0, 0, 0, 0);
                    if (m >> k & 1) x[i][w] = __ldg(reinterpret_cast<const uint4 *>(src + (row + k) * a.s_st * (F32 ? 4 : 2)) + w);
                }
            }
        };
        auto values = [&](const uint4 (&x)[W], float (&f)[8]) {
            if (F32) {
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    f[w * 4] = __uint_as_float(x[w].x); f[w * 4 + 1] = __uint_as_float(x[w].y);
                    f[w * 4 + 2] = __uint_as_float(x[w].z); f[w * 4 + 3] = __uint_as_float(x[w].w);
                }
            } else {
                const uint32_t u[4] = {x[0].x, x[0].y, x[0].z, x[0].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) { f[2 * j] = __uint_as_float(u[j] << 16); f[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u); }
            }
        };
        auto largest = [&](const uint4 (&x)[ITER][W]) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                float f[8];
                values(x[i], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(f[j]));   // NaN is passed over
            }
        };
        // ---- largest magnitude ----
        long long last = begin;
        for (long long row = begin; last >= 0; row += 32) {
            const unsigned m = members(row, last);
            if (!m) break;
            begun |= __any_sync(0xffffffffu, (m >> lane & 1) && (slot & ((1 << p.block_log2) - 1)) == 0);
            if (row == begin) {
                m0 = m;
                slot0 = slot;
                load(row, m, 0, keep);
                largest(keep);
            }
            for (int first = row == begin ? KEEP : 0; first < 32; first += KEEP) {
                if (!(m >> first)) break;
                uint4 x[ITER][W];
                load(row, m, first, x);
                largest(x);
            }
        }
        const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(most));
        const long long page = block >> (p.page_log2 - p.block_log2), in_page = block & ((1 << (p.page_log2 - p.block_log2)) - 1);
        int8_t *ep = exps + page * p.ep + in_page * p.eb;
        uint8_t *base = codes + page * p.sp;
        const int need = exp8_need<FMT>(top);
        int e = need;
        if (!begun) {
            const int old = exp8_clamp(__shfl_sync(0xffffffffu, lane == 0 ? (int)*ep : 0, 0), FMT);
            e = max(old, need);
            if (e > old) {                                                 // the block's codes, rounded to the larger step
                const float f = exp2_whole(max(old - e, -126));
                for (int r = sub; r < 1 << p.block_log2; r += RPI) {
                    uint2 *q = reinterpret_cast<uint2 *>(base + ((in_page << p.block_log2) + r) * p.ss + c8);
                    const uint2 c = *q;
                    *q = make_uint2(to_codes<FMT>(codes_to_f32<FMT>(c.x, f)), to_codes<FMT>(codes_to_f32<FMT>(c.y, f)));
                }
                __syncwarp();
            }
        }
        if (lane == 0) *ep = (int8_t)e;
        // ---- codes ----
        const float f = exp2_whole(-e);
        auto write = [&](const uint4 (&x)[ITER][W], unsigned m, int first, long long slots) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int k = first + i * RPI + sub;
                const long long to = __shfl_sync(0xffffffffu, slots, k);
                if (m >> k & 1) {
                    float v[8];
                    values(x[i], v);
                    *reinterpret_cast<uint2 *>(base + (to & slot_mask) * p.ss + c8) =
                        make_uint2(to_codes<FMT>(make_float4(v[0] * f, v[1] * f, v[2] * f, v[3] * f)), to_codes<FMT>(make_float4(v[4] * f, v[5] * f, v[6] * f, v[7] * f)));
                }
            }
        };
        write(keep, m0, 0, slot0);
        last = begin;
        for (long long row = begin; last >= 0; row += 32) {
            const unsigned m = members(row, last);
            if (!m) break;
            for (int first = row == begin ? KEEP : 0; first < 32; first += KEEP) {
                if (!(m >> first)) break;
                uint4 x[ITER][W];
                load(row, m, first, x);
                write(x, m, first, slot);
            }
        }
        __syncwarp();
    }
}

cudaError_t launch_paged8_store(const Store8Args &args, bool f32, cudaStream_t st)
{
    Store8Args a = args;
    // Rows of a block: 32 where there are enough of them for four blocks an SM, fewer otherwise (a step's few rows).
    const long long wanted = 4ll * device_sm_count();
    a.tile = 32;
    a.wpr = 1;
    while (a.wpr < 8 && a.wpr < 2 * a.pool.H) a.wpr *= 2;
    const int groups = (2 * a.pool.H + a.wpr - 1) / a.wpr;
    while (a.tile > 1 && (a.n_rows + a.tile - 1) / a.tile * a.pool.L * groups < wanted) a.tile /= 2;
    dim3 grid((unsigned)((a.n_rows + a.tile - 1) / a.tile), (unsigned)a.pool.L, (unsigned)groups);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(a); };
    const bool e4m3 = a.pool.format == CACHE_E4M3;
    if (a.pool.d == 128) {
        if (f32) e4m3 ? go(k_paged8_store<true, CACHE_E4M3, 128>) : go(k_paged8_store<true, CACHE_INT8, 128>);
        else e4m3 ? go(k_paged8_store<false, CACHE_E4M3, 128>) : go(k_paged8_store<false, CACHE_INT8, 128>);
    } else {
        if (f32) e4m3 ? go(k_paged8_store<true, CACHE_E4M3, 64>) : go(k_paged8_store<true, CACHE_INT8, 64>);
        else e4m3 ? go(k_paged8_store<false, CACHE_E4M3, 64>) : go(k_paged8_store<false, CACHE_INT8, 64>);
    }
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

// A thread takes NV codes (16 bytes of the result) of four rows' heads, of K and of V: eight loads in flight.
template <bool F32, int FMT>
__global__ void __launch_bounds__(256) k_paged8_load(const Load8Args a)
{
    constexpr int NV = F32 ? 4 : 8, U = 4;
    const Pool8 &p = a.pool;
    const int pieces = p.d / NV;
    const unsigned per_row = (unsigned)(p.H * pieces);
    const long long i0 = (long long)blockIdx.x * (256 * U) + threadIdx.x, layer = blockIdx.y;
    long long to[U];
    uint32_t ck[U][NV / 4], cv[U][NV / 4];
    float fk[U], fv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long i = i0 + u * 256;
        const long long row = ((unsigned long long)i >> 32) == 0 ? (long long)((unsigned)i / per_row) : i / per_row;
        const int rest = (int)(i - row * per_row), h = rest / pieces, c = (rest - h * pieces) * NV;
        to[u] = -1;
        const long long slot = row < a.n_rows ? __ldg(a.slot_map + row) : -1;
        if (slot >= 0 && slot < p.n_slots) {
            to[u] = layer * a.d_sl + row * a.d_st + (long long)h * a.d_sh + c;
            const long long page = slot >> p.page_log2, off = slot & ((1 << p.page_log2) - 1);
            const long long from = layer * p.sl + page * p.sp + off * p.ss + (long long)h * p.sh + c;
            const long long ex = layer * p.el + page * p.ep + (off >> p.block_log2) * p.eb + (long long)h * p.eh;
            if (NV == 8) {
                const uint2 x = __ldcs(reinterpret_cast<const uint2 *>(p.k + from)), y = __ldcs(reinterpret_cast<const uint2 *>(p.v + from));
                ck[u][0] = x.x; ck[u][NV / 4 - 1] = x.y;
                cv[u][0] = y.x; cv[u][NV / 4 - 1] = y.y;
            } else {
                ck[u][0] = __ldcs(reinterpret_cast<const uint32_t *>(p.k + from));
                cv[u][0] = __ldcs(reinterpret_cast<const uint32_t *>(p.v + from));
            }
            fk[u] = exp2_whole(exp8_clamp(__ldg(p.ke + ex), FMT));
            fv[u] = exp2_whole(exp8_clamp(__ldg(p.ve + ex), FMT));
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (to[u] < 0) continue;
#pragma unroll
        for (int comp = 0; comp < 2; ++comp) {
            const float f = comp ? fv[u] : fk[u];
            const uint32_t(&c)[NV / 4] = comp ? cv[u] : ck[u];
            void *dst = comp ? a.dst_v : a.dst_k;
            const float4 x = codes_to_f32<FMT>(c[0], f);
            if (F32) {
                __stcs(reinterpret_cast<float4 *>(static_cast<float *>(dst) + to[u]), x);
            } else {
                const float4 y = codes_to_f32<FMT>(c[NV / 4 - 1], f);
                __stcs(reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(dst) + to[u]),
                       make_uint4(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w), pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w)));
            }
        }
    }
}

cudaError_t launch_paged8_load(const Load8Args &a, bool f32, cudaStream_t st)
{
    const long long n = a.n_rows * a.pool.H * (a.pool.d / (f32 ? 4 : 8));
    dim3 grid((unsigned)((n + 1023) / 1024), (unsigned)a.pool.L);
    const bool e4m3 = a.pool.format == CACHE_E4M3;
    if (f32) e4m3 ? k_paged8_load<true, CACHE_E4M3><<<grid, 256, 0, st>>>(a) : k_paged8_load<true, CACHE_INT8><<<grid, 256, 0, st>>>(a);
    else e4m3 ? k_paged8_load<false, CACHE_E4M3><<<grid, 256, 0, st>>>(a) : k_paged8_load<false, CACHE_INT8><<<grid, 256, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace cb
