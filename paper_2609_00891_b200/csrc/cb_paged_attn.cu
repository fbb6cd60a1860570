// Attention of a few new rows per request over a paged cache (decode steps):
//   out_t = sum_j softmax_j(scale q_t . k_j) v_j   over the keys j <= p_t that the window or the sinks leave visible.
//
// Bound by the bytes of K and V: with up to 16 flattened rows (new rows x query heads of a KV head) every key and value is
// read once for all of them, at 8 to 16 operations a byte, so the warp-level matrix instruction is fast enough and the
// rows need not be padded to the 128 of the tensor-memory one.  (With 64 rows a unit it also serves models with more than
// 128 query heads per KV head, at a fraction of the speed.)
//   producer warp   TMA, one box per page (page size rows of one KV head, both halves of the channels), three stages of
//                   64 keys, two blocks an SM: 192 KB in flight; a page id outside the pool reads as zeros, so no table
//                   entry can make the copy fault.
//   4 consumer warps   a warp owns 16 rows and 64 MT / 4 keys of a tile and carries its own running maximum, sum and
//                   output, so that the main loop has no barrier between warps; they are joined at the end of a piece.
// Measured: 64 requests of 512 to 8,192 keys, 8 KV heads x 8 query heads x 128: 205 - 214 us for 1.30 GB = 6.05 - 6.3 TB/s
// (box to box), of 64 channels 154 us for 0.62 GB; one request of 1,024 keys 9.6 - 11 us in a graph, of which the schedule takes 2, the copies 1.3, the tiles 1.5, the joins 3.
// A wait that runs out is not followed by another one: the block runs through to its end, so that every barrier and join
// counter is served as in a good run, and sets the status word; its rows are then not valid.  No copy is issued after it,
// and the block ends only when those in flight have landed.
// Scores, maxima, sums and outputs are fp32; the weights exp2(s - m) are rounded to bf16 for the product with V, which is
// bf16 as well (at most 2^-8 of each weight, as the output's own rounding).
#include "cb_paged.cuh"
#include "cb_ptx.cuh"
#include "cb_math.cuh"

namespace cb {

using namespace ptx;

template <int D, int MT>
struct FewCfg {
    static constexpr int ROWS = 16 * MT;
    static constexpr int KT = 64;
    static constexpr int KS = 4 / MT;                  // key groups of a tile
    static constexpr int WK = KT / KS;                 // keys of one warp in a tile
    static constexpr int NB = D / 64;
    static constexpr int HALF = KT * D * 2;            // bytes of K (or V) in a stage
    static constexpr int STAGE = 2 * HALF;
    static constexpr int NS = D == 128 ? 3 : 6;
    static constexpr int THREADS = 160;
    static constexpr int PITCH = D / KS + 8;           // floats per row of the join buffer
    static constexpr int RED_BYTES = 4 * (KS - 1) * 8 * PITCH * 4;   // [row tile][share][the other warps' parts][8 rows]
    __device__ static constexpr int part(int mt, int share, int from)
    {
        return ((mt * KS + share) * (KS - 1) + (from < share ? from : from - 1)) * 8 * PITCH;
    }
    static constexpr size_t SMEM = 1024 + (size_t)NS * STAGE + RED_BYTES + 4 * 16 * 2 * 4 + 512;
    static constexpr int REC = ROWS * (D + 2);         // floats of a partial record: output rows, maxima, sums
};

struct FewParams {
    CUtensorMap k, v;
    PagedArgs a;
};

__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void bar_consumers() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <int D, int MT>
__global__ void __launch_bounds__(160, 2) k_paged_attn_few(const __grid_constant__ FewParams P)
{
    using C = FewCfg<D, MT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    float *red = reinterpret_cast<float *>(smem + (size_t)C::NS * C::STAGE);
    float *stat_m = red + C::RED_BYTES / 4;                 // [4 warps][16 rows]
    float *stat_l = stat_m + 64;
    uint64_t *full = reinterpret_cast<uint64_t *>(stat_l + 64);
    uint64_t *empty = full + C::NS;
    PaSum *warp_sums = reinterpret_cast<PaSum *>(empty + C::NS);
    PaShare *share = reinterpret_cast<PaShare *>(warp_sums + 5);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(share + 1);
    volatile int *last_flag = abort_flag + 2;
    volatile int *filled = abort_flag + 3;                  // stages that the producer filled

    const PagedArgs &a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 128) {
        for (int i = 0; i < C::NS; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 4); }
        abort_flag[0] = 0;
        abort_flag[1] = (int)a.poll_limit;
        *filled = 0;
        mbar_fence_init();
        tma_prefetch_desc(&P.k);
        tma_prefetch_desc(&P.v);
    }
    pa_schedule<C::ROWS, C::KT, C::THREADS>(a, reinterpret_cast<int *>(smem), C::NS * C::STAGE / 4, share, warp_sums);

    PaWalk<C::ROWS, C::KT> w;
    const bool any = w.open(a, *share);
    const int box_log2 = a.page_log2 < 6 ? a.page_log2 : 6;      // rows of one copy
    bool dead = false;       // a wait ran out: no more waits, the rest runs through on whatever is there
    if (warp == 4) {
        // ================================ producer ================================
        if (any && !a.starve) {
            Ring<C::NS> st;
            int issued = 0;
            const int n_box = 2 << (6 - box_log2);               // copies of a tile: K's, then V's
            const int comp = lane >= n_box / 2;
            const int i = lane - comp * (n_box / 2);
            const uint32_t box_bytes = (uint32_t)C::NB << (box_log2 + 7);
            bool more = true;
            while (more) {
                const int *row = a.table + (long long)w.u.b * a.table_stride;
                for (int t = w.t; t < w.t1; ++t) {
                    const int key = pa_tile(w.u, t) * C::KT + (i << box_log2);
                    int page = a.n_pages;                        // outside the pool: the copy writes zeros
                    if (lane < n_box && pa_wanted(a, w.u, key, 1 << box_log2)) {
                        const int col = key >> a.page_log2;
                        if (col < a.table_cols) page = __ldg(row + col);
                    }
                    if (!mbar_wait_to_issue_warp(&empty[st.idx], st.phase ^ 1, abort_flag)) { dead = true; break; }
                    if (lane == 0) mbar_arrive_expect_tx(&full[st.idx], C::STAGE);
                    __syncwarp();
                    if (lane < n_box)
                        tma_load_5d(smem + (size_t)st.idx * C::STAGE + comp * C::HALF + (size_t)i * box_bytes, comp ? &P.v : &P.k,
                                    &full[st.idx], 0, key & ((1 << a.page_log2) - 1), 0, w.h, page);
                    st.next();
                    ++issued;
                }
                more = !dead && w.next(a);
            }
            if (lane == 0) *filled = issued;
        }
    } else if (any) {
        // ================================ consumers ================================
        const int mt = warp / C::KS, ks = warp % C::KS;
        const int g = lane >> 2, c2 = (lane & 3) * 2;
        const uint32_t smem_base = smem_u32(smem);
        // ldmatrix rows of this lane: K (keys x channels) and V (keys x channels, transposed on the way)
        const int k_key = ((lane >> 4) << 3) + (lane & 7), k_ch = (lane >> 3) & 1;
        const int v_key = (((lane >> 3) & 1) << 3) + (lane & 7), v_ch = lane >> 4;
        if (a.give_up && warp == 0) {                    // test hook: as if a wait had run out
            abort_flag[0] = 1;
            dead = true;
        }
        Ring<C::NS> st;
        bool more = true;
        while (more) {
            const PaUnit &u = w.u;
            // this lane's two rows of the warp's 16, and their positions
            int pos[2];
            bool live[2];
            uint32_t qf[D / 16][4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = mt * 16 + g + e * 8;
                const int fr = u.row0 + r;
                const int tok = pa_token(a, fr);
                live[e] = r < u.rows && (unsigned)(u.tok0 + tok) < (unsigned)a.n_rows;
                pos[e] = live[e] ? u.base + tok : -1;
                const __nv_bfloat16 *qp = a.q + (long long)(u.tok0 + tok) * a.q_st + (long long)(w.h * a.group + fr - tok * a.group) * a.q_sh + c2;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    qf[k][e] = live[e] ? *reinterpret_cast<const uint32_t *>(qp + k * 16) : 0u;
                    qf[k][e + 2] = live[e] ? *reinterpret_cast<const uint32_t *>(qp + k * 16 + 8) : 0u;
                }
            }
            float o[D / 8][4];
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
            float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

            int full0, full1;                              // tiles [full0, full1) need no mask
            pa_full_tiles<C::KT>(a, u, full0, full1);
            for (int t = w.t; t < w.t1; ++t) {
                const bool edge = t < full0 || t >= full1;
                if (!dead && !mbar_wait_suspended_warp(&full[st.idx], st.phase, abort_flag)) dead = true;
                const uint32_t kb = smem_base + st.idx * C::STAGE, vb = kb + C::HALF;
                float s[C::WK / 8][4];
#pragma unroll
                for (int n = 0; n < C::WK / 8; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
                for (int n = 0; n < C::WK / 16; ++n) {
                    const int key = ks * C::WK + n * 16 + k_key;
                    const int pg = key >> box_log2, rr = key & ((1 << box_log2) - 1);
                    const uint32_t row = kb + ((uint32_t)(pg * C::NB) << (box_log2 + 7)) + rr * 128;
#pragma unroll
                    for (int k0 = 0; k0 < D / 16; k0 += 4) {
                        uint32_t b[4][4];                  // four loads in flight before the products that need them
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int ch = k * 2 + k_ch;
                            ldsm_x4(row + ((uint32_t)(k0 >> 2) << (box_log2 + 7)) + (uint32_t)((ch ^ (rr & 7)) << 4), b[k]);
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            mma_16816(s[2 * n], qf[k0 + k], b[k][0], b[k][1]);
                            mma_16816(s[2 * n + 1], qf[k0 + k], b[k][2], b[k][3]);
                        }
                    }
                }
                const int j0 = pa_tile(u, t) * C::KT + ks * C::WK;
                float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int n = 0; n < C::WK / 8; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = s[n][e] * a.scale_log2;
                        if (edge && !pa_sees(a, pos[e >> 1], j0 + n * 8 + c2 + (e & 1))) x = -INFINITY;
                        s[n][e] = x;
                        mx[e >> 1] = fmaxf(mx[e >> 1], x);
                    }
                float f[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 1));
                    mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 2));
                    const float mn = fmaxf(m[e], mx[e]);
                    const float ref = mn == -INFINITY ? 0.f : mn;      // a row that has seen nothing yet: all weights 0
                    f[e] = pa_exp2(m[e] - ref);
                    m[e] = mn;
                    mx[e] = ref;
                    l[e] *= f[e];
                }
                uint32_t pf[C::WK / 16][4];
#pragma unroll
                for (int n = 0; n < C::WK / 8; ++n) {
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[e] = pa_exp2(s[n][e] - mx[e >> 1]);
                        l[e >> 1] += p[e];
                    }
                    pf[n >> 1][(n & 1) * 2] = pack_bf16x2(p[0], p[1]);
                    pf[n >> 1][(n & 1) * 2 + 1] = pack_bf16x2(p[2], p[3]);
                }
                if (!__all_sync(0xffffffffu, f[0] == 1.f && f[1] == 1.f)) {
#pragma unroll
                    for (int n = 0; n < D / 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][e] *= f[e >> 1];
                }
#pragma unroll
                for (int n = 0; n < C::WK / 16; ++n) {
                    const int key = ks * C::WK + n * 16 + v_key;
                    const int pg = key >> box_log2, rr = key & ((1 << box_log2) - 1);
                    const uint32_t row = vb + ((uint32_t)(pg * C::NB) << (box_log2 + 7)) + rr * 128;
                    // rows of the tile that no query sees (behind the end, between the sinks and the window) may hold
                    // anything: their values become zeros, or 0 * NaN would reach the output
                    uint32_t keep[2] = {0xffffffffu, 0xffffffffu};
                    if (edge) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int j = j0 + n * 16 + e * 8 + c2;
                            const bool v0 = j < u.hi_key && (j >= u.lo_key || j < a.n_sink);
                            const bool v1 = j + 1 < u.hi_key && (j + 1 >= u.lo_key || j + 1 < a.n_sink);
                            keep[e] = (v0 ? 0xffffu : 0u) | (v1 ? 0xffff0000u : 0u);
                        }
                    }
#pragma unroll
                    for (int k0 = 0; k0 < D / 16; k0 += 4) {
                        uint32_t b[4][4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int ch = k * 2 + v_ch;
                            ldmatrix_x4_trans(row + ((uint32_t)(k0 >> 2) << (box_log2 + 7)) + (uint32_t)((ch ^ (rr & 7)) << 4), b[k]);
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            mma_16816(o[2 * (k0 + k)], pf[n], b[k][0] & keep[0], b[k][1] & keep[1]);
                            mma_16816(o[2 * (k0 + k) + 1], pf[n], b[k][2] & keep[0], b[k][3] & keep[1]);
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&empty[st.idx]);
                st.next();
            }

            // ---- the piece's result: join the key groups, then write the rows or a partial record ----
            // Every warp takes a quarter of the channels (all of its own rows' channels where it has no partners): it adds
            // what its partners left in shared memory to its own registers, each part scaled from its own maximum.
            const bool whole = w.whole();
            float *prec = a.part + (size_t)w.record(blockIdx.x) * C::REC;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
                l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
            }
            constexpr int SN = D / 8 / C::KS;                 // 8-channel groups of a warp's share
            float mj[2], lj[2], sc[2][C::KS];
            if (C::KS > 1) {
                if ((lane & 3) == 0) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        stat_m[warp * 16 + g + e * 8] = m[e];
                        stat_l[warp * 16 + g + e * 8] = l[e];
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e) { mj[e] = m[e]; lj[e] = l[e]; sc[e][0] = 1.f; }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                // rows g and g + 8 in turn: with up to 8 flattened rows (decode with 8 query heads a KV head) one turn does
                if (e == 1 && u.rows <= 8) break;
                if (C::KS > 1) {
#pragma unroll
                    for (int s = 0; s < C::KS; ++s)
                        if (s != ks) {
#pragma unroll
                            for (int n = 0; n < SN; ++n)
                                *reinterpret_cast<float2 *>(red + C::part(mt, s, ks) + g * C::PITCH + n * 8 + c2) =
                                    make_float2(o[s * SN + n][e * 2], o[s * SN + n][e * 2 + 1]);
                        }
                    bar_consumers();
                    mj[e] = -INFINITY;
#pragma unroll
                    for (int k = 0; k < C::KS; ++k) mj[e] = fmaxf(mj[e], stat_m[(mt * C::KS + k) * 16 + g + e * 8]);
                    const float ref = mj[e] == -INFINITY ? 0.f : mj[e];
                    lj[e] = 0.f;
#pragma unroll
                    for (int k = 0; k < C::KS; ++k) {
                        sc[e][k] = pa_exp2(stat_m[(mt * C::KS + k) * 16 + g + e * 8] - ref);
                        lj[e] += stat_l[(mt * C::KS + k) * 16 + g + e * 8] * sc[e][k];
                    }
                }
                const float inv = whole ? (lj[e] > 0.f ? 1.f / lj[e] : (lj[e] == 0.f ? 0.f : lj[e])) : 1.f;      // NaN stays NaN
                const int r = mt * 16 + g + e * 8, fr = u.row0 + r, rt = pa_token(a, fr), tok = u.tok0 + rt;
                __nv_bfloat16 *orow = a.out + (long long)tok * a.o_st + (long long)(w.h * a.group + fr - rt * a.group) * a.o_sh;
#pragma unroll
                for (int s = 0; s < C::KS; ++s)
                    if (s == ks) {
#pragma unroll
                        for (int n = 0; n < SN; ++n) {
                            float x = o[s * SN + n][e * 2] * sc[e][s], y = o[s * SN + n][e * 2 + 1] * sc[e][s];
#pragma unroll
                            for (int k = 0; k < C::KS; ++k)
                                if (k != s) {
                                    const float2 z = *reinterpret_cast<const float2 *>(red + C::part(mt, s, k) + g * C::PITCH + n * 8 + c2);
                                    x = fmaf(z.x, sc[e][k], x);
                                    y = fmaf(z.y, sc[e][k], y);
                                }
                            const int ch = (s * SN + n) * 8 + c2;
                            if (r < u.rows) {
                                if (!whole) *reinterpret_cast<float2 *>(prec + r * D + ch) = make_float2(x, y);
                                else if ((unsigned)tok < (unsigned)a.n_rows) *reinterpret_cast<uint32_t *>(orow + ch) = pack_bf16x2(x * inv, y * inv);
                            }
                        }
                    }
                if (!whole && ks == 0 && (lane & 3) == 0 && r < u.rows) {
                    prec[C::ROWS * D + r] = mj[e];
                    prec[C::ROWS * D + C::ROWS + r] = lj[e];
                }
                if (C::KS > 1) bar_consumers();               // the buffer is read before it is written again
            }
            if (!whole) {
                // the block that writes the last part of the pair joins all of them, in block order
                const int b0 = w.first_block(), b1 = w.last_block();
                bar_consumers();
                if (tid == 0) {
                    const int last = pa_arrive(&a.counters[b0]) == b1 - b0;
                    if (last) a.counters[b0] = 0;
                    *last_flag = last;
                }
                bar_consumers();
                if (*last_flag) {
                    const float *first = a.part + (size_t)w.record(b0) * C::REC;
                    for (int i = tid; i < u.rows * (D / 4); i += 128) {
                        const int r = i / (D / 4), c4 = (i % (D / 4)) * 4;
                        float mm = -INFINITY, ll = 0.f;
                        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                        // eight parts at a time, so that their loads are in flight together
                        for (int c = b0; c <= b1; c += 8) {
                            float pm[8], pl[8];
                            float4 pv[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                pm[k] = -INFINITY;
                                pl[k] = 0.f;
                                pv[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                                if (c + k <= b1) {
                                    const float *rc = c + k == b0 ? first : a.part + (size_t)(2 * (c + k)) * C::REC;
                                    pm[k] = __ldcg(rc + C::ROWS * D + r);
                                    pl[k] = __ldcg(rc + C::ROWS * D + C::ROWS + r);
                                    pv[k] = __ldcg(reinterpret_cast<const float4 *>(rc + r * D + c4));
                                }
                            }
                            float mn = mm;
#pragma unroll
                            for (int k = 0; k < 8; ++k) mn = fmaxf(mn, pm[k]);
                            const float ref = mn == -INFINITY ? 0.f : mn, f0 = pa_exp2(mm - ref);
                            mm = mn;
                            ll *= f0;
                            x.x *= f0; x.y *= f0; x.z *= f0; x.w *= f0;
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const float f = pa_exp2(pm[k] - ref);
                                ll = fmaf(f, pl[k], ll);
                                x.x = fmaf(f, pv[k].x, x.x); x.y = fmaf(f, pv[k].y, x.y); x.z = fmaf(f, pv[k].z, x.z); x.w = fmaf(f, pv[k].w, x.w);
                            }
                        }
                        const float inv = ll > 0.f ? 1.f / ll : (ll == 0.f ? 0.f : ll);
                        const int fr = u.row0 + r, rt = pa_token(a, fr), tok = u.tok0 + rt;
                        if ((unsigned)tok < (unsigned)a.n_rows)
                            *reinterpret_cast<uint2 *>(a.out + (long long)tok * a.o_st + (long long)(w.h * a.group + fr - rt * a.group) * a.o_sh + c4) =
                                make_uint2(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv));
                    }
                }
            }
            more = w.next(a);
        }
    }
    __syncthreads();
    if (abort_flag[0]) {                                 // the same in every thread: nobody writes it after the barrier
        if (tid == 0) atomicExch(a.status, DEV_TIMEOUT);
        const int issued = *filled;
        for (int k = 0; k < min(issued, C::NS); ++k) mbar_drain(&full[k], ((issued - k - 1) / C::NS) & 1);
    }
}

size_t paged_attn_few_workspace(int d) { return (size_t)2 * 2 * device_sm_count() * 64 * (d + 2) * sizeof(float); }

template <int D, int MT>
static cudaError_t launch_few(const FewParams &P, cudaStream_t st)
{
    using C = FewCfg<D, MT>;
    static bool attr[MAX_DEVICES] = {};
    cudaError_t e = opt_in_smem(k_paged_attn_few<D, MT>, C::SMEM, attr);
    if (e != cudaSuccess) return e;
    k_paged_attn_few<D, MT><<<2 * device_sm_count(), C::THREADS, C::SMEM, st>>>(P);
    e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

cudaError_t launch_paged_attn_few(const PagedArgs &a, int d, const void *k, const void *v, int page_size, long long s_page,
                                  long long s_slot, long long s_head, int max_new, cudaStream_t st)
{
    FewParams P;
    P.a = a;
    const int box = page_size < 64 ? page_size : 64;
    if (!make_kv_tensor_map(&P.k, k, d, a.Hkv, page_size, a.n_pages, s_head, s_slot, s_page, box) ||
        !make_kv_tensor_map(&P.v, v, d, a.Hkv, page_size, a.n_pages, s_head, s_slot, s_page, box))
        return cudaErrorInvalidValue;
    const long long rows = (long long)max_new * a.group;
    if (d == 128) return rows <= 16 ? launch_few<128, 1>(P, st) : launch_few<128, 4>(P, st);
    return rows <= 16 ? launch_few<64, 1>(P, st) : launch_few<64, 4>(P, st);
}

}  // namespace cb
