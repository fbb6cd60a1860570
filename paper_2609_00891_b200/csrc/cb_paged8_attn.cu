// Attention of a few new rows per request over a paged cache held in 8 bits (decode steps):
//   out_t = sum_j softmax_j(scale q_t . k_j) v_j,   k_j = code 2^e, v_j = code 2^e, e one exponent a block of rows and head.
//
// Bound by the bytes of the codes, which are read once for all query heads of a KV head.  A warp takes 16 keys of every tile
// of 64 and needs no other one until the end of a piece: it copies them into four stages of its own (cp.async; a page id
// outside the pool is filled with zeros), so that the loop has no barrier between warps, and no wait that another thread ends.
//   scores    S^T = K Q^T: the 16 keys are the rows of the warp-level matrix instruction, 8 query rows its columns, so that
//             8 flattened rows cost one instruction where the other order would pad them to 16.
//   channels  the sum over channels has any order: thread t of four takes D / 4 adjacent channels of a key, whose codes are one or
//             two 16-byte loads, and q is laid out in registers the same way.
//   outputs   O^T += V^T P^T: a pair of keys of one channel is a byte of two rows, put side by side by one permutation; the
//             output's channels have any order too, and thread g of eight takes D / 8 adjacent ones.
// Codes become fp16, which holds both formats exactly.  q is scaled by the power of two that brings its row's largest magnitude to
// 2^14 .. 2^15: fp16 then holds every bf16 value down to 2^-29 of that one exactly, and the rest to 2^-40 of it.  The weights are
// 2^6 exp2(s - m) with m at most 2^8 behind the row's maximum, so at most 2^14; they are rounded to fp16 (2^-11 of each
// weight above 2^-20 of the largest) for the product with V, and summed unrounded.  A block's exponent multiplies its scores and its
// part of the output, in fp32.
#include "cb_paged8.cuh"
#include "cb_math.cuh"
#include "cb_ptx.cuh"

namespace cb {

using namespace ptx;

template <int D, int NT>
struct Few8Cfg {
    static constexpr int ROWS = 8 * NT;
    static constexpr int KT = 64;
    static constexpr int NS = D == 128 ? 4 : 8;        // stages of a warp
    static constexpr int HALF = 16 * D;                // bytes of K (or V) in a stage
    static constexpr int STAGE = 2 * HALF;
    static constexpr int RING = NS * STAGE;            // of a warp; holds its output at the end of a piece
    static constexpr int REC = ROWS * (D + 2);         // floats of a partial record: output rows, maxima, sums
    static_assert(RING >= ROWS * D * 4, "the warp's output must fit its stages");
    static constexpr size_t SMEM = 4 * RING;
};

struct Few8Params {
    Pool8 p;
    PagedArgs a;
};

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_1688(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t b)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(b));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// 16 bytes to shared memory, or zeros.
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16u : 0u) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}

// Where the 16-byte piece c of row r of a stage stands, so that the reads below meet no bank twice.  128 channels: rows of eight
// pieces, XORed by the row; 64: two rows a line of eight pieces, XORed by twice the line.
template <int D>
__device__ __forceinline__ uint32_t piece_at(int r, int c)
{
    if (D == 128) return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4));
    return (uint32_t)((r >> 1) * 128 + (((((r & 1) << 2) | c) ^ ((r & 6))) << 4));
}

template <int D, int NT, int FMT>
__global__ void __launch_bounds__(128, 3) k_paged8_attn_few(const __grid_constant__ Few8Params P)
{
    using C = Few8Cfg<D, NT>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ PaShare share;
    __shared__ PaSum warp_sums[4];
    __shared__ float stat_m[4][C::ROWS], stat_l[4][C::ROWS];
    __shared__ int last_flag;
    const PagedArgs &a = P.a;
    const Pool8 &p = P.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t4 = lane & 3;
    constexpr int CQ = D / 4, CPT = D / 8, PIECES = D / 16;
    constexpr int ROWS_I = 32 / PIECES;                // rows of one copy instruction of the warp

    pa_schedule<C::ROWS, C::KT, 128>(a, reinterpret_cast<int *>(smem_raw), (int)(C::SMEM / 4), &share, warp_sums);
    PaWalk<C::ROWS, C::KT> w;
    if (!w.open(a, share)) return;

    uint8_t *ring = smem_raw + warp * C::RING;
    const uint32_t ring_u = smem_u32(ring);
    const int crow = lane / PIECES, cpiece = lane % PIECES;
    const int slot_mask = (1 << a.page_log2) - 1;
    bool more = true;
    while (more) {
        const PaUnit &u = w.u;
        const int n = w.t1 - w.t;
        const int *row = a.table + (long long)u.b * a.table_stride;
        const uint8_t *kb = p.k + (long long)w.h * p.sh, *vb = p.v + (long long)w.h * p.sh;
        const int8_t *eb = ((lane & 2) ? p.ve : p.ke) + (long long)w.h * p.eh;    // lanes 0 .. 3: K of both halves, V of both

        // pages of the two groups of 8 keys of this warp's step s; -1 where no key is wanted
        auto pages = [&](int s, int (&pg)[2]) {
            const int key = pa_tile(u, w.t + s) * C::KT + warp * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pg[h] = -1;
                if (s < n && pa_wanted(a, u, key + 8 * h, 8)) {
                    const int col = (key + 8 * h) >> a.page_log2;
                    if (col < a.table_cols) pg[h] = __ldg(row + col);
                }
            }
        };
        auto issue = [&](int s, int stage, const int (&pg)[2], int &ex) {
            if (s < n) {
                const int key = pa_tile(u, w.t + s) * C::KT + warp * 16;
                const uint32_t to = ring_u + stage * C::STAGE;
#pragma unroll
                for (int i = 0; i < 16 / ROWS_I; ++i) {
                    const int r = i * ROWS_I + crow, page = pg[(i * ROWS_I) >> 3];
                    const bool there = (unsigned)page < (unsigned)p.n_pages;
                    const long long from = there ? (long long)page * p.sp + (long long)((key + r) & slot_mask) * p.ss + cpiece * 16 : 0;
                    cp_async_16(to + piece_at<D>(r, cpiece), kb + from, there);
                    cp_async_16(to + C::HALF + piece_at<D>(r, cpiece), vb + from, there);
                }
                const int page = (lane & 1) ? pg[1] : pg[0];
                ex = 0;
                if (lane < 4 && (unsigned)page < (unsigned)p.n_pages)
                    ex = __ldg(eb + (long long)page * p.ep + (long long)(((key + 8 * (lane & 1)) & slot_mask) >> p.block_log2) * p.eb);
            }
            cp_async_commit();
        };

        int ex[C::NS], pg[2];
#pragma unroll
        for (int s = 0; s < C::NS - 1; ++s) {
            pages(s, pg);
            issue(s, s, pg, ex[s]);
        }
        pages(C::NS - 1, pg);

        // q: row g (and g + 8), channels t4 * CQ onwards, as fp16
        uint32_t qf[NT][D / 16][2];
        float rr[NT][2];                                   // what the scores of rows 2 t4, 2 t4 + 1 are multiplied by
        int pos[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = nt * 8 + g, fr = u.row0 + r, tok = pa_token(a, fr);
            const bool live = r < u.rows && (unsigned)(u.tok0 + tok) < (unsigned)a.n_rows;
            const uint4 *qp = reinterpret_cast<const uint4 *>(a.q + (long long)(u.tok0 + tok) * a.q_st + (long long)(w.h * a.group + fr - tok * a.group) * a.q_sh + t4 * CQ);
            uint32_t raw[D / 8];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const uint4 x = live ? __ldg(qp + i) : make_uint4(0, 0, 0, 0);
                raw[4 * i] = x.x; raw[4 * i + 1] = x.y; raw[4 * i + 2] = x.z; raw[4 * i + 3] = x.w;
#pragma unroll
                for (int j = 0; j < 4; ++j) top = max(top, max(raw[4 * i + j] << 16 & 0x7fff0000u, raw[4 * i + j] & 0x7fff0000u));
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int up = min(14 - ((int)(top >> 23) - 127), 126);       // times 2^up (an all-zero row: 2^126)
            const float f = exp2_whole(up), back = exp2_whole(-up) * a.scale_log2;
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t x = raw[2 * k + e];
                    qf[nt][k][e] = pack_f16x2(__uint_as_float(x << 16) * f, __uint_as_float(x & 0xffff0000u) * f);
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                rr[nt][e] = __shfl_sync(0xffffffffu, back, (2 * t4 + e) * 4);
                const int r2 = nt * 8 + 2 * t4 + e, tok2 = pa_token(a, u.row0 + r2);
                pos[nt][e] = r2 < u.rows && (unsigned)(u.tok0 + tok2) < (unsigned)a.n_rows ? u.base + tok2 : -1;
            }
        }
        float o[NT][D / 16][4];
        float m[NT][2], l[NT][2];                          // 2^6 below the maximum that counts, sum of this thread's weights
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[nt][e] = -INFINITY; l[nt][e] = 0.f; }
        }
        int full0, full1;                                  // tiles [full0, full1) need no mask
        pa_full_tiles<C::KT>(a, u, full0, full1);

        for (int s0 = 0; s0 < n; s0 += C::NS) {
#pragma unroll
            for (int js = 0; js < C::NS; ++js) {
                const int s = s0 + js;
                if (s >= n) break;
                cp_async_wait<C::NS - 2>();
                __syncwarp();                              // every lane's copies of this step have landed, and all are done with the one before
                issue(s + C::NS - 1, (js + C::NS - 1) % C::NS, pg, ex[(js + C::NS - 1) % C::NS]);
                pages(s + C::NS, pg);
                const uint32_t ks = ring_u + js * C::STAGE, vs = ks + C::HALF;
                const bool edge = w.t + s < full0 || w.t + s >= full1;
                const int j0 = pa_tile(u, w.t + s) * C::KT + warp * 16;
                const int ek0 = __shfl_sync(0xffffffffu, ex[js], 0), ek1 = __shfl_sync(0xffffffffu, ex[js], 1);
                const int ev0 = __shfl_sync(0xffffffffu, ex[js], 2), ev1 = __shfl_sync(0xffffffffu, ex[js], 3);

                // ---- scores: keys g and g + 8, rows 2 t4 and 2 t4 + 1 ----
                float x[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[nt][e] = 0.f;
#pragma unroll
                for (int i = 0; i < CQ / 16; ++i) {
                    const uint4 a0 = lds16(ks + piece_at<D>(g, t4 * (CQ / 16) + i)), a1 = lds16(ks + piece_at<D>(g + 8, t4 * (CQ / 16) + i));
                    const uint32_t w0[4] = {a0.x, a0.y, a0.z, a0.w}, w1[4] = {a1.x, a1.y, a1.z, a1.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t f[4];
                        codes_to_f16<FMT>(w0[j], f[0], f[2]);
                        codes_to_f16<FMT>(w1[j], f[1], f[3]);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma_f16_16816(x[nt], f, qf[nt][4 * i + j][0], qf[nt][4 * i + j][1]);
                    }
                }
                const float fk0 = exp2_whole(exp8_clamp(ek0, FMT)), fk1 = exp2_whole(exp8_clamp(ek1, FMT));
                bool grow = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[nt][e] = x[nt][e] * rr[nt][e & 1] * (e < 2 ? fk0 : fk1);
                        if (edge && !pa_sees(a, pos[nt][e & 1], j0 + g + (e < 2 ? 0 : 8))) x[nt][e] = -INFINITY;
                        grow |= x[nt][e] > m[nt][e & 1] + 14.f;
                    }
                if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float top = fmaxf(x[nt][e], x[nt][e + 2]);
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                            if (top > m[nt][e] + 14.f) {
                                const float f = pa_exp2(m[nt][e] - (top - 6.f));
                                m[nt][e] = top - 6.f;
                                l[nt][e] *= f;
#pragma unroll
                                for (int i = 0; i < D / 16; ++i) { o[nt][i][e] *= f; o[nt][i][e + 2] *= f; }
                            }
                        }
                }
                uint32_t pb[NT][2];                        // weights: row g, keys 2 t4, 2 t4 + 1 (and + 8)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float ref = m[nt][e & 1] == -INFINITY ? 0.f : m[nt][e & 1];     // a row that has seen nothing yet: all weights 0
                        y[e] = pa_exp2(x[nt][e] - ref);
                        l[nt][e & 1] += y[e];
                    }
                    pb[nt][0] = transpose_8x8(pack_f16x2(y[0], y[1]));
                    pb[nt][1] = transpose_8x8(pack_f16x2(y[2], y[3]));
                }

                // ---- outputs: channels g * CPT + 2 i, + 1 ----
                uint32_t v[4][CPT / 4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int r = 2 * t4 + (k & 1) + (k >> 1) * 8;
                    if (D == 128) {
                        const uint4 z = lds16(vs + piece_at<D>(r, g));
                        v[k][0] = z.x; v[k][1] = z.y; v[k][CPT / 4 - 2] = z.z; v[k][CPT / 4 - 1] = z.w;
                    } else {
                        const uint2 z = lds8(vs + piece_at<D>(r, g >> 1) + (g & 1) * 8);
                        v[k][0] = z.x; v[k][1] = z.y;
                    }
                    // rows that no query sees may hold anything: their values become zeros, or 0 * NaN would reach the output
                    const int j = j0 + r;
                    if (edge && !(j < u.hi_key && (j >= u.lo_key || j < a.n_sink))) {
#pragma unroll
                        for (int c = 0; c < CPT / 4; ++c) v[k][c] = 0;
                    }
                }
                const float fv0 = exp2_whole(exp8_clamp(ev0, FMT)), fv1 = exp2_whole(exp8_clamp(ev1, FMT));
                const bool same = ev0 == ev1;
#pragma unroll
                for (int i = 0; i < D / 16; i += 2) {
                    uint32_t f[2][4];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        // channels 4 c + {0, 1} and {2, 3}: (row 2 t4, row 2 t4 + 1) of each
                        codes_to_f16<FMT>(__byte_perm(v[2 * k][i / 2], v[2 * k + 1][i / 2], 0x5140), f[0][2 * k], f[0][2 * k + 1]);
                        codes_to_f16<FMT>(__byte_perm(v[2 * k][i / 2], v[2 * k + 1][i / 2], 0x7362), f[1][2 * k], f[1][2 * k + 1]);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float d[4] = {0.f, 0.f, 0.f, 0.f};
                            if (same) {
                                mma_f16_16816(d, f[k], pb[nt][0], pb[nt][1]);
                            } else {
                                float d1[4] = {0.f, 0.f, 0.f, 0.f};
                                mma_f16_1688(d, f[k][0], f[k][1], pb[nt][0]);
                                mma_f16_1688(d1, f[k][2], f[k][3], pb[nt][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[nt][i + k][e] = fmaf(d1[e], fv1, o[nt][i + k][e]);
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[nt][i + k][e] = fmaf(d[e], fv0, o[nt][i + k][e]);
                        }
                }
            }
        }
        cp_async_wait<0>();
        __syncwarp();

        // ---- the piece's result: the warps' parts meet in shared memory ----
        float *mine = reinterpret_cast<float *>(ring);     // [ROWS][D], 16-byte pieces XORed by the row
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[nt][e];
                sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                const int r = nt * 8 + 2 * t4 + e;
                if (g == 0) { stat_m[warp][r] = m[nt][e]; stat_l[warp][r] = sum; }
#pragma unroll
                for (int i = 0; i < D / 16; i += 2) {
                    const int c = (g * CPT + 2 * i) / 4;
                    *reinterpret_cast<float4 *>(mine + r * D + ((c ^ (r & 7)) << 2)) =
                        make_float4(o[nt][i][e], o[nt][i][e + 2], o[nt][i + 1][e], o[nt][i + 1][e + 2]);
                }
            }
        __syncthreads();
        const bool whole = w.whole();
        float *rec = a.part + (size_t)w.record(blockIdx.x) * C::REC;
        for (int i = tid; i < u.rows * (D / 4); i += 128) {
            const int r = i / (D / 4), c4 = i % (D / 4);
            float top = stat_m[0][r];
#pragma unroll
            for (int k = 1; k < 4; ++k) top = fmaxf(top, stat_m[k][r]);
            const float ref = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = pa_exp2(stat_m[k][r] - ref);
                sum = fmaf(f, stat_l[k][r], sum);
                const float4 z = *reinterpret_cast<const float4 *>(smem_raw + k * C::RING + (r * D + ((c4 ^ (r & 7)) << 2)) * 4);
                y.x = fmaf(f, z.x, y.x); y.y = fmaf(f, z.y, y.y); y.z = fmaf(f, z.z, y.z); y.w = fmaf(f, z.w, y.w);
            }
            if (whole) {
                const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);     // NaN stays NaN
                const int fr = u.row0 + r, rt = pa_token(a, fr), tok = u.tok0 + rt;
                if ((unsigned)tok < (unsigned)a.n_rows)
                    *reinterpret_cast<uint2 *>(a.out + (long long)tok * a.o_st + (long long)(w.h * a.group + fr - rt * a.group) * a.o_sh + c4 * 4) =
                        make_uint2(pack_bf16x2(y.x * inv, y.y * inv), pack_bf16x2(y.z * inv, y.w * inv));
            } else {
                *reinterpret_cast<float4 *>(rec + r * D + c4 * 4) = y;
                if (c4 == 0) { rec[C::ROWS * D + r] = top; rec[C::ROWS * D + C::ROWS + r] = sum; }
            }
        }
        if (!whole) {
            // the block that writes the last part of the pair joins all of them, in block order
            const int b0 = w.first_block(), b1 = w.last_block();
            __syncthreads();
            if (tid == 0) {
                const int last = pa_arrive(&a.counters[b0]) == b1 - b0;
                if (last) a.counters[b0] = 0;
                last_flag = last;
            }
            __syncthreads();
            if (last_flag) {
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
        if (more) __syncthreads();                         // the parts are read before the next piece's copies land there
    }
}

size_t paged8_attn_few_workspace(int d) { return (size_t)2 * 3 * device_sm_count() * 16 * (d + 2) * sizeof(float); }

template <int D, int NT, int FMT>
static cudaError_t launch_few8(const Few8Params &P, cudaStream_t st)
{
    using C = Few8Cfg<D, NT>;
    static bool attr[MAX_DEVICES] = {};
    cudaError_t e = opt_in_smem(k_paged8_attn_few<D, NT, FMT>, C::SMEM, attr);
    if (e != cudaSuccess) return e;
    k_paged8_attn_few<D, NT, FMT><<<3 * device_sm_count(), 128, C::SMEM, st>>>(P);
    e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

cudaError_t launch_paged8_attn_few(const PagedArgs &a, const Pool8 &pool, int max_new, cudaStream_t st)
{
    Few8Params P;
    P.a = a;
    P.p = pool;
    const bool one = (long long)max_new * a.group <= 8, e4m3 = pool.format == CACHE_E4M3;
    if (pool.d == 128) {
        if (one) return e4m3 ? launch_few8<128, 1, CACHE_E4M3>(P, st) : launch_few8<128, 1, CACHE_INT8>(P, st);
        return e4m3 ? launch_few8<128, 2, CACHE_E4M3>(P, st) : launch_few8<128, 2, CACHE_INT8>(P, st);
    }
    if (one) return e4m3 ? launch_few8<64, 1, CACHE_E4M3>(P, st) : launch_few8<64, 1, CACHE_INT8>(P, st);
    return e4m3 ? launch_few8<64, 2, CACHE_E4M3>(P, st) : launch_few8<64, 2, CACHE_INT8>(P, st);
}

}  // namespace cb
