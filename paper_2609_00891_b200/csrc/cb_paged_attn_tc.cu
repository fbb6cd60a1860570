// Attention of chunks of new rows over a paged cache on the tensor cores (tcgen05): the same sum as cb_paged_attn.cu for
// more than 16 flattened rows per request and KV head.
//
// A unit is two tiles of up to 128 flattened rows (whole tokens x the query heads of a KV head), which share every key tile
// of 128 keys.  Per thread block:
//   producer warp    TMA, one box per page and 64-channel half, ring of K and V tiles (a page id outside the pool reads as
//                    zeros).
//   clearing warp    rows of a V tile that no row of the unit sees may hold anything and 0 * NaN is NaN: a tile that has
//                    such rows lands on a barrier of its own, and this warp sets them to zero before it hands it on.
//   piece warp       describes the next piece to the softmax warps and copies its query tiles, one piece ahead.
//   MMA warp         S_i = Q_i K^T into tensor memory, then O_i += P_i V with P_i read from tensor memory, i = 0, 1 in
//                    turn: while the softmax warps work on one tile the tensor cores work on the other.
//   2 x 4 softmax warps   one thread per row: scores to registers, running maximum, exp2, weights as bf16 back over the
//                    scores in tensor memory.  The output is rescaled only when a maximum grows by more than 2^8 (weights
//                    stay below 2^8, sums and outputs are fp32), which after the first tiles is hardly ever.
// S_i of the next tile overwrites P_i, issued right after the P_i V that reads it and without a wait: this relies on the
// tensor pipe running one thread's products in the order of issue, which holds on this machine (every test, repeated runs
// bitwise) but which PTX promises only for products with one accumulator and shape.  A commit and a wait between the two
// would make it independent of that: measured, the long chunk below 1,726 -> 1,815 us.  A commit covers everything issued
// before it, so that the scores' completion also says that P_i V of the tile before is complete.
// Bound by the two tiles taking turns: ~3,100 cycles for 128 keys of both, of which the products run 2,048 and the
// special-function unit 2,048; on long runs by the board's power limit.  Measured, 64 query heads of 128 on 8 KV heads:
// 4,096 rows over 16,384 keys 1.7 - 1.75 ms = 1.1 PFLOP/s; a prompt of 8,192 rows (one request, nothing before it) 1.33 ms =
// 0.83 PFLOP/s: the line gives every block 450 tiles, but those at its begin are of one to five tiles a piece, and the first
// block walks 154 pieces where the others walk 14; a piece costs 7,600 cycles beside its tiles, the same number for every
// prompt measured.  16 requests of 2 to 16 rows over 8,192 keys 109 - 144 us (4.9 - 3.7 TB/s), by rows and page size.
#include "cb_paged.cuh"
#include "cb_ptx.cuh"
#include "cb_math.cuh"

namespace cb {

using namespace ptx;

template <int D>
struct TcAttnCfg {
    static constexpr int ROWS = 0, KT = 128;               // rows of a unit: 2 x as many whole tokens as 128 rows hold
    static constexpr int NB = D / 64;
    static constexpr int BLK = 128 * 128;                  // bytes of 128 rows of 64 channels
    static constexpr int TILE = NB * BLK;                  // a Q, K or V tile
    static constexpr int NS = D == 128 ? 5 : 10;           // K and V tiles in flight
    static constexpr int THREADS = 384;
    static constexpr int TMEM_COLS = 512;                  // S0, S1: 128 columns each, then O0, O1: D columns each
    // Quarters of a tile's weights that are handed on first, so that their product runs while the rest is computed.  Prefill of
    // 8,192 rows, three quarters against two: 64 channels 1,048 / 1,087 us, 128 channels 1,295 / 1,299 us alone and 1,700 /
    // 1,610 us for the chunk of 4,096 rows over 16,384 keys under the power limit.
    static constexpr int FIRST = D == 64 ? 3 : 2;
    static constexpr size_t SMEM = 1024 + 2 * (size_t)TILE + (size_t)NS * TILE + 1280;
    static constexpr int REC = 256 * (D + 2);              // floats of a partial record: [D / 4][256 rows][4], maxima, sums
};

struct TcAttnParams {
    CUtensorMap q, k, v;
    PagedArgs a;
    int q_bytes;                                            // of one 64-channel block of a Q tile
};

// What the softmax warps need of a piece; t0 < 0: no more pieces.
struct alignas(16) TcPiece {
    int t0, t1, full0, full1;      // key tiles of the piece; those in [full0, full1) need no mask
    int row0, rows, tok0, base;    // as in PaUnit
    int h, whole, rec, b0;         // KV head; not split; record of this block's part; first and last block of the pair
    int b1, rec0, ns, lo_tile;     // record of the first block's part
};

// Columns 0 .. n - 1 of 32 as a bit mask (n may be anything).
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

__device__ __forceinline__ int ld_acquire(const int *p)
{
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Largest of three (one instruction on sm_100).
__device__ __forceinline__ float max3(float x, float y, float z)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}

template <int D>
__global__ void __launch_bounds__(384, 1) k_paged_attn_tc(const __grid_constant__ TcAttnParams P)
{
    using C = TcAttnCfg<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *qs = smem;                                     // [2][TILE]
    uint8_t *kv = smem + 2 * (size_t)C::TILE;               // [NS][TILE]
    uint64_t *full = reinterpret_cast<uint64_t *>(kv + (size_t)C::NS * C::TILE);
    uint64_t *empty = full + C::NS;
    uint64_t *q_full = empty + C::NS;      // [2] Q tile written
    uint64_t *q_empty = q_full + 2;        // [2] its last scores of a piece complete
    uint64_t *info_full = q_empty + 2;     // [2] a piece's description written
    uint64_t *info_empty = info_full + 2;  // [2] read by the 8 softmax warps
    uint64_t *s_full = info_empty + 2;         // [2] scores complete
    uint64_t *p_ready = s_full + 2;        // [2][2] weights of the first keys and of the rest written (4 warps)
    uint64_t *o_full = p_ready + 4;        // [2] last product with V of a piece complete
    uint64_t *landed = o_full + 2;         // [NS] a V tile that has rows to clear: copied
    uint64_t *drain = landed + C::NS;
    PaSum *warp_sums = reinterpret_cast<PaSum *>(((uintptr_t)(drain + 1) + 15) & ~(uintptr_t)15);
    PaShare *share = reinterpret_cast<PaShare *>(warp_sums + 12);
    using Walk = PaWalk<C::ROWS, C::KT>;
    TcPiece *info = reinterpret_cast<TcPiece *>(((uintptr_t)(share + 1) + 15) & ~(uintptr_t)15);   // [2]
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(info + 2);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    // What is to land before the block may end after a time-out: stages that the producer filled; per stage (bits) whether its
    // last copy went to `landed`, and the parity of its next phase there; copies of each query tile.
    struct Flight { int issued; uint32_t on_landed, landings, n_query[2]; };
    Flight *flight = reinterpret_cast<Flight *>(tmem_slot + 3);
    volatile int *moves = &flight->issued;                  // counted up per stage, for the waits that outlast many tiles

    const PagedArgs &a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 256) {
        for (int i = 0; i < C::NS; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); mbar_init(&landed[i], 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
            mbar_init(&info_full[i], 1);
            mbar_init(&info_empty[i], 8);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_ready[2 * i], 4);
            mbar_init(&p_ready[2 * i + 1], 4);
            mbar_init(&o_full[i], 1);
        }
        mbar_init(drain, 1);
        abort_flag[0] = 0;
        abort_flag[1] = (int)a.poll_limit;
        *flight = Flight{};
        mbar_fence_init();
        tma_prefetch_desc(&P.q);
        tma_prefetch_desc(&P.k);
        tma_prefetch_desc(&P.v);
    }
    if (warp == 9) tmem_alloc(tmem_slot, C::TMEM_COLS);
    tc_fence_before();
    pa_schedule<C::ROWS, C::KT, C::THREADS>(a, reinterpret_cast<int *>(smem), (2 + C::NS) * C::TILE / 4, share, warp_sums);
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    const bool any = share->begin < share->end;
    const int RT = a.unit_rows >> 1;                        // rows of a tile, at most 128
    const int box_log2 = a.page_log2 < 7 ? a.page_log2 : 7;
    bool dead = false;       // a wait ran out: no more waits, the rest runs through on whatever is there

    // the softmax warps hold a row of 128 scores each: 208 + 208 + 88 registers a thread of the 3 x 168 launched with
    if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    Walk w;
    if (any) w.open(a, *share);
    if (warp == 8) {
        // ================================ producer ================================
        if (any && !a.starve) {
            Ring<C::NS> st;
            int issued = 0;
            uint32_t on_landed = 0, landings = 0;
            const int n_page = 1 << (7 - box_log2);
            const int cb = lane / n_page, i = lane - cb * n_page;        // 64-channel block and box of this lane
            bool more = true;
            while (more) {
                const int *row = a.table + (long long)w.u.b * a.table_stride;
                for (int t = w.t; t < w.t1 && !dead; ++t) {
                    const int j0 = pa_tile(w.u, t) * C::KT;
                    const int key = j0 + (i << box_log2);
                    int page = a.n_pages;                                // outside the pool: the copy writes zeros
                    if (cb < C::NB && pa_wanted(a, w.u, key, 1 << box_log2)) {
                        const int col = key >> a.page_log2;
                        if (col < a.table_cols) page = __ldg(row + col);
                    }
                    const int slot = key & ((1 << a.page_log2) - 1);
                    const bool clear = pa_clears<C::KT>(a, w.u, j0);
                    for (int comp = 0; comp < 2; ++comp) {
                        if (!mbar_wait_to_issue_warp(&empty[st.idx], st.phase ^ 1, abort_flag)) { dead = true; break; }
                        const bool cleared = comp && clear;
                        uint64_t *bar = cleared ? &landed[st.idx] : &full[st.idx];
                        on_landed = (on_landed & ~(1u << st.idx)) | ((uint32_t)cleared << st.idx);
                        landings ^= (uint32_t)cleared << st.idx;
                        uint8_t *dst = kv + (size_t)st.idx * C::TILE;
                        if (lane == 0) mbar_arrive_expect_tx(bar, C::TILE);
                        __syncwarp();
                        if (cb < C::NB)
                            tma_load_5d(dst + cb * C::BLK + ((size_t)i << (box_log2 + 7)), comp ? &P.v : &P.k, bar, 0, slot, cb, w.h, page);
                        st.next();
                        ++issued;
                        if (lane == 0) *moves = issued;
                    }
                }
                more = !dead && w.next(a);
            }
            if (lane == 0) { flight->on_landed = on_landed; flight->landings = landings; }
        }
    } else if (warp == 10) {
        // ================================ clears rows of V tiles ================================
        if (any) {
            uint32_t stage = 0, uses = 0;                  // position in the ring; bit s: parity of stage s's next landing
            bool more = true;
            while (more) {
                for (int t = w.t; t < w.t1 && !dead; ++t) {
                    const int j0 = pa_tile(w.u, t) * C::KT;
                    stage = (stage + 1) % C::NS;           // past the K tile
                    if (pa_clears<C::KT>(a, w.u, j0)) {
                        if (!mbar_wait_while_moving_warp(&landed[stage], (uses >> stage) & 1, abort_flag, moves)) { dead = true; break; }
                        uses ^= 1u << stage;
                        uint8_t *dst = kv + (size_t)stage * C::TILE;
                        // keys outside [lo_key, hi_key) and behind the sinks: nobody sees them
                        const int c0 = max(0, w.u.hi_key - j0);                                  // rows [c0, 128)
                        const int g0 = max(0, a.n_sink - j0), g1 = min(C::KT, w.u.lo_key - j0);  // rows [g0, g1)
                        const int r0 = g0 < g1 ? min(c0, g0) : c0;
                        for (int r = r0 * 8 + lane; r < C::KT * 8; r += 32) {
                            const int key_row = r >> 3;
                            if (key_row >= c0 || (key_row >= g0 && key_row < g1)) {
#pragma unroll
                                for (int cb = 0; cb < C::NB; ++cb) *reinterpret_cast<uint4 *>(dst + cb * C::BLK + r * 16) = make_uint4(0, 0, 0, 0);
                            }
                        }
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&full[stage]);
                    }
                    stage = (stage + 1) % C::NS;
                }
                more = !dead && w.next(a);
            }
        }
    } else if (warp == 11) {
        // ================================ pieces and their Q tiles ================================
        // Runs ahead of the softmax warps: the next piece's rows are loaded while the last tile of this one is worked on.
        if (any) {
            uint32_t n = 0, n_query[2] = {0, 0};
            bool more = true;
            while (more && !dead) {
                if (!mbar_wait_while_moving_warp(&info_empty[n & 1], ((n >> 1) & 1) ^ 1, abort_flag, moves)) { dead = true; break; }
                if (lane == 0) {
                    TcPiece &p = info[n & 1];
                    p.t0 = w.t; p.t1 = w.t1;
                    pa_full_tiles<C::KT>(a, w.u, p.full0, p.full1);
                    p.row0 = w.u.row0; p.rows = w.u.rows; p.tok0 = w.u.tok0; p.base = w.u.base;
                    p.h = w.h; p.whole = w.whole() ? 1 : 0; p.rec = w.record(blockIdx.x);
                    p.b0 = w.first_block(); p.b1 = w.last_block(); p.rec0 = w.record(p.b0);
                    p.ns = w.u.ns; p.lo_tile = w.u.lo_tile;
                    mbar_arrive(&info_full[n & 1]);
                }
                __syncwarp();
                ++n;
                const int tiles = w.u.rows > RT ? 2 : 1;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (i >= tiles) break;
                    if (!mbar_wait_while_moving_warp(&q_empty[i], (n_query[i] & 1) ^ 1, abort_flag, moves)) { dead = true; break; }
                    ++n_query[i];
                    // rows behind the request's are another one's, or zeros, or an earlier tile's: nobody reads their results
                    if (lane == 0) {
                        mbar_arrive_expect_tx(&q_full[i], C::NB * P.q_bytes);
                        for (int cb = 0; cb < C::NB; ++cb)
                            tma_load_4d(qs + i * C::TILE + cb * C::BLK, &P.q, &q_full[i], 0, w.h * a.group,
                                        w.u.tok0 + (w.u.qt * 2 + i) * (a.unit_tokens >> 1), cb);
                    }
                    __syncwarp();
                }
                more = w.next(a);
            }
            if (lane == 0) { flight->n_query[0] = n_query[0]; flight->n_query[1] = n_query[1]; }
            if (!dead && mbar_wait_while_moving_warp(&info_empty[n & 1], ((n >> 1) & 1) ^ 1, abort_flag, moves) && lane == 0) {
                info[n & 1].t0 = -1;
                mbar_arrive(&info_full[n & 1]);
            }
        }
    } else if (warp == 9) {
        // ================================ MMA issuer ================================
        // The whole warp walks and one elected lane issues (see elect_one).
        if (any) {
            constexpr uint32_t idesc_s = umma_idesc_bf16(128, C::KT, false, false);   // both K-major
            constexpr uint32_t idesc_o = umma_idesc_bf16(128, D, false, true);        // V: MN-major
            const uint64_t proto_k = umma_smem_desc_sw128(0, 16, 1024);
            const uint64_t proto_v = umma_smem_desc_sw128(0, C::BLK, 1024);
            const uint32_t q_addr = (smem_u32(qs) & 0x3FFFFu) >> 4, kv_addr = (smem_u32(kv) & 0x3FFFFu) >> 4;
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
            const bool leader = elect_one();
            Ring<C::NS> st;
            uint32_t nq[2] = {0, 0}, np[2] = {0, 0};
            bool more = true;
            auto scores = [&](int i, uint32_t stage, bool last) {
                const uint64_t qd = proto_k | (uint64_t)(q_addr + i * (C::TILE >> 4));
                const uint64_t kd = proto_k | (uint64_t)(kv_addr + __shfl_sync(0xffffffffu, stage, 0) * (C::TILE >> 4));
                if (leader) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = (k >> 2) * (C::BLK >> 4) + (k & 3) * 2;
                        umma_bf16_ss(tm + i * 128, qd + off, kd + off, idesc_s, k == 0 ? 0u : 1u);
                    }
                    umma_commit(&s_full[i]);
                    if (last) umma_commit(&q_empty[i]);    // the piece's last scores of this tile
                }
                __syncwarp();
            };
            // the part of the tile's keys that is handed on first, or the rest; `first`: nothing is in the output yet
            auto values = [&](int i, uint32_t stage, int half, uint32_t first) {
                const uint64_t vd = proto_v | (uint64_t)(kv_addr + __shfl_sync(0xffffffffu, stage, 0) * (C::TILE >> 4));
                if (leader) {
#pragma unroll
                    for (int k = half ? 2 * C::FIRST : 0; k < (half ? 8 : 2 * C::FIRST); ++k)
                        umma_bf16_ts(tm + 256 + i * D, tm + i * 128 + k * 8, vd + k * 128, idesc_o, k == 0 ? 1u - first : 1u);
                }
                __syncwarp();
            };
            auto commit = [&](uint64_t *bar) {
                if (leader) umma_commit(bar);
                __syncwarp();
            };
            while (more && !dead) {
                const int tiles = w.u.rows > RT ? 2 : 1;
                // K of the piece's first tile
                uint32_t ks = st.idx;
                if (!mbar_wait_suspended_warp(&full[st.idx], st.phase, abort_flag)) { dead = true; break; }
                st.next();
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (i >= tiles || dead) break;
                    if (!mbar_wait_suspended_warp(&q_full[i], nq[i]++ & 1, abort_flag)) { dead = true; break; }
                    tc_fence_after();
                    scores(i, ks, w.t + 1 == w.t1);
                }
                if (dead) break;
                commit(&empty[ks]);
                for (int t = w.t; t < w.t1 && !dead; ++t) {
                    const bool last = t + 1 == w.t1;
                    const uint32_t vs = st.idx;
                    if (!mbar_wait_suspended_warp(&full[st.idx], st.phase, abort_flag)) { dead = true; break; }
                    st.next();
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (i >= tiles || dead) break;
                        if (!mbar_wait_suspended_warp(&p_ready[2 * i], np[i] & 1, abort_flag)) { dead = true; break; }
                        tc_fence_after();
                        values(i, vs, 0, t == w.t ? 1u : 0u);
                        if (!mbar_wait_suspended_warp(&p_ready[2 * i + 1], np[i]++ & 1, abort_flag)) { dead = true; break; }
                        tc_fence_after();
                        values(i, vs, 1, 0);
                        if (last) commit(&o_full[i]);
                        if (i == tiles - 1) commit(&empty[vs]);
                        if (!last) {
                            if (i == 0) {
                                ks = st.idx;
                                if (!mbar_wait_suspended_warp(&full[st.idx], st.phase, abort_flag)) { dead = true; break; }
                                st.next();
                            }
                            scores(i, ks, t + 2 == w.t1);
                            if (i == tiles - 1) commit(&empty[ks]);
                        }
                    }
                }
                more = !dead && w.next(a);
            }
            commit(drain);                                 // every product has ended before tensor memory is freed
            mbar_drain(drain, 0);
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // ================================ softmax warps: one thread per row ================================
        const int i = warp >> 2;                           // tile
        const int r = tid & 127;                           // row in the tile
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_tm = tmem + i * 128 + lanes, o_tm = tmem + 256 + i * D + lanes;
        const float c = a.scale_log2;
        const uint64_t cc = f2_pack(c, c);
        uint32_t ns = 0, no = 0;
        if (a.give_up && any && i == 0) {                  // test hook: as if a wait had run out
            abort_flag[0] = 1;
            dead = true;
        }
        auto settle = [&](int tile, uint32_t from) {
            Walk w;
            bool more = w.open(a, *share);
            for (uint32_t k = 0; more; ++k, more = w.next(a))
                if (k >= from && !w.whole() && tile * RT < w.u.rows) {
                    int *counter = &a.counters[(2 * w.first_block() + tile) * 4 + (warp & 3)];
                    if (pa_arrive(counter) == w.last_block() - w.first_block()) *counter = 0;
                }
        };
        for (uint32_t n = 0; any; ++n) {
            if (!mbar_wait_while_moving_warp(&info_full[n & 1], (n >> 1) & 1, abort_flag, moves)) {
                // time-out: the parts that this block will not write still count, or the next call would wait for them
                if (lane == 0) settle(i, n);
                break;
            }
            const TcPiece p = info[n & 1];
            __syncwarp();
            if (lane == 0) mbar_arrive(&info_empty[n & 1]);
            if (p.t0 < 0) break;
            const int rr = i * 128 + r;                    // place in a partial record
            if (i * RT < p.rows) {
                const int fr = p.row0 + i * RT + r, rt = pa_token(a, fr), tok = p.tok0 + rt, head = p.h * a.group + fr - rt * a.group;
                const bool live = r < RT && i * RT + r < p.rows && (unsigned)tok < (unsigned)a.n_rows;
                const int pos = live ? p.base + rt : -1;
                float m = -INFINITY, l = 0.f;              // reference maximum (raw score), sum of weights
                for (int t = p.t0; t < p.t1; ++t) {
                    if (!dead && !mbar_wait_suspended_warp(&s_full[i], ns & 1, abort_flag)) dead = true;
                    ++ns;
                    tc_fence_after();
                    uint32_t s[4][32];
#pragma unroll
                    for (int x = 0; x < 4; ++x) tmem_ld_32x32(s_tm + x * 32, s[x]);
                    tmem_wait_ld();
                    if (t < p.full0 || t >= p.full1) {
                        const int j0 = (t < p.ns ? t : p.lo_tile + (t - p.ns)) * C::KT;
                        const int hi = min(pos - j0, C::KT - 1);                               // last column seen
                        const int lo = a.window > 0 ? (int)max((long long)pos - a.window + 1 - j0, -1ll) : -1;   // first one, without
                        const int sink = a.window > 0 ? a.n_sink - j0 : 0;                     // the sinks
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            // bit y: column 32 x + y is seen
                            uint32_t see = below(hi + 1 - x * 32) & ~(below(lo - x * 32) & ~below(sink - x * 32));
#pragma unroll
                            for (int y = 0; y < 32; ++y)
                                if (!(see & (1u << y))) s[x][y] = 0xff800000u;
                        }
                    }
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int y = 0; y < 32; y += 2)
#pragma unroll
                        for (int x = 0; x < 4; ++x) mx[x] = max3(mx[x], __uint_as_float(s[x][y]), __uint_as_float(s[x][y + 1]));
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    float f = 1.f;
                    if (live && (top - m) * c > 8.f) {     // also the first maximum of a row: m is -inf
                        f = pa_exp2((m - top) * c);
                        m = top;
                        l *= f;
                    }
                    if (t > p.t0 && __any_sync(0xffffffffu, f != 1.f)) {
#pragma unroll 1
                        for (int x = 0; x < D / 16; ++x) {
                            uint32_t o[16];
                            tmem_ld_32x16(o_tm + x * 16, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * f);
                            tmem_st_32x16(o_tm + x * 16, o);
                        }
                    }
                    const float mc = m == -INFINITY ? 0.f : -m * c;
                    const uint64_t mm = f2_pack(mc, mc);
                    uint64_t sum[2] = {0, 0};
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
#pragma unroll
                        for (int x = half ? C::FIRST : 0; x < (half ? 4 : C::FIRST); ++x) {
                            uint32_t p[16];
#pragma unroll
                            for (int y = 0; y < 16; ++y) {
                                const uint64_t e = f2_fma(f2_pack(__uint_as_float(s[x][2 * y]), __uint_as_float(s[x][2 * y + 1])), cc, mm);
                                float p0, p1;
                                f2_unpack(e, p0, p1);
                                p0 = pa_exp2(p0);
                                p1 = pa_exp2(p1);
                                sum[y & 1] = f2_add(sum[y & 1], f2_pack(p0, p1));
                                p[y] = pack_bf16x2(p0, p1);
                            }
                            tmem_st_32x16(s_tm + x * 16, p);
                        }
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&p_ready[2 * i + half]);
                    }
                    float s0, s1;
                    f2_unpack(f2_add(sum[0], sum[1]), s0, s1);
                    l += s0 + s1;
                }

                // ---- the piece's result ----
                if (!dead && !mbar_wait_suspended_warp(&o_full[i], no & 1, abort_flag)) dead = true;
                ++no;
                tc_fence_after();
                __nv_bfloat16 *orow = a.out + (long long)tok * a.o_st + (long long)head * a.o_sh;
                if (p.whole) {
                    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
#pragma unroll 1
                    for (int x = 0; x < D / 32; ++x) {
                        uint32_t o[32];
                        tmem_ld_32x32(o_tm + x * 32, o);
                        tmem_wait_ld();
                        if (live) {
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                uint4 v;
                                v.x = pack_bf16x2(__uint_as_float(o[y * 8 + 0]) * inv, __uint_as_float(o[y * 8 + 1]) * inv);
                                v.y = pack_bf16x2(__uint_as_float(o[y * 8 + 2]) * inv, __uint_as_float(o[y * 8 + 3]) * inv);
                                v.z = pack_bf16x2(__uint_as_float(o[y * 8 + 4]) * inv, __uint_as_float(o[y * 8 + 5]) * inv);
                                v.w = pack_bf16x2(__uint_as_float(o[y * 8 + 6]) * inv, __uint_as_float(o[y * 8 + 7]) * inv);
                                *reinterpret_cast<uint4 *>(orow + x * 32 + y * 8) = v;
                            }
                        }
                    }
                    tc_fence_before();
                } else {
                    // Rows of a warp are joined by the warp that has their last part, of any block, in block order: no warp waits
                    // for another.  A block's first piece ends a pair that the block before it finishes last, so that the
                    // other parts are mostly there already: then this part stays in tensor memory and is joined from there.
                    int *counter = &a.counters[(2 * p.b0 + i) * 4 + (warp & 3)];
                    int there_are = 0;
                    if (lane == 0) there_are = ld_acquire(counter);
                    bool join = __shfl_sync(0xffffffffu, there_are, 0) == p.b1 - p.b0;
                    const bool fresh = join;               // this block's part is not in memory
                    if (!fresh) {
                        float *rec = a.part + (size_t)p.rec * C::REC;
#pragma unroll 1
                        for (int x = 0; x < D / 32; ++x) {
                            uint32_t o[32];
                            tmem_ld_32x32(o_tm + x * 32, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int y = 0; y < 8; ++y)
                                *reinterpret_cast<float4 *>(rec + ((size_t)(x * 8 + y) * 256 + rr) * 4) =
                                    make_float4(__uint_as_float(o[y * 4]), __uint_as_float(o[y * 4 + 1]), __uint_as_float(o[y * 4 + 2]), __uint_as_float(o[y * 4 + 3]));
                        }
                        rec[256 * D + rr] = m * c;         // c > 0: -inf stays -inf
                        rec[256 * D + 256 + rr] = l;
                        __syncwarp();
                        if (lane == 0) there_are = pa_arrive(counter);
                        join = __shfl_sync(0xffffffffu, there_are, 0) == p.b1 - p.b0;
                    }
                    if (join) {
                        __syncwarp();                      // what lane 0 acquired is every lane's
                        if (lane == 0) *counter = 0;
                        const int me = (int)blockIdx.x;
                        const float *mine = a.part + 256 * D + rr;
                        auto at = [&](int b) { return (size_t)(b == p.b0 ? p.rec0 : 2 * b) * C::REC; };
                        float mm = -INFINITY, ll = 0.f;
                        for (int b = p.b0; b <= p.b1; b += 4) {           // four parts' loads in flight together
                            float pm[4], pl[4], mn = mm;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const bool own = fresh && b + k == me;
                                pm[k] = own ? m * c : b + k <= p.b1 ? __ldcg(mine + at(b + k)) : -INFINITY;
                                pl[k] = own ? l : b + k <= p.b1 ? __ldcg(mine + at(b + k) + 256) : 0.f;
                            }
#pragma unroll
                            for (int k = 0; k < 4; ++k) mn = fmaxf(mn, pm[k]);
                            const float ref = mn == -INFINITY ? 0.f : mn;
                            ll *= pa_exp2(mm - ref);
#pragma unroll
                            for (int k = 0; k < 4; ++k) ll = fmaf(pa_exp2(pm[k] - ref), pl[k], ll);
                            mm = mn;
                        }
                        const float ref = mm == -INFINITY ? 0.f : mm;
                        const float inv = ll > 0.f ? 1.f / ll : (ll == 0.f ? 0.f : ll);
#pragma unroll 1
                        for (int x = 0; x < D / 32; ++x) {
                            float acc[32];
                            uint32_t o[32];
                            tmem_ld_32x32(o_tm + x * 32, o);
#pragma unroll
                            for (int y = 0; y < 32; ++y) acc[y] = 0.f;
                            tmem_wait_ld();
                            for (int b = p.b0; b <= p.b1; b += 2) {       // two parts in flight
                                float4 v[2][8];
                                float f[2];
#pragma unroll
                                for (int k = 0; k < 2; ++k) {
                                    const bool own = fresh && b + k == me, there = !own && b + k <= p.b1;
                                    f[k] = own ? m * c : there ? __ldcg(mine + at(b + k)) : -INFINITY;
#pragma unroll
                                    for (int y = 0; y < 8; ++y)
                                        v[k][y] = there ? __ldcg(reinterpret_cast<const float4 *>(a.part + at(b + k) + ((size_t)(x * 8 + y) * 256 + rr) * 4))
                                                : own ? make_float4(__uint_as_float(o[y * 4]), __uint_as_float(o[y * 4 + 1]), __uint_as_float(o[y * 4 + 2]), __uint_as_float(o[y * 4 + 3]))
                                                      : make_float4(0.f, 0.f, 0.f, 0.f);
                                }
#pragma unroll
                                for (int k = 0; k < 2; ++k) {
                                    const float g = pa_exp2(f[k] - ref) * inv;
#pragma unroll
                                    for (int y = 0; y < 8; ++y) {
                                        acc[y * 4] = fmaf(g, v[k][y].x, acc[y * 4]);
                                        acc[y * 4 + 1] = fmaf(g, v[k][y].y, acc[y * 4 + 1]);
                                        acc[y * 4 + 2] = fmaf(g, v[k][y].z, acc[y * 4 + 2]);
                                        acc[y * 4 + 3] = fmaf(g, v[k][y].w, acc[y * 4 + 3]);
                                    }
                                }
                            }
                            if (live) {
#pragma unroll
                                for (int y = 0; y < 4; ++y)
                                    *reinterpret_cast<uint4 *>(orow + x * 32 + y * 8) =
                                        make_uint4(pack_bf16x2(acc[y * 8], acc[y * 8 + 1]), pack_bf16x2(acc[y * 8 + 2], acc[y * 8 + 3]),
                                                   pack_bf16x2(acc[y * 8 + 4], acc[y * 8 + 5]), pack_bf16x2(acc[y * 8 + 6], acc[y * 8 + 7]));
                            }
                        }
                    }
                    tc_fence_before();
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (abort_flag[0]) {                                   // the same in every thread: nobody writes it after the barrier
        if (tid == 0) atomicExch(a.status, DEV_TIMEOUT);
        // copies in flight land before the block ends
        if (warp == 9) {
            const Flight f = *flight;
            for (int k = 0; k < min(f.issued, C::NS); ++k) {
                if (f.on_landed >> k & 1) mbar_drain(&landed[k], (f.landings >> k & 1) ^ 1);
                else mbar_drain(&full[k], ((f.issued - k - 1) / C::NS) & 1);
            }
            for (int i = 0; i < 2; ++i)
                if (f.n_query[i]) mbar_drain(&q_full[i], (f.n_query[i] - 1) & 1);
        }
        __syncwarp();
    }
    if (warp == 9) tmem_dealloc(tmem, C::TMEM_COLS);
}

size_t paged_attn_tc_workspace(int d) { return (size_t)2 * device_sm_count() * 256 * (d + 2) * sizeof(float); }

template <int D>
static cudaError_t launch_tc_attn(const TcAttnParams &P, cudaStream_t st)
{
    using C = TcAttnCfg<D>;
    static bool attr[MAX_DEVICES] = {};
    cudaError_t e = opt_in_smem(k_paged_attn_tc<D>, C::SMEM, attr);
    if (e != cudaSuccess) return e;
    k_paged_attn_tc<D><<<device_sm_count(), C::THREADS, C::SMEM, st>>>(P);
    e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

cudaError_t launch_paged_attn_tc(const PagedArgs &a, int d, const void *k, const void *v, int page_size, long long s_page,
                                 long long s_slot, long long s_head, cudaStream_t st)
{
    TcAttnParams P;
    P.a = a;
    const int box = page_size < 128 ? page_size : 128;
    const int q_tokens = a.n_rows < a.unit_tokens / 2 ? a.n_rows : a.unit_tokens / 2;
    P.q_bytes = q_tokens * a.group * 128;
    if (!make_q_tensor_map(&P.q, a.q, d, a.Hkv * a.group, a.n_rows, a.q_sh, a.q_st, a.group, q_tokens) ||
        !make_kv_tensor_map(&P.k, k, d, a.Hkv, page_size, a.n_pages, s_head, s_slot, s_page, box, 1) ||
        !make_kv_tensor_map(&P.v, v, d, a.Hkv, page_size, a.n_pages, s_head, s_slot, s_page, box, 1))
        return cudaErrorInvalidValue;
    return d == 128 ? launch_tc_attn<128>(P, st) : launch_tc_attn<64>(P, st);
}

}  // namespace cb
