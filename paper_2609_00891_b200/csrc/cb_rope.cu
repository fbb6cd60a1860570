// Stand-alone rotary embedding of a strided bf16 key tensor, in place (Section 2.2, Section 3.1): removes (inverse) or
// restores the position-dependent rotation outside the fused paths.  Pure streaming: one read and one write of K.
#include "cb_internal.cuh"
#include "cb_math.cuh"
#include "cb_paged.cuh"
#include "cb_rope.cuh"

namespace cb {

struct RopeArgs {
    __nv_bfloat16 *k;
    long long sl, st, sh;
    int L, H, T, d;
    const int *pos;
    int inverse;
    uint32_t f[ROPE_MAX_FREQ];
};

// grid (token blocks, L * H); 256 threads = (d / 16 chunk pairs) x rows
__global__ void __launch_bounds__(256) k_rope_rotate(const RopeArgs a)
{
    const int HC = a.d / 16;                      // 16-byte chunk pairs per row
    const int rows = 256 / HC;
    const int lc = threadIdx.x % HC, r = threadIdx.x / HC;
    const int t = blockIdx.x * rows + r;
    if (t >= a.T) return;
    const int l = blockIdx.y / a.H, h = blockIdx.y % a.H;
    __nv_bfloat16 *row = a.k + (long long)l * a.sl + (long long)t * a.st + (long long)h * a.sh;
    uint4 *plo = reinterpret_cast<uint4 *>(row + lc * 8);
    uint4 *phi = reinterpret_cast<uint4 *>(row + a.d / 2 + lc * 8);
    const uint4 vlo = *plo, vhi = *phi;
    const unsigned ulo[4] = {vlo.x, vlo.y, vlo.z, vlo.w}, uhi[4] = {vhi.x, vhi.y, vhi.z, vhi.w};
    unsigned olo[4], ohi[4];
    const int pos = a.pos[t];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float lo[2] = {__uint_as_float(ulo[e] << 16), __uint_as_float(ulo[e] & 0xffff0000u)};
        float hi[2] = {__uint_as_float(uhi[e] << 16), __uint_as_float(uhi[e] & 0xffff0000u)};
        float nl[2], nh[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            float c, s;
            rope_cs_poly(a.f[lc * 8 + 2 * e + q], pos, c, s);
            if (a.inverse) s = -s;
            nl[q] = lo[q] * c - hi[q] * s;
            nh[q] = lo[q] * s + hi[q] * c;
        }
        __nv_bfloat162 bl = __floats2bfloat162_rn(nl[0], nl[1]), bh = __floats2bfloat162_rn(nh[0], nh[1]);
        olo[e] = *reinterpret_cast<unsigned *>(&bl);
        ohi[e] = *reinterpret_cast<unsigned *>(&bh);
    }
    *plo = make_uint4(olo[0], olo[1], olo[2], olo[3]);
    *phi = make_uint4(ohi[0], ohi[1], ohi[2], ohi[3]);
}

cudaError_t launch_rope_rotate(void *k, int L, int H, int d, long long T, long long sl, long long st, long long sh,
                               const int *pos, double base, int inverse, cudaStream_t stream)
{
    RopeArgs a;
    a.k = static_cast<__nv_bfloat16 *>(k);
    a.sl = sl; a.st = st; a.sh = sh; a.L = L; a.H = H; a.T = (int)T; a.d = d; a.pos = pos; a.inverse = inverse;
    rope_frequencies(base, d, a.f);
    const int rows = 256 / (d / 16);
    dim3 grid((unsigned)((T + rows - 1) / rows), (unsigned)(L * H));
    k_rope_rotate<<<grid, 256, 0, stream>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

// Rotary embedding with several position axes (time, height, width, ...), out of place or in place.  Every pair of
// channels turns by the position of its own axis.  The cosines and sines of a row serve all its layers and heads: a block
// takes the few rows whose pairs make 256, computes one pair a thread into shared memory and then streams those rows'
// layers and heads, four pieces of 2 x 16 bytes a thread in flight and four blocks an SM.  Bound by HBM: 8,190 rows of 64
// heads of 128 channels in 47 us (5.7 TB/s); 51 us when every thread held the angles of eight pairs in registers and
// streamed eight heads, 53 us with eight pieces in flight and fewer blocks.
// Angles are turns in 0.64 fixed point: pos * f modulo 2^64 is exact for every 32-bit position, so the angle is off by
// at most pos * 2^-56 turns (the frequency's own rounding) plus just under 2^-23 turns (the sine's argument is cut to 23
// bits, always downwards).
struct RopeAxesArgs {
    const __nv_bfloat16 *x;
    __nv_bfloat16 *out;
    long long x_sl, x_st, x_sh, o_sl, o_st, o_sh;
    int H, LH, per;               // per: (layer, head) pairs of a block
    long long T;
    const int *pos;
    long long axis_stride;
    int inverse;
    unsigned char axis[ROPE_MAX_FREQ];
    unsigned long long f[ROPE_MAX_FREQ];
};

// grid (blocks of 512 / D rows, groups of (layer, head) pairs), 256 threads
template <int D>
__global__ void __launch_bounds__(256, 4) k_rope_axes(const __grid_constant__ RopeAxesArgs a)
{
    constexpr int HC = D / 16;                        // pieces of a row: eight pairs each
    constexpr int TB = 512 / D;                       // rows of a block
    constexpr int BATCH = 4;
    // [row][quarter of a piece][piece]: cos, sin of two pairs; lanes of neighbouring pieces read neighbouring words
    __shared__ float4 cs[TB][4][HC];
    const long long t0 = (long long)blockIdx.x * TB;
    {
        const int i = threadIdx.x % (D / 2), r = threadIdx.x / (D / 2);
        float c = 1.f, s = 0.f;
        if (t0 + r < a.T) {
            const long long p = a.pos[(long long)a.axis[i] * a.axis_stride + t0 + r];
            rope_cs_turns((uint32_t)(((unsigned long long)p * a.f[i]) >> 32), c, s);
            if (a.inverse) s = -s;
        }
        reinterpret_cast<float2 *>(&cs[r][(i & 7) >> 1][i >> 3])[i & 1] = make_float2(c, s);
    }
    __syncthreads();
    const int rows = (int)min((long long)TB, a.T - t0), lh0 = blockIdx.y * a.per, n_lh = min(a.per, a.LH - lh0);
    const int items = rows * n_lh * HC;               // (row, (layer, head), piece)
    const int lc = threadIdx.x % HC;
    for (int first = threadIdx.x; first < items; first += 256 * BATCH) {
        uint4 vlo[BATCH], vhi[BATCH];
        // all are loaded before the first is stored: x and out may be the same
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int it = first + k * 256;
            if (it >= items) break;
            const int rest = it / HC, r = rest / n_lh, lh = lh0 + rest - r * n_lh, l = lh / a.H, h = lh - l * a.H;
            const __nv_bfloat16 *row = a.x + l * a.x_sl + (t0 + r) * a.x_st + h * a.x_sh + lc * 8;
            vlo[k] = *reinterpret_cast<const uint4 *>(row);
            vhi[k] = *reinterpret_cast<const uint4 *>(row + D / 2);
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int it = first + k * 256;
            if (it >= items) break;
            const int rest = it / HC, r = rest / n_lh, lh = lh0 + rest - r * n_lh, l = lh / a.H, h = lh - l * a.H;
            __nv_bfloat16 *to = a.out + l * a.o_sl + (t0 + r) * a.o_st + h * a.o_sh + lc * 8;
            const unsigned ulo[4] = {vlo[k].x, vlo[k].y, vlo[k].z, vlo[k].w}, uhi[4] = {vhi[k].x, vhi[k].y, vhi[k].z, vhi[k].w};
            unsigned olo[4], ohi[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 w = cs[r][e][lc];
                const float l0 = __uint_as_float(ulo[e] << 16), l1 = __uint_as_float(ulo[e] & 0xffff0000u);
                const float h0 = __uint_as_float(uhi[e] << 16), h1 = __uint_as_float(uhi[e] & 0xffff0000u);
                olo[e] = pack_bf16x2(l0 * w.x - h0 * w.y, l1 * w.z - h1 * w.w);
                ohi[e] = pack_bf16x2(l0 * w.y + h0 * w.x, l1 * w.w + h1 * w.z);
            }
            *reinterpret_cast<uint4 *>(to) = make_uint4(olo[0], olo[1], olo[2], olo[3]);
            *reinterpret_cast<uint4 *>(to + D / 2) = make_uint4(ohi[0], ohi[1], ohi[2], ohi[3]);
        }
    }
}

cudaError_t launch_rope_axes(const void *x, void *out, int L, int H, int d, long long T, const long long xs[3],
                             const long long os[3], const int *positions, long long axis_stride, const unsigned char *axis_of_pair,
                             double base, int inverse, cudaStream_t st)
{
    RopeAxesArgs a;
    a.x = static_cast<const __nv_bfloat16 *>(x);
    a.out = static_cast<__nv_bfloat16 *>(out);
    a.x_sl = xs[0]; a.x_st = xs[1]; a.x_sh = xs[2];
    a.o_sl = os[0]; a.o_st = os[1]; a.o_sh = os[2];
    a.H = H; a.LH = L * H; a.T = T; a.pos = positions; a.axis_stride = axis_stride; a.inverse = inverse;
    // one power and then products in extended precision (64 powers took 3 us a call, as long as the launch)
    const long double ratio = powl((long double)base, -2.0L / (long double)d);
    long double turns = 1.0L / 6.283185307179586476925286766559L;
    for (int i = 0; i < ROPE_MAX_FREQ; ++i) {
        a.axis[i] = i < d / 2 ? axis_of_pair[i] : 0;
        a.f[i] = i < d / 2 ? (unsigned long long)(turns * 18446744073709551616.0L) : 0ull;   // turns < 0.16: no wrap
        turns *= ratio;
    }
    const long long rows = 512 / d, blocks = (T + rows - 1) / rows;
    // at most 64 (layer, head) pairs a block (one round of loads), fewer where that leaves SMs without a block
    const long long want = 4ll * device_sm_count();
    long long groups = (want + blocks - 1) / blocks;
    if (groups < (a.LH + 63) / 64) groups = (a.LH + 63) / 64;
    if (groups > a.LH) groups = a.LH;
    a.per = (int)((a.LH + groups - 1) / groups);
    dim3 grid((unsigned)blocks, (unsigned)((a.LH + a.per - 1) / a.per));
    if (d == 128) k_rope_axes<128><<<grid, 256, 0, st>>>(a); else k_rope_axes<64><<<grid, 256, 0, st>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace cb
