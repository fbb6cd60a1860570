// Rows of a mapped cache (or a step's new rows) of all layers into their pages: a scatter of 16-byte pieces, fp32 rows
// rounded to bf16 (nearest even) on the way.  Bound by HBM: every row is read once and written once.
#include "cb_paged.cuh"
#include "cb_math.cuh"

namespace cb {

// grid (pieces of one layer / 256, layers); a thread moves one piece (8 channels of one head) of K and of V.
template <bool F32>
__global__ void __launch_bounds__(256) k_paged_store(const StoreArgs a)
{
    const int pieces = a.d / 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long row = i / (a.H * pieces);
    if (row >= a.n_rows) return;
    const int rest = (int)(i - row * (a.H * pieces));
    const int h = rest / pieces, c = (rest - h * pieces) * 8;
    const long long slot = a.slot_map[row];
    if (slot < 0 || slot >= a.n_slots) return;
    const long long page = slot >> a.page_log2, off = slot & ((1 << a.page_log2) - 1);
    const long long from = (long long)blockIdx.y * a.s_sl + row * a.s_st + (long long)h * a.s_sh + c;
    const long long to = (long long)blockIdx.y * a.d_sl + page * a.d_sp + off * a.d_ss + (long long)h * a.d_sh + c;
    uint4 k, v;
    if (F32) {
        const float4 *sk = reinterpret_cast<const float4 *>(static_cast<const float *>(a.src_k) + from);
        const float4 *sv = reinterpret_cast<const float4 *>(static_cast<const float *>(a.src_v) + from);
        const float4 k0 = __ldcs(sk), k1 = __ldcs(sk + 1), v0 = __ldcs(sv), v1 = __ldcs(sv + 1);
        k = make_uint4(pack_bf16x2(k0.x, k0.y), pack_bf16x2(k0.z, k0.w), pack_bf16x2(k1.x, k1.y), pack_bf16x2(k1.z, k1.w));
        v = make_uint4(pack_bf16x2(v0.x, v0.y), pack_bf16x2(v0.z, v0.w), pack_bf16x2(v1.x, v1.y), pack_bf16x2(v1.z, v1.w));
    } else {
        k = __ldcs(reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.src_k) + from));
        v = __ldcs(reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.src_v) + from));
    }
    *reinterpret_cast<uint4 *>(a.k + to) = k;
    *reinterpret_cast<uint4 *>(a.v + to) = v;
}

cudaError_t launch_paged_store(const StoreArgs &a, cudaStream_t st)
{
    const long long n = a.n_rows * a.H * (a.d / 8);
    dim3 grid((unsigned)((n + 255) / 256), (unsigned)a.L);
    if (a.src_f32) k_paged_store<true><<<grid, 256, 0, st>>>(a); else k_paged_store<false><<<grid, 256, 0, st>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace cb
