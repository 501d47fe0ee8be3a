// Queries and keys normalised head by head, rotated, and appended to the cache with the values, in one pass over the projection:
//     u' = u * gain / sqrt(mean(u^2) + eps)  over the d values of a head,   (u'_j, u'_{j + d/2}) rotated by position * base^(-2j/d)
// in fp32; every value is rounded to bf16 once, after the rotation.
#include "rope_store.h"

namespace ps {

// Sum over the d / 8 lanes (8 or 16, aligned) that share a head.
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// grid (row_blocks(T), ceil((n_q + 2 n_kv) / heads per block)), 256 threads.  A head takes D/8 threads; a thread owns the four rotation
// pairs (j, j + D/2), j = 4 * (its index in the head) .. + 3.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(NormRopeArgs a) {
    constexpr int TPH = D / 8, HALF = D / 2;
    const int t = row_of_block(blockIdx.x, a.T);
    if (t >= a.T) return;
    const RopeOut& o = a.out;
    const int hh = blockIdx.y * (256 / TPH) + threadIdx.x / TPH, j = 4 * (threadIdx.x % TPH);
    if (hh >= o.n_q + 2 * o.n_kv) return;   // whole heads: all lanes of a sum or none
    const int position = scalar_read(o.positions + t), slot = scalar_read(o.slots + t);
    float lo[4], hi[4];
    const size_t at = (size_t)t * a.ld + (size_t)hh * D + j;
    if constexpr (BF16) {
        const bf16_t* row = static_cast<const bf16_t*>(a.qkv) + at;
        const uint2 l = *reinterpret_cast<const uint2*>(row), h = *reinterpret_cast<const uint2*>(row + HALF);
        lo[0] = bf16_lo(l.x); lo[1] = bf16_hi(l.x); lo[2] = bf16_lo(l.y); lo[3] = bf16_hi(l.y);
        hi[0] = bf16_lo(h.x); hi[1] = bf16_hi(h.x); hi[2] = bf16_lo(h.y); hi[3] = bf16_hi(h.y);
    } else {
        const float* row = static_cast<const float*>(a.qkv) + at;
        for (int e = 0; e < 4; e++) lo[e] = hi[e] = 0.f;
        for (int s = 0; s < a.n_splits; s++) {
            const float4 l = *reinterpret_cast<const float4*>(row + s * a.split_stride), h = *reinterpret_cast<const float4*>(row + s * a.split_stride + HALF);
            lo[0] += l.x; lo[1] += l.y; lo[2] += l.z; lo[3] += l.w;
            hi[0] += h.x; hi[1] += h.y; hi[2] += h.z; hi[3] += h.w;
        }
    }
    if (a.gains && hh < o.n_q + o.n_kv) {
        const bf16_t* gain = a.gains + (hh < o.n_q ? 0 : D) + j;
        const uint2 gl = *reinterpret_cast<const uint2*>(gain), gh = *reinterpret_cast<const uint2*>(gain + HALF);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 4; e++) ss += lo[e] * lo[e] + hi[e] * hi[e];
        const float r = 1.0f / sqrtf(head_sum<TPH>(ss) / (float)D + a.eps);
        lo[0] *= r * bf16_lo(gl.x); lo[1] *= r * bf16_hi(gl.x); lo[2] *= r * bf16_lo(gl.y); lo[3] *= r * bf16_hi(gl.y);
        hi[0] *= r * bf16_lo(gh.x); hi[1] *= r * bf16_hi(gh.x); hi[2] *= r * bf16_lo(gh.y); hi[3] *= r * bf16_hi(gh.y);
    }
    rope_store(o, t, slot, hh, j, lo, hi, rope_angles(o, position, j));
}

hipError_t launch_qk_norm_rope(const NormRopeArgs& a, hipStream_t st) {
    if (a.T <= 0) return hipSuccess;
    const int d = a.out.d;
    if ((d != 64 && d != 128) || a.n_splits < 1 || a.n_splits > 8 || (a.bf16 && a.n_splits != 1)) return hipErrorInvalidValue;
    const int heads_per_block = 256 / (d / 8);
    const dim3 grid(row_blocks(a.T), (a.out.n_q + 2 * a.out.n_kv + heads_per_block - 1) / heads_per_block), block(256);
    if (d == 64 && a.bf16) hipLaunchKernelGGL((qk_norm_rope_kernel<64, true>), grid, block, 0, st, a);
    else if (d == 64) hipLaunchKernelGGL((qk_norm_rope_kernel<64, false>), grid, block, 0, st, a);
    else if (a.bf16) hipLaunchKernelGGL((qk_norm_rope_kernel<128, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((qk_norm_rope_kernel<128, false>), grid, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace ps
