// Rules on logits and the pick (see ps_logit_rules for what they mean):
//     seen in the prompt or the output:  z > 0 ? z / repetition : z * repetition
//     z -= frequency * (times in the output);   in the output: z -= presence;   z += bias;   not allowed: z = -inf
//     next = the lowest index of the largest z,   logprob = z_next - log sum exp z
// Products and differences are rounded one by one, as written: which token wins must not depend on where a compiler fuses them.
#include "ps_device.h"

namespace ps {

constexpr int PICK_SEG = 8192;        // tokens whose counts and biases are in LDS at a time
constexpr uint32_t IN_PROMPT = 0x80000000u;

// Running maximum, its lowest index, and the sum of exp(z - maximum).
struct Best {
    float m, s;
    int i;
};
__device__ __forceinline__ void best_add(Best& b, float z, int i) {
    if (z > b.m) {   // never for NaN, which the sum takes
        b.s = b.s * __expf(b.m - z) + 1.f;   // b.m = -inf: 0 * 0
        b.m = z; b.i = i;
    } else if (!(z == -INFINITY)) {
        b.s += __expf(z - b.m);
    }
}
// order-independent but for the rounding of the sum; ties go to the lower index
__device__ __forceinline__ Best best_join(const Best& x, const Best& y) {
    const bool first = x.m > y.m || (x.m == y.m && x.i < y.i);
    const Best &hi = first ? x : y, &lo = first ? y : x;
    Best r = hi;
    if (lo.s != 0.f) r.s += lo.s * (lo.m == hi.m ? 1.f : __expf(lo.m - hi.m));
    return r;
}

__device__ __forceinline__ float apply_rules(float z, uint32_t seen, float rep, float freq, float pres) {
#pragma clang fp contract(off)
    if (seen != 0) {
        z = z > 0.f ? z / rep : z * rep;
        const uint32_t times = seen & ~IN_PROMPT;
        if (times != 0) {
            const float f = freq * (float)times;
            z = z - f;
            z = z - pres;
        }
    }
    return z;
}

__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// One block per row, the vocabulary a segment at a time: lists are scanned for the segment's tokens, then the segment is read.
template <bool BF16>
__global__ __launch_bounds__(1024) void pick_kernel(PickArgs a) {
    __shared__ uint32_t seen[PICK_SEG];
    __shared__ int biased[PICK_SEG];    // 1 + place of the token's last bias in the list, 0: none
    __shared__ Best part[16];
    const ps_logit_rules& R = a.rules;
    const int row = blockIdx.x, V = a.vocab, tid = threadIdx.x;
    const int list = R.n_lists > 0 ? (R.row_list ? R.row_list[row] : row) : -1;
    const bool listed = list >= 0 && list < R.n_lists;
    float rep = 1.f, freq = 0.f, pres = 0.f;
    int h0 = 0, h1 = 0, ho = 0, b0 = 0, b1 = 0;
    if (listed) {
        if (R.repetition) rep = R.repetition[list];
        if (R.frequency) freq = R.frequency[list];
        if (R.presence) pres = R.presence[list];
        if (R.history) {
            h0 = clamp_to(R.history_begin[list], 0, R.n_history); h1 = clamp_to(R.history_begin[list + 1], h0, R.n_history);
            ho = R.output_begin ? clamp_to(R.output_begin[list], h0, h1) : h0;
        }
        if (R.bias_token) { b0 = clamp_to(R.bias_begin[list], 0, R.n_biases); b1 = clamp_to(R.bias_begin[list + 1], b0, R.n_biases); }
    }
    const int mask = R.mask ? (R.mask_row ? R.mask_row[row] : row) : -1;
    const bool none = mask >= R.n_masks && mask >= 0;   // no such mask: nothing is allowed
    const uint32_t* bits = mask >= 0 && !none ? R.mask + (size_t)mask * R.mask_stride : nullptr;

    Best best{-INFINITY, 0.f, 0x7fffffff};
    for (int v0 = 0; v0 < V; v0 += PICK_SEG) {
        const int n = min(PICK_SEG, V - v0);
        for (int i = tid; i < n; i += 1024) { seen[i] = 0; biased[i] = 0; }
        __syncthreads();
        for (int i = h0 + tid; i < h1; i += 1024) {
            const uint32_t t = (uint32_t)R.history[i] - (uint32_t)v0;
            if (t < (uint32_t)n) {
                if (i < ho) atomicOr(&seen[t], IN_PROMPT);
                else atomicAdd(&seen[t], 1u);
            }
        }
        if (tid == 0 && R.row_token)
            for (int r = row, up; r >= 0; r = up) {   // rows of a branch, from the leaf up; ascending parents end it
                const uint32_t t = (uint32_t)R.row_token[r] - (uint32_t)v0;
                if (t < (uint32_t)n) atomicAdd(&seen[t], 1u);
                up = R.row_prev ? R.row_prev[r] : -1;
                if (up >= r) break;
            }
        for (int i = b0 + tid; i < b1; i += 1024) {
            const uint32_t t = (uint32_t)R.bias_token[i] - (uint32_t)v0;
            if (t < (uint32_t)n) atomicMax(&biased[t], i - b0 + 1);
        }
        __syncthreads();
        for (int i = tid; i < n; i += 1024) {
            const int v = v0 + i;
            float z = BF16 ? __uint_as_float((uint32_t)static_cast<const bf16_t*>(a.logits)[(size_t)row * a.ld + v] << 16)
                           : static_cast<const float*>(a.logits)[(size_t)row * a.ld + v];
            z = apply_rules(z, seen[i], rep, freq, pres);
            if (biased[i] != 0) z += R.bias_value[b0 + biased[i] - 1];
            if (none || (bits && ((bits[v >> 5] >> (v & 31)) & 1u) == 0)) z = -INFINITY;
            if (a.out) a.out[(size_t)row * a.ldo + v] = z;
            best_add(best, z, v);
        }
        __syncthreads();
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        best = best_join(best, Best{__shfl_xor(best.m, o, 64), __shfl_xor(best.s, o, 64), __shfl_xor(best.i, o, 64)});
    if ((tid & 63) == 0) part[tid >> 6] = best;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < 16; w++) best = best_join(best, part[w]);
        const bool found = best.i != 0x7fffffff;
        if (a.next) a.next[row] = found ? best.i : -1;
        if (a.logprob) a.logprob[row] = best.m == INFINITY ? __builtin_nanf("") : found ? -logf(best.s) : best.s == 0.f ? -INFINITY : best.s;
    }
}

hipError_t launch_pick(const PickArgs& a, hipStream_t st) {
    if (a.n_rows <= 0) return hipSuccess;
    if (a.bf16) hipLaunchKernelGGL(pick_kernel<true>, dim3(a.n_rows), dim3(1024), 0, st, a);
    else hipLaunchKernelGGL(pick_kernel<false>, dim3(a.n_rows), dim3(1024), 0, st, a);
    return hipGetLastError();
}

}  // namespace ps
