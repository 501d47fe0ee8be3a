// Pieces that the attention kernels of steps and of trees have in common.
#pragma once
#include "ps_device.h"

namespace ps {

constexpr float NEG_BIG = -1.0e30f;

// K and V chunks of a pair of pages, as loaded: 16 bytes per lane per register.
template <int KS>
struct PairRegs {
    uint4 ka[KS], kb[KS], va[KS], vb[KS];
};

// Decode streams read every byte once: they load with the non-temporal hint (ldg16_stream), so that they do not push
// out of L2 what the teams of the same launch re-read (the keys and values of the prefill chunk's prefix).
template <int D>
__device__ __forceinline__ void load_pair(PairRegs<D / 32>& p, const bf16_t* pool_lane, size_t page_stride, int pa, int pb) {
    constexpr int KS = D / 32;
    const bf16_t* ca = pool_lane + (size_t)pa * page_stride;
    const bf16_t* cb = pool_lane + (size_t)pb * page_stride;
#pragma unroll
    for (int s = 0; s < KS; s++) {
        p.ka[s] = ldg16_stream(ca + s * 512);
        p.kb[s] = ldg16_stream(cb + s * 512);
    }
#pragma unroll
    for (int s = 0; s < KS; s++) {
        p.va[s] = ldg16_stream(ca + 16 * D + s * 512);
        p.vb[s] = ldg16_stream(cb + 16 * D + s * 512);
    }
}

// Running softmax state of NT query tiles against one KV stream.
template <int D, int NT>
struct TileState {
    f32x4_t o[NT][D / 16];
    float m[NT], lsum[NT];
};

// Maximum over the four lanes r, r+16, r+32, r+48 that share a query row, in the vector ALU:
// v_permlane16_swap (x, x) returns {rows 0,0,2,2 | rows 1,1,3,3} of x and v_permlane32_swap the
// {lower, lower | upper, upper} halves, so each step combines a lane with its partner in both.
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float row_quad_max(float v) {
    const u32x2_t a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a.x), __uint_as_float(a.y));
    const u32x2_t b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b.x), __uint_as_float(b.y));
}

__device__ __forceinline__ u32x2_t lds_read8(uint32_t addr, int off) {
    u32x2_t v;
    asm volatile("ds_read_b64 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(off) : "memory");
    return v;
}
// maximum of three without the quieting of signalling NaNs that fmaxf brings along
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// a * b, rounded, whatever it is added to (the compiler would make an fma of it)
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// Merge of split partials
constexpr int MERGE_MAX_WAVES = 16;
constexpr int MERGE_BATCH = 8;   // splits whose loads a wavefront has in flight

// Wavefronts that share a pass's splits: a batch each, a power of two, as many as the block has at most.
__host__ __device__ inline int merge_split_waves(int n_splits, int n_waves) {
    int nws = 1;
    while (nws < n_waves && nws * MERGE_BATCH < n_splits) nws *= 2;
    return nws;
}

}  // namespace ps
