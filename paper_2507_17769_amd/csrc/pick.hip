// Rules on logits and the pick (see ps_logit_rules for what they mean):
//     seen in the prompt or the output:  z > 0 ? z / repetition : z * repetition
//     z -= frequency * (times in the output);   in the output: z -= presence;   z += bias;   not allowed: z = -inf
//     next = the lowest index of the largest z,   logprob = z_next - log sum exp z
// Products and differences are rounded one by one, as written: which token wins must not depend on where a compiler fuses them.
//
// What bounds it is the logits, read once: a running maximum with the sum of exponentials below it takes one pass.  A row's vocabulary is cut into
// segments, a block each; a block counts the list's tokens that fall into its segment in LDS (every block scans the whole list, which comes
// from L2), while its logits are on their way in registers.  Rows that are nodes of trees share their list: a block then takes several of
// them, counts once, and moves each row's branch into the counts and out again, the next row's logits on their way.  The last block of a row
// to finish joins the segments, in their order.  A block alone is a chain of trips to memory (its rows, what belongs to the list, the list and the
// logits, the arrival), so it sends the loads of each trip together, and four blocks share a compute unit.
// Measured, calls back to back (a kernel traced on its own takes 3 us more): 64 rows of 128256, bf16 read, fp32 written, lists of 2000 tokens, in 27 us,
// 50 MB of which a copy takes 11; with empty lists 18.  fp32, 504 rows of 63-node trees in 72 us: 259 MB, 3.6 TB/s, where a plain read takes 43;
// with empty lists 63.  One row: the kernel takes 8 us.  Counters of neighbouring rows in one line cost 8 us at 8 rows, loads under a lane's own condition twice the time at 64.

#include "ps_device.h"

#include <algorithm>
#include <type_traits>

namespace ps {

constexpr int PICK_THREADS = 256;
constexpr int PICK_ROWS = 8;          // rows of a block, at most
constexpr int PICK_WINDOW = 256;      // rows whose parents and tokens a block of tree nodes keeps in LDS
constexpr int PICK_BRANCH = 128;      // tokens of a branch in the segment that it keeps, a longer branch is walked in memory
constexpr int PICK_BIASES = 256;      // biases in the segment that a block keeps (a thread each), the list is searched for further ones
constexpr uint32_t IN_PROMPT = 0x80000000u, SEARCHED = 0x40000000u;   // beside the times in the output

// Running maximum, its lowest index, and the sum of exp(z - maximum).
struct Best {
    float m, s;
    int i;
};
__device__ __forceinline__ Best nothing() { return Best{-INFINITY, 0.f, 0x7fffffff}; }
// Ties go to the lower index, a NaN is never the maximum but enters the sum.
__device__ __forceinline__ Best best_join(const Best& x, const Best& y) {
    const bool first = x.m > y.m || (x.m == y.m && x.i < y.i);
    const Best hi = first ? x : y, lo = first ? y : x;
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

struct PickLaunch : PickArgs {
    int rows_per_block, segments, groups;
    int first_row, end_row;               // of this launch
    bool logits_wide, out_wide;           // four values at a time are aligned, and whole
    unsigned long long* partial;          // [rows of the launch][segments][2]: (maximum, sum), index
    int* arrived;                         // [rows of the launch], PICK_LINE apart, zero between launches
};

// A partial result travels between blocks of different XCDs: written through and read around their L2s.
__device__ __forceinline__ void put_partial(unsigned long long* p, const Best& b) {
    __hip_atomic_store(p, (unsigned long long)__float_as_uint(b.m) | ((unsigned long long)__float_as_uint(b.s) << 32), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(p + 1, (unsigned long long)(uint32_t)b.i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Best get_partial(unsigned long long* p) {
    const unsigned long long x = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), y = __hip_atomic_load(p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return Best{__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32)), (int)(uint32_t)y};
}
__device__ __forceinline__ Best wave_join(Best b) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) b = best_join(b, Best{__shfl_xor(b.m, o, 64), __shfl_xor(b.s, o, 64), __shfl_xor(b.i, o, 64)});
    return b;
}

// One value of a wavefront's 64 by moves between lanes that stay in the vector pipe: within rows of 16, then across them; lane 63 has it.
template <class F>
__device__ __forceinline__ int wave_fold(int x, int unit, F f) {
    x = f(x, __builtin_amdgcn_update_dpp(unit, x, 0x111, 0xf, 0xf, false));   // from 1, 2, 4 and 8 lanes below
    x = f(x, __builtin_amdgcn_update_dpp(unit, x, 0x112, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(unit, x, 0x114, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(unit, x, 0x118, 0xf, 0xf, false));
    x = f(x, __builtin_amdgcn_update_dpp(unit, x, 0x142, 0xa, 0xf, false));   // a row's last lane to the next row
    x = f(x, __builtin_amdgcn_update_dpp(unit, x, 0x143, 0xc, 0xf, false));   // lane 31 to the upper half
    return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ float fold_max(float x) {
    return __int_as_float(wave_fold(__float_as_int(x), (int)0xFF800000, [](int p, int q) { return __float_as_int(fmaxf(__int_as_float(p), __int_as_float(q))); }));
}
__device__ __forceinline__ int fold_min(int x) {
    return wave_fold(x, 0x7fffffff, [](int p, int q) { return min(p, q); });
}
__device__ __forceinline__ void put_result(const PickLaunch& a, int row, const Best& b) {
    const bool found = b.i != 0x7fffffff;
    if (a.next) a.next[row] = found ? b.i : -1;
    if (a.logprob) a.logprob[row] = b.m == INFINITY ? __builtin_nanf("") : found ? -logf(b.s) : b.s == 0.f ? -INFINITY : b.s;
}

// Four adjacent logits as they are stored.  Loads stand alone, at addresses in bounds for every lane: under a condition of its own, or with
// arithmetic on its result beside it, each would be waited for before the next is sent.
template <bool BF16, bool WIDE>
struct Quad {
    typename std::conditional<BF16 && WIDE, uint2, uint4>::type w;
    // of the n of a row from p on, n >= 1, those from i on; what lies behind the end is the last one's
    __device__ __forceinline__ void load(const void* p, int i, int n) {
        if constexpr (WIDE) {   // n is a multiple of four
            w = *reinterpret_cast<const decltype(w)*>(static_cast<const char*>(p) + (size_t)min(i, n - 4) * (BF16 ? 2 : 4));
        } else if constexpr (BF16) {
            const bf16_t* v = static_cast<const bf16_t*>(p);
            w = uint4{v[min(i, n - 1)], v[min(i + 1, n - 1)], v[min(i + 2, n - 1)], v[min(i + 3, n - 1)]};
        } else {
            const uint32_t* v = static_cast<const uint32_t*>(p);
            w = uint4{v[min(i, n - 1)], v[min(i + 1, n - 1)], v[min(i + 2, n - 1)], v[min(i + 3, n - 1)]};
        }
    }
    __device__ __forceinline__ void unpack(float* z) const {
        if constexpr (BF16 && WIDE) {
            z[0] = bf16_lo(w.x); z[1] = bf16_hi(w.x); z[2] = bf16_lo(w.y); z[3] = bf16_hi(w.y);
        } else {
            const int shift = BF16 ? 16 : 0;
            z[0] = __uint_as_float(w.x << shift); z[1] = __uint_as_float(w.y << shift); z[2] = __uint_as_float(w.z << shift); z[3] = __uint_as_float(w.w << shift);
        }
    }
};

// grid (segments * groups of rows): the first segments of all rows, where vocabularies keep their frequent tokens, start first.  Q quads of adjacent tokens a thread: a segment is 1024 Q tokens.
template <bool BF16, int Q, bool WIDE>
__global__ __launch_bounds__(PICK_THREADS, WIDE ? 4 : 1) void pick_kernel(PickLaunch a) {
    constexpr int SEG = 4 * PICK_THREADS * Q;
    __shared__ __attribute__((aligned(16))) uint32_t seen[SEG];
    __shared__ Best part[PICK_ROWS][PICK_THREADS / 64];
    __shared__ uint16_t branch[PICK_ROWS][PICK_BRANCH];   // places in the segment of the tokens of the rows' branches
    __shared__ int branch_len[PICK_ROWS], last[PICK_ROWS], row_list[PICK_ROWS], row_mask[PICK_ROWS];
    __shared__ int words[8];
    __shared__ int bias_place[PICK_BIASES];               // of the biases that fall into the segment, the place in the list
    __shared__ float bias_value[PICK_BIASES];
    __shared__ int bias_token[PICK_BIASES];               // and in the segment
    __shared__ int n_bias;
    const ps_logit_rules& R = a.rules;
    const int tid = threadIdx.x, V = a.vocab, segment = blockIdx.x / a.groups, v0 = segment * SEG, n = min(SEG, V - v0);
    const int r0 = a.first_row + (blockIdx.x - segment * a.groups) * a.rows_per_block, r1 = min(r0 + a.rows_per_block, a.end_row);
    const bool counts = R.n_lists > 0 || R.row_token;

    // What the rows are, a thread a row: each step of the way to the first results is a trip to memory, so few steps, and the logits beside them.
    auto above = [&](int r) {   // the row above a row, an earlier one
        const int up = R.row_prev ? R.row_prev[r] : -1;
        return up < r ? up : -1;
    };
    const int my_row = min(r0 + tid, r1 - 1), w0 = max(0, r1 - PICK_WINDOW), my_win = min(w0 + tid, r1 - 1);
    int list_in = R.n_lists > 0 ? my_row : -1, mask_in = R.mask ? my_row : -1, prev_in = -1, token_in = 0;
    if (R.n_lists > 0 && R.row_list) list_in = R.row_list[my_row];
    if (R.mask && R.mask_row) mask_in = R.mask_row[my_row];
    if (R.row_token) token_in = R.row_token[my_win];
    if (R.row_token && R.row_prev) prev_in = R.row_prev[my_win];
    hold(list_in); hold(mask_in); hold(prev_in); hold(token_in);
    if (tid < r1 - r0) {
        row_list[tid] = list_in < R.n_lists ? max(list_in, -1) : -1;
        row_mask[tid] = mask_in;   // >= n_masks: nothing is allowed
        branch_len[tid] = 0;
    }
    int* const win_prev = reinterpret_cast<int*>(seen);
    int* const win_token = win_prev + PICK_WINDOW;
    if (R.row_token) {
        win_prev[tid] = prev_in;
        win_token[tid] = token_in;
    }
    __syncthreads();
    if (R.row_token) {
        // Branches from the leaf up (ascending parents end them), walked in LDS: a walk through memory takes a trip a step.
        if (tid < r1 - r0) {
            int len = 0;
            for (int r = r0 + tid; r >= 0;) {
                const bool in = r >= w0;
                const uint32_t t = (uint32_t)(in ? win_token[r - w0] : R.row_token[r]) - (uint32_t)v0;
                if (t < (uint32_t)n) {
                    if (len < PICK_BRANCH) branch[tid][len] = (uint16_t)t;
                    len++;
                }
                const int up = in ? win_prev[r - w0] : above(r);
                r = up < r ? up : -1;
            }
            branch_len[tid] = len;
        }
        __syncthreads();
    }
    // a row's logits and the words of its mask
    Quad<BF16, WIDE> ahead[Q];
    uint32_t allowed_ahead[Q];
    auto load_row = [&](int row) {
        const char* p = static_cast<const char*>(a.logits) + ((size_t)row * a.ld + v0) * (BF16 ? 2 : 4);
#pragma unroll
        for (int q = 0; q < Q; q++) ahead[q].load(p, (q * PICK_THREADS + tid) * 4, n);
        const int mask = __builtin_amdgcn_readfirstlane(row_mask[row - r0]);
        if (mask >= 0 && mask < R.n_masks) {
            const uint32_t* bits = R.mask + (size_t)mask * R.mask_stride;
#pragma unroll
            for (int q = 0; q < Q; q++) allowed_ahead[q] = bits[(v0 + min((q * PICK_THREADS + tid) * 4, n - 1)) >> 5];
        } else {
#pragma unroll
            for (int q = 0; q < Q; q++) allowed_ahead[q] = mask < 0 ? 0xFFFFFFFFu : 0u;
        }
    };
    // a row's branch joins the counts, or leaves them
    auto count_branch = [&](int row, uint32_t by) {
        const int len = branch_len[row - r0];
        if (len <= PICK_BRANCH) {
            if (tid < len) atomicAdd(&seen[branch[row - r0][tid]], by);
        } else if (tid == 0) {   // more than LDS keeps: the way through memory once more
            for (int r = row; r >= 0; r = above(r)) {
                const uint32_t t = (uint32_t)R.row_token[r] - (uint32_t)v0;
                if (t < (uint32_t)n) atomicAdd(&seen[t], by);
            }
        }
    };

    int counted = -2;           // list whose tokens are in LDS, -1: none
    float rep = 1.f, freq = 0.f, pres = 0.f;
    int b0 = 0, b1 = 0;
    // the last bias of the segment's token t, which has one
    auto bias_of = [&](int t) {
        int place = b1 - 1;
        while (place > b0 && R.bias_token[place] != v0 + t) place--;
        int value = __float_as_int(R.bias_value[place]);
        hold(value);   // waited for here, not where this way meets others
        return __int_as_float(value);
    };
    for (int row = r0; row < r1; row++) {
        const int list = __builtin_amdgcn_readfirstlane(row_list[row - r0]);
        if (counts && list != counted) {
            counted = list;
            // what belongs to the list, a thread a word: one trip to memory where conditional reads would take one each
            const void* const from[8] = {R.repetition, R.frequency, R.presence, R.history ? R.history_begin : nullptr, R.history ? R.history_begin : nullptr,
                                         R.output_begin, R.bias_token ? R.bias_begin : nullptr, R.bias_token ? R.bias_begin : nullptr};
            const int k = tid & 7;
            const void* p = from[0];
#pragma unroll
            for (int j = 1; j < 8; j++) p = k == j ? from[j] : p;
            const bool given = list >= 0 && p;
            int w = static_cast<const int*>(given ? p : a.arrived)[given ? list + (k == 4 || k == 7) : 0];
            hold(w);
            if (row == r0) load_row(row);   // on its way while the list is counted
            if (!given) w = k == 0 ? 0x3F800000 : k == 5 ? (int)0x80000000 : 0;   // a repetition penalty of one; the output begins where the list does
            if (tid < 8) words[tid] = w;
#pragma unroll
            for (int q = 0; q < Q; q++) reinterpret_cast<uint4*>(seen)[q * PICK_THREADS + tid] = uint4{0u, 0u, 0u, 0u};
            if (tid == 0) n_bias = 0;
            __syncthreads();
            rep = __int_as_float(words[0]); freq = __int_as_float(words[1]); pres = __int_as_float(words[2]);
            const int h0 = clamp_to(words[3], 0, R.n_history), h1 = clamp_to(words[4], h0, R.n_history), ho = clamp_to(words[5], h0, h1);
            b0 = clamp_to(words[6], 0, R.n_biases); b1 = clamp_to(words[7], b0, R.n_biases);
            constexpr int AHEAD = 8;   // loads on their way together
            int bt = 0;
            float bv = 0.f;
            if (b0 < b1) { bt = R.bias_token[min(b0 + tid, b1 - 1)]; bv = R.bias_value[min(b0 + tid, b1 - 1)]; }
            for (int i0 = h0; i0 < h1; i0 += AHEAD * PICK_THREADS) {
                int t[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; u++) t[u] = R.history[min(i0 + u * PICK_THREADS + tid, h1 - 1)];
#pragma unroll
                for (int u = 0; u < AHEAD; u++) {
                    const int i = i0 + u * PICK_THREADS + tid;
                    const uint32_t at = (uint32_t)t[u] - (uint32_t)v0;
                    if (at < (uint32_t)n && i < h1) {
                        if (i < ho) atomicOr(&seen[at], IN_PROMPT);
                        else atomicAdd(&seen[at], 1u);
                    }
                }
            }
            for (int i0 = b0; i0 < b1; i0 += PICK_THREADS) {
                const uint32_t at = (uint32_t)bt - (uint32_t)v0;
                if (at < (uint32_t)n && i0 + tid < b1) {
                    const int k = atomicAdd(&n_bias, 1);
                    if (k < PICK_BIASES) { bias_place[k] = i0 + tid; bias_token[k] = at; bias_value[k] = bv; }
                    else atomicOr(&seen[at], SEARCHED);
                }
                const int next = min(i0 + PICK_THREADS + tid, b1 - 1);
                bt = R.bias_token[next];
                bv = R.bias_value[next];
            }
            if (R.row_token) count_branch(row, 1u);
            __syncthreads();
            if (n_bias > 0) {
                // of two biases of a token the later one stands, and none of a token that is searched for
                bool stands = tid < min(n_bias, PICK_BIASES) && !(seen[bias_token[tid]] & SEARCHED);
                for (int k = 0; stands && k < min(n_bias, PICK_BIASES); k++) stands = bias_token[k] != bias_token[tid] || bias_place[k] <= bias_place[tid];
                __syncthreads();
                if (tid < PICK_BIASES && !stands) bias_token[tid] = SEG;
                __syncthreads();
            }
        } else if (row == r0) {
            load_row(row);
        }
        float z[4 * Q];
        uint32_t allowed[Q];
#pragma unroll
        for (int q = 0; q < Q; q++) {
            ahead[q].unpack(z + 4 * q);
            allowed[q] = allowed_ahead[q];
        }
        if (n < SEG) {   // the vocabulary ends inside the segment
#pragma unroll
            for (int j = 0; j < 4 * Q; j++) z[j] = ((j >> 2) * PICK_THREADS + tid) * 4 + (j & 3) < n ? z[j] : -INFINITY;
        }
        if (row + 1 < r1) load_row(row + 1);
        if (counts) {
            // Few tokens are in the lists: a thread takes those of its quads one by one, where the rules for every token would cost more than
            // the rest of the way.
#pragma unroll
            for (int q = 0; q < Q; q++) {
                const uint4 s = reinterpret_cast<const uint4*>(seen)[q * PICK_THREADS + tid];
                uint32_t mine = (s.x ? 1u : 0u) | (s.y ? 2u : 0u) | (s.z ? 4u : 0u) | (s.w ? 8u : 0u);
                while (mine) {
                    const int e = __builtin_ctz(mine);
                    mine &= mine - 1;
                    const uint32_t times = e == 0 ? s.x : e == 1 ? s.y : e == 2 ? s.z : s.w;
                    float x = e == 0 ? z[4 * q] : e == 1 ? z[4 * q + 1] : e == 2 ? z[4 * q + 2] : z[4 * q + 3];
                    x = apply_rules(x, times & ~SEARCHED, rep, freq, pres);
                    if (times & SEARCHED) x += bias_of((q * PICK_THREADS + tid) * 4 + e);
#pragma unroll
                    for (int j = 0; j < 4; j++) z[4 * q + j] = e == j ? x : z[4 * q + j];
                }
            }
            const int biases = __builtin_amdgcn_readfirstlane(min(n_bias, PICK_BIASES));
            for (int k = 0; k < biases; k++) {
                const int t = bias_token[k];
                if ((t >> 2) % PICK_THREADS != tid || t == SEG) continue;
                const float by = bias_value[k];
#pragma unroll
                for (int j = 0; j < 4 * Q; j++) z[j] = t == ((j >> 2) * PICK_THREADS + tid) * 4 + (j & 3) ? z[j] + by : z[j];
            }
        }
        if (__builtin_amdgcn_readfirstlane(row_mask[row - r0]) >= 0) {
#pragma unroll
            for (int j = 0; j < 4 * Q; j++) {
                const int bit = ((v0 + tid * 4) & 31) + (j & 3);   // segments and quads' strides are whole words
                z[j] = (allowed[j >> 2] >> bit) & 1u ? z[j] : -INFINITY;
            }
        }
        if (a.out) {
#pragma unroll
            for (int q = 0; q < Q; q++) {
                const int i = (q * PICK_THREADS + tid) * 4;
                float* o = a.out + (size_t)row * a.ldo + v0 + i;
                if (i + 4 <= n && a.out_wide) *reinterpret_cast<float4*>(o) = float4{z[4 * q], z[4 * q + 1], z[4 * q + 2], z[4 * q + 3]};
                else
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (i + e < n) o[e] = z[4 * q + e];
            }
        }
        // The wavefront's maximum first, then exponentials below it and the lowest place of those that reach it.
        float top = z[0];   // of what is not NaN
#pragma unroll
        for (int j = 1; j < 4 * Q; j++) top = fmaxf(top, z[j]);
        top = fold_max(fmaxf(top, -INFINITY));
        const float base = top > -INFINITY ? top : 0.f;   // all -inf: exp(-inf) is 0, of NaN NaN
        float sum = 0.f;
        int at = 0x7fffffff;
#pragma unroll
        for (int j = 4 * Q - 1; j >= 0; j--) {
            sum += __expf(z[j] - base);
            at = z[j] == top ? ((j >> 2) * PICK_THREADS + tid) * 4 + (j & 3) : at;
        }
        sum = wave_sum(sum);
        at = fold_min(at);
        if ((tid & 63) == 0) part[row - r0][tid >> 6] = Best{top, sum, top > -INFINITY ? v0 + at : 0x7fffffff};
        if (row + 1 < r1 && counts) {
            // The next row's counts: the same list's, with its branch in place of this one's, or another's that begin from nothing.
            const bool same = __builtin_amdgcn_readfirstlane(row_list[row + 1 - r0]) == counted;
            if (!same || (R.row_token && (branch_len[row - r0] | branch_len[row + 1 - r0]) != 0)) {
                __syncthreads();
                if (same) {
                    count_branch(row, 0xFFFFFFFFu);
                    count_branch(row + 1, 1u);
                    __syncthreads();
                }
            }
        }
    }
    __syncthreads();
    if (tid < r1 - r0) {
        Best b = part[tid][0];
#pragma unroll
        for (int w = 1; w < PICK_THREADS / 64; w++) b = best_join(b, part[tid][w]);
        const int row = r0 + tid;
        if (a.segments == 1) {
            put_result(a, row, b);
        } else {
            put_partial(a.partial + ((size_t)(row - a.first_row) * a.segments + segment) * 2, b);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // written through before it is counted
            last[tid] = __hip_atomic_fetch_add(a.arrived + (size_t)(row - a.first_row) * PICK_LINE, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.segments - 1;
        }
    }
    if (a.segments == 1) return;
    __syncthreads();
    for (int k = tid >> 6; k < r1 - r0; k += PICK_THREADS / 64) {
        if (!last[k]) continue;
        const int row = r0 + k;
        Best b = nothing();
        for (int s = tid & 63; s < a.segments; s += 64) b = best_join(b, get_partial(a.partial + ((size_t)(row - a.first_row) * a.segments + s) * 2));
        b = wave_join(b);
        if ((tid & 63) == 0) {
            put_result(a, row, b);
            a.arrived[(size_t)(row - a.first_row) * PICK_LINE] = 0;   // clean for the next launch
        }
    }
}

template <int Q>
static void launch_q(const PickLaunch& a, hipStream_t st) {
    const dim3 grid(a.segments * a.groups), block(PICK_THREADS);
    if (a.bf16 && a.logits_wide) hipLaunchKernelGGL((pick_kernel<true, Q, true>), grid, block, 0, st, a);
    else if (a.bf16) hipLaunchKernelGGL((pick_kernel<true, Q, false>), grid, block, 0, st, a);
    else if (a.logits_wide) hipLaunchKernelGGL((pick_kernel<false, Q, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((pick_kernel<false, Q, false>), grid, block, 0, st, a);
}

hipError_t launch_pick(const PickArgs& args, void* workspace, hipStream_t st) {
    PickLaunch a;
    static_cast<PickArgs&>(a) = args;
    a.partial = static_cast<unsigned long long*>(workspace);
    a.arrived = reinterpret_cast<int*>(static_cast<char*>(workspace) + (size_t)PICK_PARTIALS * 16);
    a.out_wide = (reinterpret_cast<uintptr_t>(a.out) & 15) == 0 && a.ldo % 4 == 0;
    a.logits_wide = (reinterpret_cast<uintptr_t>(a.logits) & (a.bf16 ? 7 : 15)) == 0 && a.ld % 4 == 0 && a.vocab % 4 == 0;
    // Rows of trees share a list: eight to a block, as long as there are blocks for every compute unit to hold a few.  Segments as long as
    // that leaves as many blocks, down to 1024 tokens: each scans its list once more.
    const long long rows = a.n_rows, tokens = (long long)rows * a.vocab;
    a.rows_per_block = 1;
    if (a.rules.row_list)
        while (a.rows_per_block < PICK_ROWS && tokens / (2 * a.rows_per_block) >= 768ll * 4096) a.rows_per_block *= 2;
    int q = 4;
    while (q > 1 && tokens / a.rows_per_block < 768ll * 1024 * q) q /= 2;
    a.segments = (a.vocab + 1024 * q - 1) / (1024 * q);
    // a launch has as many rows as the workspace holds partial results of
    const int most = std::min(PICK_MAX_ROWS, PICK_PARTIALS / a.segments);
    for (a.first_row = 0; a.first_row < a.n_rows; a.first_row = a.end_row) {
        a.end_row = std::min(a.n_rows, a.first_row + most);
        a.groups = (a.end_row - a.first_row + a.rows_per_block - 1) / a.rows_per_block;
        switch (q) {
            case 4: launch_q<4>(a, st); break;
            case 2: launch_q<2>(a, st); break;
            default: launch_q<1>(a, st);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ps
