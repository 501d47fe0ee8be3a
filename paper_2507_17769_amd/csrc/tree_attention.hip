// Attention of token trees over the paged cache: every new token ("node") of a sequence attends to the cached prefix, to its
// ancestors among the new tokens and to itself.
//
//     A(i) = {0 .. prefix - 1} + {prefix + j : j = i or an ancestor of i},   out_i = sum_{p in A(i)} softmax(q_i . k_p / sqrt(d)) v_p
//
// Parents come before their children, so A(i) lies within the causal range of place i and a batch is planned as a step's chunks
// and decodes are (planner.cpp): query blocks of several 16-row tiles go to teams of four wavefronts that share pairs of pages
// through a ring in LDS, single-tile blocks to streaming wavefronts.  What is new is who sees what: the pairs that reach past
// the prefix, the last few of a stream, are masked by one bit per row and position, read as a word per row and pair; the pairs of
// the prefix, all others, need no mask.  The two are loops of their own, so the long one carries nothing of the short one.
//
// Bounds and figures (16-bit cache, kernel alone, the join of partials beside it): eight chains of six, 32 query heads on 8 of 128, 80 MB: 21 + 4 us,
// HBM takes 13.  16-node trees, 317 MB: 63 + 6 us for 52; a copy of the pages alone by the same ring takes 58.  64-node trees, 64 query heads, 330 MB
// read by three query blocks each: 115 + 12 us, where the copies alone take 105 (the blocks' L2 requests) and the products alone 99; the
// matrix unit is busy a third of the time.  A deeper ring, one block of eight wavefronts a compute unit, and P.V of one tile under the softmax
// of the next were no faster.
//
// A masked place may hold anything, infinities and NaN too (a rejected branch of an overflowed draft; a page's tail that nobody
// wrote): its score is replaced, and its value must not reach a row that does not see it, which a zero weight alone does not
// give (0 * inf is NaN).  In the masked pairs non-finite values are taken out of the product; where there were any, the rows that
// do see them get them at the end of the item (see add_specials).
#include "attention_device.h"

#include <algorithm>
#include <type_traits>

namespace ps {

constexpr int TREE_WAVES = 4;   // of a block, of which a compute unit holds two
constexpr int TREE_NT = 3;      // query tiles of a wavefront, at most
constexpr int TREE_RING = 4;    // pairs of pages in LDS

// As PS_GLOBAL_TO_LDS, with the non-temporal hint: for pages that are read once.
__device__ __forceinline__ void global_to_lds_stream(const uint8_t* src, uint8_t* dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 16, 0, 2);
}

// The lane, formed anew for every item: what follows from it would otherwise be hoisted out of the loop over the items, for all kinds of
// item at once, and hold 28 registers through the loops over the pairs.
__device__ __forceinline__ int lane_id() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t & 63;
}

// What the row of token `qc` of the item's block sees of the 32 positions 32 pair .. 32 pair + 31.
__device__ __forceinline__ uint32_t visible_word(const TreeArgs& a, const AttnItem& it, int qc, int pair) {
    if (it.mask_at >= 0) return a.masks[it.mask_at + qc * it.mask_words + (pair - it.mask_pair)];
    const int left = it.pos0 + qc - 32 * pair;
    return left >= 31 ? 0xFFFFFFFFu : left < 0 ? 0u : (2u << left) - 1u;
}
// A team keeps the words of the first pairs that need them in LDS: a read from memory in the middle of the stream waits for all the pages
// on their way.  Trees of up to some 100 nodes have no further pairs; eight trees of 512 behind 4000 tokens take 316 us where chains of
// as many, whose words need no memory, take 302, one tree of 512 74 for 63.
constexpr int MASK_PAIRS = 4, MASK_ROWS = 16 * TREE_WAVES * TREE_NT;   // words of a row, tokens of a block at most
__device__ __forceinline__ uint32_t team_word(const TreeArgs& a, const AttnItem& it, const uint32_t* kept, int qc, int pair) {
    if (it.mask_at >= 0 && pair - it.mask_pair < MASK_PAIRS) return kept[(pair - it.mask_pair) * MASK_ROWS + qc];
    int w = (int)visible_word(a, it, qc, pair);
    hold(w);   // waited for here, not where the two ways meet
    return (uint32_t)w;
}
// Padding sees nothing, not even itself.
__device__ __forceinline__ bool is_padding(const TreeArgs& a, const AttnItem& it, int qc) {
    if (it.mask_at < 0) return false;
    const int p = it.pos0 + qc;
    return ((a.masks[it.mask_at + qc * it.mask_words + (p >> 5) - it.mask_pair] >> (p & 31)) & 1u) == 0;
}
// First pair that needs a mask for rows whose first token sits at pos_first.
__device__ __forceinline__ int first_masked_pair(const AttnItem& it, int pos_first) { return it.mask_at >= 0 ? it.mask_pair : (pos_first + 1) >> 5; }

// Classes of the eight bf16 values of an operand: 1.0 where the value is of the class.
enum { POS_INF, NEG_INF, NOT_A_NUMBER };
__device__ __forceinline__ uint32_t half_class(uint32_t h, int cls) {
    const bool special = (h & 0x7F80u) == 0x7F80u, nan = (h & 0x7Fu) != 0;
    const bool hit = special && (cls == NOT_A_NUMBER ? nan : !nan && ((h >> 15) & 1u) == (cls == NEG_INF ? 1u : 0u));
    return hit ? 0x3F80u : 0u;
}
__device__ __forceinline__ u32x4_t class_of(u32x4_t v, int cls) {
    u32x4_t o;
#pragma unroll
    for (int i = 0; i < 4; i++) o[i] = half_class(v[i] & 0xFFFFu, cls) | (half_class(v[i] >> 16, cls) << 16);
    return o;
}
__device__ __forceinline__ uint32_t without_specials(uint32_t w) {
    return ((w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u);
}
// of two packed pairs, the larger magnitude of either place; a pair with a magnitude of infinity or above
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t larger_halves(uint32_t x, uint32_t y) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, x & 0x7FFF7FFFu), __builtin_bit_cast(u16x2_t, y & 0x7FFF7FFFu)));
}
__device__ __forceinline__ bool is_special(uint32_t w) { return (w & 0x7FFFu) >= 0x7F80u || (w & 0x7FFF0000u) >= 0x7F800000u; }
__device__ __forceinline__ bool has_specials(u32x4_t v) { return is_special(larger_halves(larger_halves(v[0], v[1]), larger_halves(v[2], v[3]))); }
__device__ __forceinline__ f32x4_t mfma_16x16x32(u32x4_t a, bf16x8_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), b, c, 0, 0, 0);
}

__device__ __forceinline__ bf16_t* out_at(const TreeArgs& a, size_t tok, int col) {
    return a.out + (a.ldo ? tok * a.ldo + col : act_offset((int)tok, col, a.n_q * a.d));
}

// Ones where the lane's row sees the token: bits of a word (see visible_word) as an operand; g: the lane's key group.
__device__ __forceinline__ bf16x8_t seen_operand(uint32_t word, int g) {
    const uint32_t w = word >> (4 * g);
    u32x4_t seen;
    seen[0] = (w & 1u ? 0x3F80u : 0u) | (w & 2u ? 0x3F800000u : 0u);
    seen[1] = (w & 4u ? 0x3F80u : 0u) | (w & 8u ? 0x3F800000u : 0u);
    seen[2] = (w & 0x10000u ? 0x3F80u : 0u) | (w & 0x20000u ? 0x3F800000u : 0u);
    seen[3] = (w & 0x40000u ? 0x3F80u : 0u) | (w & 0x80000u ? 0x3F800000u : 0u);
    return __builtin_bit_cast(bf16x8_t, seen);
}

// After an item's rows have been stored: the non-finite values of its masked pairs, which the products left out, go to the rows that see
// them.  Three products of ones count, for each row and value of d, the +inf, -inf and NaN that it sees; every lane mends what it
// stored itself.  Rare, so it may read everything once more.
template <int D, int G, int NT>
__device__ __forceinline__ void add_specials(const TreeArgs& a, const AttnItem& it, int tok_row, int slot0, int first_pair, int last_pair, int lane) {
    constexpr int DT = D / 16, TQ = 16 / G;
    const int r = lane & 15, g = lane >> 4;
    const int32_t* pages = a.pages + it.page_off;
    const size_t page_stride = (size_t)a.n_kv * 2 * 16 * D;
    const bf16_t* v_lane = a.pool_slot + (size_t)it.kv_head * 2 * 16 * D + 16 * D + (size_t)lane * 8;
#pragma unroll 1
    for (int j = first_pair * DT; j < (last_pair + 1) * DT; j++) {
        const int pair = j / DT, dt = j % DT;
        const size_t at = (dt >> 1) * 512 + 4 * (dt & 1);
        const uint2 x = *reinterpret_cast<const uint2*>(v_lane + (size_t)pages[2 * pair] * page_stride + at);
        const uint2 y = *reinterpret_cast<const uint2*>(v_lane + (size_t)pages[min(2 * pair + 1, it.page_end - 1)] * page_stride + at);
        const u32x4_t v = {x.x, x.y, y.x, y.y};
        if (__builtin_amdgcn_ballot_w64(has_specials(v)) == 0) continue;
#pragma unroll 1
        for (int nt = 0; nt < NT; nt++) {
            const int qc = tok_row + nt * TQ;
            const bf16x8_t seen = seen_operand(visible_word(a, it, min(qc, it.q_ntok - 1), pair), g);
            const f32x4_t none = {0.f, 0.f, 0.f, 0.f};
            const f32x4_t up = mfma_16x16x32(class_of(v, POS_INF), seen, none), down = mfma_16x16x32(class_of(v, NEG_INF), seen, none),
                          nan = mfma_16x16x32(class_of(v, NOT_A_NUMBER), seen, none);
            if (qc >= it.q_ntok || is_padding(a, it, qc)) continue;
            float add[4];
            bool any = false;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                add[i] = nan[i] > 0.f || (up[i] > 0.f && down[i] > 0.f) ? __builtin_nanf("") : up[i] > 0.f ? __builtin_inff() : down[i] > 0.f ? -__builtin_inff() : 0.f;
                any = any || add[i] != 0.f;
            }
            if (!any) continue;
            if (it.partial < 0) {
                uint2* p = reinterpret_cast<uint2*>(out_at(a, (size_t)it.tok_g0 + qc, (it.kv_head * G + r % G) * D + 16 * dt + 4 * g));
                const uint2 w = *p;
                *p = uint2{pack_bf16(bf16_lo(w.x) + add[0], bf16_hi(w.x) + add[1]), pack_bf16(bf16_lo(w.y) + add[2], bf16_hi(w.y) + add[3])};
            } else {
                float4* p = reinterpret_cast<float4*>(a.part_o + (((size_t)it.partial + slot0 + nt) * 16 + r) * D + 16 * dt + 4 * g);
                const float4 w = *p;
                *p = float4{w.x + add[0], w.y + add[1], w.z + add[2], w.w + add[3]};
            }
        }
    }
}

// Scores of the keys that a row does not see become -inf: the running maximum starts at a large finite negative number, so a
// row that has seen nothing keeps it and gets weights of zero.
__device__ __forceinline__ void hide(f32x4_t& sa, f32x4_t& sb, uint32_t word, int g) {
    const uint32_t w = word >> (4 * g);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        sa[i] = (w >> i) & 1u ? sa[i] : -__builtin_inff();
        sb[i] = (w >> (16 + i)) & 1u ? sb[i] : -__builtin_inff();
    }
}

// Softmax of one tile for a pair: raw scores -> P as a packed operand, 2^(s scale2 - m).  m is a reference, not the running maximum: any
// number cancels that is the same in a row's sum and products, so it follows the maximum only when that has outgrown it by 2^16 (fp32 sums
// have room for far more).  After an item's first pairs that hardly ever happens, and a pair then needs neither the maximum across the four
// lanes of a row nor what came before rescaled, which took a third of the loop's vector instructions.  The row sums are taken from the
// rounded P by the matrix unit, so that the weights of a row add up to one exactly as rounded.  What it costs: the largest weight is rounded like
// the others, where against the maximum itself it is exactly 1.  Measured, against the maximum / as here: mean error of the values 1.9e-3 / 2.2e-3 of
// them, 1.4e-3 of it the rounding of the result; 16 trees of 64 nodes, 64 heads, 176 / 157 us, 32 heads 105 / 97, 32 trees of 16 73 / 71.
constexpr float OUTGROWN = 16.f;
template <int DT>
__device__ __forceinline__ bf16x8_t tile_softmax(const f32x4_t& sa, const f32x4_t& sb, float& m, f32x4_t (&o)[DT], f32x4_t& l, float scale2) {
    const float sv[8] = {sa[0], sa[1], sa[2], sa[3], sb[0], sb[1], sb[2], sb[3]};
    float mx = max3(max3(sv[0], sv[1], sv[2]), max3(sv[3], sv[4], sv[5]), max3(sv[6], sv[7], sv[7]));
    if (__builtin_amdgcn_ballot_w64(fmaf(mx, scale2, -m) > OUTGROWN) != 0) {
        const u32x2_t x = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        const float y = max3(__uint_as_float(x.x), __uint_as_float(x.y), mx);
        const u32x2_t z = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
        mx = max3(__uint_as_float(z.x), __uint_as_float(z.y), y);
        // only the rows that have outgrown theirs: a row's roundings are its own affair, not that of the others in its tile
        const float ms = fmaf(mx, scale2, -m) > OUTGROWN ? rounded_product(mx, scale2) : m, alpha = __builtin_amdgcn_exp2f(m - ms);
        m = ms;
#pragma unroll
        for (int dt = 0; dt < DT; dt++) { o[dt][0] *= alpha; o[dt][1] *= alpha; o[dt][2] *= alpha; o[dt][3] *= alpha; }
        l[0] *= alpha; l[1] *= alpha; l[2] *= alpha; l[3] *= alpha;
    }
    float pv[8];
#pragma unroll
    for (int i = 0; i < 8; i++) pv[i] = __builtin_amdgcn_exp2f(fmaf(sv[i], scale2, -m));
    uint4 pw;
    pw.x = pack_bf16(pv[0], pv[1]);
    pw.y = pack_bf16(pv[2], pv[3]);
    pw.z = pack_bf16(pv[4], pv[5]);
    pw.w = pack_bf16(pv[6], pv[7]);
    return as_bf16x8(pw);
}

// The assembly of max3 reads matrix results: the compiler places no waits for it, so the last product's passes are waited for here.
__device__ __forceinline__ void matrix_results(f32x4_t& a, f32x4_t& b) { asm volatile("s_nop 15\n\ts_nop 1" : "+v"(a), "+v"(b)); }
__device__ __forceinline__ void matrix_results(f32x4_t& a, f32x4_t& b, f32x4_t& c, f32x4_t& d) {
    asm volatile("s_nop 15\n\ts_nop 1" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
}
__device__ __forceinline__ void matrix_results(f32x4_t& a, f32x4_t& b, f32x4_t& c, f32x4_t& d, f32x4_t& e, f32x4_t& f) {
    asm volatile("s_nop 15\n\ts_nop 1" : "+v"(a), "+v"(b), "+v"(c), "+v"(d), "+v"(e), "+v"(f));
}

constexpr u32x4_t ONES = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};

// End of an item: the NT tiles of a wavefront go to the output (normalised) or, for an item that covers only part of its KV span, to
// partial slots it.partial + slot0 + nt.  l: each row's sum, the same in the four lanes that share the row.  Padding gets zeros, in a partial with
// a weight of its own: a sum of zero is left to rows whose scores are all -inf, and their quotient, NaN, does not depend on how a plan cuts them.
// Which 16 values of d accumulator dt holds: swapped accumulators (see team_pair) hold the neighbour's in the lanes of g >= 2.
template <bool SWAP>
__device__ __forceinline__ int dt_of(int dt, int g) { return SWAP ? dt ^ (g >> 1) : dt; }

template <int D, int G, int NT, bool SWAP>
__device__ __forceinline__ void store_rows(const TreeArgs& a, const AttnItem& it, const f32x4_t (&o)[NT][D / 16], const float (&m)[NT], const float (&l)[NT],
                                           int tok_row, int slot0, int lane) {
    constexpr int DT = D / 16, TQ = 16 / G;
    const int r = lane & 15, g = lane >> 4;
    const int head = it.kv_head * G + (r % G);
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
        const int qc = tok_row + nt * TQ;
        if (qc >= it.q_ntok) continue;   // rows beyond the block's tokens are never merged: do not store them
        const bool padding = is_padding(a, it, qc);
        if (it.partial < 0) {
            const float inv = padding ? 0.f : 1.0f / l[nt];
            const size_t tok = (size_t)it.tok_g0 + qc;
#pragma unroll
            for (int dt = 0; dt < DT; dt++) {
                const int col = head * D + 16 * dt_of<SWAP>(dt, g) + 4 * g;
                uint2 w;
                w.x = padding ? 0u : pack_bf16(o[nt][dt][0] * inv, o[nt][dt][1] * inv);
                w.y = padding ? 0u : pack_bf16(o[nt][dt][2] * inv, o[nt][dt][3] * inv);
                *reinterpret_cast<uint2*>(out_at(a, tok, col)) = w;
            }
        } else {
            const size_t slot = (size_t)it.partial + slot0 + nt;
            float* po = a.part_o + (slot * 16 + r) * D + 4 * g;
#pragma unroll
            for (int dt = 0; dt < DT; dt++)
                *reinterpret_cast<float4*>(po + 16 * dt_of<SWAP>(dt, g)) =
                    padding ? float4{0.f, 0.f, 0.f, 0.f} : float4{o[nt][dt][0], o[nt][dt][1], o[nt][dt][2], o[nt][dt][3]};
            if (g == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * 16 + r) * 2) = padding ? float2{NEG_BIG, 1.f} : float2{m[nt], l[nt]};
        }
    }
}

// ---- single-tile blocks: one wavefront -------------------------------------------------------------
// The next pair of pages is in flight in a second register set while the current one is consumed.
template <int D, bool MASK>
__device__ __forceinline__ void wave_pair(f32x4_t (&o)[1][D / 16], f32x4_t& lacc, float& m, bool& specials, PairRegs<D / 32>& p, const bf16x8_t (&qf)[D / 32],
                                          uint32_t word, int g, float scale2) {
    constexpr int KS = D / 32, DT = D / 16;
    f32x4_t sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; s++) {
        sa = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(p.ka[s]), qf[s], sa, 0, 0, 0);
        sb = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(p.kb[s]), qf[s], sb, 0, 0, 0);
    }
    matrix_results(sa, sb);
    if constexpr (MASK) {
        hide(sa, sb, word, g);
        uint32_t largest = 0;
#pragma unroll
        for (int s = 0; s < KS; s++) {
            largest = larger_halves(largest, larger_halves(larger_halves(p.va[s].x, p.va[s].y), larger_halves(p.va[s].z, p.va[s].w)));
            largest = larger_halves(largest, larger_halves(larger_halves(p.vb[s].x, p.vb[s].y), larger_halves(p.vb[s].z, p.vb[s].w)));
        }
        if (__builtin_amdgcn_ballot_w64(is_special(largest)) != 0) {
            specials = true;
#pragma unroll
            for (int s = 0; s < KS; s++) {
                p.va[s] = uint4{without_specials(p.va[s].x), without_specials(p.va[s].y), without_specials(p.va[s].z), without_specials(p.va[s].w)};
                p.vb[s] = uint4{without_specials(p.vb[s].x), without_specials(p.vb[s].y), without_specials(p.vb[s].z), without_specials(p.vb[s].w)};
            }
        }
    }
    const bf16x8_t pf = tile_softmax<DT>(sa, sb, m, o[0], lacc, scale2);
    lacc = mfma_16x16x32(ONES, pf, lacc);
    // one product per page and d-tile: each 8-byte half of a loaded register quad is an operand as it stands, where one for both pages would
    // take 64 register moves
    const uint4 pw = __builtin_bit_cast(uint4, pf);
    const s16x4_t pa = __builtin_bit_cast(s16x4_t, uint2{pw.x, pw.y}), pb = __builtin_bit_cast(s16x4_t, uint2{pw.z, pw.w});
#pragma unroll
    for (int dt = 0; dt < DT; dt++) {
        const int s = dt >> 1;
        const uint2 wa = (dt & 1) ? uint2{p.va[s].z, p.va[s].w} : uint2{p.va[s].x, p.va[s].y};
        const uint2 wb = (dt & 1) ? uint2{p.vb[s].z, p.vb[s].w} : uint2{p.vb[s].x, p.vb[s].y};
        o[0][dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, wa), pa, o[0][dt], 0, 0, 0);
        o[0][dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, wb), pb, o[0][dt], 0, 0, 0);
    }
}

template <int D, int G>
__device__ __forceinline__ void wave_item(const TreeArgs& a, const AttnItem it) {
    constexpr int KS = D / 32, DT = D / 16;
    const int lane = lane_id();
    const int r = lane & 15, g = lane >> 4;
    const int32_t* pages = a.pages + it.page_off;
    const int head = it.kv_head * G + (r % G);
    const int qc = min(r / G, it.q_ntok - 1);
    bf16x8_t qf[KS];
    const bf16_t* qrow = a.q + (size_t)(it.tok_g0 + qc) * a.ldq + head * D + 8 * g;
#pragma unroll
    for (int s = 0; s < KS; s++) qf[s] = as_bf16x8(ldg16(qrow + 32 * s));
    f32x4_t o[1][DT], lacc = {0.f, 0.f, 0.f, 0.f};
    float m = NEG_BIG;
    bool specials = false;
#pragma unroll
    for (int dt = 0; dt < DT; dt++) o[0][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const float scale2 = 1.4426950408889634f / sqrtf((float)D);  // log2(e)/sqrt(d): softmax in base 2
    const size_t page_stride = (size_t)a.n_kv * 2 * 16 * D;
    const bf16_t* pool_lane = a.pool_slot + (size_t)it.kv_head * 2 * 16 * D + (size_t)lane * 8;
    const int masked = first_masked_pair(it, it.pos0);
    // Pages in blocks of up to 64: lane l keeps the id of the block's page l, and a uniform readlane hands the ids out, so no load
    // sits between a pair's id and its data.  The item carries its first two ids: the first loads do not wait for the others.
    for (int blk = it.page_begin; blk < it.page_end; blk += 64) {
        const int n_pg = min(64, it.page_end - blk);
        const int my_pid = pages[blk + min(lane, n_pg - 1)];
        const int n_pairs = (n_pg + 1) >> 1, pair0 = blk >> 1;
        auto load = [&](PairRegs<KS>& p, int i) {
            load_pair<D>(p, pool_lane, page_stride, __builtin_amdgcn_readlane(my_pid, 2 * i), __builtin_amdgcn_readlane(my_pid, min(2 * i + 1, n_pg - 1)));
        };
        // two register sets; the steady body issues its loads unconditionally, so that the wait before each computation covers
        // exactly the older set
        PairRegs<KS> b0, b1;
        if (blk == it.page_begin) load_pair<D>(b0, pool_lane, page_stride, it.page0, it.page1);
        else load(b0, 0);
        const int n_free = min(n_pairs, masked - pair0);
        int i = 0;
        for (; i + 2 < n_free; i += 2) {
            load(b1, i + 1);
            __builtin_amdgcn_sched_barrier(0);
            wave_pair<D, false>(o, lacc, m, specials, b0, qf, 0, g, scale2);
            __builtin_amdgcn_sched_barrier(0);
            load(b0, i + 2);
            __builtin_amdgcn_sched_barrier(0);
            wave_pair<D, false>(o, lacc, m, specials, b1, qf, 0, g, scale2);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the last one or two pairs of the block that need no mask, whose values stay as they are, then the masked ones, which the stream ends with
        auto step = [&](auto mask_c) {
            constexpr bool MASK = decltype(mask_c)::value;
            load(b1, min(i + 1, n_pairs - 1));
            wave_pair<D, MASK>(o, lacc, m, specials, b0, qf, MASK ? visible_word(a, it, qc, pair0 + i) : 0, g, scale2);
#pragma unroll
            for (int s = 0; s < KS; s++) { b0.ka[s] = b1.ka[s]; b0.kb[s] = b1.kb[s]; b0.va[s] = b1.va[s]; b0.vb[s] = b1.vb[s]; }
        };
        for (; i < n_free; i++) step(std::false_type{});
        for (; i < n_pairs; i++) step(std::true_type{});
    }
    const float ml[1] = {m}, l[1] = {lacc[0]};
    store_rows<D, G, 1, false>(a, it, o, ml, l, r / G, 0, lane);
    if (specials) add_specials<D, G, 1>(a, it, r / G, 0, max(masked, it.page_begin >> 1), (it.page_end - 1) >> 1, lane);
}

// ---- teams: blocks of several tiles ---------------------------------------------------------------
// One pair of pages from ring slot `addr` (LDS byte address of this lane's 16 bytes of the slot's first KiB) for the
// wavefront's NT tiles.  The slot holds the pair as 4 KS KiB blocks [k-step s][K page a, K page b, V page a, V page b].  A V operand is an 8-byte
// half of a lane's 16 bytes: were it the same half in all lanes, two lanes would share each bank.  Lanes 8 .. 15 of every 16 read the other
// one (vswap = 8), so accumulator dt holds in its rows 8 .. 15 the values of tile dt ^ 1: its lanes of g >= 2 (see dt_of).
template <int D, int G, int NT, bool MASK>
__device__ __forceinline__ void team_pair(f32x4_t (&o)[NT][D / 16], f32x4_t (&lacc)[NT], float (&m)[NT], bool& specials, uint32_t addr, const bf16x8_t (&qf)[NT][D / 32],
                                          const TreeArgs& a, const AttnItem& it, const uint32_t* kept, int tok_row, int pair, int g, uint32_t vswap, float scale2) {
    constexpr int KS = D / 32, DT = D / 16;
    uint32_t word[NT];
    if constexpr (MASK) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) word[nt] = team_word(a, it, kept, min(tok_row + nt * (16 / G), it.q_ntok - 1), pair);
        __builtin_amdgcn_sched_barrier(0);
    }
    u32x4_t kk[2 * KS];
#pragma unroll
    for (int s = 0; s < KS; s++) {
        kk[2 * s] = lds_read16(addr, (4 * s + 0) * 1024);
        kk[2 * s + 1] = lds_read16(addr, (4 * s + 1) * 1024);
    }
    if constexpr (KS == 4)
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(kk[0]), "+v"(kk[1]), "+v"(kk[2]), "+v"(kk[3]), "+v"(kk[4]), "+v"(kk[5]), "+v"(kk[6]), "+v"(kk[7]));
    else
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(kk[0]), "+v"(kk[1]), "+v"(kk[2]), "+v"(kk[3]));
    f32x4_t sa[NT], sb[NT];
    auto scores = [&](int nt) {
        sa[nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        sb[nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; s++) {
            sa[nt] = mfma_16x16x32(kk[2 * s], qf[nt][s], sa[nt]);
            sb[nt] = mfma_16x16x32(kk[2 * s + 1], qf[nt][s], sb[nt]);
        }
    };
    bf16x8_t pf[NT];
    if constexpr (MASK) {   // tile by tile, for the registers
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            scores(nt);
            matrix_results(sa[nt], sb[nt]);
            hide(sa[nt], sb[nt], word[nt], g);
            pf[nt] = tile_softmax<DT>(sa[nt], sb[nt], m[nt], o[nt], lacc[nt], scale2);
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) scores(nt);
    }
    __builtin_amdgcn_sched_barrier(0);   // the values after the keys: they take the keys' registers, and the softmax covers their way
    u32x2_t va[DT], vb[DT];
#pragma unroll
    for (int dt = 0; dt < DT; dt++) {
        const uint32_t half = (dt & 1) ? addr ^ vswap ^ 8 : addr ^ vswap;
        va[dt] = lds_read8(half, (4 * (dt >> 1) + 2) * 1024);
        vb[dt] = lds_read8(half, (4 * (dt >> 1) + 3) * 1024);
    }
    if constexpr (!MASK) {
        if constexpr (NT == 1) matrix_results(sa[0], sb[0]);
        else if constexpr (NT == 2) matrix_results(sa[0], sb[0], sa[1], sb[1]);
        else matrix_results(sa[0], sb[0], sa[1], sb[1], sa[2], sb[2]);
#pragma unroll
        for (int nt = 0; nt < NT; nt++) pf[nt] = tile_softmax<DT>(sa[nt], sb[nt], m[nt], o[nt], lacc[nt], scale2);
    }
    if constexpr (DT == 8)
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(va[0]), "+v"(va[1]), "+v"(va[2]), "+v"(va[3]), "+v"(va[4]), "+v"(va[5]), "+v"(va[6]), "+v"(va[7]),
                     "+v"(vb[0]), "+v"(vb[1]), "+v"(vb[2]), "+v"(vb[3]), "+v"(vb[4]), "+v"(vb[5]), "+v"(vb[6]), "+v"(vb[7]));
    else
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(va[0]), "+v"(va[1]), "+v"(va[2]), "+v"(va[3]), "+v"(vb[0]), "+v"(vb[1]), "+v"(vb[2]), "+v"(vb[3]));
    if constexpr (MASK) {
        uint32_t largest = 0;
#pragma unroll
        for (int dt = 0; dt < DT; dt++) largest = larger_halves(largest, larger_halves(larger_halves(va[dt].x, va[dt].y), larger_halves(vb[dt].x, vb[dt].y)));
        if (__builtin_amdgcn_ballot_w64(is_special(largest)) != 0) {
            specials = true;
#pragma unroll
            for (int dt = 0; dt < DT; dt++) {
                va[dt] = u32x2_t{without_specials(va[dt].x), without_specials(va[dt].y)};
                vb[dt] = u32x2_t{without_specials(vb[dt].x), without_specials(vb[dt].y)};
            }
        }
    }
    __builtin_amdgcn_s_setprio(1);   // the matrix unit is fed first (see attn_kernel)
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
        lacc[nt] = mfma_16x16x32(ONES, pf[nt], lacc[nt]);
#pragma unroll
        for (int dt = 0; dt < DT; dt++) {
            const u32x4_t v = {va[dt].x, va[dt].y, vb[dt].x, vb[dt].y};
            o[nt][dt] = mfma_16x16x32(v, pf[nt], o[nt][dt]);
        }
    }
    __builtin_amdgcn_s_setprio(0);
}

// One work item on a team.  The four wavefronts of the block are RW = 4 / KW row groups of NT tiles times KW key groups: with few tiles
// the pairs of pages are dealt out to key groups, so that no wavefront is idle, and the groups' results are joined in LDS at the end.
// Per round of KW pairs: wait for the own copies of this round (those of later rounds may still be in flight), barrier (every
// wavefront's part has landed, and every wavefront has finished with the round before, whose slots are the ones to refill), issue
// the copies of the round that takes those slots, compute.  Past the item's last pair the copies fetch that pair again, into slots nobody
// reads, so that the wait counts are the same in every trip.
template <int D, int G, int NT, int KW, bool ONCE>
__device__ __forceinline__ void team_item(const TreeArgs& a, const AttnItem it, uint8_t* ring, uint32_t* kept, int wave) {
    static_assert(KW == 1 || NT == 1, "the join holds one tile a wavefront");
    constexpr int KS = D / 32, DT = D / 16, TQ = 16 / G;
    constexpr int RW = TREE_WAVES / KW, ROUNDS = TREE_RING / KW;   // rounds in the ring
    constexpr int PAIR_BYTES = 4 * KS * 1024, LPW = 4 * KS / TREE_WAVES;   // KiB blocks of a pair that a wavefront copies
    const int lane = lane_id();
    const int r = lane & 15, g = lane >> 4, rg = wave % RW, kg = wave / RW;
    const int32_t* pages = a.pages + it.page_off;
    const int head = it.kv_head * G + (r % G);
    const int n_pg = it.page_end - it.page_begin;
    int tbl = pages[it.page_begin + min(lane, n_pg - 1)];

    // Row (lane r) of tile nt is token (rg NT + nt) TQ + r / G of the block, clamped to the block's last token (rows past it
    // compute on that token's data and are not stored).
    auto row_now = [&]() { return rg * NT * TQ + (lane_id() & 15) / G; };   // formed anew: not held through the loops
    const int tok_row = row_now();
    bf16x8_t qf[NT][KS];
    auto load_queries = [&](int tok) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            const int qc = min(tok + nt * TQ, it.q_ntok - 1);
            const bf16_t* qrow = a.q + (size_t)(it.tok_g0 + qc) * a.ldq + head * D + 8 * g;
#pragma unroll
            for (int s = 0; s < KS; s++) qf[nt][s] = as_bf16x8(ldg16(qrow + 32 * s));
        }
    };
    auto hold_queries = [&]() {
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int s = 0; s < KS; s++) {   // they have arrived: else their first use, in a loop, would wait in every trip, and with it for all copies
                u32x4_t x = __builtin_bit_cast(u32x4_t, qf[nt][s]);
                asm volatile("" : "+v"(x));
                qf[nt][s] = __builtin_bit_cast(bf16x8_t, x);
            }
    };
    load_queries(tok_row);
    const int group_tok0 = rg * NT * TQ;
    const bool has_rows = group_tok0 < it.q_ntok;
    const int pos_first = it.pos0 + min(group_tok0, it.q_ntok - 1);
    const int pos_last = it.pos0 + min(group_tok0 + NT * TQ, it.q_ntok) - 1;   // nothing beyond is seen by any row of the group

    f32x4_t o[NT][DT], lacc[NT];
    float m[NT];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
        m[nt] = NEG_BIG;
        lacc[nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < DT; dt++) o[nt][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const float scale2 = 1.4426950408889634f / sqrtf((float)D);
    const uint32_t page_bytes = (uint32_t)a.n_kv * 2 * 16 * D * 2, lane16 = lane * 16, vswap = lane & 8;
    // A pair is 4 KS KiB blocks [k-step][K page a, K page b, V page a, V page b]; the wavefront copies the blocks LPW wave + k.
    const int c0 = wave * LPW;
    const uint8_t* const pool_wave = reinterpret_cast<const uint8_t*>(a.pool_slot) + (size_t)it.kv_head * 2 * 16 * D * 2 + (c0 >> 2) * 1024 + ((c0 >> 1) & 1) * 32 * D;
    const uint32_t ring0 = (uint32_t)(uintptr_t)ring;

    const int n_pairs = (n_pg + 1) >> 1, pair0 = it.page_begin >> 1;
    const int n_rounds = (n_pairs + KW - 1) / KW;
    int tb0 = 0;   // ids of 64 pages at a time in tbl, lane l holding page tb0 + l of the item's range
    hold(tbl);     // it has arrived: else every use of it in the loops would wait, and with it for all copies
    auto issue = [&](int round) {
        const int first = min(round * KW, n_pairs - 1);
        if (2 * first >= tb0 + 64) {   // a round lies within 64 pages
            tb0 += 64;
            tbl = pages[it.page_begin + tb0 + min(lane, n_pg - tb0 - 1)];
            vm_wait<0>();   // here, so that the compiler does not wait for everything where the paths join
        }
#pragma unroll
        for (int j = 0; j < KW; j++) {
            const int la = 2 * min(round * KW + j, n_pairs - 1) - tb0;
            uint8_t* dst = ring + ((round % ROUNDS) * KW + j) * PAIR_BYTES + c0 * 1024;
            const uint32_t page[2] = {(uint32_t)__builtin_amdgcn_readlane(tbl, la), (uint32_t)__builtin_amdgcn_readlane(tbl, min(la + 1, n_pg - tb0 - 1))};
            uint32_t off[2] = {lane16, lane16 + 32 * D};   // K and V of a page (of head dim 64, a wavefront copies only one)
            asm volatile("" : "+v"(off[0]), "+v"(off[1]));   // 32-bit offsets in registers of their own: scalar base + vector offset addressing
            const uint8_t* src[2] = {pool_wave + (uint64_t)page[0] * page_bytes, pool_wave + (uint64_t)page[1] * page_bytes};
#pragma unroll
            for (int k = 0; k < LPW; k++) {
                if constexpr (ONCE) global_to_lds_stream(src[k & 1] + off[k >> 1], dst + k * 1024);
                else PS_GLOBAL_TO_LDS(src[k & 1] + off[k >> 1], dst + k * 1024);
            }
        }
    };

    __builtin_amdgcn_s_barrier();   // every wavefront has finished with the ring and the words (previous item)
    if (it.mask_at >= 0) {
        const int qc = 64 * wave + lane, at = it.mask_at + min(qc, it.q_ntok - 1) * it.mask_words;
        int w[MASK_PAIRS];
#pragma unroll
        for (int k = 0; k < MASK_PAIRS; k++) w[k] = (int)a.masks[at + min(k, it.mask_words - 1)];
#pragma unroll
        for (int k = 0; k < ROUNDS - 1; k++) issue(k);
#pragma unroll
        for (int k = 0; k < MASK_PAIRS; k++) {
            hold(w[k]);
            if (qc < it.q_ntok) kept[k * MASK_ROWS + qc] = (uint32_t)w[k];   // read after the barrier of a round
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    } else {
#pragma unroll
        for (int k = 0; k < ROUNDS - 1; k++) issue(k);
    }
    hold_queries();
    // The row group sees the first n_mine pairs, the first n_free of them without a mask; of both the wavefront has every KW-th.  Past
    // them it only keeps copying and meeting the barriers: three loops, so that no accumulator is live across a branch.
    const int n_mine = !has_rows ? 0 : max(0, min(n_pairs, (pos_last >> 5) - pair0 + 1));
    const int n_free = max(0, min(n_mine, first_masked_pair(it, pos_first) - pair0));
    const int free_rounds = (n_free - kg + KW - 1) / KW, my_rounds = (n_mine - kg + KW - 1) / KW;   // of less than one pair: 0 or less
    bool specials = false;
    int i = 0;
    auto step = [&]() {
        vm_wait<(ROUNDS - 2) * KW * LPW>();
        __builtin_amdgcn_s_barrier();
        issue(i + ROUNDS - 1);
    };
    auto slot = [&]() { return ring0 + ((i % ROUNDS) * KW + kg) * PAIR_BYTES + lane16; };
    for (; i < free_rounds; i++) {
        step();
        team_pair<D, G, NT, false>(o, lacc, m, specials, slot(), qf, a, it, kept, tok_row, 0, g, vswap, scale2);
    }
    if (NT == 3 && i < my_rounds) {
        // Read once more: the masked loop needs more registers than there are beside three tiles, and queries that live through both
        // loops would be the ones it moves out, in the long loop too.
        load_queries(row_now());
        hold_queries();
    }
    const int mtok = row_now();
    for (; i < my_rounds; i++) {
        step();
        team_pair<D, G, NT, true>(o, lacc, m, specials, slot(), qf, a, it, kept, mtok, pair0 + i * KW + kg, (lane_id() >> 4), vswap, scale2);
    }
    for (; i < n_rounds; i++) step();
    vm_wait<0>();   // the surplus copies have landed before the ring is used again
    if constexpr (KW > 1) {
        // Key groups 1 .. leave maximum, sum and accumulators in LDS, group 0 joins them.
        __builtin_amdgcn_s_barrier();   // nobody reads or fills the ring any more
        float4* const mine = reinterpret_cast<float4*>(ring + (size_t)(kg * RW + rg) * (DT + 1) * 1024);
        if (kg > 0) {
#pragma unroll
            for (int dt = 0; dt < DT; dt++) mine[dt * 64 + lane] = float4{o[0][dt][0], o[0][dt][1], o[0][dt][2], o[0][dt][3]};
            mine[DT * 64 + lane] = float4{m[0], lacc[0][0], specials ? 1.f : 0.f, 0.f};
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int j = 1; j < KW; j++) {
            const float4* theirs = mine + (size_t)j * RW * (DT + 1) * 64;
            const float4 ml = theirs[DT * 64 + lane];
            const float M = fmaxf(m[0], ml.x), f = __builtin_amdgcn_exp2f(m[0] - M), h = __builtin_amdgcn_exp2f(ml.x - M);
            m[0] = M;
            lacc[0][0] = lacc[0][0] * f + ml.y * h;
            specials = specials || __builtin_amdgcn_ballot_w64(ml.z != 0.f) != 0;
#pragma unroll
            for (int dt = 0; dt < DT; dt++) {
                const float4 v = theirs[dt * 64 + lane];
                o[0][dt][0] = o[0][dt][0] * f + v.x * h; o[0][dt][1] = o[0][dt][1] * f + v.y * h;
                o[0][dt][2] = o[0][dt][2] * f + v.z * h; o[0][dt][3] = o[0][dt][3] * f + v.w * h;
            }
        }
    }
    if (!has_rows) return;
    float l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) l[nt] = lacc[nt][0];
    store_rows<D, G, NT, true>(a, it, o, m, l, row_now(), rg * NT, lane_id());
    if (specials) add_specials<D, G, NT>(a, it, row_now(), rg * NT, pair0 + n_free, pair0 + n_mine - 1, lane_id());
}

// ONCE: no sequence has a second query block that reads the same pages again.
template <int D, int G, bool ONCE>
__global__ __launch_bounds__(64 * TREE_WAVES) __attribute__((amdgpu_waves_per_eu(2, 2))) void tree_kernel(TreeArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t ring[TREE_RING * (D / 8) * 1024];   // also holds the join: 4 (D / 16 + 1) KiB
    __shared__ uint32_t kept[MASK_PAIRS * MASK_ROWS];                                       // words of masks (see team_word)
    // contiguous shares of either work list on every XCD, as in attn_kernel
    const int xcd = blockIdx.x & 7, j = blockIdx.x >> 3;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (j < a.team_per_xcd) {
        const int t = xcd * a.team_per_xcd + j;
        if (t >= a.n_team) return;
        const int i0 = a.worker_begin[t], i1 = a.worker_begin[t + 1];
        for (int i = i0; i < i1; i++) {
            const AttnItem it = a.items[i];
            const int tiles = (it.q_ntok + 16 / G - 1) / (16 / G);
            if (tiles <= 2) team_item<D, G, 1, 2, ONCE>(a, it, ring, kept, wave);
            else if (tiles <= 4) team_item<D, G, 1, 1, ONCE>(a, it, ring, kept, wave);
            else if (tiles <= 8) team_item<D, G, 2, 1, ONCE>(a, it, ring, kept, wave);
            else team_item<D, G, 3, 1, ONCE>(a, it, ring, kept, wave);
        }
    } else {
        const int w = a.n_team + (xcd * a.wave_blocks_per_xcd + (j - a.team_per_xcd)) * TREE_WAVES + wave;
        if (j - a.team_per_xcd >= a.wave_blocks_per_xcd || w >= a.n_workers) return;
        const int i0 = a.worker_begin[w], i1 = a.worker_begin[w + 1];
        for (int i = i0; i < i1; i++) wave_item<D, G>(a, a.items[i]);
    }
}

// Combine split partials of one query tile: out = sum_j 2^(m_j - M) O_j / sum_j 2^(m_j - M) l_j.
// One block per merge group, its wavefronts in a (pass, split) grid as in attn_merge_kernel.
template <int D, int G>
__global__ __launch_bounds__(64 * MERGE_MAX_WAVES) void tree_merge_kernel(TreeArgs a) {
    __shared__ float4 s_acc[MERGE_MAX_WAVES][64];
    __shared__ float2 s_ml[MERGE_MAX_WAVES][64];
    const int group = merge_group_of_block(blockIdx.x, a.n_groups);
    if (group >= a.n_groups) return;
    const int32_t* gp = reinterpret_cast<const int32_t*>(a.groups + group);
    MergeGroup mg;
    mg.tok0 = scalar_read(gp); mg.n_tok = scalar_read(gp + 1); mg.kv_head = scalar_read(gp + 2);
    mg.first_slot = scalar_read(gp + 3); mg.n_splits = scalar_read(gp + 4); mg.stride = scalar_read(gp + 5);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), NW = blockDim.x >> 6;   // NW: a power of two
    const int NWS = merge_split_waves(mg.n_splits, NW), NWP = NW / NWS, ws = wave % NWS, wp = wave / NWS;
    const int n_items = mg.n_tok * G * (D / 4);   // valid rows are the first n_tok * G of the tile
    for (int c0 = 0; c0 < n_items; c0 += 64 * NWP) {   // the same trip count for every wavefront: the barriers below
        const int c = c0 + wp * 64 + lane;
        const bool live = c < n_items;
        const int r = live ? c / (D / 4) : 0, col = live ? (c % (D / 4)) * 4 : 0;
        float M = NEG_BIG, L = 0.f;
        float4 acc = {0.f, 0.f, 0.f, 0.f};
        const int n_splits = c0 + wp * 64 < n_items ? mg.n_splits : 0;   // a wavefront past the last pass only meets the barriers
        for (int j0 = ws; j0 < n_splits; j0 += MERGE_BATCH * NWS) {
            float2 ml[MERGE_BATCH];
            float4 v[MERGE_BATCH];
#pragma unroll
            for (int j = 0; j < MERGE_BATCH; j++)
                if (j0 + j * NWS < n_splits) {
                    const size_t row = (size_t)(mg.first_slot + (j0 + j * NWS) * mg.stride) * 16 + r;
                    ml[j] = *reinterpret_cast<const float2*>(a.part_ml + row * 2);
                    v[j] = *reinterpret_cast<const float4*>(a.part_o + row * D + col);
                }
            float m_new = M;
#pragma unroll
            for (int j = 0; j < MERGE_BATCH; j++)
                if (j0 + j * NWS < n_splits) m_new = fmaxf(m_new, ml[j].x);
            const float f = __builtin_amdgcn_exp2f(M - m_new);
            M = m_new;
            L *= f; acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
#pragma unroll
            for (int j = 0; j < MERGE_BATCH; j++)
                if (j0 + j * NWS < n_splits) {
                    const float w = __builtin_amdgcn_exp2f(ml[j].x - M);
                    L += w * ml[j].y;
                    acc.x += w * v[j].x; acc.y += w * v[j].y; acc.z += w * v[j].z; acc.w += w * v[j].w;
                }
        }
        if (NWS > 1) {
            s_acc[wave][lane] = acc;
            s_ml[wave][lane] = float2{M, L};
            __syncthreads();
            if (ws == 0) {
                for (int w = 1; w < NWS; w++) M = fmaxf(M, s_ml[wave + w][lane].x);
                acc = float4{0.f, 0.f, 0.f, 0.f};
                L = 0.f;
                for (int w = 0; w < NWS; w++) {
                    const float2 q = s_ml[wave + w][lane];
                    const float4 v = s_acc[wave + w][lane];
                    const float f = __builtin_amdgcn_exp2f(q.x - M);
                    L += f * q.y;
                    acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
                }
            }
        }
        if (ws == 0 && live) {
            const float inv = 1.0f / L;
            const int head = mg.kv_head * G + r % G, tok = mg.tok0 + r / G;
            uint2 w;
            w.x = pack_bf16(acc.x * inv, acc.y * inv);
            w.y = pack_bf16(acc.z * inv, acc.w * inv);
            *reinterpret_cast<uint2*>(out_at(a, tok, head * D + col)) = w;
        }
        if (NWS > 1) __syncthreads();  // the next pass overwrites the LDS slots
    }
}

int tree_tokens_per_item(int G) { return TREE_WAVES * TREE_NT * (16 / G); }

template <int D, int G>
static hipError_t launch_dg(const TreeArgs& a_in, hipStream_t st) {
    TreeArgs a = a_in;
    a.team_per_xcd = (a.n_team + 7) >> 3;
    a.wave_blocks_per_xcd = ((a.n_workers - a.n_team + TREE_WAVES - 1) / TREE_WAVES + 7) >> 3;
    const dim3 grid((a.team_per_xcd + a.wave_blocks_per_xcd) * 8), block(64 * TREE_WAVES);
    if (a.ev_begin) (void)hipEventRecord(a.ev_begin, st);
    if (a.pages_once) hipLaunchKernelGGL((tree_kernel<D, G, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((tree_kernel<D, G, false>), grid, block, 0, st, a);
    hipError_t e = hipGetLastError();
    if (a.ev_end) (void)hipEventRecord(a.ev_end, st);
    if (e != hipSuccess || a.n_groups == 0) return e;
    // wavefronts of a block: for the most splits times the most passes (a power of two each) of any group
    const int passes = (std::max(1, a.max_merge_rows) * (D / 4) + 63) / 64;
    int nw = merge_split_waves(a.max_splits, MERGE_MAX_WAVES);
    for (int p = 1; p < passes && nw < MERGE_MAX_WAVES; p *= 2) nw *= 2;
    hipLaunchKernelGGL((tree_merge_kernel<D, G>), dim3(merge_blocks(a.n_groups)), dim3(64 * nw), 0, st, a);
    return hipGetLastError();
}

template <int D>
static hipError_t launch_d(const TreeArgs& a, hipStream_t st) {
    switch (a.n_q / a.n_kv) {
        case 1: return launch_dg<D, 1>(a, st);
        case 2: return launch_dg<D, 2>(a, st);
        case 4: return launch_dg<D, 4>(a, st);
        case 8: return launch_dg<D, 8>(a, st);
        case 16: return launch_dg<D, 16>(a, st);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_tree_attention(const TreeArgs& a, hipStream_t st) {
    if (a.n_items <= 0 || a.n_workers <= 0) return hipSuccess;
    if (a.n_team < 0 || a.n_team > a.n_workers) return hipErrorInvalidValue;
    if (a.d == 128) return launch_d<128>(a, st);
    if (a.d == 64) return launch_d<64>(a, st);
    return hipErrorInvalidValue;
}

}  // namespace ps
