// The cache rows of an accepted branch become the next positions of the prefix, in all KV slots: rows prefix + node[k] move to
// prefix + first + k.  A node's place is never before the place it moves to, so rows are moved in passes of KEEP_TILE places in ascending
// order, each read whole before it is written: no pass overwrites what a later one reads.
//
// A block is a chain of trips to memory (its list, the page numbers, the rows), so it looks all of a pass up at once, a thread a row, and sends
// the rows' loads together, at addresses in bounds for every lane.  Keys of a row lie in pieces of 16 bytes; values lie by quads of positions
// (v_elem_offset), 2 bytes a row: passes begin at pages, so a thread fills whole quads and writes 8 bytes where it read 2 four times.
// What bounds it then is lines, not bytes: a row's 16-byte key pieces and 2-byte values lie in every line of its page, so branches across 64
// nodes read most of those nodes' pages.  64 branches of 64-node trees, 8 kv heads of 128, 4 slots: 16 us, 2.7 us for one (two launches of 30 us
// with a look-up, a load and a wait for each row).
#include "ps_device.h"

namespace ps {

constexpr int KEEP_TILE = 32;      // places of a pass: two pages
constexpr int KEEP_ARGS = 960;     // words of lists in a launch's arguments (3.75 of the 4 KiB that they may take)
constexpr int KEEP_REC = 4;        // words of a sequence in front of the nodes

struct KeepArgs {
    bf16_t* pool;
    size_t slot_elems;
    const SeqInfo* seqs;
    const int32_t* pages;
    int n_kv, n_seqs;
    int32_t w[KEEP_ARGS];          // (sequence, first, its lowest node, begin) of each and of an end; then the nodes above the lowest, two to a word
};

// One block of 2 D threads per (sequence, kv head, KV slot).  A pass sits in registers between its reads and its writes: of the values, thread t
// moves one dimension of the 16 places of page t / D; of the keys the 16 bytes t % (D/8) of the places t / (D/8) and 16 further on.
template <int D>
__global__ __launch_bounds__(2 * D) void tree_keep_kernel(KeepArgs a) {
    constexpr int PIECES = D / 8;
    __shared__ size_t chunk_of[KEEP_TILE], to[KEEP_TILE / 16];   // element offsets of the places' source chunks, of the pass's pages
    __shared__ int tok_of[KEEP_TILE];                            // and the rows in the chunks
    const int32_t* rec = a.w + KEEP_REC * blockIdx.x;
    const int seq = rec[0], first = rec[1], low = rec[2], begin = rec[3], end = rec[3 + KEEP_REC];
    const uint16_t* node = reinterpret_cast<const uint16_t*>(a.w + KEEP_REC * (a.n_seqs + 1)) + begin;
    const SeqInfo s = a.seqs[seq];
    const int prefix = s.kv_len - s.n_new, n = end - begin, dst = prefix + first;
    const size_t page_elems = (size_t)a.n_kv * 2 * 16 * D;
    bf16_t* const base = a.pool + blockIdx.z * a.slot_elems + (size_t)blockIdx.y * 2 * 16 * D;
    const int32_t* const pages = a.pages + s.page_off;
    const int t = threadIdx.x, piece = (t % PIECES) * 8, row = t / PIECES, half = __builtin_amdgcn_readfirstlane(t / D), lane = t % D;
    const int v_at = 16 * D + (lane >> 5) * 512 + (lane & 31) * 4;   // + (tok >> 2) * 128 + (tok & 3): of the dimension whose place is the lane-th
    for (int p0 = dst & ~15; p0 < dst + n; p0 += KEEP_TILE) {        // places p0 + j, of which [dst, dst + n) are filled
        if (t < KEEP_TILE) {
            const int k = min(max(p0 + t - dst, 0), n - 1), p = prefix + low + node[k];
            const size_t page = pages[p >> 4];
            chunk_of[t] = page * page_elems;
            tok_of[t] = p & 15;
        } else if (t < KEEP_TILE + KEEP_TILE / 16) {
            const size_t page = pages[min((p0 >> 4) + t - KEEP_TILE, (dst + n - 1) >> 4)];
            to[t - KEEP_TILE] = page * page_elems;
        }
        __syncthreads();
        int val[16] = {};
        const uint4 key0 = *reinterpret_cast<const uint4*>(base + chunk_of[row] + k_elem_offset(tok_of[row], piece));
        const uint4 key1 = *reinterpret_cast<const uint4*>(base + chunk_of[16 + row] + k_elem_offset(tok_of[16 + row], piece));
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            if (p0 + 16 * half + i + 3 >= dst && p0 + 16 * half + i < dst + n) {   // some of the quad are filled
#pragma unroll
                for (int e = i; e < i + 4; e++) {
                    const int tok = tok_of[16 * half + e];
                    val[e] = base[chunk_of[16 * half + e] + v_at + (tok >> 2) * 128 + (tok & 3)];
                }
            }
#pragma unroll
        for (int i = 0; i < 16; i++) hold(val[i]);
        __syncthreads();   // all of the pass has been read
        auto filled = [&](int p) { return p >= dst && p < dst + n; };
        if (filled(p0 + row)) *reinterpret_cast<uint4*>(base + to[0] + k_elem_offset(row, piece)) = key0;
        if (filled(p0 + 16 + row)) *reinterpret_cast<uint4*>(base + to[1] + k_elem_offset(row, piece)) = key1;
        bf16_t* const out = base + to[half] + v_at;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int p = p0 + 16 * half + i;
            if (filled(p) && filled(p + 3)) {
                *reinterpret_cast<uint2*>(out + i * 32) = uint2{(uint32_t)(val[i] | val[i + 1] << 16), (uint32_t)(val[i + 2] | val[i + 3] << 16)};
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (filled(p + e)) out[i * 32 + e] = (bf16_t)val[i + e];
            }
        }
        __syncthreads();   // and written before the next is looked up
    }
}

hipError_t launch_tree_keep(const KeepList& l, bf16_t* pool, size_t slot_elems, int n_slots, const SeqInfo* seqs, const int32_t* pages, int n_kv, int d,
                            hipStream_t st) {
    if ((d != 64 && d != 128) || n_slots < 1 || n_slots > 65535 || n_kv > 65535) return hipErrorInvalidValue;
    KeepArgs a;
    a.pool = pool; a.slot_elems = slot_elems; a.seqs = seqs; a.pages = pages; a.n_kv = n_kv;
    // Whole sequences into a launch while they fit.  One that fits no launch, or whose nodes lie too far apart for 16 bits, goes in pieces, each
    // after the one before it.
    int i = 0, done = 0;   // next sequence, its rows that have been handed out
    while (i < l.n_seqs) {
        constexpr int MOST = KEEP_ARGS / KEEP_REC;
        int n_seqs = 0, n_nodes = 0;
        int32_t rec[MOST][KEEP_REC];
        uint16_t nodes[2 * KEEP_ARGS];
        while (i < l.n_seqs && n_seqs < MOST) {
            const int room = 2 * (KEEP_ARGS - KEEP_REC * (n_seqs + 2)) - n_nodes;
            const int32_t* const node = l.node + l.begin[i] + done;
            const int have = l.begin[i + 1] - l.begin[i] - done;
            if (room < 1 || (have > room && n_seqs > 0)) break;   // rather at the start of the next launch
            int take = 0;
            while (take < have && take < room && node[take] - node[0] < 65536) {
                nodes[n_nodes + take] = (uint16_t)(node[take] - node[0]);
                take++;
            }
            if (take > 0) {
                rec[n_seqs][0] = l.seq[i]; rec[n_seqs][1] = l.first[i] + done; rec[n_seqs][2] = node[0]; rec[n_seqs][3] = n_nodes;
                n_nodes += take;
                n_seqs++;
            }
            if (take < have) { done += take; break; }
            i++;
            done = 0;
        }
        if (n_nodes == 0) continue;
        a.n_seqs = n_seqs;
        for (int k = 0; k < n_seqs; k++)
            for (int e = 0; e < KEEP_REC; e++) a.w[KEEP_REC * k + e] = rec[k][e];
        for (int e = 0; e < KEEP_REC; e++) a.w[KEEP_REC * n_seqs + e] = n_nodes;
        int32_t* const words = a.w + KEEP_REC * (n_seqs + 1);
        nodes[n_nodes] = 0;
        for (int k = 0; k < n_nodes; k += 2) words[k / 2] = (int32_t)((uint32_t)nodes[k] | (uint32_t)nodes[k + 1] << 16);
        const dim3 grid(n_seqs, n_kv, n_slots);
        if (d == 64) hipLaunchKernelGGL(tree_keep_kernel<64>, grid, dim3(128), 0, st, a);
        else hipLaunchKernelGGL(tree_keep_kernel<128>, grid, dim3(256), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ps
