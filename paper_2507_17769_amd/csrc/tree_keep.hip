// The cache rows of an accepted branch become the next positions of the prefix, in all KV slots: rows prefix + node[k] move to
// prefix + first + k.  A node's place is never before the place it moves to, so rows are moved in passes of KEEP_TILE in ascending
// order, each read whole before it is written: no pass overwrites what a later one reads.
#include "ps_device.h"

namespace ps {

constexpr int KEEP_TILE = 32;      // rows of a pass
constexpr int KEEP_ARGS = 800;     // words of lists in a launch's arguments (3.2 of the 4 KiB that they may take)

struct KeepArgs {
    bf16_t* pool;
    size_t slot_elems;
    const SeqInfo* seqs;
    const int32_t* pages;
    int n_kv, n_seqs;
    int32_t w[KEEP_ARGS];          // [3 n_seqs + 1]: (sequence, first, begin) of each, the end of the last; then the nodes
};

// One block of D threads per (sequence, kv head, KV slot).  A pass sits in registers between its reads and its writes: thread t moves
// value t of every row, and of the keys the 16 bytes t % (D/8) of the rows t / (D/8), + 8, ...
template <int D>
__global__ __launch_bounds__(D) void tree_keep_kernel(KeepArgs a) {
    constexpr int GROUPS = D / 8, ROWS = D / GROUPS, KEYS = KEEP_TILE / ROWS;
    const int32_t* rec = a.w + 3 * blockIdx.x;
    const int seq = rec[0], first = rec[1], begin = rec[2], end = rec[5];
    const int32_t* node = a.w + 3 * a.n_seqs + 3 + begin;
    const SeqInfo s = a.seqs[seq];
    const int prefix = s.kv_len - s.n_new, n = end - begin;
    bf16_t* const base = a.pool + blockIdx.z * a.slot_elems + (size_t)blockIdx.y * 2 * 16 * D;
    auto chunk = [&](int p) { return base + (size_t)a.pages[s.page_off + (p >> 4)] * a.n_kv * 2 * 16 * D; };
    const int t = threadIdx.x, kg = (t % GROUPS) * 8, kr = t / GROUPS;
    for (int k0 = 0; k0 < n; k0 += KEEP_TILE) {
        uint4 key[KEYS];
        bf16_t val[KEEP_TILE];
#pragma unroll
        for (int i = 0; i < KEYS; i++) {
            const int k = k0 + i * ROWS + kr;
            if (k < n) {
                const int p = prefix + node[k];
                key[i] = *reinterpret_cast<const uint4*>(chunk(p) + k_elem_offset(p & 15, kg));
            }
        }
#pragma unroll
        for (int i = 0; i < KEEP_TILE; i++)
            if (k0 + i < n) {
                const int p = prefix + node[k0 + i];
                val[i] = chunk(p)[16 * D + v_elem_offset(p & 15, t)];
            }
        __syncthreads();   // all of the pass has been read
#pragma unroll
        for (int i = 0; i < KEYS; i++) {
            const int k = k0 + i * ROWS + kr;
            if (k < n) {
                const int p = prefix + first + k;
                *reinterpret_cast<uint4*>(chunk(p) + k_elem_offset(p & 15, kg)) = key[i];
            }
        }
#pragma unroll
        for (int i = 0; i < KEEP_TILE; i++)
            if (k0 + i < n) {
                const int p = prefix + first + k0 + i;
                chunk(p)[16 * D + v_elem_offset(p & 15, t)] = val[i];
            }
        __syncthreads();   // and written before the next is read: a later row is never among them, but a line may be
    }
}

hipError_t launch_tree_keep(const KeepList& l, bf16_t* pool, size_t slot_elems, int n_slots, const SeqInfo* seqs, const int32_t* pages, int n_kv, int d,
                            hipStream_t st) {
    if ((d != 64 && d != 128) || n_slots < 1 || n_slots > 65535 || n_kv > 65535) return hipErrorInvalidValue;
    KeepArgs a;
    a.pool = pool; a.slot_elems = slot_elems; a.seqs = seqs; a.pages = pages; a.n_kv = n_kv;
    // whole sequences into a launch while they fit; one that fits no launch goes in pieces, launch after launch
    int i = 0, done = 0;   // next sequence, its rows that have been handed out
    while (i < l.n_seqs) {
        int n_seqs = 0, n_nodes = 0;
        int32_t rec[KEEP_ARGS / 4][3], nodes[KEEP_ARGS];
        while (i < l.n_seqs && n_seqs < KEEP_ARGS / 4 && 3 * (n_seqs + 2) + n_nodes < KEEP_ARGS) {
            const int have = l.begin[i + 1] - l.begin[i] - done, room = KEEP_ARGS - 3 * (n_seqs + 2) - n_nodes;
            if (have > room && n_seqs > 0) break;   // rather at the start of the next launch
            const int take = have < room ? have : room;
            rec[n_seqs][0] = l.seq[i]; rec[n_seqs][1] = l.first[i] + done; rec[n_seqs][2] = n_nodes;
            for (int k = 0; k < take; k++) nodes[n_nodes + k] = l.node[l.begin[i] + done + k];
            n_nodes += take;
            n_seqs++;
            if (take < have) { done += take; break; }
            i++;
            done = 0;
        }
        if (n_nodes == 0) continue;
        a.n_seqs = n_seqs;
        for (int k = 0; k < n_seqs; k++) { a.w[3 * k] = rec[k][0]; a.w[3 * k + 1] = rec[k][1]; a.w[3 * k + 2] = rec[k][2]; }
        a.w[3 * n_seqs] = a.w[3 * n_seqs + 1] = 0;
        a.w[3 * n_seqs + 2] = n_nodes;
        for (int k = 0; k < n_nodes; k++) a.w[3 * n_seqs + 3 + k] = nodes[k];
        const dim3 grid(n_seqs, n_kv, n_slots);
        if (d == 64) hipLaunchKernelGGL(tree_keep_kernel<64>, grid, dim3(64), 0, st, a);
        else hipLaunchKernelGGL(tree_keep_kernel<128>, grid, dim3(128), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ps
