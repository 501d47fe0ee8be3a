#include "tree_plan.h"

#include <algorithm>

namespace ps {

static inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// What a team takes for a pair of pages, in units of a third of what HBM takes to bring it to one of 256 compute units (0.7 us), by
// the tiles of its query block.  Trees of one, six, 16 and 48 nodes side by side, us: 71, with 3 for all 72, with 3, 5 and 8 139 (70B
// heads 87, 93 and 96); 24 trees of 16 beside two of 200: 80, 86 and 85.
static int pair_weight(int tiles) { return tiles <= 4 ? 3 : tiles <= 8 ? 4 : 5; }

// What a run takes besides its pairs, in pairs: to begin and to leave its rows (queries, page numbers and the first pages arrive, partials go),
// and for each pair with a mask.  Measured as the ends of the workers: those of three runs ended half as late again as those of one when only
// pairs were counted (126 us to 85 at 64-node trees of 64 heads).  START from 3 to 8 gives the same time to within 2%.
constexpr int START = 4, MASKED = 2;
constexpr int SHORT = 4;   // no cut leaves a run of fewer pairs

constexpr int GANG = 4;   // query blocks that read the same pages at the same time, at most

// The work list of the tree attention kernel, in the form that build_attention_plan gives a step's (AttnPlan): every (sequence, KV
// head, query block) is a stream of page pairs; streams one after another are cut into runs of equal weight, one per worker, so
// that all workers end together; a stream that was cut leaves partials and merge groups.
//
// The query blocks of a sequence hold the same number of tiles, to within one.  Up to GANG of them form a gang: they read the same
// pages, so they are cut at the same places and run side by side on neighbouring blocks of one XCD, where the first to ask for a
// page brings it into the L2 that serves the others.  Workers are therefore dealt out by gang size: streaming wavefronts for
// single-tile blocks, teams in units of one, two, three and four for the gangs.
static void build_tree_attention_plan(const PlanConfig& cfg, TreePlan& plan) {
    plan.items.clear();
    plan.groups.clear();
    plan.worker_begin.assign(1, 0);
    plan.n_partial_slots = plan.n_partial_items = plan.n_team_workers = 0;
    plan.two_blocks_per_cu = false;
    const int TQ = 16 / cfg.group, max_tiles = cfg.prefill_tokens / TQ;

    struct Stream { int seq, q0, qb, blocks, qn, np, w, free; };   // `blocks` query blocks of qb tokens from token q0 on, qn tokens in all; pages; pairs before the masks
    std::vector<Stream> pool[GANG + 1];                      // [0]: streaming wavefronts
    int64_t units[GANG + 1] = {}, pairs_team = 0, pairs_wave = 0;
    for (int s = 0; s < plan.n_seqs; s++) {
        const SeqInfo& sq = plan.seqs[s];
        const int tiles = ceil_div(sq.n_new, TQ), blocks = ceil_div(tiles, max_tiles), qb = ceil_div(tiles, blocks) * TQ;
        const int gangs = ceil_div(ceil_div(sq.n_new, qb), GANG), per_gang = ceil_div(ceil_div(sq.n_new, qb), gangs);
        for (int q0 = 0; q0 < sq.n_new; q0 += per_gang * qb) {
            const int qn = std::min(per_gang * qb, sq.n_new - q0), n = ceil_div(qn, qb), c = tiles == 1 ? 0 : n;
            const Stream st{s, q0, qb, n, qn, ceil_div(sq.kv_len - sq.n_new + q0 + qn, PS_PAGE_SIZE), c == 0 ? 1 : pair_weight(ceil_div(std::min(qb, qn), TQ)), (sq.kv_len - sq.n_new + q0) / 32};
            pool[c].push_back(st);
            const int64_t pairs = (int64_t)ceil_div(st.np, 2) * cfg.n_kv_heads;
            units[c] += (pairs + (int64_t)cfg.n_kv_heads * (START + MASKED * (ceil_div(st.np, 2) - st.free))) * st.w;
            (c == 0 ? pairs_wave : pairs_team) += pairs * n;
        }
    }
    if (pairs_team + pairs_wave == 0) return;

    // Blocks with teams: one to a compute unit, two where the runs are long enough (24 pairs a unit): twice the workers leave twice the partials.  One
    // everywhere: 16 trees of 64 nodes 64 -> 75 us at 8B heads, 104 -> 125 at 70B; two everywhere: four trees of eight 18 -> 21 and 21 -> 27.
    // Streaming wavefronts alone keep HBM busy from 13/16 of one block to a unit on, and leave fewer partials: single nodes behind 512 to 4096 tokens,
    // 8, 32 and 128 sequences, 18.5, 46 and 190 us, with all units 19.8, 47 and 193; behind 100 to 700 tokens, 8 and 128 sequences, 13.7 and 45 for 13.7 and 46.
    const int cus = std::max(8, cfg.compute_units), places = std::max(2 * cus, cfg.block_slots);
    int64_t team_units = 0;
    for (int c = 1; c <= GANG; c++) team_units += units[c] * c;
    int n_team = 0, n_wave = 0, workers[GANG + 1] = {};
    if (cfg.n_workers > 0) {
        n_team = pairs_team ? cfg.n_workers : 0;
        n_wave = pairs_wave ? cfg.n_workers : 0;
    } else if (!pairs_team) {
        n_wave = 4 * (13 * cus / 16);
    } else {
        const int blocks = pairs_team + pairs_wave / 4 < 24 * (int64_t)cus ? cus : places;
        n_team = blocks;
        if (pairs_wave) {
            // a stream's pair costs its block what HBM takes for it; every XCD gets the same number of either kind: whole eighths
            n_team = (int)(blocks * ((double)team_units / ((double)team_units + 3.0 * pairs_wave)) + 4) / 8 * 8;
            n_team = std::min(std::max(8, n_team), blocks - 8);
            n_wave = 4 * (blocks - n_team);
        }
    }
    // in proportion to the work, in whole gangs, no run shorter than some four pairs (eight single nodes 18.4 us; two pairs the same, eight 19.6)
    for (int c = 1, left = n_team; c <= GANG; c++) {
        if (!units[c]) continue;
        int64_t pairs = 0;
        for (const Stream& st : pool[c]) pairs += (int64_t)ceil_div(st.np, 2) * cfg.n_kv_heads;
        int n = (int)((double)n_team * (double)(units[c] * c) / (double)team_units / c + 0.5);
        n = std::min(n, left / c);
        workers[c] = (int)std::max<int64_t>(1, std::min<int64_t>(n, pairs / 4));
        left = std::max(0, left - workers[c] * c);
    }
    if (n_wave) workers[0] = (int)std::max<int64_t>(1, std::min<int64_t>(n_wave, pairs_wave / 4));

    struct Run { int worker, stream, head, pair, pairs, split; };
    std::vector<Run> runs;
    std::vector<int> slot;   // first partial slot of a (stream, head) and query block, -1: not cut
    for (int k = 0; k <= GANG; k++) {
        const int c = k < GANG ? k + 1 : 0;   // teams first
        const std::vector<Stream>& streams = pool[c];
        if (streams.empty()) continue;
        const int n = workers[c], width = std::max(1, c), base = (int)plan.worker_begin.size() - 1;
        // Worker w ends where the cumulative weight reaches (w + 1) / n of it, to within SHORT pairs, so rounding never accumulates.  KV head
        // by head: the contiguous share of an XCD streams whole heads.
        int64_t total = units[c];
        for (int i = 1; i < n; i++) total += START * streams[(size_t)i * streams.size() / n].w;   // of the runs that begin at a cut
        const int64_t part = total / n, rest = total % n;
        auto boundary = [&](int w) { return part * (w + 1) + rest * (w + 1) / n; };
        runs.clear();
        slot.assign(streams.size() * cfg.n_kv_heads * width, -1);
        int w = 0;
        int64_t done = 0;
        for (int h = 0; h < cfg.n_kv_heads; h++)
            for (size_t i = 0; i < streams.size(); i++) {
                const Stream& st = streams[i];
                const int n_pairs = ceil_div(st.np, 2);
                int pair = 0, splits = 0;
                while (pair < n_pairs) {
                    const bool used = !runs.empty() && runs.back().worker == w;
                    const int64_t left = (w + 1 < n ? boundary(w) : INT64_MAX / 2) - done;
                    int take = (int)std::min<int64_t>(n_pairs - pair, left / st.w - START);
                    if (take < std::min(SHORT, n_pairs - pair) && used) { w++; continue; }   // not worth beginning
                    if (take < n_pairs - pair && n_pairs - pair - take < SHORT) take = n_pairs - pair;   // nor what would remain
                    take = std::max(take, std::min(SHORT, n_pairs - pair));
                    runs.push_back(Run{w, (int)i, h, pair, take, splits++});
                    pair += take;
                    done += (int64_t)(take + START) * st.w;
                    if (pair == n_pairs) done += (int64_t)MASKED * (n_pairs - st.free) * st.w;
                    if (w + 1 < n && done >= boundary(w)) w++;
                }
                if (splits == 1) continue;
                for (int b = 0; b < st.blocks; b++) {
                    const int q0 = st.q0 + b * st.qb, qn = std::min(st.qb, st.q0 + st.qn - q0), tiles = ceil_div(qn, TQ), first = plan.n_partial_slots;
                    slot[(h * streams.size() + i) * width + b] = first;
                    for (int t = 0; t < tiles; t++)
                        plan.groups.push_back(MergeGroup{plan.seqs[st.seq].tok0 + q0 + t * TQ, std::min(TQ, qn - t * TQ), h, first + t, splits, tiles, 0, 0});
                    plan.n_partial_slots += splits * tiles;
                    plan.n_partial_items += splits;
                }
            }
        size_t at = 0;
        for (int v = 0; v < n; v++) {
            size_t end = at;
            while (end < runs.size() && runs[end].worker == v) end++;
            for (int b = 0; b < width; b++) {
                for (size_t r = at; r < end; r++) {
                    const Run& run = runs[r];
                    const Stream& st = streams[run.stream];
                    const SeqInfo& sq = plan.seqs[st.seq];
                    const int q0 = st.q0 + b * st.qb, qn = std::min(st.qb, st.q0 + st.qn - q0), tiles = ceil_div(qn, TQ);
                    const int s0 = slot[(run.head * streams.size() + run.stream) * width + b], p0 = 2 * run.pair;
                    plan.items.push_back(AttnItem{st.seq, run.head, q0, qn, p0, std::min(st.np, p0 + 2 * run.pairs), s0 < 0 ? -1 : s0 + run.split * tiles,
                                                  base + v * width + b, sq.tok0 + q0, sq.kv_len - sq.n_new + q0, sq.page_off, plan.pages[sq.page_off + p0],
                                                  plan.pages[sq.page_off + std::min(p0 + 1, st.np - 1)], -1, 0, 0});
                }
                plan.worker_begin.push_back((int32_t)plan.items.size());
            }
            at = end;
        }
        if (c > 0) plan.n_team_workers += n * width;
    }
}

ps_status build_tree_plan(const ps_seq* seqs, int n_seqs, const int32_t* parents, const PlanConfig& cfg, TreePlan& plan, std::string& err) {
    build_indices(seqs, n_seqs, plan);
    plan.masks.clear();
    plan.row_seq.resize(plan.n_tokens);
    plan.row_prev.resize(plan.n_tokens);
    struct Mask { int64_t at; int32_t words, pair; };
    std::vector<Mask> mask(n_seqs, Mask{-1, 0, 0});
    for (int s = 0; s < n_seqs; s++) {
        const int n = seqs[s].n_new, t0 = plan.cu_seqlens[s], prefix = seqs[s].kv_len - n;
        const int32_t* par = parents ? parents + t0 : nullptr;
        bool chain = true;
        for (int i = 0; i < n; i++) {
            const int p = par ? par[i] : i - 1;
            const auto who = [&]() { return "seq " + std::to_string(s) + " (req " + std::to_string(seqs[s].req_id) + "), node " + std::to_string(i) + ": "; };
            if (p != PS_TREE_PAD && (p < -1 || p >= i)) {
                err = who() + "parent " + std::to_string(p) + " is neither an earlier node nor -1 (the cached prefix) nor PS_TREE_PAD";
                return PS_EINVAL;
            }
            if (p >= 0 && par && par[p] == PS_TREE_PAD) { err = who() + "its parent is padding"; return PS_EINVAL; }
            chain = chain && p == i - 1;
            plan.row_seq[t0 + i] = s;
            plan.row_prev[t0 + i] = p < 0 ? -1 : t0 + p;
            plan.positions[t0 + i] = p < 0 ? prefix : plan.positions[t0 + p] + 1;
        }
        if (chain) continue;
        if (n > PS_TREE_MAX_NODES) {
            err = "seq " + std::to_string(s) + " (req " + std::to_string(seqs[s].req_id) + "): more than " + std::to_string(PS_TREE_MAX_NODES) + " nodes in a tree";
            return PS_ERANGE;
        }
        Mask& m = mask[s];
        m.pair = prefix / 32;
        m.words = (prefix + n - 1) / 32 - m.pair + 1;
        m.at = (int64_t)plan.masks.size();
        if (m.at + (int64_t)n * m.words > INT32_MAX) { err = "the trees of the batch need more than 2^31 mask words"; return PS_ERANGE; }
        plan.masks.resize(plan.masks.size() + (size_t)n * m.words, 0u);
        uint32_t* w = plan.masks.data() + m.at;
        for (int i = 0; i < n; i++, w += m.words) {
            if (par[i] == PS_TREE_PAD) continue;
            if (par[i] >= 0) std::copy(plan.masks.data() + m.at + (size_t)par[i] * m.words, plan.masks.data() + m.at + (size_t)(par[i] + 1) * m.words, w);
            else w[0] = (1u << (prefix & 31)) - 1u;   // what the first word holds of the prefix
            const int p = prefix + i;
            w[(p >> 5) - m.pair] |= 1u << (p & 31);
        }
    }
    build_tree_attention_plan(cfg, plan);
    for (AttnItem& it : plan.items) {
        const Mask& m = mask[it.seq];
        it.mask_at = m.at < 0 ? -1 : (int32_t)(m.at + (int64_t)it.q_tok0 * m.words);
        it.mask_words = m.words;
        it.mask_pair = m.pair;
    }
    return PS_OK;
}

}  // namespace ps
