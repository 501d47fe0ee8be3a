#include "tree_plan.h"

#include <algorithm>

namespace ps {

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
    build_attention_plan(cfg, plan);
    for (AttnItem& it : plan.items) {
        const Mask& m = mask[it.seq];
        it.mask_at = m.at < 0 ? -1 : (int32_t)(m.at + (int64_t)it.q_tok0 * m.words);
        it.mask_words = m.words;
        it.mask_pair = m.pair;
    }
    return PS_OK;
}

}  // namespace ps
