// Checks of the plan of token trees, compiled for the host by test_host_tree.py: over random batches, every work item's mask words lie
// within the masks and say for each token and position of the item what the parents say, positions are prefix + depth, the items cover
// every position that a token sees exactly once, and malformed parents are refused.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "tree_plan.h"

using namespace ps;

#define REQUIRE(cond)                                  \
    if (!(cond)) {                                     \
        printf("%s: case %d line %d\n", #cond, n, __LINE__); \
        return 1;                                      \
    }

int main() {
    std::mt19937 rng(11);
    auto up_to = [&](int k) { return (int)(rng() % (unsigned)(k + 1)); };
    int n = 0;
    int64_t checked = 0;
    for (; n < 1500; n++) {
        PlanConfig cfg;
        cfg.n_kv_heads = 1 + up_to(2);
        cfg.group = 1 << up_to(4);
        cfg.prefill_tokens = 4 * (1 + up_to(2)) * (16 / cfg.group);
        cfg.n_workers = n % 3 == 0 ? 1 + up_to(40) : 0;
        cfg.max_position = 1 << 20;
        const int n_seqs = up_to(5);
        std::vector<ps_seq> seqs;
        std::vector<std::vector<int32_t>> tables;
        std::vector<int32_t> parents;
        std::vector<bool> bad_seen;
        for (int s = 0; s < n_seqs; s++) {
            const int q = 1 + up_to(n % 5 == 0 ? 200 : 40), prefix = up_to(n % 4 == 0 ? 3 : 300), kind = up_to(3);
            tables.emplace_back((q + prefix + 15) / 16, 0);
            seqs.push_back(ps_seq{s, q, q + prefix, nullptr, (int32_t)tables.back().size()});
            const int pad = kind == 2 ? up_to(q) : 0;
            for (int i = 0; i < q; i++) parents.push_back(kind == 0 ? i - 1 : i >= q - pad ? PS_TREE_PAD : i == 0 ? -1 : up_to(i) - 1);
        }
        int page = 0;
        for (size_t i = 0; i < seqs.size(); i++) {
            for (int32_t& p : tables[i]) p = page++;
            seqs[i].page_table = tables[i].data();
        }
        TreePlan plan;
        std::string err;
        REQUIRE(build_tree_plan(seqs.data(), n_seqs, parents.data(), cfg, plan, err) == PS_OK);
        std::vector<std::vector<std::vector<int>>> seen(n_seqs);   // [sequence][kv head] of token x position, counted
        for (int s = 0; s < n_seqs; s++) seen[s].assign(cfg.n_kv_heads, std::vector<int>((size_t)seqs[s].n_new * seqs[s].kv_len, 0));
        for (const AttnItem& it : plan.items) {
            const ps_seq& q = seqs[it.seq];
            const int prefix = q.kv_len - q.n_new, t0 = plan.cu_seqlens[it.seq];
            for (int i = 0; i < it.q_ntok; i++) {
                const int tok = it.q_tok0 + i;
                std::vector<bool> anc(q.n_new, false);
                const int par0 = parents[t0 + tok];
                if (par0 != PS_TREE_PAD)
                    for (int j = tok; j >= 0; j = parents[t0 + j]) anc[j] = true;
                for (int p = it.page_begin * 16; p < it.page_end * 16; p++) {
                    bool want = p < q.kv_len && par0 != PS_TREE_PAD && (p < prefix || anc[p - prefix]), got;
                    if (it.mask_at < 0) {
                        got = p <= it.pos0 + i;
                    } else if (p / 32 < it.mask_pair) {
                        got = true;   // no mask there: padding is taken out at the end
                        want = want || (par0 == PS_TREE_PAD && p < prefix);
                    } else {
                        REQUIRE(p / 32 - it.mask_pair < it.mask_words || p >= q.kv_len);
                        if (p / 32 - it.mask_pair >= it.mask_words) continue;
                        const int64_t w = it.mask_at + (int64_t)i * it.mask_words + p / 32 - it.mask_pair;
                        REQUIRE(w >= 0 && w < (int64_t)plan.masks.size());
                        got = plan.masks[w] >> (p & 31) & 1;
                    }
                    REQUIRE(got == want);
                    if (p < q.kv_len && got && par0 != PS_TREE_PAD) seen[it.seq][it.kv_head][(size_t)tok * q.kv_len + p]++;
                    checked++;
                }
            }
        }
        for (int s = 0; s < n_seqs; s++) {
            const int t0 = plan.cu_seqlens[s], prefix = seqs[s].kv_len - seqs[s].n_new;
            for (int i = 0; i < seqs[s].n_new; i++) {
                int depth = 0, want = parents[t0 + i] == PS_TREE_PAD ? 0 : prefix;
                for (int j = parents[t0 + i]; j >= 0; j = parents[t0 + j]) depth++;
                REQUIRE(plan.positions[t0 + i] == prefix + depth);
                REQUIRE(plan.row_seq[t0 + i] == s && plan.row_prev[t0 + i] == (parents[t0 + i] < 0 ? -1 : t0 + parents[t0 + i]));
                REQUIRE(plan.slots[t0 + i] == seqs[s].page_table[(prefix + i) / 16] * 16 + (prefix + i) % 16);
                if (want) want += depth + 1; else if (parents[t0 + i] != PS_TREE_PAD) want = depth + 1;
                for (int h = 0; h < cfg.n_kv_heads; h++) {
                    int sum = 0;
                    for (int p = 0; p < seqs[s].kv_len; p++) {
                        const int c = seen[s][h][(size_t)i * seqs[s].kv_len + p];
                        REQUIRE(c <= 1);
                        sum += c;
                    }
                    REQUIRE(sum == want);
                }
            }
        }
        // a parent that is not an earlier node, or is padding
        if (!parents.empty()) {
            const int s = up_to(n_seqs - 1), t0 = plan.cu_seqlens[s], i = up_to(seqs[s].n_new - 1);
            std::vector<int32_t> wrong = parents;
            wrong[t0 + i] = up_to(1) ? i + up_to(3) : -3 - up_to(3);
            REQUIRE(build_tree_plan(seqs.data(), n_seqs, wrong.data(), cfg, plan, err) == PS_EINVAL && !err.empty());
            if (seqs[s].n_new > 1) {
                wrong = parents;
                wrong[t0] = PS_TREE_PAD;
                wrong[t0 + 1] = 0;
                REQUIRE(build_tree_plan(seqs.data(), n_seqs, wrong.data(), cfg, plan, err) == PS_EINVAL);
            }
        }
    }
    // too many nodes in a tree, as many in a chain
    std::vector<int32_t> table(200), par(PS_TREE_MAX_NODES + 1);
    for (int i = 0; i < 200; i++) table[i] = i;
    for (size_t i = 0; i < par.size(); i++) par[i] = (int)i - 1;
    ps_seq q{1, PS_TREE_MAX_NODES + 1, PS_TREE_MAX_NODES + 20, table.data(), 200};
    PlanConfig cfg;
    cfg.max_position = 1 << 20;
    TreePlan plan;
    std::string err;
    REQUIRE(build_tree_plan(&q, 1, par.data(), cfg, plan, err) == PS_OK && plan.masks.empty());
    REQUIRE(build_tree_plan(&q, 1, nullptr, cfg, plan, err) == PS_OK && plan.masks.empty());
    par.back() = 5;
    REQUIRE(build_tree_plan(&q, 1, par.data(), cfg, plan, err) == PS_ERANGE);
    q.n_new--; q.kv_len--;
    par[PS_TREE_MAX_NODES - 1] = 5;
    REQUIRE(build_tree_plan(&q, 1, par.data(), cfg, plan, err) == PS_OK && !plan.masks.empty());
    printf("OK %lld positions\n", (long long)checked);
    return 0;
}
