// Host side of a batch of token trees: validation of the parents, positions and the masks of who sees what.  No HIP calls.
#pragma once
#include "planner.h"

namespace ps {

struct TreePlan : StepPlan {
    std::vector<uint32_t> masks;     // see AttnItem; sequences whose tokens are plain chains have none
    std::vector<int32_t> row_seq;    // [T] sequence of a token
    std::vector<int32_t> row_prev;   // [T] row of its parent, -1: none
};

// Fills plan for the batch; parents as in ps_tree_plan (null: chains).  The batch is valid (validate_batch), cfg.prefill_tokens set.
// PS_EINVAL / PS_ERANGE with a message in err for malformed parents; plan is then unspecified.
ps_status build_tree_plan(const ps_seq* seqs, int n_seqs, const int32_t* parents, const PlanConfig& cfg, TreePlan& plan, std::string& err);

}  // namespace ps
