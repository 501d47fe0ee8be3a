// The context behind the C ABI and what its source files share: error reporting, device memory, the layer stack of a step.
#pragma once
#include <deque>
#include <string>

#include "planner.h"
#include "tree_plan.h"

namespace ps {

struct LayerWeights {
    bf16_t *wqkv_t = nullptr, *wo_t = nullptr, *wgu_t = nullptr, *wd_t = nullptr, *g_attn = nullptr, *g_ffn = nullptr;
    bf16_t* qk_gains = nullptr;   // [2][head_dim]: of the query heads, of the key heads
    bool qk_norm = false;         // heads are normalised
    bool ready = false;
};

struct Staging {  // pinned host buffer for one step's metadata
    void* host = nullptr;
    size_t bytes = 0;
};

// Memory of a step's four projections: the largest over them (see gemm_sizes).
struct LayerNeeds {
    size_t act_bytes, part_bytes, skfrag_bytes;
    int skcnt_n;
};

// Where the buffers of a step lie in the static scratch array; `total` may exceed the array.
struct StaticLayout {
    size_t xn, q, attn, act, x1, xmid, part, part_o, part_ml, meta, skfrag, skcnt, total;
    size_t act_bytes, part_bytes, skfrag_bytes;
    int skcnt_n;
};

struct StepMemory {
    GemmOptions gemm;      // of the layers' projections
    LayerNeeds needs;
    StaticLayout layout;
};

// Device buffers of one step besides its inputs and outputs: the library's growing workspaces (ps_step,
// ps_step_tokens) or pieces of the static scratch array (ps_step_static).
struct StepBufs {
    bf16_t *xn = nullptr, *q = nullptr, *attn = nullptr, *act = nullptr;
    float *x1 = nullptr, *xmid = nullptr, *part = nullptr, *part_o = nullptr, *part_ml = nullptr;
    size_t part_bytes = 0, act_bytes = 0;
    float* skfrag = nullptr;
    size_t skfrag_bytes = 0;
    int* skcnt = nullptr;
    int skcnt_n = 0;
    GemmOptions gemm;      // of the layer projections
    char* meta = nullptr;  // static steps only: device copy of the metadata
};

// One pass of a batch through the layer stack: where its metadata lies on the device and what surrounds it.
struct StackRun {
    const StepBufs* bufs;
    int T;
    const int32_t *positions, *slots;   // device [T]
    const AttnArgs* attn;               // work lists of the batch; queries, cache and output are those of the layer
    const TreeArgs* tree;               // not null: attention of trees, with these work lists instead
    const void* fetch_src;              // metadata that the first kernel brings over (see launch_rmsnorm), or null
    void* fetch_dst;
    size_t fetch_bytes;
    const void* x_in;
    void* x_out;
    bool out_f32;
    ps_step_stats* stats;
};

}  // namespace ps

using namespace ps;

struct ps_ctx {
    ps_model_desc desc{};
    bool host_only = false;
    int device = 0;        // current at ps_create
    uint64_t id = 0;       // of this context among all of the process: a plan of another one is refused
    hipStream_t stream = nullptr;
    std::string err;

    std::vector<LayerWeights> layers;
    float* rope_cs = nullptr;  // [max_position][d/2] (cos, sin)

    // KV pool + allocator
    bf16_t* pool = nullptr;
    int n_pool_pages = -1;
    int n_kv_slots = 0;
    size_t slot_elems = 0;  // elements per physical layer slot
    uint64_t pool_id = 0;   // counts ps_kv_alloc: plans made for an earlier pool are refused
    std::deque<int32_t> free_list;
    std::unordered_map<int64_t, std::vector<int32_t>> owned;
    std::vector<uint8_t> page_seen;

    // workspaces
    int cap_tokens = 0;
    bf16_t *ws_xn = nullptr, *ws_q = nullptr, *ws_attn = nullptr, *ws_act = nullptr;
    float *ws_x1 = nullptr, *ws_xmid = nullptr;
    // model head (ps_init_head): embedding table, final gain, repacked output matrix; its workspaces
    bf16_t *embedding = nullptr, *g_final = nullptr, *wout_t = nullptr;
    int vocab = 0;
    bool head_ready = false;
    bf16_t* ws_embed = nullptr;   // [cap_tokens][hidden] bf16: embedding rows of the step's tokens
    float* ws_final = nullptr;    // [cap_tokens][hidden] fp32: output of the last layer
    float* ws_logits = nullptr;   // fp32 partials of the output projection, [splits][n_seqs][vocab]
    size_t logits_bytes = 0;
    int32_t* ws_next = nullptr;   // [cap] greedy tokens when the caller passes none
    int next_cap = 0;
    void* ws_pick = nullptr;      // see launch_pick: of fixed size, so that the call never allocates
    hipEvent_t ev_head[4] = {nullptr, nullptr, nullptr, nullptr};
    float* ws_part = nullptr;  // fp32 GEMM partials [splits][T][N], shared by the three projections
    size_t part_bytes = 0;
    size_t act_bytes = 0;
    float *part_o = nullptr, *part_ml = nullptr;
    int cap_part_slots = 0;
    // tiled GEMM: parked accumulators of partial K runs and one counter per tile (zero between launches)
    float* ws_skfrag = nullptr;
    size_t skfrag_bytes = 0;
    int* ws_skcnt = nullptr;
    int skcnt_n = 0;
    // Device copies of the staging ring (same 8 slots).  The copy of step n+1's metadata runs on
    // copy_stream while step n's kernels execute; the main stream only waits for the slot's event.
    char* dev_meta = nullptr;
    size_t dev_meta_slot = 0;  // bytes per slot
    hipStream_t copy_stream = nullptr;
    hipEvent_t meta_ready[8] = {};
    // Ring of 8 pinned buffers in two halves.  One event per half, recorded after the half's last
    // copy has been enqueued, tells when all four buffers of that half may be overwritten: one
    // event record per four steps instead of one per step.
    Staging staging[8];
    hipEvent_t half_done[2] = {nullptr, nullptr};
    bool half_pending[2] = {false, false};
    int staging_next = 0;

    // options / debug
    int opt_attn_workers = 0;
    int opt_attn_teams = 0;
    int opt_attn_prefill_weight = 22;
    int worker_slots = 2048;   // eight to a compute unit; without a device those of a whole MI355X
    int opt_gemm_split_k = 0;
    int opt_gemm_tile = 0;
    int opt_gemm_whole_tiles = 0;
    int opt_gemm_wreg = 0;
    bool opt_poison = false;
    int opt_only_layer = -1;
    bool opt_out_f32 = false;
    int tap_layer = -1;
    ps_taps taps{};

    // optional event pairs around every attention launch (see ps_attention_times)
    int opt_time_attention = 0;   // 0 = off, N = bracket the attention launch of every Nth step
    int64_t step_counter = 0;
    std::vector<hipEvent_t> attn_ev;  // ring of 2 * ATTN_EV_PAIRS events
    int attn_ev_count = 0;            // pairs recorded since the last ps_attention_times

    // ps_step_static: this device's copy of the scratch array, a pinned ring for the metadata (allocated by ps_create)
    unsigned char* static_scratch = nullptr;
    char* static_host = nullptr;
    hipEvent_t static_ev[4] = {nullptr, nullptr, nullptr, nullptr};
    bool static_pending[4] = {false, false, false, false};
    int static_next = 0;

    // optional event pairs around the four projection launches of a layer (see ps_gemm_times)
    int opt_time_gemm = 0;            // 0 = off, N = bracket them in every Nth step
    std::vector<hipEvent_t> gemm_ev;  // ring of 8 * GEMM_EV_RECS events: record r holds pairs (qkv, o, gate/up, down)
    int gemm_ev_count = 0;            // records (one per layer of a timed step) since the last ps_gemm_times

    hipEvent_t ev[PS_N_STAGES * 2 + 2] = {};
    bool have_events = false;
    StepPlan plan;
    StepMemory memory{};   // goes with it
};

namespace ps {

ps_status fail(ps_ctx* c, ps_status s, const std::string& msg);
ps_status hip_fail(ps_ctx* c, hipError_t e, const char* what);
#define HIP_TRY(c, call)                                   \
    do {                                                   \
        hipError_t e__ = (call);                           \
        if (e__ != hipSuccess) return hip_fail(c, e__, #call); \
    } while (0)

template <typename T>
ps_status dev_alloc(ps_ctx* c, T** p, size_t bytes, const char* what) {
    *p = nullptr;
    if (bytes == 0) return PS_OK;
    hipError_t e = hipMalloc(reinterpret_cast<void**>(p), bytes);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        *p = nullptr;
        return fail(c, PS_ENOMEM, std::string("device allocation failed for ") + what + " (" + std::to_string(bytes) + " bytes): " + hipGetErrorString(e));
    }
    return PS_OK;
}
template <typename T>
void dev_free(T*& p) {
    if (p) (void)hipFree(p);
    p = nullptr;
}

inline int qkv_cols(const ps_model_desc& d) { return (d.n_q_heads + 2 * d.n_kv_heads) * d.head_dim; }
inline size_t align16(size_t x) { return (x + 15) & ~(size_t)15; }

PlanConfig plan_config(const ps_ctx* c);
GemmOptions gemm_options(const ps_ctx* c);
GemmOptions head_options(const ps_ctx* c);
LayerNeeds layer_needs(const ps_ctx* c, int T, const GemmOptions& o);
ps_status ensure_workspaces(ps_ctx* c, int T, int n_part_slots, int head_rows, const LayerNeeds& needs, const GemmOptions& o);
ps_status ensure_logits(ps_ctx* c, size_t bytes);
void free_workspaces(ps_ctx* c);
StepBufs workspace_bufs(ps_ctx* c, const GemmOptions& o);
ps_status run_stack(ps_ctx* c, const StackRun& r);
ps_status poison(ps_ctx* c, const StepBufs& W, int T, int n_part_slots);
void set_work_lists(const StepPlan& p, const ps_model_desc& d, AttnArgs* a);

}  // namespace ps
