// C ABI of the operators on drafted tokens: trees, normalised heads, tree attention, keeping a branch, rules on logits, and the
// step that uses them together.  See include/polystep.h for the contract of every entry point.
#include <algorithm>
#include <cstring>
#include <new>

#include "context.h"

// A batch of trees: its plan, and the plan's device side in one buffer.  Freed without its context: that may be gone.
struct ps_tree {
    const ps_ctx* ctx = nullptr;
    uint64_t ctx_id = 0, pool_id = 0;
    int device = 0;
    bool host_only = false, planned = false;
    TreePlan plan;
    TreeArgs args{};            // work lists on the device
    const int32_t *positions = nullptr, *slots = nullptr, *row_seq = nullptr, *row_prev = nullptr;   // device, [T]
    char* dev = nullptr;
    size_t dev_bytes = 0;
    float *part_o = nullptr, *part_ml = nullptr;
    int cap_part_slots = 0;
    // pinned buffers that plans and token ids travel in, two of each in turn; an event tells when one has been read
    struct Pinned {
        char* host = nullptr;
        size_t bytes = 0;
        hipEvent_t read = nullptr;
        bool pending = false;
    };
    Pinned meta[2], tokens[2];
    int next_meta = 0, next_tokens = 0;
    int32_t* dev_tokens = nullptr;
    int cap_tokens = 0;
};

namespace {

// The context's device is current while one of its calls runs.
struct OnDevice {
    int before = -1;
    explicit OnDevice(const ps_ctx* c) { enter(c->host_only ? -1 : c->device); }
    explicit OnDevice(int device) { enter(device); }
    void enter(int device) {
        int now = -1;
        if (device >= 0 && hipGetDevice(&now) == hipSuccess && now != device && hipSetDevice(device) == hipSuccess) before = now;
    }
    ~OnDevice() {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

// Nothing throws across the C boundary.
template <typename F>
ps_status guarded(ps_ctx* c, const char* name, F f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return fail(c, PS_ENOMEM, std::string(name) + ": out of host memory");
    } catch (...) {
        return fail(c, PS_EDEVICE, std::string(name) + ": unexpected failure");
    }
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Whether n rows of two tensors share memory: bytes of a row, and from one to the next.  Rows of the same distance may lie between each other's.
bool rows_meet(const void* a, int64_t row_a, int64_t step_a, const void* b, int64_t row_b, int64_t step_b, int64_t n) {
    const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a));   // of b behind a
    if (d >= (n - 1) * step_a + row_a || -d >= (n - 1) * step_b + row_b) return false;
    if (n == 1 || step_a != step_b) return true;
    const int64_t at = (d % step_a + step_a) % step_a;
    return at < row_a || at + row_b > step_a;
}

// A pinned buffer of at least `bytes` that nothing reads any more.
ps_status pinned(ps_ctx* c, ps_tree::Pinned& b, size_t bytes) {
    if (b.pending) {
        HIP_TRY(c, hipEventSynchronize(b.read));
        b.pending = false;
    }
    if (!b.read) HIP_TRY(c, hipEventCreateWithFlags(&b.read, hipEventDisableTiming));
    if (b.bytes < bytes) {
        if (b.host) (void)hipHostFree(b.host);
        b.host = nullptr;
        b.bytes = 0;
        const size_t want = align16(std::max(bytes + bytes / 2, (size_t)1 << 14));
        if (hipHostMalloc(reinterpret_cast<void**>(&b.host), want, hipHostMallocDefault) != hipSuccess) {
            (void)hipGetLastError();
            b.host = nullptr;
            return fail(c, PS_ENOMEM, "pinned buffer allocation failed");
        }
        b.bytes = want;
    }
    return PS_OK;
}
ps_status send(ps_ctx* c, ps_tree::Pinned& b, void* dev, size_t bytes) {
    HIP_TRY(c, launch_copy_bytes(b.host, dev, align16(bytes), c->stream));
    HIP_TRY(c, hipEventRecord(b.read, c->stream));
    b.pending = true;
    return PS_OK;
}

PlanConfig tree_plan_config(const ps_ctx* c) {
    PlanConfig pc = plan_config(c);
    pc.prefill_tokens = tree_tokens_per_item(pc.group);
    return pc;
}

// Common to the calls that take a planned tree.
ps_status check_tree(ps_ctx* c, const ps_tree* t, const char* name) {
    if (!t) return fail(c, PS_EINVAL, std::string(name) + ": null tree");
    if (c->host_only) return fail(c, PS_ESTATE, std::string(name) + ": host-only context");
    if (!t->planned) return fail(c, PS_ESTATE, std::string(name) + ": the tree is not planned (call ps_tree_plan)");
    if (t->ctx != c || t->ctx_id != c->id) return fail(c, PS_ESTATE, std::string(name) + ": the tree was planned for another context");
    if (!c->pool) return fail(c, PS_ESTATE, std::string(name) + ": no KV pool (call ps_kv_alloc)");
    if (t->pool_id != c->pool_id) return fail(c, PS_ESTATE, std::string(name) + ": the KV pool was replaced after ps_tree_plan");
    return PS_OK;
}
// Calls whose host side a graph would not repeat (buffers that grow, pinned memory that later calls fill again, flags of the context).
ps_status check_not_captured(ps_ctx* c, const char* name) {
    hipStreamCaptureStatus now = hipStreamCaptureStatusNone;
    const hipError_t e = hipStreamIsCapturing(c->stream, &now);
    if (e != hipSuccess) (void)hipGetLastError();   // the default stream while another one is captured
    if (e != hipSuccess || now != hipStreamCaptureStatusNone) return fail(c, PS_ESTATE, std::string(name) + ": cannot be captured into a graph");
    return PS_OK;
}
ps_status check_layer(ps_ctx* c, int32_t layer, const char* name) {
    if (layer < 0 || layer >= c->desc.n_layers) return fail(c, PS_ERANGE, std::string(name) + ": layer index out of range");
    return PS_OK;
}
bf16_t* slot_of(const ps_ctx* c, int layer) { return c->pool + (size_t)(layer % c->n_kv_slots) * c->slot_elems; }

ps_status upload(ps_ctx* c, ps_tree* t, const TreePlan& p) {
    struct Piece { const void* src; size_t bytes, at; };
    Piece pieces[] = {{p.positions.data(), p.positions.size() * 4, 0},
                      {p.slots.data(), p.slots.size() * 4, 0},
                      {p.row_seq.data(), p.row_seq.size() * 4, 0},
                      {p.row_prev.data(), p.row_prev.size() * 4, 0},
                      {p.seqs.data(), p.seqs.size() * sizeof(SeqInfo), 0},
                      {p.pages.data(), p.pages.size() * 4, 0},
                      {p.items.data(), p.items.size() * sizeof(AttnItem), 0},
                      {p.worker_begin.data(), p.worker_begin.size() * 4, 0},
                      {p.groups.data(), p.groups.size() * sizeof(MergeGroup), 0},
                      {p.masks.data(), p.masks.size() * 4, 0}};
    size_t total = 0;
    for (Piece& x : pieces) { x.at = total; total = align16(total + x.bytes); }
    ps_status st;
    if (t->dev_bytes < total) {
        HIP_TRY(c, hipStreamSynchronize(c->stream));
        dev_free(t->dev);
        t->dev_bytes = 0;
        const size_t want = align16(std::max(total + total / 2, (size_t)1 << 14));
        if ((st = dev_alloc(c, &t->dev, want, "tree plan")) != PS_OK) return st;
        t->dev_bytes = want;
    }
    if (p.n_partial_slots > t->cap_part_slots) {
        HIP_TRY(c, hipStreamSynchronize(c->stream));
        dev_free(t->part_o); dev_free(t->part_ml);
        t->cap_part_slots = 0;
        const int cap = p.n_partial_slots + p.n_partial_slots / 2 + 64;
        if ((st = dev_alloc(c, &t->part_o, (size_t)cap * 16 * c->desc.head_dim * 4, "tree attention partials")) != PS_OK) return st;
        if ((st = dev_alloc(c, &t->part_ml, (size_t)cap * 16 * 2 * 4, "tree attention partial stats")) != PS_OK) return st;
        t->cap_part_slots = cap;
    }
    ps_tree::Pinned& b = t->meta[t->next_meta];
    if ((st = pinned(c, b, total)) != PS_OK) return st;
    t->next_meta ^= 1;
    for (const Piece& x : pieces)
        if (x.bytes) memcpy(b.host + x.at, x.src, x.bytes);
    if ((st = send(c, b, t->dev, total)) != PS_OK) return st;
    auto at = [&](int i) { return t->dev + pieces[i].at; };
    t->positions = reinterpret_cast<const int32_t*>(at(0));
    t->slots = reinterpret_cast<const int32_t*>(at(1));
    t->row_seq = reinterpret_cast<const int32_t*>(at(2));
    t->row_prev = reinterpret_cast<const int32_t*>(at(3));
    TreeArgs& a = t->args;
    a.seqs = reinterpret_cast<const SeqInfo*>(at(4));
    a.pages = reinterpret_cast<const int32_t*>(at(5));
    a.items = reinterpret_cast<const AttnItem*>(at(6));
    a.worker_begin = reinterpret_cast<const int32_t*>(at(7));
    a.groups = reinterpret_cast<const MergeGroup*>(at(8));
    a.masks = reinterpret_cast<const uint32_t*>(at(9));
    a.part_o = t->part_o; a.part_ml = t->part_ml;
    set_work_lists(p, c->desc, &a);
    return PS_OK;
}

RopeOut rope_out(const ps_ctx* c, const ps_tree* t, int layer, bf16_t* q) {
    return RopeOut{q, slot_of(c, layer), t->positions, t->slots, reinterpret_cast<const float2*>(c->rope_cs), c->desc.n_q_heads, c->desc.n_kv_heads, c->desc.head_dim};
}

// Everything about rules that the host can see.
ps_status check_rules(ps_ctx* c, const ps_logit_rules& r, int n_rows, int vocab, const char* name) {
    const auto bad = [&](const char* what) { return fail(c, PS_EINVAL, std::string(name) + ": " + what); };
    if (r.n_lists < 0 || r.n_history < 0 || r.n_biases < 0 || r.n_masks < 0) return bad("negative count in the rules");
    if (r.n_lists == 0 && (r.history || r.repetition || r.frequency || r.presence || r.bias_token || r.row_list || r.row_token)) return bad("rules of lists with n_lists 0");
    if (r.n_lists > 0 && !r.row_list && r.n_lists != n_rows) return bad("without row_list n_lists must be the number of rows");
    if (r.history && !r.history_begin) return bad("history without history_begin");
    if (r.output_begin && !r.history) return bad("output_begin without history");
    if (r.bias_token && (!r.bias_begin || !r.bias_value)) return bad("bias_token without bias_begin and bias_value");
    if (r.row_prev && !r.row_token) return bad("row_prev without row_token");
    if (r.mask && r.mask_stride < (vocab + 31) / 32) return bad("mask_stride below ceil(vocab / 32)");
    if (r.mask && !r.mask_row && r.n_masks != n_rows) return bad("without mask_row n_masks must be the number of rows");
    if (!r.mask && (r.mask_row || r.n_masks)) return bad("mask_row or n_masks without mask");
    const void* words[] = {r.history, r.history_begin, r.output_begin, r.repetition, r.frequency, r.presence, r.bias_token, r.bias_value, r.bias_begin,
                           r.mask, r.mask_row, r.row_list, r.row_token, r.row_prev};
    for (const void* p : words)
        if (!aligned(p, 4)) return bad("the rules' arrays must be 4-byte aligned");
    return PS_OK;
}

}  // namespace

extern "C" ps_status ps_tree_create(ps_ctx* c, ps_tree** out) {
    if (!c || !out) return fail(c, PS_EINVAL, "ps_tree_create: null argument");
    *out = nullptr;
    ps_tree* t = new (std::nothrow) ps_tree();
    if (!t) return fail(c, PS_ENOMEM, "ps_tree_create: out of host memory");
    t->ctx = c; t->ctx_id = c->id; t->device = c->device; t->host_only = c->host_only;
    *out = t;
    return PS_OK;
}

extern "C" void ps_tree_destroy(ps_tree* t) {
    if (!t) return;
    if (!t->host_only) {
        OnDevice on(t->device);
        (void)hipDeviceSynchronize();
        dev_free(t->dev); dev_free(t->part_o); dev_free(t->part_ml); dev_free(t->dev_tokens);
        for (ps_tree::Pinned* b : {&t->meta[0], &t->meta[1], &t->tokens[0], &t->tokens[1]}) {
            if (b->host) (void)hipHostFree(b->host);
            if (b->read) (void)hipEventDestroy(b->read);
        }
    }
    delete t;
}

extern "C" ps_status ps_tree_plan(ps_ctx* c, ps_tree* t, const ps_seq* seqs, int32_t n_seqs, const int32_t* parents) {
    if (!c || !t) return fail(c, PS_EINVAL, "ps_tree_plan: null argument");
    if (t->ctx != c || t->ctx_id != c->id) return fail(c, PS_ESTATE, "ps_tree_plan: the tree belongs to another context");
    t->planned = false;
    return guarded(c, "ps_tree_plan", [&]() -> ps_status {
        if (!c->host_only && !c->pool) return fail(c, PS_ESTATE, "ps_tree_plan: no KV pool (call ps_kv_alloc)");
        OnDevice on(c);
        std::string err;
        ps_status st;
        if (!c->host_only && (st = check_not_captured(c, "ps_tree_plan")) != PS_OK) return st;
        const PlanConfig pc = tree_plan_config(c);
        st = validate_batch(seqs, n_seqs, pc, c->page_seen, err);
        if (st == PS_OK) st = build_tree_plan(seqs, n_seqs, parents, pc, t->plan, err);
        if (st != PS_OK) return fail(c, st, "ps_tree_plan: " + err);
        t->args = TreeArgs{};
        t->args.pages_once = std::all_of(t->plan.seqs.begin(), t->plan.seqs.end(), [&](const SeqInfo& s) { return s.n_new <= pc.prefill_tokens; });
        if (!c->host_only && n_seqs > 0 && (st = upload(c, t, t->plan)) != PS_OK) return st;
        t->pool_id = c->pool_id;
        t->planned = true;
        return PS_OK;
    });
}

extern "C" ps_status ps_tree_indices(ps_ctx* c, const ps_tree* t, int32_t* cu_seqlens, int32_t* positions, int32_t* slot_mapping) {
    if (!c || !t) return fail(c, PS_EINVAL, "ps_tree_indices: null argument");
    if (!t->planned) return fail(c, PS_ESTATE, "ps_tree_indices: the tree is not planned (call ps_tree_plan)");
    const TreePlan& p = t->plan;
    if (cu_seqlens) std::copy(p.cu_seqlens.begin(), p.cu_seqlens.end(), cu_seqlens);
    if (positions) std::copy(p.positions.begin(), p.positions.end(), positions);
    if (slot_mapping) std::copy(p.slots.begin(), p.slots.end(), slot_mapping);
    return PS_OK;
}

extern "C" ps_status ps_init_qk_norm(ps_ctx* c, int32_t layer, const void* g_q, const void* g_k) {
    if (!c) return PS_EINVAL;
    if (c->host_only) return fail(c, PS_ESTATE, "ps_init_qk_norm: host-only context");
    ps_status st = check_layer(c, layer, "ps_init_qk_norm");
    if (st != PS_OK) return st;
    if (!g_q != !g_k) return fail(c, PS_EINVAL, "ps_init_qk_norm: gains for only one of queries and keys");
    LayerWeights& L = c->layers[layer];
    if (!g_q) { L.qk_norm = false; return PS_OK; }
    if (!aligned(g_q, 16) || !aligned(g_k, 16)) return fail(c, PS_EINVAL, "ps_init_qk_norm: gains must be 16-byte aligned");
    OnDevice on(c);
    if ((st = check_not_captured(c, "ps_init_qk_norm")) != PS_OK) return st;
    const size_t bytes = (size_t)c->desc.head_dim * 2;
    if (!L.qk_gains && (st = dev_alloc(c, &L.qk_gains, 2 * bytes, "qk gains")) != PS_OK) return st;
    L.qk_norm = false;
    HIP_TRY(c, launch_copy_bytes(g_q, L.qk_gains, bytes, c->stream));
    HIP_TRY(c, launch_copy_bytes(g_k, L.qk_gains + c->desc.head_dim, bytes, c->stream));
    L.qk_norm = true;
    return PS_OK;
}

extern "C" ps_status ps_qk_norm_rope(ps_ctx* c, int32_t layer, const ps_tree* t, const void* qkv, int32_t dtype, int64_t ld, void* q) {
    const char* name = "ps_qk_norm_rope";
    if (!c) return PS_EINVAL;
    ps_status st = check_tree(c, t, name);
    if (st != PS_OK || (st = check_layer(c, layer, name)) != PS_OK) return st;
    if (t->plan.n_tokens == 0) return PS_OK;
    if (!qkv || !q) return fail(c, PS_EINVAL, "ps_qk_norm_rope: null qkv or q");
    if (dtype != PS_F32 && dtype != PS_BF16) return fail(c, PS_EINVAL, "ps_qk_norm_rope: dtype must be PS_F32 or PS_BF16");
    const size_t size = dtype == PS_F32 ? 4 : 2;
    if (ld < qkv_cols(c->desc)) return fail(c, PS_EINVAL, "ps_qk_norm_rope: ld is smaller than a row");
    if (!aligned(qkv, 16) || !aligned(q, 16) || (ld * size) % 16) return fail(c, PS_EINVAL, "ps_qk_norm_rope: qkv, its rows and q must be 16-byte aligned");
    const int64_t q_row = (int64_t)c->desc.n_q_heads * c->desc.head_dim * 2;
    if (rows_meet(qkv, qkv_cols(c->desc) * (int64_t)size, ld * (int64_t)size, q, q_row, q_row, t->plan.n_tokens)) return fail(c, PS_EINVAL, "ps_qk_norm_rope: qkv and q overlap");
    OnDevice on(c);
    const LayerWeights& L = c->layers[layer];
    const NormRopeArgs a{qkv, dtype == PS_BF16, 1, 0, ld, rope_out(c, t, layer, static_cast<bf16_t*>(q)), L.qk_norm ? L.qk_gains : nullptr, c->desc.rms_eps, t->plan.n_tokens};
    HIP_TRY(c, launch_qk_norm_rope(a, c->stream));
    return PS_OK;
}

extern "C" ps_status ps_tree_attention(ps_ctx* c, int32_t layer, const ps_tree* t, const void* q, int64_t ldq, void* out, int64_t ldo) {
    const char* name = "ps_tree_attention";
    if (!c) return PS_EINVAL;
    ps_status st = check_tree(c, t, name);
    if (st != PS_OK || (st = check_layer(c, layer, name)) != PS_OK) return st;
    if (t->plan.n_tokens == 0) return PS_OK;
    if (!q || !out) return fail(c, PS_EINVAL, "ps_tree_attention: null q or out");
    const int row = c->desc.n_q_heads * c->desc.head_dim;
    if (ldq < row || ldo < row || ldq > INT32_MAX) return fail(c, PS_EINVAL, "ps_tree_attention: a row stride is smaller than a row, or ldq above 2^31 - 1");
    if (!aligned(q, 16) || !aligned(out, 16) || ldq % 8 || ldo % 8) return fail(c, PS_EINVAL, "ps_tree_attention: q, out and their rows must be 16-byte aligned");
    if (rows_meet(q, row * 2, ldq * 2, out, row * 2, ldo * 2, t->plan.n_tokens)) return fail(c, PS_EINVAL, "ps_tree_attention: q and out overlap");
    OnDevice on(c);
    TreeArgs a = t->args;
    a.q = static_cast<const bf16_t*>(q); a.ldq = (int)ldq; a.pool_slot = slot_of(c, layer);
    a.out = static_cast<bf16_t*>(out); a.ldo = ldo;
    HIP_TRY(c, launch_tree_attention(a, c->stream));
    return PS_OK;
}

extern "C" ps_status ps_tree_keep(ps_ctx* c, const ps_tree* t, const int32_t* n_keep, const int32_t* nodes) {
    const char* name = "ps_tree_keep";
    if (!c) return PS_EINVAL;
    ps_status st = check_tree(c, t, name);
    if (st != PS_OK) return st;
    const TreePlan& p = t->plan;
    if (p.n_seqs == 0) return PS_OK;
    if (!n_keep) return fail(c, PS_EINVAL, "ps_tree_keep: null n_keep");
    return guarded(c, name, [&]() -> ps_status {
        // of every sequence, the nodes that are not where they belong already: those from the first such node on
        std::vector<int32_t> seq, first, begin, node;
        int64_t at = 0;
        for (int s = 0; s < p.n_seqs; s++) {
            const int n = n_keep[s], have = p.seqs[s].n_new;
            if (n < 0 || n > have) return fail(c, PS_ERANGE, "ps_tree_keep: seq " + std::to_string(s) + " has " + std::to_string(have) + " nodes, not " + std::to_string(n));
            if (n > 0 && !nodes) return fail(c, PS_EINVAL, "ps_tree_keep: null nodes");
            int k0 = -1;
            for (int k = 0; k < n; k++) {
                const int32_t v = nodes[at + k];
                if (v < 0 || v >= have) return fail(c, PS_ERANGE, "ps_tree_keep: seq " + std::to_string(s) + " has no node " + std::to_string(v));
                if (k > 0 && v <= nodes[at + k - 1]) return fail(c, PS_EINVAL, "ps_tree_keep: the nodes of seq " + std::to_string(s) + " are not ascending");
                if (k0 < 0 && v != k) {
                    k0 = k;
                    seq.push_back(s); first.push_back(k); begin.push_back((int32_t)node.size());
                }
                if (k0 >= 0) node.push_back(v);
            }
            at += n;
        }
        if (seq.empty()) return PS_OK;
        begin.push_back((int32_t)node.size());
        OnDevice on(c);
        const KeepList l{(int)seq.size(), seq.data(), first.data(), begin.data(), node.data()};
        HIP_TRY(c, launch_tree_keep(l, c->pool, c->slot_elems, c->n_kv_slots, t->args.seqs, t->args.pages, c->desc.n_kv_heads, c->desc.head_dim, c->stream));
        return PS_OK;
    });
}

extern "C" ps_status ps_pick_tokens(ps_ctx* c, const void* logits, int32_t dtype, int64_t ld, int32_t n_rows, int32_t vocab, const ps_logit_rules* rules,
                                    float* out, int64_t ldo, int32_t* next_tokens, float* logprobs) {
    const char* name = "ps_pick_tokens";
    if (!c) return PS_EINVAL;
    if (c->host_only) return fail(c, PS_ESTATE, "ps_pick_tokens: host-only context");
    if (n_rows < 0 || n_rows > (1 << 24)) return fail(c, PS_ERANGE, "ps_pick_tokens: n_rows outside [0, 2^24]");
    if (vocab < 1 || vocab > (1 << 20)) return fail(c, PS_ERANGE, "ps_pick_tokens: vocab outside [1, 2^20]");
    if (dtype != PS_F32 && dtype != PS_BF16) return fail(c, PS_EINVAL, "ps_pick_tokens: dtype must be PS_F32 or PS_BF16");
    if (n_rows == 0) return PS_OK;
    if (!logits) return fail(c, PS_EINVAL, "ps_pick_tokens: null logits");
    if (ld < vocab || (out && ldo < vocab)) return fail(c, PS_EINVAL, "ps_pick_tokens: a row stride is smaller than a row");
    if (!aligned(logits, dtype == PS_F32 ? 4 : 2) || !aligned(out, 4) || !aligned(next_tokens, 4) || !aligned(logprobs, 4))
        return fail(c, PS_EINVAL, "ps_pick_tokens: a tensor is not aligned to its elements");
    const int64_t size = dtype == PS_F32 ? 4 : 2;
    const bool in_place = out == logits && dtype == PS_F32 && (ld == ldo || n_rows == 1);
    if (out && !in_place && rows_meet(logits, vocab * size, ld * size, out, vocab * 4ll, ldo * 4, n_rows))
        return fail(c, PS_EINVAL, "ps_pick_tokens: out overlaps logits and is not fp32 logits themselves");
    PickArgs a{logits, dtype == PS_BF16, ld, n_rows, vocab, ps_logit_rules{}, out, ldo, next_tokens, logprobs};
    if (rules) {
        const ps_status st = check_rules(c, *rules, n_rows, vocab, name);
        if (st != PS_OK) return st;
        a.rules = *rules;
    }
    OnDevice on(c);
    HIP_TRY(c, launch_pick(a, c->ws_pick, c->stream));
    return PS_OK;
}

extern "C" ps_status ps_verify_tokens(ps_ctx* c, const ps_tree* tree, const int32_t* token_ids, const ps_logit_rules* rules, int32_t* next_tokens,
                                      float* logprobs, float* logits, float* hidden) {
    const char* name = "ps_verify_tokens";
    if (!c) return PS_EINVAL;
    ps_status st = check_tree(c, tree, name);
    if (st != PS_OK || (st = check_not_captured(c, name)) != PS_OK) return st;
    ps_tree* t = const_cast<ps_tree*>(tree);   // its buffers for token ids
    const TreePlan& p = t->plan;
    const ps_model_desc& d = c->desc;
    const int T = p.n_tokens, V = c->vocab, H = d.hidden;
    for (int l = 0; l < d.n_layers; l++)
        if (!c->layers[l].ready) return fail(c, PS_ESTATE, "ps_verify_tokens: layer " + std::to_string(l) + " has no weights (call ps_init_layer)");
    if (!c->head_ready) return fail(c, PS_ESTATE, "ps_verify_tokens: no model head (call ps_init_head)");
    if (c->opt_only_layer >= 0) return fail(c, PS_ESTATE, "ps_verify_tokens: option only_layer is set");
    if (rules) {
        if (rules->row_list || rules->row_token || rules->row_prev) return fail(c, PS_EINVAL, "ps_verify_tokens: row_list, row_token and row_prev are the tree's");
        if (rules->n_lists != 0 && rules->n_lists != p.n_seqs) return fail(c, PS_EINVAL, "ps_verify_tokens: n_lists must be 0 or the number of sequences");
        ps_logit_rules r = *rules;
        if (r.n_lists) r.row_list = t->row_seq;
        if ((st = check_rules(c, r, T, V, name)) != PS_OK) return st;
    }
    if (T == 0) return PS_OK;
    if (!token_ids) return fail(c, PS_EINVAL, "ps_verify_tokens: null token ids");
    for (int i = 0; i < T; i++)
        if (token_ids[i] < 0 || token_ids[i] >= V)
            return fail(c, PS_ERANGE, "ps_verify_tokens: token " + std::to_string(i) + " has id " + std::to_string(token_ids[i]) + " outside the vocabulary of " + std::to_string(V));
    return guarded(c, name, [&]() -> ps_status {
        OnDevice on(c);
        c->step_counter++;
        if (!c->ws_embed && c->cap_tokens > 0) {  // workspaces were sized before the head existed
            HIP_TRY(c, hipStreamSynchronize(c->stream));
            free_workspaces(c);
        }
        const GemmOptions o = gemm_options(c);
        ps_status st;
        if ((st = ensure_workspaces(c, T, 0, T, layer_needs(c, T, o), o)) != PS_OK) return st;
        if (!logits && (st = ensure_logits(c, (size_t)T * V * sizeof(float))) != PS_OK) return st;
        if (T > t->cap_tokens) {
            HIP_TRY(c, hipStreamSynchronize(c->stream));
            dev_free(t->dev_tokens);
            t->cap_tokens = 0;
            const int cap = (T + T / 4 + 63) & ~3;
            if ((st = dev_alloc(c, &t->dev_tokens, (size_t)cap * 4, "token ids")) != PS_OK) return st;
            t->cap_tokens = cap;
        }
        ps_tree::Pinned& b = t->tokens[t->next_tokens];
        if ((st = pinned(c, b, (size_t)T * 4)) != PS_OK) return st;
        t->next_tokens ^= 1;
        memcpy(b.host, token_ids, (size_t)T * 4);
        if ((st = send(c, b, t->dev_tokens, (size_t)T * 4)) != PS_OK) return st;

        StepBufs W = workspace_bufs(c, o);
        W.part_o = t->part_o; W.part_ml = t->part_ml;
        if (c->opt_poison && (st = poison(c, W, T, p.n_partial_slots)) != PS_OK) return st;
        HIP_TRY(c, launch_embed_gather(c->embedding, t->dev_tokens, c->ws_embed, T, H, c->stream));
        float* const x = hidden ? hidden : c->ws_final;
        const StackRun run{&W, T, t->positions, t->slots, nullptr, &t->args, nullptr, nullptr, 0, c->ws_embed, x, true, nullptr};
        if ((st = run_stack(c, run)) != PS_OK) return st;

        float* const z = logits ? logits : c->ws_logits;
        HIP_TRY(c, launch_rmsnorm(x, true, c->g_final, W.xn, T, H, d.rms_eps, c->stream));
        GemmArgs g{};
        g.A = W.xn; g.Wp = c->wout_t; g.M = T; g.N = V; g.K = H; g.kind = GemmOut::PARTIAL_F32;
        g.out = z; g.out_bytes = (size_t)T * V * sizeof(float);
        g.opt = head_options(c);
        g.sk_frag = W.skfrag; g.sk_frag_bytes = W.skfrag_bytes; g.sk_counters = W.skcnt; g.sk_n_counters = W.skcnt_n;
        int n_splits = 1;
        HIP_TRY(c, launch_gemm(g, &n_splits, c->stream));
        if (n_splits != 1) return fail(c, PS_EDEVICE, "ps_verify_tokens: output projection was split");
        PickArgs a{z, false, V, T, V, ps_logit_rules{}, rules ? logits : nullptr, V, next_tokens, logprobs};
        if (rules) {
            a.rules = *rules;
            if (rules->n_lists) { a.rules.row_list = t->row_seq; a.rules.row_token = t->dev_tokens; a.rules.row_prev = t->row_prev; }
        }
        if (a.out || a.next || a.logprob) HIP_TRY(c, launch_pick(a, c->ws_pick, c->stream));
        return PS_OK;
    });
}

extern "C" ps_status ps_kv_pool(ps_ctx* c, void** pool, int64_t* bytes) {
    if (!c || !pool || !bytes) return fail(c, PS_EINVAL, "ps_kv_pool: null argument");
    if (c->host_only) return fail(c, PS_ESTATE, "ps_kv_pool: host-only context");
    if (!c->pool) return fail(c, PS_ESTATE, "ps_kv_pool: no KV pool (call ps_kv_alloc)");
    *pool = c->pool;
    *bytes = (int64_t)(c->slot_elems * c->n_kv_slots * 2);
    return PS_OK;
}
