// Decayed linear attention over prompts (stepq_linattn_prefill): the workspace, and which kernels a
// call runs.
#include "device.cuh"
#include "linattn_prefill.cuh"

namespace stepq {
namespace {

// The workspace's parts, each at a multiple of 256 bytes.
struct Workspace {
    size_t table, sequences, splits, totals, states, bytes;
    Workspace(int Hv, int B, const la::Split &split) {
        const auto part = [&](size_t n) {
            const size_t at = bytes;
            bytes += (n + 255) / 256 * 256;
            return at;
        };
        bytes = 0;
        part(sizeof(la::PlanHeader));
        table = part((size_t)split.most * sizeof(la::Segment));
        sequences = part((size_t)B * sizeof(la::Sequence));
        splits = part((size_t)split.parts * sizeof(la::SplitSequence));
        const size_t held = split.states();
        totals = part(held * Hv * 4);
        states = part(held * Hv * kN * 4);
    }
};

// bf16 calls whose sequences are no longer than a block of the terms' kernel are its, without a plan:
// 16 tokens of 32 heads, calls in a row, take 20 us for one sequence, 71 for 64 and 256 for 256; 64
// tokens at a time 24, 81 and 282. 16 sequences of 32 tokens take 28 us by
// blocks of 16 and 24 by 64.
constexpr int kFewTokens = 16;

}  // namespace

size_t linattn_workspace_bytes(const stepq_config *cfg, int B, int tokens, int max_len) {
    return Workspace(cfg->n_value_heads, B, la::split_of(cfg->n_value_heads, B, tokens, max_len)).bytes;
}

stepq_status launch_linattn_prefill(const stepq_config *cfg, int layer, float *pool, int pool_slots,
                                    const int32_t *slots, const uint8_t *resume, const int32_t *cu, int B,
                                    int tokens, int max_len, const stepq_linattn_io *io, const stepq_norm *norm,
                                    void *workspace, cudaStream_t s) {
    la::PrefillArgs a{};
    const uint64_t per_layer = (uint64_t)kN * cfg->n_value_heads;
    a.pool = pool;
    a.slot_floats = per_layer * cfg->n_layers;
    a.layer_off = per_layer * layer;
    a.pool_slots = pool_slots;
    a.B = B;
    a.tokens = tokens;
    a.Hk = cfg->n_key_heads;
    a.Hv = cfg->n_value_heads;
    a.slots = slots; a.cu = cu; a.resume = resume;
    a.q = io->q; a.k = io->k; a.v = io->v; a.gate = io->gate; a.y = io->y;
    a.qs = io->q_stride; a.ks = io->k_stride; a.vs = io->v_stride; a.gs = io->gate_stride; a.ys = io->y_stride;
    a.norm = la::norm_args(norm);
    a.err = device_error_word();
    a.stall = stall_knob();
    const la::Split split = la::split_of(a.Hv, B, tokens, max_len);
    const Workspace w(a.Hv, B, split);
    uint8_t *base = (uint8_t *)workspace;
    a.plan = (la::PlanHeader *)base;
    a.table = (la::Segment *)(base + w.table);
    a.sequences = (la::Sequence *)(base + w.sequences);
    a.split = (la::SplitSequence *)(base + w.splits);
    a.totals = (float *)(base + w.totals);
    a.states = (float *)(base + w.states);
    a.segment = split.segment;
    const int items = split.most * a.Hv, parts = split.parts * a.Hv, splits = B < split.parts ? B : split.parts;
    const bool few = (max_len > 0 ? max_len : tokens) <= kFewTokens;
    if (few || !la::linattn_chunks_takes(cfg, io)) {
        const auto terms = [&](const la::PrefillArgs *args, bool out) {
            return la::launch_linattn_terms(io->dtype, args, out ? items : parts, out, norm != nullptr, s);
        };
        if (!split.parts) {                                 // a segment is a sequence
            a.plan = nullptr;
            return terms(&a, true);
        }
        stepq_status st = terms(nullptr, false);           // what may be refused comes before the first launch
        if (st == STEPQ_OK) st = terms(nullptr, true);
        if (st == STEPQ_OK) st = la::launch_linattn_plan(a, s);
        if (st == STEPQ_OK) st = terms(&a, false);
        if (st == STEPQ_OK) st = la::launch_linattn_join(a, splits, s);
        return st == STEPQ_OK ? terms(&a, true) : st;
    }
    const int sms = sm_count();
    la::ChunkMaps maps;                                    // what may be refused comes before the first launch
    stepq_status st = la::prepare_linattn_chunks(a, parts > 0, maps);
    if (st == STEPQ_OK) st = la::launch_linattn_plan(a, s);
    if (st == STEPQ_OK && parts) st = la::launch_linattn_chunks(a, maps, parts < sms ? parts : sms, false, s);
    if (st == STEPQ_OK && parts) st = la::launch_linattn_join(a, splits, s);
    return st == STEPQ_OK ? la::launch_linattn_chunks(a, maps, items < sms ? items : sms, true, s) : st;
}

}  // namespace stepq
