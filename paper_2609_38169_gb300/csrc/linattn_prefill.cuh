// What the prompt kernels of decayed linear attention share: arguments, the plan that
// linattn_plan.cu lays down in the workspace, and the launches.
#pragma once

#include <cuda.h>

#include "linattn.cuh"

namespace stepq {
namespace la {

constexpr int kChunk = 64;             // tokens a chunk of the tensor-core kernel

// Consecutive tokens of one sequence that a CTA takes with one head: a whole sequence, or, of
// one that is split, Split::segment tokens or what is left.
struct alignas(16) Segment {
    int row, len;                      // first row, tokens
    int slot;
    int id;                            // place of its state in the workspace, where its sequence is split
    int in, out;                       // kState*: where the state before it comes from, where the one after it goes
    int pad[2];
};
enum { kStateZero, kStatePool, kStateWork };           // in; out: kStateZero is none
struct PlanHeader {
    int segments;
    int parts, splits;                 // the first segments of the table, whose own parts come first; split sequences
    int next[2];                       // the items taken so far by the two passes
    int pad[3];
};
struct Sequence {
    int id, segments;                  // id: its first segment's, where there are several
};
struct alignas(16) SplitSequence {
    int b, id, segments, pad;
};

struct PrefillArgs {
    float *pool;
    uint64_t slot_floats, layer_off;
    int pool_slots, B, tokens, Hk, Hv;
    const int32_t *slots, *cu;
    const uint8_t *resume;
    const void *q, *k, *v;
    const float *gate;
    void *y;
    int64_t qs, ks, vs, gs, ys;
    NormArgs norm;
    unsigned int *err;
    StallKnob stall;
    // the plan; without one (linattn_terms.cu alone) an item is a sequence
    PlanHeader *plan;
    Segment *table;                    // by falling length
    Sequence *sequences;
    SplitSequence *split;
    float *totals, *states;            // [their segments][Hv]: products of a segment's decays; states before the segments
    int segment;                       // tokens
};

// First row and length of sequence b, and its slot; false (and the device error) if either
// is out of range. lead: the thread that raises it.
__device__ __forceinline__ bool sequence(const PrefillArgs &a, int b, bool lead, int &start, int &len, int &slot) {
    const int each = a.tokens / a.B;
    start = a.cu ? a.cu[b] : b * each;
    const int end = a.cu ? a.cu[b + 1] : start + each;
    slot = a.slots[b];
    const bool bounds = start >= 0 && end >= start && end <= a.tokens;
    len = bounds ? end - start : 0;
    if (!bounds) {
        if (lead) raise_error(a.err, STEPQ_ERR_ARG);
        return false;
    }
    if (slot < 0 || slot >= a.pool_slots) {
        if (lead) raise_error(a.err, STEPQ_ERR_SLOT_RANGE);
        return false;
    }
    return true;
}
// Sequence b against those after it, `threads` of them at a time: two with tokens and one slot raise
// the device error.
__device__ __forceinline__ bool has_tokens(const PrefillArgs &a, int b) {
    return !a.cu || (a.cu[b] >= 0 && a.cu[b + 1] > a.cu[b] && a.cu[b + 1] <= a.tokens);
}
__device__ __forceinline__ void check_slot(const PrefillArgs &a, int b, int thread, int threads) {
    const int slot = a.slots[b];
    for (int j = b + 1 + thread; j < a.B; j += threads)
        if (a.slots[j] == slot && slot >= 0 && slot < a.pool_slots && has_tokens(a, b) && has_tokens(a, j))
            raise_error(a.err, STEPQ_ERR_DUP_SLOT);
}
__device__ __forceinline__ float *pool_page(const PrefillArgs &a, int slot, int h) {
    return a.pool + (uint64_t)slot * a.slot_floats + a.layer_off + (uint64_t)h * kN;
}

// Tokens of a segment for a call, the most segments it can make, and the most of them that are
// parts: a split sequence has `segment` tokens for each segment but its last, and one token or more
// for that, so there are no more split sequences than parts, and no more than 2 x parts segments of theirs.
struct Split {
    int segment, most, parts;          // parts = 0: no sequence is split
    int states() const { return 2 * parts < most || !parts ? 2 * parts : most; }
};
Split split_of(int Hv, int B, int tokens, int max_len);

// linattn_plan.cu: the segments; the states before the segments of split sequences from the
// segments' own parts
stepq_status launch_linattn_plan(const PrefillArgs &a, cudaStream_t s);
stepq_status launch_linattn_join(const PrefillArgs &a, int splits, cudaStream_t s);
// linattn_terms.cu. a = nullptr: only what a launch needs of the runtime
stepq_status launch_linattn_terms(int dtype, const PrefillArgs *a, int items, bool out, bool norm, cudaStream_t s);
// linattn_chunks.cu. prepare: what a launch needs of the runtime and the driver; parts: also the
// pass with out = false, which forms only the segments' own parts of the state
struct ChunkMaps {
    CUtensorMap of[3];                 // k, q, v
};
bool linattn_chunks_takes(const stepq_config *cfg, const stepq_linattn_io *io);
stepq_status prepare_linattn_chunks(const PrefillArgs &a, bool parts, ChunkMaps &maps);
stepq_status launch_linattn_chunks(const PrefillArgs &a, const ChunkMaps &maps, int grid, bool out, cudaStream_t s);

}  // namespace la
}  // namespace stepq
