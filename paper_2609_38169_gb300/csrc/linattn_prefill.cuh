// What the prompt kernels of decayed linear attention share: arguments and the walk over
// their work.
#pragma once

#include "linattn.cuh"

namespace stepq {
namespace la {

constexpr int kChunk = 64;             // tokens a chunk of the tensor-core kernel

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
    int items;                         // (sequence, head) pairs
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

// The work of one CTA of a persistent grid: items blockIdx.x, + gridDim.x, ... that have
// tokens. Every warp walks it alike.
struct Items {
    const PrefillArgs &a;
    int item, h, row, len;
    __device__ __forceinline__ explicit Items(const PrefillArgs &args) : a(args), item((int)blockIdx.x - (int)gridDim.x) {}
    // lead: the thread that raises what is wrong with a sequence (one of a CTA's warps)
    __device__ __forceinline__ bool next(bool lead = false) {
#pragma unroll 1
        for (item += gridDim.x; item < a.items; item += gridDim.x) {
            b = item / a.Hv;
            h = item - b * a.Hv;
            if (sequence(a, b, lead, row, len, slot) && len > 0) return true;
        }
        return false;
    }
    __device__ __forceinline__ float *page() const {
        return a.pool + (uint64_t)slot * a.slot_floats + a.layer_off + (uint64_t)h * kN;
    }
    __device__ __forceinline__ const float *state_in() const { return !a.resume || a.resume[b] ? page() : nullptr; }
    __device__ __forceinline__ float *state_out() const { return page(); }
    __device__ __forceinline__ float *total_out() const { return nullptr; }

  private:
    int b, slot;
};

// linattn_chunks.cu
bool linattn_chunks_takes(const stepq_config *cfg, const stepq_linattn_io *io);
stepq_status launch_linattn_chunks(const PrefillArgs &a, int items, bool out, cudaStream_t s);

}  // namespace la
}  // namespace stepq
