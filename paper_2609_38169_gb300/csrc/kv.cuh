// Shared parts of the paged key-value cache's kernels: the pages' layout and the calls'
// arguments with their types erased.
//
// A page holds page_tokens tokens of every (layer, key head): the rows of K in token order,
// the rows of V, and for codes of 8 and 4 bits the fp16 scale of each row of K, then of V.
#pragma once

#include <cstdint>

#include "linattn.cuh"

namespace stepq {
namespace kv {

__host__ __device__ constexpr int bits_of(int format) { return format == STEPQ_KV_INT4 ? 4 : format == STEPQ_KV_INT8 ? 8 : 16; }
__host__ __device__ constexpr int row_bytes(int format, int dim) { return dim * bits_of(format) / 8; }
__host__ __device__ constexpr bool coded(int format) { return bits_of(format) < 16; }

// One layer of the pages.
struct Pages {
    uint8_t *base;                  // of the layer in page 0
    uint32_t page_bytes;
    uint32_t segment;               // bytes of one head's part of a page
    int n_pages, shift;             // page_tokens = 1 << shift
    const int32_t *table;
    int64_t table_stride;
    int width;                      // entries of a row of the table
    int n_heads;
    unsigned int *err;

    __device__ __forceinline__ int slot(int token) const { return token & ((1 << shift) - 1); }
    __device__ __forceinline__ uint8_t *at(int page, int head) const {
        return base + (uint64_t)(uint32_t)page * page_bytes + (uint64_t)head * segment;
    }
};

inline Pages pages_of(const stepq_kv_config *c, int layer, const stepq_kv_pages *p) {
    Pages g{};
    g.segment = (uint32_t)c->page_tokens * (2 * row_bytes(c->format, c->head_dim) + (coded(c->format) ? 4 : 0));
    g.page_bytes = g.segment * (uint32_t)(c->n_heads * c->n_layers);
    g.base = (uint8_t *)p->pages + (uint64_t)g.segment * c->n_heads * layer;
    g.n_pages = p->n_pages;
    while ((1 << g.shift) < c->page_tokens) g.shift++;
    g.table = p->table;
    g.table_stride = p->table_stride;
    g.width = p->table_width;
    g.n_heads = c->n_heads;
    g.err = device_error_word();
    return g;
}

// A call of stepq_kv_attend.
struct AttendArgs {
    Pages pg;
    const int32_t *lens;
    int B, groups, hq;              // groups: query heads a key head
    int dtype;
    const void *q;
    void *y;
    float *lse;
    int64_t qs, ys;
    float scale;                    // log2(e) times the call's
    int window;
    int whole;                      // clusters take whole sequences: no parts
    int stages;                     // of each warp's ring
    float *parts;                   // workspace, laid out as kv_attend.cuh says at Joined
};

// kv_launch.cuh, instantiated for each format in a file of its own
template <int F>
stepq_status launch_attend(const stepq_kv_config *c, const AttendArgs &args, int64_t most, cudaStream_t s);
template <int F>
size_t attend_workspace(const stepq_kv_config *c, int groups, int64_t rows, int64_t most);

}  // namespace kv
}  // namespace stepq
