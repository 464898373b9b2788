// C-ABI entry points of the paged key-value cache: argument checks, then the launches.
#include <climits>
#include <cmath>

#include "internal.h"

using namespace stepq;

namespace {

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

int row_bits(int format) { return format == STEPQ_KV_INT4 ? 4 : format == STEPQ_KV_INT8 ? 8 : 16; }

size_t page_bytes(const stepq_kv_config *c) {
    const size_t row = (size_t)c->head_dim * row_bits(c->format) / 8;
    return (size_t)c->n_layers * c->n_heads * c->page_tokens * (2 * row + (row_bits(c->format) < 16 ? 4 : 0));
}

stepq_status check_config(const stepq_kv_config *c) {
    if (!c || c->n_layers < 1 || c->n_heads < 1 || c->format < STEPQ_KV_BF16 || c->format > STEPQ_KV_INT4 ||
        c->n_heads > (1 << 14) || c->n_layers > (1 << 16))
        return STEPQ_ERR_ARG;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return STEPQ_ERR_UNSUPPORTED;
    if (c->page_tokens < 8 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1)))
        return STEPQ_ERR_UNSUPPORTED;
    return page_bytes(c) < (1ull << 32) ? STEPQ_OK : STEPQ_ERR_UNSUPPORTED;
}

stepq_status check_pages(const stepq_kv_config *c, int layer, const stepq_kv_pages *p, int B) {
    const stepq_status st = check_config(c);
    if (st != STEPQ_OK) return st;
    if (layer < 0 || layer >= c->n_layers || !p || B < 0) return STEPQ_ERR_ARG;
    if (!p->pages || p->n_pages < 1 || p->table_width < 0 || p->table_stride < 0 || (B > 0 && p->table_width > 0 && !p->table) ||
        (int64_t)p->table_width * c->page_tokens > (1 << 30))
        return STEPQ_ERR_ARG;
    return aligned(p->pages, 16) && aligned(p->table, 4) ? STEPQ_OK : STEPQ_ERR_ALIGN;
}

// Rows of a vector type at `stride` elements.
stepq_status check_rows(int dtype, const void *p, int64_t stride) {
    if (!p || stride < 0) return STEPQ_ERR_ARG;
    return aligned(p, 16) && stride % (dtype == STEPQ_F32 ? 4 : 8) == 0 ? STEPQ_OK : STEPQ_ERR_ALIGN;
}

stepq_status check_transfer(const stepq_kv_config *c, int layer, const stepq_kv_pages *p, const int32_t *starts,
                            const int32_t *cu, int B, int tokens, const stepq_kv_rows *r, bool out) {
    stepq_status st = check_pages(c, layer, p, B);
    if (st != STEPQ_OK) return st;
    if (tokens < 0 || tokens > (1 << 30) || !r || r->dtype < STEPQ_F32 || r->dtype > STEPQ_F16) return STEPQ_ERR_ARG;
    if (B == 0 || tokens == 0) return STEPQ_OK;
    if (!starts || (!cu && tokens % B)) return STEPQ_ERR_ARG;
    if (!aligned(starts, 4) || !aligned(cu, 4)) return STEPQ_ERR_ALIGN;
    if ((st = check_rows(r->dtype, r->k, r->k_stride)) != STEPQ_OK) return st;
    if ((st = check_rows(r->dtype, r->v, r->v_stride)) != STEPQ_OK) return st;
    const int64_t width = (int64_t)c->n_heads * c->head_dim;
    if (out && tokens > 1 && (r->k_stride < width || r->v_stride < width)) return STEPQ_ERR_ARG;
    return STEPQ_OK;
}

// Whether q_heads are shared by the key heads evenly, and rows of them make a grid.
bool heads_fit(const stepq_kv_config *c, int q_heads, int B) {
    return q_heads >= 1 && q_heads % c->n_heads == 0 && (long long)B * q_heads <= INT_MAX / 8;
}

}  // namespace

extern "C" size_t stepq_kv_page_bytes(const stepq_kv_config *c) { return check_config(c) == STEPQ_OK ? page_bytes(c) : 0; }

extern "C" stepq_status stepq_kv_append(const stepq_kv_config *cfg, int layer, const stepq_kv_pages *pages,
                                        const int32_t *starts, const int32_t *cu_seqlens, int B, int tokens,
                                        const stepq_kv_rows *rows, stepq_stream_t stream) {
    const stepq_status st = check_transfer(cfg, layer, pages, starts, cu_seqlens, B, tokens, rows, false);
    if (st != STEPQ_OK || B == 0 || tokens == 0) return st;
    return launch_kv_rows(true, cfg, layer, pages, starts, cu_seqlens, B, tokens, rows, (cudaStream_t)stream);
}

extern "C" stepq_status stepq_kv_read(const stepq_kv_config *cfg, int layer, const stepq_kv_pages *pages,
                                      const int32_t *starts, const int32_t *cu_seqlens, int B, int tokens,
                                      const stepq_kv_rows *rows, stepq_stream_t stream) {
    const stepq_status st = check_transfer(cfg, layer, pages, starts, cu_seqlens, B, tokens, rows, true);
    if (st != STEPQ_OK || B == 0 || tokens == 0) return st;
    return launch_kv_rows(false, cfg, layer, pages, starts, cu_seqlens, B, tokens, rows, (cudaStream_t)stream);
}

extern "C" size_t stepq_kv_workspace_bytes(const stepq_kv_config *cfg, int q_heads, int B, int max_len) {
    if (check_config(cfg) != STEPQ_OK || B <= 0 || max_len < 0 || !heads_fit(cfg, q_heads, B)) return 0;
    return kv_workspace_bytes(cfg, q_heads, B, max_len ? max_len : 1 << 30);
}

extern "C" stepq_status stepq_kv_attend(const stepq_kv_config *cfg, int layer, const stepq_kv_pages *pages,
                                        const int32_t *lens, int B, const stepq_kv_query *q, void *workspace,
                                        size_t workspace_bytes, stepq_stream_t stream) {
    stepq_status st = check_pages(cfg, layer, pages, B);
    if (st != STEPQ_OK) return st;
    if (!q || q->dtype < STEPQ_F32 || q->dtype > STEPQ_F16 || !std::isfinite(q->scale) || q->window < 0 ||
        q->max_len < 0 || !heads_fit(cfg, q->n_heads, B))
        return STEPQ_ERR_ARG;
    if (B == 0) return STEPQ_OK;
    if (!lens) return STEPQ_ERR_ARG;
    if (!aligned(lens, 4) || !aligned(q->lse, 4)) return STEPQ_ERR_ALIGN;
    if ((st = check_rows(q->dtype, q->q, q->q_stride)) != STEPQ_OK) return st;
    if ((st = check_rows(q->dtype, q->y, q->y_stride)) != STEPQ_OK) return st;
    if (B > 1 && q->y_stride < (int64_t)q->n_heads * cfg->head_dim) return STEPQ_ERR_ARG;
    if (q->y == q->q && B > 1 && q->y_stride != q->q_stride) return STEPQ_ERR_ARG;
    const int64_t width = (int64_t)pages->table_width * cfg->page_tokens;
    const int64_t most = q->max_len && q->max_len < width ? q->max_len : width;
    const size_t need = kv_workspace_bytes(cfg, q->n_heads, B, most);
    if (need && (!workspace || workspace_bytes < need)) return STEPQ_ERR_ARG;
    if (need && !aligned(workspace, 256)) return STEPQ_ERR_ALIGN;
    return launch_kv_attend(cfg, layer, pages, lens, B, q, most, workspace, (cudaStream_t)stream);
}
