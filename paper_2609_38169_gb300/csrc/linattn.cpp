// C-ABI entry points of decayed linear attention and the group norm: argument checks, then
// the launches.
#include <climits>
#include <cmath>

#include "internal.h"

using namespace stepq;

namespace {

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

int type_bytes(int dtype) { return dtype == STEPQ_F32 ? 4 : 2; }

stepq_status check_norm(const stepq_norm *n) {
    if (n->act < STEPQ_ACT_NONE || n->act > STEPQ_ACT_SIGMOID || (n->center & ~1) || (n->shared & ~1) ||
        !(n->eps >= 0.f) || std::isinf(n->eps))
        return STEPQ_ERR_ARG;
    if (!aligned(n->weight, 4) || !aligned(n->bias, 4)) return STEPQ_ERR_ALIGN;
    return STEPQ_OK;
}

// What the calls of decayed linear attention have in common. rows: of the vectors.
stepq_status check_call(const stepq_config *cfg, int layer, const float *pool, int pool_slots,
                        const int32_t *slots, int B, int rows, const stepq_linattn_io *io,
                        const stepq_norm *norm) {
    stepq_status st = validate_config(cfg, false);
    if (st != STEPQ_OK) return st;
    if (cfg->gate_kind != STEPQ_GATE_SCALAR) return STEPQ_ERR_UNSUPPORTED;
    if (layer < 0 || layer >= cfg->n_layers || !pool || pool_slots <= 0 || B < 0 || rows < 0 || !io)
        return STEPQ_ERR_ARG;
    if (io->dtype < STEPQ_F32 || io->dtype > STEPQ_F16) return STEPQ_ERR_ARG;
    if ((long long)B * cfg->n_value_heads > INT_MAX / 8) return STEPQ_ERR_ARG;     // the grid's size
    if (norm && (st = check_norm(norm)) != STEPQ_OK) return st;
    if (B == 0 || rows == 0) return STEPQ_OK;
    if (!slots || !io->q || !io->k || !io->v || !io->gate || !io->y) return STEPQ_ERR_ARG;
    const int64_t zs = norm && norm->z ? norm->z_stride : 0;
    if (io->q_stride < 0 || io->k_stride < 0 || io->v_stride < 0 || io->gate_stride < 0 || zs < 0 ||
        (rows > 1 && io->y_stride < (int64_t)kD * cfg->n_value_heads))
        return STEPQ_ERR_ARG;
    const int64_t step = 16 / type_bytes(io->dtype);
    if ((io->q_stride | io->k_stride | io->v_stride | io->y_stride | zs) & (step - 1)) return STEPQ_ERR_ALIGN;
    if (!aligned(pool, 16) || !aligned(slots, 4) || !aligned(io->q, 16) || !aligned(io->k, 16) ||
        !aligned(io->v, 16) || !aligned(io->y, 16) || !aligned(io->gate, 4) || (norm && !aligned(norm->z, 16)))
        return STEPQ_ERR_ALIGN;
    return STEPQ_OK;
}

}  // namespace

extern "C" stepq_status stepq_linattn_decode_step(const stepq_config *cfg, int layer, float *pool,
                                                  int pool_slots, const int32_t *slots, int B,
                                                  const stepq_linattn_io *io, const stepq_norm *norm,
                                                  stepq_stream_t stream) {
    const stepq_status st = check_call(cfg, layer, pool, pool_slots, slots, B, B, io, norm);
    if (st != STEPQ_OK || B == 0) return st;
    return launch_linattn_decode(cfg, layer, pool, pool_slots, slots, B, io, norm, (cudaStream_t)stream);
}

extern "C" size_t stepq_linattn_workspace_bytes(const stepq_config *cfg, int B, int tokens, int max_len) {
    if (validate_config(cfg, false) != STEPQ_OK || B <= 0 || tokens <= 0 || max_len < 0) return 0;
    if ((long long)B * cfg->n_value_heads > INT_MAX / 8) return 0;
    return linattn_workspace_bytes(cfg, B, tokens, max_len);
}

extern "C" stepq_status stepq_linattn_prefill(const stepq_config *cfg, int layer, float *pool, int pool_slots,
                                              const int32_t *slots, const uint8_t *resume,
                                              const int32_t *cu_seqlens, int B, int tokens, int max_len,
                                              const stepq_linattn_io *io, const stepq_norm *norm,
                                              void *workspace, size_t workspace_bytes, stepq_stream_t stream) {
    const stepq_status st = check_call(cfg, layer, pool, pool_slots, slots, B, tokens, io, norm);
    if (st != STEPQ_OK) return st;
    if (max_len < 0) return STEPQ_ERR_ARG;
    if (B == 0 || tokens == 0) return STEPQ_OK;
    if (!cu_seqlens && tokens % B) return STEPQ_ERR_ARG;
    if (!aligned(cu_seqlens, 4)) return STEPQ_ERR_ALIGN;
    const size_t need = linattn_workspace_bytes(cfg, B, tokens, max_len);
    if (need && (!workspace || workspace_bytes < need)) return STEPQ_ERR_ARG;
    if (need && !aligned(workspace, 256)) return STEPQ_ERR_ALIGN;
    return launch_linattn_prefill(cfg, layer, pool, pool_slots, slots, resume, cu_seqlens, B, tokens, max_len, io,
                                  norm, workspace, (cudaStream_t)stream);
}

extern "C" stepq_status stepq_group_norm(int dtype, int64_t rows, int groups, int width, const void *x,
                                         int64_t x_stride, void *out, int64_t out_stride,
                                         const stepq_norm *norm, stepq_stream_t stream) {
    if (dtype < STEPQ_F32 || dtype > STEPQ_F16 || rows < 0 || groups < 1 || width < 1 || !norm) return STEPQ_ERR_ARG;
    const stepq_status st = check_norm(norm);
    if (st != STEPQ_OK) return st;
    const int64_t channels = (int64_t)groups * width;
    if (channels > INT_MAX || rows > (1ll << 40) / groups) return STEPQ_ERR_ARG;
    if (rows == 0) return STEPQ_OK;
    if (!x || !out || x_stride < 0 || (rows > 1 && out_stride < channels) || (norm->z && norm->z_stride < 0))
        return STEPQ_ERR_ARG;
    // in place only row by row: else a row would be written before another one is read there
    if (rows > 1 && ((out == x && out_stride != x_stride) || (out == norm->z && out_stride != norm->z_stride)))
        return STEPQ_ERR_ARG;
    const uintptr_t e = (uintptr_t)type_bytes(dtype);
    if (!aligned(x, e) || !aligned(out, e) || !aligned(norm->z, e)) return STEPQ_ERR_ALIGN;
    return launch_group_norm(dtype, rows, groups, width, x, x_stride, out, out_stride, norm, (cudaStream_t)stream);
}
