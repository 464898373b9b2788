// Decayed linear attention over prompts: S_t = g_t S_{t-1} + k_t v_t^T, y_t = S_t^T q_t for
// the tokens of packed sequences, token by token.
//
// One CTA of 128 threads per (sequence, value head): thread j holds column j of the state
// in registers, so neither the update nor the readout crosses threads; q and k reach all
// threads as shared-memory broadcasts. 3 x 128^2 FMA-pipe operations a token and head bound it.
#include "async.cuh"
#include "device.cuh"
#include "linattn_prefill.cuh"

namespace stepq {
namespace la {

constexpr int kBlockTokens = 16;       // tokens staged at a time

template <class T>
__global__ void __launch_bounds__(kD) linattn_prefill_tokens_kernel(PrefillArgs a) {
    __shared__ __align__(16) float qs[kBlockTokens][kD], ks[kBlockTokens][kD], vy[kBlockTokens][kD];
    __shared__ float gs[kBlockTokens];
    const int j = threadIdx.x, w = j >> 5, l = j & 31;
    griddep_wait();
    griddep_launch();
    const int b = blockIdx.x / a.Hv, h = blockIdx.x - b * a.Hv, hk = h / (a.Hv / a.Hk);
    int start, len, slot;
    if (!sequence(a, b, j == 0, start, len, slot) || len == 0) return;
    float *S = a.pool + (uint64_t)slot * a.slot_floats + a.layer_off + (uint64_t)h * kN + j;
    uint64_t s[kD / 2];                                  // rows 2 i, 2 i + 1 of column j
    const bool from_slot = !a.resume || a.resume[b];
#pragma unroll
    for (int i = 0; i < kD / 2; i++)
        s[i] = from_slot ? f2(S[(2 * i) * kD], S[(2 * i + 1) * kD]) : 0;
    for (int t0 = 0; t0 < len; t0 += kBlockTokens) {
        const int n = min(kBlockTokens, len - t0);
        const int64_t row = (int64_t)start + t0;
        for (int t = 0; t < n; t++) {
            qs[t][j] = to_f32(((const T *)a.q)[(row + t) * a.qs + hk * kD + j]);
            ks[t][j] = to_f32(((const T *)a.k)[(row + t) * a.ks + hk * kD + j]);
            vy[t][j] = to_f32(((const T *)a.v)[(row + t) * a.vs + h * kD + j]);
        }
        if (j < n) gs[j] = a.gate[(row + j) * a.gs + h];
        __syncthreads();
        for (int t = 0; t < n; t++) {
            const uint64_t g = f2s(gs[t]), v = f2s(vy[t][j]);
            uint64_t y0 = 0, y1 = 0;
#pragma unroll
            for (int i = 0; i < kD / 2; i += 2) {
                const uint4 k = *(const uint4 *)&ks[t][2 * i], q = *(const uint4 *)&qs[t][2 * i];
                s[i] = ffma2(u2pair(k.x, k.y), v, fmul2(g, s[i]));
                s[i + 1] = ffma2(u2pair(k.z, k.w), v, fmul2(g, s[i + 1]));
                y0 = ffma2(u2pair(q.x, q.y), s[i], y0);
                y1 = ffma2(u2pair(q.z, q.w), s[i + 1], y1);
            }
            const uint64_t y = fadd2(y0, y1);
            vy[t][j] = f2lo(y) + f2hi(y);                // v of this thread's column is used up
        }
        __syncthreads();
        for (int t = w; t < n; t += 4) {
            const float4 r = *(const float4 *)&vy[t][4 * l];
            float y[1][4] = {{r.x, r.y, r.z, r.w}};
            if (a.norm.on) {
                Vec<T, 4> z{};
                if (a.norm.z) z = *(const Vec<T, 4> *)((const T *)a.norm.z + (row + t) * a.norm.z_stride + h * kD + 4 * l);
                norm_head<T, 1>(a.norm, HeadAffine(a.norm, h, l), &z, y);
            }
            store_vec<T, 4>((T *)a.y + (row + t) * a.ys + h * kD + 4 * l, y[0]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kD / 2; i++) {
        S[(2 * i) * kD] = f2lo(s[i]);
        S[(2 * i + 1) * kD] = f2hi(s[i]);
    }
}

}  // namespace la

namespace {

// The workspace's parts, each at a multiple of 256 bytes.
struct Workspace {
    size_t table, sequences, totals, states, bytes;
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
        totals = part(split.on ? (size_t)split.most * Hv * 4 : 0);
        states = part(split.on ? (size_t)split.most * Hv * kN * 4 : 0);
    }
};

// The tensor-core kernel takes 64 tokens at a time with its operands in flight; for a few tokens
// the walk token by token is done sooner: (measured rule below).
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
    const bool few = (max_len > 0 ? max_len : tokens) <= kFewTokens;
    if (few || !la::linattn_chunks_takes(cfg, io))
        return la::by_type(io->dtype, [&](auto t) {
            return launch_overlapped(la::linattn_prefill_tokens_kernel<decltype(t)>, B * a.Hv, kD, 0, s, a);
        });
    const la::Split split = la::split_of(a.Hv, B, tokens, max_len);
    const Workspace w(a.Hv, B, split);
    uint8_t *base = (uint8_t *)workspace;
    a.plan = (la::PlanHeader *)base;
    a.table = (la::Segment *)(base + w.table);
    a.sequences = (la::Sequence *)(base + w.sequences);
    a.totals = (float *)(base + w.totals);
    a.states = (float *)(base + w.states);
    a.segment = split.segment;
    const long long items = (long long)split.most * a.Hv;
    const int grid = items < sm_count() ? (int)items : sm_count();
    la::ChunkMaps maps;                                    // what may be refused comes before the first launch
    stepq_status st = la::prepare_linattn_chunks(a, split.on, maps);
    if (st == STEPQ_OK) st = la::launch_linattn_plan(a, s);
    if (st == STEPQ_OK && split.on) st = la::launch_linattn_chunks(a, maps, grid, false, s);
    if (st == STEPQ_OK && split.on) st = la::launch_linattn_join(a, s);
    return st == STEPQ_OK ? la::launch_linattn_chunks(a, maps, grid, true, s) : st;
}

}  // namespace stepq
