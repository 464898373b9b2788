// Decayed linear attention over prompts on the FMA units, eight tokens at a time: the form for
// fp32 and fp16 vectors (whose products bf16 operands would cut), and for a few tokens.
//
// With c_t = g_1 .. g_t and w_ts = g_{s+1} .. g_t inside a block of eight tokens:
//   y_t = c_t S_0^T q_t + sum_{s<=t} w_ts (q_t . k_s) v_s,   S_8 = c_8 S_0 + sum_s w_8s k_s v_s^T,
// two multiply-adds per state element and token (three token by token, where the decay takes
// one). The state stays in registers: a warp holds all 128 rows of 16 columns, lane 4 r + c rows
// 32 m + 4 r + e (m, e = 0..3) of columns 4 c .. + 3, in pairs of rows, so that q and k come from
// shared memory as the pairs that the packed multiply-add takes. The readouts' sums over the
// eight row lanes r leave token r's in lane r (28 shuffles for 8 x 4 values), which adds its
// block's part.
//
// The FMA units and the chain of a block bound it: 3 x 333 tokens of 32 heads in fp32, 96 CTAs of
// two warps a scheduler on 152 multiprocessors, take 95 us (token by token: 215; with P formed in
// the block that takes it, three barriers: 104; the vectors' and states' bytes alone: 11).
// 16 x 1024 tokens (512 CTAs) take 1.10 ms, half the FMA rate, in fp16 as in fp32; two CTAs a
// multiprocessor, registers spilled, 14% more. 16 warps of 8 columns: 8% more, for twice the
// shared-memory reads. CTAs of 64 or 32 columns: 18 and 21% more, every CTA forming P.
#include "async.cuh"
#include "device.cuh"
#include "linattn_prefill.cuh"

namespace stepq {
namespace la {

constexpr int kBlockTokens = 8;

struct BlockStage {
    float q[kBlockTokens][kD], k[kBlockTokens][kD], v[kBlockTokens][kD], g[kBlockTokens];
};

template <class T, bool OUT, bool NORM>
__global__ void __launch_bounds__(256) linattn_blocks_kernel(PrefillArgs a) {
    constexpr int TB = kBlockTokens, J = 4;
    static_assert(TB == 8, "a warp a token");
    __shared__ __align__(16) BlockStage stage[3];            // read, ready, and being filled
    __shared__ __align__(16) float P[2][TB][TB];
    __shared__ __align__(16) float ys[2][NORM ? TB : 1][kD];
    const int tid = threadIdx.x, w = tid >> 5, l = tid & 31, r = l >> 2, c = l & 3;
    griddep_wait();
    griddep_launch();
    const int col = 4 * J * w + J * c;
    const int part = blockIdx.x / a.Hv, h = blockIdx.x - part * a.Hv, hk = h / (a.Hv / a.Hk);
    int row, len;
    const float *in = nullptr;
    float *out, *total_to = nullptr, total = 1.f;           // a part's decay
    if (a.plan) {
        if (part >= a.plan->segments) return;
        const Segment s = a.table[part];
        float *work = a.states + ((uint64_t)s.id * a.Hv + h) * kN, *page = pool_page(a, s.slot, h);
        if (!OUT && s.out == kStatePool) return;         // a sequence's last segment has no part to hand on
        row = s.row;
        len = s.len;
        if (OUT) in = s.in == kStateZero ? nullptr : s.in == kStatePool ? page : work;
        out = !OUT ? work + (uint64_t)a.Hv * kN : s.out == kStatePool ? page : nullptr;
        total_to = !OUT ? a.totals + (uint64_t)s.id * a.Hv + h : nullptr;
    } else {
        int slot;
        if (!sequence(a, part, tid == 0, row, len, slot) || len == 0) return;
        out = pool_page(a, slot, h);
        in = !a.resume || a.resume[part] ? out : nullptr;
    }
    uint64_t S[4][2][J];                                 // rows 32 m + 4 r + 2 p, + 1 of column col + j
#pragma unroll
    for (int m = 0; m < 4; m++)
#pragma unroll
        for (int p = 0; p < 2; p++) {
            float x[J] = {}, y[J] = {};
            if (in) {
                load_vec<float, J>(&in[(32 * m + 4 * r + 2 * p) * kD + col], x);
                load_vec<float, J>(&in[(32 * m + 4 * r + 2 * p + 1) * kD + col], y);
            }
#pragma unroll
            for (int j = 0; j < J; j++) S[m][p][j] = f2(x[j], y[j]);
        }
    // A block's vectors on their way: warp t brings token t, four channels a lane.
    const int t = w, ch = 4 * l;
    Vec<T, 4> nq, nk, nv;
    float ng = 1.f;
    const auto fetch = [&](int t0) {
        const Vec<T, 4> zero{};
        const int64_t at = (int64_t)row + t0 + t;
        const bool valid = t0 + t < len;
        nq = OUT && valid ? *(const Vec<T, 4> *)((const T *)a.q + at * a.qs + hk * kD + ch) : zero;
        nv = valid ? *(const Vec<T, 4> *)((const T *)a.v + at * a.vs + h * kD + ch) : zero;
        nk = valid ? *(const Vec<T, 4> *)((const T *)a.k + at * a.ks + hk * kD + ch) : zero;
        if (tid < TB) ng = t0 + tid < len ? a.gate[((int64_t)row + t0 + tid) * a.gs + h] : 1.f;
    };
    const auto put = [&](BlockStage &s) {
        if constexpr (sizeof(T) == 2) {
            // The conversions stay here: moved up to the loads, they would wait for them there (25% slower).
            uint32_t *q = (uint32_t *)&nq, *k = (uint32_t *)&nk, *v = (uint32_t *)&nv;
            asm volatile("" : "+r"(q[0]), "+r"(q[1]), "+r"(k[0]), "+r"(k[1]), "+r"(v[0]), "+r"(v[1])::"memory");
        }
        const auto f4 = [](const Vec<T, 4> &x) { return make_float4(to_f32(x.e[0]), to_f32(x.e[1]), to_f32(x.e[2]), to_f32(x.e[3])); };
        if (OUT) *(float4 *)&s.q[t][ch] = f4(nq);
        *(float4 *)&s.k[t][ch] = f4(nk);
        *(float4 *)&s.v[t][ch] = f4(nv);
        if (tid < TB) s.g[tid] = ng;
    };
    // P of token t = w: 4 channels a lane, eight keys' sums reduced together
    const auto scores = [&](const BlockStage &s, float (*P)[TB]) {
        float g[TB], p[TB];
        load_vec<float, 4>(s.g, *(float(*)[4]) & g[0]);
        load_vec<float, 4>(s.g + 4, *(float(*)[4]) & g[4]);
        const float4 q = *(const float4 *)&s.q[t][4 * l];
#pragma unroll
        for (int i = 0; i < TB; i++) {
            const float4 k = *(const float4 *)&s.k[i][4 * l];
            p[i] = fmaf(q.x, k.x, q.y * k.y) + fmaf(q.z, k.z, q.w * k.w);
        }
#pragma unroll
        for (int b = 0; b < 3; b++) {                        // lane bit 4 - b chooses key bit 2 - b
            const int half = 4 >> b;
            const bool up = l & (16 >> b);
#pragma unroll
            for (int i = 0; i < half; i++) {
                const float give = up ? p[i] : p[i + half];
                p[i] = (up ? p[i + half] : p[i]) + __shfl_xor_sync(0xffffffffu, give, 16 >> b);
            }
        }
        p[0] += __shfl_xor_sync(0xffffffffu, p[0], 2);
        p[0] += __shfl_xor_sync(0xffffffffu, p[0], 1);
        const int key = l >> 2;
        float wt = 1.f;
#pragma unroll
        for (int j = 1; j < TB; j++) wt *= j > key && j <= t ? g[j] : 1.f;
        if ((l & 3) == 0) P[t][key] = key <= t ? p[0] * wt : 0.f;
    };
    fetch(0);
    put(stage[0]);
    if (len > TB) {
        fetch(TB);
        put(stage[1]);
    }
    if (OUT) {
        __syncthreads();
        scores(stage[0], P[0]);
    }
    // Token w of block n, a block late: the readouts are in shared memory then, and the next block's
    // products fill the waits of its sums.
    const HeadAffine affine(a.norm, h, l);
    Vec<T, 4> z{};
    const auto normalise = [&](int n) {
        if (TB * n + w >= len) return;
        float u[1][4];
        if constexpr (sizeof(T) == 2) {                      // z's too
            uint32_t *word = (uint32_t *)&z;
            asm volatile("" : "+r"(word[0]), "+r"(word[1])::"memory");
        }
        load_vec<float, 4>(&ys[n & 1][w][4 * l], u[0]);
        norm_head<T, 1>(a.norm, affine, &z, u);
        store_vec<T, 4>((T *)a.y + ((int64_t)row + TB * n + w) * a.ys + h * kD + 4 * l, u[0]);
    };
    int at_stage = 0;                                        // n mod 3
    for (int t0 = 0, n = 0; t0 < len; t0 += TB, n++) {
        // One barrier a block: it shows the next block's vectors and this one's P, formed ahead.
        __syncthreads();
        const BlockStage &s = stage[at_stage], &next = stage[at_stage == 2 ? 0 : at_stage + 1];
        BlockStage &last = stage[at_stage == 0 ? 2 : at_stage - 1];
        at_stage = at_stage == 2 ? 0 : at_stage + 1;
        if (t0 + 2 * TB < len) fetch(t0 + 2 * TB);
        if (NORM) {
            if (n) normalise(n - 1);
            if (a.norm.z && t0 + w < len)
                z = *(const Vec<T, 4> *)((const T *)a.norm.z + ((int64_t)row + t0 + w) * a.norm.z_stride + h * kD + 4 * l);
        }
        float g[TB];
        load_vec<float, 4>(s.g, *(float(*)[4]) & g[0]);
        load_vec<float, 4>(s.g + 4, *(float(*)[4]) & g[4]);
        if (OUT) {
            // S_0^T q_t: this lane's rows, then the sum over the row lanes
            float y[TB][J];
#pragma unroll
            for (int t = 0; t < TB; t++) {
                uint64_t acc[J] = {};
#pragma unroll
                for (int m = 0; m < 4; m++) {
                    const ulonglong2 q = *(const ulonglong2 *)&s.q[t][32 * m + 4 * r];
#pragma unroll
                    for (int j = 0; j < J; j++) acc[j] = ffma2(q.y, S[m][1][j], ffma2(q.x, S[m][0][j], acc[j]));
                }
#pragma unroll
                for (int j = 0; j < J; j++) y[t][j] = f2lo(acc[j]) + f2hi(acc[j]);
            }
#pragma unroll
            for (int b = 0; b < 3; b++) {                // lane bit 4 - b (row lane bit 2 - b) chooses token bit 2 - b
                const int half = 4 >> b;
                const bool up = l & (16 >> b);
#pragma unroll
                for (int t = 0; t < half; t++)
#pragma unroll
                    for (int j = 0; j < J; j++) {
                        const float give = up ? y[t][j] : y[t + half][j];
                        y[t][j] = (up ? y[t + half][j] : y[t][j]) + __shfl_xor_sync(0xffffffffu, give, 16 >> b);
                    }
            }
            // token r: its part of the state before the block, then the block's own
            float ct = 1.f;
#pragma unroll
            for (int j = 0; j < TB; j++) ct *= j <= r ? g[j] : 1.f;
            float o[J], pr[TB];
            load_vec<float, 4>(&P[n & 1][r][0], *(float(*)[4]) & pr[0]);
            load_vec<float, 4>(&P[n & 1][r][4], *(float(*)[4]) & pr[4]);
#pragma unroll
            for (int j = 0; j < J; j++) o[j] = ct * y[0][j];
#pragma unroll
            for (int i = 0; i < TB; i++) {
                float v[J];
                load_vec<float, J>(&s.v[i][col], v);
#pragma unroll
                for (int j = 0; j < J; j++) o[j] = i <= r ? fmaf(pr[i], v[j], o[j]) : o[j];   // a later token's v may be anything
            }
            const int64_t at = (int64_t)row + t0;
            if (NORM) {
                store_vec<float, J>(&ys[n & 1][r][col], o);
            } else if (t0 + r < len) {
                store_vec<T, J>((T *)a.y + (at + r) * a.ys + h * kD + col, o);
            }
        }
        // S_8
        float w8[TB], all = 1.f;
#pragma unroll
        for (int i = TB - 1; i >= 0; i--) {
            w8[i] = all;
            all *= g[i];
        }
        if (!OUT) total *= all;
        const uint64_t all2 = f2s(all);
#pragma unroll
        for (int m = 0; m < 4; m++)
#pragma unroll
            for (int j = 0; j < J; j++) {
                S[m][0][j] = fmul2(S[m][0][j], all2);
                S[m][1][j] = fmul2(S[m][1][j], all2);
            }
#pragma unroll
        for (int i = 0; i < TB; i++) {
            float v[J];
            load_vec<float, J>(&s.v[i][col], v);
            uint64_t v2[J];
#pragma unroll
            for (int j = 0; j < J; j++) v2[j] = f2s(w8[i] * v[j]);
#pragma unroll
            for (int m = 0; m < 4; m++) {
                const ulonglong2 k = *(const ulonglong2 *)&s.k[i][32 * m + 4 * r];
#pragma unroll
                for (int j = 0; j < J; j++) {
                    S[m][0][j] = ffma2(k.x, v2[j], S[m][0][j]);
                    S[m][1][j] = ffma2(k.y, v2[j], S[m][1][j]);
                }
            }
        }
        if (OUT && t0 + TB < len) scores(next, P[~n & 1]);
        if (t0 + 2 * TB < len) put(last);
    }
    if (NORM) {
        __syncthreads();
        normalise((len - 1) / TB);
    }
    if (!OUT && tid == 0) *total_to = total;
    if (out)
#pragma unroll
        for (int m = 0; m < 4; m++)
#pragma unroll
            for (int p = 0; p < 2; p++) {
                float x[J], y[J];
#pragma unroll
                for (int j = 0; j < J; j++) {
                    x[j] = f2lo(S[m][p][j]);
                    y[j] = f2hi(S[m][p][j]);
                }
                float *at = &out[(32 * m + 4 * r + 2 * p) * kD + col];
                store_vec<float, J>(at, x);
                store_vec<float, J>(at + kD, y);
            }
}

template <class T, bool OUT>
static stepq_status launch_blocks(const PrefillArgs &a, long long items, cudaStream_t s) {
    if (OUT && a.norm.on) return launch_overlapped(linattn_blocks_kernel<T, OUT, OUT>, (int)items, 256, 0, s, a);
    return launch_overlapped(linattn_blocks_kernel<T, OUT, false>, (int)items, 256, 0, s, a);
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

// bf16 sequences of few tokens, where they are no more than fill the GPU's multiprocessors twice:
// blocks of eight need no plan before them (calls in a row, 16 tokens of 32 heads: 21 to 24 us for
// one sequence to eight, 64 tokens at a time on the tensor cores 27; of 16 sequences 34 against 30,
// of 64 sequences 133 against 81).
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
    a.totals = (float *)(base + w.totals);
    a.states = (float *)(base + w.states);
    a.segment = split.segment;
    const long long items = (long long)split.most * a.Hv;
    const bool few = (max_len > 0 ? max_len : tokens) <= kFewTokens && items <= 2 * sm_count();
    if (few || !la::linattn_chunks_takes(cfg, io)) {
        if (!split.on) a.plan = nullptr;                   // a segment is a sequence
        return la::by_type(io->dtype, [&](auto t) {
            using T = decltype(t);
            if (!split.on) return la::launch_blocks<T, true>(a, (long long)B * a.Hv, s);
            stepq_status st = la::launch_linattn_plan(a, s);
            if (st == STEPQ_OK) st = la::launch_blocks<T, false>(a, items, s);
            if (st == STEPQ_OK) st = la::launch_linattn_join(a, s);
            return st == STEPQ_OK ? la::launch_blocks<T, true>(a, items, s) : st;
        });
    }
    const int grid = items < sm_count() ? (int)items : sm_count();
    la::ChunkMaps maps;                                    // what may be refused comes before the first launch
    stepq_status st = la::prepare_linattn_chunks(a, split.on, maps);
    if (st == STEPQ_OK) st = la::launch_linattn_plan(a, s);
    if (st == STEPQ_OK && split.on) st = la::launch_linattn_chunks(a, maps, grid, false, s);
    if (st == STEPQ_OK && split.on) st = la::launch_linattn_join(a, s);
    return st == STEPQ_OK ? la::launch_linattn_chunks(a, maps, grid, true, s) : st;
}

}  // namespace stepq
