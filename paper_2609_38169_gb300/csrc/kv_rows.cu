// Rows of K and V into the pages, and back.
//
// A code of b bits is u = clamp(rne(x / s), -q, q) + 2^(b-1) with q = 2^(b-1) - 1 and the row's
// scale s = fp16(clamp(absmax / q, 2^-14, 65504)); it stands for (u - 2^(b-1)) s. x / s is the
// rounded quotient: for x of 16 bits its distance from a border between two codes is zero
// or above 2^-20 of it, so every such code is the one of the exact quotient.
//
// One warp per token, which finds its sequence and page once for all heads. A lane takes
// eight channels, D / 8 lanes a row, so that a warp has 32 / (D / 8) rows at once.
#include <type_traits>

#include "device.cuh"
#include "kv.cuh"

namespace stepq {
namespace kv {

constexpr int kWarps = 4;

struct RowsArgs {
    Pages pg;
    const int32_t *starts, *cu;
    int B, tokens;
    void *k, *v;                    // read only by the append
    int64_t ks, vs;
};

// The sequence of packed row i: the last whose first row is not above it. Empty sequences and
// bounds out of order come out as the sequence that the halving ends at; the caller checks
// that it holds the row.
__device__ __forceinline__ int find_sequence(const int32_t *cu, int B, int i, int lane) {
    int lo = 0, n = B;                                       // among sequences lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const bool below = lane * step < n && cu[at] <= i;
        const unsigned m = __ballot_sync(0xffffffffu, below);
        const int last = m ? 31 - __clz(m) : 0;
        n = min(step, n - last * step);
        lo += last * step;
    }
    return lo;
}

// Eight channels of a row.
template <class T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]) {
    if (sizeof(T) == 4) {
        const float4 a = ((const float4 *)p)[0], b = ((const float4 *)p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const la::Vec<T, 8> v = *(const la::Vec<T, 8> *)p;
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = la::to_f32(v.e[i]);
    }
}
template <class T>
__device__ __forceinline__ void store8(T *p, const float (&x)[8]) {
    if (sizeof(T) == 4) {
        ((float4 *)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        ((float4 *)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        la::store_vec<T, 8>(p, x);
    }
}

// Where a token's rows go: its page and place, or page -1.
struct Place { int page, slot; };
__device__ __forceinline__ Place place_of(const RowsArgs &a, int i, int lane) {
    int b, first;
    if (a.cu) {
        b = find_sequence(a.cu, a.B, i, lane);
        first = a.cu[b];
        if (i < first || i >= a.cu[b + 1]) {
            if (lane == 0 && (i < a.cu[a.B] && i >= a.cu[0])) raise_error(a.pg.err, STEPQ_ERR_ARG);
            return {-1, 0};
        }
    } else {
        const int each = a.tokens / a.B;
        b = i / each;
        first = b * each;
    }
    const int start = a.starts[b];
    const long long pos = (long long)start + (i - first);
    if (start < 0 || (pos >> a.pg.shift) >= a.pg.width) {
        if (lane == 0) raise_error(a.pg.err, STEPQ_ERR_SLOT_RANGE);
        return {-1, 0};
    }
    const int page = a.pg.table[b * a.pg.table_stride + (pos >> a.pg.shift)];
    if (page < 0 || page >= a.pg.n_pages) {
        if (lane == 0) raise_error(a.pg.err, STEPQ_ERR_SLOT_RANGE);
        return {-1, 0};
    }
    return {page, a.pg.slot((int)pos)};
}

template <int F, int D, class T>
__global__ void __launch_bounds__(32 * kWarps) kv_append_kernel(RowsArgs a) {
    constexpr int RB = row_bytes(F, D), L = D / 8, PER = 32 / L;
    const int lane = threadIdx.x & 31, i = blockIdx.x * kWarps + (threadIdx.x >> 5);
    griddep_wait();
    griddep_launch();
    if (i >= a.tokens) return;
    const Place p = place_of(a, i, lane);
    if (p.page < 0) return;
    const int rows = 2 * a.pg.n_heads, c = lane % L, pt = 1 << a.pg.shift;
    for (int r0 = 0; r0 < rows; r0 += PER) {
        const int r = r0 + lane / L;                         // head by head, K before V
        const bool on = r < rows;
        const int h = r >> 1, part = r & 1;
        float x[8] = {};
        if (on) load8<T>((const T *)(part ? a.v : a.k) + i * (part ? a.vs : a.ks) + h * D + 8 * c, x);
        uint8_t *seg = a.pg.at(p.page, h);
        uint8_t *row = seg + (part * pt + p.slot) * RB;
        if (!coded(F)) {
            using C = typename std::conditional<F == STEPQ_KV_BF16, la::bf16, la::f16>::type;
            if (on) store8<C>((C *)row + 8 * c, x);
            continue;
        }
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) top = fmaxf(top, fabsf(x[e]));
#pragma unroll
        for (int o = 1; o < L; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        constexpr float q = F == STEPQ_KV_INT8 ? 127.f : 7.f;
        const uint16_t sb = f16_bits(fminf(fmaxf(__fdiv_rn(top, q), kF16Min), kF16Max));
        const float s = f16_val(sb);
        uint32_t u[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float t = x[e] == x[e] ? fminf(fmaxf(rintf(__fdiv_rn(x[e], s)), -q), q) : 0.f;
            u[e] = (uint32_t)(int)(t + (q + 1.f));
        }
        if (!on) continue;
        if (F == STEPQ_KV_INT8) {
            const uint32_t w0 = u[0] | u[1] << 8 | u[2] << 16 | u[3] << 24, w1 = u[4] | u[5] << 8 | u[6] << 16 | u[7] << 24;
            ((uint2 *)row)[c] = make_uint2(w0, w1);
        } else {
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 8; e++) w |= u[e] << (4 * e);
            ((uint32_t *)row)[c] = w;
        }
        if (c == 0) ((uint16_t *)(seg + 2 * pt * RB))[part * pt + p.slot] = sb;
    }
}

template <int F, int D, class T>
__global__ void __launch_bounds__(32 * kWarps) kv_read_kernel(RowsArgs a) {
    constexpr int RB = row_bytes(F, D), L = D / 8, PER = 32 / L;
    const int lane = threadIdx.x & 31, i = blockIdx.x * kWarps + (threadIdx.x >> 5);
    griddep_wait();
    griddep_launch();
    if (i >= a.tokens) return;
    const Place p = place_of(a, i, lane);
    if (p.page < 0) return;
    const int rows = 2 * a.pg.n_heads, c = lane % L, pt = 1 << a.pg.shift;
    for (int r = lane / L; r < rows; r += PER) {
        const int h = r >> 1, part = r & 1;
        const uint8_t *seg = a.pg.at(p.page, h);
        const uint8_t *row = seg + (part * pt + p.slot) * RB;
        float x[8];
        if (!coded(F)) {
            using C = typename std::conditional<F == STEPQ_KV_BF16, la::bf16, la::f16>::type;
            load8<C>((const C *)row + 8 * c, x);
        } else {
            const float s = f16_val(((const uint16_t *)(seg + 2 * pt * RB))[part * pt + p.slot]);
            if (F == STEPQ_KV_INT8) {
                const uint2 w = ((const uint2 *)row)[c];
#pragma unroll
                for (int e = 0; e < 8; e++) x[e] = (float)((int)((e < 4 ? w.x : w.y) >> (8 * (e & 3)) & 255u) - 128) * s;
            } else {
                const uint32_t w = ((const uint32_t *)row)[c];
#pragma unroll
                for (int e = 0; e < 8; e++) x[e] = (float)((int)(w >> (4 * e) & 15u) - 8) * s;
            }
        }
        store8<T>((T *)(part ? a.v : a.k) + i * (part ? a.vs : a.ks) + h * D + 8 * c, x);
    }
}

// Runs f(format) with the pages' format as a compile-time constant.
template <class Fn>
auto by_format(const stepq_kv_config *c, Fn &&f) {
    switch (c->format) {
    case STEPQ_KV_BF16: return f(std::integral_constant<int, STEPQ_KV_BF16>{});
    case STEPQ_KV_F16: return f(std::integral_constant<int, STEPQ_KV_F16>{});
    case STEPQ_KV_INT8: return f(std::integral_constant<int, STEPQ_KV_INT8>{});
    default: return f(std::integral_constant<int, STEPQ_KV_INT4>{});
    }
}
// Runs f(format, dim).
template <class Fn>
stepq_status by_layout(const stepq_kv_config *c, Fn &&f) {
    return by_format(c, [&](auto fmt) {
        return c->head_dim == 64    ? f(fmt, std::integral_constant<int, 64>{})
               : c->head_dim == 128 ? f(fmt, std::integral_constant<int, 128>{})
                                    : f(fmt, std::integral_constant<int, 256>{});
    });
}

}  // namespace kv

stepq_status launch_kv_rows(bool append, const stepq_kv_config *cfg, int layer, const stepq_kv_pages *pages,
                            const int32_t *starts, const int32_t *cu, int B, int tokens, const stepq_kv_rows *rows,
                            cudaStream_t s) {
    kv::RowsArgs a{};
    a.pg = kv::pages_of(cfg, layer, pages);
    a.starts = starts;
    a.cu = cu;
    a.B = B;
    a.tokens = tokens;
    a.k = rows->k; a.v = rows->v; a.ks = rows->k_stride; a.vs = rows->v_stride;
    const int grid = (tokens + kv::kWarps - 1) / kv::kWarps;
    return kv::by_layout(cfg, [&](auto f, auto d) {
        return la::by_type(rows->dtype, [&](auto t) {
            auto *kernel = append ? kv::kv_append_kernel<decltype(f)::value, decltype(d)::value, decltype(t)>
                                  : kv::kv_read_kernel<decltype(f)::value, decltype(d)::value, decltype(t)>;
            return launch_overlapped(kernel, grid, 32 * kv::kWarps, 0, s, a);
        });
    });
}

size_t kv_workspace_bytes(const stepq_kv_config *cfg, int q_heads, int64_t rows, int64_t most) {
    return kv::by_format(cfg, [&](auto f) {
        return kv::attend_workspace<decltype(f)::value>(cfg, q_heads / cfg->n_heads, rows, most);
    });
}

stepq_status launch_kv_attend(const stepq_kv_config *cfg, int layer, const stepq_kv_pages *pages, const int32_t *lens,
                              int B, const stepq_kv_query *q, int64_t most, void *workspace, cudaStream_t s) {
    kv::AttendArgs a{};
    a.pg = kv::pages_of(cfg, layer, pages);
    a.lens = lens;
    a.B = B;
    a.groups = q->n_heads / cfg->n_heads;
    a.hq = q->n_heads;
    a.dtype = q->dtype;
    a.q = q->q; a.y = q->y; a.lse = q->lse; a.qs = q->q_stride; a.ys = q->y_stride;
    a.scale = q->scale * 1.44269504f;
    a.window = q->window;
    a.parts = (float *)workspace;
    return kv::by_format(cfg, [&](auto f) { return kv::launch_attend<decltype(f)::value>(cfg, a, most, s); });
}

}  // namespace stepq
