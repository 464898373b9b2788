// Rows of K and V into the pages, and back.
//
// A code of b bits is u = clamp(rne(x / s), -q, q) + 2^(b-1) with q = 2^(b-1) - 1 and the row's
// scale s = fp16(clamp(absmax / q, 2^-14, 65504)); it stands for (u - 2^(b-1)) s. x / s is the
// rounded quotient: for x of 16 bits its distance from a border between two codes is zero
// or above 2^-20 of it, so every such code is the one of the exact quotient.
//
// A warp takes K or V of one token and up to kRows rows a lane: a lane has eight channels, D / 8
// lanes a row, so that a warp holds 32 / (D / 8) heads at once. All its loads are on their way
// before it looks at the first value (the append's before it has found the token's sequence and
// page). HBM bounds both calls on paper; what they have to be kept from is the issue slots (75% busy in the
// append, 54 to 61% in reading). 20,011 tokens of 8 heads from bf16 into 8 bits 26 us, 4.7 TB/s; 32,299 back
// 31 us, 6.4 TB/s; 64,000 out of 4 bits 54 us, 6.1 TB/s.
#include <type_traits>

#include "device.cuh"
#include "kv.cuh"

namespace stepq {
namespace kv {

constexpr int kWarps = 4, kRows = 4;

struct RowsArgs {
    Pages pg;
    const int32_t *starts, *cu;
    int B, tokens, each, warps;     // each: tokens a warp, where heads are few; warps: that have rows
    void *k, *v;                    // read only by the append
    int64_t ks, vs;
};

// The sequence of packed row i: the last whose first row is not above it. Bounds out of order come out as the
// sequence that the halving ends at; the caller checks that it holds the row.
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

// Eight channels of a row as they lie in memory, and as pairs of fp32.
template <class T> struct alignas(16) Eight { T e[8]; };
__device__ __forceinline__ void pairs(const Eight<float> &v, uint64_t (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = f2(v.e[2 * i], v.e[2 * i + 1]);
}
template <class T>
__device__ __forceinline__ void pairs(const Eight<T> &v, uint64_t (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = f2(la::to_f32(v.e[2 * i]), la::to_f32(v.e[2 * i + 1]));
}
template <class T>
__device__ __forceinline__ void store8(T *p, const uint64_t (&x)[4]) {
    if (sizeof(T) == 4) {
        ((float4 *)p)[0] = make_float4(f2lo(x[0]), f2hi(x[0]), f2lo(x[1]), f2hi(x[1]));
        ((float4 *)p)[1] = make_float4(f2lo(x[2]), f2hi(x[2]), f2lo(x[3]), f2hi(x[3]));
    } else {
        la::Vec<T, 8> v;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            v.e[2 * i] = la::from_f32<T>(f2lo(x[i]));
            v.e[2 * i + 1] = la::from_f32<T>(f2hi(x[i]));
        }
        *(la::Vec<T, 8> *)p = v;
    }
}

// Reports bounds that are not ascending within [0, tokens]: warp w behind those that have rows looks at the 32
// sequences from 32 w on. (By the warps that have rows, 20,011 tokens into 8 bits and back took 56.9 us, so 56.3.)
__device__ __forceinline__ void check_bounds(const RowsArgs &a, int w, int lane) {
    const long long j = 32ll * w + lane;
    if (!a.cu || blockIdx.y > 0 || j >= a.B) return;
    const int first = a.cu[j], next = a.cu[j + 1];
    if (first < 0 || next < first || next > a.tokens) raise_error(a.pg.err, STEPQ_ERR_ARG);
}

// Where a token's rows go: its page and place, or page -1. Sequence b holds it, or one behind b.
struct Place { int page, slot; };
__device__ __forceinline__ Place place_in(const RowsArgs &a, int b, int i, bool report) {
    int first;
    if (a.cu) {
        first = a.cu[b];
        int next = a.cu[b + 1];
        while (i >= next && b + 1 < a.B) {
            first = next;
            next = a.cu[++b + 1];
        }
        if (i < first || i >= next || first < 0 || next > a.tokens) return {-1, 0};
    } else {
        const int each = a.tokens / a.B;
        b = i / each;
        first = b * each;
    }
    const int start = a.starts[b];
    const long long pos = (long long)start + (i - first);
    if (start < 0 || (pos >> a.pg.shift) >= a.pg.width) {
        if (report) raise_error(a.pg.err, STEPQ_ERR_SLOT_RANGE);
        return {-1, 0};
    }
    const int page = a.pg.table[b * a.pg.table_stride + (pos >> a.pg.shift)];
    if (page < 0 || page >= a.pg.n_pages) {
        if (report) raise_error(a.pg.err, STEPQ_ERR_SLOT_RANGE);
        return {-1, 0};
    }
    return {page, a.pg.slot((int)pos)};
}

// A quotient a / s by one correction: t = a y with y near 1 / s, then t + (a - t s) y, whose sum is rounded
// once (P. Markstein, Computation of elementary functions on the IBM RISC System/6000, 1990). With y
// within 2^-22 that sum is a / s up to 2^-44 of it. For s of 11 bits and a of 24 no quotient other than
// a rounding border itself is so near one (a - m s is a multiple of 2^-36 of a for every border m of
// 25 bits, and is not zero: m s has more bits than a), so the result is the rounded quotient.
__device__ __forceinline__ float quotient(float a, float s, float y) {
    const float t = a * y;
    return fmaf(fmaf(-t, s, a), y, t);
}
__device__ __forceinline__ float reciprocal_near(float s) {   // 1 unit in 2^-23
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(s));
    return y;
}

// The bits of the largest magnitude of a lane's eight values as an fp32 (NaN is above all): as
// unsigned numbers magnitudes are ordered, two of 16 bits at a time.
template <class T>
__device__ __forceinline__ uint32_t magnitude(const Eight<T> &v, uint32_t most) {
    const uint4 w = *(const uint4 *)&v;
    const uint32_t m = 0x7fff7fffu, t = __vimax3_u16x2(w.x & m, w.y & m, w.z & m);
    return __vimax3_u16x2(t, w.w & m, most);
}
__device__ __forceinline__ uint32_t magnitude(const Eight<float> &v, uint32_t most) {
#pragma unroll
    for (int e = 0; e < 8; e++) most = max(most, __float_as_uint(v.e[e]) & 0x7fffffffu);
    return most;
}
template <class T, int L>
__device__ __forceinline__ float row_magnitude(const Eight<T> &v, bool on) {
    uint32_t most = on ? magnitude(v, 0u) : 0u;
#pragma unroll
    for (int o = 1; o < L; o *= 2) {
        const uint32_t x = __shfl_xor_sync(0xffffffffu, most, o);
        most = sizeof(T) == 4 ? max(most, x) : __vmaxu2(most, x);
    }
    if (sizeof(T) == 4) return __uint_as_float(most);
    const uint16_t top = (uint16_t)max(most & 0xffffu, most >> 16);
    return la::to_f32(*(const T *)&top);
}

// A lane's eight channels c of a row into the page: all lanes of a warp call it, those with `on` have a row.
template <int F, int D, class T>
__device__ __forceinline__ void put_row(const Eight<T> &in, bool on, uint8_t *row, uint8_t *scale, int c) {
    constexpr int L = D / 8;
    if (!coded(F)) {
        using C = typename std::conditional<F == STEPQ_KV_BF16, la::bf16, la::f16>::type;
        uint64_t x[4];
        pairs(in, x);
        if (on) store8<C>((C *)row + 8 * c, x);
        return;
    }
    uint64_t x[4];
    if (on) pairs(in, x);
    else x[0] = x[1] = x[2] = x[3] = 0;
    constexpr float q = F == STEPQ_KV_INT8 ? 127.f : 7.f;
    constexpr int half = F == STEPQ_KV_INT8 ? 128 : 8;
    float top = row_magnitude<T, L>(in, on);
    const bool far = !(top <= 65504.f * q);
    if (__any_sync(0xffffffffu, far)) {
        // a scale at its bound, or values that are not finite: NaN becomes zero, the others are clamped
        top = 0.f;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float t = e & 1 ? f2hi(x[e / 2]) : f2lo(x[e / 2]);
            v[e] = t == t ? t : 0.f;
            top = fmaxf(top, fabsf(v[e]));
        }
#pragma unroll
        for (int o = 1; o < L; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        top = fminf(top, 65504.f * q);
#pragma unroll
        for (int e = 0; e < 4; e++)
            x[e] = f2(fminf(fmaxf(v[2 * e], -top), top), fminf(fmaxf(v[2 * e + 1], -top), top));
    }
    const uint16_t sb = f16_bits(fmaxf(quotient(top, q, 1.f / q), kF16Min));
    const float s = f16_val(sb), y = reciprocal_near(s);
    // Quotients plus 1.5 2^23 + 2^(b-1): the sum's lowest bits are the code. |x| <= top, so that
    // no quotient is above q by more than the scale's rounding.
    constexpr uint32_t magic = 0x4b400000u + half;
    uint64_t u[4];
    const uint64_t ss = f2s(-s), yy = f2s(y);
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const uint64_t t = fmul2(x[e], yy);
        u[e] = fadd2(ffma2(ffma2(t, ss, x[e]), yy, t), f2s(12582912.f + half));
    }
    if (!on) return;
    auto code = [&](int e) { return (uint32_t)(u[e >> 1] >> (32 * (e & 1))); };
    if (F == STEPQ_KV_INT8) {
        uint2 w;
        w.x = __byte_perm(__byte_perm(code(0), code(1), 0x0040), __byte_perm(code(2), code(3), 0x0040), 0x5410);
        w.y = __byte_perm(__byte_perm(code(4), code(5), 0x0040), __byte_perm(code(6), code(7), 0x0040), 0x5410);
        ((uint2 *)row)[c] = w;
    } else {
        // what stands above the codes adds up to a constant (mod 2^32)
        uint32_t w = code(7);
#pragma unroll
        for (int e = 6; e >= 0; e--) w = w * 16u + code(e);
        ((uint32_t *)row)[c] = w - (magic - half) * 0x11111111u;
    }
    if (c == 0) *(uint16_t *)scale = sb;
}

// And back: eight channels as they lie in the page, to dst.
template <int F> using Held = la::Vec<uint32_t, bits_of(F) / 4>;
template <int F, class T>
__device__ __forceinline__ void take_row(const Held<F> &w, uint16_t scale, T *dst) {
    using C = typename std::conditional<F == STEPQ_KV_BF16, la::bf16, la::f16>::type;
    uint64_t x[4];
    if constexpr (!coded(F)) {
        pairs(*(const Eight<C> *)&w, x);
    } else {
        // 2^23 + u 2^k less 2^23 + 2^(b-1) 2^k is exact, and so is s 2^-k
        const float s = f16_val(scale);
#pragma unroll
        for (int e = 0; e < 4; e++) {
            if constexpr (F == STEPQ_KV_INT8) {
                const uint32_t v = w.e[e / 2];
                x[e] = u2pair(__byte_perm(v, 0x4b000000u, 0x7650 + 2 * (e & 1)), __byte_perm(v, 0x4b000000u, 0x7651 + 2 * (e & 1)));
                x[e] = fmul2(fadd2(x[e], f2s(-8388736.f)), f2s(s));
            } else {
                const uint32_t v = e < 2 ? w.e[0] : w.e[0] >> 16;
                constexpr float pow16[4] = {1.f, 16.f, 256.f, 4096.f};
                const int k = 2 * (e & 1);
                x[e] = u2pair(and_or(v, 15u << (4 * k), 0x4b000000u), and_or(v, 240u << (4 * k), 0x4b000000u));
                x[e] = fadd2(x[e], f2(-8388608.f - 8.f * pow16[k], -8388608.f - 8.f * pow16[k + 1]));
                x[e] = fmul2(x[e], f2(s * (1.f / pow16[k]), s * (1.f / pow16[k + 1])));
            }
        }
    }
    store8<T>(dst, x);
}

// A lane's rows: token i, K or V (part), heads h0 + n * PER, channels 8 c on.
template <int D>
struct Mine {
    static constexpr int L = D / 8, PER = 32 / L;
    int i, lane, c, part, h0;
    __device__ __forceinline__ Mine() {
        i = blockIdx.x * kWarps + (threadIdx.x >> 5);
        lane = threadIdx.x & 31;
        c = lane % L;
        part = blockIdx.y & 1;
        h0 = (blockIdx.y >> 1) * PER * kRows + lane / L;
    }
    __device__ __forceinline__ Place place(const RowsArgs &a) const {
        return place_in(a, a.cu ? find_sequence(a.cu, a.B, i, lane) : 0, i, lane == 0);
    }
};

template <int F, int D, class T>
__global__ void __launch_bounds__(32 * kWarps) kv_append_kernel(RowsArgs a) {
    constexpr int RB = row_bytes(F, D);
    const Mine<D> m;
    griddep_wait();
    griddep_launch();
    if (m.i >= a.tokens) return check_bounds(a, m.i - a.tokens, m.lane);
    const T *src = (const T *)(m.part ? a.v : a.k) + m.i * (m.part ? a.vs : a.ks) + m.h0 * D + 8 * m.c;
    Eight<T> in[kRows];
#pragma unroll
    for (int n = 0; n < kRows; n++)
        if (m.h0 + n * m.PER < a.pg.n_heads) in[n] = *(const Eight<T> *)(src + n * m.PER * D);
    const Place p = m.place(a);
    if (p.page < 0) return;
    uint8_t *seg = a.pg.at(p.page, m.h0);
    const int pt = 1 << a.pg.shift, at = (m.part * pt + p.slot) * RB, at_scale = 2 * pt * RB + 2 * (m.part * pt + p.slot);
#pragma unroll
    for (int n = 0; n < kRows; n++, seg += m.PER * a.pg.segment) {
        if (m.h0 - m.lane / m.L + n * m.PER >= a.pg.n_heads) return;         // no lane has a row
        put_row<F, D, T>(in[n], m.h0 + n * m.PER < a.pg.n_heads, seg + at, seg + at_scale, m.c);
    }
}

template <int F, int D, class T>
__global__ void __launch_bounds__(32 * kWarps) kv_read_kernel(RowsArgs a) {
    constexpr int RB = row_bytes(F, D);
    const Mine<D> m;
    griddep_wait();
    griddep_launch();
    if (m.i >= a.tokens) return check_bounds(a, m.i - a.tokens, m.lane);
    const Place p = m.place(a);
    if (p.page < 0) return;
    const uint8_t *seg = a.pg.at(p.page, m.h0);
    const int pt = 1 << a.pg.shift, at = (m.part * pt + p.slot) * RB, at_scale = 2 * pt * RB + 2 * (m.part * pt + p.slot);
    Held<F> w[kRows];
    uint16_t sb[kRows];
#pragma unroll
    for (int n = 0; n < kRows; n++, seg += m.PER * a.pg.segment)
        if (m.h0 + n * m.PER < a.pg.n_heads) {
            w[n] = ((const Held<F> *)(seg + at))[m.c];
            if (coded(F)) sb[n] = *(const uint16_t *)(seg + at_scale);
        }
    T *dst = (T *)(m.part ? a.v : a.k) + m.i * (m.part ? a.vs : a.ks) + m.h0 * D + 8 * m.c;
#pragma unroll
    for (int n = 0; n < kRows; n++) {
        if (m.h0 + n * m.PER >= a.pg.n_heads) return;
        take_row<F, T>(w[n], sb[n], dst + n * m.PER * D);
    }
}

// The same for prompts where heads are so few that they would leave half of a warp without a row: a
// warp takes a.each tokens, rows n * PER + lane / L of their (token, head). 44,691 tokens of one head
// into 4 bits and back 30 us, a token a warp 50.
template <int D>
struct Few {
    static constexpr int L = D / 8, PER = 32 / L;
    int c, part, token[kRows], head[kRows];
    bool on[kRows];
    Place p[kRows];
    __device__ __forceinline__ Few(const RowsArgs &a, int warp) {
        const int lane = threadIdx.x & 31, first = warp * a.each, H = a.pg.n_heads;
        c = lane % L;
        part = blockIdx.y;
        const int b = a.cu ? find_sequence(a.cu, a.B, first, lane) : 0;
#pragma unroll
        for (int n = 0; n < kRows; n++) {
            const int row = n * PER + lane / L;
            token[n] = first + row / H;
            head[n] = row % H;
            on[n] = row < a.each * H && token[n] < a.tokens;
            p[n] = {-1, 0};
            if (on[n]) p[n] = place_in(a, b, token[n], c == 0);
            on[n] = p[n].page >= 0;
        }
    }
};

template <int F, int D, class T>
__global__ void __launch_bounds__(32 * kWarps) kv_append_few_kernel(RowsArgs a) {
    constexpr int RB = row_bytes(F, D);
    griddep_wait();
    griddep_launch();
    const int warp = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (warp >= a.warps) return check_bounds(a, warp - a.warps, threadIdx.x & 31);
    const Few<D> m(a, warp);
    const T *src = (const T *)(m.part ? a.v : a.k) + 8 * m.c;
    const int64_t stride = m.part ? a.vs : a.ks;
    Eight<T> in[kRows];
#pragma unroll
    for (int n = 0; n < kRows; n++)
        if (m.on[n]) in[n] = *(const Eight<T> *)(src + m.token[n] * stride + m.head[n] * D);
    const int pt = 1 << a.pg.shift;
#pragma unroll
    for (int n = 0; n < kRows; n++) {
        uint8_t *seg = m.on[n] ? a.pg.at(m.p[n].page, m.head[n]) : a.pg.base;
        const int at = m.part * pt + m.p[n].slot;
        put_row<F, D, T>(in[n], m.on[n], seg + at * RB, seg + 2 * pt * RB + 2 * at, m.c);
    }
}

template <int F, int D, class T>
__global__ void __launch_bounds__(32 * kWarps) kv_read_few_kernel(RowsArgs a) {
    constexpr int RB = row_bytes(F, D);
    griddep_wait();
    griddep_launch();
    const int warp = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (warp >= a.warps) return check_bounds(a, warp - a.warps, threadIdx.x & 31);
    const Few<D> m(a, warp);
    const int pt = 1 << a.pg.shift;
    Held<F> w[kRows];
    uint16_t sb[kRows];
#pragma unroll
    for (int n = 0; n < kRows; n++)
        if (m.on[n]) {
            const uint8_t *seg = a.pg.at(m.p[n].page, m.head[n]);
            const int at = m.part * pt + m.p[n].slot;
            w[n] = ((const Held<F> *)(seg + at * RB))[m.c];
            if (coded(F)) sb[n] = *(const uint16_t *)(seg + 2 * pt * RB + 2 * at);
        }
    T *dst = (T *)(m.part ? a.v : a.k) + 8 * m.c;
    const int64_t stride = m.part ? a.vs : a.ks;
#pragma unroll
    for (int n = 0; n < kRows; n++)
        if (m.on[n]) take_row<F, T>(w[n], sb[n], dst + m.token[n] * stride + m.head[n] * D);
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
    const int at_once = 256 / cfg->head_dim, per_warp = kv::kRows * at_once;
    const bool few = 2 * cfg->n_heads <= at_once && tokens >= 8192;      // enough to fill the GPU
    a.each = few ? per_warp / cfg->n_heads : 1;
    a.warps = (tokens + a.each - 1) / a.each;
    const int64_t warps = a.warps + (cu ? (B + 31ll) / 32 : 0);          // some for the bounds
    const dim3 grid((unsigned)((warps + kv::kWarps - 1) / kv::kWarps),
                    2 * ((cfg->n_heads + per_warp - 1) / per_warp));
    return kv::by_layout(cfg, [&](auto f, auto d) {
        return la::by_type(rows->dtype, [&](auto t) {
            constexpr int F = decltype(f)::value, D = decltype(d)::value;
            using T = decltype(t);
            auto *kernel = append ? kv::kv_append_kernel<F, D, T> : kv::kv_read_kernel<F, D, T>;
            if constexpr (D <= 128)
                if (few) kernel = append ? kv::kv_append_few_kernel<F, D, T> : kv::kv_read_few_kernel<F, D, T>;
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
