// Shared parts of the decayed linear-attention kernels and the group norm: element types,
// the activation and the norm's arguments.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "async.cuh"
#include "internal.h"

namespace stepq {
namespace la {

using bf16 = __nv_bfloat16;
using f16 = __half;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(f16 x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ f16 from_f32<f16>(float x) { return __float2half_rn(x); }

// N consecutive elements that one vector of up to 16 bytes holds.
template <class T, int N> struct alignas(N * sizeof(T)) Vec { T e[N]; };
template <class T, int N>
__device__ __forceinline__ void load_vec(const T *p, float (&x)[N]) {
    const Vec<T, N> v = *(const Vec<T, N> *)p;
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = to_f32(v.e[i]);
}
template <class T, int N>
__device__ __forceinline__ void store_vec(T *p, const float (&x)[N]) {
    Vec<T, N> v;
#pragma unroll
    for (int i = 0; i < N; i++) v.e[i] = from_f32<T>(x[i]);
    *(Vec<T, N> *)p = v;
}

// stepq_norm with z's type erased; on = 0: y leaves as it is.
struct NormArgs {
    const float *w, *b;
    const void *z;
    int64_t z_stride;
    float eps;
    int act, center, shared, on;
};
inline NormArgs norm_args(const stepq_norm *n) {
    if (!n) return NormArgs{};
    return {n->weight, n->bias, n->z, n->z_stride, n->eps, n->act, n->center, n->shared, 1};
}

// act(x). Vectors of 16 bits leave a result 8 or 11 bits: the fast exponential and reciprocal (a
// few units in 2^-23, and 2^-24 |x| from the exponent's product) are far below that. fp32 results
// take expf and the rounded quotient.
__device__ __forceinline__ float fast_sigmoid(float scaled) {  // of x, scaled = -x / ln 2
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(scaled));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
}
constexpr float kToExponent = -1.44269504f;

template <class T>
__device__ __forceinline__ float activation(int act, float x) {
    if (act == STEPQ_ACT_NONE) return x;
    if (sizeof(T) == 2) return (act == STEPQ_ACT_SIGMOID ? 1.f : x) * fast_sigmoid(x * kToExponent);
    return (act == STEPQ_ACT_SIGMOID ? 1.f : x) / (1.f + expf(-x));
}

// A pair of a 16-bit type's.
__device__ __forceinline__ uint64_t activation2(int act, uint64_t x) {
    if (act == STEPQ_ACT_NONE) return x;
    const uint64_t t = fmul2(x, f2s(kToExponent)), r = f2(fast_sigmoid(f2lo(t)), fast_sigmoid(f2hi(t)));
    return act == STEPQ_ACT_SIGMOID ? r : fmul2(x, r);
}

// out = u act(z) or act(u) of one channel, u = xc * rstd * w + b with xc = x - mean.
template <class T>
__device__ __forceinline__ float norm_out(const NormArgs &n, float xc, float rstd, float w, float b, float z) {
    const float u = fmaf(xc * rstd, w, b), a = activation<T>(n.act, n.z ? z : u);
    return n.z ? u * a : a;
}

__device__ __forceinline__ float rstd_of(float var, float eps) { return rsqrtf(var + eps); }

// The affine parameters of lane l's channels 4 l .. 4 l + 3 of head h.
struct HeadAffine {
    float w[4], b[4];
    __device__ __forceinline__ HeadAffine(const NormArgs &n, int h, int lane) {
        const int c = 4 * lane + (n.shared ? 0 : h * kD);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            w[i] = n.w ? n.w[c + i] : 1.f;
            b[i] = n.b ? n.b[c + i] : 0.f;
        }
    }
};

// One head's readouts of N tokens in a warp, lane l holding channels 4 l .. 4 l + 3 (z: of the
// gate, if there is one). Mean m and centred sum of squares q of ever larger parts in one
// butterfly: of two parts of n values each, m = (m1 + m2) / 2 and q = q1 + q2 + (m1 - m2)^2 n / 2,
// which cancels nothing; the sum of squares about zero is q + 128 m^2.
template <class T, int N>
__device__ __forceinline__ void norm_head(const NormArgs &n, const HeadAffine &p, const Vec<T, 4> *z, float (&y)[N][4]) {
    float m[N], q[N];
#pragma unroll
    for (int i = 0; i < N; i++) {
        m[i] = 0.25f * ((y[i][0] + y[i][1]) + (y[i][2] + y[i][3]));
        q[i] = 0.f;
#pragma unroll
        for (int e = 0; e < 4; e++) q[i] = fmaf(y[i][e] - m[i], y[i][e] - m[i], q[i]);
    }
    float half = 2.f;                                       // of the values in a part
#pragma unroll
    for (int o = 1; o < 32; o *= 2, half *= 2.f)
#pragma unroll
        for (int i = 0; i < N; i++) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m[i], o), d = m[i] - m2;
            q[i] += __shfl_xor_sync(0xffffffffu, q[i], o);
            q[i] = fmaf(d * half, d, q[i]);
            m[i] = 0.5f * (m[i] + m2);
        }
#pragma unroll
    for (int i = 0; i < N; i++) {
        const float c = n.center ? m[i] : 0.f;
        const float r = rstd_of(fmaf(m[i] - c, m[i], q[i] * (1.f / kD)), n.eps);
#pragma unroll
        for (int e = 0; e < 4; e++) y[i][e] = norm_out<T>(n, y[i][e] - c, r, p.w[e], p.b[e], to_f32(z[i].e[e]));
    }
}

// Runs f(T{}) for the element type of a call.
template <class F>
inline stepq_status by_type(int dtype, F &&f) {
    return dtype == STEPQ_F32 ? f(float{}) : dtype == STEPQ_BF16 ? f(bf16{}) : f(f16{});
}

}  // namespace la
}  // namespace stepq
