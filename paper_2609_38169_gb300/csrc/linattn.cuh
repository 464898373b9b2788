// Shared parts of the decayed linear-attention kernels and the group norm: element types,
// the activation and the norm's arguments.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

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

// Vectors of 16 bits leave a result 8 or 11 bits: the fast exponential and quotient (a few
// units in 2^-23, and 2^-24 |x| from the exponent's product) are far below that. fp32
// results take expf and the rounded quotient.
template <class T>
__device__ __forceinline__ float activation(int act, float x) {
    if (act == STEPQ_ACT_NONE) return x;
    const float num = act == STEPQ_ACT_SILU ? x : 1.f;
    if (sizeof(T) == 2) return __fdividef(num, 1.f + __expf(-x));
    return num / (1.f + expf(-x));
}

// out = u act(z) or act(u) of one channel, u = xc * rstd * w + b with xc = x - mean.
template <class T>
__device__ __forceinline__ float norm_out(const NormArgs &n, float xc, float rstd, float w, float b, float z) {
    const float u = fmaf(xc * rstd, w, b);
    return n.z ? u * activation<T>(n.act, z) : activation<T>(n.act, u);
}

__device__ __forceinline__ float rstd_of(float var, float eps) { return rsqrtf(var + eps); }

// One head's readouts of a token in a warp, lane l holding channels N l .. N l + N - 1 of N * 32.
// h: the head; row: the token's row (of z).
template <class T, int N>
__device__ __forceinline__ void norm_head(const NormArgs &n, int h, int64_t row, int lane, float (&y)[N]) {
    constexpr int W = 32 * N;
    float m = 0.f;
    if (n.center) {
#pragma unroll
        for (int i = 0; i < N; i++) m += y[i];
#pragma unroll
        for (int o = 16; o; o >>= 1) m += __shfl_xor_sync(0xffffffffu, m, o);
        m *= 1.f / W;
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < N; i++) {
        y[i] -= m;
        ss = fmaf(y[i], y[i], ss);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float r = rstd_of(ss * (1.f / W), n.eps);
    const int c = N * lane, pc = c + (n.shared ? 0 : h * W);
    float z[N] = {};
    if (n.z) load_vec<T, N>((const T *)n.z + row * n.z_stride + (int64_t)h * W + c, z);
#pragma unroll
    for (int i = 0; i < N; i++)
        y[i] = norm_out<T>(n, y[i], r, n.w ? n.w[pc + i] : 1.f, n.b ? n.b[pc + i] : 0.f, z[i]);
}

// Runs f(T{}) for the element type of a call.
template <class F>
inline stepq_status by_type(int dtype, F &&f) {
    return dtype == STEPQ_F32 ? f(float{}) : dtype == STEPQ_BF16 ? f(bf16{}) : f(f16{});
}

}  // namespace la
}  // namespace stepq
