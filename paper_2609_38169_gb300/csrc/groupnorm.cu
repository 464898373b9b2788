// Group norm of rows of channels with an activation or a gate (stepq_norm).
//
// A warp per group: the group's values stay in registers between the mean, the centred
// sum of squares (fp32, two passes over registers: no cancellation) and the output, so x and
// z are read once and out written once; HBM bounds it. Groups too wide for that are read
// again from the cache.
#include "async.cuh"
#include "device.cuh"
#include "linattn.cuh"

namespace stepq {
namespace la {

struct GroupArgs {
    const void *x;
    void *out;
    int64_t x_stride, out_stride, items;      // item = row * groups + group
    int groups, width;
    NormArgs norm;
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// V elements a vector, K vectors a lane (K = 0: any number, read again for each pass).
template <class T, int V, int K>
__global__ void __launch_bounds__(256) group_norm_kernel(GroupArgs a) {
    griddep_wait();
    griddep_launch();
    const int l = threadIdx.x & 31, vecs = a.width / V;
    const float inv = 1.f / (float)a.width;
    const int64_t warps = (int64_t)gridDim.x * 8;
    for (int64_t it = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); it < a.items; it += warps) {
        const int64_t row = it / a.groups;
        const int grp = (int)(it - row * a.groups);
        const int64_t c0 = (int64_t)grp * a.width;
        const T *x = (const T *)a.x + row * a.x_stride + c0;
        const T *z = a.norm.z ? (const T *)a.norm.z + row * a.norm.z_stride + c0 : nullptr;
        T *out = (T *)a.out + row * a.out_stride + c0;
        const int64_t p0 = a.norm.shared ? 0 : c0;
        const auto emit = [&](int e, const float (&xc)[V], float r) {
            float zv[V] = {}, o[V];
            if (z) load_vec<T, V>(z + e, zv);
#pragma unroll
            for (int i = 0; i < V; i++)
                o[i] = norm_out<T>(a.norm, xc[i], r, a.norm.w ? a.norm.w[p0 + e + i] : 1.f,
                                   a.norm.b ? a.norm.b[p0 + e + i] : 0.f, zv[i]);
            store_vec<T, V>(out + e, o);
        };
        if constexpr (K > 0) {
            float v[K][V];
            float m = 0.f, ss = 0.f;
#pragma unroll
            for (int n = 0; n < K; n++) {
                const int e = V * (l + 32 * n);
                if (l + 32 * n < vecs) load_vec<T, V>(x + e, v[n]);
                else
#pragma unroll
                    for (int i = 0; i < V; i++) v[n][i] = 0.f;
#pragma unroll
                for (int i = 0; i < V; i++) m += v[n][i];
            }
            m = a.norm.center ? warp_sum(m) * inv : 0.f;
#pragma unroll
            for (int n = 0; n < K; n++)
#pragma unroll
                for (int i = 0; i < V; i++) {
                    v[n][i] = l + 32 * n < vecs ? v[n][i] - m : 0.f;
                    ss = fmaf(v[n][i], v[n][i], ss);
                }
            const float r = rstd_of(warp_sum(ss) * inv, a.norm.eps);
#pragma unroll
            for (int n = 0; n < K; n++)
                if (l + 32 * n < vecs) emit(V * (l + 32 * n), v[n], r);
        } else {
            float v[V], m = 0.f, ss = 0.f;
            if (a.norm.center) {
                for (int n = l; n < vecs; n += 32) {
                    load_vec<T, V>(x + V * n, v);
#pragma unroll
                    for (int i = 0; i < V; i++) m += v[i];
                }
                m = warp_sum(m) * inv;
            }
            for (int n = l; n < vecs; n += 32) {
                load_vec<T, V>(x + V * n, v);
#pragma unroll
                for (int i = 0; i < V; i++) ss = fmaf(v[i] - m, v[i] - m, ss);
            }
            const float r = rstd_of(warp_sum(ss) * inv, a.norm.eps);
            for (int n = l; n < vecs; n += 32) {
                load_vec<T, V>(x + V * n, v);
#pragma unroll
                for (int i = 0; i < V; i++) v[i] -= m;
                emit(V * n, v, r);
            }
        }
    }
}

}  // namespace la

stepq_status launch_group_norm(int dtype, int64_t rows, int groups, int width, const void *x, int64_t x_stride,
                               void *out, int64_t out_stride, const stepq_norm *norm, cudaStream_t s) {
    la::GroupArgs a{};
    a.x = x; a.out = out;
    a.x_stride = x_stride; a.out_stride = out_stride;
    a.items = rows * groups;
    a.groups = groups; a.width = width;
    a.norm = la::norm_args(norm);
    const int64_t most = 16ll * sm_count(), ctas = (a.items + 7) / 8;
    const int grid = (int)(ctas < most ? ctas : most);
    return la::by_type(dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / sizeof(T);
        const auto on = [&](const void *p, int64_t stride) {
            return !p || ((uintptr_t)p % 16 == 0 && stride % V == 0);
        };
        if (width % V == 0 && on(x, x_stride) && on(out, out_stride) && on(norm->z, norm->z_stride)) {
            const int k = (width / V + 31) / 32;
            if (k <= 1) return launch_overlapped(la::group_norm_kernel<T, V, 1>, grid, 256, 0, s, a);
            if (k <= 4) return launch_overlapped(la::group_norm_kernel<T, V, 4>, grid, 256, 0, s, a);
            return launch_overlapped(la::group_norm_kernel<T, V, 0>, grid, 256, 0, s, a);
        }
        if (width <= 256) return launch_overlapped(la::group_norm_kernel<T, 1, 8>, grid, 256, 0, s, a);
        return launch_overlapped(la::group_norm_kernel<T, 1, 0>, grid, 256, 0, s, a);
    });
}

}  // namespace stepq
