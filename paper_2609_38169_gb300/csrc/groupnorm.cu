// Group norm of rows of channels with an activation or a gate (stepq_norm).
//
// A team of 1 to 32 lanes, or a CTA, per group: the group's values stay in registers between the
// mean, the centred sum of squares (fp32, two passes over registers: no cancellation) and the
// output, so x and z are read once and out written once, and HBM bounds it: 65536 rows of 32
// gated groups of 128 in bf16 take 241 us, 6.7 TB/s. A thread copies its own vectors two groups
// ahead into its own places of shared memory (one ahead in registers: 485 us, a warp a group with
// none: 719; places for four: 5% slower).
#include "async.cuh"
#include "device.cuh"
#include "linattn.cuh"

#include <numeric>
#include <type_traits>

namespace stepq {
namespace la {

struct GroupArgs {
    const void *x;
    void *out;
    int64_t x_stride, out_stride, items;      // item = row * groups + group
    int groups, width, lanes;                 // lanes: of a team in a warp
    int fixed;                                // a team's items are of one group
    NormArgs norm;
};

constexpr int kWarpTeamThreads = 256, kCtaTeamThreads = 512;

// The elements as fp32 pairs, and back: 16-bit ones a word at a time, half the byte moves of one
// by one.
template <class T, int V>
__device__ __forceinline__ void to_pairs(const Vec<T, V> &x, uint64_t (&p)[V / 2]) {
    const uint32_t *word = (const uint32_t *)x.e;
#pragma unroll
    for (int i = 0; i < V / 2; i++) {
        if constexpr (std::is_same<T, bf16>::value) {
            p[i] = u2pair(word[i] << 16, word[i] & 0xFFFF0000u);
        } else if constexpr (std::is_same<T, f16>::value) {
            const float2 f = __half22float2(*(const __half2 *)&word[i]);
            p[i] = f2(f.x, f.y);
        } else {
            p[i] = f2(x.e[2 * i], x.e[2 * i + 1]);
        }
    }
}
template <class T, int V>
__device__ __forceinline__ void from_pairs(const uint64_t (&p)[V / 2], Vec<T, V> &x) {
#pragma unroll
    for (int i = 0; i < V / 2; i++) {
        const float lo = f2lo(p[i]), hi = f2hi(p[i]);
        if constexpr (std::is_same<T, bf16>::value) {
            *(__nv_bfloat162 *)&x.e[2 * i] = __floats2bfloat162_rn(lo, hi);
        } else if constexpr (std::is_same<T, f16>::value) {
            *(__half2 *)&x.e[2 * i] = __floats2half2_rn(lo, hi);
        } else {
            x.e[2 * i] = lo;
            x.e[2 * i + 1] = hi;
        }
    }
}
template <int V>
__device__ __forceinline__ void affine_pairs(const float *p, float other, uint64_t (&x)[V / 2]) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        const ulonglong2 t = p ? *(const ulonglong2 *)(p + i) : make_ulonglong2(f2s(other), f2s(other));
        x[i / 2] = t.x;
        x[i / 2 + 1] = t.y;
    }
}

// Sum over a team: some lanes of a warp, or the CTA.
template <bool CTA>
__device__ __forceinline__ float team_sum(float x, int lanes, float (*part)[kCtaTeamThreads / 32], int &turn) {
    for (int o = CTA ? 16 : lanes / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if constexpr (CTA) {
        float *p = part[turn];                               // two in turn: one barrier a sum
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) p[threadIdx.x >> 5] = x;
        __syncthreads();
        x = 0.f;
        for (int i = 0; i < (int)blockDim.x / 32; i++) x += p[i];
    }
    return x;
}

// out = act(z) u or act(u) (stepq_norm) of a vector.
template <class T, int V, bool GATED, int ACT>
__device__ __forceinline__ void emit(T *out, const uint64_t (&u)[V / 2], const Vec<T, V> &zv) {
    uint64_t z[V / 2], o[V / 2];
    to_pairs<T, V>(zv, z);
#pragma unroll
    for (int i = 0; i < V / 2; i++) {
        const uint64_t s = GATED ? z[i] : u[i];
        if constexpr (sizeof(T) == 2) o[i] = activation2(ACT, s);
        else o[i] = f2(activation<T>(ACT, f2lo(s)), activation<T>(ACT, f2hi(s)));
        if (GATED) o[i] = fmul2(u[i], o[i]);
    }
    Vec<T, V> x;
    from_pairs<T, V>(o, x);
    *(Vec<T, V> *)out = x;
}

// f of the call's form (gated, activation) as constants.
template <class F>
__device__ __forceinline__ void by_form(const NormArgs &n, F &&f) {
    using std::integral_constant;
    const auto act = [&](auto gated) {
        if (n.act == STEPQ_ACT_SILU) f(gated, integral_constant<int, STEPQ_ACT_SILU>{});
        else if (n.act == STEPQ_ACT_SIGMOID) f(gated, integral_constant<int, STEPQ_ACT_SIGMOID>{});
        else f(gated, integral_constant<int, STEPQ_ACT_NONE>{});
    };
    if (n.z) act(integral_constant<bool, true>{});
    else act(integral_constant<bool, false>{});
}

// The items of a thread's team: first, and every `step` from there.
struct Items {
    const GroupArgs &a;
    int team;
    int64_t row, rows;                                       // rows: a step's, where a team keeps its group
    int grp;
    __device__ __forceinline__ Items(const GroupArgs &a, int team, int64_t first, int64_t step) : a(a), team(team), rows(step / a.groups) { locate(first); }
    __device__ __forceinline__ void locate(int64_t it) {
        row = (it + team) / a.groups;
        grp = (int)(it + team - row * a.groups);
    }
    __device__ __forceinline__ void advance(int64_t it) {
        if (a.fixed) row += rows;
        else locate(it);
    }
    template <class T> __device__ __forceinline__ const T *x() const { return (const T *)a.x + row * a.x_stride + (int64_t)grp * a.width; }
    template <class T> __device__ __forceinline__ const T *z() const { return (const T *)a.norm.z + row * a.norm.z_stride + (int64_t)grp * a.width; }
    template <class T> __device__ __forceinline__ T *out() const { return (T *)a.out + row * a.out_stride + (int64_t)grp * a.width; }
    __device__ __forceinline__ int affine() const { return a.norm.shared ? 0 : grp * a.width; }
};

// Vectors of 16 bytes, K a thread, copied ahead of their item: two or three a lane of a team in a
// warp, four where the CTA is the team (rows of 4096 in bf16 171 us, with two 183; 7168 113 and 136). The affine parameters stay in
// registers where a team's items have the same. Four times the CTAs that fit: the multiprocessors
// get out of step, and HBM's reads and writes mix (one: 267 us for 241).
constexpr int kDepth = 3, kWaves = 4, kCtaVectors = 4;
constexpr int ring_bytes(int K, int threads) { return kDepth * 2 * K * 16 * threads; }
// CTAs of 256 threads a multiprocessor: what the registers of values and parameters leave (16-bit
// types at three, registers spilled: 20% slower; fp32 at two: 8%).
template <class T>
constexpr int kResident = sizeof(T) == 2 ? 2 : 3;

template <class T, int K, bool CTA>
__global__ void __launch_bounds__(CTA ? kCtaTeamThreads : kWarpTeamThreads, CTA ? 1 : kResident<T>) group_norm_kernel(GroupArgs a) {
    constexpr int V = 16 / sizeof(T), H = V / 2;
    __shared__ float part[2][kCtaTeamThreads / 32];
    extern __shared__ __align__(16) uint8_t ring[];
    int turn = 0;
    griddep_wait();
    griddep_launch();
    const int tid = threadIdx.x, lanes = CTA ? (int)blockDim.x : a.lanes, tl = CTA ? tid : tid & (lanes - 1), vecs = a.width / V;
    const int teams = CTA ? 1 : kWarpTeamThreads / lanes, team = CTA ? 0 : tid / lanes;
    const int leader = CTA ? 0 : (tid & ~31) / lanes;        // the warp's first team
    const float inv = 1.f / (float)a.width;
    const int64_t step = (int64_t)gridDim.x * teams, first = (int64_t)blockIdx.x * teams;
    Items now(a, team, first, step), ahead = now;
    uint64_t w[K][H], b[K][H];
    const auto affine = [&](int p0) {
#pragma unroll
        for (int n = 0; n < K; n++) {
            const int e = tl + lanes * n;
            if (e >= vecs) continue;
            affine_pairs<V>(a.norm.w ? a.norm.w + p0 + V * e : nullptr, 1.f, w[n]);
            affine_pairs<V>(a.norm.b ? a.norm.b + p0 + V * e : nullptr, 0.f, b[n]);
        }
    };
    const bool keep = a.fixed || a.norm.shared;
    if (keep) affine(now.affine());
    const auto place = [&](int stage, int which, int n) {
        return (Vec<T, V> *)(ring + (((stage * 2 + which) * K + n) * (int)blockDim.x + tid) * 16);
    };
    int64_t ahead_it = first;
    const auto fetch = [&](int stage) {
        const bool valid = ahead_it + team < a.items;
        const T *x = ahead.x<T>(), *z = ahead.z<T>();
#pragma unroll
        for (int n = 0; n < K; n++) {
            const int e = tl + lanes * n;
            const bool there = valid && e < vecs;            // else zeros
            cp_async16_or_zero(place(stage, 0, n), there ? x + V * e : (const T *)a.x, there);
            if (a.norm.z) cp_async16_or_zero(place(stage, 1, n), there ? z + V * e : (const T *)a.norm.z, there);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        ahead_it += step;
        ahead.advance(ahead_it);
    };
#pragma unroll 1
    for (int d = 0; d < kDepth - 1; d++) fetch(d);
    int stage = 0;
    for (int64_t it = first; it + leader < a.items; it += step, now.advance(it)) {
        const bool valid = it + team < a.items;              // a warp's teams take their shuffles together
        T *out = now.out<T>();
        Vec<T, V> zv[K];
        uint64_t v[K][H], m2 = 0, q2 = 0;
        asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 2) : "memory");
#pragma unroll
        for (int n = 0; n < K; n++) {
            to_pairs<T, V>(*place(stage, 0, n), v[n]);
            if (a.norm.z) zv[n] = *place(stage, 1, n);
        }
        fetch(stage == 0 ? kDepth - 1 : stage - 1);          // the place read a step ago
        stage = stage + 1 == kDepth ? 0 : stage + 1;
        if (!keep && valid) affine(now.affine());
        float m = 0.f;
        if (a.norm.center) {
#pragma unroll
            for (int n = 0; n < K; n++)
#pragma unroll
                for (int i = 0; i < H; i++) m2 = fadd2(m2, v[n][i]);
            m = team_sum<CTA>(f2lo(m2) + f2hi(m2), lanes, part, turn) * inv;
        }
#pragma unroll
        for (int n = 0; n < K; n++) {
            const uint64_t mm = f2s(tl + lanes * n < vecs ? m : 0.f);
#pragma unroll
            for (int i = 0; i < H; i++) {
                v[n][i] = fsub2(v[n][i], mm);
                q2 = ffma2(v[n][i], v[n][i], q2);
            }
        }
        const uint64_t r = f2s(rstd_of(team_sum<CTA>(f2lo(q2) + f2hi(q2), lanes, part, turn) * inv, a.norm.eps));
#pragma unroll
        for (int n = 0; n < K; n++)
#pragma unroll
            for (int i = 0; i < H; i++) v[n][i] = ffma2(fmul2(v[n][i], r), w[n][i], b[n][i]);
        by_form(a.norm, [&](auto gated, auto act) {
#pragma unroll
            for (int n = 0; n < K; n++)
                if (valid && tl + lanes * n < vecs)
                    emit<T, V, decltype(gated)::value, decltype(act)::value>(out + V * (tl + lanes * n), v[n], zv[n]);
        });
    }
}

// Single elements, at most kScalars a lane of a team: rows that start at no multiple of 16 bytes or
// have groups of no such width. 4099 x 12 groups of 75 in fp32 take 19 us (1.6 TB/s): requests of
// 4 bytes a lane that touch several lines each, the parameters' among them, and some 45
// instructions an element. 8 a lane 21; copied a group ahead in registers 23 to 27.
constexpr int kScalars = 16;

template <class T>
__global__ void __launch_bounds__(kWarpTeamThreads, 4) group_norm_scalars_kernel(GroupArgs a) {
    griddep_wait();
    griddep_launch();
    const int tid = threadIdx.x, lanes = a.lanes, tl = tid & (lanes - 1), team = tid / lanes;
    const int teams = kWarpTeamThreads / lanes, leader = (tid & ~31) / lanes;
    const float inv = 1.f / (float)a.width;
    const int64_t step = (int64_t)gridDim.x * teams, first = (int64_t)blockIdx.x * teams;
    Items now(a, team, first, step);
    float (*no_part)[kCtaTeamThreads / 32] = nullptr;
    int no_turn = 0;
    for (int64_t it = first; it + leader < a.items; it += step, now.advance(it)) {
        const int mine = it + team < a.items ? a.width - tl : 0;   // element tl + n lanes is there for n lanes < mine
        const T *x = now.x<T>() + tl, *z = a.norm.z ? now.z<T>() + tl : nullptr;
        float v[kScalars], zv[kScalars], m = 0.f, ss = 0.f;
#pragma unroll
        for (int n = 0; n < kScalars; n++) {
            v[n] = n * lanes < mine ? to_f32(x[n * lanes]) : 0.f;
            zv[n] = z && n * lanes < mine ? to_f32(z[n * lanes]) : 0.f;
            m += v[n];
        }
        m = a.norm.center ? team_sum<false>(m, lanes, no_part, no_turn) * inv : 0.f;
#pragma unroll
        for (int n = 0; n < kScalars; n++) {
            v[n] = n * lanes < mine ? v[n] - m : 0.f;
            ss = fmaf(v[n], v[n], ss);
        }
        const float r = rstd_of(team_sum<false>(ss, lanes, no_part, no_turn) * inv, a.norm.eps);
        T *out = now.out<T>() + tl;
        const int p0 = now.affine() + tl;
#pragma unroll
        for (int n = 0; n < kScalars; n++) {
            if (n * lanes >= a.width) break;                 // (no lane has one)
            const int e = n * lanes;
            if (e < mine)
                out[e] = from_f32<T>(norm_out<T>(a.norm, v[n], r, a.norm.w ? a.norm.w[p0 + e] : 1.f, a.norm.b ? a.norm.b[p0 + e] : 0.f, zv[n]));
        }
    }
}

// Groups of any width, read again for each pass, a CTA a group.
template <class T, int V>
__global__ void __launch_bounds__(kCtaTeamThreads) group_norm_wide_kernel(GroupArgs a) {
    __shared__ float part[2][kCtaTeamThreads / 32];
    int turn = 0;
    griddep_wait();
    griddep_launch();
    const int threads = blockDim.x, vecs = a.width / V;
    const float inv = 1.f / (float)a.width;
    Items now(a, 0, blockIdx.x, gridDim.x);
    for (int64_t it = blockIdx.x; it < a.items; it += gridDim.x, now.advance(it)) {
        const T *x = now.x<T>(), *z = a.norm.z ? now.z<T>() : nullptr;
        float v[V], m = 0.f, ss = 0.f;
        if (a.norm.center) {
            for (int n = threadIdx.x; n < vecs; n += threads) {
                load_vec<T, V>(x + V * n, v);
#pragma unroll
                for (int i = 0; i < V; i++) m += v[i];
            }
            m = team_sum<true>(m, 32, part, turn) * inv;
        }
        for (int n = threadIdx.x; n < vecs; n += threads) {
            load_vec<T, V>(x + V * n, v);
#pragma unroll
            for (int i = 0; i < V; i++) ss = fmaf(v[i] - m, v[i] - m, ss);
        }
        const float r = rstd_of(team_sum<true>(ss, 32, part, turn) * inv, a.norm.eps);
        const int p0 = now.affine();
        T *out = now.out<T>();
        for (int n = threadIdx.x; n < vecs; n += threads) {
            float zv[V] = {};
            load_vec<T, V>(x + V * n, v);
            if (z) load_vec<T, V>(z + V * n, zv);
#pragma unroll
            for (int i = 0; i < V; i++)
                v[i] = norm_out<T>(a.norm, v[i] - m, r, a.norm.w ? a.norm.w[p0 + V * n + i] : 1.f, a.norm.b ? a.norm.b[p0 + V * n + i] : 0.f, zv[i]);
            store_vec<T, V>(out + V * n, v);
        }
    }
}

// teams: of a CTA; resident: CTAs a multiprocessor.
static stepq_status launch_groups(void (*kernel)(GroupArgs), GroupArgs &a, int teams, int resident, int threads, int smem, cudaStream_t s) {
    const int64_t most = (int64_t)(resident > 0 ? resident : 1) * sm_count(), ctas = (a.items + teams - 1) / teams;
    int grid = (int)(ctas < most ? ctas : most);
    // A grid whose teams keep their group costs an eighth of the CTAs at most.
    const int part = a.groups / std::gcd(a.groups, teams);
    a.fixed = ctas <= most || part * 8ll <= grid;
    if (ctas > most && a.fixed) grid -= grid % part;
    return launch_overlapped(kernel, grid, threads, smem, s, a);
}

template <class T, int K, bool CTA>
static stepq_status launch_vectors(GroupArgs &a, int threads, cudaStream_t s) {
    static SmemOptIn opt_in;
    const auto kernel = group_norm_kernel<T, K, CTA>;
    const stepq_status st = opt_in((const void *)kernel, ring_bytes(K, CTA ? kCtaTeamThreads : threads));
    if (st != STEPQ_OK) return st;
    return launch_groups(kernel, a, CTA ? 1 : threads / a.lanes, CTA ? 256 * kResident<T> / threads : kWaves * kResident<T>,
                         threads, ring_bytes(K, threads), s);
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
    return la::by_type(dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / sizeof(T);
        const auto on = [&](const void *p, int64_t stride) {
            return !p || ((uintptr_t)p % 16 == 0 && stride % V == 0);
        };
        const auto warps = [](int64_t threads) {
            const int64_t n = (threads + 31) / 32 * 32;
            return (int)(n < la::kCtaTeamThreads ? n : la::kCtaTeamThreads);
        };
        const bool vectors = width % V == 0 && on(x, x_stride) && on(out, out_stride) && on(norm->z, norm->z_stride) &&
                             on(norm->weight, 0) && on(norm->bias, 0);
        const int vecs = width / V, pieces = vectors ? vecs : width, a_lane = vectors ? 2 : la::kScalars;
        a.lanes = 1;
        while (a.lanes < 32 && a_lane * a.lanes < pieces) a.lanes *= 2;
        if (vectors && vecs <= 2 * 32) return la::launch_vectors<T, 2, false>(a, la::kWarpTeamThreads, s);
        if (vectors && vecs <= 3 * 32) return la::launch_vectors<T, 3, false>(a, la::kWarpTeamThreads, s);
        if (vectors && vecs <= la::kCtaVectors * la::kCtaTeamThreads)
            return la::launch_vectors<T, la::kCtaVectors, true>(a, warps((vecs + la::kCtaVectors - 1) / la::kCtaVectors), s);
        if (!vectors && width <= la::kScalars * 32)
            return la::launch_groups(la::group_norm_scalars_kernel<T>, a, la::kWarpTeamThreads / a.lanes, 4, la::kWarpTeamThreads, 0, s);
        const int threads = vectors ? la::kCtaTeamThreads : warps(width / la::kScalars);
        return la::launch_groups(vectors ? la::group_norm_wide_kernel<T, V> : la::group_norm_wide_kernel<T, 1>, a, 1,
                                 1024 / threads, threads, 0, s);
    });
}

}  // namespace stepq
