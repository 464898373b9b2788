// Decayed linear attention over prompts, 16 tokens at a time on the tensor cores, every factor a
// sum of bf16 terms: the form for fp32 and fp16 vectors, and for a few tokens of bf16.
//
// With c_t = g_1 .. g_t and w_ts = g_{s+1} .. g_t inside a block of 16 tokens:
//   Y^T = (S_0^T Q^T) diag(c_t) + V^T P^T,   P_ts = w_ts (q_t . k_s), zero for s > t
//   S_16 = c_16 S_0 + U,   U^T = V^T K',   K'_s = w_16s k_s
// A factor is the sum of terms, each the rest of those before rounded to bf16: an fp32 value is three
// exactly, an fp16 value two. Of a product the pairs of terms i and j (from 0) with i + j <= 2 are
// taken; those left out are below 2^-24 of it together. fp16 and bf16: q, k and v are two terms
// or one; S and P are two (2^-17 of each value is lost: the readout is rounded to 2^-12 or 2^-9); K'
// has three here too, since states are kept in fp32. U is formed apart from S and added to it in fp32, smaller
// pairs first: what the tensor core's sums truncate does not add up from block to block.
//
// One CTA of eight warps per segment and head; warp w holds S^T of value columns 16 w .. + 15 in
// registers, laid out as an accumulator of U^T, which is the layout of the left factor S^T too.
// So a block's products need no exchange of the state: only P does, whose sums over the channels
// are split over the warps. That is why these are warp-level products. Out of tensor memory the
// twelve tiles of one chunk's terms take 192 KB of shared memory for 64 tokens, with no room for a
// second chunk beside it; for 32 tokens two would fit, which is not built. Vectors are split into
// their terms once, by the thread that loads them, into swizzled rows of 256 bytes; P is formed a
// block ahead; two barriers a block.
//
// The products' rate and latency bound it (216 of a warp a block in fp32, 160 in fp16; the pipe 79%
// busy where a CTA runs): 16 x 1024 tokens of 32 heads take 0.88 ms in fp32, 0.66 in fp16; 3 x 333 tokens in fp32
// 76 us. In blocks of eight tokens on the FMA units the same took 1.10 and 1.10 ms, and 95 us; token by
// token 215 us. 16-bit vectors leave room for two CTAs a multiprocessor (fp16 with one: 0.83 ms);
// in fp32 two spill (1.00 ms).
#include "async.cuh"
#include "device.cuh"
#include "linattn_prefill.cuh"

#include <type_traits>

namespace stepq {
namespace la {
namespace tm {

constexpr int TB = 16;                                       // tokens a block
constexpr int kRows = TB * kD;                               // elements of a term's tile
constexpr int kPitchP = 24;                                  // of P's rows: eight of them in eight places of 16 bytes

template <class T> constexpr int kTerms = sizeof(T) == 4 ? 3 : std::is_same<T, bf16>::value ? 1 : 2;   // of q, k and v
template <class T> constexpr int kInner = sizeof(T) == 4 ? 3 : 2;                                      // of S and P
template <class T> constexpr int kTileBytes = (3 * kTerms<T> + 3) * kRows * 2;
constexpr int kPartBytes = 8 * TB * TB * 4, kPBytes = 3 * TB * kPitchP * 2, kYBytes = 2 * TB * kD * 4;
template <class T, bool NORM> constexpr int kSmemBytes = 2 * kTileBytes<T> + kPartBytes + kPBytes + (NORM ? kYBytes : 0);

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four 8 x 8 tiles, lane i giving the address of row i % 8 of tile i / 8; TRANS: each transposed.
template <bool TRANS>
__device__ __forceinline__ void load_tiles(uint32_t (&r)[4], const bf16 *row) {
    if (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_addr(row)) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_addr(row)) : "memory");
}
// The terms of two values, a pair a word. But the last of several, none rounds to infinity: the largest
// finite values keep finite terms, and an infinite one has an infinite last.
template <int N>
__device__ __forceinline__ void split(uint64_t x, uint32_t (&t)[N]) {
#pragma unroll
    for (int i = 0; i < N; i++) {
        if (i + 1 < N) asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(t[i]) : "f"(f2hi(x)), "f"(f2lo(x)));
        else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(t[i]) : "f"(f2hi(x)), "f"(f2lo(x)));
        if (i + 1 < N) x = fsub2(x, u2pair(t[i] << 16, t[i] & 0xFFFF0000u));
    }
}
// d += the product of A's and B's terms i and j, i + j <= 2, smaller ones first; SETS > 1: those of
// each order i + j apart, so that fewer of the products wait for one another.
template <int NA, int NB, int SETS>
__device__ __forceinline__ void product(float (&d)[SETS][4], const uint32_t (&A)[NA][4], const uint32_t (&B0)[NB], const uint32_t (&B1)[NB]) {
#pragma unroll
    for (int sum = 2; sum >= 0; sum--)
#pragma unroll
        for (int i = 0; i < NA; i++)
            if (sum - i >= 0 && sum - i < NB) mma(d[sum < SETS ? sum : SETS - 1], A[i], B0[sum - i], B1[sum - i]);
}
template <int SETS>
__device__ __forceinline__ float total_of(const float (&d)[SETS][4], int e) {   // smaller ones first
    float x = d[SETS - 1][e];
#pragma unroll
    for (int m = SETS - 2; m >= 0; m--) x += d[m][e];
    return x;
}
// Element (token, 8 chunk) of a tile: rows of 256 bytes, their 16-byte pieces exchanged so that
// eight rows' equal pieces lie in different banks.
__device__ __forceinline__ int at(int token, int chunk) { return token * kD + 8 * (chunk ^ (token & 7)); }

template <class T, bool OUT, bool NORM>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) linattn_terms_kernel(PrefillArgs a) {
    constexpr int N = kTerms<T>, NS = kInner<T>;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, w = tid >> 5, l = tid & 31, g = l >> 2, c = l & 3;
    griddep_wait();
    griddep_launch();
    const int part = blockIdx.x / a.Hv, h = blockIdx.x - part * a.Hv, hk = h / (a.Hv / a.Hk);
    int row, len;
    const float *in = nullptr;
    float *out, *total_to = nullptr, total = 1.f;            // a part's decay
    if (a.plan) {
        if (part >= (OUT ? a.plan->segments : a.plan->parts)) return;
        const Segment s = a.table[part];
        float *work = a.states + ((uint64_t)s.id * a.Hv + h) * kN, *page = pool_page(a, s.slot, h);
        row = s.row;
        len = s.len;
        if (OUT) in = s.in == kStateZero ? nullptr : s.in == kStatePool ? page : work;
        out = !OUT ? work + (uint64_t)a.Hv * kN : s.out == kStatePool ? page : nullptr;
        total_to = !OUT ? a.totals + (uint64_t)s.id * a.Hv + h : nullptr;
    } else {
        int slot;
        if (!sequence(a, part, tid == 0, row, len, slot) || len == 0) return;
        if (h == 0) check_slot(a, part, tid, 256);
        out = pool_page(a, slot, h);
        in = !a.resume || a.resume[part] ? out : nullptr;
    }
    // A stage: q, k, v in N terms each, K' in three.
    const auto tile = [&](int stage, int which, int term) {
        return (bf16 *)(smem + stage * kTileBytes<T>) + (which * N + term) * kRows;
    };
    float *sums = (float *)(smem + 2 * kTileBytes<T>);       // [warp][16 t][16 s]
    bf16 *P = (bf16 *)(smem + 2 * kTileBytes<T> + kPartBytes);   // [term][16 t][kPitchP]
    float *ys = (float *)(smem + 2 * kTileBytes<T> + kPartBytes + kPBytes);   // [2][16][128]

    // Tile j of S^T: key rows 8 j + 2 c, + 1 of a product's rows g and g + 8, which are value columns
    // 2 g and 2 g + 1 of the warp's 16: V's tiles hold a group's even columns before its odd ones, so
    // that a thread's two are one access to states and readouts.
    float S[16][4];
    const int vcol = 16 * w + 2 * g;
#pragma unroll
    for (int j = 0; j < 16; j++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const float2 x = in ? *(const float2 *)&in[(8 * j + 2 * c + e) * kD + vcol] : make_float2(0.f, 0.f);
            S[j][e] = x.x;
            S[j][e + 2] = x.y;
        }

    // A block's vectors on their way: token t of it, channels 8 ch .. + 7; the decay of token l % 16.
    const int t = tid >> 4, ch = tid & 15;
    Vec<T, 8> nq{}, nk{}, nv{};
    float ng = 1.f;
    const auto fetch = [&](int t0) {
        const Vec<T, 8> zero{};
        const int64_t r = (int64_t)row + t0 + t;
        const bool valid = t0 + t < len;
        const auto get = [&](const void *p, int64_t stride, int head) {
            Vec<T, 8> x = zero;
            if (valid) {
                const Vec<T, 16 / sizeof(T)> *from = (const Vec<T, 16 / sizeof(T)> *)((const T *)p + r * stride + head * kD + 8 * ch);
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; i++) ((Vec<T, 16 / sizeof(T)> *)&x)[i] = from[i];
            }
            return x;
        };
        if (OUT) nq = get(a.q, a.qs, hk);
        nk = get(a.k, a.ks, hk);
        nv = get(a.v, a.vs, h);
        const int j = l & 15;
        ng = t0 + j < len ? a.gate[((int64_t)row + t0 + j) * a.gs + h] : 1.f;
    };
    // Products of the block's decays from token l % 16 + 1 on.
    const auto suffix = [&](float gate) {
        float x = __shfl_down_sync(0xffffffffu, gate, 1, 16);
        x = (l & 15) == 15 ? 1.f : x;
#pragma unroll
        for (int o = 1; o < 16; o *= 2) {
            const float y = __shfl_down_sync(0xffffffffu, x, o, 16);
            x *= (l & 15) + o < 16 ? y : 1.f;
        }
        return x;
    };
    const auto put = [&](int stage) {
        if constexpr (sizeof(T) == 2) {                      // the conversions stay here, behind the loads' way
            uint32_t *q = (uint32_t *)&nq, *k = (uint32_t *)&nk, *v = (uint32_t *)&nv;
            asm volatile("" : "+r"(q[0]), "+r"(q[1]), "+r"(q[2]), "+r"(q[3]), "+r"(k[0]), "+r"(k[1]), "+r"(k[2]), "+r"(k[3]),
                         "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3])::"memory");
        }
        const uint64_t wt = f2s(__shfl_sync(0xffffffffu, suffix(ng), t));
        const auto terms = [&](const Vec<T, 8> &x, int which, uint64_t scale, auto n) {
            constexpr int M = decltype(n)::value;
            uint32_t r[4][M];
#pragma unroll
            for (int i = 0; i < 4; i++) split<M>(fmul2(f2(to_f32(x.e[2 * i]), to_f32(x.e[2 * i + 1])), scale), r[i]);
#pragma unroll
            for (int m = 0; m < M; m++) {
                if (which == 2) {                            // even columns, odd columns
                    bf16 *at0 = tile(stage, 2, m) + 4 * (ch & 1);
                    const int g16 = ch & ~1;
                    *(uint2 *)(at0 + at(t, g16)) = make_uint2(__byte_perm(r[0][m], r[1][m], 0x5410), __byte_perm(r[2][m], r[3][m], 0x5410));
                    *(uint2 *)(at0 + at(t, g16 + 1)) = make_uint2(__byte_perm(r[0][m], r[1][m], 0x7632), __byte_perm(r[2][m], r[3][m], 0x7632));
                } else {
                    *(uint4 *)(tile(stage, which, m) + at(t, ch)) = make_uint4(r[0][m], r[1][m], r[2][m], r[3][m]);
                }
            }
        };
        if (OUT) {
            terms(nq, 0, f2s(1.f), std::integral_constant<int, N>{});
            terms(nk, 1, f2s(1.f), std::integral_constant<int, N>{});
        }
        terms(nv, 2, f2s(1.f), std::integral_constant<int, N>{});
        terms(nk, 3, wt, std::integral_constant<int, 3>{});
    };
    // Q K^T of a stage over this warp's 16 channels.
    const int r8 = l & 7, t8 = l >> 3;                       // a tile's row, and which tile, of load_tiles
    const auto scores = [&](int stage) {
        uint32_t A[N][4], B[N][4];
#pragma unroll
        for (int m = 0; m < N; m++) {
            load_tiles<false>(A[m], tile(stage, 0, m) + at(8 * (t8 & 1) + r8, 2 * w + (t8 >> 1)));
            load_tiles<false>(B[m], tile(stage, 1, m) + at(8 * (t8 >> 1) + r8, 2 * w + (t8 & 1)));
        }
#pragma unroll
        for (int i = 0; i < 2; i++) {
            uint32_t b0[N], b1[N];
#pragma unroll
            for (int m = 0; m < N; m++) {
                b0[m] = B[m][2 * i];
                b1[m] = B[m][2 * i + 1];
            }
            float p[1][4] = {};
            product(p, A, b0, b1);
            *(float2 *)&sums[w * TB * TB + g * TB + 8 * i + 2 * c] = make_float2(p[0][0], p[0][1]);
            *(float2 *)&sums[w * TB * TB + (g + 8) * TB + 8 * i + 2 * c] = make_float2(p[0][2], p[0][3]);
        }
    };
    // P of token t and key l % 16 from the warps' sums, as terms.
    const auto weigh = [&](float gate) {
        const int s = l & 15;
        float p = 0.f;
#pragma unroll
        for (int i = 0; i < 8; i++) p += sums[i * TB * TB + t * TB + s];
        const float wt = suffix(s <= t ? gate : 1.f);
        p = s <= t ? p * wt : 0.f;
        uint32_t r[NS];
        split<NS>(f2(p, 0.f), r);
#pragma unroll
        for (int m = 0; m < NS; m++) *(uint16_t *)&P[(m * TB + t) * kPitchP + s] = (uint16_t)r[m];
    };
    // Tokens 2 w and 2 w + 1 of block n, a block late: the next products fill the waits of their sums.
    const HeadAffine affine(a.norm, h, l);
    Vec<T, 4> z[2] = {};
    const auto normalise = [&](int n) {
        if constexpr (sizeof(T) == 2) {
            uint32_t *word = (uint32_t *)z;
            asm volatile("" : "+r"(word[0]), "+r"(word[1]), "+r"(word[2]), "+r"(word[3])::"memory");
        }
        float u[2][4];
#pragma unroll
        for (int i = 0; i < 2; i++) load_vec<float, 4>(&ys[((n & 1) * TB + 2 * w + i) * kD + 4 * l], u[i]);
        norm_head<T, 2>(a.norm, affine, z, u);
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int k = TB * n + 2 * w + i;
            if (k < len) store_vec<T, 4>((T *)a.y + ((int64_t)row + k) * a.ys + h * kD + 4 * l, u[i]);
        }
    };

    float g0, g1 = 1.f;                                      // decays of this block and of the next, token l % 16
    fetch(0);
    put(0);
    g0 = ng;
    if (len > TB) {
        fetch(TB);
        put(1);
        g1 = ng;
    }
    if (OUT) {
        __syncthreads();
        scores(0);
        __syncthreads();
        weigh(g0);
    }
    for (int t0 = 0, n = 0; t0 < len; t0 += TB, n++) {
        const int stage = n & 1;
        __syncthreads();                                     // this block's P, the next one's vectors
        if (t0 + 2 * TB < len) fetch(t0 + 2 * TB);
        if (NORM) {
            if (n) normalise(n - 1);
            if (a.norm.z)
#pragma unroll
                for (int i = 0; i < 2; i++)
                    if (t0 + 2 * w + i < len)
                        z[i] = *(const Vec<T, 4> *)((const T *)a.norm.z + ((int64_t)row + t0 + 2 * w + i) * a.norm.z_stride + h * kD + 4 * l);
        }
        if (OUT && t0 + TB < len) scores(stage ^ 1);
        // Products of the decays to token l % 16, and of all.
        float pre = g0;
#pragma unroll
        for (int o = 1; o < 16; o *= 2) {
            const float y = __shfl_up_sync(0xffffffffu, pre, o, 16);
            pre *= (l & 15) >= o ? y : 1.f;
        }
        const float all = __shfl_sync(0xffffffffu, pre, 15);
        if (!OUT) total *= all;
        uint32_t V[N][4];
#pragma unroll
        for (int m = 0; m < N; m++) load_tiles<true>(V[m], tile(stage, 2, m) + at(8 * (t8 >> 1) + r8, 2 * w + (t8 & 1)));
        if (OUT) {
            float y[2][NS][4] = {};
#pragma unroll
            for (int j = 0; j < 8; j++) {
                uint32_t A[NS][4], B[N][4];
#pragma unroll
                for (int e = 0; e < 4; e++) {                // its rows g (+ 8), key rows 16 j + 2 c (+ 8)
                    uint32_t x[NS];
                    const float *s = &S[2 * j + (e >> 1)][2 * (e & 1)];
                    split<NS>(f2(s[0], s[1]), x);
#pragma unroll
                    for (int m = 0; m < NS; m++) A[m][e] = x[m];
                }
#pragma unroll
                for (int m = 0; m < N; m++) load_tiles<false>(B[m], tile(stage, 0, m) + at(8 * (t8 >> 1) + r8, 2 * j + (t8 & 1)));
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    uint32_t b0[N], b1[N];
#pragma unroll
                    for (int m = 0; m < N; m++) {
                        b0[m] = B[m][2 * i];
                        b1[m] = B[m][2 * i + 1];
                    }
                    product(y[i], A, b0, b1);
                }
            }
            uint32_t B[NS][4];
#pragma unroll
            for (int m = 0; m < NS; m++) load_tiles<false>(B[m], &P[(m * TB + 8 * (t8 >> 1) + r8) * kPitchP + 8 * (t8 & 1)]);
#pragma unroll
            for (int i = 0; i < 2; i++) {
                uint32_t b0[NS], b1[NS];
#pragma unroll
                for (int m = 0; m < NS; m++) {
                    b0[m] = B[m][2 * i];
                    b1[m] = B[m][2 * i + 1];
                }
                float o[1][4] = {};
                product(o, V, b0, b1);
#pragma unroll
                for (int e = 0; e < 2; e++) {                // token 8 i + 2 c (+ 1)
                    const int tk = 8 * i + 2 * c + e;
                    const float ct = __shfl_sync(0xffffffffu, pre, tk);
                    const float r[2] = {fmaf(ct, total_of(y[i], e), o[0][e]), fmaf(ct, total_of(y[i], e + 2), o[0][e + 2])};
                    if (NORM) store_vec<float, 2>(&ys[(stage * TB + tk) * kD + vcol], r);
                    else if (t0 + tk < len) store_vec<T, 2>((T *)a.y + ((int64_t)row + t0 + tk) * a.ys + h * kD + vcol, r);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            uint32_t B[3][4];
#pragma unroll
            for (int m = 0; m < 3; m++) load_tiles<true>(B[m], tile(stage, 3, m) + at(8 * (t8 & 1) + r8, j + (t8 >> 1)));
#pragma unroll
            for (int i = 0; i < 2; i++) {
                uint32_t b0[3], b1[3];
#pragma unroll
                for (int m = 0; m < 3; m++) {
                    b0[m] = B[m][2 * i];
                    b1[m] = B[m][2 * i + 1];
                }
                float u[1][4] = {};
                product(u, V, b0, b1);
#pragma unroll
                for (int e = 0; e < 4; e++) S[j + i][e] = fmaf(S[j + i][e], all, u[0][e]);
            }
        }
        __syncthreads();                                     // the stage is read, the sums of the next P are there
        if (OUT && t0 + TB < len) weigh(g1);
        g0 = g1;
        if (t0 + 2 * TB < len) {
            put(stage);
            g1 = ng;
        }
    }
    if (NORM) {
        __syncthreads();
        normalise((len - 1) / TB);
    }
    if (!OUT && tid == 0) *total_to = total;
    if (out)
#pragma unroll
        for (int j = 0; j < 16; j++)
#pragma unroll
            for (int e = 0; e < 2; e++) *(float2 *)&out[(8 * j + 2 * c + e) * kD + vcol] = make_float2(S[j][e], S[j][e + 2]);
}

template <class T, bool OUT, bool NORM>
static stepq_status launch(const PrefillArgs *a, int items, cudaStream_t s) {
    static SmemOptIn opt;
    const auto kernel = linattn_terms_kernel<T, OUT, NORM>;
    const stepq_status st = opt((const void *)kernel, kSmemBytes<T, NORM>);
    return st != STEPQ_OK || !a ? st : launch_overlapped(kernel, items, 256, kSmemBytes<T, NORM>, s, *a);
}

template <class T>
static stepq_status launch_type(const PrefillArgs *a, int items, bool out, bool norm, cudaStream_t s) {
    return !out ? launch<T, false, false>(a, items, s) : norm ? launch<T, true, true>(a, items, s) : launch<T, true, false>(a, items, s);
}

}  // namespace tm

stepq_status launch_linattn_terms(int dtype, const PrefillArgs *a, int items, bool out, bool norm, cudaStream_t s) {
    return by_type(dtype, [&](auto t) { return tm::launch_type<decltype(t)>(a, items, out, norm, s); });
}

}  // namespace la
}  // namespace stepq
