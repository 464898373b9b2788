// Attention of one new token over a paged cache, split over its length.
//
// For the query heads that share a key head, s_t = c q . k_t and
//   y = sum_t 2^(s_t - R) v_t / sum_t 2^(s_t - R),  c = scale log2(e),
// for any reference R near the largest s_t. Parts of the tokens give (R, l, O), l the sum of
// weights and O that of weighted v, and parts join as sum_i 2^(R_i - R) O_i over the same sum of
// the l_i.
//
// Work: the tokens of every (sequence, key head) are cut into tiles; all tiles in a row are
// dealt out in equal shares to the CTAs, which find theirs from the lengths on the device. A
// CTA's share is pieces of one or more sequences; a piece that is a whole sequence gives its
// outputs, one that is not leaves (R, l, O) in the workspace, and a second kernel joins those.
// Within a CTA each warp takes every fourth tile, through its own ring of shared memory filled
// by 16-byte asynchronous copies, and waits for no other warp until the piece ends.
//
// Products by mma.sync m16n8k16 with tokens (for K) and channels (for V) as the 16 rows and
// eight query heads as the columns, so that no part of a product is padding where eight heads
// share a key head. HBM bounds the call as long as these keep up; tcgen05 would want 128 rows of
// tokens of which each is used for 8 columns, and codes would have to go back to shared memory.
// The order of channels within a product is free, so a lane takes whole 16-byte pieces of a
// row and the queries are laid out to match. Codes u enter K's product as the fp16 subnormal
// u 2^-24 (a mask or a byte permute), its offset 2^(b-1) sum q is subtracted from the sum; for V,
// where that would cancel over all tokens, u - 2^(b-1) is formed first, exactly.
//
// Roundings: q enters as a sum of QT terms of the cache's 16-bit type, weights as a sum of PT,
// everything between in fp32. One term of fp16 has 2^-12, half of bf16's eighth of a unit, two
// of fp16 2^-23, two of bf16 2^-17, three 2^-25; see Terms.
#pragma once

#include <type_traits>

#include "device.cuh"
#include "kv.cuh"

namespace stepq {
namespace kv {

constexpr int kAttWarps = 4;
constexpr float kLow = -3.402823466e+38f;

// Workspace: for each CTA c two parts (2 c: the piece that its share begins with, 2 c + 1: one
// that it ends with) of HT heads, [HT][D] of O and then R and l [HT] each; behind the parts an
// int4 for each CTA that says which parts the piece begun by it and ended by others has.
struct Joined {
    int count, first, b, vh;        // first part; the others are 2 (c + 1), 2 (c + 2), ..
};
template <int HT, int D> __host__ __device__ constexpr int part_floats() { return HT * (D + 2); }

template <int F> struct Compute { using T = la::f16; };
template <> struct Compute<STEPQ_KV_BF16> { using T = la::bf16; };

// Shape of a variant.
template <int F_, int D_, int NT_, int QT_, int PT_>
struct Shape {
    static constexpr int F = F_, D = D_, NT = NT_, QT = QT_, PT = PT_;
    static constexpr int HT = 8 * NT;                        // heads of a CTA
    static constexpr int RB = row_bytes(F, D);
    static constexpr bool CODED = coded(F);
    // tokens of a tile: 8 KB of K and V where that is 16 to 64 of them
    static constexpr int TT = RB * 2 * 64 <= 8192 ? 64 : RB * 2 * 32 <= 8192 ? 32 : 16;
    static constexpr int TILE = 2 * TT * RB + (CODED ? 4 * TT : 0);
    static constexpr int STAGES = 3;
    static constexpr int RING = kAttWarps * STAGES * TILE;
    static constexpr int MERGE = kAttWarps * HT * (D + 2) * 4;
    static constexpr int OFF_Q = RING > MERGE ? RING : MERGE;          // [QT][NT][D / 16][32] uint2
    static constexpr int OFF_HEAD = OFF_Q + QT * NT * (D / 16) * 256;  // float [2][HT]: factor, offset
    static constexpr int OFF_SCAN = OFF_HEAD + 2 * HT * 4;             // int64 [kAttWarps + 2]
    static constexpr int SMEM = OFF_SCAN + 8 * (kAttWarps + 4);
    static constexpr int RESIDENT = SMEM <= 75 * 1024 ? 3 : SMEM <= 113 * 1024 ? 2 : 1;
    static constexpr int KP = RB / 4 < 16 ? RB / 4 : 16;     // bytes a lane reads of a row of K at once
    static constexpr int VP = RB / 8 < 16 ? RB / 8 : 16;     // and of V
    static constexpr int KS = D / 16;                        // steps of K's product
    static constexpr int MT = D / 16;                        // row tiles of V's
    static constexpr bool QREG = QT * NT * KS <= 16;         // queries kept in registers
    using C = typename Compute<F>::T;
};

// ------------------------------------------------------------------ building blocks
template <class C>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    if (std::is_same<C, la::bf16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit elements, row lane / 4 and columns 2 (lane % 4), + 1, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi, la::bf16) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi, la::f16) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 unpack(uint32_t v, la::bf16) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack(uint32_t v, la::f16) {
    return __half22float2(*(const __half2 *)&v);
}
__device__ __forceinline__ uint32_t hadd2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("add.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <int N> struct alignas(4 * N) Words { uint32_t w[N]; };
template <int BYTES>
__device__ __forceinline__ Words<BYTES / 4> lds(const uint8_t *tile, uint32_t at) {
    return *(const Words<BYTES / 4> *)(tile + at);
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

// Place of byte `at` (row * RB + byte) of a tile's rows: 16-byte pieces change places within 128
// bytes so that the lanes that read at once meet no bank twice. They read 64 bytes each of
// rows r and r + 1 (K), or up to 32 of rows r, r + 2, r + 4 and r + 6 (V).
template <int RB>
__device__ __forceinline__ uint32_t k_place(int row, int byte) {
    return (uint32_t)(row * RB + byte) ^ (RB >= 128 ? (row & 1) << 6 : 0);
}
template <int RB>
__device__ __forceinline__ uint32_t v_place(int row, int byte) {
    return (uint32_t)(row * RB + byte) ^ (RB >= 64 ? ((row >> 1) & 3) << 5 : ((row >> 2) & 1) << 5);
}

// A lane's piece of a row of K as pairs of the compute type, in the order of q_channel().
template <int F, int N>
__device__ __forceinline__ void k_pairs(const Words<N> &x, uint32_t (&p)[N * 16 / bits_of(F)]) {
#pragma unroll
    for (int i = 0; i < N; i++) {
        if constexpr (F == STEPQ_KV_INT8) {
            p[2 * i] = __byte_perm(x.w[i], 0u, 0x4140);
            p[2 * i + 1] = __byte_perm(x.w[i], 0u, 0x4342);
        } else if constexpr (F == STEPQ_KV_INT4) {
            const uint32_t y = x.w[i] >> 8;
            p[4 * i] = x.w[i] & 0x000f000fu;
            p[4 * i + 1] = x.w[i] & 0x00f000f0u;
            p[4 * i + 2] = y & 0x000f000fu;
            p[4 * i + 3] = y & 0x00f000f0u;
        } else {
            p[i] = x.w[i];
        }
    }
}
// Channel of half `half` of pair j (of one piece's) as k_pairs() leaves them.
template <int F>
__host__ __device__ constexpr int q_channel(int j, int half) {
    return F == STEPQ_KV_INT4 ? 8 * (j / 4) + j % 4 + 4 * half : 2 * j + half;
}
template <int F>
__host__ __device__ constexpr float q_factor(int j) { return F == STEPQ_KV_INT4 && (j & 1) ? 0.0625f : 1.f; }

// A lane's pieces of two tokens' rows of V as pairs of tokens, p[channel]: one 2^-24 of the code
// without its offset, and for the odd channels of 4 bits 2^-20.
template <int F, int N>
__device__ __forceinline__ void v_pairs(const Words<N> &a, const Words<N> &b, uint32_t (&p)[N * 32 / bits_of(F)]) {
#pragma unroll
    for (int i = 0; i < N; i++) {
        if constexpr (F == STEPQ_KV_INT8) {
            const uint32_t lo = __byte_perm(a.w[i], b.w[i], 0x5140), hi = __byte_perm(a.w[i], b.w[i], 0x7362);
            p[4 * i] = hadd2(__byte_perm(lo, 0u, 0x4140), 0x80808080u);
            p[4 * i + 1] = hadd2(__byte_perm(lo, 0u, 0x4342), 0x80808080u);
            p[4 * i + 2] = hadd2(__byte_perm(hi, 0u, 0x4140), 0x80808080u);
            p[4 * i + 3] = hadd2(__byte_perm(hi, 0u, 0x4342), 0x80808080u);
        } else if constexpr (F == STEPQ_KV_INT4) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint32_t x = __byte_perm(a.w[i], b.w[i], h ? 0x7632 : 0x5410), y = x >> 8;
                p[8 * i + 4 * h] = hadd2(x & 0x000f000fu, 0x80088008u);
                p[8 * i + 4 * h + 1] = hadd2(x & 0x00f000f0u, 0x80808080u);
                p[8 * i + 4 * h + 2] = hadd2(y & 0x000f000fu, 0x80088008u);
                p[8 * i + 4 * h + 3] = hadd2(y & 0x00f000f0u, 0x80808080u);
            }
        } else {
            p[2 * i] = __byte_perm(a.w[i], b.w[i], 0x5410);
            p[2 * i + 1] = __byte_perm(a.w[i], b.w[i], 0x7632);
        }
    }
}
// What V's product is to be multiplied by, by the parity of the channel.
template <int F>
__host__ __device__ constexpr float v_factor(int odd) {
    return !coded(F) ? 1.f : F == STEPQ_KV_INT4 && odd ? 1048576.f : 16777216.f;
}

__device__ __forceinline__ float load_any(const void *p, int64_t i, int dtype) {
    return dtype == STEPQ_F32 ? ((const float *)p)[i]
           : dtype == STEPQ_BF16 ? la::to_f32(((const la::bf16 *)p)[i]) : la::to_f32(((const la::f16 *)p)[i]);
}
// Four consecutive channels.
__device__ __forceinline__ void store4_any(void *p, int64_t i, int dtype, const float (&x)[4]) {
    if (dtype == STEPQ_F32) la::store_vec<float, 4>((float *)p + i, x);
    else if (dtype == STEPQ_BF16) la::store_vec<la::bf16, 4>((la::bf16 *)p + i, x);
    else la::store_vec<la::f16, 4>((la::f16 *)p + i, x);
}

// Tokens [lo, hi) of a row that count, and its tiles (one for a row without any).
struct Span { int lo, hi, tile0, tiles; };
template <int TT>
__device__ __forceinline__ Span span_of(const AttendArgs &a, int len) {
    Span s;
    const long long most = (long long)a.pg.width << a.pg.shift;
    s.hi = len < 0 ? 0 : len > most ? (int)most : len;
    s.lo = a.window > 0 && s.hi > a.window ? s.hi - a.window : 0;
    s.tile0 = s.lo / TT;
    s.tiles = max(1, (s.hi + TT - 1) / TT - s.tile0);
    return s;
}

// ------------------------------------------------------------------ the kernel
template <class S>
__global__ void __launch_bounds__(32 * kAttWarps, S::RESIDENT) kv_attend_kernel(AttendArgs a) {
    extern __shared__ __align__(128) uint8_t smem[];
    using C = typename S::C;
    constexpr int D = S::D, TT = S::TT, RB = S::RB, NT = S::NT, HT = S::HT, F = S::F;
    const int tid = threadIdx.x, w = tid >> 5, l = tid & 31, r = l >> 2, c = l & 3;
    const int chunks = (a.groups + HT - 1) / HT, VH = a.pg.n_heads * chunks;
    float *head_k = (float *)(smem + S::OFF_HEAD), *head_off = head_k + HT;
    long long *scan = (long long *)(smem + S::OFF_SCAN);
    griddep_wait();
    griddep_launch();

    // The share: tiles [t, end) of all, in the order (sequence, virtual head, tile); b and the
    // tiles of the sequences before it.
    long long t = 0, end = 0, share = 0, before = 0;
    int b = 0;
    if (!a.whole) {
        const int per = (a.B + 32 * kAttWarps - 1) / (32 * kAttWarps), i0 = min(a.B, tid * per), i1 = min(a.B, i0 + per);
        long long mine = 0;
        for (int i = i0; i < i1; i++) mine += span_of<TT>(a, a.lens[i]).tiles;
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const long long x = __shfl_up_sync(0xffffffffu, upto, o);
            if (l >= o) upto += x;
        }
        if (l == 31) scan[w] = upto;
        __syncthreads();
        long long total = 0;
#pragma unroll
        for (int i = 0; i < kAttWarps; i++) {
            if (i < w) upto += scan[i];
            total += scan[i];
        }
        total *= VH;
        share = max((total + gridDim.x - 1) / gridDim.x, (long long)(2 * kAttWarps));
        t = share * blockIdx.x;
        end = min(total, t + share);
        if (t < total && t >= (upto - mine) * VH && t < upto * VH) {
            long long p = upto - mine;
            int i = i0;
            for (;; i++) {
                const int n = span_of<TT>(a, a.lens[i]).tiles;
                if (t < (p + n) * VH) break;
                p += n;
            }
            scan[kAttWarps] = p;
            scan[kAttWarps + 1] = i;
        }
        __syncthreads();
        before = scan[kAttWarps];
        b = (int)scan[kAttWarps + 1];
        if (tid == 0)                                        // no piece goes on in other CTAs, unless one does below
            ((Joined *)(a.parts + (size_t)2 * gridDim.x * part_floats<HT, D>()))[blockIdx.x] = Joined{0, 0, 0, 0};
        if (t >= total) return;
    } else {
        t = blockIdx.x;
        end = (long long)a.B * VH;
    }

    const uint32_t ring = smem_addr(smem) + w * S::STAGES * S::TILE;
    while (t < end) {
        // The piece: virtual head vh of sequence b, its tiles from `from`, n of them.
        int vh, from, n;
        if (a.whole) {
            b = (int)(t / VH);
            vh = (int)(t - (long long)b * VH);
        }
        const int len = a.lens[b];
        const Span sp = span_of<TT>(a, len);
        if (a.whole) {
            from = 0;
            n = sp.tiles;
        } else {
            const long long in = t - before * VH;
            vh = (int)(in / sp.tiles);
            from = (int)(in - (long long)vh * sp.tiles);
            n = (int)min((long long)(sp.tiles - from), end - t);
        }
        if (tid == 0 && from == 0 && vh == 0) {
            if (len < 0) raise_error(a.pg.err, STEPQ_ERR_ARG);
            if (len > sp.hi && len > 0) raise_error(a.pg.err, STEPQ_ERR_SLOT_RANGE);
        }
        const int hk = vh / chunks, g0 = (vh - hk * chunks) * HT, nh = min(HT, a.groups - g0);
        const int h0 = hk * a.groups + g0;                   // first query head

        __syncthreads();                                     // the last piece's shared memory is free
        // Queries, as pairs in the order of K's pieces: step ks of the product, pair (0, 1) of
        // lane 4 head + c.
        uint32_t *qf = (uint32_t *)(smem + S::OFF_Q);
        for (int h = w; h < HT; h += kAttWarps) {
            constexpr int N = D / 32;
            float x[N], top = 0.f;
#pragma unroll
            for (int e = 0; e < N; e++) {
                x[e] = h < nh ? load_any(a.q, b * a.qs + (int64_t)(h0 + h) * D + 32 * e + l, a.dtype) : 0.f;
                top = fmaxf(top, fabsf(x[e]));
            }
            float k = a.scale, off = 0.f;
            if (std::is_same<C, la::f16>::value) {
                // scaled by a power of two to at most 2^15, where fp16 keeps 2^-40 of the largest
#pragma unroll
                for (int o = 1; o < 32; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const int ex = top > 0.f && top < INFINITY ? 14 - ilogbf(top) : 0;
#pragma unroll
                for (int e = 0; e < N; e++) x[e] = ldexpf(x[e], ex);
                k = ldexpf(k, -ex);
            }
#pragma unroll
            for (int e = 0; e < N; e++) {
                // channel -> piece of KP bytes, pair j in it, half; pieces 4 i + c go to lane c
                constexpr int PC = S::KP * 8 / bits_of(F), JP = PC / 2;          // channels, pairs of a piece
                const int ch = 32 * e + l, piece = ch / PC, in = ch % PC;
                int j, half;
                if (F == STEPQ_KV_INT4) {
                    j = 4 * (in / 8) + in % 4;
                    half = in / 4 % 2;
                } else {
                    j = in / 2;
                    half = in % 2;
                }
                const int pair = (piece / 4) * JP + j, lane = 4 * (h % 8) + piece % 4;
                float rest = x[e] * q_factor<F>(j);
#pragma unroll
                for (int i = 0; i < S::QT; i++) {
                    const C v = la::from_f32<C>(rest);
                    rest -= la::to_f32(v);
                    off += la::to_f32(v) / q_factor<F>(j);
                    ((C *)qf)[((((i * NT + h / 8) * S::KS + pair / 2) * 32 + lane) * 2 + pair % 2) * 2 + half] = v;
                }
            }
            if (S::CODED) {
#pragma unroll
                for (int o = 1; o < 32; o *= 2) off += __shfl_xor_sync(0xffffffffu, off, o);
                off *= F == STEPQ_KV_INT8 ? 128.f / 16777216.f : 8.f / 16777216.f;
                k *= 16777216.f;
            }
            if (l == 0) {
                head_k[h] = k;
                head_off[h] = off;
            }
        }
        __syncthreads();

        float hf[NT][2], ho[NT][2], R[NT][2], sum[NT][2], O[NT][S::MT][4];
        uint2 qr[S::QREG ? S::QT : 1][S::QREG ? NT : 1][S::QREG ? S::KS : 1];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
#pragma unroll
            for (int e = 0; e < 2; e++) {
                hf[nt][e] = head_k[8 * nt + 2 * c + e];
                ho[nt][e] = head_off[8 * nt + 2 * c + e];
                R[nt][e] = kLow;
                sum[nt][e] = 0.f;
            }
#pragma unroll
            for (int m = 0; m < S::MT; m++)
#pragma unroll
                for (int e = 0; e < 4; e++) O[nt][m][e] = 0.f;
        }
        if constexpr (S::QREG) {
#pragma unroll
            for (int i = 0; i < S::QT; i++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int ks = 0; ks < S::KS; ks++)
                        qr[i][nt][ks] = ((const uint2 *)qf)[((i * NT + nt) * S::KS + ks) * 32 + l];
        }

        // This warp's tiles: from + w, from + w + kAttWarps, ... below from + n.
        const int count = n > w ? (n - w + kAttWarps - 1) / kAttWarps : 0;
        const int token0 = (sp.tile0 + from + w) * TT;       // of the warp's first tile
        const int32_t *table = a.pg.table + b * a.pg.table_stride;
        // page of octet l (eight tokens) of the warp's tile i, -1 for none
        auto page_ids = [&](int i) {
            if (l >= TT / 8 || i >= count) return -1;
            const int tok = token0 + i * kAttWarps * TT + 8 * l;
            if (tok >= sp.hi || tok + 8 <= sp.lo) return -1;
            const int id = table[tok >> a.pg.shift];
            if (id >= 0 && id < a.pg.n_pages) return id;
            raise_error(a.pg.err, STEPQ_ERR_SLOT_RANGE);
            return -1;
        };
        auto copy_tile = [&](int i, int ids) {
            const uint32_t dst = ring + (i % S::STAGES) * S::TILE;
            const int tok0 = token0 + i * kAttWarps * TT;
            constexpr int PER = RB / 16, N = TT * PER / 32;
#pragma unroll
            for (int j = 0; j < N; j++) {
                const int ch = 32 * j + l, row = ch / PER, byte = ch % PER * 16, tok = tok0 + row;
                const int id = __shfl_sync(0xffffffffu, ids, row / 8);
                const bool ok = id >= 0 && tok >= sp.lo && tok < sp.hi;
                const uint8_t *src = a.pg.at(ok ? id : 0, hk) + (ok ? a.pg.slot(tok) * RB + byte : 0);
                copy16(dst + k_place<RB>(row, byte), src, ok);
                copy16(dst + TT * RB + v_place<RB>(row, byte), src + (ok ? RB << a.pg.shift : 0), ok);
            }
            if (S::CODED && l < TT / 8) {
                const bool ok = ids >= 0;
                const uint8_t *src = a.pg.at(ok ? ids : 0, hk) + (ok ? (2 * RB << a.pg.shift) + 2 * a.pg.slot(tok0 + 8 * l) : 0);
                copy16(dst + 2 * TT * RB + 16 * l, src, ok);
                copy16(dst + 2 * TT * RB + 2 * TT + 16 * l, src + (ok ? 2 << a.pg.shift : 0), ok);
            }
        };

        int ids = page_ids(0);
#pragma unroll
        for (int i = 0; i < S::STAGES - 1; i++) {
            if (i < count) copy_tile(i, ids);
            asm volatile("cp.async.commit_group;" ::: "memory");
            ids = page_ids(i + 1);
        }
        for (int i = 0; i < count; i++) {
            asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 2) : "memory");
            __syncwarp();                                    // all lanes' copies of tile i; all have read tile i - 1
            if (i + S::STAGES - 1 < count) copy_tile(i + S::STAGES - 1, ids);
            asm volatile("cp.async.commit_group;" ::: "memory");
            ids = page_ids(i + S::STAGES);
            const uint8_t *st = smem + (w * S::STAGES + i % S::STAGES) * S::TILE;
            const int tok0 = token0 + i * kAttWarps * TT;
            const bool edge = tok0 < sp.lo || tok0 + TT > sp.hi;

            // scores, tokens 16 g + r and + 8 by heads 2 c and 2 c + 1
            constexpr int G = TT / 16;
            float s[NT][G][4];
#pragma unroll
            for (int g = 0; g < G; g++) {
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int e = 0; e < 4; e++) s[nt][g][e] = 0.f;
                constexpr int NP = RB / (4 * S::KP), JP = S::KP * 4 / bits_of(F);    // pieces, pairs of each
#pragma unroll
                for (int p = 0; p < NP; p++) {
                    const int byte = (4 * p + c) * S::KP;
                    uint32_t x[JP], y[JP];
                    k_pairs<F>(lds<S::KP>(st, k_place<RB>(16 * g + r, byte)), x);
                    k_pairs<F>(lds<S::KP>(st, k_place<RB>(16 * g + r + 8, byte)), y);
#pragma unroll
                    for (int j = 0; j < JP / 2; j++) {
                        const int ks = p * (JP / 2) + j;
#pragma unroll
                        for (int nt = 0; nt < NT; nt++)
#pragma unroll
                            for (int q = 0; q < S::QT; q++) {
                                uint2 v;
                                if constexpr (S::QREG) v = qr[q][nt][ks];
                                else v = ((const uint2 *)qf)[((q * NT + nt) * S::KS + ks) * 32 + l];
                                mma<C>(s[nt][g], x[2 * j], y[2 * j], x[2 * j + 1], y[2 * j + 1], v.x, v.y);
                            }
                    }
                }
            }
            // base-2 exponents; masked ones are -inf
            float sv[G][2];
#pragma unroll
            for (int g = 0; g < G; g++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const int row = 16 * g + r + 8 * h;
                    float sk = 1.f;
                    sv[g][h] = 1.f;
                    if (S::CODED) {
                        const uint16_t *sc = (const uint16_t *)(st + 2 * TT * RB);
                        sk = f16_val(sc[row]);
                        sv[g][h] = fmaxf(f16_val(sc[TT + row]), kF16Min);    // 0 or NaN: of no token
                    }
                    const bool out = edge && (tok0 + row < sp.lo || tok0 + row >= sp.hi);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            float &x = s[nt][g][2 * h + e];
                            x = S::CODED ? (x - ho[nt][e]) * (hf[nt][e] * sk) : x * hf[nt][e];
                            if (out) x = -INFINITY;
                        }
                }
            // Weights 2^(s - R) sv of at most 2^15. R rises, to 7 below the largest exponent
            // (of the weight), only when one would be above: seldom after the first tiles.
            float wt[NT][G][4], most = 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int g = 0; g < G; g++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        wt[nt][g][e] = exp2_fast(s[nt][g][e] - R[nt][e & 1]);
                        most = fmaxf(most, wt[nt][g][e] * sv[g][e >> 1]);
                    }
            if (__any_sync(0xffffffffu, most > 32768.f)) {
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        float top = kLow;
#pragma unroll
                        for (int g = 0; g < G; g++)
#pragma unroll
                            for (int h = 0; h < 2; h++)
                                top = fmaxf(top, s[nt][g][2 * h + e] + (S::CODED ? log2f(sv[g][h]) : 0.f));
#pragma unroll
                        for (int o = 4; o < 32; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        const float up = fmaxf(R[nt][e], top - 7.f), f = exp2_fast(R[nt][e] - up);
                        R[nt][e] = up;
                        sum[nt][e] *= f;
#pragma unroll
                        for (int m = 0; m < S::MT; m++) {
                            O[nt][m][e] *= f;
                            O[nt][m][2 + e] *= f;
                        }
#pragma unroll
                        for (int g = 0; g < G; g++)
#pragma unroll
                            for (int h = 0; h < 2; h++) wt[nt][g][2 * h + e] = exp2_fast(s[nt][g][2 * h + e] - up);
                    }
            }
            // weighted v: heads' weights by tokens become the right factor by a transposition
#pragma unroll
            for (int g = 0; g < G; g++) {
                uint32_t p[NT][S::PT][2];
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        float x = wt[nt][g][2 * h], y = wt[nt][g][2 * h + 1];
                        sum[nt][0] += x;
                        sum[nt][1] += y;
                        x *= sv[g][h];
                        y *= sv[g][h];
#pragma unroll
                        for (int i = 0; i < S::PT; i++) {
                            const uint32_t v = pack(x, y, C{});
                            if (i + 1 < S::PT) {
                                const float2 f = unpack(v, C{});
                                x -= f.x;
                                y -= f.y;
                            }
                            p[nt][i][h] = transpose8(v);
                        }
                    }
                constexpr int NP = RB / (8 * S::VP), CH = S::VP * 8 / bits_of(F);    // pieces, channels of each
#pragma unroll
                for (int q = 0; q < NP; q++) {
                    const int byte = (8 * q + r) * S::VP, row = 16 * g + 2 * c;
                    const uint8_t *at = st + TT * RB;
                    uint32_t x[CH], y[CH];
                    v_pairs<F>(lds<S::VP>(at, v_place<RB>(row, byte)), lds<S::VP>(at, v_place<RB>(row + 1, byte)), x);
                    v_pairs<F>(lds<S::VP>(at, v_place<RB>(row + 8, byte)), lds<S::VP>(at, v_place<RB>(row + 9, byte)), y);
#pragma unroll
                    for (int m = 0; m < CH / 2; m++)
#pragma unroll
                        for (int nt = 0; nt < NT; nt++)
#pragma unroll
                            for (int i = 0; i < S::PT; i++)
                                mma<C>(O[nt][q * (CH / 2) + m], x[2 * m], x[2 * m + 1], y[2 * m], y[2 * m + 1], p[nt][i][0], p[nt][i][1]);
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        // The four warps' parts, through the rings' memory.
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int e = 0; e < 2; e++)
#pragma unroll
                for (int o = 4; o < 32; o *= 2) sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], o);
        __syncthreads();
        float *mine = (float *)smem + w * HT * (D + 2);
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int h = 8 * nt + 2 * c + e;
                constexpr int MP = S::VP * 4 / bits_of(F);    // row tiles of a piece
#pragma unroll
                for (int m = 0; m < S::MT; m++)
                    *(float2 *)(mine + h * D + (8 * (m / MP) + r) * (2 * MP) + 2 * (m % MP)) =
                        make_float2(O[nt][m][e] * v_factor<F>(0), O[nt][m][2 + e] * v_factor<F>(1));
                if (r == 0) {
                    mine[HT * D + h] = R[nt][e];
                    mine[HT * D + HT + h] = sum[nt][e];
                }
            }
        __syncthreads();
        const bool all = n == sp.tiles;
        // a part that is not all of its sequence: its first piece in this CTA's share or the last
        float *part = a.parts + (size_t)(2 * blockIdx.x + (t == share * blockIdx.x ? 0 : 1)) * part_floats<HT, D>();
        for (int i = tid; i < nh * (D / 4); i += 32 * kAttWarps) {
            const int h = i / (D / 4), d = 4 * (i % (D / 4));
            const float *src = (const float *)smem;
            float top = kLow;
#pragma unroll
            for (int x = 0; x < kAttWarps; x++) top = fmaxf(top, src[x * HT * (D + 2) + HT * D + h]);
            float total = 0.f, o[4] = {};
#pragma unroll
            for (int x = 0; x < kAttWarps; x++) {
                const float *from_w = src + x * HT * (D + 2);
                const float f = exp2_fast(from_w[HT * D + h] - top);
                total = fmaf(f, from_w[HT * D + HT + h], total);
                const float4 v = *(const float4 *)(from_w + h * D + d);
                o[0] = fmaf(f, v.x, o[0]);
                o[1] = fmaf(f, v.y, o[1]);
                o[2] = fmaf(f, v.z, o[2]);
                o[3] = fmaf(f, v.w, o[3]);
            }
            if (all) {
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] = total != 0.f ? o[e] / total : 0.f;
                store4_any(a.y, b * a.ys + (int64_t)(h0 + h) * D + d, a.dtype, o);
                if (a.lse && d == 0)
                    a.lse[(int64_t)b * a.hq + h0 + h] = total != 0.f ? (top + log2f(total)) * 0.693147181f : -INFINITY;
            } else {
                *(float4 *)(part + h * D + d) = make_float4(o[0], o[1], o[2], o[3]);
                if (d == 0) {
                    part[HT * D + h] = top;
                    part[HT * D + HT + h] = total;
                }
            }
        }
        if (!a.whole && tid == 0 && from + n < sp.tiles && from == 0) {
            // begun here, ended by CTA blockIdx.x + count - 1
            const long long last = (t + sp.tiles - 1) / share;
            ((Joined *)(a.parts + (size_t)2 * gridDim.x * part_floats<HT, D>()))[blockIdx.x] =
                Joined{(int)(last - blockIdx.x) + 1, 2 * (int)blockIdx.x + (t == share * blockIdx.x ? 0 : 1), b, vh};
        }
        if (a.whole) {
            t += gridDim.x;
        } else {
            t += n;
            if (vh == VH - 1 && from + n == sp.tiles) {
                before += sp.tiles;
                b++;
            }
        }
    }
}

// Joins the parts of the piece that CTA blockIdx.x of the kernel above began and others ended.
template <int HT, int D>
__global__ void __launch_bounds__(256) kv_join_kernel(AttendArgs a) {
    griddep_wait();
    griddep_launch();
    const Joined j = ((const Joined *)(a.parts + (size_t)2 * gridDim.x * part_floats<HT, D>()))[blockIdx.x];
    if (j.count == 0) return;
    const int chunks = (a.groups + HT - 1) / HT, hk = j.vh / chunks, g0 = (j.vh - hk * chunks) * HT;
    const int nh = min(HT, a.groups - g0), h0 = hk * a.groups + g0;
    auto part = [&](int i) {
        return a.parts + (size_t)(i == 0 ? j.first : 2 * (blockIdx.x + i)) * part_floats<HT, D>();
    };
    for (int i = threadIdx.x; i < nh * (D / 4); i += 256) {
        const int h = i / (D / 4), d = 4 * (i % (D / 4));
        float top = kLow, total = 0.f, o[4] = {};
#pragma unroll 8
        for (int x = 0; x < j.count; x++) top = fmaxf(top, part(x)[HT * D + h]);
#pragma unroll 4
        for (int x = 0; x < j.count; x++) {
            const float *p = part(x);
            const float f = exp2_fast(p[HT * D + h] - top);
            total = fmaf(f, p[HT * D + HT + h], total);
            const float4 v = *(const float4 *)(p + h * D + d);
            o[0] = fmaf(f, v.x, o[0]);
            o[1] = fmaf(f, v.y, o[1]);
            o[2] = fmaf(f, v.z, o[2]);
            o[3] = fmaf(f, v.w, o[3]);
        }
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] = total != 0.f ? o[e] / total : 0.f;
        store4_any(a.y, j.b * a.ys + (int64_t)(h0 + h) * D + d, a.dtype, o);
        if (a.lse && d == 0)
            a.lse[(int64_t)j.b * a.hq + h0 + h] = total != 0.f ? (top + log2f(total)) * 0.693147181f : -INFINITY;
    }
}

}  // namespace kv
}  // namespace stepq
