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
// Where sequences are few and short enough, a cluster of CTAs takes each instead, whole, and
// joins its parts through distributed shared memory: no workspace and no second kernel.
// Within a CTA each warp takes every fourth tile, through its own ring of shared memory filled
// by 16-byte asynchronous copies, and waits for no other warp until the piece ends. The ring
// runs on into the next piece's tiles, which arrive while this piece's parts are put together.
//
// Products by mma.sync m16n8k16 with tokens (for K) and channels (for V) as the 16 rows and
// eight query heads as the columns, so that no part of a product is padding where eight heads
// share a key head. HBM bounds the call as long as these keep up; tcgen05 would want 128 rows of
// tokens of which each is used for 8 columns, and codes would have to go back to shared memory.
// Measured (both kernels; 8 key heads of 128 channels, pages of 16 or 64 tokens): 256 x 8,191 tokens in 4 bits
// and 64 query heads 367 us, 6.1 TB/s, where the integer pipe is busy half of the time at half the issue
// rate; 128 x 4,096 in 8 bits 174 us, 6.3 TB/s; 64 ragged sequences of 131,072 in bf16 85 us, 6.3 TB/s, 4 us
// of which pass before the first tile is asked for and 4 in the second kernel; 37 tokens 4.1 us.
// The order of channels within a product is free, so a lane takes whole 16-byte pieces of a
// row and the queries are laid out to match. Codes become fp16 exactly. For bf16 vectors over 4 bits those of
// K enter as they are, u 2^-24 (a mask leaves a subnormal number), and their offset 8 sum q is
// subtracted from the sum. The tensor cores line products up by the exponents of normal numbers, as if u were
// 1024, which cuts such sums off after some 17 bits: a score is within D 2^-17 of scale times its row's scale
// times the largest |q|, 1e-4 for normal queries and keys of 128 channels, where a weight's one term is within
// 5e-4 and the output's rounding within 4e-3. Codes without their offset take an instruction more for a pair: 256 x
// 8,191 tokens 397 us, so 367. Elsewhere they enter so: fp16 vectors over 4 bits take 1 to 4% longer for it,
// 8 bits nothing.
//
// Between the products (whose factors are sums of 16-bit terms, see Shape) everything is fp32.
#pragma once

#include <type_traits>

#include "device.cuh"
#include "kv.cuh"

namespace stepq {
namespace kv {

constexpr int kAttWarps = 4, kParts = 8 * kAttWarps;           // warps of a CTA, of a cluster
constexpr float kLow = -3.402823466e+38f;

// Workspace: for each CTA c two parts (2 c: the piece that its share begins with, 2 c + 1: one
// that it ends with) of HT heads, [HT][D] of O and then R and l [HT] each. Behind them, for each
// (sequence, virtual head) or, where those are more than the CTAs, for each CTA, which parts the
// piece has that it begins and others end.
struct Joined {
    int count, first, b, vh;        // parts; the first one's number, the others are those of the next CTAs
};
template <int HT, int D> __host__ __device__ constexpr int part_floats() { return HT * (D + 2); }

template <int F> struct Compute { using T = la::f16; };
template <> struct Compute<STEPQ_KV_BF16> { using T = la::bf16; };

// Shape of a variant. LARGE: of calls whose warps take many tiles (codes of up to 128 head channels).
// Queries and weights enter the products as sums of QT and PT terms of the pages' 16-bit type (fp16 for
// codes), as many as the vectors' type T asks for:
//  * queries of bf16 and fp16 are one term of fp16 (exactly, down to 2^-39 of their head's largest; of RAW every
//    second pair down to 2^-35), of bf16 one or two; of fp32 two of fp16 are within 2^-22, three of bf16 within 2^-24.
//  * outputs in bf16: a weight's one term of fp16 is within 2^-11, an eighth of the output's own rounding;
//    of bf16 it would have that rounding again, and two are within 2^-16. Outputs in fp16 take two terms
//    of either; in fp32 two of fp16, three of bf16.
template <int F_, int D_, int NT_, class T_, bool LARGE_ = false>
struct Shape {
    using T = T_;
    static constexpr bool LARGE = LARGE_;
    using Larger = Shape<F_, D_, NT_, T_, coded(F_) && NT_ * D_ <= 128>;
    static constexpr int F = F_, D = D_, NT = NT_;
    static constexpr bool BF16 = std::is_same<T, la::bf16>::value, WIDE = std::is_same<T, float>::value;
    static constexpr int QT = F == STEPQ_KV_BF16 ? (BF16 ? 1 : WIDE ? 3 : 2) : (WIDE ? 2 : 1);
    static constexpr int PT = F == STEPQ_KV_BF16 ? (WIDE ? 3 : 2) : (BF16 ? 1 : 2);
    static constexpr int HT = 8 * NT;                        // heads of a CTA
    static constexpr int RB = row_bytes(F, D);
    static constexpr bool CODED = coded(F);
    // A tile: 4 KB of codes of up to 128 head channels, else 8 or 16; 16 to 64 tokens. Twice as much
    // leaves less to do a token, and takes longer until the first output: 256 x 8,191 tokens in 4 bits
    // 409 us, LARGE 372; 128 x 4,096 in 8 bits 189 and 178; 8 x 24 in 4 bits 5.4 and 6.4.
    static constexpr int WANT = CODED ? (LARGE ? 64 : 32) * (NT * D > 128 ? NT * D : 128) : 64 * (D > 128 ? D : 128);
    static constexpr int FIT = WANT / (2 * RB), TT = FIT > 64 ? 64 : FIT;
    static constexpr int ST = NT * D >= 256 || TT == 16 ? 16 : 32;       // taken at once
    static_assert(TT >= 16 && TT % ST == 0, "a tile is whole parts");
    static constexpr int TILE = 2 * TT * RB + (CODED ? 4 * TT : 0);
    static constexpr int OFF_HEAD = QT * NT * (D / 16) * 256;          // behind the queries [QT][NT][D / 16][32] uint2:
                                                                       // float [2][HT]: factor, offset
    static constexpr int OFF_SUM = OFF_HEAD + 2 * HT * 4;              // float [kAttWarps][2][HT]: R, l
    static constexpr int OFF_SCAN = OFF_SUM + kAttWarps * 2 * HT * 4;  // int64 [kAttWarps + 3]
    // of clusters: float [HT][kParts + 2], int [kParts], float4 [kAttWarps][32]
    static constexpr int OFF_PART = (OFF_SCAN + 8 * (kAttWarps + 3) + 15) / 16 * 16;
    static constexpr int OFF_RING = (OFF_PART + (HT * (kParts + 2) + kParts) * 4 + kAttWarps * 512 + 127) / 128 * 128;
    // CTAs of a multiprocessor with rings of so many stages, by shared memory and by registers
    // (16 heads of 64 channels and fp32 vectors: 64 x 4,096 tokens in 8 bits 118 us with three, 76 with two)
    static constexpr int BY_REGS = NT * D >= 256 || (NT == 2 && WIDE) ? 2 : 3;
    static constexpr int smem(int stages) { return OFF_RING + kAttWarps * stages * TILE; }
    static constexpr int resident(int stages) {
        const int n = 227 * 1024 / (smem(stages) + 1024);
        return n < BY_REGS ? n : BY_REGS;
    }
    // What a piece costs beside its tiles, in tiles: a share of many short pieces took longer than others.
    // 69 ragged sequences, 94,875 tokens in fp16, 5 key heads of 128 (us): none 50.8, 4 extra 45.7, 7 43.4, 10 43.0,
    // 20 43.0; 16 query heads each 65.8, 50.5, 47.5, 44.5, 44.0; 100 ragged, 300,000 tokens in
    // 4 bits 63.1, 52.5 (4 extra), 47.6 (10). Equal lengths: no change.
    static constexpr int EXTRA = 10;
    // Tiles a warp up to which clusters take whole sequences: 8 light ones, 2 heavy ones. 32 ragged sequences of
    // 500 tokens, 4 key heads of 128 with 16 query heads in 8 bits: up to 8 tiles 21.5 us, in shares 14.9;
    // 8 x 1,500 in fp16, 8 key heads with 4: 13.1 and 14.9.
    static constexpr int ROOM = 16384 / (TT * NT * D), WHOLE = ROOM > 8 ? 8 : ROOM < 2 ? 2 : ROOM;
    static constexpr int STAGES = CODED && !LARGE ? 3 : 2;   // of calls that fill the GPU
    static_assert(TILE >= HT * D * 4, "a warp's part is put together in one stage of its ring");
    static constexpr int KP = RB / 4 < 16 ? RB / 4 : 16;     // bytes a lane reads of a row of K at once
    static constexpr int VP = RB / 8 < 16 ? RB / 8 : 16;     // and of V
    static constexpr int KS = D / 16;                        // steps of K's product
    static constexpr int MT = D / 16;                        // row tiles of V's
    static constexpr bool QREG = QT * NT * KS <= 16;         // queries kept in registers
    using C = typename Compute<F>::T;
    static constexpr bool RAW = F == STEPQ_KV_INT4 && BF16;  // K's codes enter with their offset, at 2^-24
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
// d += A B for the terms B[t] of a right factor. The tensor cores' sums are cut off, not rounded, which adds up
// over many steps: for fp32 outputs (WIDE) each product's own sum, the smallest term
// first, is added with rounding.
template <class C, bool WIDE, int T, class Term>
__device__ __forceinline__ void mma_terms(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, Term &&term) {
    if (WIDE) {
        float sum[4] = {};
#pragma unroll
        for (int t = T - 1; t >= 0; t--) {
            const uint2 b = term(t);
            mma<C>(sum, a0, a1, a2, a3, b.x, b.y);
        }
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            const uint64_t v = fadd2(f2(d[e], d[e + 1]), f2(sum[e], sum[e + 1]));
            d[e] = f2lo(v);
            d[e + 1] = f2hi(v);
        }
    } else {
#pragma unroll
        for (int t = 0; t < T; t++) {
            const uint2 b = term(t);
            mma<C>(d, a0, a1, a2, a3, b.x, b.y);
        }
    }
}
template <int N> struct alignas(4 * N) Words { uint32_t w[N]; };
template <int BYTES>
__device__ __forceinline__ Words<BYTES / 4> lds(const uint8_t *tile, uint32_t at) {
    return *(const Words<BYTES / 4> *)(tile + at);
}
// Pages pass through L2 once a call: what else lies there stays (when it was added, with the usual order of
// eviction and with this one: 200,003 tokens of 2 x 256 channels 75 and 71 us; 524,288 of 8 x 128 in 8 bits 185 and 181).
__device__ __forceinline__ uint64_t streaming() {
    uint64_t p;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

// This thread's groups of copies have landed, but for the newest N.
template <int N>
__device__ __forceinline__ void wait_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Place of byte `at` (row * RB + byte) of a tile's rows: 16-byte pieces change places within 128
// bytes so that the lanes that read at once meet no bank twice. They read 64 bytes each of
// rows r and r + 1 (K), of V 16 of eight rows (16 bits) or up to 32 of rows r, r + 2, r + 4 and r + 6.
template <int RB>
__device__ __forceinline__ uint32_t k_place(int row, int byte) {
    return (uint32_t)(row * RB + byte) ^ (RB >= 128 ? (row & 1) << 6 : 0);
}
template <int F, int RB>
__device__ __forceinline__ uint32_t v_place(int row, int byte) {
    return (uint32_t)(row * RB + byte) ^ (!coded(F) ? (row & 7) << 4 : RB >= 64 ? ((row >> 1) & 3) << 5 : ((row >> 2) & 1) << 5);
}

__device__ __forceinline__ uint32_t hadd2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("add.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// Codes without their offset as pairs of fp16, exactly: 0x6400 | u is 1024 + u, less 1024 + 2^(b-1);
// 0x6400 | 16 u is 1024 + 16 u, of which a 16th less 64 + 8.
__device__ __forceinline__ uint32_t codes8(uint32_t w, uint32_t bytes) { return hadd2(__byte_perm(w, 0x64646464u, bytes), 0xe480e480u); }
__device__ __forceinline__ uint32_t codes4(uint32_t w) { return hadd2(and_or(w, 0x000f000fu, 0x64006400u), 0xe408e408u); }
__device__ __forceinline__ uint32_t codes4_high(uint32_t w) {
    return hfma2(and_or(w, 0x00f000f0u, 0x64006400u), 0x2c002c00u, 0xd480d480u);
}

// A lane's piece of a row of K as pairs of the compute type, in the order that Queries::put() gives
// the queries. RAW: codes with their offset at 2^-24, for the odd pairs 2^-20.
template <int F, bool RAW, int N>
__device__ __forceinline__ void k_pairs(const Words<N> &x, uint32_t (&p)[N * 16 / bits_of(F)]) {
#pragma unroll
    for (int i = 0; i < N; i++) {
        const uint32_t w = x.w[i];
        if constexpr (F == STEPQ_KV_INT8) {
            p[2 * i] = codes8(w, 0x4140);
            p[2 * i + 1] = codes8(w, 0x4342);
        } else if constexpr (F == STEPQ_KV_INT4) {
            const uint32_t y = w >> 8;
            p[4 * i] = RAW ? w & 0x000f000fu : codes4(w);
            p[4 * i + 1] = RAW ? w & 0x00f000f0u : codes4_high(w);
            p[4 * i + 2] = RAW ? y & 0x000f000fu : codes4(y);
            p[4 * i + 3] = RAW ? y & 0x00f000f0u : codes4_high(y);
        } else {
            p[i] = w;
        }
    }
}

// Four 8 x 8 matrices of 16-bit elements, transposed: lanes 8 i .. 8 i + 7 give the rows of matrix i.
__device__ __forceinline__ void load_transposed(uint32_t (&m)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(m[0]), "=r"(m[1]), "=r"(m[2]), "=r"(m[3]) : "r"(at) : "memory");
}
// A lane's pieces of two tokens' rows of V as pairs of tokens, p[channel].
template <int F, int N>
__device__ __forceinline__ void v_pairs(const Words<N> &a, const Words<N> &b, uint32_t (&p)[N * 32 / bits_of(F)]) {
#pragma unroll
    for (int i = 0; i < N; i++) {
        if constexpr (F == STEPQ_KV_INT8) {
            const uint32_t lo = __byte_perm(a.w[i], b.w[i], 0x5140), hi = __byte_perm(a.w[i], b.w[i], 0x7362);
            p[4 * i] = codes8(lo, 0x4140);
            p[4 * i + 1] = codes8(lo, 0x4342);
            p[4 * i + 2] = codes8(hi, 0x4140);
            p[4 * i + 3] = codes8(hi, 0x4342);
        } else {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint32_t x = __byte_perm(a.w[i], b.w[i], h ? 0x7632 : 0x5410), y = x >> 8;
                p[8 * i + 4 * h] = codes4(x);
                p[8 * i + 4 * h + 1] = codes4_high(x);
                p[8 * i + 4 * h + 2] = codes4(y);
                p[8 * i + 4 * h + 3] = codes4_high(y);
            }
        }
    }
}

// Thread-block clusters: this CTA's place, the barrier of all their threads (which shows each other's
// shared memory), and where CTA `rank` has what lies here at p.
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <class P>
__device__ __forceinline__ const P *in_cluster(const P *p, uint32_t rank) {
    uint64_t r;
    asm("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(p), "r"(rank));
    return (const P *)r;
}

// A piece: tiles from .. from + n - 1 of the `tiles` of sequence b, virtual head vh, whose tokens
// [lo, hi) count (a row without any has one tile).
struct Piece {
    int b, vh, from, n, lo, hi, tile0, tiles;
    int turn;                       // of this warp: it takes tiles from + turn, and every `turns`-th after it
    int bad;                        // status of its length
};
template <int TT>
__device__ __forceinline__ void set_span(const AttendArgs &a, int len, Piece &p) {
    const long long most = (long long)a.pg.width << a.pg.shift;
    p.hi = len < 0 ? 0 : len > most ? (int)most : len;
    p.bad = len < 0 ? STEPQ_ERR_ARG : len > most ? STEPQ_ERR_SLOT_RANGE : 0;
    p.lo = p.tile0 = 0;
    if (a.window > 0) {
        p.lo = max(0, p.hi - a.window);
        p.tile0 = p.lo / TT;
    }
    p.tiles = max(1, (p.hi + TT - 1) / TT - p.tile0);
}
template <int TT>
__device__ __forceinline__ int tiles_of(const AttendArgs &a, int len) {
    Piece p;
    set_span<TT>(a, len, p);
    return p.tiles;
}

// a / b, mostly of numbers below 2^32 (a division of 64 bits takes some hundred instructions).
__device__ __forceinline__ long long divided(long long a, long long b) {
    if (((a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
    return a / b;
}
// 2^e for e in [-126, 127].
__device__ __forceinline__ float power2(int e) { return __int_as_float((e + 127) << 23); }

// Queries of a warp's heads w, w + kAttWarps, ..: lane l has pairs 32 k + l of each head's channels,
// pair u the channels 2 u and 2 u + 1, of 4-bit codes 8 (u / 4) + u % 4 and the fourth after it.
template <class S>
struct Queries {
    static constexpr int H = S::HT / kAttWarps, N = S::D / 64;
    static constexpr bool FOURTH = S::F == STEPQ_KV_INT4;
    float2 x[H][N];
    template <class T>
    __device__ __forceinline__ void load_as(const T *q, int nh, int w, int l) {
#pragma unroll
        for (int i = 0; i < H; i++)
#pragma unroll
            for (int k = 0; k < N; k++) {
                const int h = w + i * kAttWarps, u = 32 * k + l;
                const T *at = q + h * S::D + (FOURTH ? 8 * (u / 4) + u % 4 : 2 * u);
                x[i][k] = make_float2(0.f, 0.f);
                if (h < nh && FOURTH) x[i][k] = make_float2(la::to_f32(at[0]), la::to_f32(at[4]));
                else if (h < nh) {
                    const la::Vec<T, 2> v = *(const la::Vec<T, 2> *)at;
                    x[i][k] = make_float2(la::to_f32(v.e[0]), la::to_f32(v.e[1]));
                }
            }
    }
    __device__ __forceinline__ void load(const AttendArgs &a, int b, int h0, int nh, int w, int l) {
        const int64_t at = b * a.qs + (int64_t)h0 * S::D;
        load_as((const typename S::T *)a.q + at, nh, w, l);
    }
    // To shared memory as pairs in the order of K's pieces: of step ks of the product, pair (0, 1)
    // of lane 4 head + c; with each head's factor of the scores and the offset of the codes.
    __device__ __forceinline__ void put(const AttendArgs &a, uint8_t *smem, int w, int l) {
        using C = typename S::C;
        constexpr int F = S::F;
        uint32_t *qf = (uint32_t *)smem;
        float *head_k = (float *)(smem + S::OFF_HEAD), *head_off = head_k + S::HT;
#pragma unroll
        for (int i = 0; i < H; i++) {
            const int h = w + i * kAttWarps;
            float k = a.scale, off = 0.f;
            if (std::is_same<C, la::f16>::value) {
                // scaled by a power of two to below 2^15: fp16 then keeps 2^-39 of the largest
                float top = 0.f;
#pragma unroll
                for (int e = 0; e < N; e++) top = fmax3(top, fabsf(x[i][e].x), fabsf(x[i][e].y));
#pragma unroll
                for (int o = 1; o < 32; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const int ex = max(-126, min(126, 141 - (__float_as_int(top) >> 23)));
#pragma unroll
                for (int e = 0; e < N; e++) x[i][e] = make_float2(x[i][e].x * power2(ex), x[i][e].y * power2(ex));
                k *= power2(-ex);
            }
#pragma unroll
            for (int e = 0; e < N; e++) {
                // pieces of KP bytes go to lanes c in turn: piece, and pair j of it
                constexpr int PC = S::KP * 8 / bits_of(F), JP = PC / 2;          // channels, pairs of a piece
                const int u = 32 * e + l, piece = u / JP, j = u % JP;
                const int pair = (piece / 4) * JP + j, lane = 4 * (h % 8) + piece % 4;
                const float f = S::RAW && (j & 1) ? 0.0625f : 1.f;     // of a code at 2^-20
                float2 rest = make_float2(x[i][e].x * f, x[i][e].y * f);
                float used = 0.f;
#pragma unroll
                for (int t = 0; t < S::QT; t++) {
                    const uint32_t v = pack(rest.x, rest.y, C{});
                    const float2 b = unpack(v, C{});
                    rest = make_float2(rest.x - b.x, rest.y - b.y);
                    used += b.x + b.y;
                    qf[(((t * S::NT + h / 8) * S::KS + pair / 2) * 32 + lane) * 2 + pair % 2] = v;
                }
                off += S::RAW && (j & 1) ? 16.f * used : used;
            }
            if (S::RAW) {
#pragma unroll
                for (int o = 1; o < 32; o *= 2) off += __shfl_xor_sync(0xffffffffu, off, o);
                off *= 8.f * 0x1p-24f;
            }
            if (l == 0) {
                head_k[h] = k;
                head_off[h] = off;
            }
        }
    }
};

// Channels d .. d + 3 of query head h from the sums o of weighted values and `total` of weights.
template <class T>
__device__ __forceinline__ void put_output(const AttendArgs &a, int b, int h, int d, float top, float total, float (&o)[4], int D) {
    const float f = total != 0.f ? 1.f / total : 0.f;
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] = total != 0.f ? o[e] * f : 0.f;
    const int64_t at = b * a.ys + (int64_t)h * D + d;
    la::store_vec<T, 4>((T *)a.y + at, o);
    if (a.lse && d == 0) a.lse[(int64_t)b * a.hq + h] = total != 0.f ? (top + log2f(total)) * 0.693147181f : -INFINITY;
}

// ------------------------------------------------------------------ the kernel
template <class S>
__global__ void __launch_bounds__(32 * kAttWarps, S::BY_REGS) kv_attend_kernel(AttendArgs a) {
    extern __shared__ __align__(128) uint8_t smem[];
    using C = typename S::C;
    constexpr int D = S::D, TT = S::TT, RB = S::RB, NT = S::NT, HT = S::HT, F = S::F;
    const int tid = threadIdx.x, w = tid >> 5, l = tid & 31, r = l >> 2, c = l & 3;
    const int chunks = (a.groups + HT - 1) / HT, VH = a.pg.n_heads * chunks;
    const int items = a.B * VH;                              // far below 2^31: the host sees to it
    const float *head_k = (const float *)(smem + S::OFF_HEAD), *head_off = head_k + HT;
    float *sums = (float *)(smem + S::OFF_SUM);
    long long *scan = (long long *)(smem + S::OFF_SCAN);
    Joined *joined = (Joined *)(a.parts + (size_t)2 * gridDim.x * part_floats<HT, D>());
    griddep_wait();
    griddep_launch();

    // Calls for whole sequences: the CTAs of a cluster take a sequence's tiles in turn.
    const int ctas = a.whole ? (int)cluster_size() : 1, rank = a.whole ? (int)cluster_rank() : 0;
    const int stages = a.stages;                             // S::STAGES, or 1 where no warp has more tiles
    const int turns = ctas * kAttWarps;

    // The share: `left` tiles of all, in the order (sequence, virtual head, tile), from tile `from`
    // of virtual head vh of sequence b on; len is lens[b]. Every piece counts EXTRA tiles more, behind its own.
    long long left = 0, share = 0, past = 0;                 // past: of the share before the piece at hand
    int item = blockIdx.x / ctas;                            // of calls for whole sequences
    int b = 0, vh = 0, from = 0, len = 0;
    if (!a.whole) {
        const int per = (a.B + 32 * kAttWarps - 1) / (32 * kAttWarps), i0 = min(a.B, tid * per), i1 = min(a.B, i0 + per);
        long long mine = 0;
        for (int i = i0; i < i1; i++) mine += tiles_of<TT>(a, a.lens[i]) + S::EXTRA;
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
        share = max(divided(total + gridDim.x - 1, gridDim.x), (long long)(2 * kAttWarps));
        const long long t = share * blockIdx.x;
        left = min(total - t, share);
        if (t < total && t >= (upto - mine) * VH && t < upto * VH) {
            long long p = upto - mine;
            int i = i0, n;
            for (;; i++) {
                n = tiles_of<TT>(a, a.lens[i]) + S::EXTRA;
                if (t < (p + n) * VH) break;
                p += n;
            }
            const long long in = t - p * VH;
            scan[kAttWarps] = i;
            const long long head = divided(in, n);
            scan[kAttWarps + 1] = head;
            scan[kAttWarps + 2] = in - head * n;
        }
        __syncthreads();
        if (tid == 0 && items > (int)gridDim.x) joined[blockIdx.x].count = 0;     // unless a piece goes on elsewhere
        if (left <= 0) return;
        b = (int)scan[kAttWarps];
        vh = (int)scan[kAttWarps + 1];
        from = (int)scan[kAttWarps + 2];
        len = a.lens[b];
        const int n = tiles_of<TT>(a, len);
        if (from >= n) {                                     // in the extra ones behind a piece
            past = n + S::EXTRA - from;
            left -= past;
            from = 0;
            if (++vh == VH) {
                vh = 0;
                if (++b < a.B) len = a.lens[b];
            }
        }
    }

    // The next piece of the share, n = 0 behind the last.
    auto next_piece = [&]() {
        Piece p{};
        if (a.whole) {
            if (item >= items) return p;
            p.b = item / VH;
            p.vh = item - p.b * VH;
            item += gridDim.x / ctas;
            len = a.lens[p.b];
            set_span<TT>(a, len, p);
            p.n = p.tiles;
            p.turn = rank * kAttWarps + w;
        } else {
            if (left <= 0) return p;
            p.b = b;
            p.vh = vh;
            p.from = from;
            set_span<TT>(a, len, p);
            p.n = (int)min((long long)(p.tiles - from), left);
            p.turn = (w + (int)left) & (kAttWarps - 1);      // the share's tiles go round the warps
            left -= p.n;
            from += p.n;
            if (from == p.tiles) {
                left -= S::EXTRA;
                from = 0;
                if (++vh == VH) {
                    vh = 0;
                    if (++b < a.B) len = a.lens[b];
                }
            }
        }
        return p;
    };
    auto count_of = [&](const Piece &p) { return p.n > p.turn ? (p.n - p.turn + turns - 1) / turns : 0; };

    // What is copied next: `more` tiles of a piece, the first at token `tok`; ids: the pages of
    // that tile's octets (eight tokens), -1 behind the table. A page that holds a whole
    // tile is looked up once.
    struct {
        const int32_t *table;
        uint64_t head;
        int tok, more, lo, hi, ids[TT / 8];
    } f{};
    const bool one_page = (1 << a.pg.shift) >= TT;
    const int table_end = a.pg.width << a.pg.shift;
    auto load_ids = [&]() {                                  // nothing here waits for the sequence's length
        if (one_page) {
            f.ids[0] = f.tok < table_end ? f.table[f.tok >> a.pg.shift] : -1;
        } else {
#pragma unroll
            for (int o = 0; o < TT / 8; o++) f.ids[o] = f.tok + 8 * o < table_end ? f.table[(f.tok + 8 * o) >> a.pg.shift] : -1;
        }
    };
    auto fetch_from = [&](const Piece &p) {
        f.table = a.pg.table + p.b * a.pg.table_stride;
        f.head = (uint64_t)(p.vh / chunks) * a.pg.segment;
        f.tok = (p.tile0 + p.from + p.turn) * TT;
        f.more = count_of(p);
        f.lo = p.lo;
        f.hi = p.hi;
        load_ids();
    };
    const uint32_t ring = smem_addr(smem) + S::OFF_RING + w * stages * S::TILE;
    const uint8_t *ring_at = smem + S::OFF_RING + w * stages * S::TILE;
    // Stages are taken in turn: to_fill the next that copies go to, to_read the next that is read.
    int to_fill = 0, to_read = 0, ahead = 0;                 // ahead: tiles copied and not yet read
    // A step copies 512 bytes of rows, 16 a lane: the change of place within 128 bytes is that of the
    // lane's part of the offset and, apart from it, that of the step's.
    const uint32_t k_lane = k_place<RB>(16 * l / RB, 16 * l % RB), v_lane = v_place<F, RB>(16 * l / RB, 16 * l % RB);
    const uint64_t policy = streaming();
    auto copy_tile = [&]() {
        const uint32_t dst = ring + to_fill * S::TILE, to_v = RB << a.pg.shift;
        constexpr int N = TT * RB / 512;                     // steps
        const uint8_t *layer = a.pg.base + f.head;
        const int slot = a.pg.slot(f.tok);
        auto steps = [&](int j0, int n, const uint8_t *k) {  // n steps from j0 on, from k on
            const uint8_t *v = k + to_v;
#pragma unroll
            for (int x = 0; x < n; x++) {
                const int j = j0 + x;
                const uint32_t kj = k_place<RB>(512 * j / RB, 512 * j % RB) ^ (512 * j), vj = v_place<F, RB>(512 * j / RB, 512 * j % RB) ^ (512 * j);
                copy16(dst + 512 * j + (k_lane ^ kj), k + 512 * x, policy);
                copy16(dst + TT * RB + 512 * j + (v_lane ^ vj), v + 512 * x, policy);
            }
        };
        const bool inside = f.tok >= f.lo && f.tok + TT <= f.hi;
        const bool one = one_page && inside && (uint32_t)f.ids[0] < (uint32_t)a.pg.n_pages;
        bool several = inside && !one_page;
        if (one) {
            const uint8_t *page = layer + (uint64_t)(uint32_t)f.ids[0] * a.pg.page_bytes;
            steps(0, N, page + (slot * RB + 16 * l));
            if (S::CODED && l < TT / 4) {                    // K's scales, then V's
                const bool is_v = l >= TT / 8;
                copy16(dst + 2 * TT * RB + 16 * l, page + 2 * to_v + 2 * slot + 16 * (l & (TT / 8 - 1)) + (is_v ? 2 << a.pg.shift : 0), policy);
            }
        } else {
            int mine = f.ids[0];                                 // the page of octet l
#pragma unroll
            for (int o = 0; o < TT / 8; o++) {
                several = several && (uint32_t)f.ids[o] < (uint32_t)a.pg.n_pages;
                if (o > 0 && !one_page) mine = l == o ? f.ids[o] : mine;
            }
            const uint8_t *page = layer + (uint64_t)(uint32_t)mine * a.pg.page_bytes;
            if (several) {
                constexpr int PER = RB >= 64 ? RB / 64 : 1;      // steps of an octet, or octets of a step in two halves
#pragma unroll
                for (int j0 = 0; j0 < N; j0 += PER) {
                    constexpr int two = RB < 64;
                    const int o = 512 * j0 / (8 * RB), id = two && l >= 16 ? f.ids[o + two] : f.ids[o];
                    steps(j0, PER, layer + (uint64_t)(uint32_t)id * a.pg.page_bytes + a.pg.slot(f.tok + 8 * o + (two && l >= 16 ? 8 : 0)) * RB + 16 * l % (8 * RB));
                }
                if (S::CODED && l < TT / 8) {
                    const uint8_t *src = page + 2 * to_v + 2 * a.pg.slot(f.tok + 8 * l);
                    copy16(dst + 2 * TT * RB + 16 * l, src, policy);
                    copy16(dst + 2 * TT * RB + 2 * TT + 16 * l, src + (2 << a.pg.shift), policy);
                }
            } else {
                // rows that are no tokens, or in no page, become zeros
                const int tok_l = f.tok + 8 * l;
                const bool counts = l < TT / 8 && tok_l < f.hi && tok_l + 8 > f.lo;
                if ((uint32_t)mine >= (uint32_t)a.pg.n_pages) {
                    if (counts) raise_error(a.pg.err, STEPQ_ERR_SLOT_RANGE);
                    mine = -1;
                }
#pragma unroll
                for (int j = 0; j < N; j++) {
                    const int at = 512 * j + 16 * l, row = at / RB, byte = at % RB, tok = f.tok + row;
                    const int id = __shfl_sync(0xffffffffu, mine, row / 8);
                    const bool ok = id >= 0 && tok >= f.lo && tok < f.hi;
                    const uint8_t *src = ok ? layer + (uint64_t)(uint32_t)id * a.pg.page_bytes + a.pg.slot(tok) * RB + byte : a.pg.base;
                    copy16(dst + k_place<RB>(row, byte), src, ok);
                    copy16(dst + TT * RB + v_place<F, RB>(row, byte), src + (ok ? to_v : 0), ok);
                }
                if (S::CODED && l < TT / 8) {
                    const bool ok = mine >= 0 && counts;
                    const uint8_t *src = ok ? page + 2 * to_v + 2 * a.pg.slot(tok_l) : a.pg.base;
                    copy16(dst + 2 * TT * RB + 16 * l, src, ok);
                    copy16(dst + 2 * TT * RB + 2 * TT + 16 * l, src + (ok ? 2 << a.pg.shift : 0), ok);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++to_fill == stages) to_fill = 0;
        ahead++;
        f.more--;
        f.tok += turns * TT;
    };

    // What this lane reads of a tile: piece c of row r of K; of V in 16 bits a matrix's row of 16 bytes,
    // of codes piece r of rows 2 c and 2 c + 1. 8 rows, and 8 pieces of V, further on lie the same.
    const uint32_t k_at = k_place<RB>(r, c * S::KP);
    const uint32_t v_at = S::CODED ? v_place<F, RB>(2 * c, r * S::VP) : TT * RB + v_place<F, RB>((l & 7) + (l >> 4) * 8, (l >> 3 & 1) * 16);
    const uint32_t v_at1 = v_place<F, RB>(2 * c + 1, r * S::VP);

    Piece p = next_piece();
    auto first_head = [&](const Piece &x) { return x.vh / chunks * a.groups + x.vh % chunks * HT; };
    auto heads_of = [&](const Piece &x) { return min(HT, a.groups - x.vh % chunks * HT); };
    fetch_from(p);
    // A warp's part of a piece goes through the stage of its ring that was read last.
    auto stage_of = [&](int x, int stage) { return smem + S::OFF_RING + (x * stages + stage) * S::TILE; };
    struct {
        int b, h0, nh;
        bool all;                                            // the piece is its whole sequence
        float *part;                                         // else where it goes
    } out{};
    bool first = true;

    for (;; first = false) {
        const Piece q = p.n > 0 ? next_piece() : p;
        bool rest = p.n > 0 && q.n > 0;                      // q's tiles are not looked at yet
        Queries<S> qs;
        qs.load(a, p.b, first_head(p), p.n > 0 ? heads_of(p) : 0, w, l);
        if (!first) {
            // the warps' parts of the piece before
            auto leave = [&](int h, int d, float top, float total, float(&o)[4]) {
                if (out.all) {
                    put_output<typename S::T>(a, out.b, out.h0 + h, d, top, total, o, D);
                } else {
                    *(float4 *)(out.part + h * D + d) = make_float4(o[0], o[1], o[2], o[3]);
                    if (d == 0) {
                        out.part[HT * D + h] = top;
                        out.part[HT * D + HT + h] = total;
                    }
                }
            };
            auto add = [](float(&o)[4], float k, const float4 &v) {
                o[0] = fmaf(k, v.x, o[0]);
                o[1] = fmaf(k, v.y, o[1]);
                o[2] = fmaf(k, v.z, o[2]);
                o[3] = fmaf(k, v.w, o[3]);
            };
            if (ctas == 1) {
                __syncthreads();
                for (int i = tid; i < out.nh * (D / 4); i += 32 * kAttWarps) {
                    const int h = i / (D / 4), d = 4 * (i % (D / 4));
                    float top = kLow, total = 0.f, o[4] = {};
#pragma unroll
                    for (int x = 0; x < kAttWarps; x++) top = fmaxf(top, sums[2 * x * HT + h]);
#pragma unroll
                    for (int x = 0; x < kAttWarps; x++) {
                        const float k = exp2_fast(sums[2 * x * HT + h] - top);
                        total = fmaf(k, sums[(2 * x + 1) * HT + h], total);
                        add(o, k, *(const float4 *)((const float *)stage_of(x, ((const int *)scan)[x]) + h * D + d));
                    }
                    leave(h, d, top, total, o);
                }
            } else {
                // Weights of all warps' parts, a lane each; then each CTA a share of the channels, its
                // warp x the parts of every CTA's warp x.
                cluster_sync();
                float *weight = (float *)(smem + S::OFF_PART);
                int *stage = (int *)(weight + HT * (kParts + 2));
                float4 *half = (float4 *)(smem + S::OFF_PART + (HT * (kParts + 2) + kParts) * 4);
                for (int h = w; h < out.nh; h += kAttWarps) {
                    float R = kLow, sum = 0.f;
                    if (l < turns) {
                        const float *rl = in_cluster((const float *)sums, l / kAttWarps) + 2 * (l % kAttWarps) * HT + h;
                        R = rl[0];
                        sum = rl[HT];
                        if (h == w) stage[l] = in_cluster((const int *)scan, l / kAttWarps)[l % kAttWarps];
                    }
                    float top = R;
#pragma unroll
                    for (int o = 1; o < 32; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const float k = exp2_fast(R - top);
                    sum *= k;
#pragma unroll
                    for (int o = 1; o < 32; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    weight[h * (kParts + 2) + l] = k;
                    if (l == 0) {
                        weight[h * (kParts + 2) + kParts] = top;
                        weight[h * (kParts + 2) + kParts + 1] = sum;
                    }
                }
                __syncthreads();
                const int n = out.nh * (D / 4), each = (n + ctas - 1) / ctas, end = min(n, (rank + 1) * each);
                for (int i0 = rank * each; i0 < end; i0 += 32) {
                    const int i = i0 + l, h = i / (D / 4), d = 4 * (i % (D / 4));
                    const float *k = weight + h * (kParts + 2);
                    float o[4] = {};
                    if (i < end) {
#pragma unroll 8
                        for (int z = 0; z < ctas; z++) {
                            const float *part = (const float *)stage_of(w, stage[z * kAttWarps + w]) + h * D + d;
                            add(o, k[z * kAttWarps + w], *(const float4 *)in_cluster(part, z));
                        }
                        half[w * 32 + l] = make_float4(o[0], o[1], o[2], o[3]);
                    }
                    __syncthreads();
                    if (w == 0 && i < end) {
#pragma unroll
                        for (int x = 1; x < kAttWarps; x++) add(o, 1.f, half[x * 32 + l]);
                        leave(h, d, k[kParts], k[kParts + 1], o);
                    }
                    __syncthreads();
                }
            }
        }
        if (ctas > 1 && !first) cluster_sync();              // the others have read this CTA's
        if (p.n == 0) break;
        qs.put(a, smem, w, l);
        __syncthreads();                                     // the queries are there, the parts before have been read
        if (tid == 0 && p.bad) raise_error(a.pg.err, p.bad);
        const int slot = 2 * (int)blockIdx.x + (first ? 0 : 1);
        out = {p.b, first_head(p), heads_of(p), p.n == p.tiles, a.parts + (size_t)slot * part_floats<HT, D>()};
        if (!a.whole && tid == 0 && p.from == 0) {
            // begun here, and ended here or by one of the next CTAs
            const Joined j{out.all ? 0 : (int)divided(past + p.tiles - 1, share) + 1, slot, p.b, p.vh};
            if (items <= (int)gridDim.x) joined[p.b * VH + p.vh] = j;
            else if (j.count) joined[blockIdx.x] = j;
        }
        past += p.from + p.n == p.tiles ? p.n + S::EXTRA : p.n;
        const int count = count_of(p), tok_first = (p.tile0 + p.from + p.turn) * TT;

        // The largest weight, 2^-low. 2^15 leaves the least bits that terms in fp16 lose; in bf16 V may be as large as
        // fp32 goes, which sums of n tokens with weights of 1 / n at most do not pass, and weights have fp32's exponents.
        const int low = F == STEPQ_KV_BF16 ? 32 - __clz(p.hi - p.lo) : -15;
        const float most_wt = power2(-low);

        // pairs are of heads 2 c and 2 c + 1
        uint64_t hf[NT], ho[NT], R[NT], sum[NT];
        float O[NT][S::MT][4];
        const uint2 *qf = (const uint2 *)smem;
        uint2 qr[S::QREG ? S::QT : 1][S::QREG ? NT : 1][S::QREG ? S::KS : 1];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            hf[nt] = *(const uint64_t *)(head_k + 8 * nt + 2 * c);
            ho[nt] = *(const uint64_t *)(head_off + 8 * nt + 2 * c);
            R[nt] = f2s(kLow);
            sum[nt] = 0;
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
                    for (int ks = 0; ks < S::KS; ks++) qr[i][nt][ks] = qf[((i * NT + nt) * S::KS + ks) * 32 + l];
        }

        // Before the first tile is read all stages but one are on their way, those behind p's last
        // with q's tiles; then one more a tile.
        if (f.more == 0 && rest) {
            fetch_from(q);
            rest = false;
        }
        for (int i = min(0, ahead - (stages - 1));; i++) {
            __syncwarp();                                    // all have read the tile before
            if (f.more > 0 && ahead < (i >= 0 && i < count ? stages : stages - 1)) {
                copy_tile();
                if (f.more == 0 && rest) {
                    fetch_from(q);
                    rest = false;
                } else {
                    load_ids();
                }
            }
            if (i < 0) continue;
            if (i == count) break;
            // the copies of this tile have landed once no more than those behind it are open
            if (ahead == S::STAGES) wait_but<S::STAGES - 1>();
            else wait_but<0>();
            __syncwarp();
            const uint8_t *st = ring_at + to_read * S::TILE;
            if (++to_read == stages) to_read = 0;
            ahead--;
            constexpr int G = S::ST / 16;
#pragma unroll 1
            for (int sub = 0; sub < TT; sub += S::ST) {
                const int tok0 = tok_first + i * turns * TT + sub;
                const bool edge = tok0 < p.lo || tok0 + S::ST > p.hi;
                const uint8_t *rows = st + sub * RB;

                // scores, tokens 16 g + r and + 8 by heads 2 c and 2 c + 1
                float s[NT][G][4];
#pragma unroll
                for (int g = 0; g < G; g++) {
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int e = 0; e < 4; e++) s[nt][g][e] = 0.f;
                    constexpr int NP = RB / (4 * S::KP), JP = S::KP * 4 / bits_of(F);    // pieces, pairs of each
#pragma unroll
                    for (int x = 0; x < NP; x++) {
                        // pieces 4 x + c: an odd x differs from an even one in the bit that rows change
                        const uint8_t *at = rows + ((x & 1) * 4 * S::KP ^ k_at) + (x >> 1) * 8 * S::KP + 16 * g * RB;
                        uint32_t k0[JP], k8[JP];
                        k_pairs<F, S::RAW>(lds<S::KP>(at, 0), k0);
                        k_pairs<F, S::RAW>(lds<S::KP>(at, 8 * RB), k8);
#pragma unroll
                        for (int j = 0; j < JP / 2; j++) {
                            const int ks = x * (JP / 2) + j;
#pragma unroll
                            for (int nt = 0; nt < NT; nt++)
                                mma_terms<C, S::WIDE, S::QT>(s[nt][g], k0[2 * j], k8[2 * j], k0[2 * j + 1], k8[2 * j + 1], [&](int t) {
                                    if constexpr (S::QREG) return qr[t][nt][ks];
                                    else return qf[((t * NT + nt) * S::KS + ks) * 32 + l];
                                });
                        }
                    }
                }
                // base-2 exponents x = (s - ho) sk hf, rounded before the reference is taken from them: a difference of
                // large scores is then a difference of what the reference was found from. Masked ones are -inf.
                // sv: V's scales, for the reference at least 2^-24 (1 where there is no token); least: the least as it is.
                float sv[G][2], least = 1.f;
                auto v_scale = [&](int g, int h) {
                    return f16_val(((const uint16_t *)(st + 2 * TT * RB))[TT + sub + 16 * g + r + 8 * h]);
                };
                uint64_t x[NT][G][2];
#pragma unroll
                for (int g = 0; g < G; g++)
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        float sk = 1.f;
                        sv[g][h] = 1.f;
                        if (S::CODED) {
                            sk = f16_val(((const uint16_t *)(st + 2 * TT * RB))[sub + 16 * g + r + 8 * h]) * (S::RAW ? 0x1p24f : 1.f);
                            sv[g][h] = fmaxf(fabsf(v_scale(g, h)), 0x1p-24f);
                            least = fminf(least, v_scale(g, h));
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) {
                            x[nt][g][h] = f2(s[nt][g][2 * h], s[nt][g][2 * h + 1]);
                            if (S::RAW) x[nt][g][h] = fsub2(x[nt][g][h], ho[nt]);
                            if (S::CODED) x[nt][g][h] = fmul2(x[nt][g][h], f2s(sk));
                            x[nt][g][h] = fmul2(x[nt][g][h], hf[nt]);        // may be large, where sk makes up for it
                        }
                    }
                if (edge) {
#pragma unroll
                    for (int g = 0; g < G; g++)
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            const int tok = tok0 + 16 * g + r + 8 * h;
                            if (tok >= p.lo && tok < p.hi) continue;
                            sv[g][h] = 1.f;                  // what lies there may be infinite: its weight of 0 stays 0
#pragma unroll
                            for (int nt = 0; nt < NT; nt++) x[nt][g][h] = f2s(-INFINITY);
                        }
                }
                // Weights 2^(s - R) sv of at most `most_wt`. R rises, until the largest is 8 bits below,
                // only when one would be above: seldom after the first tiles.
                uint64_t wt[NT][G][2], wv[NT][G][2];
                auto weights = [&](int nt) {
                    const uint64_t less_r = f2(-f2lo(R[nt]), -f2hi(R[nt]));
                    float most = 0.f;
#pragma unroll
                    for (int g = 0; g < G; g++)
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            const uint64_t t = fadd2(x[nt][g][h], less_r);
                            wt[nt][g][h] = f2(exp2_fast(f2lo(t)), exp2_fast(f2hi(t)));
                            wv[nt][g][h] = S::CODED ? fmul2(wt[nt][g][h], f2s(sv[g][h])) : wt[nt][g][h];
                            most = fmax3(most, f2lo(wv[nt][g][h]), f2hi(wv[nt][g][h]));
                        }
                    return most;
                };
                float most = weights(0);
                if (NT > 1) most = fmaxf(most, weights(NT - 1));
                // Rows of zeros, of a page that nothing was written to or of none, have code 0 and scale 0: their values take
                // the scale as it is. (With a vote of their own 256 x 8,191 tokens in 4 bits took 371 us, so 368.)
                const bool zeros = S::CODED && least <= 0.f;
                if (__any_sync(0xffffffffu, zeros || most > most_wt)) {
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        float up[2], f[2];
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            float top = kLow;
                            auto half = [&](uint64_t v) { return e ? f2hi(v) : f2lo(v); };
#pragma unroll
                            for (int g = 0; g < G; g++)
#pragma unroll
                                for (int h = 0; h < 2; h++)
                                    top = fmaxf(top, half(x[nt][g][h]) + (S::CODED ? log2f(sv[g][h]) : 0.f));
#pragma unroll
                            for (int o = 4; o < 32; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                            up[e] = fmaxf(half(R[nt]), top + (float)(low + 8));
                            f[e] = exp2_fast(half(R[nt]) - up[e]);
#pragma unroll
                            for (int m = 0; m < S::MT; m++) {
                                O[nt][m][e] *= f[e];
                                O[nt][m][2 + e] *= f[e];
                            }
                        }
                        R[nt] = f2(up[0], up[1]);
                        sum[nt] = fmul2(sum[nt], f2(f[0], f[1]));
                        weights(nt);
#pragma unroll
                        for (int g = 0; g < G; g++)
#pragma unroll
                            for (int h = 0; h < 2; h++)
                                if (zeros && sv[g][h] != 1.f) wv[nt][g][h] = fmul2(wt[nt][g][h], f2s(v_scale(g, h)));
                    }
                }
                // weighted v: heads' weights by tokens become the right factor by a transposition
#pragma unroll
                for (int g = 0; g < G; g++) {
                    uint2 pw[NT][S::PT];
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            sum[nt] = fadd2(sum[nt], wt[nt][g][h]);
                            uint64_t left = wv[nt][g][h];
#pragma unroll
                            for (int t = 0; t < S::PT; t++) {
                                const uint32_t v = pack(f2lo(left), f2hi(left), C{});
                                if (t + 1 < S::PT) {
                                    const float2 u = unpack(v, C{});
                                    left = fsub2(left, f2(u.x, u.y));
                                }
                                (h ? pw[nt][t].y : pw[nt][t].x) = transpose8(v);
                            }
                        }
                    if constexpr (!S::CODED) {
                        // row tile m: channels 16 m + r and 16 m + 8 + r
#pragma unroll
                        for (int m = 0; m < S::MT; m++) {
                            uint32_t v[4];
                            load_transposed(v, smem_addr(rows) + (v_at ^ ((m & 3) << 5)) + (m >> 2) * 128 + 16 * g * RB);
#pragma unroll
                            for (int nt = 0; nt < NT; nt++)
                                mma_terms<C, S::WIDE, S::PT>(O[nt][m], v[0], v[1], v[2], v[3], [&](int t) { return pw[nt][t]; });
                        }
                    } else {
                        constexpr int NP = RB / (8 * S::VP), CH = S::VP * 8 / bits_of(F);    // pieces, channels of each
#pragma unroll
                        for (int z = 0; z < NP; z++) {
                            const uint8_t *at = rows + TT * RB + 8 * z * S::VP + 16 * g * RB;
                            uint32_t x[CH], y[CH];
                            v_pairs<F>(lds<S::VP>(at, v_at), lds<S::VP>(at, v_at1), x);
                            v_pairs<F>(lds<S::VP>(at, v_at + 8 * RB), lds<S::VP>(at, v_at1 + 8 * RB), y);
#pragma unroll
                            for (int m = 0; m < CH / 2; m++)
#pragma unroll
                                for (int nt = 0; nt < NT; nt++)
                                    mma_terms<C, S::WIDE, S::PT>(O[nt][z * (CH / 2) + m], x[2 * m], x[2 * m + 1], y[2 * m], y[2 * m + 1],
                                                                 [&](int t) { return pw[nt][t]; });
                        }
                    }
                }
            }
        }

        __syncwarp();
        const int stage = to_read == 0 ? stages - 1 : to_read - 1;
        float *mine = (float *)stage_of(w, stage);
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                float total = e ? f2hi(sum[nt]) : f2lo(sum[nt]);
#pragma unroll
                for (int o = 4; o < 32; o *= 2) total += __shfl_xor_sync(0xffffffffu, total, o);
                const int h = 8 * nt + 2 * c + e;
                constexpr int MP = S::VP * 4 / bits_of(F);    // row tiles of a piece
#pragma unroll
                for (int m = 0; m < S::MT; m++) {
                    if (S::CODED) {
                        *(float2 *)(mine + h * D + (8 * (m / MP) + r) * (2 * MP) + 2 * (m % MP)) =
                            make_float2(O[nt][m][e], O[nt][m][2 + e]);
                    } else {
                        mine[h * D + 16 * m + r] = O[nt][m][e];
                        mine[h * D + 16 * m + 8 + r] = O[nt][m][2 + e];
                    }
                }
                if (r == 0) {
                    sums[(w * 2) * HT + h] = e ? f2hi(R[nt]) : f2lo(R[nt]);
                    sums[(w * 2 + 1) * HT + h] = total;
                }
            }
        if (l == 0) ((int *)scan)[w] = stage;
        p = q;
    }
}

// Joins the parts of piece blockIdx.x: of head blockIdx.y, a warp every eighth part, whose first are on
// their way before the weights are known; where pieces are MANY (gridDim.y < HT) of every gridDim.y-th
// head, or, if the piece has few parts, of a head a warp (256 x 8,191 tokens of 8 key heads in 4 bits, both
// kernels: 372 us with a CTA for every head of every piece, 365 so).
constexpr int kJoinWarps = 8, kJoinAhead = 6, kMostParts = 1024;
template <int D>
struct JoinLane {
    static constexpr int N = D / 32, V = N < 4 ? N : 4;      // a lane's channels, of them side by side
    la::Vec<float, V> v[N / V];
    static __device__ __forceinline__ int channel(int e, int l) { return V * (32 * (e / V) + l) + e % V; }
    __device__ __forceinline__ JoinLane(const float *p, int l) {
#pragma unroll
        for (int e = 0; e < N / V; e++) v[e] = ((const la::Vec<float, V> *)p)[32 * e + l];
    }
    __device__ __forceinline__ JoinLane() {}
    __device__ __forceinline__ void add_to(float (&o)[N], float k) const {
#pragma unroll
        for (int e = 0; e < N; e++) o[e] = fmaf(k, v[e / V].e[e % V], o[e]);
    }
};
template <int HT, int D, class T, bool MANY>
__global__ void __launch_bounds__(32 * kJoinWarps) kv_join_kernel(AttendArgs a, int ctas) {
    __shared__ float os[kJoinWarps][D], weight[kMostParts], red[2][kJoinWarps];
    const int tid = threadIdx.x, w = tid >> 5, l = tid & 31;
    griddep_wait();
    griddep_launch();
    const Joined j = ((const Joined *)(a.parts + (size_t)2 * ctas * part_floats<HT, D>()))[blockIdx.x];
    if (j.count == 0) return;
    const int chunks = (a.groups + HT - 1) / HT, g0 = j.vh % chunks * HT;
    const int nh = min(HT, a.groups - g0), h0 = j.vh / chunks * a.groups + g0;
    auto part = [&](int i) {
        return a.parts + (size_t)(i == 0 ? j.first : 2 * ((j.first >> 1) + i)) * part_floats<HT, D>();
    };
    constexpr int N = JoinLane<D>::N;
    if (MANY && j.count <= kJoinWarps) {
        for (int h = w + blockIdx.y * kJoinWarps; h < nh; h += gridDim.y * kJoinWarps) {
            JoinLane<D> parts[kJoinWarps];
#pragma unroll
            for (int i = 0; i < kJoinWarps; i++)
                if (i < j.count) parts[i] = JoinLane<D>(part(i) + h * D, l);
            const float *x = part(min(l, j.count - 1));
            const float R = l < j.count ? x[HT * D + h] : kLow;
            float top = R;
#pragma unroll
            for (int o = 1; o < kJoinWarps; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            top = __shfl_sync(0xffffffffu, top, 0);
            const float k = exp2_fast(R - top);
            float total = l < j.count ? k * x[HT * D + HT + h] : 0.f, o[N] = {};
#pragma unroll
            for (int s = 1; s < kJoinWarps; s *= 2) total += __shfl_xor_sync(0xffffffffu, total, s);
            total = __shfl_sync(0xffffffffu, total, 0);
#pragma unroll
            for (int i = 0; i < kJoinWarps; i++)
                if (i < j.count) parts[i].add_to(o, __shfl_sync(0xffffffffu, k, i));
            // a lane's channels come together through shared memory, four side by side
#pragma unroll
            for (int e = 0; e < N; e++) os[w][JoinLane<D>::channel(e, l)] = o[e];
            __syncwarp();
            for (int d = 4 * l; d < D; d += 128) {
                const float4 v = *(const float4 *)&os[w][d];
                float y[4] = {v.x, v.y, v.z, v.w};
                put_output<T>(a, j.b, h0 + h, d, top, total, y, D);
            }
            __syncwarp();
        }
        return;
    }
    for (int h = blockIdx.y; h < nh; h += MANY ? gridDim.y : HT) {
        JoinLane<D> ahead[kJoinAhead];
#pragma unroll
        for (int i = 0; i < kJoinAhead; i++)
            if (w + i * kJoinWarps < j.count) ahead[i] = JoinLane<D>(part(w + i * kJoinWarps) + h * D, l);
        float top = kLow, total = 0.f, o[N] = {};
        for (int i = tid; i < j.count; i += 32 * kJoinWarps) {
            weight[i] = part(i)[HT * D + h];
            top = fmaxf(top, weight[i]);
        }
#pragma unroll
        for (int s = 1; s < 32; s *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
        if (l == 0) red[0][w] = top;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < kJoinWarps; x++) top = fmaxf(top, red[0][x]);
        for (int i = tid; i < j.count; i += 32 * kJoinWarps) {
            weight[i] = exp2_fast(weight[i] - top);
            total = fmaf(weight[i], part(i)[HT * D + HT + h], total);
        }
#pragma unroll
        for (int s = 1; s < 32; s *= 2) total += __shfl_xor_sync(0xffffffffu, total, s);
        if (l == 0) red[1][w] = total;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kJoinAhead; i++)
            if (w + i * kJoinWarps < j.count) ahead[i].add_to(o, weight[w + i * kJoinWarps]);
#pragma unroll 4
        for (int i = w + kJoinAhead * kJoinWarps; i < j.count; i += kJoinWarps) JoinLane<D>(part(i) + h * D, l).add_to(o, weight[i]);
#pragma unroll
        for (int e = 0; e < N; e++) os[w][JoinLane<D>::channel(e, l)] = o[e];
        __syncthreads();
        for (int d = 4 * tid; d < D; d += 4 * 32 * kJoinWarps) {
            float sum = 0.f, y[4] = {};
#pragma unroll
            for (int x = 0; x < kJoinWarps; x++) {
                sum += red[1][x];
#pragma unroll
                for (int e = 0; e < 4; e++) y[e] += os[x][d + e];
            }
            put_output<T>(a, j.b, h0 + h, d, top, sum, y, D);
        }
        __syncthreads();                                     // before the next head's
    }
}

}  // namespace kv
}  // namespace stepq
