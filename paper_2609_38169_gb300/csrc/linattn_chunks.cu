// Decayed linear attention over prompts in bf16, 64 tokens at a time on the tensor cores:
// S_t = g_t S_{t-1} + k_t v_t^T, y_t = S_t^T q_t (stepq_linattn_prefill).
//
// Within a chunk of C tokens, with S_0 the state before it and products of decays
// c_t = g_1 .. g_t and w_ts = g_{s+1} .. g_t (s <= t; all <= 1, no quotient is formed, so a
// decay of zero or a product below fp32's range is simply a zero):
//   Y^T = (S_0^T Q^T) diag(c_t) + V^T P^T,   P_ts = w_ts (q_t . k_s), zero for s > t
//   S_C = c_C S_0 + U,   U^T = V^T K',   K'_s = w_Cs k_s
// Four products a chunk, all with M = 128 (lane = value channel, or token):
//   scores  Q K^T            A = Q, B = K in smem        N = 64, K = 128   (rows 64.. unused)
//   QS      S_0^T Q^T        A = S^T in tmem, B = Q      N = 64, K = 128   x 2 (head, rest)
//   PV      V^T P^T          A = V^T, B = P in smem      N = 64, K = 64    x 2 (head, rest)
//   KV      V^T K'           A = V^T, B = K' in smem     N = 128, K = 64   x 3
// q, k and v are bf16 and enter as they are, from where TMA put them. What is fp32 enters as
// a sum of bf16: K' as three truncated terms, exactly; S and P as a truncated head and a
// rounded rest (2^-17 of each value; the result is rounded to 2^-9). The state itself stays
// in fp32 registers of the chain's warps and U is formed apart from it, so what is added from
// chunk to chunk is rounded to nearest (the tensor core's own sums truncate).
//
// One persistent CTA of 19 warps per SM:
//   warps 0-7    the chain: S <- c_C S + U, its split into tensor memory, and Y (lane = value
//                channel j, warps w and w + 4 sharing lanes 32 (w % 4) ..)
//   warps 8-15   quadrants 0, 1 (lanes = tokens): P; quadrants 2, 3: K'
//   warp 16      issues the MMAs
//   warp 17      loads q, k and v (TMA, two places each)
//   warp 18      decays: their products over the chunk
// Hand-over by mbarriers, every wait bounded.
#include <cuda.h>

#include "async.cuh"
#include "device.cuh"
#include "linattn_prefill.cuh"
#include "tcgen05.cuh"

namespace stepq {
namespace la {
namespace ch {

constexpr int C = kChunk;
constexpr int kPlaces = 2;                              // of q, k and v
constexpr int kGateRing = 4;
constexpr int kBlock = 19 * 32 + 32;                    // registers are shared out by warpgroups
constexpr int kRegs = 96, kRegsChain = 136, kRegsOperand = 80, kRegsIssue = 48;
static_assert(256 * (kRegsChain + kRegsOperand) + 128 * kRegsIssue <= kBlock * kRegs, "register shares");
constexpr uint32_t kColU = 0, kColSh = 128, kColSl = 192, kColP = 256, kColY1 = 320, kColY2 = 384, kCols = 512;

constexpr int kTile = C * 128;                          // 64 rows of 128 bytes: 64 channels of a chunk
constexpr int kOffQ = 0;                                // [place][2 tiles]
constexpr int kOffK = kOffQ + kPlaces * 2 * kTile;
constexpr int kOffV = kOffK + kPlaces * 2 * kTile;
constexpr int kOffKp = kOffV + kPlaces * 2 * kTile;     // K': 3 terms x 2 tiles
constexpr int kOffP = kOffKp + 3 * 2 * kTile;           // P: head, rest
constexpr int kOffY = kOffP + 2 * kTile;                // float [C][kYRow] readouts to normalise
constexpr int kYRow = 132;
struct Gates {
    float g[C], c[C], wk[C];                            // decays, c_t, w_Cs (0 past the last token)
    float suf[32], pre[32];                             // w_{31,s} of the first half, c_t / c_31 of the second
    float total, pad[3];                                // c_C
};
constexpr int kOffG = kOffY + C * kYRow * 4;
constexpr int kOffBar = kOffG + kGateRing * (int)sizeof(Gates);
enum {
    kFullQ, kFullK = kFullQ + kPlaces, kFullV = kFullK + kPlaces, kFreeQ = kFullV + kPlaces, kFreeK = kFreeQ + kPlaces,
    kFreeV = kFreeK + kPlaces, kFullG = kFreeV + kPlaces, kFreeG = kFullG + kGateRing, kScores = kFreeG + kGateRing,
    kScoresFree, kPReady, kKpReady, kSReady, kUFree, kYFree, kQs, kKv, kPv, kDrain, kBars
};
constexpr int kOffTmem = kOffBar + kBars * 8;
constexpr int kSmem = kOffTmem + 16;
static_assert(kSmem <= kSmemMax, "one CTA's shared memory");
static_assert(kOffBar % 8 == 0 && kOffG % 16 == 0, "alignment");

constexpr uint32_t kIdescScores = tc::idesc_bf16(128, 64, 0, 0);
constexpr uint32_t kIdescQs = tc::idesc_bf16(128, 64, 0, 0);
constexpr uint32_t kIdescPv = tc::idesc_bf16(128, 64, 1, 0);
constexpr uint32_t kIdescKv = tc::idesc_bf16(128, 128, 1, 1);

struct Maps {
    CUtensorMap q, k, v;
};

struct Ctx {
    const PrefillArgs &a;
    uint8_t *smem;
    uint64_t *bars;
    // warp-uniform: true once the phase of the given parity has completed
    __device__ __forceinline__ bool wait(int bar, uint32_t parity) const {
        return __all_sync(0xffffffffu, mbar_wait(&bars[bar], parity, a.stall.wait_cycles));
    }
    // The phase of use n of a ring of R places; `again`: that it was given back before.
    template <int R> __device__ __forceinline__ bool wait_full(int bar, uint32_t n) const {
        return wait(bar + n % R, (n / R) & 1u);
    }
    template <int R> __device__ __forceinline__ bool wait_free(int bar, uint32_t n) const {
        return n < R || wait(bar + n % R, (n / R - 1) & 1u);
    }
    // One arrival for the warp, after what its lanes did.
    __device__ __forceinline__ void arrive(int bar) const {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&bars[bar]);
    }
    __device__ __forceinline__ const Gates &gates(uint32_t n) const {
        return ((const Gates *)(smem + kOffG))[n % kGateRing];
    }
};

__device__ __forceinline__ uint32_t high_halves(float a, float b) {      // truncated to bf16, a low
    return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
}
__device__ __forceinline__ float head_of(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t rounded_halves(float a, float b) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    return d;
}
// Two fp32 values as a truncated bf16 head and a rounded rest each.
__device__ __forceinline__ void split2(float a, float b, uint32_t &head, uint32_t &rest) {
    head = high_halves(a, b);
    rest = rounded_halves(a - head_of(a), b - head_of(b));
}

// Warp 18: the decays of every chunk and their products, a block of 32 tokens per half.
__device__ __forceinline__ bool decays(const Ctx &x) {
    const PrefillArgs &a = x.a;
    const int l = threadIdx.x & 31;
    uint32_t n = 0;
    for (Items it(a); it.next();) {
        for (int t0 = 0; t0 < it.len; t0 += C, n++) {
            const int m = it.len - t0;                      // tokens from here on
            const float *g = a.gate + ((int64_t)it.row + t0) * a.gs + it.h;
            const float g0 = l < m ? g[(int64_t)l * a.gs] : 1.f, g1 = l + 32 < m ? g[(int64_t)(l + 32) * a.gs] : 1.f;
            float p0 = g0, p1 = g1;                         // inclusive from the block's start
            float s0 = __shfl_down_sync(0xffffffffu, g0, 1), s1 = __shfl_down_sync(0xffffffffu, g1, 1);
            if (l == 31) s0 = s1 = 1.f;                     // exclusive to the block's end
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const float u0 = __shfl_up_sync(0xffffffffu, p0, o), u1 = __shfl_up_sync(0xffffffffu, p1, o);
                const float d0 = __shfl_down_sync(0xffffffffu, s0, o), d1 = __shfl_down_sync(0xffffffffu, s1, o);
                if (l >= o) p0 *= u0, p1 *= u1;
                if (l + o < 32) s0 *= d0, s1 *= d1;
            }
            const float all0 = __shfl_sync(0xffffffffu, p0, 31), all1 = __shfl_sync(0xffffffffu, p1, 31);
            if (!x.wait_free<kGateRing>(kFreeG, n)) return false;
            Gates &o = ((Gates *)(x.smem + kOffG))[n % kGateRing];
            o.g[l] = g0;
            o.g[32 + l] = g1;
            o.c[l] = p0;
            o.c[32 + l] = all0 * p1;
            o.wk[l] = l < m ? s0 * all1 : 0.f;
            o.wk[32 + l] = l + 32 < m ? s1 : 0.f;
            o.suf[l] = s0;
            o.pre[l] = p1;
            if (l == 0) o.total = all0 * all1;
            x.arrive(kFullG + n % kGateRing);
        }
    }
    return true;
}

// Warp 17: q, k and v of every chunk.
template <bool OUT>
__device__ __forceinline__ bool load(const Ctx &x, const Maps &maps) {
    const PrefillArgs &a = x.a;
    const int grp = a.Hv / a.Hk;
    const uint32_t lead = tc::elect();
    uint32_t count[3] = {0, 0, 0};                          // chunks of k, q and v started
    bool ok = true;
    const auto fetch = [&](int which, const CUtensorMap *map, int full, int free, int off, int ch, int row) {
        const uint32_t n = count[which];
        if (!x.wait_free<kPlaces>(free, n)) return false;
        uint8_t *dst = x.smem + off + (n % kPlaces) * 2 * kTile;
        if (lead) {
            mbar_arrive_tx(&x.bars[full + n % kPlaces], 2 * kTile);
            tma_load_2d(dst, map, ch, row, &x.bars[full + n % kPlaces]);
            tma_load_2d(dst + kTile, map, ch + 64, row, &x.bars[full + n % kPlaces]);
        }
        __syncwarp();
        count[which]++;
        return true;
    };
    for (Items it(a); ok && it.next();) {
        const int hk = it.h / grp;
        if (it.item == a.stall.withhold_item) ok = false;   // test switch: these copies never start
        for (int t0 = 0; ok && t0 < it.len; t0 += C) {
            const int row = it.row + t0;
            ok = fetch(0, &maps.k, kFullK, kFreeK, kOffK, hk * kD, row) &&
                 (!OUT || fetch(1, &maps.q, kFullQ, kFreeQ, kOffQ, hk * kD, row)) &&
                 fetch(2, &maps.v, kFullV, kFreeV, kOffV, it.h * kD, row);
        }
    }
    // no copy is in flight when the CTA ends
    const int full[3] = {kFullK, kFullQ, kFullV};
#pragma unroll
    for (int i = 0; i < 3; i++)
        for (uint32_t m = count[i] < kPlaces ? 0 : count[i] - kPlaces; m < count[i]; m++)
            ok = x.wait_full<kPlaces>(full[i], m) && ok;
    return ok;
}

// Warp 16: the MMAs.
template <bool OUT>
__device__ __forceinline__ bool issue(const Ctx &x, uint32_t tm) {
    const uint32_t lead = tc::elect();
    uint32_t chunks = 0;
    for (Items it(x.a); it.next();) chunks += (uint32_t)(it.len + C - 1) / C;
    const auto at = [&](int off, uint32_t n) { return x.smem + off + (n % kPlaces) * 2 * kTile; };
    const auto scores = [&](uint32_t n) {
        if (!x.wait_full<kPlaces>(kFullQ, n) || !x.wait_full<kPlaces>(kFullK, n) || (n > 0 && !x.wait(kScoresFree, (n - 1) & 1u)))
            return false;
        tc::fence_after();
        const uint64_t q = tc::sdesc_sw128(at(kOffQ, n), 16, 1024), k = tc::sdesc_sw128(at(kOffK, n), 16, 1024);
#pragma unroll
        for (int s = 0; s < 8; s++) {
            const uint64_t step = (s >> 2) * (kTile / 16) + (s & 3) * 2;
            tc::mma_f16_ss(lead, tm + kColP, q + step, k + step, kIdescScores, s > 0);
        }
        tc::commit(lead, &x.bars[kScores]);
        tc::commit(lead, &x.bars[kFreeK + n % kPlaces]);
        return true;
    };
    const uint64_t kp = tc::sdesc_sw128(x.smem + kOffKp, kTile, 1024), p = tc::sdesc_sw128(x.smem + kOffP, 16, 1024);
    bool ok = true;
    if (OUT && chunks > 0) ok = scores(0);
    for (uint32_t n = 0; ok && n < chunks; n++) {
        const uint32_t ph = n & 1u;
        if (!(ok = x.wait(kKpReady, ph) && x.wait_full<kPlaces>(kFullV, n) && (n == 0 || x.wait(kUFree, ph ^ 1u)))) break;
        tc::fence_after();
        const uint64_t v = tc::sdesc_sw128(at(kOffV, n), kTile, 1024);
#pragma unroll
        for (int s = 0; s < 12; s++)                      // the smallest terms first
            tc::mma_f16_ss(lead, tm + kColU, v + (s & 3) * 128, kp + (2 - s / 4) * (2 * kTile / 16) + (s & 3) * 128, kIdescKv,
                           s > 0);
        tc::commit(lead, &x.bars[kKv]);
        if (!OUT) {
            tc::commit(lead, &x.bars[kFreeV + n % kPlaces]);
            continue;
        }
        if (!(ok = x.wait(kSReady, ph) && (n == 0 || x.wait(kYFree, ph ^ 1u)))) break;
        tc::fence_after();
        const uint64_t q = tc::sdesc_sw128(at(kOffQ, n), 16, 1024);
#pragma unroll
        for (int s = 0; s < 16; s++) {
            const int e = s & 7;
            tc::mma_f16_ts(lead, tm + kColY1, tm + (s < 8 ? kColSl : kColSh) + 8 * e, q + (e >> 2) * (kTile / 16) + (e & 3) * 2,
                           kIdescQs, s > 0);
        }
        tc::commit(lead, &x.bars[kQs]);
        tc::commit(lead, &x.bars[kFreeQ + n % kPlaces]);
        if (n + 1 < chunks && !(ok = scores(n + 1))) break;
        if (!(ok = x.wait(kPReady, ph))) break;
        tc::fence_after();
#pragma unroll
        for (int s = 0; s < 8; s++)
            tc::mma_f16_ss(lead, tm + kColY2, v + (s & 3) * 128, p + (s < 4 ? kTile / 16 : 0) + (s & 3) * 2, kIdescPv, s > 0);
        tc::commit(lead, &x.bars[kPv]);
        tc::commit(lead, &x.bars[kFreeV + n % kPlaces]);
    }
    // every MMA has ended before the tensor memory is given back
    tc::commit(lead, &x.bars[kDrain]);
    return x.wait(kDrain, 0) && ok;
}

// Warps 8-15, quadrants 2 and 3: K' = w_Cs k_s as three truncated bf16 terms. A warp takes
// 32 tokens (lane = token) of one tile of 64 channels, so that 8 lanes' 16-byte pieces of a
// swizzled tile lie in different banks. In a chunk with fewer tokens the rows past the last
// belong to other sequences: zeros take their place here and in V.
template <bool OUT>
__device__ __forceinline__ bool scale_keys(const Ctx &x, int w) {
    const PrefillArgs &a = x.a;
    const int l = threadIdx.x & 31, s = 32 * (w & 1) + l, tile = w >> 1;       // w 0..3
    uint32_t n = 0;
    for (Items it(a); it.next();) {
        for (int t0 = 0; t0 < it.len; t0 += C, n++) {
            const int m = it.len - t0;
            if (!x.wait_full<kGateRing>(kFullG, n) || !x.wait_full<kPlaces>(kFullK, n)) return false;
            const float f = x.gates(n).wk[s];
            if (n > 0 && !x.wait(kKv, (n - 1) & 1u)) return false;
            const uint8_t *k = x.smem + kOffK + ((n % kPlaces) * 2 + tile) * kTile + s * 128;
            uint8_t *kp = x.smem + kOffKp + tile * kTile + s * 128;
            const bool valid = s < m;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int o = (i ^ (s & 7)) * 16;
                const uint4 r = *(const uint4 *)(k + o);
                const uint32_t in[4] = {r.x, r.y, r.z, r.w};
                uint32_t t[3][4];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    float lo = valid ? __uint_as_float(in[e] << 16) * f : 0.f;
                    float hi = valid ? __uint_as_float(in[e] & 0xFFFF0000u) * f : 0.f;
                    t[0][e] = high_halves(lo, hi);
                    lo -= head_of(lo);
                    hi -= head_of(hi);
                    t[1][e] = high_halves(lo, hi);
                    lo -= head_of(lo);
                    hi -= head_of(hi);
                    t[2][e] = high_halves(lo, hi);
                }
#pragma unroll
                for (int u = 0; u < 3; u++) *(uint4 *)(kp + u * 2 * kTile + o) = make_uint4(t[u][0], t[u][1], t[u][2], t[u][3]);
            }
            if (m < C) {
                if (!x.wait_full<kPlaces>(kFullV, n)) return false;
                if (!valid)
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        *(uint4 *)(x.smem + kOffV + ((n % kPlaces) * 2 + tile) * kTile + s * 128 + i * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_async_smem();
            x.arrive(kKpReady);
            x.arrive(kFreeK + n % kPlaces);
        }
    }
    return true;
}

// Warps 8-15, quadrants 0 and 1: P of tokens t = 32 quad + lane over keys 32 half .. + 31, for
// the three of the four blocks that are not all zero. Diagonal blocks: w_ts by a running
// product down the row; the block below them: the product of its two parts.
__device__ __forceinline__ bool weigh_scores(const Ctx &x, uint32_t tm, int quad, int half) {
    const int l = threadIdx.x & 31, t = 32 * quad + l;
    const uint32_t tl = tm + ((uint32_t)(32 * quad) << 16) + kColP + 32 * half;
    uint8_t *row = x.smem + kOffP + t * 128;
    uint32_t n = 0;
    for (Items it(x.a); it.next();) {
        for (int t0 = 0; t0 < it.len; t0 += C, n++) {
            const uint32_t ph = n & 1u;
            if (!x.wait_full<kGateRing>(kFullG, n)) return false;
            const Gates &g = x.gates(n);
            const float pre = g.pre[l];
            if (!x.wait(kScores, ph)) return false;
            tc::fence_after();
            float p[32], w = 0.f;
            {
                float u[16];
                tc::ld16(tl, u);
#pragma unroll
                for (int e = 0; e < 16; e++) p[e] = u[e];
                tc::ld16(tl + 16, u);
#pragma unroll
                for (int e = 0; e < 16; e++) p[16 + e] = u[e];
            }
            tc::fence_before();
            x.arrive(kScoresFree);
            if (quad != half) {
#pragma unroll
                for (int e = 0; e < 32; e++) p[e] *= g.suf[e] * pre;
            } else {
#pragma unroll
                for (int e = 31; e >= 0; e--) {
                    w = l == e ? 1.f : w * g.g[32 * half + (e + 1 & 31)];
                    p[e] = l >= e ? p[e] * w : 0.f;
                }
            }
            if (n > 0 && !x.wait(kPv, ph ^ 1u)) return false;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                uint32_t h[4], r[4];
#pragma unroll
                for (int e = 0; e < 4; e++) split2(p[8 * i + 2 * e], p[8 * i + 2 * e + 1], h[e], r[e]);
                const int o = ((4 * half + i) ^ (t & 7)) * 16;
                *(uint4 *)(row + o) = make_uint4(h[0], h[1], h[2], h[3]);
                *(uint4 *)(row + kTile + o) = make_uint4(r[0], r[1], r[2], r[3]);
            }
            fence_async_smem();
            x.arrive(kPReady);
        }
    }
    return true;
}

// Barrier over the 256 threads of warps 0-7; returns the OR of their predicates.
__device__ __forceinline__ bool chain_any(bool p) {
    uint32_t r;
    asm volatile(
        "{ .reg .pred p, q; setp.ne.u32 p, %1, 0; barrier.cta.red.or.pred q, 1, 256, p; selp.u32 %0, 1, 0, q; }"
        : "=r"(r)
        : "r"((uint32_t)p)
        : "memory");
    return r != 0;
}

// Warps 0-7: the state and the outputs. This thread: value channel j, key channels
// 64 half .. + 63 of the state, tokens 32 half .. + 31 of the outputs.
template <bool OUT, bool NORM>
__device__ __forceinline__ bool chain(const Ctx &x, uint32_t tm) {
    const PrefillArgs &a = x.a;
    const int w = threadIdx.x >> 5, l = threadIdx.x & 31, quad = w & 3, half = w >> 2, j = 32 * quad + l;
    const uint32_t tl = tm + ((uint32_t)(32 * quad) << 16);
    float *ys = (float *)(x.smem + kOffY);
    uint32_t n = 0;
    float s[64];
    const auto publish = [&]() {                            // S^T's head and rest as an operand
#pragma unroll
        for (int i = 0; i < 4; i++) {
            uint32_t h[8], r[8];
#pragma unroll
            for (int e = 0; e < 8; e++) split2(s[16 * i + 2 * e], s[16 * i + 2 * e + 1], h[e], r[e]);
            tc::st8(tl + kColSh + 32 * half + 8 * i, h);
            tc::st8(tl + kColSl + 32 * half + 8 * i, r);
        }
        tc::wait_st();
        tc::fence_before();
        x.arrive(kSReady);
    };
    // A wait ran out: the other warps meet this one at the chunk's next barrier.
    const auto give_up = [&]() {
        if (NORM) chain_any(true);
        return false;
    };
    for (Items it(a); it.next();) {
        const float *in = it.state_in();
#pragma unroll
        for (int e = 0; e < 64; e++) s[e] = in ? in[(64 * half + e) * kD + j] : 0.f;
        if (OUT) publish();
        float total = 1.f;                                  // the segment's decay
        for (int t0 = 0; t0 < it.len; t0 += C, n++) {
            const uint32_t ph = n & 1u;
            const bool last = t0 + C >= it.len;
            if (!x.wait_full<kGateRing>(kFullG, n) || !x.wait(kKv, ph)) return give_up();
            tc::fence_after();
            const Gates &g = x.gates(n);
            const float gc = g.total;
            total *= gc;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                float u[16];
                tc::ld16(tl + kColU + 64 * half + 16 * i, u);
#pragma unroll
                for (int e = 0; e < 16; e++) s[16 * i + e] = fmaf(gc, s[16 * i + e], u[e]);
            }
            tc::fence_before();
            x.arrive(kUFree);
            if (!OUT) {
                x.arrive(kFreeG + n % kGateRing);
                continue;
            }
            if (!x.wait(kQs, ph)) return give_up();
            tc::fence_after();
            if (!last) publish();
            if (!x.wait(kPv, ph)) return give_up();
            tc::fence_after();
            const int64_t row = (int64_t)it.row + t0;
            const int m = min(C, it.len - t0);
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int c0 = 32 * half + 16 * i;
                float y1[16], y2[16];
                tc::ld16(tl + kColY1 + c0, y1);
                tc::ld16(tl + kColY2 + c0, y2);
                bf16 *y = (bf16 *)a.y + (row + c0) * a.ys + it.h * kD + j;
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const float r = fmaf(g.c[c0 + e], y1[e], y2[e]);
                    if (NORM) ys[(c0 + e) * kYRow + j] = r;
                    else if (c0 + e < m) y[e * a.ys] = __float2bfloat16_rn(r);
                }
            }
            tc::fence_before();
            x.arrive(kYFree);
            x.arrive(kFreeG + n % kGateRing);
            if (NORM) {
                if (chain_any(false)) return false;
                for (int t = w; t < m; t += 8) {
                    const float4 r = *(const float4 *)&ys[t * kYRow + 4 * l];
                    float y[4] = {r.x, r.y, r.z, r.w};
                    norm_head<bf16, 4>(a.norm, it.h, row + t, l, y);
                    store_vec<bf16, 4>((bf16 *)a.y + (row + t) * a.ys + it.h * kD + 4 * l, y);
                }
                chain_any(false);
            }
        }
        float *out = it.state_out();
        if (out)
#pragma unroll
            for (int e = 0; e < 64; e++) out[(64 * half + e) * kD + j] = s[e];
        if (!OUT && threadIdx.x == 0) *it.total_out() = total;
    }
    return true;
}

template <bool OUT, bool NORM>
__global__ void __launch_bounds__(kBlock, 1) linattn_chunks_kernel(PrefillArgs a, const __grid_constant__ Maps maps) {
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t *bars = (uint64_t *)(smem + kOffBar);
    uint32_t *tbase = (uint32_t *)(smem + kOffTmem);
    const int tid = threadIdx.x, w = __shfl_sync(0xffffffffu, tid >> 5, 0);
    if (w == 0) {
        tc::tmem_alloc(tbase, kCols);
        tc::tmem_relinquish();
    }
    if (tid == 0) {
        for (int i = 0; i < kPlaces; i++) {
            mbar_init(&bars[kFullQ + i], 1);
            mbar_init(&bars[kFullK + i], 1);
            mbar_init(&bars[kFullV + i], 1);
            mbar_init(&bars[kFreeQ + i], 1);
            mbar_init(&bars[kFreeK + i], OUT ? 5 : 4);      // the scores, four warps of K'
            mbar_init(&bars[kFreeV + i], 1);
        }
        for (int i = 0; i < kGateRing; i++) {
            mbar_init(&bars[kFullG + i], 1);
            mbar_init(&bars[kFreeG + i], 8);
        }
        mbar_init(&bars[kScores], 1);
        mbar_init(&bars[kScoresFree], 3);
        mbar_init(&bars[kPReady], 3);
        mbar_init(&bars[kKpReady], 4);
        mbar_init(&bars[kSReady], 8);
        mbar_init(&bars[kUFree], 8);
        mbar_init(&bars[kYFree], 8);
        mbar_init(&bars[kQs], 1);
        mbar_init(&bars[kKv], 1);
        mbar_init(&bars[kPv], 1);
        mbar_init(&bars[kDrain], 1);
        mbar_init_fence();
    }
    if (OUT && w >= 8 && w < 10) {                          // P's block above the diagonal stays zero
        for (int i = tid - 256; i < 2 * 32 * 4; i += 64) {
            const int t = (i >> 2) & 31, o = ((4 + (i & 3)) ^ (t & 7)) * 16;
            *(uint4 *)(smem + kOffP + (i >> 7) * kTile + t * 128 + o) = make_uint4(0, 0, 0, 0);
        }
        fence_async_smem();
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    griddep_wait();
    griddep_launch();
    const uint32_t tm = *tbase;
    const Ctx x{a, smem, bars};
    bool ok = true;
    if (w < 8) {
        tc::regs_inc<kRegsChain>();
        ok = chain<OUT, NORM>(x, tm);
    } else if (w < 16) {
        tc::regs_dec<kRegsOperand>();
        const int quad = w & 3, half = (w - 8) >> 2;
        if (quad >= 2) ok = scale_keys<OUT>(x, 2 * half + quad - 2);
        else if (OUT && quad >= half) ok = weigh_scores(x, tm, quad, half);
    } else {
        tc::regs_dec<kRegsIssue>();
        if (w == 16) ok = issue<OUT>(x, tm);
        else if (w == 17) ok = load<OUT>(x, maps);
        else if (w == 18) ok = decays(x);
    }
    if (!ok) raise_error(a.err, STEPQ_ERR_TIMEOUT);
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    if (w == 0) {
        tc::fence_after();
        tc::tmem_dealloc(tm, kCols);
    }
}

// The encoder of tensor maps, from the driver.
using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                            const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static Encode encoder() {
    static std::atomic<void *> fn{nullptr};
    void *p = fn.load(std::memory_order_acquire);
    if (!p) {
        cudaDriverEntryPointQueryResult found;
        if (cuda_status(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found)) !=
                STEPQ_OK ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        fn.store(p, std::memory_order_release);
    }
    return (Encode)p;
}
// [rows][channels] bf16, a box of 64 channels x 64 rows; rows past the last read as zero.
static bool encode(Encode f, CUtensorMap *map, const void *p, int channels, int rows, int64_t stride) {
    const cuuint64_t dims[2] = {(cuuint64_t)channels, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {64, C}, one[2] = {1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (void *)p, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool OUT, bool NORM>
static stepq_status launch(const PrefillArgs &a, const Maps &maps, int items, cudaStream_t s) {
    const auto kernel = linattn_chunks_kernel<OUT, NORM>;
    static SmemOptIn opt;
    const stepq_status st = opt((const void *)kernel, kSmem);
    if (st != STEPQ_OK) return st;
    // the register shares are taken from what the kernel is launched with
    static std::atomic<int> regs{0};
    if (regs.load(std::memory_order_relaxed) == 0) {
        cudaFuncAttributes f{};
        const stepq_status e = cuda_status(cudaFuncGetAttributes(&f, (const void *)kernel));
        if (e != STEPQ_OK) return e;
        regs.store(f.numRegs, std::memory_order_relaxed);
    }
    if (regs.load(std::memory_order_relaxed) < kRegs) return STEPQ_ERR_CUDA;
    const int grid = sm_count();
    return launch_overlapped(kernel, grid < items ? grid : items, kBlock, kSmem, s, a, maps);
}

}  // namespace ch

// The rows of q, k and v as TMA takes them: a row per token that holds at least the heads'
// channels.
bool linattn_chunks_takes(const stepq_config *cfg, const stepq_linattn_io *io) {
    const int64_t hk = (int64_t)kD * cfg->n_key_heads, hv = (int64_t)kD * cfg->n_value_heads;
    constexpr int64_t most = (1ll << 39);
    return io->dtype == STEPQ_BF16 && io->q_stride >= hk && io->k_stride >= hk && io->v_stride >= hv &&
           io->q_stride < most && io->k_stride < most && io->v_stride < most;
}

stepq_status launch_linattn_chunks(const PrefillArgs &a, int items, bool out, cudaStream_t s) {
    const ch::Encode f = ch::encoder();
    ch::Maps maps;
    if (!f || !ch::encode(f, &maps.q, a.q, kD * a.Hk, a.tokens, a.qs) || !ch::encode(f, &maps.k, a.k, kD * a.Hk, a.tokens, a.ks) ||
        !ch::encode(f, &maps.v, a.v, kD * a.Hv, a.tokens, a.vs))
        return STEPQ_ERR_CUDA;
    if (!out) return ch::launch<false, false>(a, maps, items, s);
    return a.norm.on ? ch::launch<true, true>(a, maps, items, s) : ch::launch<true, false>(a, maps, items, s);
}

}  // namespace la
}  // namespace stepq
