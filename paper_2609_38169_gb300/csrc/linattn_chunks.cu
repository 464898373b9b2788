// Decayed linear attention over prompts in bf16, 64 tokens at a time on the tensor cores:
// S_t = g_t S_{t-1} + k_t v_t^T, y_t = S_t^T q_t (stepq_linattn_prefill).
//
// Within a chunk of C tokens, with S_0 the state before it and products of decays
// c_t = g_1 .. g_t and w_ts = g_{s+1} .. g_t (s <= t; all <= 1, no quotient is formed, so a
// decay of zero or a product below fp32's range is simply a zero):
//   Y^T = (S_0^T Q^T) diag(c_t) + V^T P^T,   P_ts = w_ts (q_t . k_s), zero for s > t
//   S_C = c_C S_0 + U,   U^T = V^T K',   K'_s = w_Cs k_s
// Four products a chunk, all with M = 128 (lane = value channel, or token):
//   scores  Q K^T            A = Q, B = K in smem         N = 64, K = 128   (rows 64.. unused)
//   QS      S_0^T Q^T        A = S^T in tmem, B = Q       N = 64, K = 128   x 2 (head, rest of S)
//   PV      V^T P^T          A = V^T in tmem, B = P       N = 64, K = 64    x 2 (head, rest of P)
//   KV      V^T K'           A = V^T in tmem, B = K'      N = 128, K = 64   x 3
// Shared-memory bandwidth is what they and the warps compete for (128 bytes a cycle: with V
// read from there by PV and KV and the readouts passing through it, its use added up to the
// chunk's whole time, 4100 cycles), so V is transposed once into tensor memory.
// q, k and v are bf16 and enter as they are. What is fp32 enters as
// a sum of bf16: K' as three truncated terms, exactly, since states are kept in fp32; S and P
// as a head and a rest, both rounded (2^-17 of each value; the result is rounded to
// 2^-9). The state itself stays in fp32 registers and U is formed apart from it, so what is
// added from chunk to chunk is rounded to nearest (the tensor core's own sums truncate).
//
// One persistent CTA of 28 warps per SM:
//   warps 0-7    the state: S <- c_C S + U, its split into tensor memory (lane = value channel,
//                warps w and w + 4 sharing lanes 32 (w % 4) ..)
//   8 warps      V^T, and the outputs (lanes likewise)
//   3 warps      P (lanes = tokens), a 32 x 32 block each
//   1 warp       loads q, k and v (TMA, two places each); decays and their products
//   2 warps      issue the MMAs: scores and PV; KV and QS
//   6 warps      K' (8 where only the segments' parts are formed)
// Hand-over by mbarriers, every wait bounded. Loops keep few unrolled steps: unrolled, the
// warps' code did not fit the instruction caches (a third of the stalls of issuing warps).
//
// 128 prompts of 512 tokens, 16 key and 32 value heads: 445 us, 4,150 cycles a chunk and head
// (token by token 5,490 us; the bytes alone 283). Nothing is used up: issue slots 61%, shared
// memory 39%, the tensor pipe 34%, HBM 60%; what is left are the hand-overs between warps.
#include "async.cuh"
#include "device.cuh"
#include "linattn_prefill.cuh"
#include "tcgen05.cuh"

namespace stepq {
namespace la {
namespace ch {

constexpr int C = kChunk;
constexpr int kPlaces = 2;                              // of q, k, v and P
constexpr int kBlock = 28 * 32;                         // registers are shared out by warpgroups
constexpr int kOutWarps = 8, kFirst = 8 + kOutWarps;    // P, P, loads, MMAs, MMAs, P, then K'
// K': the six after those; where no outputs are formed, the first two that would form P as well (the
// pass for the parts alone of 16384 tokens: 68 us for 72).
template <bool OUT> constexpr int kScaleWarps = OUT ? 6 : 8;
constexpr int kRegs = 72, kRegsState = 112, kRegsOut = 64, kRegsOperand = 48;
static_assert(256 * (kRegsState + kRegsOut) + 384 * kRegsOperand <= kBlock * kRegs, "register shares");
constexpr uint32_t kColU = 0, kColSh = 128, kColSl = 192, kColP = 256, kColY1 = 320, kColY2 = 384, kColV = 448,
                   kCols = 512;                         // V^T: two places of 32

constexpr int kTile = C * 128;                          // 64 rows of 128 bytes: 64 channels of a chunk
constexpr int kOffK = 0, kOffQ = kOffK + kPlaces * 2 * kTile, kOffV = kOffQ + kPlaces * 2 * kTile;   // [place][2 tiles]
constexpr int kOffKp = kOffV + kPlaces * 2 * kTile;     // K': [term][2 tiles]
constexpr int kOffP = kOffKp + 3 * 2 * kTile;           // P: [place][head, rest]
// Where readouts are normalised, P has one place, to make room for them, the gate and the
// affine map: float [C][128], bf16 [C][128], float [2][128].
template <bool NORM> constexpr int kPlacesP = NORM ? 1 : kPlaces;
template <bool NORM> constexpr int kOffY = kOffP + kPlacesP<NORM> * 2 * kTile;
template <bool NORM> constexpr int kOffZ = kOffY<NORM> + (NORM ? C * kD * 4 : 0);
template <bool NORM> constexpr int kOffAffine = kOffZ<NORM> + (NORM ? C * kD * 2 : 0);
struct alignas(16) Gates {
    float next[C], c[C], wk[C];                         // g_{t+1}, c_t, w_Cs (0 past the last token)
    float suf[32], pre[32];                             // w_{31,s} of the first half, c_t / c_31 of the second
    float total, pad[3];                                // c_C
};
constexpr int kRing = 4;                                // places of decays and of items
// Cycles: waits are measured with a 32-bit clock, which has to be seen past the limit before it wraps.
constexpr long long kLongestWait = 1ll << 31;
struct alignas(16) Item {
    const float *in;                                    // the state before the segment, or null: zero
    float *out, *total;                                 // the state after it, its decays' product, or null
    int row, len, h, pad;                               // len 0: no more items
};
template <bool NORM> constexpr int kOffG = kOffAffine<NORM> + (NORM ? 2 * kD * 4 : 0);
template <bool NORM> constexpr int kOffItem = kOffG<NORM> + kRing * (int)sizeof(Gates);
template <bool NORM> constexpr int kOffBar = kOffItem<NORM> + kRing * (int)sizeof(Item);
enum {
    kFullK, kFullQ = kFullK + kPlaces, kFullV = kFullQ + kPlaces, kFreeK = kFullV + kPlaces, kFreeQ = kFreeK + kPlaces,
    kFreeV = kFreeQ + kPlaces, kVtReady = kFreeV + kPlaces, kVtFree = kVtReady + kPlaces, kPReady = kVtFree + kPlaces,
    kKpReady = kPReady + kPlaces, kKpFree = kKpReady + 2,
    kFullG = kKpFree + 2, kFreeG = kFullG + kRing, kFullItem = kFreeG + kRing,
    kFreeItem = kFullItem + kRing, kScores = kFreeItem + kRing, kSReady, kUFree, kYFree, kQs, kKv, kPv, kDrainA, kDrainB, kBars
};
template <bool NORM> constexpr int kOffTmem = kOffBar<NORM> + kBars * 8;
template <bool NORM> constexpr int kOffStop = kOffTmem<NORM> + 8;      // uint32 [2] of each group of warps
template <bool NORM> constexpr int kSmem = kOffStop<NORM> + 40;
static_assert(kSmem<true> <= kSmemMax && kSmem<false> <= kSmemMax, "one CTA's shared memory");

constexpr uint32_t kIdescScores = tc::idesc_bf16(128, 64, 0, 0);
constexpr uint32_t kIdescQs = tc::idesc_bf16(128, 64, 0, 0);
constexpr uint32_t kIdescPv = tc::idesc_bf16(128, 64, 0, 0);
constexpr uint32_t kIdescKv = tc::idesc_bf16(128, 128, 0, 1);

template <bool NORM>
struct Ctx {
    const PrefillArgs &a;
    uint8_t *smem;
    uint64_t *bars;
    mutable uint32_t limit;                                 // of a wait, in cycles; 0: one has run out
    static constexpr int R = kRing;
    // Waits for the phase of the given parity. Once a wait has run out no other of this warp
    // holds: the warps reach their ends without early exits, and the outputs are undefined.
    __device__ __forceinline__ void wait(int bar, uint32_t parity) const {
        const uint32_t t0 = (uint32_t)clock();
        while (!mbar_test(&bars[bar], parity))
            if ((uint32_t)clock() - t0 > limit) {
                limit = 0;
                break;
            }
        __syncwarp();
    }
    // Use n of a ring of N places: filled; given back after use n - N.
    template <int N> __device__ __forceinline__ void wait_full(int bar, uint32_t n) const { wait(bar + n % N, (n / N) & 1u); }
    template <int N> __device__ __forceinline__ void wait_free(int bar, uint32_t n) const {
        wait(bar + n % N, ((n / N) & 1u) ^ 1u);             // before a barrier's first phase its parity is 1
    }
    // Use n of a single place: the one before has ended.
    __device__ __forceinline__ void wait_last(int bar, uint32_t n) const {
        wait(bar, (n & 1u) ^ 1u);
    }
    // One arrival for the warp, after what its lanes did.
    __device__ __forceinline__ void arrive(int bar) const {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&bars[bar]);
    }
    __device__ __forceinline__ Gates &gates(uint32_t n) const { return ((Gates *)(smem + kOffG<NORM>))[n % R]; }
    __device__ __forceinline__ volatile uint32_t *stopped() const { return (volatile uint32_t *)(smem + kOffStop<NORM>); }
    __device__ __forceinline__ Item &item(uint32_t n) const { return ((Item *)(smem + kOffItem<NORM>))[n % R]; }
};

// Barriers of the groups of warps. Within a group one warp waits for the phases and the
// others for it: a waiting warp tests every 140 cycles or so, and 28 of them took half of
// the SM's issue slots.
enum { kSyncNone, kSyncState, kSyncOut, kSyncKeys, kSyncScores };
template <int ID, int WARPS>
__device__ __forceinline__ void group_sync() {
    asm volatile("barrier.cta.sync %0, %1;" ::"n"(ID), "n"(32 * WARPS) : "memory");
}

// A warp's walk over the items that the loads' warp hands out. The warps of a group walk it
// in step: they end where their first one (`leader`) ends, after which none of them is left
// at one of the group's barriers.
template <bool NORM, int ID = kSyncNone, int WARPS = 1>
struct Items {
    const Ctx<NORM> &x;
    bool leader;
    uint32_t n = 0;
    const float *in;
    float *out, *total;
    int row, len, h;
    __device__ __forceinline__ explicit Items(const Ctx<NORM> &c, bool first = true) : x(c), leader(first) {}
    __device__ __forceinline__ bool next() {
        if (leader) x.template wait_full<kRing>(kFullItem, n);
        bool stop = x.limit == 0;                           // a wait ran out: nothing more
        if (WARPS > 1) {
            // Two words in turn: the leader may come to the next item before another warp has read this
            // one's, but not to the one after that, since they meet in between.
            volatile uint32_t *word = x.stopped() + 2 * ID + n % 2;
            if (leader) *word = stop;
            group_sync<ID, WARPS>();
            stop = *word;
        }
        const Item &i = x.item(n);
        in = i.in;
        out = i.out;
        total = i.total;
        row = i.row;
        len = stop ? 0 : i.len;
        h = i.h;
        x.arrive(kFreeItem + n++ % kRing);
        return len > 0;
    }
};

// The pieces of a pair of fp32 values: both truncated to bf16 (the first in the low half),
// what remains of them (exact), and both rounded to bf16.
__device__ __forceinline__ uint32_t heads(uint64_t p) {
    return __byte_perm((uint32_t)p, (uint32_t)(p >> 32), 0x7632);
}
__device__ __forceinline__ uint64_t rests(uint64_t p) {
    return fsub2(p, u2pair((uint32_t)p & 0xFFFF0000u, (uint32_t)(p >> 32) & 0xFFFF0000u));
}
__device__ __forceinline__ uint32_t rounded(uint64_t p) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(f2hi(p)), "f"(f2lo(p)));
    return d;
}
// A pair's heads rounded to nearest and, rounded too, what remains of them: 2^-17 of each value is lost,
// twice as much after truncated heads. A head does not round to infinity: finite values keep a rest.
__device__ __forceinline__ void head_rest(uint64_t p, uint32_t &h, uint32_t &r) {
    asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(f2hi(p)), "f"(f2lo(p)));
    r = rounded(fsub2(p, u2pair(h << 16, h & 0xFFFF0000u)));
}
__device__ __forceinline__ uint64_t pair_at(const float *p) {           // 8-byte aligned
    return *(const uint64_t *)p;
}

// The decays of every chunk and their products, a block of 32 tokens per half, and
// k, q and v.
template <bool OUT, bool NORM>
__device__ __forceinline__ void load(const Ctx<NORM> &x, const ChunkMaps &maps) {
    const PrefillArgs &a = x.a;
    const int grp = a.Hv / a.Hk, l = threadIdx.x & 31;
    const uint32_t lead = tc::elect();
    uint32_t n = 0, started = 0;                            // chunks; copies, three a chunk
    const int segments = OUT ? a.plan->segments : a.plan->parts;
    int i = 0;                                              // segment * Hv + head
    Segment it;
    // The longest segment and head left.
    const auto take = [&]() {
        if (lead) i = atomicAdd(&a.plan->next[OUT], 1);
        i = __reduce_max_sync(0xffffffffu, i);
        it.len = 0;
        if (i / a.Hv < segments) it = a.table[i / a.Hv];
    };
    take();
    for (uint32_t k = 0;; k++) {
        x.template wait_free<kRing>(kFreeItem, k);
        const int h = i % a.Hv, row = it.row, len = it.len;
        if (lead) {
            Item &o = x.item(k);
            float *work = a.states + ((uint64_t)it.id * a.Hv + h) * kN, *page = pool_page(a, it.slot, h);
            o.row = row;
            o.len = len;
            o.h = h;
            o.in = !OUT || it.in == kStateZero ? nullptr : it.in == kStatePool ? page : work;
            o.out = !OUT ? work + (uint64_t)a.Hv * kN : it.out == kStatePool ? page : nullptr;
            o.total = OUT ? nullptr : a.totals + (uint64_t)it.id * a.Hv + h;
        }
        x.arrive(kFullItem + k % kRing);
        if (len == 0 || x.limit == 0) break;
        if (i == a.stall.withhold_item) {                   // test switch: these copies never start
            x.limit = 0;
            break;
        }
        const int hk = h / grp;
        const float *gate = a.gate + (int64_t)row * a.gs + h;
        const auto decay = [&](int t) { return t < len ? gate[(int64_t)t * a.gs] : 1.f; };
        float g0 = decay(l), g1 = decay(32 + l);
#pragma unroll 1
        for (int t0 = 0; t0 < len; t0 += C, n++) {
            const int m = len - t0;
            float p0 = g0, p1 = g1;                         // inclusive from the block's start
            float n0 = __shfl_down_sync(0xffffffffu, g0, 1), n1 = __shfl_down_sync(0xffffffffu, g1, 1);
            if (l == 31) n0 = n1 = 1.f;
            float s0 = n0, s1 = n1;                         // exclusive to the block's end
            g0 = decay(t0 + C + l);                         // the next chunk's
            g1 = decay(t0 + C + 32 + l);
#pragma unroll 1
            for (int o = 1; o < 32; o *= 2) {
                const float u0 = __shfl_up_sync(0xffffffffu, p0, o), u1 = __shfl_up_sync(0xffffffffu, p1, o);
                const float d0 = __shfl_down_sync(0xffffffffu, s0, o), d1 = __shfl_down_sync(0xffffffffu, s1, o);
                if (l >= o) p0 *= u0, p1 *= u1;
                if (l + o < 32) s0 *= d0, s1 *= d1;
            }
            const float all0 = __shfl_sync(0xffffffffu, p0, 31), all1 = __shfl_sync(0xffffffffu, p1, 31);
            x.template wait_free<x.R>(kFreeG, n);
            Gates &o = x.gates(n);
            o.next[l] = n0;
            o.next[32 + l] = n1;
            o.c[l] = p0;
            o.c[32 + l] = all0 * p1;
            o.wk[l] = l < m ? s0 * all1 : 0.f;
            o.wk[32 + l] = l + 32 < m ? s1 : 0.f;
            o.suf[l] = s0;
            o.pre[l] = p1;
            if (l == 0) o.total = all0 * all1;
            x.arrive(kFullG + n % x.R);
#pragma unroll 1
            for (int e = 0; e < 3; e++) {                   // k, q, v
                if (!OUT && e == 1) {
                    started++;
                    continue;
                }
                x.template wait_free<kPlaces>(kFreeK + e * kPlaces, n);
                if (x.limit == 0) goto drain;               // nothing more is started
                started++;
                uint64_t *full = &x.bars[kFullK + e * kPlaces + n % kPlaces];
                uint8_t *dst = x.smem + (e * kPlaces + n % kPlaces) * 2 * kTile;
                const int ch = (e == 2 ? h : hk) * kD;
                if (lead) {
                    mbar_arrive_tx(full, 2 * kTile);
                    tma_load_2d(dst, &maps.of[e], ch, row + t0, full);
                    tma_load_2d(dst + kTile, &maps.of[e], ch + 64, row + t0, full);
                }
                __syncwarp();
            }
            if (t0 == 0) take();                            // the next one, known long before it is due
        }
    }
drain:                                                      // no copy is in flight when the CTA ends
#pragma unroll 1
    for (uint32_t u = started < 3 * kPlaces ? 0 : started - 3 * kPlaces; u < started; u++)
        if (OUT || u % 3 != 1) mbar_wait(&x.bars[kFullK + (u % 3) * kPlaces + u / 3 % kPlaces], (u / 3 / kPlaces) & 1u, x.a.stall.wait_cycles);
}

// Descriptor of the two tiles of chunk n in one of the loaded operands' places.
template <bool NORM>
__device__ __forceinline__ uint64_t operand(const Ctx<NORM> &x, int off, uint32_t n, uint32_t lbo) {
    return tc::sdesc_sw128(x.smem + off + (n % kPlaces) * 2 * kTile, lbo, 1024);
}

// Scores and PV. The scores of a chunk are formed ahead of the PV of the one before.
template <bool NORM>
__device__ __forceinline__ void issue_scores(const Ctx<NORM> &x, uint32_t tm) {
    const uint32_t lead = tc::elect();
    Items<NORM> it(x);
    int left = 0;                                           // tokens of the item
    bool more = true;
#pragma unroll 1
    for (uint32_t n = 0; more; n++) {
        const uint32_t m = n - 1;
        left -= C;
        if (left <= 0) {
            more = it.next();
            left = it.len;
        }
        if (n > 0) x.template wait_full<kPlaces>(kPReady, m);       // the scores of chunk m have been read
        if (more) {
            x.template wait_full<kPlaces>(kFullK, n);
            x.template wait_full<kPlaces>(kFullQ, n);
            tc::fence_after();
            const uint64_t q = operand(x, kOffQ, n, 16), k = operand(x, kOffK, n, 16);
#pragma unroll 1
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int s = 0; s < 4; s++)
                    tc::mma_f16_ss(lead, tm + kColP, q + i * (kTile / 16) + s * 2, k + i * (kTile / 16) + s * 2, kIdescScores,
                                   i > 0 || s > 0);
            tc::commit(lead, &x.bars[kScores]);
            tc::commit(lead, &x.bars[kFreeK + n % kPlaces]);
            tc::commit(lead, &x.bars[kFreeQ + n % kPlaces]);
        }
        if (n == 0) continue;
        x.template wait_full<kPlaces>(kVtReady, m);
        x.wait_last(kYFree, m);
        tc::fence_after();
        const uint64_t p = operand(x, kOffP, kPlacesP<NORM> > 1 ? m : 0, 16);
#pragma unroll 1
        for (int i = 1; i >= 0; i--)                        // rest, head
#pragma unroll
            for (int s = 0; s < 4; s++)
                tc::mma_f16_ts(lead, tm + kColY2, tm + kColV + 32 * (m % kPlaces) + 8 * s, p + i * (kTile / 16) + s * 2, kIdescPv,
                               i < 1 || s > 0);
        tc::commit(lead, &x.bars[kPv]);
        tc::commit(lead, &x.bars[kVtFree + m % kPlaces]);
    }
    // every MMA has ended before the tensor memory is given back
    tc::commit(lead, &x.bars[kDrainA]);
    if (!mbar_wait(&x.bars[kDrainA], 0, x.a.stall.wait_cycles)) x.limit = 0;
}

// KV and QS.
template <bool OUT, bool NORM>
__device__ __forceinline__ void issue_state(const Ctx<NORM> &x, uint32_t tm) {
    const uint32_t lead = tc::elect();
    const uint64_t kp = tc::sdesc_sw128(x.smem + kOffKp, kTile, 1024);
    Items<NORM> it(x);
    int left = 0;
#pragma unroll 1
    for (uint32_t n = 0;; n++) {
        left -= C;
        if (left <= 0) {
            if (!it.next()) break;
            left = it.len;
        }
        x.template wait_full<kPlaces>(kVtReady, n);
        x.wait_last(kUFree, n);
#pragma unroll 1
        for (uint32_t h = 0; h < 2; h++) {                // the chunk's halves, so that one is scaled under the other
            x.wait(kKpReady + h, n & 1u);
            tc::fence_after();
#pragma unroll 1
            for (int i = 2; i >= 0; i--)                  // the smallest terms first
#pragma unroll
                for (int s = 0; s < 2; s++)
                    tc::mma_f16_ts(lead, tm + kColU, tm + kColV + 32 * (n % kPlaces) + 8 * (2 * h + s),
                                   kp + i * (2 * kTile / 16) + (2 * h + s) * 128, kIdescKv, h > 0 || i < 2 || s > 0);
            tc::commit(lead, &x.bars[kKpFree + h]);
        }
        tc::commit(lead, &x.bars[kKv]);
        tc::commit(lead, &x.bars[kVtFree + n % kPlaces]);
        if (!OUT) continue;
        x.template wait_full<kPlaces>(kFullQ, n);
        x.wait_last(kYFree, n);
        x.wait(kSReady, n & 1u);
        tc::fence_after();
        const uint64_t q = operand(x, kOffQ, n, 16);
#pragma unroll 1
        for (int i = 0; i < 4; i++)                       // rest, head; each its two halves of K
#pragma unroll
            for (int s = 0; s < 4; s++)
                tc::mma_f16_ts(lead, tm + kColY1, tm + (i < 2 ? kColSl : kColSh) + 32 * (i & 1) + 8 * s,
                               q + (i & 1) * (kTile / 16) + s * 2, kIdescQs, i > 0 || s > 0);
        tc::commit(lead, &x.bars[kQs]);
        tc::commit(lead, &x.bars[kFreeQ + n % kPlaces]);
    }
    tc::commit(lead, &x.bars[kDrainB]);
    if (!mbar_wait(&x.bars[kDrainB], 0, x.a.stall.wait_cycles)) x.limit = 0;
}

// K' = w_Cs k_s as three truncated bf16 terms. A unit is a 16-byte piece of 32 tokens (lane =
// token) of a tile, so that 8 lanes' pieces of the swizzled rows lie in different banks. In a
// chunk with fewer tokens the rows past the last belong to other sequences: zeros take
// their place.
template <bool OUT, bool NORM>
__device__ __forceinline__ void scale(const Ctx<NORM> &x, int w) {
    constexpr int W = kScaleWarps<OUT>;
    const PrefillArgs &a = x.a;
    const int l = threadIdx.x & 31;
    uint32_t n = 0;
    for (Items<NORM, kSyncKeys, W> it(x, w == 0); it.next();) {
#pragma unroll 1
        for (int t0 = 0; t0 < it.len; t0 += C, n++) {
            const int m = it.len - t0, place = (n % kPlaces) * 2 * kTile;
            if (w == 0) {
                x.template wait_full<x.R>(kFullG, n);
                x.template wait_full<kPlaces>(kFullK, n);
            }
            const Gates &g = x.gates(n);
#pragma unroll 1
            for (int h = 0; h < 2; h++) {
                if (w == 0) x.wait_last(kKpFree + h, n);
                group_sync<kSyncKeys, W>();
                const int s = 32 * h + l;
                const uint64_t f = f2s(g.wk[s]);
#pragma unroll 1
                for (int u = (w + 4 * h) % W; u < 16; u += W) {
                    uint8_t *at = x.smem + (u >> 3) * kTile + s * 128 + ((u & 7) ^ (l & 7)) * 16;
                    uint4 r = *(const uint4 *)(at + kOffK + place);
                    if (s >= m) r = make_uint4(0, 0, 0, 0);
                    const uint32_t in[4] = {r.x, r.y, r.z, r.w};
                    uint32_t t[3][4];
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        uint64_t p = fmul2(u2pair(in[e] << 16, in[e] & 0xFFFF0000u), f);
                        t[0][e] = heads(p);
                        p = rests(p);
                        t[1][e] = heads(p);
                        t[2][e] = heads(rests(p));
                    }
#pragma unroll
                    for (int i = 0; i < 3; i++)
                        *(uint4 *)(at + kOffKp + i * 2 * kTile) = make_uint4(t[i][0], t[i][1], t[i][2], t[i][3]);
                }
                fence_async_smem();
                x.arrive(kKpReady + h);
            }
            x.arrive(kFreeK + n % kPlaces);
            x.arrive(kFreeG + n % x.R);
        }
    }
}

// V^T of chunk n, m tokens, into tensor memory: 16 channels (half h) of this warp's
// quadrant. Rows past the last token belong to other sequences: zeros take their place.
template <bool NORM>
__device__ __forceinline__ void transpose_v(const Ctx<NORM> &x, uint32_t tm, uint32_t n, int m, int h) {
    const int l = threadIdx.x & 31, quad = (threadIdx.x >> 5) & 3;
    // ldmatrix: this lane's row of the four 8 x 8 matrices (tokens 0-7 | 8-15) x (channels 0-7 | 8-15)
    const int row = (l & 7) + 8 * (l >> 4), piece = 4 * (quad & 1) + ((l >> 3) & 1);
    x.template wait_full<kPlaces>(kFullV, n);
    x.template wait_free<kPlaces>(kVtFree, n);
    tc::fence_after();
    const uint8_t *v = x.smem + kOffV + (n % kPlaces) * 2 * kTile + (quad >> 1) * kTile + row * 128;
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 4; i++)                             // 16 tokens
        tc::load_transposed(v + i * 16 * 128 + ((piece + 2 * h) ^ (l & 7)) * 16, r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
    if (m < C)
#pragma unroll
        for (int i = 0; i < 16; i++) {                      // tokens 2 (l & 3) and + 1 of the 8 at 8 (i >> 1)
            const int t = 8 * (i >> 1) + 2 * (l & 3);
            r[i] = t + 1 < m ? r[i] : t < m ? r[i] & 0xFFFFu : 0u;
        }
    tc::st_16x32(tm + ((uint32_t)(32 * quad + 16 * h) << 16) + kColV + 32 * (n % kPlaces), r);
    tc::wait_st();
    tc::fence_before();
    x.arrive(kVtReady + n % kPlaces);
    x.arrive(kFreeV + n % kPlaces);
}

// P of tokens t = 32 quad + lane over keys 32 half .. + 31, 16 keys at a time;
// the block above the diagonal stays zero. Diagonal blocks: w_ts by a running product down
// the row (zero above the diagonal); the block below them: the product of its two parts.
template <bool NORM>
__device__ __forceinline__ void weigh_scores(const Ctx<NORM> &x, uint32_t tm, int quad, int half) {
    const int l = threadIdx.x & 31, t = 32 * quad + l;
    const uint32_t tl = tm + ((uint32_t)(32 * quad) << 16) + kColP;
    uint32_t n = 0;
    for (Items<NORM, kSyncScores, 3> it(x, quad == 0); it.next();) {
#pragma unroll 1
        for (int t0 = 0; t0 < it.len; t0 += C, n++) {
            if (quad == 0) {
                x.template wait_full<x.R>(kFullG, n);
                if (kPlacesP<NORM> > 1) x.template wait_free<kPlaces>(kVtFree, n);     // PV has read the place
                else x.wait_last(kPv, n);
                x.wait(kScores, n & 1u);
            }
            group_sync<kSyncScores, 3>();
            tc::fence_after();
            const Gates &g = x.gates(n);
            uint8_t *row = x.smem + kOffP + (n % kPlacesP<NORM>) * 2 * kTile + t * 128;
            const uint64_t pre = f2s(g.pre[l]);
            const int m = it.len - t0;                      // keys past the last: other sequences' rows
            float w = 0.f;
#pragma unroll 1
            for (int b = 2 * half + 1; b >= 2 * half; b--) { // keys 16 b .. + 15
                uint32_t u[16];
                tc::ld16(tl + 16 * b, u);
                uint64_t f[8];                              // the weights
                if (half < quad) {
#pragma unroll
                    for (int i = 0; i < 8; i++) f[i] = fmul2(pair_at(&g.suf[16 * b + 2 * i]), pre);
                } else {
                    const int d = t - 16 * b;
                    const float4 *nx = (const float4 *)&g.next[16 * b];
#pragma unroll
                    for (int i = 7; i >= 0; i -= 2) {
                        const float4 v = nx[i >> 1];
                        const float w3 = d == 2 * i + 1 ? 1.f : w * v.w, w2 = d == 2 * i ? 1.f : w3 * v.z;
                        const float w1 = d == 2 * i - 1 ? 1.f : w2 * v.y;
                        w = d == 2 * i - 2 ? 1.f : w1 * v.x;
                        f[i] = f2(w2, w3);
                        f[i - 1] = f2(w, w1);
                    }
                }
                if (m < 16 * b + 16)
#pragma unroll
                    for (int i = 0; i < 16; i++) u[i] = 16 * b + i < m ? u[i] : 0u;
                uint32_t h[8], r[8];
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    head_rest(fmul2(u2pair(u[2 * i], u[2 * i + 1]), f[i]), h[i], r[i]);
                }
                const int o0 = ((2 * b) ^ (t & 7)) * 16, o1 = ((2 * b + 1) ^ (t & 7)) * 16;
                *(uint4 *)(row + o0) = make_uint4(h[0], h[1], h[2], h[3]);
                *(uint4 *)(row + o1) = make_uint4(h[4], h[5], h[6], h[7]);
                *(uint4 *)(row + kTile + o0) = make_uint4(r[0], r[1], r[2], r[3]);
                *(uint4 *)(row + kTile + o1) = make_uint4(r[4], r[5], r[6], r[7]);
            }
            tc::fence_before();
            fence_async_smem();
            x.arrive(kPReady + n % kPlaces);
            x.arrive(kFreeG + n % x.R);
        }
    }
}

// The state. This thread: value channel j, key channels 64 half .. + 63, in pairs.
template <bool OUT, bool NORM>
__device__ __forceinline__ void states(const Ctx<NORM> &x, uint32_t tm) {
    const PrefillArgs &a = x.a;
    const int w = threadIdx.x >> 5, l = threadIdx.x & 31, quad = w & 3, half = w >> 2, j = 32 * quad + l;
    const uint32_t tl = tm + ((uint32_t)(32 * quad) << 16);
    uint32_t n = 0;
    uint64_t s[32];
    for (Items<NORM, kSyncState, 8> it(x, w == 0); it.next();) {
        const float *in = it.in;
#pragma unroll
        for (int e = 0; e < 32; e++)
            s[e] = in ? f2(in[(64 * half + 2 * e) * kD + j], in[(64 * half + 2 * e + 1) * kD + j]) : 0;
        float total = 1.f;                                  // the segment's decay
#pragma unroll 1
        for (int t0 = 0; t0 < it.len; t0 += C, n++) {
            if (OUT) {                                      // S^T's head and rest as an operand
                if (w == 0) x.wait_last(kQs, n);
                group_sync<kSyncState, 8>();
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    uint32_t h[8], r[8];
#pragma unroll
                    for (int e = 0; e < 8; e++) head_rest(s[8 * i + e], h[e], r[e]);
                    tc::st8(tl + kColSh + 32 * half + 8 * i, h);
                    tc::st8(tl + kColSl + 32 * half + 8 * i, r);
                }
                tc::wait_st();
                tc::fence_before();
                x.arrive(kSReady);
            }
            if (w == 0) {
                x.template wait_full<x.R>(kFullG, n);
                x.wait(kKv, n & 1u);
            }
            group_sync<kSyncState, 8>();
            tc::fence_after();
            const float gc = x.gates(n).total;
            const uint64_t g2 = f2s(gc);
            total *= gc;
#pragma unroll
            for (int i = 0; i < 2; i++) {
                uint64_t u[16];
                tc::ld32_pairs(tl + kColU + 64 * half + 32 * i, u);
#pragma unroll
                for (int e = 0; e < 16; e++) s[16 * i + e] = ffma2(g2, s[16 * i + e], u[e]);
            }
            tc::fence_before();
            x.arrive(kUFree);
            x.arrive(kFreeG + n % x.R);
        }
        float *out = it.out;
        if (out)
#pragma unroll
            for (int e = 0; e < 32; e++) {
                out[(64 * half + 2 * e) * kD + j] = f2lo(s[e]);
                out[(64 * half + 2 * e + 1) * kD + j] = f2hi(s[e]);
            }
        if (!OUT && threadIdx.x == 0) *it.total = total;
    }
}

// u act(z) or act(u) for a pair of channels (stepq_norm), u = y A + B, by selects alone: branches
// cost a normalised prompt a tenth of its time.
struct GateForm {
    bool gated, none, sigmoid;
    __device__ __forceinline__ explicit GateForm(const NormArgs &n)
        : gated(n.z), none(n.act == STEPQ_ACT_NONE), sigmoid(n.act == STEPQ_ACT_SIGMOID) {}
    __device__ __forceinline__ uint64_t operator()(uint64_t y, uint64_t A, uint64_t B, uint64_t z) const {
        const uint64_t one = f2s(1.f), u = ffma2(y, A, B), t = gated ? z : u, x = fmul2(t, f2s(kToExponent));
        const uint64_t r = f2(fast_sigmoid(f2lo(x)), fast_sigmoid(f2hi(x)));
        return fmul2(fmul2(sigmoid ? one : t, none ? one : r), gated ? u : one);
    }
};

// Normalises the chunk's readouts ys [C][128], its first m tokens, into y. Eight lanes a token,
// lane k of them channels 32 i + 4 k .. + 3: with 32 lanes a token the sums' five steps took as
// long as the rest. Means and centred sums of squares of ever larger parts: see norm_head.
__device__ __forceinline__ void norm_chunk(const PrefillArgs &a, const float *ys, const bf16 *zs, const float *affine, bf16 *y,
                                           int m, int w, int l) {
    const int k = l & 7;
    const GateForm gate(a.norm);
#pragma unroll 1
    for (int t = 4 * w + (l >> 3); t < C; t += 32) {
        uint64_t v[8];
        float mean = 0.f;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float4 u = *(const float4 *)&ys[t * kD + 32 * i + 4 * k];
            v[2 * i] = f2(u.x, u.y);
            v[2 * i + 1] = f2(u.z, u.w);
            mean += (u.x + u.y) + (u.z + u.w);
        }
        mean *= 1.f / 16;
        uint64_t q2 = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint64_t d = fsub2(v[i], f2s(mean));
            q2 = ffma2(d, d, q2);
        }
        float q = f2lo(q2) + f2hi(q2);
#pragma unroll
        for (int o = 1; o < 8; o *= 2) {
            const float m2 = __shfl_xor_sync(0xffffffffu, mean, o), d = mean - m2;
            q += __shfl_xor_sync(0xffffffffu, q, o);
            q = fmaf(d * (8.f * o), d, q);
            mean = 0.5f * (mean + m2);
        }
        const float c = a.norm.center ? mean : 0.f, r = rstd_of(fmaf(mean - c, mean, q * (1.f / kD)), a.norm.eps);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int ch = 32 * i + 4 * k;
            const ulonglong2 w4 = *(const ulonglong2 *)&affine[ch], b4 = *(const ulonglong2 *)&affine[kD + ch];
            uint2 z = *(const uint2 *)&zs[t * kD + ch];
            if (!a.norm.z) z = make_uint2(0, 0);
            const uint64_t o0 = gate(fsub2(v[2 * i], f2s(c)), fmul2(w4.x, f2s(r)), b4.x, u2pair(z.x << 16, z.x & 0xFFFF0000u));
            const uint64_t o1 = gate(fsub2(v[2 * i + 1], f2s(c)), fmul2(w4.y, f2s(r)), b4.y, u2pair(z.y << 16, z.y & 0xFFFF0000u));
            if (t < m) *(uint2 *)(y + t * a.ys + ch) = make_uint2(rounded(o0), rounded(o1));
        }
    }
}

// V^T of the next chunk, and the outputs. This thread: value channel j of tokens 32 half .. + 31,
// a warp's 64 bytes of a token straight from registers (16-byte pieces by way of stmatrix and
// shared memory: a tenth fewer instructions, but 5% slower for the shared memory they take);
// or, to be normalised, through shared memory, where a token's 128 channels come together.
template <bool OUT, bool NORM>
__device__ __forceinline__ void outputs(const Ctx<NORM> &x, uint32_t tm) {
    constexpr int W = kOutWarps;
    const PrefillArgs &a = x.a;
    const int w = (threadIdx.x >> 5) - 8, l = threadIdx.x & 31, quad = w & 3, half = w >> 2, j = 32 * quad + l;
    const uint32_t tl = tm + ((uint32_t)(32 * quad) << 16) + 32 * half;
    float *ys = (float *)(x.smem + kOffY<NORM>), *affine = (float *)(x.smem + kOffAffine<NORM>);
    bf16 *zs = (bf16 *)(x.smem + kOffZ<NORM>);
    uint32_t n = 0;
    // V^T runs a chunk ahead, into the next item's first: that item is known by then
    Items<NORM, kSyncOut, W> ahead(x, w == 0);
    bool more = ahead.next();
    int next = ahead.len;                                   // tokens of its item from chunk v on
    uint32_t v = 0;
    while (more) {
        const int row = ahead.row, len = ahead.len, h = ahead.h;
        bf16 *y = (bf16 *)a.y + (int64_t)row * a.ys + h * kD;
        const bf16 *z = (const bf16 *)a.norm.z + (int64_t)row * a.norm.z_stride + h * kD;
        if (NORM) {                                         // (no warp reads the last item's any more)
            const int c = threadIdx.x & (kD - 1), pc = c + (a.norm.shared ? 0 : h * kD);
            if (threadIdx.x & kD) affine[c] = a.norm.w ? a.norm.w[pc] : 1.f;
            else affine[kD + c] = a.norm.b ? a.norm.b[pc] : 0.f;
        }
#pragma unroll 1
        for (int t0 = 0; t0 < len; t0 += C, n++) {
#pragma unroll 1
            for (; v <= n + 1; v++, next -= C) {
                if (next <= 0) {
                    more = ahead.next();
                    next = ahead.len;
                    if (!more) break;
                }
                transpose_v(x, tm, v, next, half);
            }
            if (!OUT) continue;
            const int m = min(C, len - t0);
            if (NORM && a.norm.z)                           // the gate, on its way before it is needed
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int t = 2 * w + (l >> 4) + 16 * i;
                    cp_async16_or_zero(zs + t * kD + 8 * (l & 15), z + min(t, m - 1) * a.norm.z_stride + 8 * (l & 15), t < m);
                }
            if (w == 0) {
                x.template wait_full<x.R>(kFullG, n);
                x.wait(kPv, n & 1u);
                x.wait(kQs, n & 1u);
            }
            group_sync<kSyncOut, W>();
            tc::fence_after();
            const float *c = x.gates(n).c + 32 * half;
            bf16 *yt = y + 32 * half * a.ys + j;
#pragma unroll 1
            for (int i = 0; i < 32; i += 16) {
                uint32_t y1[16], y2[16];
                tc::ld16_two(tl + kColY1 + i, y1, tl + kColY2 + i, y2);
                if (i == 16) {
                    tc::fence_before();
                    x.arrive(kYFree);
                }
                float *p = ys + (32 * half + i) * kD + j;
                const int left = m - 32 * half - i;
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const uint64_t u = ffma2(pair_at(&c[i + e]), u2pair(y1[e], y1[e + 1]), u2pair(y2[e], y2[e + 1]));
                    if (NORM) {
                        p[e * kD] = f2lo(u);
                        p[(e + 1) * kD] = f2hi(u);
                    } else {
                        const uint32_t b = rounded(u);
                        if (e < left) *(uint16_t *)yt = (uint16_t)b;
                        yt += a.ys;
                        if (e + 1 < left) *(uint16_t *)yt = (uint16_t)(b >> 16);
                        yt += a.ys;
                    }
                }
            }
            x.arrive(kFreeG + n % x.R);
            if (NORM) {
                cp_async_wait_all();
                group_sync<kSyncOut, W>();
                norm_chunk(a, ys, zs, affine, y, m, w, l);
                group_sync<kSyncOut, W>();                  // the readouts' and the gate's places are free again
                z += C * a.norm.z_stride;
            }
            y += C * a.ys;
        }
    }
}

template <bool OUT, bool NORM>
__global__ void __launch_bounds__(kBlock, 1) linattn_chunks_kernel(PrefillArgs a, const __grid_constant__ ChunkMaps maps) {
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t *bars = (uint64_t *)(smem + kOffBar<NORM>);
    uint32_t *tbase = (uint32_t *)(smem + kOffTmem<NORM>);
    const int tid = threadIdx.x, w = __shfl_sync(0xffffffffu, tid >> 5, 0);
    if (w == 0) {
        tc::tmem_alloc(tbase, kCols);
        tc::tmem_relinquish();
    }
    if (tid < kBars) {
        int count = 1;                                      // TMA, the end of MMAs, the decays, items
        if (tid >= kFreeK && tid < kFreeQ) count = kScaleWarps<OUT> + (OUT ? 1 : 0);            // K', the scores
        if (tid >= kFreeQ && tid < kFreeV) count = OUT ? 2 : 1;                            // scores, QS
        if (tid >= kFreeV && tid < kVtFree) count = kOutWarps;                             // V^T (and kVtReady)
        if (tid >= kVtFree && tid < kPReady) count = OUT ? 2 : 1;                          // KV, PV
        if (tid >= kPReady && tid < kKpReady) count = 3;
        if (tid >= kKpReady && tid < kKpFree) count = kScaleWarps<OUT>;
        if (tid >= kFreeG && tid < kFullItem) count = 8 + kScaleWarps<OUT> + (OUT ? 3 + kOutWarps : 0);     // state, K', P, outputs
        if (tid >= kFreeItem && tid < kScores) count = 9 + kScaleWarps<OUT> + kOutWarps + (OUT ? 4 : 0);    // and the MMAs
        if (tid >= kSReady && tid < kYFree) count = 8;
        if (tid == kYFree) count = kOutWarps;
        mbar_init(&bars[tid], count);
        mbar_init_fence();
    }
    if (OUT && w >= 8 && w < 10) {                          // P's block above the diagonal stays zero
        for (int i = tid - 256; i < kPlacesP<NORM> * 2 * 32 * 4; i += 64) {
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
    const Ctx<NORM> x{a, smem, bars, (uint32_t)min(a.stall.wait_cycles, kLongestWait)};
    if (w < 8) {
        tc::regs_inc<kRegsState>();
        states<OUT>(x, tm);
    } else if (w < kFirst) {
        tc::regs_dec<kRegsOut>();
        outputs<OUT>(x, tm);
    } else {
        tc::regs_dec<kRegsOperand>();
        const int i = w - kFirst;
        if (i == 2) load<OUT>(x, maps);
        else if (i == 4) issue_state<OUT>(x, tm);
        else if (i >= 6) scale<OUT>(x, i - 6);
        else if (!OUT && i < 2) scale<OUT>(x, i + 6);
        else if (OUT) {
            if (i == 3) issue_scores(x, tm);
            else weigh_scores(x, tm, w & 3, i == 1);
        }
    }
    if (x.limit == 0) raise_error(a.err, STEPQ_ERR_TIMEOUT);
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

// The shared memory a launch takes, and the registers that its warps share out.
template <bool OUT, bool NORM>
static stepq_status prepare() {
    const auto kernel = (const void *)linattn_chunks_kernel<OUT, NORM>;
    static SmemOptIn opt;
    const stepq_status st = opt(kernel, kSmem<NORM>);
    if (st != STEPQ_OK) return st;
    static std::atomic<int> regs{0};                    // kept once known
    if (regs.load(std::memory_order_relaxed) == 0) {
        cudaFuncAttributes f{};
        const stepq_status e = cuda_status(cudaFuncGetAttributes(&f, kernel));
        if (e != STEPQ_OK) return e;
        regs.store(f.numRegs, std::memory_order_relaxed);
    }
    return regs.load(std::memory_order_relaxed) < kRegs ? STEPQ_ERR_CUDA : STEPQ_OK;
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

stepq_status prepare_linattn_chunks(const PrefillArgs &a, bool parts, ChunkMaps &maps) {
    const ch::Encode f = ch::encoder();
    if (!f || !ch::encode(f, &maps.of[0], a.k, kD * a.Hk, a.tokens, a.ks) ||
        !ch::encode(f, &maps.of[1], a.q, kD * a.Hk, a.tokens, a.qs) || !ch::encode(f, &maps.of[2], a.v, kD * a.Hv, a.tokens, a.vs))
        return STEPQ_ERR_CUDA;
    const stepq_status st = parts ? ch::prepare<false, false>() : STEPQ_OK;
    if (st != STEPQ_OK) return st;
    return a.norm.on ? ch::prepare<true, true>() : ch::prepare<true, false>();
}

stepq_status launch_linattn_chunks(const PrefillArgs &a, const ChunkMaps &maps, int grid, bool out, cudaStream_t s) {
    using namespace ch;
    if (!out) return launch_overlapped(linattn_chunks_kernel<false, false>, grid, kBlock, kSmem<false>, s, a, maps);
    if (a.norm.on) return launch_overlapped(linattn_chunks_kernel<true, true>, grid, kBlock, kSmem<true>, s, a, maps);
    return launch_overlapped(linattn_chunks_kernel<true, false>, grid, kBlock, kSmem<false>, s, a, maps);
}

}  // namespace la
}  // namespace stepq
