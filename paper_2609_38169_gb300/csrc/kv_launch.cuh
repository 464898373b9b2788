// Choice of a variant of the attention kernels, and their launch.
#pragma once

#include "kv_attend.cuh"

namespace stepq {
namespace kv {

// Runs f(Shape{}) for the variant of a call; more than 8 query heads a key head go in sixteens, but for
// 256 channels of codes, whose sixteens have little room (64 x 4,096 tokens of two key heads with 16 query heads
// each, us: in 4 bits 73, in eights 64; 8 bits and fp32 vectors 215 and 95; 2 x 900 tokens 21 and 10. Long calls in
// 8 bits with 16-bit vectors lose by it, 80 and 86).
template <int F, class Fn>
auto by_shape(int head_dim, int groups, int dtype, Fn &&f) {
    auto types = [&](auto d, auto nt) {
        constexpr int D = decltype(d)::value, NT = decltype(nt)::value;
        return dtype == STEPQ_F32    ? f(Shape<F, D, NT, float>{})
               : dtype == STEPQ_BF16 ? f(Shape<F, D, NT, la::bf16>{})
                                     : f(Shape<F, D, NT, la::f16>{});
    };
    auto heads = [&](auto d) {
        if constexpr (!coded(F) || decltype(d)::value < 256)
            if (groups > 8) return types(d, std::integral_constant<int, 2>{});
        return types(d, std::integral_constant<int, 1>{});
    };
    return head_dim == 64    ? heads(std::integral_constant<int, 64>{})
           : head_dim == 128 ? heads(std::integral_constant<int, 128>{})
                             : heads(std::integral_constant<int, 256>{});
}
template <class S> using Half = Shape<S::F, S::D, 1, typename S::T>;

// CTAs of a call, from what the host knows: its rows and the most tokens that one has. cluster > 0:
// clusters of that many take whole sequences. A warp then has up to S::WHOLE tiles, however short
// the others' sequences are; beyond that equal shares are worth the parts and the second kernel.
// A window makes all longer sequences equal, and twice as many tiles worth it: 33 sequences of 1,000
// tokens' window, 10 heads of 64 (8 tiles a warp and more) 15.5 us, in shares 20.8. Without one, 7 of 14,000 in
// 8 bits (14 tiles a warp) take 16.5 us, in shares 14.3.
struct Grid { int ctas, cluster, stages; };
template <class S>
Grid grid_of(const stepq_kv_config *c, int groups, int64_t rows, int64_t most, bool equal) {
    const int64_t tiles = (most + S::TT - 1) / S::TT, sms = sm_count();
    const int64_t heads = rows * c->n_heads * ((groups + S::HT - 1) / S::HT);
    const int64_t places = sms * S::resident(S::STAGES), resident = places < kMostParts ? places : kMostParts;
    // A cluster lies within one part of the chip, where the places behind the last whole one are lost: of 152, 304
    // and 456 places, clusters of 4 find 144, 296 and 440, of 8 find 120, 288 and 408.
    auto lost = [](int c) { return c < 4 ? 0 : c < 8 ? 16 : 48; };
    int cluster = 1;                                         // as many as find places and two tiles a warp
    while (cluster < 8 && 2 * cluster * heads <= resident - lost(2 * cluster) && tiles > 2 * kAttWarps * cluster) cluster *= 2;
    const bool whole = tiles <= (equal ? 2 : 1) * S::WHOLE * kAttWarps * cluster && (heads <= resident || tiles <= 2 * kAttWarps);
    Grid g{0, whole ? cluster : 0, S::STAGES};
    if (whole && tiles <= kAttWarps * cluster && heads * cluster <= sms * S::resident(1) - lost(cluster)) {
        // a tile a warp needs one stage, which lets more CTAs in
        g.ctas = (int)heads * cluster;
        g.stages = 1;
    } else if (whole) {
        // more sequences than places: a CTA takes several, and has the next one's tiles copied meanwhile
        g.ctas = (int)(heads < resident ? heads : resident) * cluster;
    } else {
        const int64_t ctas = (heads * tiles + 2 * kAttWarps - 1) / (2 * kAttWarps);
        g.ctas = (int)(ctas < resident ? ctas : resident);
    }
    return g;
}
template <class S>
size_t parts_bytes(const Grid &g) {
    if (g.cluster) return 0;
    return (size_t)g.ctas * (2 * sizeof(float) * part_floats<S::HT, S::D>() + sizeof(Joined));
}

template <int F>
size_t attend_workspace(const stepq_kv_config *c, int groups, int64_t rows, int64_t most) {
    size_t need = 0;
    auto add = [&](auto sh) {
        using S = decltype(sh);
        const size_t n = parts_bytes<S>(grid_of<S>(c, groups, rows, most, false));
        if (n > need) need = n;
    };
    for (int dtype = STEPQ_F32; dtype <= STEPQ_F16; dtype++)
        by_shape<F>(c->head_dim, groups, dtype, [&](auto sh) {
            using S = decltype(sh);
            add(sh);
            add(typename S::Larger{});
            if constexpr (S::NT > 1) {
                add(Half<S>{});
                add(typename Half<S>::Larger{});
            }
            return 0;
        });
    return need;
}

template <class S>
stepq_status launch_shape(const Grid &g, int64_t pieces, AttendArgs a, cudaStream_t s) {
    static SmemOptIn opt;
    a.whole = g.cluster;
    a.stages = g.stages;
    stepq_status st = opt((const void *)kv_attend_kernel<S>, kSmemMax);
    if (st != STEPQ_OK) return st;
    st = launch_clusters(kv_attend_kernel<S>, g.ctas, g.cluster ? g.cluster : 1, 32 * kAttWarps, S::smem(g.stages), s, a);
    if (st != STEPQ_OK || g.cluster) return st;
    // CTAs for every head of a piece as far as they all run at once
    const int joins = (int)(pieces < g.ctas ? pieces : g.ctas), at_once = 8 * sm_count() / joins;
    const int each = at_once < 1 ? 1 : at_once < S::HT ? at_once : S::HT;
    auto *join = each < S::HT ? kv_join_kernel<S::HT, S::D, typename S::T, true> : kv_join_kernel<S::HT, S::D, typename S::T, false>;
    return launch_overlapped(join, dim3((unsigned)joins, (unsigned)each), 32 * kJoinWarps, 0, s, a, g.ctas);
}

template <class S>
stepq_status launch_tiles(const stepq_kv_config *c, const AttendArgs &a, int64_t most, bool equal, cudaStream_t s) {
    using L = typename S::Larger;
    const Grid g = grid_of<S>(c, a.groups, a.B, most, equal);
    const int64_t pieces = (int64_t)a.B * c->n_heads * ((a.groups + S::HT - 1) / S::HT);
    // large tiles from 16 small ones a warp on (15 x 19,625 tokens in 4 bits, 19 a warp: 54 us, large 49;
    // 26 x 1,201 with fp32 vectors, 4 a warp: 18.4 and 20.3)
    if constexpr (L::LARGE)
        if (!g.cluster && pieces * ((most + S::TT - 1) / S::TT) >= 16ll * kAttWarps * g.ctas)
            return launch_shape<L>(grid_of<L>(c, a.groups, a.B, most, equal), pieces, a, s);
    return launch_shape<S>(g, pieces, a, s);
}

template <int F>
stepq_status launch_attend(const stepq_kv_config *c, const AttendArgs &a, int64_t most, cudaStream_t s) {
    constexpr int kTile = 64;                                // the largest, in which a window ends
    const bool equal = a.window > 0 && (int64_t)a.window + kTile < most;
    if (equal) most = a.window + kTile;
    return by_shape<F>(c->head_dim, a.groups, a.dtype, [&](auto sh) {
        using S = decltype(sh);
        // in eights where sixteens would leave half of the GPU without a CTA (2 x 900 tokens of 128 channels, four
        // key heads with 16 query heads each, us: 8 bits 12.3 in sixteens, 8.9 in eights; 4 bits 14.1 and 8.8; bf16
        // 9.8 and 8.2. 32 ragged sequences of 500 tokens, 8 heads of 64 channels in 4 bits 18 and 33)
        if constexpr (S::NT > 1) {
            const Grid g = grid_of<S>(c, a.groups, a.B, most, equal);
            if (g.cluster && 2 * g.ctas <= sm_count()) return launch_tiles<Half<S>>(c, a, most, equal, s);
        }
        return launch_tiles<S>(c, a, most, equal, s);
    });
}

}  // namespace kv
}  // namespace stepq
