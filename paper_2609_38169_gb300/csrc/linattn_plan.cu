// The work of a prompt call laid out on the device, where the sequences' lengths are: segments
// in the order of falling length, which the CTAs of the tensor-core kernel take one after
// another; and the states before the segments of split sequences.
#include "async.cuh"
#include "device.cuh"
#include "linattn_prefill.cuh"

namespace stepq {
namespace la {

// A GB300's multiprocessors. A constant, since the bytes that a call asks for depend on it: they are the
// same whatever device is current when they are asked for, and without one.
constexpr int kSms = 152;

// One CTA per SM takes a segment and head at a time, longest first, so the time of a call is
// about its share W = tokens x Hv / 152 tokens a CTA, or the longest item's length L. Splitting
// a sequence lets its segments run side by side, but the state before each has to be there:
// a pass over k and v alone for the segments' own parts (about 0.55 of the full pass) and a
// scan. It pays where L > 1.6 W. A segment is W / 3 tokens, so that the last round of items is
// short (one prompt of 4096 tokens, 32 heads: 78 us, by W / 4 or W / 6 85; of 16384 209, by W / 2
// 220, W / 4 212, W / 6 223), but not less than 256, whose 128 KiB of state traffic are half of its
// vectors'. Of the 16384 tokens' time the parts take 68 us, the scan 11, the full pass 122; 32 CTAs
// by themselves 470.
Split split_of(int Hv, int B, int tokens, int max_len) {
    const int longest = max_len > 0 && max_len < tokens ? max_len : max_len > 0 ? tokens : (tokens + B - 1) / B;
    const double share = (double)tokens * Hv / kSms;
    Split s{tokens, B, 0};
    if (longest > 512 && longest > 1.6 * share) {
        const int q = (int)(share / 3);
        s.segment = q < 256 ? 256 : (q + kChunk - 1) / kChunk * kChunk;
        s.parts = tokens / s.segment;
        s.most = B + s.parts;
    }
    return s;
}

// Buckets of lengths in chunks: exponent and three bits of mantissa. The last is for the parts: the
// segments of split sequences but each one's last, all of the greatest length.
constexpr int kBuckets = 256, kParts = kBuckets - 1;
__device__ __forceinline__ int bucket_of(int len) {
    const int chunks = (len + kChunk - 1) / kChunk;
    return min(kParts - 1, (int)(__float_as_uint((float)chunks) >> 20) - (127 << 3));
}

// CTA 0: counting sort of the segments by bucket; within one the order is arbitrary, which
// changes no result. Sequences out of range raise the error and make no segment. The workspace is
// laid out for sequences that share no row. Around a sequence whose bounds descend others may share
// rows: if those to be split have more rows together than there are, the call raises the error and
// has no segments at all. The other CTAs look for slots given twice, a sequence a warp at a time.
__global__ void __launch_bounds__(1024) linattn_plan_kernel(PrefillArgs a) {
    __shared__ int count[kBuckets], states, splits;     // states: segments of split sequences
    __shared__ unsigned long long rows;                 // of the sequences to be split
    const int tid = threadIdx.x;
    if (tid < kBuckets) count[tid] = 0;
    if (tid == 0) {
        states = splits = 0;
        rows = 0;
    }
    __syncthreads();
    griddep_wait();
    griddep_launch();
    if (blockIdx.x) {
        for (int b = (blockIdx.x - 1) * 32 + (tid >> 5); b < a.B; b += (gridDim.x - 1) * 32) check_slot(a, b, tid & 31, 32);
        return;
    }
    for (int b = tid; b < a.B; b += 1024) {
        int row, len, slot;
        if (!sequence(a, b, true, row, len, slot)) len = 0;
        const int n = (len + a.segment - 1) / a.segment;
        a.sequences[b] = {n > 1 ? atomicAdd(&states, n) : 0, n};
        if (n > 1) {
            atomicAdd(&rows, (unsigned long long)len);
            atomicAdd(&splits, 1);
            atomicAdd(&count[kParts], n - 1);
        }
        if (n > 0) atomicAdd(&count[bucket_of(len - (n - 1) * a.segment)], 1);
    }
    __syncthreads();
    if (rows > (unsigned long long)a.tokens) {
        for (int b = tid; b < a.B; b += 1024) a.sequences[b] = {0, 0};
        if (tid == 0) {
            *a.plan = PlanHeader{};
            raise_error(a.err, STEPQ_ERR_ARG);
        }
        return;
    }
    // first place of each bucket, the longest first
    if (tid < 32) {
        int run = 0;
        for (int c = kBuckets - 32; c >= 0; c -= 32) {
            const int mine = count[c + 31 - tid];
            int sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int up = __shfl_up_sync(0xffffffffu, sum, o);
                if (tid >= o) sum += up;
            }
            count[c + 31 - tid] = run + sum - mine;
            run += __shfl_sync(0xffffffffu, sum, 31);
        }
        if (tid == 0) *a.plan = PlanHeader{run, states - splits, splits, {0, 0}, {}};
    }
    __syncthreads();
    for (int b = tid; b < a.B; b += 1024) {
        int row, len, slot;
        if (!sequence(a, b, false, row, len, slot)) continue;
        const Sequence q = a.sequences[b];
        if (q.segments > 1) a.split[atomicSub(&splits, 1) - 1] = {b, q.id, q.segments, 0};
        for (int i = 0; i < q.segments; i++) {
            Segment s{row + i * a.segment, min(a.segment, len - i * a.segment), slot, q.id + i, 0, 0, {}};
            s.in = q.segments > 1 ? kStateWork : !a.resume || a.resume[b] ? kStatePool : kStateZero;
            s.out = i == q.segments - 1 ? kStatePool : kStateZero;
            a.table[atomicAdd(&count[i < q.segments - 1 ? kParts : bucket_of(s.len)], 1)] = s;
        }
    }
}

// States before the segments of a split sequence: S_0 from the slot or zero, and
// S_{i+1} = (product of segment i's decays) S_i + U_i, where U_i lies in S_{i+1}'s place. A
// CTA takes 1024 elements of one sequence and head; two states a segment through L2.
// The next kernel starts with this one's end, not under it: its CTAs, placed around this one's, would
// take multiprocessors in twos while others are free (1500 tokens of 7 heads in fp16: 106 us for 83).
__global__ void __launch_bounds__(256) linattn_join_kernel(PrefillArgs a) {
    griddep_wait();
    const int part = blockIdx.x & 15, item = blockIdx.x >> 4, i = item / a.Hv, h = item - i * a.Hv;
    const SplitSequence q = a.split[i];                     // (on its way with the number of them)
    if (i >= a.plan->splits) return;
    const int e = part * 1024 + 4 * threadIdx.x;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!a.resume || a.resume[q.b]) s = *(const float4 *)(pool_page(a, a.slots[q.b], h) + e);
    float *at = a.states + ((uint64_t)q.id * a.Hv + h) * kN + e;
    const float *total = a.totals + (uint64_t)q.id * a.Hv + h;
    const uint64_t step = (uint64_t)a.Hv * kN;
    *(float4 *)at = s;
    constexpr int N = 4;                                // segments read ahead
    for (int j = 1; j < q.segments; j += N) {
        float4 u[N];
        float g[N];
#pragma unroll
        for (int n = 0; n < N; n++)
            if (j + n < q.segments) {
                u[n] = *(const float4 *)(at + (j + n) * step);
                g[n] = total[(j + n - 1) * a.Hv];
            }
#pragma unroll
        for (int n = 0; n < N; n++)
            if (j + n < q.segments) {
                s = make_float4(fmaf(g[n], s.x, u[n].x), fmaf(g[n], s.y, u[n].y), fmaf(g[n], s.z, u[n].z), fmaf(g[n], s.w, u[n].w));
                *(float4 *)(at + (j + n) * step) = s;
            }
    }
}

stepq_status launch_linattn_plan(const PrefillArgs &a, cudaStream_t s) {
    const int pairs = a.B < 2 ? 0 : (a.B + 31) / 32;
    return launch_overlapped(linattn_plan_kernel, 1 + (pairs < kSms ? pairs : kSms), 1024, 0, s, a);
}
stepq_status launch_linattn_join(const PrefillArgs &a, int splits, cudaStream_t s) {
    return launch_overlapped(linattn_join_kernel, splits * a.Hv * 16, 256, 0, s, a);
}

}  // namespace la
}  // namespace stepq
