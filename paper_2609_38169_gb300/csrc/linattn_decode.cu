// Decayed linear attention, one token: X = g S + k v^T in place, y = X^T q, for every
// (slot, value head) of a batch.
//
// One CTA per state: 128 x 128 fp32 read and written once, 128 KiB against 5 x 128^2
// operations, so HBM bounds it: 1024 slots of 32 heads take 616 us, 7.0 TB/s. All loads of a
// thread (16 x 16 bytes) are issued before the first is used.
#include "async.cuh"
#include "device.cuh"
#include "linattn.cuh"

namespace stepq {
namespace la {

struct DecodeArgs {
    float *pool;
    uint64_t slot_floats, layer_off;
    int pool_slots, nb, Hk, Hv;
    const int32_t *slots;
    const void *q, *k, *v;
    const float *gate;
    void *y;
    int64_t qs, ks, vs, gs, ys;
    NormArgs norm;
    unsigned int *err;
};

template <class T>
__global__ void __launch_bounds__(kThreads) linattn_decode_kernel(DecodeArgs a) {
    __shared__ float kq[2][kD];
    __shared__ float red[8][kD];
    const int tid = threadIdx.x, w = tid >> 5, l = tid & 31;
    griddep_wait();
    griddep_launch();
    const int b = blockIdx.x / a.Hv, h = blockIdx.x - b * a.Hv, hk = h / (a.Hv / a.Hk);
    const int slot = a.slots[b];
    // entry i of the batch against those after it
    if ((int)blockIdx.x < a.nb)
        for (int i = blockIdx.x, j = i + 1 + tid; j < a.nb; j += kThreads) {
            const int s = a.slots[i];
            if (a.slots[j] == s && s >= 0 && s < a.pool_slots) raise_error(a.err, STEPQ_ERR_DUP_SLOT);
        }
    if (slot < 0 || slot >= a.pool_slots) {
        if (tid == 0) raise_error(a.err, STEPQ_ERR_SLOT_RANGE);
        return;
    }
    float4 *S = (float4 *)(a.pool + (uint64_t)slot * a.slot_floats + a.layer_off + (uint64_t)h * kN);
    float4 s[16];
#pragma unroll
    for (int p = 0; p < 16; p++) s[p] = S[(8 * p + w) * 32 + l];
    if (tid < kD) kq[0][tid] = to_f32(((const T *)a.k)[b * a.ks + hk * kD + tid]);
    else kq[1][tid - kD] = to_f32(((const T *)a.q)[b * a.qs + hk * kD + tid - kD]);
    const float g = a.gate[b * a.gs + h];
    float v[4];
    load_vec<T, 4>((const T *)a.v + b * a.vs + h * kD + 4 * l, v);
    __syncthreads();
    float y[1][4] = {};
#pragma unroll
    for (int p = 0; p < 16; p++) {
        const int i = 8 * p + w;
        const float ki = kq[0][i], qi = kq[1][i];
        s[p] = make_float4(fmaf(ki, v[0], g * s[p].x), fmaf(ki, v[1], g * s[p].y), fmaf(ki, v[2], g * s[p].z),
                           fmaf(ki, v[3], g * s[p].w));
        S[i * 32 + l] = s[p];
        y[0][0] = fmaf(qi, s[p].x, y[0][0]);
        y[0][1] = fmaf(qi, s[p].y, y[0][1]);
        y[0][2] = fmaf(qi, s[p].z, y[0][2]);
        y[0][3] = fmaf(qi, s[p].w, y[0][3]);
    }
    *(float4 *)&red[w][4 * l] = make_float4(y[0][0], y[0][1], y[0][2], y[0][3]);
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int o = 1; o < 8; o++) {
        const float4 r = *(const float4 *)&red[o][4 * l];
        y[0][0] += r.x;
        y[0][1] += r.y;
        y[0][2] += r.z;
        y[0][3] += r.w;
    }
    if (a.norm.on) {
        Vec<T, 4> z{};
        if (a.norm.z) z = *(const Vec<T, 4> *)((const T *)a.norm.z + b * a.norm.z_stride + h * kD + 4 * l);
        norm_head<T, 1>(a.norm, HeadAffine(a.norm, h, l), &z, y);
    }
    store_vec<T, 4>((T *)a.y + b * a.ys + h * kD + 4 * l, y[0]);
}

}  // namespace la

stepq_status launch_linattn_decode(const stepq_config *cfg, int layer, float *pool, int pool_slots,
                                   const int32_t *slots, int B, const stepq_linattn_io *io,
                                   const stepq_norm *norm, cudaStream_t s) {
    la::DecodeArgs a{};
    const uint64_t per_layer = (uint64_t)kN * cfg->n_value_heads;
    a.pool = pool;
    a.slot_floats = per_layer * cfg->n_layers;
    a.layer_off = per_layer * layer;
    a.pool_slots = pool_slots;
    a.nb = B;
    a.Hk = cfg->n_key_heads;
    a.Hv = cfg->n_value_heads;
    a.slots = slots;
    a.q = io->q; a.k = io->k; a.v = io->v; a.gate = io->gate; a.y = io->y;
    a.qs = io->q_stride; a.ks = io->k_stride; a.vs = io->v_stride; a.gs = io->gate_stride; a.ys = io->y_stride;
    a.norm = la::norm_args(norm);
    a.err = device_error_word();
    return la::by_type(io->dtype, [&](auto t) {
        return launch_overlapped(la::linattn_decode_kernel<decltype(t)>, B * a.Hv, kThreads, 0, s, a);
    });
}

}  // namespace stepq
