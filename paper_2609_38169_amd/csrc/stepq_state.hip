// One token of a batch of requests on full-precision states, in place.
#include "stepq_seq.h"

namespace stepq {
namespace {

struct StateArgs {
    float *state;
    const int32_t *ids;
    const void *q, *k, *v;
    Gate alpha, beta;        // beta.p NULL: 1
    float *o;
    int32_t n_states, Hv, Hqk, dk, batch;
};

constexpr int kThreads = 256;

// One workgroup per (request, head).  A thread holds 4 neighbouring columns of
// every RG-th row in registers, so that the state is read once and written
// once, 16 bytes a lane:
//   ks = S^T k, qs = S^T q in one pass (sums over the rows: within the thread,
//   the wave, then across the waves in LDS);
//   u = beta (v - alpha ks);  o = alpha qs + (q.k) u  (= S'^T q);  S' = alpha S + k u^T.
// Bound by memory: 8 d_k d_v bytes per tile.  512 requests x 32 heads of
// 128 x 128: 2.15 GB in 422 us, 5.1 TB/s, what a large copy reaches; one request
// of 4 heads of 64 x 64: 4.1 us, a launch.
template <typename T, int DV, bool DELTA>
__global__ __launch_bounds__(kThreads) void state_step_kernel(StateArgs a)
{
    constexpr int CG = DV / 4, RG = kThreads / CG, R = 128 / RG, NW = kThreads / 64;
    __shared__ float sk[128], sq[128];
    __shared__ float4 red[NW][2][CG];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int b = blockIdx.x / a.Hv, h = blockIdx.x - b * a.Hv, hq = h / (a.Hv / a.Hqk);
    const int cg = tid % CG, rg = tid / CG;
    const size_t bh = static_cast<size_t>(b) * a.Hv + h;
    float *o = a.o + bh * DV;
    const int id = a.ids[b];
    if (id < 0 || id >= a.n_states) {
        if (tid < DV) o[tid] = 0.0f;
        return;
    }
    float4 *S = reinterpret_cast<float4 *>(a.state + (static_cast<size_t>(id) * a.Hv + h) * a.dk * DV);
    float4 x[R];
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const int i = rg + RG * n;
        x[n] = i < a.dk ? S[static_cast<size_t>(i) * CG + cg] : make_float4(0, 0, 0, 0);
    }
    if (tid < 128) {
        const size_t at = (static_cast<size_t>(b) * a.Hqk + hq) * a.dk + tid;
        sk[tid] = tid < a.dk ? widen(static_cast<const T *>(a.k)[at]) : 0.0f;
        sq[tid] = tid < a.dk ? widen(static_cast<const T *>(a.q)[at]) : 0.0f;
    }
    const float al = a.alpha.at(bh), be = a.beta.p ? a.beta.at(bh) : 1.0f;
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = widen(static_cast<const T *>(a.v)[bh * DV + cg * 4 + j]);
    __syncthreads();
    float ks[4] = {}, qs[4] = {}, qk = sq[lane] * sk[lane] + sq[lane + 64] * sk[lane + 64];
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const float ki = sk[rg + RG * n], qi = sq[rg + RG * n];
        const float e[4] = {x[n].x, x[n].y, x[n].z, x[n].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (DELTA) ks[j] = fmaf(ki, e[j], ks[j]);
            qs[j] = fmaf(qi, e[j], qs[j]);
        }
    }
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) qk += __shfl_xor(qk, m);
#pragma unroll
    for (int m = CG; m < 64; m <<= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (DELTA) ks[j] += __shfl_xor(ks[j], m);
            qs[j] += __shfl_xor(qs[j], m);
        }
    if (lane < CG) {
        if (DELTA) red[wave][0][lane] = make_float4(ks[0], ks[1], ks[2], ks[3]);
        red[wave][1][lane] = make_float4(qs[0], qs[1], qs[2], qs[3]);
    }
    __syncthreads();
    float4 tk = make_float4(0, 0, 0, 0), tq = tk;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (DELTA) {
            const float4 y = red[w][0][cg];
            tk.x += y.x, tk.y += y.y, tk.z += y.z, tk.w += y.w;
        }
        const float4 z = red[w][1][cg];
        tq.x += z.x, tq.y += z.y, tq.z += z.z, tq.w += z.w;
    }
    float u[4] = {v[0], v[1], v[2], v[3]};
    if (DELTA) u[0] -= al * tk.x, u[1] -= al * tk.y, u[2] -= al * tk.z, u[3] -= al * tk.w;
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] *= be;
    if (rg == 0) {
        float4 y;
        y.x = fmaf(qk, u[0], al * tq.x), y.y = fmaf(qk, u[1], al * tq.y);
        y.z = fmaf(qk, u[2], al * tq.z), y.w = fmaf(qk, u[3], al * tq.w);
        reinterpret_cast<float4 *>(o)[cg] = y;
    }
#pragma unroll
    for (int n = 0; n < R; ++n) {
        const int i = rg + RG * n;
        if (i < a.dk) {
            const float ki = sk[i];
            float4 y;
            y.x = fmaf(ki, u[0], al * x[n].x), y.y = fmaf(ki, u[1], al * x[n].y);
            y.z = fmaf(ki, u[2], al * x[n].z), y.w = fmaf(ki, u[3], al * x[n].w);
            S[static_cast<size_t>(i) * CG + cg] = y;
        }
    }
}

template <typename T>
void launch(const StateArgs &a, int dv, bool delta, hipStream_t s)
{
    const dim3 grid(static_cast<unsigned>(a.batch) * a.Hv);
    if (dv == 128) {
        if (delta) state_step_kernel<T, 128, true><<<grid, kThreads, 0, s>>>(a);
        else state_step_kernel<T, 128, false><<<grid, kThreads, 0, s>>>(a);
    } else {
        if (delta) state_step_kernel<T, 64, true><<<grid, kThreads, 0, s>>>(a);
        else state_step_kernel<T, 64, false><<<grid, kThreads, 0, s>>>(a);
    }
}

}  // namespace
}  // namespace stepq

using namespace stepq;

extern "C" stepq_status stepq_state_step(const stepq_state_desc *d, float *state, const int32_t *ids, int32_t batch,
                                         const void *q, const void *k, const void *v, const void *alpha,
                                         const void *beta, float *o, void *stream)
{
    if (!d) return bad("desc is NULL");
    if (d->n_v_heads < 1 || d->n_qk_heads < 1 || d->n_v_heads % d->n_qk_heads)
        return bad("head counts must be >= 1 and n_v_heads a multiple of n_qk_heads");
    if (d->d_k < 1 || d->d_k > 128 || (d->d_v != 64 && d->d_v != 128))
        return set_error(STEPQ_E_UNSUPPORTED, "d_k must be 1 .. 128 and d_v 64 or 128");
    if (!known_dtype(d->act_dtype) || !known_dtype(d->gate_dtype)) return bad("unknown activation or gate dtype");
    if (d->rule != STEPQ_RULE_DECAY && d->rule != STEPQ_RULE_DELTA) return bad("unknown rule");
    if (d->n_states < 0 || batch < 0) return bad("negative count");
    if (batch > d->n_states) return bad("more requests than states");
    if (static_cast<int64_t>(batch) * d->n_v_heads >= (int64_t(1) << 24))        // a launch has less than 2^32 threads
        return set_error(STEPQ_E_UNSUPPORTED, "2^24 or more (request, head) tiles in one call: split the batch");
    if (batch == 0) return STEPQ_OK;
    if (!state || !ids || !q || !k || !v || !alpha || !o) return bad("NULL state, ids, activation or output pointer");
    if (!aligned(state, 16) || !aligned(o, 16)) return bad("state and o must be 16-byte aligned");
    const int32_t gf = d->gate_dtype == STEPQ_F32;
    StateArgs a{state, ids, q, k, v, {alpha, gf}, {beta, gf}, o, d->n_states, d->n_v_heads, d->n_qk_heads, d->d_k, batch};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->act_dtype == STEPQ_BF16) launch<bf16_t>(a, d->d_v, d->rule == STEPQ_RULE_DELTA, s);
    else launch<float>(a, d->d_v, d->rule == STEPQ_RULE_DELTA, s);
    return launched("state step launch");
}
