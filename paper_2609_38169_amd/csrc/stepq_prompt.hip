// Prompts: packed sequences through the gated recurrences of stepq_rule.
#include "stepq_seq.h"

namespace stepq {
namespace {

struct PromptArgs {
    const int32_t *cu;
    const void *q, *k, *v;
    Gate alpha, beta;        // beta.p NULL: 1
    void *o;
    const float *state_in;   // NULL: zeros
    const int32_t *in_ids;
    float *state_out;
    int64_t sq, sk, sv, so;  // token strides
    int32_t T, n_seq, Hv, Hqk, dk, dv, n_in;
};

// The recurrence itself, token by token: a thread holds one column of the
// state, a workgroup 64 columns of one (sequence, head).
template <typename T, int DK, bool DELTA>
__global__ __launch_bounds__(64) void prompt_tokens_kernel(PromptArgs a)
{
    constexpr int N = 16;
    __shared__ float sk[N][DK], sq[N][DK], sa[N], sb[N];
    const int blocks = a.dv / 64, x = blockIdx.x;
    const int col = (x % blocks) * 64 + threadIdx.x, h = x / blocks % a.Hv, s = x / blocks / a.Hv;
    const int hq = h / (a.Hv / a.Hqk);
    const int from = min(max(a.cu[s], 0), a.T), to = min(max(a.cu[s + 1], from), a.T);
    const int src = a.state_in ? (a.in_ids ? a.in_ids[s] : s) : -1;
    float S[DK];
    const float *in = a.state_in + (static_cast<size_t>(src) * a.Hv + h) * a.dk * a.dv + col;
#pragma unroll
    for (int i = 0; i < DK; ++i)
        S[i] = src >= 0 && src < a.n_in && i < a.dk ? in[static_cast<size_t>(i) * a.dv] : 0.0f;
    for (int t0 = from; t0 < to; t0 += N) {
        __syncthreads();
        for (int e = threadIdx.x; e < N * DK; e += 64) {
            const int t = t0 + e / DK, i = e % DK;
            const bool in_range = t < to && i < a.dk;
            sk[e / DK][i] = in_range ? widen(static_cast<const T *>(a.k)[t * a.sk + hq * a.dk + i]) : 0.0f;
            sq[e / DK][i] = in_range ? widen(static_cast<const T *>(a.q)[t * a.sq + hq * a.dk + i]) : 0.0f;
        }
        if (threadIdx.x < N && t0 + threadIdx.x < to) {
            const size_t g = static_cast<size_t>(t0 + threadIdx.x) * a.Hv + h;
            sa[threadIdx.x] = a.alpha.at(g);
            sb[threadIdx.x] = a.beta.p ? a.beta.at(g) : 1.0f;
        }
        __syncthreads();
        for (int n = 0; n < N && t0 + n < to; ++n) {
            const size_t t = t0 + n;
            float u = widen(static_cast<const T *>(a.v)[t * a.sv + h * a.dv + col]), ks = 0.0f, y = 0.0f;
#pragma unroll
            for (int i = 0; i < DK; ++i) {
                if (i % 32 == 0) __builtin_amdgcn_sched_barrier(0);   // few rows of k in flight: no spills
                S[i] *= sa[n];
                if (DELTA) ks = fmaf(S[i], sk[n][i], ks);
            }
            u = sb[n] * (u - ks);
#pragma unroll
            for (int i = 0; i < DK; ++i) {
                if (i % 32 == 0) __builtin_amdgcn_sched_barrier(0);
                S[i] = fmaf(sk[n][i], u, S[i]);
                y = fmaf(S[i], sq[n][i], y);
            }
            static_cast<T *>(a.o)[t * a.so + h * a.dv + col] = narrow<T>(y);
        }
    }
    float *out = a.state_out + (static_cast<size_t>(s) * a.Hv + h) * a.dk * a.dv + col;
#pragma unroll
    for (int i = 0; i < DK; ++i)
        if (i < a.dk) out[static_cast<size_t>(i) * a.dv] = S[i];
}

template <typename T, int DK>
void launch(const PromptArgs &a, bool delta, hipStream_t s)
{
    const dim3 grid(static_cast<unsigned>(a.n_seq) * a.Hv * (a.dv / 64));
    if (delta) prompt_tokens_kernel<T, DK, true><<<grid, 64, 0, s>>>(a);
    else prompt_tokens_kernel<T, DK, false><<<grid, 64, 0, s>>>(a);
}

stepq_status check(const stepq_prompt_desc *d)
{
    if (!d) return bad("desc is NULL");
    if (d->n_v_heads < 1 || d->n_qk_heads < 1 || d->n_v_heads % d->n_qk_heads)
        return bad("head counts must be >= 1 and n_v_heads a multiple of n_qk_heads");
    if (d->d_k < 1 || d->d_k > 128 || (d->d_v != 64 && d->d_v != 128))
        return set_error(STEPQ_E_UNSUPPORTED, "d_k must be 1 .. 128 and d_v 64 or 128");
    if (!known_dtype(d->act_dtype) || !known_dtype(d->gate_dtype)) return bad("unknown activation or gate dtype");
    if (d->rule != STEPQ_RULE_DECAY && d->rule != STEPQ_RULE_DELTA) return bad("unknown rule");
    if (d->n_tokens < 0 || d->n_seq < 0 || d->n_states_in < 0) return bad("negative count");
    if (d->n_tokens >= (int64_t(1) << 31))
        return set_error(STEPQ_E_UNSUPPORTED, "2^31 tokens or more in one call: split the batch");
    if (static_cast<int64_t>(d->n_seq) * d->n_v_heads > (int64_t(1) << 24))
        return set_error(STEPQ_E_UNSUPPORTED, "more than 2^24 (sequence, head) pairs in one call: split the batch");
    const int64_t qk = int64_t(d->n_qk_heads) * d->d_k, vo = int64_t(d->n_v_heads) * d->d_v;
    if ((d->q_stride && d->q_stride < qk) || (d->k_stride && d->k_stride < qk) || (d->v_stride && d->v_stride < vo) ||
        (d->o_stride && d->o_stride < vo))
        return bad("a token stride is smaller than a token");
    return STEPQ_OK;
}

}  // namespace
}  // namespace stepq

using namespace stepq;

extern "C" stepq_status stepq_prompt_workspace(const stepq_prompt_desc *d, size_t *bytes)
{
    if (const stepq_status st = check(d)) return st;
    if (!bytes) return bad("bytes is NULL");
    *bytes = 0;
    return STEPQ_OK;
}

extern "C" stepq_status stepq_prompt(const stepq_prompt_desc *d, const int32_t *cu_seqlens, const void *q,
                                     const void *k, const void *v, const void *alpha, const void *beta, void *o,
                                     const float *state_in, const int32_t *in_ids, float *state_out, void *workspace,
                                     size_t workspace_bytes, void *stream)
{
    if (const stepq_status st = check(d)) return st;
    if (d->n_seq == 0) return STEPQ_OK;
    if (!cu_seqlens || !state_out) return bad("NULL cu_seqlens or state_out");
    if (d->n_tokens && (!q || !k || !v || !alpha || !o)) return bad("NULL activation or output pointer");
    if (!state_in && in_ids) return bad("in_ids without state_in");
    if (state_in && !in_ids && d->n_states_in < d->n_seq) return bad("fewer states in state_in than sequences");
    if (state_in == state_out && in_ids) return bad("state_out must not be state_in where in_ids chooses the states");
    const int64_t qk = int64_t(d->n_qk_heads) * d->d_k, vo = int64_t(d->n_v_heads) * d->d_v;
    const int32_t gf = d->gate_dtype == STEPQ_F32;
    PromptArgs a{cu_seqlens, q, k, v, {alpha, gf}, {beta, gf}, o, state_in, in_ids, state_out,
                 d->q_stride ? d->q_stride : qk, d->k_stride ? d->k_stride : qk, d->v_stride ? d->v_stride : vo,
                 d->o_stride ? d->o_stride : vo, static_cast<int32_t>(d->n_tokens), d->n_seq, d->n_v_heads,
                 d->n_qk_heads, d->d_k, d->d_v, d->n_states_in};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool delta = d->rule == STEPQ_RULE_DELTA;
    if (d->act_dtype == STEPQ_BF16) {
        if (d->d_k > 64) launch<bf16_t, 128>(a, delta, s);
        else launch<bf16_t, 64>(a, delta, s);
    } else {
        if (d->d_k > 64) launch<float, 128>(a, delta, s);
        else launch<float, 64>(a, delta, s);
    }
    return launched("prompt launch");
}
