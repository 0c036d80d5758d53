// moe_token_logprobs and its gradient: log probabilities of given ids, entropy and the best alternatives of rows of logits.
#include <float.h>

#include "scalar_math.h"

namespace moe {

constexpr int LP_THREADS = 256;
constexpr int LP_WAVES = LP_THREADS / WAVE;

__device__ __forceinline__ float lp_max(float v, float *scratch)
{
#pragma unroll
    for (int o = 1; o < WAVE; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, WAVE));
    if (threadIdx.x % WAVE == 0) scratch[threadIdx.x / WAVE] = v;
    __syncthreads();
    for (int i = 0; i < LP_WAVES; ++i) v = fmaxf(v, scratch[i]);
    __syncthreads();
    return v;
}
__device__ __forceinline__ float lp_sum(float v, float *scratch)
{
    v = sum_over<WAVE>(v);
    if (threadIdx.x % WAVE == 0) scratch[threadIdx.x / WAVE] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < LP_WAVES; ++i) v += scratch[i];
    __syncthreads();
    return v;
}

// one workgroup per row: the maximum, the sums, then the alternatives one by one
template <class X>
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_kernel(const X *__restrict__ logits, size_t stride, const int32_t *__restrict__ target,
                                                                    int V, int k, float *__restrict__ logprob, float *__restrict__ entropy,
                                                                    float *__restrict__ lse, int32_t *__restrict__ top_idx,
                                                                    float *__restrict__ top_logprob)
{
    __shared__ float scratch[LP_WAVES];
    __shared__ int scratch_id[LP_WAVES];
    const size_t n = blockIdx.x;
    const X *row = logits + n * stride;
    float m = -FLT_MAX;                                  // finite where everything is masked: the sum is then zero
    for (int i = threadIdx.x; i < V; i += LP_THREADS) m = fmaxf(m, value_of(row[i]));
    m = lp_max(m, scratch);
    float s = 0.f, t = 0.f;
    for (int i = threadIdx.x; i < V; i += LP_THREADS) {
        const float d = value_of(row[i]) - m, e = exp_of<true>(d);
        s += e;
        if (e != 0.f) t = fmaf(d, e, t);                 // a masked logit: zero, not zero times infinity
    }
    s = lp_sum(s, scratch);
    t = lp_sum(t, scratch);
    const bool none = s == 0.f;
    const float log_s = logf(s);
    if (threadIdx.x == 0) {
        const int a = target[n];
        logprob[n] = a < 0 || a >= V ? 0.f : none ? -INFINITY : value_of(row[a]) - m - log_s;
        entropy[n] = none ? 0.f : log_s - t / s;
        lse[n] = none ? -INFINITY : m + log_s;
    }
    float after = INFINITY;
    int after_id = -1;
    for (int j = 0; j < k; ++j) {                        // the largest behind the one before: smaller, or equal with a higher id
        float best = -INFINITY;
        int id = V;
        for (int i = threadIdx.x; i < V; i += LP_THREADS) {
            float v = value_of(row[i]);
            if (v != v) v = -INFINITY;
            if ((v < after || (v == after && i > after_id)) && (v > best || id == V)) best = v, id = i;
        }
#pragma unroll
        for (int o = 1; o < WAVE; o <<= 1) {
            const float ov = __shfl_xor(best, o, WAVE);
            const int oi = __shfl_xor(id, o, WAVE);
            argmax_merge(best, id, ov, oi);
        }
        if (threadIdx.x % WAVE == 0) scratch[threadIdx.x / WAVE] = best, scratch_id[threadIdx.x / WAVE] = id;
        __syncthreads();
        for (int i = 0; i < LP_WAVES; ++i) argmax_merge(best, id, scratch[i], scratch_id[i]);
        __syncthreads();
        if (threadIdx.x == 0) {
            top_idx[n * k + j] = id;
            top_logprob[n * k + j] = none ? -INFINITY : best - m - log_s;
        }
        after = best;
        after_id = id;
    }
}

template <class X>
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_backward_kernel(const X *logits, size_t stride, const int32_t *__restrict__ target,
                                                                             const float *__restrict__ lse, const float *__restrict__ entropy,
                                                                             const float *__restrict__ dlogprob, const float *__restrict__ dentropy,
                                                                             int V, X *dlogits, size_t dstride)
{
    const size_t n = blockIdx.x;
    const int a = target[n];
    const float g = a < 0 || a >= V ? 0.f : dlogprob[n], q = dentropy ? dentropy[n] : 0.f, z = lse[n], H = dentropy ? entropy[n] : 0.f;
    for (int i = threadIdx.x; i < V; i += LP_THREADS) {
        const float lp = value_of(logits[n * stride + i]) - z, p = exp_of<true>(lp);
        float d = 0.f;
        if (z != -INFINITY) {                            // nothing was left of the row
            d = p == 0.f ? 0.f : -p * fmaf(q, lp + H, g);
            if (i == a) d += g;
        }
        store_value(dlogits + n * dstride + i, d);
    }
}

static int logprobs_check(const char *who, int N, int V, long long stride, int dtype)
{
    MOE_REQUIRE(N >= 0 && V > 0, MOE_ERR_INVALID_ARG, "%s: N=%d V=%d out of range", who, N, V);
    MOE_REQUIRE(stride >= V, MOE_ERR_INVALID_ARG, "%s: rows of %d logits lie %lld apart", who, V, stride);
    MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
    return MOE_OK;
}

}  // namespace moe

using namespace moe;

extern "C" size_t moe_token_logprobs_workspace_bytes(int N, int V, int k, int dtype)
{
    (void)N, (void)V, (void)k, (void)dtype;
    return 0;
}

extern "C" int moe_token_logprobs(const void *logits, long long row_stride, const int32_t *target, int N, int V, int dtype, int k,
                                  float *logprob, float *entropy, float *lse, int32_t *top_idx, float *top_logprob, void *ws, size_t ws_bytes,
                                  void *stream)
{
    const int rc = logprobs_check("moe_token_logprobs", N, V, row_stride, dtype);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE(k >= 0 && k <= MOE_MAX_TOPK && k <= V, MOE_ERR_INVALID_ARG, "moe_token_logprobs: k=%d out of range (k <= %d, k <= V)", k, MOE_MAX_TOPK);
    if (N == 0) return MOE_OK;
    MOE_REQUIRE(logits && target && logprob && entropy && lse && (k == 0 || (top_idx && top_logprob)), MOE_ERR_INVALID_ARG,
                "moe_token_logprobs: null pointer");
    hipStream_t st = (hipStream_t)stream;
    if (dtype == MOE_BF16)
        hipLaunchKernelGGL(token_logprobs_kernel<bf16_t>, dim3(N), dim3(LP_THREADS), 0, st, (const bf16_t *)logits, (size_t)row_stride, target, V, k,
                           logprob, entropy, lse, top_idx, top_logprob);
    else
        hipLaunchKernelGGL(token_logprobs_kernel<float>, dim3(N), dim3(LP_THREADS), 0, st, (const float *)logits, (size_t)row_stride, target, V, k,
                           logprob, entropy, lse, top_idx, top_logprob);
    MOE_CHECK_LAUNCH("moe_token_logprobs");
    return MOE_OK;
}

extern "C" int moe_token_logprobs_backward(const void *logits, long long row_stride, const int32_t *target, const float *lse,
                                           const float *entropy, const float *dlogprob, const float *dentropy, int N, int V, int dtype,
                                           void *dlogits, long long dlogits_stride, void *stream)
{
    const int rc = logprobs_check("moe_token_logprobs_backward", N, V, row_stride < dlogits_stride ? row_stride : dlogits_stride, dtype);
    if (rc != MOE_OK || N == 0) return rc;
    MOE_REQUIRE(logits && target && lse && dlogprob && dlogits && (entropy || !dentropy), MOE_ERR_INVALID_ARG,
                "moe_token_logprobs_backward: null pointer");
    MOE_REQUIRE(dlogits != logits || dlogits_stride == row_stride, MOE_ERR_INVALID_ARG,
                "moe_token_logprobs_backward: dlogits lies on logits with another stride");
    hipStream_t st = (hipStream_t)stream;
    if (dtype == MOE_BF16)
        hipLaunchKernelGGL(token_logprobs_backward_kernel<bf16_t>, dim3(N), dim3(LP_THREADS), 0, st, (const bf16_t *)logits, (size_t)row_stride,
                           target, lse, entropy, dlogprob, dentropy, V, (bf16_t *)dlogits, (size_t)dlogits_stride);
    else
        hipLaunchKernelGGL(token_logprobs_backward_kernel<float>, dim3(N), dim3(LP_THREADS), 0, st, (const float *)logits, (size_t)row_stride,
                           target, lse, entropy, dlogprob, dentropy, V, (float *)dlogits, (size_t)dlogits_stride);
    MOE_CHECK_LAUNCH("moe_token_logprobs_backward");
    return MOE_OK;
}
