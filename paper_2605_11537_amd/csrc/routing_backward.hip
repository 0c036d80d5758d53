// The gradient of sorting tokens by expert and back: moe_combine_topk_backward, moe_dispatch_topk_backward, moe_route_topk_backward.
#include "scalar_math.h"

namespace moe {

constexpr int RB_THREADS = 256;
typedef unsigned rb_u32x4_t __attribute__((ext_vector_type(4)));

// the values of a 16-byte piece
template <bool BF16>
__device__ __forceinline__ float piece_value(const rb_u32x4_t &p, int q)
{
    if (!BF16) return __uint_as_float(p[q & 3]);
    const uint32_t w = p[(q >> 1) & 3];
    return __uint_as_float(q & 1 ? w & 0xffff0000u : w << 16);
}
template <bool BF16>
__device__ __forceinline__ rb_u32x4_t piece_of(const float (&v)[BF16 ? 8 : 4])
{
    constexpr int V = BF16 ? 8 : 4;
    rb_u32x4_t r;
#pragma unroll
    for (int q = 0; q < 4; ++q) r[q] = BF16 ? pack_bf16x2(v[(2 * q) % V], v[(2 * q + 1) % V]) : __float_as_uint(v[q % V]);
    return r;
}

// one wavefront per token: its dout once, the k rows of y it met, their gradients
template <bool BF16>
__global__ __launch_bounds__(RB_THREADS) void combine_backward_kernel(const rb_u32x4_t *__restrict__ dout, const rb_u32x4_t *__restrict__ y_perm,
                                                                      const int32_t *__restrict__ inv, const float *__restrict__ weight, int T,
                                                                      int k, int vec_per_row, int residual, rb_u32x4_t *__restrict__ dy_perm,
                                                                      float *__restrict__ dweight, rb_u32x4_t *__restrict__ dx)
{
    constexpr int V = BF16 ? 8 : 4;
    const int s = blockIdx.x * (RB_THREADS / WAVE) + threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
    if (s >= T) return;
    int pos[MOE_MAX_TOPK];
    float p[MOE_MAX_TOPK], dot[MOE_MAX_TOPK];
    bool any = false;
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        pos[j] = j < k ? inv[(size_t)j * T + s] : -1;
        p[j] = j < k ? weight[(size_t)j * T + s] : 0.f;
        dot[j] = 0.f;
        any = any || pos[j] >= 0;
    }
    const rb_u32x4_t zero = {0, 0, 0, 0};
    for (int c = lane; c < vec_per_row; c += WAVE) {
        const rb_u32x4_t g = dout[(size_t)s * vec_per_row + c];
        if (dx) dx[(size_t)s * vec_per_row + c] = residual || !any ? g : zero;
#pragma unroll
        for (int j = 0; j < MOE_MAX_TOPK; ++j) {
            if (pos[j] < 0) continue;
            if (dweight) {
                const rb_u32x4_t y = y_perm[(size_t)pos[j] * vec_per_row + c];
#pragma unroll
                for (int q = 0; q < V; ++q) dot[j] = fmaf(piece_value<BF16>(g, q), piece_value<BF16>(y, q), dot[j]);
            }
            float v[V];
#pragma unroll
            for (int q = 0; q < V; ++q) v[q] = p[j] * piece_value<BF16>(g, q);
            dy_perm[(size_t)pos[j] * vec_per_row + c] = piece_of<BF16>(v);
        }
    }
    if (!dweight) return;
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        if (j >= k) continue;
        const float sum = sum_over<WAVE>(dot[j]);
        if (lane == 0) dweight[(size_t)j * T + s] = sum;
    }
}

// one wavefront per token: the gradients of its k copies, added in choice order behind dx_add
template <bool BF16>
__global__ __launch_bounds__(RB_THREADS) void dispatch_backward_kernel(const rb_u32x4_t *__restrict__ dx_perm, const int32_t *__restrict__ inv,
                                                                       const rb_u32x4_t *dx_add, int T, int k, int vec_per_row, rb_u32x4_t *dx)
{
    constexpr int V = BF16 ? 8 : 4;
    const int s = blockIdx.x * (RB_THREADS / WAVE) + threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
    if (s >= T) return;
    int pos[MOE_MAX_TOPK];
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) pos[j] = j < k ? inv[(size_t)j * T + s] : -1;
    for (int c = lane; c < vec_per_row; c += WAVE) {
        rb_u32x4_t g[MOE_MAX_TOPK], a = {0, 0, 0, 0};
        if (dx_add) a = dx_add[(size_t)s * vec_per_row + c];
#pragma unroll
        for (int j = 0; j < MOE_MAX_TOPK; ++j)
            if (pos[j] >= 0) g[j] = dx_perm[(size_t)pos[j] * vec_per_row + c];
        float v[V];
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] = piece_value<BF16>(a, q);
#pragma unroll
        for (int j = 0; j < MOE_MAX_TOPK; ++j) {
            if (pos[j] < 0) continue;
#pragma unroll
            for (int q = 0; q < V; ++q) v[q] += piece_value<BF16>(g[j], q);
        }
        dx[(size_t)s * vec_per_row + c] = piece_of<BF16>(v);
    }
}

// one wavefront per token, its logits held in registers
constexpr int RB_LOGITS = MOE_MAX_EXPERTS / WAVE;

__global__ __launch_bounds__(RB_THREADS) void route_backward_kernel(const float *__restrict__ logits, const int32_t *__restrict__ idx,
                                                                    const float *__restrict__ dweight, int T, int E, int k, int renormalize,
                                                                    float *__restrict__ dlogits)
{
    const int s = blockIdx.x * (RB_THREADS / WAVE) + threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
    if (s >= T) return;
    const float *row = logits + (size_t)s * E;
    int e[MOE_MAX_TOPK];
    float dw[MOE_MAX_TOPK], w[MOE_MAX_TOPK];
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        const int id = j < k ? idx[(size_t)j * T + s] : -1;
        e[j] = id >= 0 && id < E ? id : -1;
        dw[j] = e[j] >= 0 ? dweight[(size_t)j * T + s] : 0.f;
        w[j] = e[j] >= 0 ? row[e[j]] : -INFINITY;
        top = fmaxf(top, w[j]);
    }
    float v[RB_LOGITS], total = 0.f;
    if (!renormalize) {
#pragma unroll
        for (int i = 0; i < RB_LOGITS; ++i) {
            const int c = i * WAVE + lane;
            v[i] = c < E ? row[c] : -INFINITY;
            top = fmaxf(top, v[i]);
        }
#pragma unroll
        for (int o = 1; o < WAVE; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, WAVE));
#pragma unroll
        for (int i = 0; i < RB_LOGITS; ++i) {
            v[i] = i * WAVE + lane < E ? exp_of<true>(v[i] - top) : 0.f;
            total += v[i];
        }
        total = sum_over<WAVE>(total);
    }
    float mean = 0.f;
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        w[j] = e[j] >= 0 ? exp_of<true>(w[j] - top) : 0.f;
        if (renormalize) total += w[j];
    }
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        w[j] = e[j] >= 0 ? w[j] / total : 0.f;
        mean = fmaf(w[j], dw[j], mean);
    }
#pragma unroll
    for (int i = 0; i < RB_LOGITS; ++i) {
        const int c = i * WAVE + lane;
        if (c >= E) continue;
        float g = renormalize ? 0.f : -(v[i] / total) * mean;
#pragma unroll
        for (int j = 0; j < MOE_MAX_TOPK; ++j)
            if (e[j] == c) g += renormalize ? w[j] * (dw[j] - mean) : w[j] * dw[j];
        dlogits[(size_t)s * E + c] = g;
    }
}

static int rows_check(const char *who, int T, int k, int d, int dtype)
{
    MOE_REQUIRE(T >= 0 && d > 0 && k >= 1 && k <= MOE_MAX_TOPK, MOE_ERR_INVALID_ARG, "%s: T=%d d=%d k=%d out of range (k <= %d)", who, T, d, k,
                MOE_MAX_TOPK);
    MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
    const size_t row = (size_t)d * (dtype == MOE_F32 ? 4 : 2);
    MOE_REQUIRE(row % 16 == 0, MOE_ERR_INVALID_ARG, "%s: row size %zu bytes is not a multiple of 16", who, row);
    return MOE_OK;
}

}  // namespace moe

using namespace moe;

extern "C" int moe_combine_topk_backward(const void *dout, const void *y_perm, const int32_t *inv, const float *expert_weight, int T, int k,
                                         int d, int dtype, int residual, void *dy_perm, float *dweight, void *dx, void *stream)
{
    const int rc = rows_check("moe_combine_topk_backward", T, k, d, dtype);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE(residual == 0 || residual == 1, MOE_ERR_INVALID_ARG, "moe_combine_topk_backward: residual must be 0 or 1");
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(dout && inv && expert_weight && dy_perm && (y_perm || !dweight), MOE_ERR_INVALID_ARG, "moe_combine_topk_backward: null pointer");
    MOE_REQUIRE(dy_perm != dout && dy_perm != y_perm && dx != dout && dx != dy_perm && (!dx || dx != y_perm), MOE_ERR_INVALID_ARG,
                "moe_combine_topk_backward: an output aliases another tensor");
    MOE_REQUIRE(aligned16(dout) && aligned16(y_perm) && aligned16(dy_perm) && aligned16(dx), MOE_ERR_INVALID_ARG,
                "moe_combine_topk_backward: tensor misaligned");
    const int vec = (int)((size_t)d * (dtype == MOE_F32 ? 4 : 2) / 16);
    auto kern = dtype == MOE_BF16 ? combine_backward_kernel<true> : combine_backward_kernel<false>;
    hipLaunchKernelGGL(kern, dim3(ceil_div(T, RB_THREADS / WAVE)), dim3(RB_THREADS), 0, (hipStream_t)stream, (const rb_u32x4_t *)dout,
                       (const rb_u32x4_t *)y_perm, inv, expert_weight, T, k, vec, residual, (rb_u32x4_t *)dy_perm, dweight, (rb_u32x4_t *)dx);
    MOE_CHECK_LAUNCH("moe_combine_topk_backward");
    return MOE_OK;
}

extern "C" int moe_dispatch_topk_backward(const void *dx_perm, const int32_t *inv, const void *dx_add, int T, int k, int d, int dtype, void *dx,
                                          void *stream)
{
    const int rc = rows_check("moe_dispatch_topk_backward", T, k, d, dtype);
    if (rc != MOE_OK || T == 0) return rc;
    MOE_REQUIRE(dx_perm && inv && dx, MOE_ERR_INVALID_ARG, "moe_dispatch_topk_backward: null pointer");
    MOE_REQUIRE(dx != dx_perm, MOE_ERR_INVALID_ARG, "moe_dispatch_topk_backward: dx aliases dx_perm");
    MOE_REQUIRE(aligned16(dx_perm) && aligned16(dx_add) && aligned16(dx), MOE_ERR_INVALID_ARG, "moe_dispatch_topk_backward: tensor misaligned");
    const int vec = (int)((size_t)d * (dtype == MOE_F32 ? 4 : 2) / 16);
    auto kern = dtype == MOE_BF16 ? dispatch_backward_kernel<true> : dispatch_backward_kernel<false>;
    hipLaunchKernelGGL(kern, dim3(ceil_div(T, RB_THREADS / WAVE)), dim3(RB_THREADS), 0, (hipStream_t)stream, (const rb_u32x4_t *)dx_perm, inv,
                       (const rb_u32x4_t *)dx_add, T, k, vec, (rb_u32x4_t *)dx);
    MOE_CHECK_LAUNCH("moe_dispatch_topk_backward");
    return MOE_OK;
}

extern "C" int moe_route_topk_backward(const float *logits, const int32_t *expert_idx, const float *dweight, int T, int E, int k,
                                       int renormalize, float *dlogits, void *stream)
{
    MOE_REQUIRE(T >= 0 && E > 0 && k >= 1 && k <= MOE_MAX_TOPK && k <= E, MOE_ERR_INVALID_ARG,
                "moe_route_topk_backward: T=%d E=%d k=%d out of range (k <= %d, k <= E)", T, E, k, MOE_MAX_TOPK);
    MOE_REQUIRE(renormalize == 0 || renormalize == 1, MOE_ERR_INVALID_ARG, "moe_route_topk_backward: renormalize must be 0 or 1");
    MOE_REQUIRE(E <= MOE_MAX_EXPERTS, MOE_ERR_UNSUPPORTED, "moe_route_topk_backward: E=%d > %d", E, MOE_MAX_EXPERTS);
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(logits && expert_idx && dweight && dlogits, MOE_ERR_INVALID_ARG, "moe_route_topk_backward: null pointer");
    MOE_REQUIRE(dlogits != logits && dlogits != dweight, MOE_ERR_INVALID_ARG, "moe_route_topk_backward: dlogits aliases an input");
    hipLaunchKernelGGL(route_backward_kernel, dim3(ceil_div(T, RB_THREADS / WAVE)), dim3(RB_THREADS), 0, (hipStream_t)stream, logits, expert_idx,
                       dweight, T, E, k, renormalize, dlogits);
    MOE_CHECK_LAUNCH("moe_route_topk_backward");
    return MOE_OK;
}
