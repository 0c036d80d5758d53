// The gradient of sorting tokens by expert and back: moe_combine_topk_backward, moe_dispatch_topk_backward, moe_route_topk_backward.
// Rows are moved once and memory binds.  65536 tokens of 768 bf16, one choice: combine 76 us (5.0 TB/s), dispatch 56 us (5.2 TB/s), the gate over 256
// experts 26 us (5.1 TB/s), renormalised, which reads no other logits, 15 us; 4096 tokens, three choices: 10 and 7 us, of which launch and first load are half.
#include <float.h>

#include "row_groups.h"
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

// The row of this thread's group of 2^lg lanes (256 at most: a workgroup), in a grid of rows_grid.
__device__ __forceinline__ unsigned rb_row(int lg, int &lane)
{
    lane = threadIdx.x & ((1 << lg) - 1);
    return (((blockIdx.y << ROWS_GRID_LG) + blockIdx.x) << (8 - lg)) + (threadIdx.x >> lg);
}

// The row of x_perm that an assignment went to, below rows; -1: none.  An entry of inv beyond the rows names none.
__device__ __forceinline__ int rb_place(const int32_t *inv, size_t a, unsigned rows)
{
    const int r = inv[a];
    return (unsigned)r < rows ? r : -1;
}

// A group of lanes per token: its dout once, PIECES pieces a lane at a time, the rows of y it met (KMAX at most, all asked for before the
// first is used), their gradients.  dweight: lanes' sums, then the wavefronts' in their order where a workgroup shares a row.
template <bool BF16, int PIECES, int KMAX>
__global__ __launch_bounds__(RB_THREADS) void combine_backward_kernel(const rb_u32x4_t *__restrict__ dout, const rb_u32x4_t *__restrict__ y_perm,
                                                                      const int32_t *__restrict__ inv, const float *__restrict__ weight, int T,
                                                                      int k, int vec_per_row, int lg, int residual, rb_u32x4_t *__restrict__ dy_perm,
                                                                      float *__restrict__ dweight, rb_u32x4_t *__restrict__ dx)
{
    constexpr int V = BF16 ? 8 : 4;
    __shared__ float sums[RB_THREADS / WAVE][KMAX];
    int lane;
    const unsigned s = rb_row(lg, lane);
    if (s >= (unsigned)T) return;                        // where a workgroup has a row: the whole workgroup
    const int lanes = 1 << lg;
    int pos[KMAX];
    float p[KMAX], dot[KMAX];
    bool any = false;
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
        pos[j] = -1, p[j] = dot[j] = 0.f;
        if (j >= k) continue;
        pos[j] = rb_place(inv, (size_t)j * T + s, (unsigned)k * T);
        p[j] = weight[(size_t)j * T + s];
        any = any || pos[j] >= 0;
    }
    const bool pass = residual || !any;
    for (int c0 = lane; c0 < vec_per_row; c0 += lanes * PIECES) {
        rb_u32x4_t g[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            if (c0 + i * lanes < vec_per_row) g[i] = dout[(size_t)s * vec_per_row + c0 + i * lanes];
        rb_u32x4_t y[KMAX][PIECES];
        if (dweight) {
#pragma unroll
            for (int j = 0; j < KMAX; ++j) {
                if (pos[j] < 0) continue;
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
                    if (c0 + i * lanes < vec_per_row) y[j][i] = y_perm[(size_t)pos[j] * vec_per_row + c0 + i * lanes];
            }
        }
#pragma unroll
        for (int j = 0; j < KMAX; ++j) {
            if (pos[j] < 0) continue;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                if (c0 + i * lanes >= vec_per_row) continue;
                float v[V];
#pragma unroll
                for (int q = 0; q < V; ++q) v[q] = p[j] * piece_value<BF16>(g[i], q);
                dy_perm[(size_t)pos[j] * vec_per_row + c0 + i * lanes] = piece_of<BF16>(v);
                if (dweight) {
#pragma unroll
                    for (int q = 0; q < V; ++q) dot[j] = fmaf(piece_value<BF16>(g[i], q), piece_value<BF16>(y[j][i], q), dot[j]);
                }
            }
        }
        if (dx) {
            const rb_u32x4_t zero = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                if (c0 + i * lanes < vec_per_row) dx[(size_t)s * vec_per_row + c0 + i * lanes] = pass ? g[i] : zero;
        }
    }
    if (!dweight) return;
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
        if (j >= k) break;
        float v = dot[j];
        if (lg >= 1) v += group_exchange<0>(v);
        if (lg >= 2) v += group_exchange<1>(v);
        if (lg >= 3) v += group_exchange<2>(v);
        if (lg >= 4) v += group_exchange<3>(v);
        if (lg >= 5) v += group_exchange<4>(v);
        if (lg >= 6) v += group_exchange<5>(v);
        if (lg <= 6 && lane == 0) dweight[(size_t)j * T + s] = v;
        if (lg > 6 && lane % WAVE == 0) sums[lane / WAVE][j] = v;
    }
    if (lg <= 6) return;
    __syncthreads();
    if (lane < k) {
        float v = sums[0][lane];
        for (int w = 1; w < lanes / WAVE; ++w) v += sums[w][lane];
        dweight[(size_t)lane * T + s] = v;
    }
}

// A group of lanes per token: the gradients of its k copies, added in choice order behind dx_add.
template <bool BF16>
__global__ __launch_bounds__(RB_THREADS) void dispatch_backward_kernel(const rb_u32x4_t *__restrict__ dx_perm, const int32_t *__restrict__ inv,
                                                                       const rb_u32x4_t *dx_add, int T, int k, int vec_per_row, int lg, rb_u32x4_t *dx)
{
    constexpr int V = BF16 ? 8 : 4;
    int lane;
    const unsigned s = rb_row(lg, lane);
    if (s >= (unsigned)T) return;
    int pos[MOE_MAX_TOPK];
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) pos[j] = j < k ? rb_place(inv, (size_t)j * T + s, (unsigned)k * T) : -1;
    for (int c = lane; c < vec_per_row; c += 1 << lg) {
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

// The largest logit is never below the lowest finite value: a row (with renormalize, its chosen logits) that is masked throughout has exponentials of
// 0, a total of 0 and a gradient of 0, and no infinity is taken from another.  A NaN passes into the total.  A token without a choice has none of either,
// whatever its logits hold.
// LANES lanes per token, RB_LOGITS logits a lane in registers (one wavefront to every token and 1024 places asked: 61 us for 65536 x 256); PIECES:
// four consecutive ones (rows begin on 16 bytes).  With renormalize the other experts' logits take no part and are not read.
constexpr int RB_LOGITS = 16;

template <int LANES, bool PIECES>
__global__ __launch_bounds__(RB_THREADS) void route_backward_kernel(const float *__restrict__ logits, const int32_t *__restrict__ idx,
                                                                    const float *__restrict__ dweight, int T, int E, int k, int renormalize,
                                                                    float *__restrict__ dlogits)
{
    constexpr int P = PIECES ? 4 : 1;
    typedef float piece_t __attribute__((ext_vector_type(P)));
    int lane;
    const unsigned s = rb_row(LANES == 64 ? 6 : LANES == 16 ? 4 : 2, lane);
    if (s >= (unsigned)T) return;
    const float *row = logits + (size_t)s * E;
    int e[MOE_MAX_TOPK];
    float dw[MOE_MAX_TOPK], w[MOE_MAX_TOPK];
    float top = -FLT_MAX;
    bool any = false;
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        e[j] = -1, dw[j] = 0.f, w[j] = -INFINITY;
        if (j >= k) continue;
        const int id = idx[(size_t)j * T + s];
        const float d = dweight[(size_t)j * T + s];
        if (id >= 0 && id < E) e[j] = id, dw[j] = d, w[j] = row[id], any = true;
        top = fmaxf(top, w[j]);
    }
    const auto place = [&](int i) { return i / P * P * LANES + lane * P; };     // of the piece that i lies in
    float v[RB_LOGITS], total = 0.f;
    if (!renormalize) {
#pragma unroll
        for (int i = 0; i < RB_LOGITS; i += P) {
            piece_t x = -INFINITY;
            if (place(i) < E) x = *(const piece_t *)(row + place(i));
#pragma unroll
            for (int q = 0; q < P; ++q) {
                if constexpr (P > 1) v[i + q] = x[q];
                else v[i] = x[0];
                top = fmaxf(top, v[i + q]);
            }
        }
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, WAVE));
#pragma unroll
        for (int i = 0; i < RB_LOGITS; ++i) {
            v[i] = place(i) < E ? exp_of<true>(v[i] - top) : 0.f;
            total += v[i];
        }
        total = sum_over<LANES>(total);
    }
    float mean = 0.f;
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        if (j >= k) continue;
        w[j] = e[j] >= 0 ? exp_of<true>(w[j] - top) : 0.f;
        if (renormalize) total += w[j];
    }
    const float share = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        if (j >= k) continue;
        w[j] = e[j] >= 0 ? w[j] * share : 0.f;
        mean = fmaf(w[j], dw[j], mean);
    }
    const float all = renormalize ? 0.f : -mean * share, off = renormalize ? mean : 0.f;
#pragma unroll
    for (int i = 0; i < RB_LOGITS; ++i) v[i] = renormalize || !any ? 0.f : v[i] * all;
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        if (j >= k) break;
        const float more = w[j] * (dw[j] - off);
        const int at = e[j] - lane * P;                  // the place in this lane, if it has it
#pragma unroll
        for (int i = 0; i < RB_LOGITS; ++i) v[i] += at == i / P * P * LANES + i % P ? more : 0.f;
    }
#pragma unroll
    for (int i = 0; i < RB_LOGITS; i += P) {
        if (place(i) >= E) continue;
        piece_t x;
#pragma unroll
        for (int q = 0; q < P; ++q) x[q] = v[i + q];
        *(piece_t *)(dlogits + (size_t)s * E + place(i)) = x;
    }
}

// combine's gradient: log2 of the lanes per row, one piece per lane and trip, a wavefront's at most or a whole workgroup; -1: 32 lanes with
// three pieces each, for one choice (with more, their rows keep a lane's loads in flight) and rows that they hold at once: bf16, 64 lanes and these in
// us, 4096 x 640 5.9 and 5.1, 20000 x 640 22.1 and 18.6, 20000 x 768 27.2 and 25.4, 65536 x 512 52.3 and 51.8, x 768 78.3 and 75.6, fewer tokens
// alike.  Wider rows take them two trips: 4096 x 896 6.7 and 7.1, 65536 x 1024 99.6 and 100.5, 131072 x 1024 196 and 198.
static int combine_backward_lanes(int k, int vec_per_row)
{
    const int lg = row_lanes(vec_per_row);
    if (lg <= 5) return lg;
    return lg > 7 ? 8 : k == 1 && vec_per_row <= 3 * 32 ? -1 : 6;
}
static int dispatch_backward_lanes(int T, int vec_per_row)
{
    const int lg = combine_topk_lanes(T, vec_per_row);
    return lg < 8 ? lg : 8;
}

static int rows_check(const char *who, int T, int k, int d, int dtype)
{
    MOE_REQUIRE(T >= 0 && d > 0 && k >= 1 && k <= MOE_MAX_TOPK, MOE_ERR_INVALID_ARG, "%s: T=%d d=%d k=%d out of range (k <= %d)", who, T, d, k,
                MOE_MAX_TOPK);
    MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
    MOE_REQUIRE((long long)T * k <= INT32_MAX, MOE_ERR_INVALID_ARG, "%s: T=%d tokens of k=%d choices", who, T, k);
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
    const int lg = combine_backward_lanes(k, vec), wide = lg < 0;
#define MOE_CMB_BACK(B)                                               \
    (wide     ? combine_backward_kernel<B, 3, 1>                      \
     : k == 1 ? combine_backward_kernel<B, 1, 1>                      \
     : k <= 4 ? combine_backward_kernel<B, 1, 4>                      \
              : combine_backward_kernel<B, 1, MOE_MAX_TOPK>)
    auto kern = dtype == MOE_BF16 ? MOE_CMB_BACK(true) : MOE_CMB_BACK(false);
#undef MOE_CMB_BACK
    hipLaunchKernelGGL(kern, rows_grid(T, wide ? 5 : lg), dim3(RB_THREADS), 0, (hipStream_t)stream, (const rb_u32x4_t *)dout,
                       (const rb_u32x4_t *)y_perm, inv, expert_weight, T, k, vec, wide ? 5 : lg, residual, (rb_u32x4_t *)dy_perm, dweight,
                       (rb_u32x4_t *)dx);
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
    const int lg = dispatch_backward_lanes(T, vec);
    hipLaunchKernelGGL(kern, rows_grid(T, lg), dim3(RB_THREADS), 0, (hipStream_t)stream, (const rb_u32x4_t *)dx_perm, inv,
                       (const rb_u32x4_t *)dx_add, T, k, vec, lg, (rb_u32x4_t *)dx);
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
    const bool pieces = E % 4 == 0 && aligned16(logits) && aligned16(dlogits);
#define MOE_GATE(L)                                                                                                                            \
    hipLaunchKernelGGL((pieces ? route_backward_kernel<L, true> : route_backward_kernel<L, false>), rows_grid(T, L == 64 ? 6 : L == 16 ? 4 : 2), \
                       dim3(RB_THREADS), 0, (hipStream_t)stream, logits, expert_idx, dweight, T, E, k, renormalize, dlogits)
    if (E <= 4 * RB_LOGITS) MOE_GATE(4);
    else if (E <= 16 * RB_LOGITS) MOE_GATE(16);
    else MOE_GATE(64);
#undef MOE_GATE
    MOE_CHECK_LAUNCH("moe_route_topk_backward");
    return MOE_OK;
}
