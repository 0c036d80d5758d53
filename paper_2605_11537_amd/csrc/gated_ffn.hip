// Gated experts over rows sorted by expert, y = (act(x W_gate) * (x W_up)) W_down, and their gradient.
//
// Forward, two launches: g and u = x [W_gate | W_up] and h = act(g) u in one (a workgroup has the same columns of both matrices, so that a lane holds g
// and u of an element), then y = h W_down.  Backward, three: dh = dy W_down^T with dg = dh u act'(g) and du = dh act(g) written as they come, dx = dg
// W_gate^T + du W_up^T as one sum over both, and the weights' gradients x^T [dg | du] and h^T dy, expert by expert over its rows.
//
// h, dg and du are rounded once to the tensors' type, as operands of the products behind them; g and u are kept in binary32 for the gradient (states): a
// second rounding to bfloat16 in the chain would make the gradients' error 1.7 times that of rounding them once, 1.4 times without.
#include "product.h"
#include "scalar_math.h"

namespace moe {
namespace {

constexpr int GATED_MAX_WIDTH = 1 << 20;       // byte offsets inside a tile's rows fit 31 bits
constexpr int MAX_GROUPS = MOE_MAX_EXPERTS;

// ------------------------------------------------------------------------------------------------- activations
// e^(-g^2 / 2) and the normal distribution's Phi(g).  For bfloat16 results the rational form of Abramowitz and Stegun, 7.1.26: off by 1.5e-7.
template <bool PRECISE>
__device__ __forceinline__ void normal_of(float g, float &bell, float &phi)
{
    const float x = fabsf(g) * 0.707106781f;
    bell = exp_of<PRECISE>(-0.5f * g * g);
    float tail;                                // erfc(x)
    if (PRECISE) tail = erfcf(x);
    else {
        const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
        tail = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f) * bell;
    }
    phi = g < 0.f ? 0.5f * tail : fmaf(-0.5f, tail, 1.f);
}

template <bool PRECISE>
__device__ __forceinline__ float act_of(int activation, float g)
{
    if (activation == MOE_ACT_SILU) {
        float s, rest;
        gate_of<PRECISE>(g, 0.f, s, rest);
        return g * s;
    }
    if (activation == MOE_ACT_GELU) {
        float bell, phi;
        normal_of<PRECISE>(g, bell, phi);
        return g * phi;
    }
    return g > 0.f ? g : g != g ? g : 0.f;
}

template <bool PRECISE>
__device__ __forceinline__ float act_of(int activation, float g, float &slope)
{
    if (activation == MOE_ACT_SILU) {
        float s, rest;
        gate_of<PRECISE>(g, 0.f, s, rest);
        slope = s * fmaf(g, rest, 1.f);
        return g * s;
    }
    if (activation == MOE_ACT_GELU) {
        float bell, phi;
        normal_of<PRECISE>(g, bell, phi);
        slope = fmaf(g * 0.398942280f, bell, phi);
        return g * phi;
    }
    slope = g > 0.f ? 1.f : g != g ? g : 0.f;
    return g > 0.f ? g : g != g ? g : 0.f;
}

// g and u of four neighbouring columns lie side by side, so that both products' lanes read and write 32 bytes
__device__ __forceinline__ float *states_at(float *gu, size_t row, int F, int column) { return gu + (row * F + column) * 2; }

struct GatedArgs {
    const void *x, *w_gate, *w_up, *w_down, *dy;
    const int32_t *offset;
    int R, E, d, F, activation;
    void *h, *y, *dgu, *dx, *dw_gate, *dw_up, *dw_down;
    float *gu;
};

// ------------------------------------------------------------------------------------------------- products over rows sorted by expert
enum GatedStep { GATED_HIDDEN, GATED_DOWN, GATED_DHIDDEN, GATED_DX };

template <int STEP, class TILE>
__global__ __launch_bounds__(TILE::THREADS, TILE::WAVES / 4) void gated_rows_kernel(GatedArgs p, int tall)
{
    typedef typename TILE::T T;
    constexpr int Z = sizeof(T);
    __shared__ __align__(1024) char smem[TILE::LDS];
    __shared__ int prefix[MAX_GROUPS + 1];
    const RowTiles tiles = {prefix, p.offset, p.E, p.R, TILE::BM};
    tiles.count();
    const int N = STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d;
    const int n_m = __builtin_amdgcn_readfirstlane(prefix[p.E]), n_n = tiles_of(N, TILE::HALF_N);
    const unsigned d_bytes = p.d * Z, f_bytes = p.F * Z;
    const unsigned lda = STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? d_bytes : STEP == GATED_DOWN ? f_bytes : 2 * f_bytes;
    const unsigned ldb = STEP == GATED_HIDDEN || STEP == GATED_DX ? f_bytes : d_bytes;
    const TILE tile((product_lds_t *)smem, lda, ldb);
    const bool with_states = p.gu != nullptr;
    Units units(n_m * n_n);
    tile.run(
        [&](Job &j) {
            int u, m, n, lo, hi;
            if (!units.take(u)) return false;
            product_place(u, n_m, n_n, tall, m, n);
            j.group = tiles.find(m, lo, hi);
            j.m0 = lo;
            j.rows = hi - lo < TILE::BM ? hi - lo : TILE::BM;
            j.n0 = n * TILE::HALF_N;
            j.columns = N - j.n0 < TILE::HALF_N ? N - j.n0 : TILE::HALF_N;
            j.runs = 1;
            const size_t w = (size_t)j.group * p.d * f_bytes;          // the expert's first byte in each of its matrices
            if (STEP == GATED_HIDDEN) {
                j.k = p.d;
                j.a[0] = source_along(p.x, (size_t)lo * d_bytes, d_bytes, j.rows, TILE::BM);
                j.b[0] = source_across(p.w_gate, w, f_bytes, j.n0 * Z);
                j.b[1] = source_across(p.w_up, w, f_bytes, j.n0 * Z);
            } else if (STEP == GATED_DOWN) {
                j.k = p.F;
                j.a[0] = source_along(p.h, (size_t)lo * f_bytes, f_bytes, j.rows, TILE::BM);
                j.b[0] = source_across(p.w_down, w, d_bytes, j.n0 * Z);
            } else if (STEP == GATED_DHIDDEN) {
                j.k = p.d;
                j.a[0] = source_along(p.dy, (size_t)lo * d_bytes, d_bytes, j.rows, TILE::BM);
                j.b[0] = source_along(p.w_down, w + (size_t)j.n0 * d_bytes, d_bytes, j.columns, TILE::HALF_N);
            } else {
                j.k = p.F;
                j.runs = 2;
                j.a[0] = source_along(p.dgu, (size_t)lo * 2 * f_bytes, 2 * f_bytes, j.rows, TILE::BM);
                j.a[1] = j.a[0];
                j.a[1].base += f_bytes;
                j.b[0] = source_along(p.w_gate, w + (size_t)j.n0 * f_bytes, f_bytes, j.columns, TILE::HALF_N);
                j.b[1] = source_along(p.w_up, w + (size_t)j.n0 * f_bytes, f_bytes, j.columns, TILE::HALF_N);
            }
            return true;
        },
        [&](const Job &j, typename TILE::Sums &sums) {
#pragma unroll
            for (int mb = 0; mb < TILE::MB; ++mb) {
                const int row = tile.of_row(mb);
                if (row >= j.rows) continue;
                const size_t r = (size_t)(j.m0 + row);
#pragma unroll
                for (int nb = 0; nb < TILE::NB; ++nb) {
                    const int column = tile.of_column(nb);
                    if (column >= j.columns) continue;
                    const int n = j.n0 + column;
                    const product_f32x4 v = sums[0][mb][nb];
                    if constexpr (STEP == GATED_HIDDEN) {
                        const product_f32x4 up = sums[1][mb][nb];
                        product_f32x4 h;
#pragma unroll
                        for (int i = 0; i < 4; ++i) h[i] = act_of<Z == 4>(p.activation, v[i]) * up[i];
                        store4((T *)p.h + r * p.F + n, h);
                        if (with_states) {
                            float *gu = states_at(p.gu, r, p.F, n);
                            store4(gu, v);
                            store4(gu + 4, up);
                        }
                    } else if constexpr (STEP == GATED_DHIDDEN) {
                        const float *gu = states_at(p.gu, r, p.F, n);
                        const product_f32x4 g = *reinterpret_cast<const product_f32x4 *>(gu), up = *reinterpret_cast<const product_f32x4 *>(gu + 4);
                        product_f32x4 dg, du;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float slope;
                            du[i] = v[i] * act_of<Z == 4>(p.activation, g[i], slope);
                            dg[i] = v[i] * up[i] * slope;
                        }
                        T *to = (T *)p.dgu + r * 2 * p.F + n;
                        store4(to, dg);
                        store4(to + p.F, du);
                    } else store4((T *)(STEP == GATED_DOWN ? p.y : p.dx) + r * p.d + n, v);
                }
            }
        });
}

// ------------------------------------------------------------------------------------------------- the weights' gradients
// DOWN: dW_down = h^T dy, F x d; else dW_gate and dW_up = x^T [dg | du], d x 2F.  An expert without rows gets zeros.
template <bool DOWN, class TILE>
__global__ __launch_bounds__(TILE::THREADS, TILE::WAVES / 4) void gated_weights_kernel(GatedArgs p, int tall)
{
    typedef typename TILE::T T;
    constexpr int Z = sizeof(T);
    __shared__ __align__(1024) char smem[TILE::LDS];
    const RowTiles tiles = {nullptr, p.offset, p.E, p.R, 1};
    const int M = DOWN ? p.F : p.d, N = DOWN ? p.d : 2 * p.F;
    const int n_m = tiles_of(M, TILE::BM), n_n = tiles_of(N, TILE::BN);
    const unsigned lda = M * Z, ldb = N * Z;
    const TILE tile((product_lds_t *)smem, lda, ldb);
    Units units(p.E * n_m * n_n);
    tile.run(
        [&](Job &j) {
            int u, m, n;
            if (!units.take(u)) return false;
            const int e = u / (n_m * n_n);
            product_place(u - e * n_m * n_n, n_m, n_n, tall, m, n);
            const int lo = __builtin_amdgcn_readfirstlane(tiles.first(e)), hi = __builtin_amdgcn_readfirstlane(tiles.end(e, lo));
            j.group = e;
            j.m0 = m * TILE::BM;
            j.n0 = n * TILE::BN;
            j.rows = M - j.m0 < TILE::BM ? M - j.m0 : TILE::BM;
            j.columns = N - j.n0 < TILE::BN ? N - j.n0 : TILE::BN;
            j.runs = 1;
            j.k = hi - lo;
            j.a[0] = source_across(DOWN ? p.h : p.x, (size_t)lo * lda, lda, j.m0 * Z);
            j.b[0] = source_across(DOWN ? p.dy : p.dgu, (size_t)lo * ldb, ldb, j.n0 * Z);
            return true;
        },
        [&](const Job &j, typename TILE::Sums &sums) {
            const size_t w = (size_t)j.group * p.d * p.F;
#pragma unroll
            for (int mb = 0; mb < TILE::MB; ++mb) {
                const int row = tile.of_row(mb);
                if (row >= j.rows) continue;
#pragma unroll
                for (int nb = 0; nb < TILE::NB; ++nb) {
                    const int column = tile.of_column(nb);
                    if (column >= j.columns) continue;
                    const int n = j.n0 + column;
                    T *to;
                    if (DOWN) to = (T *)p.dw_down + w + (size_t)(j.m0 + row) * p.d + n;
                    else to = (T *)(n < p.F ? p.dw_gate : p.dw_up) + w + (size_t)(j.m0 + row) * p.F + (n < p.F ? n : n - p.F);
                    store4(to, sums[0][mb][nb]);
                }
            }
        });
}

// ------------------------------------------------------------------------------------------------- host
template <class TILE>
constexpr int resident() { return 256 * (160 * 1024 / (TILE::LDS + 4 * (MAX_GROUPS + 4))); }

template <int STEP, class TILE>
void launch_rows(const GatedArgs &p, hipStream_t st)
{
    const int N = STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d;
    const long long units = ((long long)p.R / TILE::BM + (p.E < p.R ? p.E : p.R)) * tiles_of(N, TILE::HALF_N);
    hipLaunchKernelGGL((gated_rows_kernel<STEP, TILE>), dim3(product_grid(units, resident<TILE>())), dim3(TILE::THREADS), 0, st, p, 8);
}
template <bool DOWN, class TILE>
void launch_weights(const GatedArgs &p, hipStream_t st)
{
    const int M = DOWN ? p.F : p.d, N = DOWN ? p.d : 2 * p.F;
    const long long units = (long long)p.E * tiles_of(M, TILE::BM) * tiles_of(N, TILE::BN);
    hipLaunchKernelGGL((gated_weights_kernel<DOWN, TILE>), dim3(product_grid(units, resident<TILE>())), dim3(TILE::THREADS), 0, st, p, 8);
}

// rows of an expert for which a tile of so many rows is taken
bool tall_tiles(int R, int E) { return R / E >= 96; }

template <class T>
struct Tiles;
template <>
struct Tiles<bf16_t> {
    template <Order B, int HALVES = 1>
    using Tall = Tile<bf16_t, ALONG_K, B, 256, 256, 2, 4, HALVES>;
    template <Order B, int HALVES = 1>
    using Flat = Tile<bf16_t, ALONG_K, B, 64, 128, 1, 4, HALVES>;
    using Weights = Tile<bf16_t, ACROSS_K, ACROSS_K, 256, 256, 2, 4>;
};
template <>
struct Tiles<float> {
    template <Order B, int HALVES = 1>
    using Tall = Tile<float, ALONG_K, B, 128, 128, 2, 2, HALVES>;
    template <Order B, int HALVES = 1>
    using Flat = Tile<float, ALONG_K, B, 32, 128, 1, 4, HALVES>;
    using Weights = Tile<float, ACROSS_K, ACROSS_K, 128, 128, 2, 2>;
};

template <class T>
void forward(const GatedArgs &p, hipStream_t st)
{
    if (tall_tiles(p.R, p.E)) {
        launch_rows<GATED_HIDDEN, typename Tiles<T>::template Tall<ACROSS_K, 2>>(p, st);
        launch_rows<GATED_DOWN, typename Tiles<T>::template Tall<ACROSS_K>>(p, st);
    } else {
        launch_rows<GATED_HIDDEN, typename Tiles<T>::template Flat<ACROSS_K, 2>>(p, st);
        launch_rows<GATED_DOWN, typename Tiles<T>::template Flat<ACROSS_K>>(p, st);
    }
}
template <class T>
void backward(const GatedArgs &p, hipStream_t st)
{
    if (p.R == 0) {                            // zeros for every weight
    } else if (tall_tiles(p.R, p.E)) {
        launch_rows<GATED_DHIDDEN, typename Tiles<T>::template Tall<ALONG_K>>(p, st);
        if (p.dx) launch_rows<GATED_DX, typename Tiles<T>::template Tall<ALONG_K>>(p, st);
    } else {
        launch_rows<GATED_DHIDDEN, typename Tiles<T>::template Flat<ALONG_K>>(p, st);
        if (p.dx) launch_rows<GATED_DX, typename Tiles<T>::template Flat<ALONG_K>>(p, st);
    }
    if (p.dw_gate) launch_weights<false, typename Tiles<T>::Weights>(p, st);
    if (p.dw_down) launch_weights<true, typename Tiles<T>::Weights>(p, st);
}

size_t hidden_bytes(int R, int F, int dtype) { return align_up((size_t)R * F * (dtype == MOE_F32 ? 4 : 2), 256); }

int gated_check(const char *who, int R, int E, int d, int F, int dtype, int activation)
{
    MOE_REQUIRE(R >= 0 && E > 0 && d > 0 && F > 0, MOE_ERR_INVALID_ARG, "%s: R=%d E=%d d=%d F=%d out of range", who, R, E, d, F);
    MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
    MOE_REQUIRE(activation == MOE_ACT_SILU || activation == MOE_ACT_GELU || activation == MOE_ACT_RELU, MOE_ERR_INVALID_ARG,
                "%s: unknown activation %d", who, activation);
    MOE_REQUIRE(d % 8 == 0 && F % 8 == 0, MOE_ERR_INVALID_ARG, "%s: d=%d and F=%d must be multiples of 8", who, d, F);
    MOE_REQUIRE(E <= MOE_MAX_EXPERTS && d <= GATED_MAX_WIDTH && F <= GATED_MAX_WIDTH / 2, MOE_ERR_UNSUPPORTED, "%s: E=%d d=%d F=%d beyond the kernels",
                who, E, d, F);
    MOE_REQUIRE(((long long)R / 16 + E) * (tiles_of(d, 32) + tiles_of(F, 32)) < 1ll << 30 && (long long)E * tiles_of(d, 32) * tiles_of(F, 32) < 1ll << 30,
                MOE_ERR_UNSUPPORTED, "%s: R=%d E=%d d=%d F=%d: more tiles than an int counts", who, R, E, d, F);
    return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" size_t moe_gated_ffn_states_bytes(int R, int F, int dtype)
{
    return R <= 0 || F <= 0 ? 0 : hidden_bytes(R, F, dtype) + (size_t)R * F * 8;
}

extern "C" size_t moe_gated_ffn_workspace_bytes(int R, int E, int d, int F, int dtype)
{
    (void)E;
    (void)d;
    return R <= 0 || F <= 0 ? 0 : hidden_bytes(R, F, dtype);
}

extern "C" size_t moe_gated_ffn_backward_workspace_bytes(int R, int E, int d, int F, int dtype)
{
    (void)E;
    (void)d;
    return R <= 0 || F <= 0 ? 0 : 2 * hidden_bytes(R, F, dtype);
}

extern "C" int moe_gated_ffn(const void *x, const int32_t *expert_offset, const void *w_gate, const void *w_up, const void *w_down, int R, int E, int d,
                             int F, int dtype, int activation, void *y, void *states, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = gated_check("moe_gated_ffn", R, E, d, F, dtype, activation);
    if (rc != MOE_OK || R == 0) return rc;
    MOE_REQUIRE(x && w_gate && w_up && w_down && y && (expert_offset || E == 1), MOE_ERR_INVALID_ARG, "moe_gated_ffn: null pointer");
    MOE_REQUIRE(y != x && y != w_gate && y != w_up && y != w_down && y != states && states != x, MOE_ERR_INVALID_ARG,
                "moe_gated_ffn: an output aliases another tensor");
    MOE_REQUIRE(aligned16(x) && aligned16(w_gate) && aligned16(w_up) && aligned16(w_down) && aligned16(y) && aligned16(states), MOE_ERR_INVALID_ARG,
                "moe_gated_ffn: tensor misaligned");
    const size_t need = states ? 0 : moe_gated_ffn_workspace_bytes(R, E, d, F, dtype);
    MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE, "moe_gated_ffn: workspace of %zu bytes given, %zu needed",
                ws ? ws_bytes : 0, need);
    GatedArgs p = {};
    p.x = x, p.w_gate = w_gate, p.w_up = w_up, p.w_down = w_down, p.offset = expert_offset;
    p.R = R, p.E = E, p.d = d, p.F = F, p.activation = activation;
    p.h = states ? states : ws, p.y = y;
    p.gu = states ? (float *)((char *)states + hidden_bytes(R, F, dtype)) : nullptr;
    if (dtype == MOE_BF16) forward<bf16_t>(p, (hipStream_t)stream);
    else forward<float>(p, (hipStream_t)stream);
    MOE_CHECK_LAUNCH("moe_gated_ffn");
    return MOE_OK;
}

extern "C" int moe_gated_ffn_backward(const void *dy, const void *x, const int32_t *expert_offset, const void *w_gate, const void *w_up,
                                      const void *w_down, const void *states, int R, int E, int d, int F, int dtype, int activation, void *dx,
                                      void *dw_gate, void *dw_up, void *dw_down, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = gated_check("moe_gated_ffn_backward", R, E, d, F, dtype, activation);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE(!dw_gate == !dw_up, MOE_ERR_INVALID_ARG, "moe_gated_ffn_backward: dw_gate and dw_up come together");
    MOE_REQUIRE((R == 0 || (dy && x && w_gate && w_up && w_down && states)) && (expert_offset || E == 1 || R == 0), MOE_ERR_INVALID_ARG,
                "moe_gated_ffn_backward: null pointer");
    const void *in[] = {dy, x, w_gate, w_up, w_down, states};
    void *out[] = {dx, dw_gate, dw_up, dw_down};
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; out[i] && j < 6; ++j)
            MOE_REQUIRE(out[i] != in[j], MOE_ERR_INVALID_ARG, "moe_gated_ffn_backward: an output aliases another tensor");
        for (int j = 0; out[i] && j < i; ++j)
            MOE_REQUIRE(out[i] != out[j], MOE_ERR_INVALID_ARG, "moe_gated_ffn_backward: an output aliases another tensor");
        MOE_REQUIRE(aligned16(out[i]), MOE_ERR_INVALID_ARG, "moe_gated_ffn_backward: tensor misaligned");
    }
    for (const void *p : in) MOE_REQUIRE(aligned16(p), MOE_ERR_INVALID_ARG, "moe_gated_ffn_backward: tensor misaligned");
    const size_t need = moe_gated_ffn_backward_workspace_bytes(R, E, d, F, dtype);
    MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE,
                "moe_gated_ffn_backward: workspace of %zu bytes given, %zu needed", ws ? ws_bytes : 0, need);
    GatedArgs p = {};
    p.x = x, p.w_gate = w_gate, p.w_up = w_up, p.w_down = w_down, p.dy = dy, p.offset = expert_offset;
    p.R = R, p.E = E, p.d = d, p.F = F, p.activation = activation;
    p.h = const_cast<void *>(states), p.gu = (float *)((char *)const_cast<void *>(states) + hidden_bytes(R, F, dtype));
    p.dgu = ws, p.dx = dx, p.dw_gate = dw_gate, p.dw_up = dw_up, p.dw_down = dw_down;
    if (dtype == MOE_BF16) backward<bf16_t>(p, (hipStream_t)stream);
    else backward<float>(p, (hipStream_t)stream);
    MOE_CHECK_LAUNCH("moe_gated_ffn_backward");
    return MOE_OK;
}
