// Gated experts over rows sorted by expert, y = (act(x W_gate) * (x W_up)) W_down, and their gradient.
//
// Forward, two launches: g and u = x [W_gate | W_up] and h = act(g) u in one (a workgroup has the same columns of both matrices, so that a lane holds g
// and u of an element), then y = h W_down.  Backward, three: dh = dy W_down^T with dg = dh u act'(g) and du = dh act(g) written as they come, dx = dg
// W_gate^T + du W_up^T as one sum over both, and the weights' gradients x^T [dg | du] and h^T dy, expert by expert over its rows.  dh goes with dW_down
// in one launch and dx with the other two where there is work enough.
//
// Bound by the matrix instructions with many rows of an expert, by the stream of the weights with few, by launches and round trips with one.  A
// training step's 18 d F operations a row are beside the states, 10 F bytes a row (bfloat16) written and read.
//
// h, dg and du are rounded once to the tensors' type, as operands of the products behind them; g and u are kept in binary32 for the gradient (states): a
// second rounding to bfloat16 in the chain would make the gradients' error 1.7 times that of rounding them once, 1.4 times without.
#include "product.h"
#include "scalar_math.h"
#include "gated_ffn_rules.h"

#include <type_traits>

namespace moe {
namespace {

constexpr int MAX_GROUPS = MOE_MAX_EXPERTS;

// ------------------------------------------------------------------------------------------------- activations
// s = 1 / (1 + e^-g) and 1 - s, from an exponential that is at most 1: both keep their relative accuracy, and s reaches 0 (g s would grow again with |g| if it did
// not).
template <bool PRECISE>
__device__ __forceinline__ void sigmoid_of(float g, float &s, float &rest)
{
    const float e = exp_of<PRECISE>(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.f + e), er = e * r;
    s = g < 0.f ? er : r;
    rest = g < 0.f ? r : er;
}

// e^(-g^2 / 2) and the normal distribution's Phi(g).  For bfloat16 results e^(x^2) erfc(x) = t P(t) with t = 1 / (1 + 0.43 x) and a P of degree 7 that was fitted
// for the least relative error on 0 <= x <= 9.6 (behind it the bell is no normal number any more): 8.5e-8, evaluated in binary32 4e-7.
template <bool PRECISE>
__device__ __forceinline__ void normal_of(float g, float &bell, float &phi)
{
    const float x = fabsf(g) * 0.707106781f;
    bell = exp_of<PRECISE>(-0.5f * g * g);
    float tail;                                // erfc(x)
    if (PRECISE) tail = erfcf(x);
    else {
        constexpr float P[8] = {0.242514968f, 0.24436973f, 0.204987422f, 0.246721953f, -0.0854886025f, 0.383441329f, -0.310215741f, 0.0736690089f};
        const float t = __builtin_amdgcn_rcpf(fmaf(0.43f, x, 1.f));
        float v = P[7];
#pragma unroll
        for (int i = 6; i >= 0; --i) v = fmaf(t, v, P[i]);
        tail = t * v * bell;
    }
    phi = g < 0.f ? 0.5f * tail : fmaf(-0.5f, tail, 1.f);
}

template <bool PRECISE>
__device__ __forceinline__ float act_of(int activation, float g)
{
    if (activation == MOE_ACT_SILU) {
        float s, rest;
        sigmoid_of<PRECISE>(g, s, rest);
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
        sigmoid_of<PRECISE>(g, s, rest);
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

struct GatedArgs {
    const void *x, *w_gate, *w_up, *w_down, *dy;
    const int32_t *offset;
    int R, E, d, F, activation;
    void *h, *y, *dgu, *dx, *dw_gate, *dw_up, *dw_down;
    float *gu;
    int parts;                                 // of an expert's rows, whose weight gradients are summed by themselves ...
    float *sums;                               // ... here: [parts] of the three gradients behind each other, if there is more than one
};

// ------------------------------------------------------------------------------------------------- products over rows sorted by expert
enum GatedStep { GATED_HIDDEN, GATED_DOWN, GATED_DHIDDEN, GATED_DX };

// this lane's place in the block of the wavefront's first rows and columns
template <class TILE>
__device__ __forceinline__ float *gated_states(const TILE &tile, const RowTiles &tiles, const Job &j, const GatedArgs &p)
{
    const int row = j.m0 + tile.first_row() - tiles.first(j.group), column = j.n0 + tile.first_column();
    const size_t block = (size_t)(tiles.blocks[j.group] + row / 16) * states_columns(p.F) + column / 16;
    return p.gu + block * GATED_BLOCK + (threadIdx.x & 63) * 4;
}

// STEP's tiles of type TILE: `units` of the parts of n_m x n_n tiles of BIG_M rows x BIG_N columns (of a half), from tile `first` on
// SPLIT: the workgroup's wavefronts have a tile each, of the same place, and share its k; `shared` holds their sums, which the first one adds and writes.
template <int STEP, class TILE, int BIG_M, int BIG_N, int SPLIT = 1>
__device__ __forceinline__ void gated_rows(const GatedArgs &p, const RowTiles &tiles, char *smem, int n_m, int n_n, int first, Units units, int tall,
                                           product_f32x4 *shared = nullptr)
{
    typedef typename TILE::T T;
    constexpr int Z = sizeof(T), PARTS_M = BIG_M / TILE::BM, PARTS_N = BIG_N / TILE::HALF_N, PARTS = PARTS_M * PARTS_N;
    const int N = STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d;
    const unsigned d_bytes = p.d * Z, f_bytes = p.F * Z;
    const unsigned lda = STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? d_bytes : STEP == GATED_DOWN ? f_bytes : 2 * f_bytes;
    const unsigned ldb = STEP == GATED_HIDDEN || STEP == GATED_DX ? f_bytes : d_bytes;
    const TILE tile((product_lds_t *)smem, lda, ldb);
    const bool with_states = p.gu != nullptr;
    tile.template run<SPLIT == 1 ? TILE::MB * Writer<TILE, T>::STORES : 0>(
        [&](Job &j) {
            int u, m, n, lo, hi;
            do {
                if (!units.take(u)) return false;
                product_place(first + u / PARTS, n_m, n_n, tall, m, n);
                j.group = tiles.find(m, lo, hi);
                lo += u % PARTS / PARTS_N * TILE::BM;
                j.n0 = n * BIG_N + u % PARTS_N * TILE::HALF_N;
            } while (PARTS > 1 && (lo >= hi || j.n0 >= N));             // a part behind the last row or column
            j.m0 = lo;
            j.rows = hi - lo < TILE::BM ? hi - lo : TILE::BM;
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
            if constexpr (SPLIT > 1) share_k<TILE, SPLIT>(j, ldb);
            return true;
        },
        [&](const Job &j, typename TILE::Sums &sums) {
            if constexpr (SPLIT > 1)
                if (!join_sums<TILE, SPLIT>(sums, shared)) return;
            if constexpr (STEP == GATED_HIDDEN) {
                const Writer<TILE, T> h(tile, (T *)p.h + (size_t)j.m0 * p.F + j.n0, f_bytes, j.rows, j.columns);
                float *const gu = gated_states(tile, tiles, j, p);
                const size_t row_of_blocks = (size_t)states_columns(p.F) * GATED_BLOCK;
                const int last = states_columns(p.F) - 1 - (j.n0 + tile.first_column()) / 16;      // block of columns from this wavefront's first on
#pragma unroll
                for (int mb = 0; mb < TILE::MB; ++mb) {
                    product_f32x4 v[TILE::NB];
                    const bool there = with_states && tile.first_row() + mb * 16 < j.rows;         // uniform
#pragma unroll
                    for (int nb = 0; nb < TILE::NB; ++nb) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[nb][i] = act_of<Z == 4>(p.activation, sums[0][mb][nb][i]) * sums[1][mb][nb][i];
                        if (there && nb <= last) {
                            float *const at = gu + mb * row_of_blocks + nb * GATED_BLOCK;
                            store4(at, sums[0][mb][nb]);
                            store4(at + 256, sums[1][mb][nb]);
                        }
                    }
                    h.row(mb, v);
                }
            } else if constexpr (STEP == GATED_DHIDDEN) {
                T *const to = (T *)p.dgu + (size_t)j.m0 * 2 * p.F + j.n0;
                const Writer<TILE, T> dg(tile, to, 2 * f_bytes, j.rows, j.columns), du(tile, to + p.F, 2 * f_bytes, j.rows, j.columns);
                const float *const gu = gated_states(tile, tiles, j, p);
                const size_t row_of_blocks = (size_t)states_columns(p.F) * GATED_BLOCK;
                const int last = states_columns(p.F) - 1 - (j.n0 + tile.first_column()) / 16;
                // the states of a row of blocks are asked for a row ahead
                product_f32x4 gate[2][TILE::NB], up[2][TILE::NB];
                auto ask = [&](int mb) {
                    const bool there = tile.first_row() + mb * 16 < j.rows;
#pragma unroll
                    for (int nb = 0; nb < TILE::NB; ++nb) {
                        const product_f32x4 *at = reinterpret_cast<const product_f32x4 *>(there && nb <= last ? gu + mb * row_of_blocks + nb * GATED_BLOCK : p.gu);
                        gate[mb & 1][nb] = at[0];
                        up[mb & 1][nb] = at[64];
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                ask(0);
#pragma unroll
                for (int mb = 0; mb < TILE::MB; ++mb) {
                    if (mb + 1 < TILE::MB) ask(mb + 1);
                    product_f32x4 vg[TILE::NB], vu[TILE::NB];
#pragma unroll
                    for (int nb = 0; nb < TILE::NB; ++nb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float slope;
                            const float v = sums[0][mb][nb][i];
                            vu[nb][i] = v * act_of<Z == 4>(p.activation, gate[mb & 1][nb][i], slope);
                            vg[nb][i] = v * (up[mb & 1][nb][i] * slope);       // behind a shut gate 0, whatever dh u is
                        }
                    dg.row(mb, vg);
                    du.row(mb, vu);
                }
            } else {
                const Writer<TILE, T> to(tile, (T *)(STEP == GATED_DOWN ? p.y : p.dx) + (size_t)j.m0 * p.d + j.n0, d_bytes, j.rows, j.columns);
#pragma unroll
                for (int mb = 0; mb < TILE::MB; ++mb) to.row(mb, sums[0][mb]);
            }
        });
}

// Many rows: tiles of 256 x 256 (hidden: 256 x 128 of both matrices, so that g and u of an element meet in a lane), one workgroup of eight wavefronts to a
// compute unit that goes from tile to tile; binary32 128 x 128, two workgroups.  Bound by the matrix instructions and, in front of them, by the stages' way from
// LDS; hidden beside that by the states that a tile writes at its end.  8192 x 1024 x 4096, one expert: hidden 208 us (0.66 PFLOP/s: of a tile's 50 us the
// products take 26, the states' stores 13, the activation 4.5), down 98 (0.70), dh, which waits for the states at its tiles' ends, 168.
template <int STEP, class SIZES>
__global__ __launch_bounds__(Whole<SIZES>::THREADS, 2) void gated_rows_kernel(GatedArgs p, int tall)
{
    typedef typename Whole<SIZES>::Tile Big;
    __shared__ __align__(1024) char smem[Whole<SIZES>::LDS];
    __shared__ int tables[3][MAX_GROUPS + 1];
    const RowTiles tiles = {tables[0], tables[1], tables[2], p.offset, p.E, p.R, Big::BM};
    tiles.count();
    const int n_m = __builtin_amdgcn_readfirstlane(tiles.prefix[p.E]), n_n = tiles_of(STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d, Big::HALF_N);
    in_rounds<SIZES>(n_m * n_n, [&](auto sized, int first, int past) {
        typedef typename decltype(sized)::Type Part;
        constexpr int parts = Big::BM / Part::BM * (Big::HALF_N / Part::HALF_N);
        gated_rows<STEP, Part, Big::BM, Big::HALF_N>(p, tiles, smem, n_m, n_n, first, Units((past - first) * parts, first > 0), tall);
    });
}

// Tiles of 16 rows x 32 columns or 32 x 64 (hidden: 32 of both matrices), in so few workgroups that a stage's way from memory counts: four wavefronts, each with
// its quarter of k, its own ring and no barrier while it runs.  One row, 768 x 2048: 6.8 and 7.0 us; with the wavefronts beside each other and one ring 9.8 and
// 11.0.  Forward of 60 rows, 768 x 2048, 18 us, in tiles of 64 x 128 34.  Binary32, 958 rows, 32 experts of 512 x 1376: dx 78 us, 35 TFLOP/s.
template <int STEP, class TILE>
__global__ __launch_bounds__(4 * WAVE) void gated_shared_kernel(GatedArgs p)
{
    constexpr int SPLIT = 4;
    __shared__ __align__(1024) char smem[SPLIT * TILE::LDS];
    __shared__ product_f32x4 shared[SHARED_SUMS<TILE, SPLIT>];
    __shared__ int tables[3][MAX_GROUPS + 1];
    const RowTiles tiles = {tables[0], tables[1], tables[2], p.offset, p.E, p.R, TILE::BM};
    tiles.count();
    const int n_m = __builtin_amdgcn_readfirstlane(tiles.prefix[p.E]), n_n = tiles_of(STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d, TILE::HALF_N);
    char *const ring = smem + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * TILE::LDS;
    gated_rows<STEP, TILE, TILE::BM, TILE::HALF_N, SPLIT>(p, tiles, ring, n_m, n_n, 0, Units(n_m * n_n), 8, shared);
}

// Few rows of an expert: tiles of 32 or 64 rows x 128 columns (hidden: 64 of both matrices), several small workgroups to a compute unit, whose rings together
// keep enough of the weights on their way.  Bound by that stream.  768 x 2048: 34 rows of 26 experts 31 and 19 us (5.3 and 4.2 TB/s; of the second
// there are 156 tiles for 256 compute units); 2181 rows of 128 179 and 83 (4.5 and 4.9).  In binary32 the products cost as much: 958 rows, 32 experts of 512 x
// 1376, hidden 58 us, 46 TFLOP/s.
template <int STEP, class TILE>
__global__ __launch_bounds__(TILE::THREADS, 2) void gated_few_rows_kernel(GatedArgs p)
{
    __shared__ __align__(1024) char smem[TILE::LDS];
    __shared__ int tables[3][MAX_GROUPS + 1];
    const RowTiles tiles = {tables[0], tables[1], tables[2], p.offset, p.E, p.R, TILE::BM};
    tiles.count();
    const int n_m = __builtin_amdgcn_readfirstlane(tiles.prefix[p.E]), n_n = tiles_of(STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d, TILE::HALF_N);
    gated_rows<STEP, TILE, TILE::BM, TILE::HALF_N>(p, tiles, smem, n_m, n_n, 0, Units(n_m * n_n), 8);
}

// ------------------------------------------------------------------------------------------------- the weights' gradients
// Experts have different numbers of rows: an XCD's range of units holds an eighth of every expert's tiles.
__host__ __device__ constexpr int gated_weights_share(int tiles) { return (tiles + 7) / 8; }

// DOWN: dW_down = h^T dy, F x d; else dW_gate and dW_up = x^T [dg | du], d x 2F.  An expert without rows gets zeros.
template <bool DOWN, class TILE, int BIG_M, int BIG_N>
__device__ __forceinline__ void gated_weights(const GatedArgs &p, const RowTiles &tiles, char *smem, int n_m, int n_n, int first, Units units, int tall)
{
    typedef typename TILE::T T;
    constexpr int Z = sizeof(T), PARTS_N = BIG_N / TILE::BN, PARTS = BIG_M / TILE::BM * PARTS_N;
    const int M = DOWN ? p.F : p.d, N = DOWN ? p.d : 2 * p.F;
    const unsigned lda = M * Z, ldb = N * Z;
    const TILE tile((product_lds_t *)smem, lda, ldb);
    const int per = gated_weights_share(n_m * n_n);
    tile.template run<TILE::MB * Writer<TILE, T>::STORES>(
        [&](Job &j) {
            int u, m, n, e, t;
            do {
                if (!units.take(u)) return false;
                const int big = first + u / PARTS, groups = p.E * p.parts, xcd = big / (groups * per), in = big - xcd * groups * per;
                e = in / per;
                t = xcd * per + in - e * per;
                if (t >= n_m * n_n) continue;
                j.group = e;
                e /= p.parts;
                product_place(t, n_m, n_n, tall, m, n);
                j.m0 = m * BIG_M + u % PARTS / PARTS_N * TILE::BM;
                j.n0 = n * BIG_N + u % PARTS_N * TILE::BN;
            } while (t >= n_m * n_n || (PARTS > 1 && (j.m0 >= M || j.n0 >= N)));
            int lo = __builtin_amdgcn_readfirstlane(tiles.first(e)), hi = __builtin_amdgcn_readfirstlane(tiles.end(e));
            if (p.parts > 1) {                 // this part's rows
                const int part = (tiles_of(hi - lo, p.parts) + 63) / 64 * 64, from = lo + (j.group - e * p.parts) * part;
                hi = from + part < hi ? from + part : hi;
                lo = from < hi ? from : hi;
            }
            j.rows = M - j.m0 < TILE::BM ? M - j.m0 : TILE::BM;
            j.columns = N - j.n0 < TILE::BN ? N - j.n0 : TILE::BN;
            j.runs = 1;
            j.k = hi - lo;
            j.a[0] = source_across(DOWN ? p.h : p.x, (size_t)lo * lda, lda, j.m0 * Z);
            j.b[0] = source_across(DOWN ? p.dy : p.dgu, (size_t)lo * ldb, ldb, j.n0 * Z);
            return true;
        },
        [&](const Job &j, typename TILE::Sums &sums) {
            const size_t all = (size_t)p.E * p.d * p.F, e = j.group / p.parts, ld = DOWN ? p.d : p.F;
            const size_t at = e * p.d * p.F + j.m0 * ld + j.n0;
            auto write = [&](auto *gate, auto *up, auto *down) {
                typedef std::remove_pointer_t<decltype(gate)> U;
                if (DOWN || j.n0 < p.F) {      // two matrices' columns side by side
                    const Writer<TILE, U> to(tile, (DOWN ? down : gate) + at, ld * sizeof(U), j.rows, DOWN || j.columns < p.F - j.n0 ? j.columns : p.F - j.n0);
#pragma unroll
                    for (int mb = 0; mb < TILE::MB; ++mb) to.row(mb, sums[0][mb]);
                }
                if (!DOWN && j.n0 + j.columns > p.F) {
                    const Writer<TILE, U> to(tile, up + at - p.F, ld * sizeof(U), j.rows, j.columns, p.F - j.n0);
#pragma unroll
                    for (int mb = 0; mb < TILE::MB; ++mb) to.row(mb, sums[0][mb]);
                }
            };
            if (p.parts > 1) {
                float *const part = p.sums + (j.group - e * p.parts) * 3 * all;
                write(part, part + all, part + 2 * all);
            } else write((T *)p.dw_gate, (T *)p.dw_up, (T *)p.dw_down);
        });
}

// Sums over rows: both operands lie across k and are transposed on their way from LDS, k is an expert's rows, of any number.  Bound by the matrix
// instructions with some hundred rows to an expert (8192 x 1024 x 4096: dW_down 122 us, 0.56 PFLOP/s: 64 tiles, as 256 quarters), by writing the gradients
// with few (958 rows, 32 experts of 512 x 1376 in binary32: 72 and 43 us for 180 and 90 MB).
template <bool DOWN, class SIZES>
__global__ __launch_bounds__(Whole<SIZES>::THREADS, 2) void gated_weights_kernel(GatedArgs p, int tall)
{
    typedef typename Whole<SIZES>::Tile Big;
    __shared__ __align__(1024) char smem[Whole<SIZES>::LDS];
    __shared__ int tables[3][MAX_GROUPS + 1];
    const RowTiles tiles = {tables[0], tables[1], tables[2], p.offset, p.E, p.R, Big::BM};
    tiles.count();
    const int n_m = tiles_of(DOWN ? p.F : p.d, Big::BM), n_n = tiles_of(DOWN ? p.d : 2 * p.F, Big::BN);
    in_rounds<SIZES>(8 * p.E * p.parts * gated_weights_share(n_m * n_n), [&](auto sized, int first, int past) {
        typedef typename decltype(sized)::Type Part;
        gated_weights<DOWN, Part, Big::BM, Big::BN>(p, tiles, smem, n_m, n_n, first, Units((past - first) * (Big::BM / Part::BM * (Big::BN / Part::BN)), first > 0), tall);
    });
}

// The parts' sums added in their order, rounded once.
template <class T>
__global__ __launch_bounds__(256) void gated_join_kernel(const float *sums, int parts, size_t all, T *dw_gate, T *dw_up, T *dw_down)
{
    T *const to = blockIdx.y == 0 ? dw_gate : blockIdx.y == 1 ? dw_up : dw_down;
    if (!to) return;
    const float *from = sums + blockIdx.y * all;
    for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; i < all; i += (size_t)gridDim.x * 1024) {
        product_f32x4 v = *reinterpret_cast<const product_f32x4 *>(from + i);
        for (int s = 1; s < parts; ++s) v += *reinterpret_cast<const product_f32x4 *>(from + s * 3 * all + i);
        store4(to + i, v);
    }
}

// ------------------------------------------------------------------------------------------------- both, where there is work for the whole chip
// dh with dW_down, dx with dW_gate and dW_up: two products that need nothing of each other share a launch, so that the last round of one does not leave
// compute units without work, and the tiles that wait for memory (dh's for the states) run beside such as do not.  16 experts of 1024 x 2816, 15747
// rows: 368 and 449 us (0.49 and 0.81 PFLOP/s), as four launches 364 and 525; a step of 8 experts of 2048 x 1408 and 16384 rows 960 us, without the first pair
// 1020, without both 1095; of 64 of 512 x 1376 and 24576 rows 748, 735 and 731: there the
// rule that pairs them loses 2 %.
template <int STEP, class ROWS, class WEIGHTS>
__global__ __launch_bounds__(Whole<ROWS>::THREADS, 2) void gated_pair_kernel(GatedArgs p, int tall)
{
    typedef typename Whole<ROWS>::Tile Rows;
    typedef typename Whole<WEIGHTS>::Tile Weights;
    constexpr bool DOWN = STEP == GATED_DHIDDEN;
    __shared__ __align__(1024) char smem[Rows::LDS > Weights::LDS ? Rows::LDS : Weights::LDS];
    __shared__ int tables[3][MAX_GROUPS + 1];
    const RowTiles tiles = {tables[0], tables[1], tables[2], p.offset, p.E, p.R, Rows::BM};
    tiles.count();
    const int n_m = __builtin_amdgcn_readfirstlane(tiles.prefix[p.E]), n_n = tiles_of(STEP == GATED_DHIDDEN ? p.F : p.d, Rows::HALF_N);
    const int w_m = tiles_of(DOWN ? p.F : p.d, Weights::BM), w_n = tiles_of(DOWN ? p.d : 2 * p.F, Weights::BN), per = gated_weights_share(w_m * w_n);
    // costs in stages: a tile's and what its writes take (dh's with its states)
    const int rows = __builtin_amdgcn_readfirstlane(tiles.end(p.E - 1));
    const int cost_rows = STEP == GATED_DHIDDEN ? p.d / Rows::STAGE_K + 20 : 2 * p.F / Rows::STAGE_K + 4, cost_weights = rows / p.E / Weights::STAGE_K + 5;
    const int slot = blockIdx.x >> 3, slots = gridDim.x >> 3;
    const Shares shares((n_m * n_n + 7) >> 3, cost_rows, p.E * per, cost_weights, slots);
    const bool first = slot < shares.mine;
    if (first) {
        gated_rows<STEP, Rows, Rows::BM, Rows::HALF_N>(p, tiles, smem, n_m, n_n, 0, Units(n_m * n_n, slot, shares.mine, 0, n_m * n_n), tall);
        __syncthreads();                       // the buffers change their sizes
    }
    const int total = 8 * p.E * per;
    gated_weights<DOWN, Weights, Weights::BM, Weights::BN>(
        p, tiles, smem, w_m, w_n, 0, first ? Units(total, slot, shares.mine, shares.rest, total) : Units(total, slot - shares.mine, slots - shares.mine, 0, shares.rest), tall);
}

// ------------------------------------------------------------------------------------------------- host
template <int STEP, class SIZES>
void launch_rows(const GatedArgs &p, hipStream_t st)
{
    typedef typename Whole<SIZES>::Tile Big;
    const int N = STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d;
    const long long units = ((long long)p.R / Big::BM + (p.E < p.R ? p.E : p.R)) * tiles_of(N, Big::HALF_N);
    hipLaunchKernelGGL((gated_rows_kernel<STEP, SIZES>), dim3(product_grid(units, PRODUCT_CUS * SIZES::PER_CU)), dim3(Big::THREADS), 0, st, p, 8);
}
template <int STEP, class TILE>
void launch_few_rows(const GatedArgs &p, hipStream_t st)
{
    const int N = STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d;
    const long long units = ((long long)p.R / TILE::BM + (p.E < p.R ? p.E : p.R)) * tiles_of(N, TILE::HALF_N);
    constexpr int per_cu = 160 * 1024 / (TILE::LDS + 12 * (MAX_GROUPS + 4));
    const long long grid = units < PRODUCT_CUS * per_cu ? units : PRODUCT_CUS * per_cu;
    hipLaunchKernelGGL((gated_few_rows_kernel<STEP, TILE>), dim3((unsigned)((grid + 7) / 8 * 8)), dim3(TILE::THREADS), 0, st, p);
}
template <int STEP, class TILE>
void launch_shared(const GatedArgs &p, hipStream_t st)
{
    const int N = STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d;
    const long long units = ((long long)p.R / TILE::BM + (p.E < p.R ? p.E : p.R)) * tiles_of(N, TILE::HALF_N);
    hipLaunchKernelGGL((gated_shared_kernel<STEP, TILE>), dim3((unsigned)(((units < PRODUCT_CUS ? units : PRODUCT_CUS) + 7) / 8 * 8)), dim3(4 * WAVE), 0, st, p);
}
template <bool DOWN, class SIZES>
void launch_weights(const GatedArgs &p, hipStream_t st)
{
    typedef typename Whole<SIZES>::Tile Big;
    const long long units = (long long)p.E * p.parts * (tiles_of(DOWN ? p.F : p.d, Big::BM) * tiles_of(DOWN ? p.d : 2 * p.F, Big::BN) + 7);
    hipLaunchKernelGGL((gated_weights_kernel<DOWN, SIZES>), dim3(product_grid(units, PRODUCT_CUS * SIZES::PER_CU)), dim3(Big::THREADS), 0, st, p, 8);
}

template <class T, Order B, int HALVES>
struct Few;
template <Order B, int HALVES>
struct Few<bf16_t, B, HALVES> {
    typedef Tile<bf16_t, ALONG_K, B, 64, 64, 2, 2, HALVES, 3> Small;
    typedef Tile<bf16_t, ALONG_K, B, 64, 128, 1, 4, HALVES> Mid;
    typedef Tile<bf16_t, ALONG_K, B, 32, 128, 1, 4, HALVES, 3> Low;
    typedef Tile<bf16_t, ALONG_K, B, 32, 64, 1, 1, HALVES, 2> Shared;
    typedef Tile<bf16_t, ALONG_K, B, 16, 32 * HALVES, 1, 1, HALVES, HALVES == 2 ? 3 : 5> Tiny;
};
template <Order B, int HALVES>
struct Few<float, B, HALVES> {
    typedef Tile<float, ALONG_K, B, 32, 128, 1, 4, HALVES, 3> Mid;
    typedef Mid Low;
    typedef Tile<float, ALONG_K, B, 32, 64, 1, 1, HALVES, 2> Shared;
    typedef Tile<float, ALONG_K, B, 16, 32 * HALVES, 1, 1, HALVES, HALVES == 2 ? 3 : 5> Tiny;
};

template <int STEP, class T>
void launch_step(const GatedArgs &p, hipStream_t st)
{
    constexpr Order B = STEP == GATED_HIDDEN || STEP == GATED_DOWN ? ACROSS_K : ALONG_K;
    constexpr int HALVES = STEP == GATED_HIDDEN ? 2 : 1;
    typedef Few<T, B, HALVES> few;
    const int N = STEP == GATED_HIDDEN || STEP == GATED_DHIDDEN ? p.F : p.d;
    constexpr bool long_sum = STEP == GATED_DOWN || STEP == GATED_DX;          // over F or 2 F, few columns
    switch (gated_rows_rule(p.R, p.E, N, 64 / HALVES, sizeof(T) == 4 ? MOE_F32 : MOE_BF16, long_sum)) {
    case GATED_TINY: launch_shared<STEP, typename few::Tiny>(p, st); break;
    case GATED_SHARED: launch_shared<STEP, typename few::Shared>(p, st); break;
    case GATED_LOW: launch_few_rows<STEP, typename few::Low>(p, st); break;
    case GATED_MID: launch_few_rows<STEP, typename few::Mid>(p, st); break;
    case GATED_SMALL:
        if constexpr (sizeof(T) == 2 && long_sum) {
            launch_few_rows<STEP, typename few::Small>(p, st);
            break;
        }
    default: launch_rows<STEP, Sizes<T, ALONG_K, B, HALVES>>(p, st);
    }
}

template <class T>
void forward(const GatedArgs &p, hipStream_t st)
{
    launch_step<GATED_HIDDEN, T>(p, st);
    launch_step<GATED_DOWN, T>(p, st);
}
template <int STEP, class T>
void launch_pair(const GatedArgs &p, hipStream_t st)
{
    typedef Sizes<T, ALONG_K, ALONG_K> rows;
    typedef Sizes<T, ACROSS_K, ACROSS_K> weights;
    hipLaunchKernelGGL((gated_pair_kernel<STEP, rows, weights>), dim3(PRODUCT_CUS * rows::PER_CU), dim3(Whole<rows>::THREADS), 0, st, p, 8);
}
template <class T>
void backward(const GatedArgs &p, hipStream_t st)
{
    const int dtype = sizeof(T) == 4 ? MOE_F32 : MOE_BF16;
    GatedArgs q = p;
    q.parts = 1;
    // By the sizes alone.  Where only one product of a pair is wanted it has the pair's tiles and parts, so that its sums have the same order.
    typedef Sizes<T, ALONG_K, ALONG_K> rows;
    const bool down = p.R > 0 && gated_pairs(p.R, p.E, p.d, p.F, dtype, true), up = p.R > 0 && gated_pairs(p.R, p.E, p.d, p.F, dtype, false);
    if (p.R > 0) {                             // else zeros for every weight
        if (down && p.dw_down) launch_pair<GATED_DHIDDEN, T>(q, st);
        else if (down) launch_rows<GATED_DHIDDEN, rows>(q, st);
        else launch_step<GATED_DHIDDEN, T>(p, st);
        if (up && p.dx && p.dw_gate) launch_pair<GATED_DX, T>(q, st);
        else if (up && p.dx) launch_rows<GATED_DX, rows>(q, st);
        else if (p.dx) launch_step<GATED_DX, T>(p, st);
    }
    if (p.dw_gate && !(up && p.dx)) launch_weights<false, Sizes<T, ACROSS_K, ACROSS_K>>(up ? q : p, st);
    if (p.dw_down && !down) launch_weights<true, Sizes<T, ACROSS_K, ACROSS_K>>(p, st);
    if (p.parts > 1 && ((p.dw_gate && !up) || (p.dw_down && !down))) {
        const size_t all = (size_t)p.E * p.d * p.F;
        hipLaunchKernelGGL(gated_join_kernel<T>, dim3((unsigned)(all / 1024 < 1024 ? all / 1024 + 1 : 1024), 3), dim3(256), 0, st, p.sums, p.parts, all,
                           up ? nullptr : (T *)p.dw_gate, up ? nullptr : (T *)p.dw_up, down ? nullptr : (T *)p.dw_down);
    }
}

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

extern "C" size_t moe_gated_ffn_states_bytes(int R, int E, int F, int dtype)
{
    return R <= 0 || E <= 0 || F <= 0 ? 0 : hidden_bytes(R, F, dtype) + states_blocks(R, E) * states_columns(F) * GATED_BLOCK * 4;
}

extern "C" size_t moe_gated_ffn_workspace_bytes(int R, int E, int d, int F, int dtype)
{
    return R <= 0 || E <= 0 || d <= 0 || F <= 0 ? 0 : hidden_bytes(R, F, dtype);
}

extern "C" size_t moe_gated_ffn_backward_workspace_bytes(int R, int E, int d, int F, int dtype)
{
    if (R <= 0 || E <= 0 || d <= 0 || F <= 0) return 0;
    const int parts = gated_parts(R, E, d, F, dtype);
    return 2 * hidden_bytes(R, F, dtype) + (parts > 1 ? (size_t)parts * 3 * E * d * F * 4 : 0);
}

extern "C" int moe_gated_ffn(const void *x, const int32_t *expert_offset, const void *w_gate, const void *w_up, const void *w_down, int R, int E, int d,
                             int F, int dtype, int activation, void *y, void *states, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = gated_check("moe_gated_ffn", R, E, d, F, dtype, activation);
    if (rc != MOE_OK || R == 0) return rc;
    MOE_REQUIRE(x && w_gate && w_up && w_down && y && (expert_offset || E == 1), MOE_ERR_INVALID_ARG, "moe_gated_ffn: null pointer");
    MOE_REQUIRE(aligned16(x) && aligned16(w_gate) && aligned16(w_up) && aligned16(w_down) && aligned16(y) && aligned16(states), MOE_ERR_INVALID_ARG,
                "moe_gated_ffn: tensor misaligned");
    const size_t need = states ? 0 : moe_gated_ffn_workspace_bytes(R, E, d, F, dtype);
    MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE, "moe_gated_ffn: workspace of %zu bytes given, %zu needed",
                ws ? ws_bytes : 0, need);
    const size_t z = dtype == MOE_F32 ? 4 : 2, rows = (size_t)R * d * z, weights = (size_t)E * d * F * z;
    const Span spans[] = {{x, rows, false}, {expert_offset, (E + 1) * sizeof(int32_t), false}, {w_gate, weights, false}, {w_up, weights, false},
                          {w_down, weights, false}, {y, rows, true}, {states, moe_gated_ffn_states_bytes(R, E, F, dtype), true}, {states ? nullptr : ws, need, true}};
    MOE_REQUIRE(spans_apart(spans), MOE_ERR_INVALID_ARG, "moe_gated_ffn: an output, the states or the workspace aliases another tensor");
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
    const void *in[] = {dy, x, w_gate, w_up, w_down, states, dx, dw_gate, dw_up, dw_down};
    for (const void *p : in) MOE_REQUIRE(aligned16(p), MOE_ERR_INVALID_ARG, "moe_gated_ffn_backward: tensor misaligned");
    const size_t need = moe_gated_ffn_backward_workspace_bytes(R, E, d, F, dtype);
    MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE,
                "moe_gated_ffn_backward: workspace of %zu bytes given, %zu needed", ws ? ws_bytes : 0, need);
    const size_t z = dtype == MOE_F32 ? 4 : 2, rows = (size_t)R * d * z, weights = (size_t)E * d * F * z;
    const Span spans[] = {{dy, rows, false}, {x, rows, false}, {expert_offset, (E + 1) * sizeof(int32_t), false}, {w_gate, weights, false}, {w_up, weights, false},
                          {w_down, weights, false}, {states, moe_gated_ffn_states_bytes(R, E, F, dtype), false}, {dx, rows, true}, {dw_gate, weights, true},
                          {dw_up, weights, true}, {dw_down, weights, true}, {ws, need, true}};
    MOE_REQUIRE(spans_apart(spans), MOE_ERR_INVALID_ARG, "moe_gated_ffn_backward: an output or the workspace aliases another tensor");
    if (!dw_gate && !dw_down && (!dx || R == 0)) return MOE_OK;        // nothing is wanted
    GatedArgs p = {};
    p.x = x, p.w_gate = w_gate, p.w_up = w_up, p.w_down = w_down, p.dy = dy, p.offset = expert_offset;
    p.R = R, p.E = E, p.d = d, p.F = F, p.activation = activation;
    p.h = const_cast<void *>(states), p.gu = (float *)((char *)const_cast<void *>(states) + hidden_bytes(R, F, dtype));
    p.parts = R > 0 ? gated_parts(R, E, d, F, dtype) : 1;
    p.sums = (float *)((char *)ws + 2 * hidden_bytes(R, F, dtype));
    p.dgu = ws, p.dx = dx, p.dw_gate = dw_gate, p.dw_up = dw_up, p.dw_down = dw_down;
    if (dtype == MOE_BF16) backward<bf16_t>(p, (hipStream_t)stream);
    else backward<float>(p, (hipStream_t)stream);
    MOE_CHECK_LAUNCH("moe_gated_ffn_backward");
    return MOE_OK;
}
