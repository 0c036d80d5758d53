// Log probabilities of given ids under a head over a large vocabulary, z = h W^T + b, without the logits in memory, and their gradient.
//
// Forward: a workgroup makes a tile of logits in registers and leaves of each of its rows the maximum, the sum of e^(z - maximum) and, where it has
// the target's column, that logit; a second launch joins a row's tiles.  Backward: the logits are made again, piece of the vocabulary by piece, and
// leave as dz = dlogprob ([v = target] - p), from which two products make the rows' part of dh and the piece's rows of dW.
//
// dz is rounded once to the tensors' type, as the operand of those products.  It is divided by the largest |dlogprob| first, and dh and dW are multiplied by
// it in binary32: with the loss a mean all rows have the same dlogprob, which would put the same rounding error on every target's -1.
//
// p = e^(z - lse), but lse = m + log s has been rounded, and beside a large m that takes a part of log s or all of it: 64 ids of -1e9 had p = 1 each.  Where a
// row's |lse| is far from zero the backward call makes all rows' m and s once more (a launch that only prepares the rows where none is) and takes p = e^(z - m) / s,
// so that they add up to one: 8192 x 768 x 50257 2000 us, where rows are far 2620.  The logits are the same bits in all passes: every tile adds an element's k in the
// same order.
#include "product.h"
#include "scalar_math.h"
#include "head_logprobs_rules.h"

namespace moe {
namespace {

constexpr float HEAD_NONE = -__builtin_inff();

struct HeadArgs {
    const void *h, *w;
    const float *b, *lse, *dlogprob;
    const int32_t *target;
    int N, d, V;
    int v0, columns;                           // backward: the piece's first id, its ids
    int *far;                                  // backward: whether a row is far from zero
    float2 *again;                             // a row's maxima and sums made again, [N, n_again]
    int n_again;
    int n_n;                                   // forward: slots of a row
    float2 *tiles;                             // forward [N, n_n]: maximum, sum
    float *at_target;                          // forward [N]
    float *largest;                            // backward: |dlogprob|
    void *clean;                               // backward: h with zeros for the padded rows, or NULL
    bool scan;                                 // backward: every workgroup of the first launch looks at all rows
    void *dz;
    float *db;                                 // backward [slots of a wavefront's rows, V], or NULL
};

__device__ __forceinline__ float finite_or(float m, float other) { return m == HEAD_NONE ? other : m; }

// Whether a row's lse does not hold log s: below the limit half a step of it is 2^-19 (binary32) or 2^-14 (bfloat16, whose dz is rounded by 2^-8) at most.
template <class T>
__device__ __forceinline__ bool far_from_zero(float lse)
{
    return fabsf(lse) >= (sizeof(T) == 4 ? 64.f : 2048.f) && fabsf(lse) < __builtin_inff();
}

// the tile's logits with their bias; columns behind the vocabulary are masked
template <class TILE>
__device__ __forceinline__ void add_bias(const TILE &tile, const Job &j, const float *b, int V, typename TILE::Sums &z)
{
    if (!b && j.columns == TILE::BN) return;
#pragma unroll
    for (int nb = 0; nb < TILE::NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int v = j.n0 + tile.of_column(nb) + i;
            const float bias = v >= V ? HEAD_NONE : b ? b[v] : 0.f;
#pragma unroll
            for (int mb = 0; mb < TILE::MB; ++mb) z[0][mb][nb][i] = v >= V ? HEAD_NONE : z[0][mb][nb][i] + bias;
        }
}

// over the four lane groups that hold a row's columns: rows of 16 lanes, then halves of 32, exchanged among registers
__device__ __forceinline__ float row_max(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float row_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
// e^x for x <= 0 up to some tens, a logit beside its row's maximum or log sum.  Binary32: with the exponent's product taken along.  bfloat16: one rounding, off by
// |x| 2^-24 of an e^x that counts the less the larger |x| is; x 2^-24 e^x is at most 0.4 of that step of lse, and dz is rounded by 2^-8 behind it.
template <class T>
__device__ __forceinline__ float exp_beside(float z, float beside)
{
    return exp_of<sizeof(T) == 4>(z - beside);
}

// where column `in` of a wavefront's is one of this lane's: block, register
template <class TILE>
__device__ __forceinline__ bool holds_column(int in)
{
    return in >= 0 && in < TILE::WAVE_N && ((in >> 2) & 3) == (int)((threadIdx.x & 63) >> 4);
}

// What the backward calls begin with.  Workgroups from `first` on: h with zeros for the padded rows, which may hold anything: what dW's sums are made of.
template <int THREADS>
__device__ __forceinline__ void head_clean(const HeadArgs &p, int pieces, int first)
{
    const uint4 *const h = (const uint4 *)p.h;
    uint4 *const to = (uint4 *)p.clean;
    const size_t total = (size_t)p.N * pieces, step = (size_t)(gridDim.x - first) * THREADS;
    for (size_t i = (size_t)(blockIdx.x - first) * THREADS + threadIdx.x; i < total; i += step) {
        const int id = p.target[i / pieces];
        to[i] = id >= 0 && id < p.V ? h[i] : make_uint4(0, 0, 0, 0);
    }
}
// The first workgroup writes the largest |dlogprob| of a row that counts, 1 where that is 0 or no number, and whether such a row is far from zero.  -> that.
template <class T, int THREADS>
__device__ __forceinline__ bool head_scan(const HeadArgs &p)
{
    __shared__ float waves[THREADS / WAVE];
    float m = 0.f;
    bool any = false;
#pragma unroll 8
    for (int i = threadIdx.x; i < p.N; i += THREADS) {
        const int id = p.target[i];
        const float g = blockIdx.x > 0 ? 0.f : fabsf(p.dlogprob[i]), l = p.lse[i];
        if (id >= 0 && id < p.V) m = fmaxf(m, g), any |= far_from_zero<T>(l);
    }
    any = __syncthreads_or(any);
    if (blockIdx.x > 0) return any;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < THREADS / WAVE; ++w) m = fmaxf(m, waves[w]);
        *p.largest = m > 0.f && m < __builtin_inff() ? m : 1.f;
        *p.far = any;
    }
    return any;
}
// In a launch of its own, where rows are many.
template <class T>
__global__ __launch_bounds__(512) void head_begin_kernel(HeadArgs p)
{
    if (blockIdx.x > 0) head_clean<512>(p, p.d * (int)sizeof(T) / 16, 1);
    else head_scan<T, 512>(p);
}
// By the kernels that make rows again, -> whether they have to.
template <class T, int THREADS>
__device__ __forceinline__ bool head_begin(const HeadArgs &p)
{
    if (!p.scan) return *p.far;
    if (p.clean) head_clean<THREADS>(p, p.d * (int)sizeof(T) / 16, 0);
    return head_scan<T, THREADS>(p);
}

// `units` of the parts of n_m x n_n tiles of BIG_M x BIG_N, from tile `first` on (below likewise); here all have BIG_N columns, for which a row has one slot.
// SPLIT: the workgroup's wavefronts share a tile's k.
template <class TILE, int BIG_M, int BIG_N, int SPLIT = 1>
__device__ __forceinline__ void head_forward(const HeadArgs &p, char *smem, float2 *parts, int n_m, int n_n, int first, Units units, int tall,
                                             product_f32x4 *shared = nullptr)
{
    typedef typename TILE::T T;
    constexpr int WN = TILE::BN / TILE::WAVE_N, PARTS_N = BIG_N / TILE::BN, PARTS = BIG_M / TILE::BM * PARTS_N;
    const unsigned d_bytes = p.d * sizeof(T);
    const TILE tile((product_lds_t *)smem, d_bytes, d_bytes);
    tile.template run<0>(
        [&](Job &j) {
            int u, m, n;
            do {
                if (!units.take(u)) return false;
                product_place(first + u / PARTS, n_m, n_n, tall, m, n);
                j.m0 = m * BIG_M + u % PARTS / PARTS_N * TILE::BM;
                j.n0 = n * BIG_N + u % PARTS_N * TILE::BN;
            } while (PARTS > 1 && (j.m0 >= p.N || j.n0 >= p.V));
            j.rows = p.N - j.m0 < TILE::BM ? p.N - j.m0 : TILE::BM;
            j.columns = p.V - j.n0 < TILE::BN ? p.V - j.n0 : TILE::BN;
            j.k = p.d;
            j.runs = 1;
            j.a[0] = source_along(p.h, (size_t)j.m0 * d_bytes, d_bytes, j.rows, TILE::BM);
            j.b[0] = source_along(p.w, (size_t)j.n0 * d_bytes, d_bytes, j.columns, TILE::BN);
            if constexpr (SPLIT > 1) share_k<TILE, SPLIT>(j, d_bytes);
            return true;
        },
        [&](const Job &j, typename TILE::Sums &z) {
            bool mine = true;
            if constexpr (SPLIT > 1) mine = join_sums<TILE, SPLIT>(z, shared);
            if (mine) add_bias(tile, j, p.b, p.V, z);
            const int lane = threadIdx.x & 63;
            int targets[TILE::MB];
#pragma unroll
            for (int mb = 0; mb < TILE::MB; ++mb) targets[mb] = mine && tile.of_row(mb) < j.rows ? p.target[j.m0 + tile.of_row(mb)] : -1;
            if (mine)
#pragma unroll
            for (int mb = 0; mb < TILE::MB; ++mb) {
                const int row = tile.of_row(mb), target = targets[mb];
                float m = HEAD_NONE;
#pragma unroll
                for (int nb = 0; nb < TILE::NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) m = fmaxf(m, z[0][mb][nb][i]);
                const int in = target - j.n0 - tile.wn * TILE::WAVE_N;
                if (holds_column<TILE>(in) && target < p.V) {
                    float hit = 0.f;
#pragma unroll
                    for (int nb = 0; nb < TILE::NB; ++nb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) hit = in >> 4 == nb && (in & 3) == i ? z[0][mb][nb][i] : hit;
                    p.at_target[j.m0 + row] = hit;
                }
                m = row_max(m);
                const float beside = finite_or(m, 0.f);
                float s = 0.f;
#pragma unroll
                for (int nb = 0; nb < TILE::NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s += exp_beside<T>(z[0][mb][nb][i], beside);
                s = row_sum(s);
                if (lane < 16) parts[tile.wn * TILE::BM + row] = make_float2(m, s);
            }
            __syncthreads();
            for (int row = threadIdx.x; row < j.rows; row += TILE::THREADS) {
                float m = HEAD_NONE, s = 0.f;
#pragma unroll
                for (int w = 0; w < WN; ++w) m = fmaxf(m, parts[w * TILE::BM + row].x);
                const float beside = finite_or(m, 0.f);
#pragma unroll
                for (int w = 0; w < WN; ++w) {
                    const float2 part = parts[w * TILE::BM + row];         // of masked columns alone: a sum of 0, times 1 and not e^-m
                    s += part.y * exp_of<true>(finite_or(part.x, beside) - beside);
                }
                p.tiles[(size_t)(j.m0 + row) * n_n + j.n0 / TILE::BN] = make_float2(m, s);
            }
        });
}

// Bound by the matrix instructions and their stages' way from LDS: 8192 x 768 x 50257 653 us, 0.97 PFLOP/s; the same tiles without
// maxima and exponentials, which have no product beside them, reach 1.15 to 1.2 (k = 1024).  Binary32, 777 x 320 x 5003: 33 us, 75 TFLOP/s.
template <class SIZES, bool AGAIN>
__global__ __launch_bounds__(Whole<SIZES>::THREADS, 2) void head_forward_kernel(HeadArgs p, int tall)
{
    typedef typename Whole<SIZES>::Tile Big;
    __shared__ __align__(1024) char smem[Whole<SIZES>::LDS];
    __shared__ float2 parts[4 * Big::BM];
    if constexpr (AGAIN)
        if (!head_begin<typename Big::T, Big::THREADS>(p)) return;
    const int n_m = tiles_of(p.N, Big::BM), n_n = tiles_of(p.V, Big::BN);
    in_rounds<SIZES>(n_m * n_n, [&](auto sized, int first, int past) {
        static_assert(decltype(sized)::Type::BN == Big::BN, "one slot for a row's columns of a tile");
        typedef typename decltype(sized)::Type Part;
        head_forward<Part, Big::BM, Big::BN>(p, smem, parts, n_m, n_n, first, Units((past - first) * (Big::BM / Part::BM * (Big::BN / Part::BN)), first > 0), tall);
    });
}
// Few rows: bound by the stream of W.  3 x 768 x 131072: 30 us, 6.7 TB/s (a part of W is still in the cache beside the memory).
template <class TILE, bool AGAIN>
__global__ __launch_bounds__(TILE::THREADS, 2) void head_forward_few_kernel(HeadArgs p)
{
    __shared__ __align__(1024) char smem[TILE::LDS];
    __shared__ float2 parts[4 * TILE::BM];
    if constexpr (AGAIN)
        if (!head_begin<typename TILE::T, TILE::THREADS>(p)) return;
    const int n_m = tiles_of(p.N, TILE::BM), n_n = tiles_of(p.V, TILE::BN);
    head_forward<TILE, TILE::BM, TILE::BN>(p, smem, parts, n_m, n_n, 0, Units(n_m * n_n), 8);
}

// As tiles of 16 rows x 32 columns, where these are few (a predictor's head over its experts, a few tokens): four wavefronts share a tile's k, and
// nothing is computed beside 32 ids.  With gradient, us, and in tiles of 64 x 128 or more (both without the 2 us in which rows are looked at): 18 x 2048 x 8 in binary32 40, 177; 60 x 1024 x 2000 in binary32
// 68, 136, in bfloat16 35, 45; 1000 x 256 x 128 34, 38; 4096 x 256 x 8 40, 39.
template <class TILE, bool AGAIN>
__global__ __launch_bounds__(4 * WAVE) void head_forward_tiny_kernel(HeadArgs p)
{
    constexpr int SPLIT = 4;
    __shared__ __align__(1024) char smem[SPLIT * TILE::LDS];
    __shared__ product_f32x4 shared[SHARED_SUMS<TILE, SPLIT>];
    __shared__ float2 parts[TILE::BM];
    if constexpr (AGAIN)
        if (!head_begin<typename TILE::T, 4 * WAVE>(p)) return;
    const int n_m = tiles_of(p.N, TILE::BM), n_n = tiles_of(p.V, TILE::BN);
    char *const ring = smem + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * TILE::LDS;
    head_forward<TILE, TILE::BM, TILE::BN, SPLIT>(p, ring, parts, n_m, n_n, 0, Units(n_m * n_n), 8, shared);
}

// A row's tiles' maxima and sums -> lse and the target's log probability, or with `again` the maximum and the sum.  ROWS rows to a workgroup of four
// wavefronts: one each, or with few rows, whose tiles would be many trips one behind another, all four on one (3 x 131072: 5 us, one wavefront 7.7).
template <int ROWS>
__global__ __launch_bounds__(256) void head_join_kernel(const float2 *tiles, const float *at_target, const int32_t *target, int N, int V, int n_n,
                                                        float *logprob, float *lse, const int *far, float2 *again)
{
    if (far && !*far) return;
    constexpr int LANES = 256 / ROWS;
    const int row = blockIdx.x * ROWS + threadIdx.x / LANES, lane = threadIdx.x & 63;
    if (ROWS > 1 && row >= N) return;
    const float2 *t = tiles + (size_t)row * n_n;
    float m = HEAD_NONE, s = 0.f;
    for (int i = threadIdx.x % LANES; i < n_n; i += LANES) {
        const float2 v = t[i];
        const float both = fmaxf(m, v.x), beside = finite_or(both, 0.f);
        s = s * exp_of<true>(finite_or(m, beside) - beside) + v.y * exp_of<true>(finite_or(v.x, beside) - beside);
        m = both;
    }
    float all = m;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) all = fmaxf(all, __shfl_xor(all, o, 64));
    s *= exp_of<true>(finite_or(m, finite_or(all, 0.f)) - finite_or(all, 0.f));
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
    if (ROWS == 1) {
        __shared__ float2 waves[4];
        if (lane == 0) waves[threadIdx.x >> 6] = make_float2(all, s);
        __syncthreads();
        all = fmaxf(fmaxf(waves[0].x, waves[1].x), fmaxf(waves[2].x, waves[3].x));
        s = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) s += waves[w].y * exp_of<true>(finite_or(waves[w].x, finite_or(all, 0.f)) - finite_or(all, 0.f));
    }
    if (threadIdx.x % LANES == 0) {
        if (again) {
            again[row] = make_float2(all, s);
            return;
        }
        const float beside = finite_or(all, 0.f), l = logf(s);         // -infinity where every id is masked
        lse[row] = beside + l;
        const int id = target[row];
        const bool on = id >= 0 && id < V;
        const float z = on ? at_target[row] : 0.f;
        logprob[row] = !on ? 0.f : z == HEAD_NONE && s == s ? z : (z - beside) - l;
    }
}

// dz lies in blocks of 512 bytes of columns, all rows of one behind all of the last: both products walk it in long runs.  (As a matrix of 50257 columns each
// row of a stage was on a page of its own.)
template <class T>
struct DZ {
    static constexpr int COLUMNS = HEAD_DZ_ROW / (int)sizeof(T);
};

template <class TILE, int BIG_M, int BIG_N, int SPLIT = 1>
__device__ __forceinline__ void head_dlogits(const HeadArgs &p, char *smem, int n_m, int n_n, int first, Units units, int tall,
                                             product_f32x4 *shared = nullptr)
{
    typedef typename TILE::T T;
    constexpr int PARTS_N = BIG_N / TILE::BN, PARTS = BIG_M / TILE::BM * PARTS_N;
    const unsigned d_bytes = p.d * sizeof(T);
    const TILE tile((product_lds_t *)smem, d_bytes, d_bytes);
    const float largest = *p.largest;
    const bool far = *p.far;
    tile.template run<SPLIT == 1 ? TILE::MB * Writer<TILE, T>::STORES : 0>(
        [&](Job &j) {
            int u, m, n;
            do {
                if (!units.take(u)) return false;
                product_place(first + u / PARTS, n_m, n_n, tall, m, n);
                j.m0 = m * BIG_M + u % PARTS / PARTS_N * TILE::BM;
                j.n0 = p.v0 + n * BIG_N + u % PARTS_N * TILE::BN;
            } while (PARTS > 1 && (j.m0 >= p.N || j.n0 >= p.v0 + p.columns));
            j.rows = p.N - j.m0 < TILE::BM ? p.N - j.m0 : TILE::BM;
            const int left = p.v0 + p.columns - j.n0;
            j.columns = left < TILE::BN ? left : TILE::BN;
            j.k = p.d;
            j.runs = 1;
            j.a[0] = source_along(p.h, (size_t)j.m0 * d_bytes, d_bytes, j.rows, TILE::BM);
            j.b[0] = source_along(p.w, (size_t)j.n0 * d_bytes, d_bytes, j.columns, TILE::BN);
            if constexpr (SPLIT > 1) share_k<TILE, SPLIT>(j, d_bytes);
            return true;
        },
        [&](const Job &j, typename TILE::Sums &z) {
            if constexpr (SPLIT > 1)
                if (!join_sums<TILE, SPLIT>(z, shared)) return;
            add_bias(tile, j, p.b, p.V, z);
            const int at = j.n0 - p.v0;        // behind the last id there are zeros up to the tile's end
            const Writer<TILE, T> to(tile, (T *)p.dz + ((size_t)(at / DZ<T>::COLUMNS) * p.N + j.m0) * DZ<T>::COLUMNS + at % DZ<T>::COLUMNS, HEAD_DZ_ROW, j.rows, TILE::BN);
            // what the rows need, asked for at once
            int targets[TILE::MB];
            float weights[TILE::MB], lses[TILE::MB], shares[TILE::MB];
#pragma unroll
            for (int mb = 0; mb < TILE::MB; ++mb) {
                const int row = j.m0 + (tile.of_row(mb) < j.rows ? tile.of_row(mb) : 0);
                targets[mb] = p.target[row];
                weights[mb] = p.dlogprob[row];
                lses[mb] = p.lse[row];
                shares[mb] = 1.f;
            }
            if (far) {                         // uniform
#pragma unroll
                for (int mb = 0; mb < TILE::MB; ++mb) {
                    const float2 *again = p.again + (size_t)(j.m0 + (tile.of_row(mb) < j.rows ? tile.of_row(mb) : 0)) * p.n_again;
                    float m = HEAD_NONE, s = 0.f;          // of a far row finite
                    for (int i = 0; i < p.n_again; ++i) m = fmaxf(m, again[i].x);
                    for (int i = 0; i < p.n_again; ++i) s += again[i].y * exp_of<true>(again[i].x - m);
                    if (far_from_zero<T>(lses[mb])) lses[mb] = m, shares[mb] = 1.f / s;
                }
            }
            product_f32x4 down[TILE::NB];      // sums over this lane's rows
#pragma unroll
            for (int nb = 0; nb < TILE::NB; ++nb) down[nb] = product_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int mb = 0; mb < TILE::MB; ++mb) {
                const int target = tile.of_row(mb) < j.rows ? targets[mb] : -1;
                const bool on = target >= 0 && target < p.V;
                const float g = on ? weights[mb] / largest : 0.f, lse = on ? finite_or(lses[mb], 0.f) : 0.f;
                const float gp = g * shares[mb];
                product_f32x4 dz[TILE::NB];
#pragma unroll
                for (int nb = 0; nb < TILE::NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) dz[nb][i] = on ? -gp * exp_beside<T>(z[0][mb][nb][i], lse) : 0.f;
                const int in = target - j.n0 - tile.wn * TILE::WAVE_N;
                if (on && holds_column<TILE>(in)) {
#pragma unroll
                    for (int nb = 0; nb < TILE::NB; ++nb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) dz[nb][i] += in >> 4 == nb && (in & 3) == i ? g : 0.f;
                }
#pragma unroll
                for (int nb = 0; nb < TILE::NB; ++nb) down[nb] += dz[nb];
                to.row(mb, dz);
            }
            if (p.db) {
#pragma unroll
                for (int nb = 0; nb < TILE::NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float s = sum_over<16>(down[nb][i]);
                        const int v = j.n0 + tile.of_column(nb) + i;
                        // a slot for a wavefront's rows, of which all tiles of the launch have the same number
                        if ((threadIdx.x & 15) == 0 && v < p.V && j.m0 + tile.wm * TILE::WAVE_M < p.N)
                            p.db[(size_t)(j.m0 / TILE::WAVE_M + tile.wm) * p.V + v] = s;
                    }
            }
        });
}

// The forward's product again, and dz of its tile to memory: 8192 x 768 x 50257 727 us, 0.87 PFLOP/s; the exponentials and 800 MB of dz beside the product.
template <class SIZES>
__global__ __launch_bounds__(Whole<SIZES>::THREADS, 2) void head_dlogits_kernel(HeadArgs p, int tall)
{
    typedef typename Whole<SIZES>::Tile Big;
    __shared__ __align__(1024) char smem[Whole<SIZES>::LDS];
    const int n_m = tiles_of(p.N, Big::BM), n_n = tiles_of(p.columns, Big::BN);
    in_rounds<SIZES>(n_m * n_n, [&](auto sized, int first, int past) {
        static_assert(decltype(sized)::Type::WAVE_M == Big::WAVE_M, "one slot for a wavefront's rows");
        typedef typename decltype(sized)::Type Part;
        head_dlogits<Part, Big::BM, Big::BN>(p, smem, n_m, n_n, first, Units((past - first) * (Big::BM / Part::BM * (Big::BN / Part::BN)), first > 0), tall);
    });
}
template <class TILE>
__global__ __launch_bounds__(TILE::THREADS, 2) void head_dlogits_few_kernel(HeadArgs p)
{
    __shared__ __align__(1024) char smem[TILE::LDS];
    const int n_m = tiles_of(p.N, TILE::BM), n_n = tiles_of(p.columns, TILE::BN);
    head_dlogits<TILE, TILE::BM, TILE::BN>(p, smem, n_m, n_n, 0, Units(n_m * n_n), 8);
}
template <class TILE>
__global__ __launch_bounds__(4 * WAVE) void head_dlogits_tiny_kernel(HeadArgs p)
{
    constexpr int SPLIT = 4;
    __shared__ __align__(1024) char smem[SPLIT * TILE::LDS];
    __shared__ product_f32x4 shared[SHARED_SUMS<TILE, SPLIT>];
    const int n_m = tiles_of(p.N, TILE::BM), n_n = tiles_of(p.columns, TILE::BN);
    char *const ring = smem + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * TILE::LDS;
    head_dlogits<TILE, TILE::BM, TILE::BN, SPLIT>(p, ring, n_m, n_n, 0, Units(n_m * n_n), 8, shared);
}

// ------------------------------------------------------------------------------------------------- the two products of the gradient
struct HeadGradArgs {
    const void *dz, *h, *w;
    int N, d, columns, v0;
    int parts, part;                           // dh: k in so many parts of so many columns
    bool add;                                  // dh: behind an earlier piece
    float *dh;                                 // [parts, N, d]
    void *dw;
    int dw_parts, dw_part;                     // dW: rows in so many parts of so many; with more than one their sums go to
    float *dw_sums;                            // [dw_parts, columns, d]
    const float *largest;
};

template <class TILE, int BIG_M, int BIG_N>
__device__ __forceinline__ void head_dh(const HeadGradArgs &p, char *smem, int n_m, int n_n, int first, Units units, int tall)
{
    typedef typename TILE::T T;
    constexpr int Z = sizeof(T), PARTS_N = BIG_N / TILE::BN, PARTS = BIG_M / TILE::BM * PARTS_N;
    const unsigned lda = HEAD_DZ_ROW, ldb = p.d * Z;
    const TILE tile((product_lds_t *)smem, lda, ldb);
    tile.template run<TILE::MB * Writer<TILE, float>::STORES>(
        [&](Job &j) {
            int u, m, n;
            do {
                if (!units.take(u)) return false;
                const int big = first + u / PARTS;
                j.group = big / (n_m * n_n);
                product_place(big - j.group * n_m * n_n, n_m, n_n, tall, m, n);
                j.m0 = m * BIG_M + u % PARTS / PARTS_N * TILE::BM;
                j.n0 = n * BIG_N + u % PARTS_N * TILE::BN;
            } while (PARTS > 1 && (j.m0 >= p.N || j.n0 >= p.d));
            const int k0 = j.group * p.part;
            j.rows = p.N - j.m0 < TILE::BM ? p.N - j.m0 : TILE::BM;
            j.columns = p.d - j.n0 < TILE::BN ? p.d - j.n0 : TILE::BN;
            j.runs = 1;
            j.k = p.columns - k0 < p.part ? (p.columns - k0 > 0 ? p.columns - k0 : 0) : p.part;
            j.block = (size_t)p.N * HEAD_DZ_ROW;
            j.a[0] = source_along(p.dz, k0 / DZ<T>::COLUMNS * j.block + (size_t)j.m0 * lda, lda, j.rows, TILE::BM);
            j.b[0] = source_across(p.w, (size_t)(p.v0 + k0) * ldb, ldb, j.n0 * Z);
            return true;
        },
        [&](const Job &j, typename TILE::Sums &sums) {
            float *const first = p.dh + ((size_t)j.group * p.N + j.m0) * p.d + j.n0;
            const Writer<TILE, float> to(tile, first, p.d * 4, j.rows, j.columns);
#pragma unroll
            for (int mb = 0; mb < TILE::MB; ++mb) {
                if (p.add) {                   // uniform
                    const int row = tile.of_row(mb);
#pragma unroll
                    for (int nb = 0; nb < TILE::NB; ++nb)
                        if (row < j.rows && tile.of_column(nb) < j.columns)
                            sums[0][mb][nb] += *reinterpret_cast<const product_f32x4 *>(first + (size_t)row * p.d + tile.of_column(nb));
                }
                to.row(mb, sums[0][mb]);
            }
        });
}

// dh = dz W, k the piece's ids in parts, whose sums go to memory in binary32.  Alone at 8192 x 768 x 50257 607 us (1.04 PFLOP/s); 777 x 320 x 5003 in binary32 48 (52
// TFLOP/s: reads of 4 bytes bring W across k into lanes).
template <class SIZES>
__global__ __launch_bounds__(Whole<SIZES>::THREADS, 2) void head_dh_kernel(HeadGradArgs p, int tall)
{
    typedef typename Whole<SIZES>::Tile Big;
    __shared__ __align__(1024) char smem[Whole<SIZES>::LDS];
    const int n_m = tiles_of(p.N, Big::BM), n_n = tiles_of(p.d, Big::BN);
    in_rounds<SIZES>(p.parts * n_m * n_n, [&](auto sized, int first, int past) {
        typedef typename decltype(sized)::Type Part;
        head_dh<Part, Big::BM, Big::BN>(p, smem, n_m, n_n, first, Units((past - first) * (Big::BM / Part::BM * (Big::BN / Part::BN)), first > 0), tall);
    });
}
template <class TILE>
__global__ __launch_bounds__(TILE::THREADS, 2) void head_dh_few_kernel(HeadGradArgs p)
{
    __shared__ __align__(1024) char smem[TILE::LDS];
    const int n_m = tiles_of(p.N, TILE::BM), n_n = tiles_of(p.d, TILE::BN);
    head_dh<TILE, TILE::BM, TILE::BN>(p, smem, n_m, n_n, 0, Units(p.parts * n_m * n_n), 8);
}

template <class TILE, int BIG_M, int BIG_N>
__device__ __forceinline__ void head_dw(const HeadGradArgs &p, char *smem, int n_m, int n_n, int first, Units units, int tall)
{
    typedef typename TILE::T T;
    constexpr int Z = sizeof(T), PARTS_N = BIG_N / TILE::BN, PARTS = BIG_M / TILE::BM * PARTS_N;
    const unsigned lda = HEAD_DZ_ROW, ldb = p.d * Z;
    const TILE tile((product_lds_t *)smem, lda, ldb);
    const float largest = *p.largest;
    tile.template run<TILE::MB * Writer<TILE, T>::STORES>(
        [&](Job &j) {
            int u, m, n;
            do {
                if (!units.take(u)) return false;
                const int big = first + u / PARTS;
                j.group = big / (n_m * n_n);
                product_place(big - j.group * n_m * n_n, n_m, n_n, tall, m, n);
                j.m0 = m * BIG_M + u % PARTS / PARTS_N * TILE::BM;
                j.n0 = n * BIG_N + u % PARTS_N * TILE::BN;
            } while (PARTS > 1 && (j.m0 >= p.columns || j.n0 >= p.d));
            const int k0 = j.group * p.dw_part;
            j.rows = p.columns - j.m0 < TILE::BM ? p.columns - j.m0 : TILE::BM;
            j.columns = p.d - j.n0 < TILE::BN ? p.d - j.n0 : TILE::BN;
            j.runs = 1;
            j.k = p.N - k0 < p.dw_part ? (p.N - k0 > 0 ? p.N - k0 : 0) : p.dw_part;
            j.a[0] = source_across(p.dz, ((size_t)(j.m0 / DZ<T>::COLUMNS) * p.N + k0) * HEAD_DZ_ROW, lda, j.m0 % DZ<T>::COLUMNS * Z);
            j.b[0] = source_across(p.h, (size_t)k0 * ldb, ldb, j.n0 * Z);
            return true;
        },
        [&](const Job &j, typename TILE::Sums &sums) {
            if (p.dw_parts > 1) {
                const Writer<TILE, float> to(tile, p.dw_sums + ((size_t)j.group * p.columns + j.m0) * p.d + j.n0, p.d * 4, j.rows, j.columns);
#pragma unroll
                for (int mb = 0; mb < TILE::MB; ++mb) to.row(mb, sums[0][mb]);
                return;
            }
            const Writer<TILE, T> to(tile, (T *)p.dw + (size_t)(p.v0 + j.m0) * p.d + j.n0, p.d * Z, j.rows, j.columns);
#pragma unroll
            for (int mb = 0; mb < TILE::MB; ++mb) {
#pragma unroll
                for (int nb = 0; nb < TILE::NB; ++nb) sums[0][mb][nb] *= largest;
                to.row(mb, sums[0][mb]);
            }
        });
}

// dW = dz^T h, k the rows; where tiles are few and rows many, in parts.  Alone at 8192 x 768 x 50257 619 us (1.02 PFLOP/s); 777 x 320 x 5003 in binary32 36.
template <class SIZES>
__global__ __launch_bounds__(Whole<SIZES>::THREADS, 2) void head_dw_kernel(HeadGradArgs p, int tall)
{
    typedef typename Whole<SIZES>::Tile Big;
    __shared__ __align__(1024) char smem[Whole<SIZES>::LDS];
    const int n_m = tiles_of(p.columns, Big::BM), n_n = tiles_of(p.d, Big::BN);
    in_rounds<SIZES>(p.dw_parts * n_m * n_n, [&](auto sized, int first, int past) {
        typedef typename decltype(sized)::Type Part;
        head_dw<Part, Big::BM, Big::BN>(p, smem, n_m, n_n, first, Units((past - first) * (Big::BM / Part::BM * (Big::BN / Part::BN)), first > 0), tall);
    });
}

// Both, where there is work for the whole chip: they need nothing of each other, and the last round of one leaves no compute units without work.
// 8192 x 768 x 50257: 1195 to 1240 us (1.04 PFLOP/s), one after the other 1226 and 8 more for the parts of dh, which are more then.
template <class DH, class DW>
__global__ __launch_bounds__(Whole<DH>::THREADS, 2) void head_pair_kernel(HeadGradArgs p, int tall)
{
    typedef typename Whole<DH>::Tile Dh;
    typedef typename Whole<DW>::Tile Dw;
    __shared__ __align__(1024) char smem[Dh::LDS > Dw::LDS ? Dh::LDS : Dw::LDS];
    const int h_m = tiles_of(p.N, Dh::BM), h_n = tiles_of(p.d, Dh::BN), w_m = tiles_of(p.columns, Dw::BM), w_n = tiles_of(p.d, Dw::BN);
    const int n1 = w_m * w_n, n2 = p.parts * h_m * h_n;
    const int slot = blockIdx.x >> 3, slots = gridDim.x >> 3;
    const Shares shares((n1 + 7) >> 3, p.N / Dw::STAGE_K + 4, (n2 + 7) >> 3, p.part / Dh::STAGE_K + 6, slots);
    const bool first = slot < shares.mine;
    if (first) {
        head_dw<Dw, Dw::BM, Dw::BN>(p, smem, w_m, w_n, 0, Units(n1, slot, shares.mine, 0, n1), tall);
        __syncthreads();                       // the buffers change their sizes
    }
    head_dh<Dh, Dh::BM, Dh::BN>(p, smem, h_m, h_n, 0,
                                first ? Units(n2, slot, shares.mine, shares.rest, n2) : Units(n2, slot - shares.mine, slots - shares.mine, 0, shares.rest), tall);
}

// ------------------------------------------------------------------------------------------------- rows
// What they end with: the parts' sums, in their order, times the largest |dlogprob|.  Workgroups 0 .. dh_blocks-1 dh, then dW (a single piece's, in parts), then
// db.
template <class T>
__global__ __launch_bounds__(256) void head_end_kernel(HeadGradArgs p, const int32_t *target, int V, T *dh, int dh_blocks, int dw_blocks, const float *db_sums,
                                                       int db_parts, float *db)
{
    const float scale = *p.largest;
    int block = blockIdx.x;
    if (block < dh_blocks) {
        const size_t total = (size_t)p.N * p.d;
        for (size_t i = ((size_t)block * 256 + threadIdx.x) * 4; i < total; i += (size_t)dh_blocks * 1024) {
            const int id = target[i / p.d];
            product_f32x4 v = {0.f, 0.f, 0.f, 0.f};
            if (id >= 0 && id < V)
                for (int s = 0; s < p.parts; ++s) v += *reinterpret_cast<const product_f32x4 *>(p.dh + s * total + i);
            store4(dh + i, v * scale);
        }
        return;
    }
    block -= dh_blocks;
    if (block < dw_blocks) {
        const size_t total = (size_t)p.columns * p.d;
        for (size_t i = ((size_t)block * 256 + threadIdx.x) * 4; i < total; i += (size_t)dw_blocks * 1024) {
            product_f32x4 v = {0.f, 0.f, 0.f, 0.f};
            for (int s = 0; s < p.dw_parts; ++s) v += *reinterpret_cast<const product_f32x4 *>(p.dw_sums + s * total + i);
            store4((T *)p.dw + (size_t)p.v0 * p.d + i, v * scale);
        }
        return;
    }
    const int v = (block - dw_blocks) * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;      // four wavefronts share a column's parts
    __shared__ double quarter[4][64];
    double s = 0.;
    for (int i = w; v < V && i < db_parts; i += 4) s += db_sums[(size_t)i * V + v];
    quarter[w][threadIdx.x & 63] = s;
    __syncthreads();
    if (w == 0 && v < V) db[v] = (float)((((quarter[0][threadIdx.x] + quarter[1][threadIdx.x]) + quarter[2][threadIdx.x]) + quarter[3][threadIdx.x]) * scale);
}

__global__ __launch_bounds__(256) void head_clear_kernel(unsigned *p, size_t words)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (size_t)gridDim.x * 256) p[i] = 0;
}

// ------------------------------------------------------------------------------------------------- host
void launch_clear(void *p, size_t bytes, hipStream_t st)
{
    const size_t words = bytes / 4;            // rows are multiples of 16 bytes
    hipLaunchKernelGGL(head_clear_kernel, dim3((unsigned)(words / 256 < 2048 ? words / 256 + 1 : 2048)), dim3(256), 0, st, (unsigned *)p, words);
}

// tiles of 64, 32 (binary32 only) and 16 rows
template <class T, Order A, Order B>
using Flat = Tile<T, A, B, 64, HEAD_FEW_COLUMNS, 1, 4, 1, 2, A == ALONG_K && B == ACROSS_K ? DZ<T>::COLUMNS : 0>;
template <class T, Order A, Order B>
using Low = Tile<T, A, B, sizeof(T) == 4 ? 32 : 64, HEAD_FEW_COLUMNS, 1, 4, 1, 2, A == ALONG_K && B == ACROSS_K ? DZ<T>::COLUMNS : 0>;
template <class T, Order A, Order B>
using Few = Tile<T, A, B, 16, HEAD_FEW_COLUMNS, 1, 4, 1, 2, A == ALONG_K && B == ACROSS_K ? DZ<T>::COLUMNS : 0>;

// parts of a tile with all of its columns, and with all of its rows
template <class T>
struct RowParts;
template <>
struct RowParts<bf16_t> : Sizes<bf16_t, ALONG_K, ALONG_K> {
    typedef Sized<Tile<bf16_t, ALONG_K, ALONG_K, 64, 256, 2, 4, 1, 3>> Quarter;
    typedef Sized<Tile<bf16_t, ALONG_K, ALONG_K, 32, 256, 2, 4, 1, 4>> Eighth;
    typedef Eighth Sixteenth;
};
template <>
struct RowParts<float> : Sizes<float, ALONG_K, ALONG_K> {
    typedef Sized<Tile<float, ALONG_K, ALONG_K, 32, 128, 2, 2, 1, 3>> Quarter;
    typedef Sized<Tile<float, ALONG_K, ALONG_K, 16, 128, 1, 4, 1, 3>> Eighth;
    typedef Eighth Sixteenth;
};
template <class T>
struct ColumnParts;
template <>
struct ColumnParts<bf16_t> : Sizes<bf16_t, ALONG_K, ALONG_K> {
    typedef Sized<Tile<bf16_t, ALONG_K, ALONG_K, 256, 128, 2, 4, 1, 3>> Half;
    typedef Sized<Tile<bf16_t, ALONG_K, ALONG_K, 256, 64, 2, 4, 1, 3>> Quarter;
    typedef Quarter Eighth;
    typedef Quarter Sixteenth;
};
template <>
struct ColumnParts<float> : Sizes<float, ALONG_K, ALONG_K> {
    typedef Sized<Tile<float, ALONG_K, ALONG_K, 128, 64, 2, 2, 1, 3>> Half;
    typedef Sized<Tile<float, ALONG_K, ALONG_K, 128, 32, 2, 2, 1, 3>> Quarter;
    typedef Quarter Eighth;
    typedef Quarter Sixteenth;
};
// dh: A in dz's blocks
template <class T>
struct DhParts;
template <>
struct DhParts<bf16_t> {
    typedef Sized<Tile<bf16_t, ALONG_K, ACROSS_K, 256, 256, 2, 4, 1, 2, DZ<bf16_t>::COLUMNS>> Whole;
    typedef Sized<Tile<bf16_t, ALONG_K, ACROSS_K, 128, 256, 2, 4, 1, 3, DZ<bf16_t>::COLUMNS>> Half;
    typedef Sized<Tile<bf16_t, ALONG_K, ACROSS_K, 128, 128, 2, 4, 1, 4, DZ<bf16_t>::COLUMNS>> Quarter;
    typedef Sized<Tile<bf16_t, ALONG_K, ACROSS_K, 128, 64, 4, 2, 1, 6, DZ<bf16_t>::COLUMNS>> Eighth;
    typedef Sized<Tile<bf16_t, ALONG_K, ACROSS_K, 64, 64, 4, 2, 1, 8, DZ<bf16_t>::COLUMNS>> Sixteenth;
    static constexpr int PER_CU = 1;
};
template <>
struct DhParts<float> {
    typedef Sized<Tile<float, ALONG_K, ACROSS_K, 128, 128, 2, 2, 1, 2, DZ<float>::COLUMNS>> Whole;
    typedef Sized<Tile<float, ALONG_K, ACROSS_K, 64, 128, 2, 2, 1, 3, DZ<float>::COLUMNS>> Half;
    typedef Sized<Tile<float, ALONG_K, ACROSS_K, 64, 64, 2, 2, 1, 4, DZ<float>::COLUMNS>> Quarter;
    typedef Sized<Tile<float, ALONG_K, ACROSS_K, 32, 64, 2, 2, 1, 6, DZ<float>::COLUMNS>> Eighth;
    typedef Eighth Sixteenth;
    static constexpr int PER_CU = 2;
};

template <class TILE>
dim3 few_grid(long long units, int more_lds)
{
    const long long most = PRODUCT_CUS * (160 * 1024 / (TILE::LDS + more_lds));
    return dim3((unsigned)(((units < most ? units : most) + 7) / 8 * 8));
}

// KERNEL for tiles of PARTS' sizes, or KERNEL_few for tiles of 64, 32 or 16 rows, by the number of rows; M, N, TIMES: D and how often; further template arguments
#define HEAD_BY_ROWS(KERNEL, PARTS, A, B, ARGS, ST, M, N, TIMES, LDS_ROWS, ...)                                                                       \
    do {                                                                                                                                       \
        typedef PARTS<T> sizes;                                                                                                                \
        typedef typename Whole<sizes>::Tile big;                                                                                               \
        typedef Flat<T, A, B> flat;                                                                                                            \
        typedef Low<T, A, B> low;                                                                                                              \
        typedef Few<T, A, B> few;                                                                                                              \
        const HeadRows rows = head_rows(M, sizeof(T) == 4 ? MOE_F32 : MOE_BF16);                                                               \
        if (rows == HEAD_TALL_TILES)                                                                                                           \
            hipLaunchKernelGGL((KERNEL##_kernel<sizes, ##__VA_ARGS__>),                                                                        \
                               dim3(product_grid((long long)TIMES * tiles_of(M, big::BM) * tiles_of(N, big::BN), PRODUCT_CUS * sizes::PER_CU)), \
                               dim3(big::THREADS), 0, ST, ARGS, 8);                                                                            \
        else if (rows == HEAD_FLAT_TILES)                                                                                                      \
            hipLaunchKernelGGL((KERNEL##_few_kernel<flat, ##__VA_ARGS__>),                                                                     \
                               few_grid<flat>((long long)TIMES * tiles_of(M, flat::BM) * tiles_of(N, flat::BN), LDS_ROWS * flat::BM),          \
                               dim3(flat::THREADS), 0, ST, ARGS);                                                                              \
        else if (rows == HEAD_LOW_TILES)                                                                                                       \
            hipLaunchKernelGGL((KERNEL##_few_kernel<low, ##__VA_ARGS__>),                                                                      \
                               few_grid<low>((long long)TIMES * tiles_of(M, low::BM) * tiles_of(N, low::BN), LDS_ROWS * low::BM),             \
                               dim3(low::THREADS), 0, ST, ARGS);                                                                              \
        else                                                                                                                                   \
            hipLaunchKernelGGL((KERNEL##_few_kernel<few, ##__VA_ARGS__>),                                                                      \
                               few_grid<few>((long long)TIMES * tiles_of(M, few::BM) * tiles_of(N, few::BN), LDS_ROWS * few::BM),              \
                               dim3(few::THREADS), 0, ST, ARGS);                                                                               \
    } while (0)

// p.tiles, p.at_target -> logprob and lse; AGAIN: what the backward calls begin with, and p.again where a row is far from zero
template <class T, bool AGAIN>
void forward(const HeadArgs &p, float *logprob, float *lse, hipStream_t st)
{
    const int N = p.N;
    typedef Tile<T, ALONG_K, ALONG_K, HEAD_TINY_ROWS, HEAD_TINY_COLUMNS, 1, 1, 1, 5> tiny;
    if (head_tiny(N, p.V))
        hipLaunchKernelGGL((head_forward_tiny_kernel<tiny, AGAIN>), few_grid<tiny>((long long)tiles_of(N, tiny::BM) * tiles_of(p.V, tiny::BN), 3 * tiny::LDS),
                           dim3(4 * WAVE), 0, st, p);
    else HEAD_BY_ROWS(head_forward, RowParts, ALONG_K, ALONG_K, p, st, N, p.V, 1, 32, AGAIN);
    if (AGAIN && p.tiles == p.again) return;   // who needs them joins them
    if (N <= 512 && p.n_n > 64)
        hipLaunchKernelGGL(head_join_kernel<1>, dim3(N), dim3(256), 0, st, p.tiles, p.at_target, p.target, N, p.V, p.n_n, logprob, lse, p.far, p.again);
    else
        hipLaunchKernelGGL(head_join_kernel<4>, dim3(tiles_of(N, 4)), dim3(256), 0, st, p.tiles, p.at_target, p.target, N, p.V, p.n_n, logprob, lse, p.far, p.again);
}

template <class T>
void backward(HeadArgs p, const HeadShape &g, char *ws, T *dh, T *dw, float *db, hipStream_t st)
{
    const int N = p.N;
    float *const dh_parts = (float *)(ws + g.dh_at), *const db_parts = (float *)(ws + g.db_at);
    p.largest = (float *)ws;
    p.far = (int *)ws + 1;
    p.clean = dw ? ws + g.rows_at : nullptr;
    p.scan = N <= HEAD_SCAN_ROWS;
    p.again = (float2 *)(ws + g.again_at);
    p.n_again = g.n_again;
    p.n_n = head_row_slots(N, p.V, sizeof(T) == 4 ? MOE_F32 : MOE_BF16);
    p.at_target = (float *)(ws + g.dz_at);
    p.tiles = p.n_again == p.n_n ? p.again : (float2 *)(ws + g.dz_at + head_targets_bytes(N));
    p.dz = ws + g.dz_at;
    p.db = db ? db_parts : nullptr;
    auto blocks_for = [](size_t work, size_t each) { return (int)(work / each < 2048 ? work / each + 1 : 2048); };
    if (!p.scan) hipLaunchKernelGGL(head_begin_kernel<T>, dim3(1 + (dw ? blocks_for((size_t)N * p.d * sizeof(T) / 16, 512) : 0)), dim3(512), 0, st, p);
    forward<T, true>(p, nullptr, nullptr, st);
    HeadGradArgs q = {};
    for (int v0 = 0; v0 < p.V; v0 += g.piece) {
        p.v0 = v0;
        p.columns = p.V - v0 < g.piece ? p.V - v0 : g.piece;
        typedef Tile<T, ALONG_K, ALONG_K, HEAD_TINY_ROWS, HEAD_TINY_COLUMNS, 1, 1, 1, 5> tiny;
        if (head_tiny(N, p.V)) hipLaunchKernelGGL(head_dlogits_tiny_kernel<tiny>, few_grid<tiny>((long long)tiles_of(N, tiny::BM) * tiles_of(p.V, tiny::BN), 3 * tiny::LDS), dim3(4 * WAVE), 0, st, p);
        else HEAD_BY_ROWS(head_dlogits, ColumnParts, ALONG_K, ALONG_K, p, st, N, p.columns, 1, 0);
        q.dz = p.dz, q.h = ws + g.rows_at, q.w = p.w, q.N = N, q.d = p.d, q.columns = p.columns, q.v0 = v0;
        q.parts = g.parts, q.part = (int)align_up(tiles_of(p.columns, g.parts), DZ<T>::COLUMNS), q.add = v0 > 0;
        q.dh = dh_parts, q.dw = dw, q.largest = p.largest;
        q.dw_parts = g.dw_parts, q.dw_part = (int)align_up(tiles_of(N, g.dw_parts), 64), q.dw_sums = (float *)(ws + g.dw_at);
        if (dh && dw && g.paired) {
            typedef DhParts<T> sizes;
            hipLaunchKernelGGL((head_pair_kernel<sizes, Sizes<T, ACROSS_K, ACROSS_K>>), dim3(PRODUCT_CUS * sizes::PER_CU),
                               dim3(Whole<sizes>::THREADS), 0, st, q, 8);
            continue;
        }
        if (dh) HEAD_BY_ROWS(head_dh, DhParts, ALONG_K, ACROSS_K, q, st, N, p.d, g.parts, 0);
        if (dw) {
            typedef Sizes<T, ACROSS_K, ACROSS_K> sizes;
            typedef typename Whole<sizes>::Tile big;
            hipLaunchKernelGGL((head_dw_kernel<sizes>),
                               dim3(product_grid((long long)g.dw_parts * tiles_of(p.columns, big::BM) * tiles_of(p.d, big::BN), PRODUCT_CUS * sizes::PER_CU)),
                               dim3(big::THREADS), 0, st, q, 8);
        }
    }
    const int dh_blocks = dh ? blocks_for((size_t)N * p.d, 1024) : 0, dw_blocks = dw && g.dw_parts > 1 ? blocks_for((size_t)q.columns * p.d, 1024) : 0;
    const int db_blocks = db ? tiles_of(p.V, 64) : 0;
    if (dh_blocks + dw_blocks + db_blocks)
        hipLaunchKernelGGL(head_end_kernel<T>, dim3(dh_blocks + dw_blocks + db_blocks), dim3(256), 0, st, q, p.target, p.V, dh, dh_blocks, dw_blocks, db_parts,
                           g.db_rows, db);
}

int head_check(const char *who, int N, int d, int V, int dtype)
{
    MOE_REQUIRE(N >= 0 && d > 0 && V > 0, MOE_ERR_INVALID_ARG, "%s: N=%d d=%d V=%d out of range", who, N, d, V);
    MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
    MOE_REQUIRE(d % 8 == 0, MOE_ERR_INVALID_ARG, "%s: d=%d must be a multiple of 8", who, d);
    MOE_REQUIRE(d <= HEAD_MAX_WIDTH && V <= HEAD_MAX_IDS && N <= HEAD_MAX_ROWS && (long long)ceil_div(N, 16) * ceil_div(V, 128) < 1ll << 30 &&
                    (long long)ceil_div(d, 64) * ceil_div(V, 64) < 1ll << 30 && (long long)ceil_div(d, 64) * ceil_div(N, 16) < 1ll << 24,
                MOE_ERR_UNSUPPORTED, "%s: N=%d d=%d V=%d beyond the kernels", who, N, d, V);
    return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" size_t moe_head_logprobs_workspace_bytes(int N, int d, int V, int dtype)
{
    (void)d;
    if (N <= 0 || V <= 0) return 0;
    return head_scores_bytes(N, V, dtype);
}

extern "C" int moe_head_logprobs(const void *h, const void *w_head, const float *b_head, const int32_t *target, int N, int d, int V, int dtype,
                                 float *logprob, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = head_check("moe_head_logprobs", N, d, V, dtype);
    if (rc != MOE_OK || N == 0) return rc;
    MOE_REQUIRE(h && w_head && target && logprob && lse, MOE_ERR_INVALID_ARG, "moe_head_logprobs: null pointer");
    MOE_REQUIRE(aligned16(h) && aligned16(w_head), MOE_ERR_INVALID_ARG, "moe_head_logprobs: tensor misaligned");
    const size_t need = moe_head_logprobs_workspace_bytes(N, d, V, dtype);
    MOE_REQUIRE(ws && ws_bytes >= need && aligned16(ws), MOE_ERR_WORKSPACE, "moe_head_logprobs: workspace of %zu bytes given, %zu needed",
                ws ? ws_bytes : 0, need);
    const size_t z = dtype == MOE_F32 ? 4 : 2;
    const Span spans[] = {{h, (size_t)N * d * z, false}, {w_head, (size_t)V * d * z, false}, {b_head, (size_t)V * 4, false}, {target, (size_t)N * 4, false},
                          {logprob, (size_t)N * 4, true}, {lse, (size_t)N * 4, true}, {ws, need, true}};
    MOE_REQUIRE(spans_apart(spans), MOE_ERR_INVALID_ARG, "moe_head_logprobs: an output or the workspace aliases another tensor");
    HeadArgs p = {};
    p.h = h, p.w = w_head, p.b = b_head, p.target = target, p.N = N, p.d = d, p.V = V;
    p.n_n = head_row_slots(N, V, dtype);
    p.at_target = (float *)ws;
    p.tiles = (float2 *)((char *)ws + head_targets_bytes(N));
    if (dtype == MOE_BF16) forward<bf16_t, false>(p, logprob, lse, (hipStream_t)stream);
    else forward<float, false>(p, logprob, lse, (hipStream_t)stream);
    MOE_CHECK_LAUNCH("moe_head_logprobs");
    return MOE_OK;
}

extern "C" size_t moe_head_logprobs_backward_workspace_bytes(int N, int d, int V, int dtype)
{
    return N <= 0 || d <= 0 || V <= 0 ? 0 : head_shape(N, d, V, dtype).bytes;
}

extern "C" int moe_head_logprobs_backward(const void *h, const void *w_head, const float *b_head, const int32_t *target, const float *lse,
                                          const float *dlogprob, int N, int d, int V, int dtype, void *dh, void *dw_head, float *db_head, void *ws,
                                          size_t ws_bytes, void *stream)
{
    const int rc = head_check("moe_head_logprobs_backward", N, d, V, dtype);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE(N == 0 || (h && w_head && target && lse && dlogprob), MOE_ERR_INVALID_ARG, "moe_head_logprobs_backward: null pointer");
    MOE_REQUIRE(aligned16(h) && aligned16(w_head) && aligned16(dh) && aligned16(dw_head), MOE_ERR_INVALID_ARG,
                "moe_head_logprobs_backward: tensor misaligned");
    if (!dw_head && !db_head && (!dh || N == 0)) return MOE_OK;        // nothing is wanted
    const HeadShape g = N > 0 ? head_shape(N, d, V, dtype) : HeadShape();
    MOE_REQUIRE(N == 0 || (ws && ws_bytes >= g.bytes && aligned16(ws)), MOE_ERR_WORKSPACE,
                "moe_head_logprobs_backward: workspace of %zu bytes given, %zu needed", ws ? ws_bytes : 0, g.bytes);
    const size_t z = dtype == MOE_F32 ? 4 : 2, n = (size_t)N * 4;
    const Span spans[] = {{h, (size_t)N * d * z, false}, {w_head, (size_t)V * d * z, false}, {b_head, (size_t)V * 4, false}, {target, n, false}, {lse, n, false},
                          {dlogprob, n, false}, {dh, (size_t)N * d * z, true}, {dw_head, (size_t)V * d * z, true}, {db_head, (size_t)V * 4, true},
                          {ws, N > 0 ? g.bytes : 0, true}};
    MOE_REQUIRE(spans_apart(spans), MOE_ERR_INVALID_ARG, "moe_head_logprobs_backward: an output or the workspace aliases another tensor");
    hipStream_t st = (hipStream_t)stream;
    if (N == 0) {                              // sums over nothing
        if (dw_head) launch_clear(dw_head, (size_t)V * d * (dtype == MOE_F32 ? 4 : 2), st);
        if (db_head) launch_clear(db_head, (size_t)V * 4, st);
        MOE_CHECK_LAUNCH("moe_head_logprobs_backward");
        return MOE_OK;
    }
    HeadArgs p = {};
    p.h = h, p.w = w_head, p.b = b_head, p.target = target, p.lse = lse, p.dlogprob = dlogprob, p.N = N, p.d = d, p.V = V;
    if (dtype == MOE_BF16) backward<bf16_t>(p, g, (char *)ws, (bf16_t *)dh, (bf16_t *)dw_head, db_head, st);
    else backward<float>(p, g, (char *)ws, (float *)dh, (float *)dw_head, db_head, st);
    MOE_CHECK_LAUNCH("moe_head_logprobs_backward");
    return MOE_OK;
}
