// moe_token_logprobs and its gradient: log probabilities of given ids, entropy and the best alternatives of rows of logits.
//
// With m the largest logit, d = x - m, s = sum e^d and t = sum d e^d: lse = m + log s, log p_i = d_i - log s, entropy = log s - t / s.  Parts
// of a row join by bringing (m, s, t) to the larger maximum: s e^(m - M), (t + (m - M) s) e^(m - M).
// A row is read once, into registers.  The sums are found while it arrives.  The alternatives then cost next to nothing: a bound that k logits
// reach for certain (the k-th largest of the maxima of sixteen groups of threads), the few logits that reach it collected, and each ranked
// among them.  Rows where more than LP_LIST reach it (equal logits) or fewer than k lie above minus infinity take k searches of the registers:
// 8192 x 50257 bf16, k = 4, 1150 us for equal logits and 1030 for rows with five left, 179 else; 2048 x 32000 fp32, k = 8, 374, 352 and 49.
// Measured: 8192 x 50257 bf16, k = 4, 170 to 179 us (4.6 to 4.8 TB/s; memory, and some nine vector operations a logit beside it), 2048 x 32000 fp32 48 us
// (5.5 TB/s); 32768 x 256 fp32, k = 1, 9 us (3.7 TB/s); k = 8, where the searches' operations bind, 65536 x 256 22 us bf16 and 29 fp32, 32768 x 1000 40
// and 52.  In parts: 1500 x 131072 bf16 98 us (4.0 TB/s), 4000 x 50257 fp32 179 us (4.5 TB/s), 3 x 131072 12 us.  The gradient reads and writes once: 342
// us (4.8 TB/s) for the first, 13 us (5.2 TB/s) for the third.
#include <float.h>

#include "scalar_math.h"
#include "token_logprobs_rules.h"

namespace moe {

constexpr int LP_THREADS = 256;        // of a workgroup over short rows, and of the gradient's
constexpr int LP_GROUPS = 16;
constexpr int LP_LIST = 64;
typedef unsigned lp_u32x4_t __attribute__((ext_vector_type(4)));

template <class X> struct LogitPiece;
template <> struct LogitPiece<float> {
    static constexpr int N = 4;
    static constexpr unsigned MASKED = 0xff800000u;        // minus infinity
    static __device__ __forceinline__ float get(const lp_u32x4_t &p, int q) { return __uint_as_float(p[q]); }
};
template <> struct LogitPiece<bf16_t> {
    static constexpr int N = 8;
    static constexpr unsigned MASKED = 0xff80ff80u;
    static __device__ __forceinline__ float get(const lp_u32x4_t &p, int q)
    {
        return __uint_as_float(q & 1 ? p[q >> 1] & 0xffff0000u : p[q >> 1] << 16);
    }
};

// A logit as the alternatives see it: no number counts as masked (the maximum of a NaN and a value is the value).
__device__ __forceinline__ float lp_ranked(float x) { return fmaxf(x, -INFINITY); }

// Sums under a maximum.  It is never below the lowest finite value: a row that is masked throughout has s = 0, and no infinity is taken
// from another; a NaN passes into s.
struct LogitSums {
    float m, s, t;
    __device__ __forceinline__ void add(float x)
    {
        const float d = x - m, e = __builtin_amdgcn_exp2f(d * LOG2E);
        s += e;
        t = fmaf(fmaxf(d, -1e4f), e, t);                 // d off minus infinity, which times zero would be no number
    }
    // to >= m.  Products rounded as they are: one that a sum over lanes took in unrounded would differ from lane to lane.
    __device__ __forceinline__ void raise(float to)
    {
#pragma clang fp contract(off)
        const float d = fmaxf(m - to, -1e4f), e = exp_of<true>(d);
        t = (t + d * s) * e;
        s *= e;
        m = to;
    }
};
// a reduction over groups of LANES lanes
template <int LANES, int STEP = 0, class V, class F>
__device__ __forceinline__ V lp_over(V v, F f)
{
    if constexpr ((1 << STEP) < LANES) return lp_over<LANES, STEP + 1>(f(v, group_exchange<STEP>(v)), f);
    else return v;
}
template <int LANES>
__device__ __forceinline__ float lp_max_lanes(float v)
{
    return lp_over<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}
// the lanes' sums under the largest of their maxima
template <int LANES>
__device__ __forceinline__ void lp_join_lanes(LogitSums &a)
{
    a.raise(lp_max_lanes<LANES>(a.m));
    a.s = sum_over<LANES>(a.s);
    a.t = sum_over<LANES>(a.t);
}

struct LogprobOut {
    float *logprob, *entropy, *lse;
    int32_t *top_idx;
    float *top_logprob;
};

// what a row's sums give; xt: the target's logit
__device__ __forceinline__ void lp_finish(const LogitSums &a, float log_s, size_t n, int target, int V, float xt, const LogprobOut &o)
{
    const bool none = a.s == 0.f;
    o.logprob[n] = target < 0 || target >= V ? 0.f : none ? -INFINITY : xt - a.m - log_s;
    o.entropy[n] = none ? 0.f : log_s - a.t / a.s;
    o.lse[n] = none ? -INFINITY : a.m + log_s;
}
__device__ __forceinline__ float lp_of(float x, const LogitSums &a, float log_s) { return a.s == 0.f ? -INFINITY : x - a.m - log_s; }

// Short rows: LANES lanes each, LP_SMALL logits a lane in registers.  PIECES: rows begin on 16 bytes.
template <class X, int LANES, bool PIECES>
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_short_kernel(const X *__restrict__ logits, size_t stride,
                                                                          const int32_t *__restrict__ target, int N, int V, int k, LogprobOut out)
{
    typedef LogitPiece<X> piece;
    constexpr int P = PIECES ? piece::N : 1;             // consecutive logits of a lane
    const unsigned n = blockIdx.x * (LP_THREADS / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
    if (n >= (unsigned)N) return;
    const X *row = logits + n * stride;
    const int wanted = target[n];                        // asked for with the row, not behind the sums
    const float wanted_v = wanted >= 0 && wanted < V ? value_of(row[wanted]) : 0.f;
    // behind the row: masked, and after every logit of the row where equals are ranked
    float v[LP_SMALL];
#pragma unroll
    for (int i = 0; i < LP_SMALL; i += P) {
        const int at = i * LANES + lane * P;
        if (PIECES) {
            lp_u32x4_t p;
            if (at + P <= V) p = *(const lp_u32x4_t *)(row + at);
#pragma unroll
            for (int q = 0; q < P; ++q) v[i + q] = at + P <= V ? piece::get(p, q) : -INFINITY;
            if (at < V && at + P > V) {
#pragma unroll
                for (int q = 0; q < P; ++q) v[i + q] = at + q < V ? value_of(row[at + q]) : -INFINITY;
            }
        } else {
            v[i] = at < V ? value_of(row[at]) : -INFINITY;
        }
    }
    const auto place = [&](int i) { return i / P * P * LANES + lane * P + i % P; };
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < LP_SMALL; ++i) top = fmaxf(top, v[i]);
    top = lp_max_lanes<LANES>(top);
    LogitSums a = {fmaxf(top, -FLT_MAX), 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < LP_SMALL; ++i) a.add(v[i]);
    a.s = sum_over<LANES>(a.s);
    a.t = sum_over<LANES>(a.t);
    const float log_s = logf(a.s);
    if (lane == 0) lp_finish(a, log_s, n, wanted, V, wanted_v, out);
    if (k == 0) return;
    const auto put = [&](int j, float x, int id) {
        if (lane != 0) return;
        out.top_idx[(size_t)n * k + j] = id;
        out.top_logprob[(size_t)n * k + j] = lp_of(x, a, log_s);
    };
    if constexpr (sizeof(X) == 2) {
        // value and place in one word that grows with the value and falls with the place: one maximum finds both
        unsigned key[LP_SMALL];
#pragma unroll
        for (int i = 0; i < LP_SMALL; ++i) {
            const unsigned u = __float_as_uint(lp_ranked(v[i]) + 0.f);                 // -0 is 0
            key[i] = ((u ^ ((unsigned)((int)u >> 31) | 0x80000000u)) & 0xffff0000u) | (0xffffu - place(i));
        }
        for (int j = 0; j < k; ++j) {
            unsigned best = 0;
#pragma unroll
            for (int i = 0; i < LP_SMALL; ++i) best = max(best, key[i]);
            best = (unsigned)lp_over<LANES>((int)best, [](int x, int y) { return (int)max((unsigned)x, (unsigned)y); });
            if (j + 1 < k) {
#pragma unroll
                for (int i = 0; i < LP_SMALL; ++i) key[i] = key[i] == best ? 0u : key[i];
            }
            const unsigned u = best & 0xffff0000u;
            put(j, __uint_as_float(u >> 31 ? u ^ 0x80000000u : ~u & 0xffff0000u), (int)(0xffffu - (best & 0xffffu)));
        }
    } else {
#pragma unroll
        for (int i = 0; i < LP_SMALL; ++i) v[i] = lp_ranked(v[i]);
        for (int j = 0; j < k; ++j) {
            if (j > 0) {
                top = -INFINITY;
#pragma unroll
                for (int i = 0; i < LP_SMALL; ++i) top = fmaxf(top, v[i]);
                top = lp_max_lanes<LANES>(top);
            }
            int id = INT32_MAX;
#pragma unroll
            for (int i = LP_SMALL - 1; i >= 0; --i) id = v[i] == top ? place(i) : id;
            id = lp_over<LANES>(id, [](int x, int y) { return min(x, y); });
            if (j + 1 < k) {
#pragma unroll
                for (int i = 0; i < LP_SMALL; ++i) v[i] = place(i) == id ? NAN : v[i];     // taken
            }
            put(j, top, id);
        }
    }
}

// The best k of (value, id) entries of LDS, each ranked by those before it: entry of rank r to put(r, value, id).
template <class F>
__device__ __forceinline__ void lp_rank(const float *value, const int *id, int count, int k, F put)
{
    const int at = threadIdx.x;
    if (at >= count) return;
    const float v = value[at];
    const int i = id[at];
    int rank = 0;
    for (int j = 0; j < count; ++j) {
        const float ov = value[j];
        rank += ov > v || (ov == v && id[j] < i) ? 1 : 0;
    }
    if (rank < k) put(rank, v, i);
}

// Long rows: a workgroup takes a part of a row, LP_VECS pieces a thread in registers; 64 registers, so that two workgroups of 1024 share a compute unit
// and one loads while the other sums (one alone: 8192 x 50257 400 us); the builds for parts spill 50 of
// them in bf16 and 11 in fp32, most of it for the search behind a full list.  WHOLE: the part is the row; else its numbers go to
// a record of LP_RECORD floats.
template <class X, bool WHOLE>
__global__ __launch_bounds__(LP_MAX_THREADS, 8) void token_logprobs_kernel(const X *__restrict__ logits, size_t stride,
                                                                        const int32_t *__restrict__ target, int V, int parts, int part, int k,
                                                                        int threads, float *__restrict__ records, LogprobOut out)
{
    typedef LogitPiece<X> piece;
    constexpr int P = piece::N;
    __shared__ float wave_m[LP_MAX_THREADS / WAVE], wave_s[LP_MAX_THREADS / WAVE], wave_t[LP_MAX_THREADS / WAVE];
    __shared__ float groups[LP_GROUPS], list_v[LP_LIST];
    __shared__ int list_id[LP_LIST], listed;
    const unsigned n = blockIdx.x, which = WHOLE ? 0 : blockIdx.y;
    const int lo = which * part, len = min(part, V - lo), tid = threadIdx.x, lane = tid % WAVE;
    const int wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
    const int waves = threads / WAVE;
    const X *row = logits + n * stride + lo;
    // pieces of 16 bytes from the first address that is one; what lies before and behind them is one logit a thread
    const int head = min(len, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(X)), pieces = (len - head) / P;
    const int behind = head + pieces * P, ends = len - pieces * P;
    const int end_at = tid < head ? tid : behind + (tid - head);       // this thread's single logit, for tid < ends
    const lp_u32x4_t *body = (const lp_u32x4_t *)(row + head);
    const int wanted = target[n];                        // asked for with the row, not behind the sums
    const float wanted_v = wanted >= lo && wanted < lo + len ? value_of(row[wanted - lo]) : 0.f;
    lp_u32x4_t held[LP_VECS];
    X single = 0;
    if (tid < ends) single = row[end_at];
#pragma unroll
    for (int i = 0; i < LP_VECS; ++i) {                   // masked behind the last piece
        held[i] = {piece::MASKED, piece::MASKED, piece::MASKED, piece::MASKED};
        if (i * threads + tid < pieces) held[i] = body[i * threads + tid];
    }
    if (tid == 0) listed = 0;
    const float end_v = tid < ends ? value_of(single) : -INFINITY;
    float top = end_v;
#pragma unroll
    for (int i = 0; i < LP_VECS; ++i) {
        if (i * threads + wave * WAVE >= pieces) break;  // the whole wavefront
#pragma unroll
        for (int q = 0; q < P; ++q) top = fmaxf(top, piece::get(held[i], q));
    }
    // the groups of threads that the bound is taken from: threads / LP_GROUPS neighbours, a wavefront at most
    float most = lp_max_lanes<4>(top);
    {
        const int size = threads / LP_GROUPS;
        float group = most;
        most = fmaxf(most, group_exchange<2>(most));
        if (size >= 8) group = most;
        most = fmaxf(most, group_exchange<3>(most));
        if (size >= 16) group = most;
        most = fmaxf(most, group_exchange<4>(most));
        if (size >= 32) group = most;
        most = fmaxf(most, group_exchange<5>(most));
        if (size >= 64) group = most;
        if (tid % size == 0) groups[tid / size] = group;
    }
    LogitSums a = {fmaxf(most, -FLT_MAX), 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < LP_VECS; ++i) {
        if (i * threads + wave * WAVE >= pieces) break;
#pragma unroll
        for (int q = 0; q < P; ++q) a.add(piece::get(held[i], q));
    }
    if (ends) a.add(end_v);
    a.s = sum_over<WAVE>(a.s);
    a.t = sum_over<WAVE>(a.t);
    if (lane == 0) wave_m[wave] = a.m, wave_s[wave] = a.s, wave_t[wave] = a.t;
    __syncthreads();
    {                                                    // the wavefronts' sums, one a lane
        const int w = lane % LP_GROUPS;
        a.m = w < waves ? wave_m[w] : -FLT_MAX;
        a.s = w < waves ? wave_s[w] : 0.f;
        a.t = w < waves ? wave_t[w] : 0.f;
        lp_join_lanes<LP_GROUPS>(a);
    }
    const float log_s = logf(a.s);
    float *record = WHOLE ? nullptr : records + ((size_t)n * parts + which) * LP_RECORD;
    if (tid == 0) {
        if (WHOLE) lp_finish(a, log_s, n, wanted, V, wanted_v, out);
        else record[0] = a.m, record[1] = a.s, record[2] = a.t, record[3] = wanted_v;
    }
    if (k == 0) return;
    const auto put = [&](int rank, float v, int id) {
        if (WHOLE) {
            out.top_idx[(size_t)n * k + rank] = id;
            out.top_logprob[(size_t)n * k + rank] = lp_of(v, a, log_s);
        } else {
            record[4 + rank] = v;
            record[4 + MOE_MAX_TOPK + rank] = __int_as_float(id + lo);
        }
    };
    // the bound: the least of the groups' maxima that fewer than k are above
    const float mine = groups[lane % LP_GROUPS];
    unsigned few = 0;
#pragma unroll
    for (int j = 0; j < LP_GROUPS; ++j) {
        const float o = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), j));
        few |= __popcll(__ballot(mine > o) & ((1u << LP_GROUPS) - 1)) < k ? 1u << j : 0u;
    }
    const float bound = -lp_max_lanes<LP_GROUPS>(few >> lane % LP_GROUPS & 1 ? -mine : -INFINITY);
    int count = LP_LIST + 1;
    if (bound > -INFINITY) {
        if (top >= bound) {
            const auto offer = [&](float v, int id) {
                if (v >= bound) {
                    const int at = atomicAdd(&listed, 1);
                    if (at < LP_LIST) list_v[at] = v, list_id[at] = id;
                }
            };
#pragma unroll
            for (int i = 0; i < LP_VECS; ++i) {
                if (i * threads + wave * WAVE >= pieces) break;
                asm("" : "+v"(held[i]));               // unpacked again: the logits themselves would fill the registers
                float best = piece::get(held[i], 0);
#pragma unroll
                for (int q = 1; q < P; ++q) best = fmaxf(best, piece::get(held[i], q));
                if (best < bound) continue;
#pragma unroll
                for (int q = 0; q < P; ++q) offer(piece::get(held[i], q), head + (i * threads + tid) * P + q);
            }
            if (tid < ends) offer(end_v, end_at);
        }
        __syncthreads();
        count = listed;
    }
    if (count <= LP_LIST) {
        lp_rank(list_v, list_id, count, k, put);
        return;
    }
    // one by one: the largest behind the one before, smaller or equal with a higher id
    float after = INFINITY;
    int after_id = -1;
    for (int j = 0; j < min(k, len); ++j) {
        float best = -INFINITY;
        int id = INT32_MAX;
        const auto offer = [&](float x, int at) {
            const float v = lp_ranked(x);
            if ((v < after || (v == after && at > after_id)) && (v > best || (v == best && at < id))) best = v, id = at;
        };
        if (tid < ends) offer(end_v, end_at);
#pragma unroll
        for (int i = 0; i < LP_VECS; ++i) {
            asm("" : "+v"(held[i]));
            if (i * threads + tid >= pieces) continue;
#pragma unroll
            for (int q = 0; q < P; ++q) offer(piece::get(held[i], q), head + (i * threads + tid) * P + q);
        }
        argmax_over<WAVE>(best, id);
        __syncthreads();                               // the round before has been read
        if (lane == 0) list_v[wave] = best, list_id[wave] = id;
        __syncthreads();
        best = list_v[0], id = list_id[0];
        for (int w = 1; w < waves; ++w) argmax_merge(best, id, list_v[w], list_id[w]);
        if (tid == 0) put(j, best, id);
        after = best;
        after_id = id;
    }
    if (!WHOLE && tid == 0)
        for (int j = len; j < k; ++j) record[4 + j] = -INFINITY, record[4 + MOE_MAX_TOPK + j] = __int_as_float(INT32_MAX);
}

// the parts of a row, one lane each; a lane's best entries are in order, so only the first that is left can be the next
__global__ __launch_bounds__(WAVE) void token_logprobs_join_kernel(const float *__restrict__ records, const int32_t *__restrict__ target, int V,
                                                                   int parts, int part, int k, LogprobOut out)
{
    const size_t n = blockIdx.x;
    const int lane = threadIdx.x;
    const float *record = records + (n * parts + min(lane, parts - 1)) * LP_RECORD;
    LogitSums a = {-FLT_MAX, 0.f, 0.f};
    if (lane < parts) a = {record[0], record[1], record[2]};
    float best[MOE_MAX_TOPK];
    int ids[MOE_MAX_TOPK];
#pragma unroll
    for (int j = 0; j < MOE_MAX_TOPK; ++j) {
        best[j] = j < k && lane < parts ? record[4 + j] : -INFINITY;
        ids[j] = j < k && lane < parts ? __float_as_int(record[4 + MOE_MAX_TOPK + j]) : INT32_MAX;
    }
    const int wanted = target[n];
    const float wanted_v = wanted >= 0 && wanted < V ? records[(n * parts + wanted / part) * LP_RECORD + 3] : 0.f;
    lp_join_lanes<WAVE>(a);
    const float log_s = logf(a.s);
    if (lane == 0) lp_finish(a, log_s, n, wanted, V, wanted_v, out);
    for (int j = 0; j < k; ++j) {
        float v = best[0];
        int i = ids[0];
        argmax_over<WAVE>(v, i);
        if (i == ids[0]) {
#pragma unroll
            for (int q = 0; q + 1 < MOE_MAX_TOPK; ++q) best[q] = best[q + 1], ids[q] = ids[q + 1];
            best[MOE_MAX_TOPK - 1] = -INFINITY, ids[MOE_MAX_TOPK - 1] = INT32_MAX;
        }
        if (lane == 0) {
            out.top_idx[n * k + j] = i;
            out.top_logprob[n * k + j] = lp_of(v, a, log_s);
        }
    }
}

// The gradient, elementwise: -p (g + q (log p + H)), and g more at the target.  log p = x - lse - rest: lse = m + log s has been rounded, and beside a
// large m that takes a part of log s or all of it.  rest is what the row's own sum then says, log sum e^(x - lse); 0 where lse holds.
template <class X>
struct LogprobSlope {
    static constexpr bool PRECISE = sizeof(X) == 4;
    // from where a row is summed again: an lse below is off by 2^-19 (binary32) or 2^-14 (bfloat16, whose results round by 2^-8) at most
    static constexpr float FAR = PRECISE ? 64.f : 2048.f;
    float lse, rest, base, q, g;
    int target;
    bool none;
    __device__ __forceinline__ float at(float x, int i) const
    {
        const float lp = x - lse - rest, p = exp_of<PRECISE>(lp);
        float d = p * fmaf(-q, lp, base);
        d = p == 0.f || none ? 0.f : d;                  // a masked logit: log p is no number to multiply with
        return i == target && !none ? d + g : d;
    }
};

// 2^lg threads share a row; blockIdx.y: its run of 2^lg * LP_SLOPE_PIECES pieces.  A row far from zero is the first run's alone, which reads it twice (8192 x
// 20000 fp32 259 us, all rows far 396; 8192 x 50257 bf16 340 and 751; 4 x 131072 fp32 5 and 139).  dlogits may lie on it, so all of it is read before any is
// written: by the threads of one wavefront, or by the workgroup with a barrier, which the two rows of a workgroup do not share.
template <class X>
__global__ __launch_bounds__(LP_THREADS) void token_logprobs_backward_kernel(const X *logits, size_t stride, const int32_t *__restrict__ target,
                                                                             const float *__restrict__ lse, const float *__restrict__ entropy,
                                                                             const float *__restrict__ dlogprob, const float *__restrict__ dentropy,
                                                                             int N, int V, int lg, X *dlogits, size_t dstride)
{
    typedef LogitPiece<X> piece;
    constexpr int P = piece::N;
    __shared__ float wave_sum[LP_THREADS / WAVE];
    const unsigned n = blockIdx.x * (LP_THREADS >> lg) + (threadIdx.x >> lg);
    const int lanes = 1 << lg, lane = threadIdx.x & (lanes - 1);
    if (n >= (unsigned)N) return;
    const X *row = logits + n * stride;
    X *out = dlogits + n * dstride;
    LogprobSlope<X> f;
    f.target = target[n];
    f.lse = lse[n];
    f.q = dentropy ? dentropy[n] : 0.f;
    const float slope = dlogprob[n];                     // asked for with the others, not behind the target
    const bool padded = f.target < 0 || f.target >= V;
    f.g = padded ? 0.f : slope;
    f.none = f.lse == -INFINITY || (padded && f.q == 0.f);     // nothing to pass on, whatever a padded position's logits hold
    f.base = -f.g - (dentropy ? f.q * entropy[n] : 0.f);
    f.rest = 0.f;
    if (fabsf(f.lse) >= f.FAR && !f.none) {              // the whole group of threads
        const int sharers = lanes < LP_THREADS ? min(lanes, WAVE) : LP_THREADS;
        if (blockIdx.y != 0 || lane >= sharers) return;
        float sum = 0.f;
#pragma unroll 4
        for (int c = lane; c < V; c += sharers) sum += exp_of<true>(value_of(row[c]) - f.lse);
        for (int o = 1; o < sharers && o < WAVE; o <<= 1) sum += __shfl_xor(sum, o, WAVE);
        if (sharers > WAVE) {
            if (lane % WAVE == 0) wave_sum[lane / WAVE] = sum;
            __syncthreads();
            sum = 0.f;
            for (int w = 0; w < LP_THREADS / WAVE; ++w) sum += wave_sum[w];
        }
        f.rest = logf(sum);
        for (int c = lane; c < V; c += sharers) store_value(out + c, f.at(value_of(row[c]), c));
        return;
    }
    const int run = lanes * LP_SLOPE_PIECES;
    if ((((uintptr_t)row ^ (uintptr_t)out) & 15) == 0) {
        const int head = min(V, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(X)), pieces = (V - head) / P;
        const lp_u32x4_t *body = (const lp_u32x4_t *)(row + head);
        lp_u32x4_t *to = (lp_u32x4_t *)(out + head), held[LP_SLOPE_PIECES];
        const int first = blockIdx.y * run + lane;
#pragma unroll
        for (int i = 0; i < LP_SLOPE_PIECES; ++i)
            if (first + i * lanes < pieces) held[i] = body[first + i * lanes];
#pragma unroll
        for (int i = 0; i < LP_SLOPE_PIECES; ++i) {
            const int at = first + i * lanes;
            if (at >= pieces) continue;
            lp_u32x4_t r;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int c = head + at * P + w * (P / 4);
                if constexpr (P == 4) r[w] = __float_as_uint(f.at(piece::get(held[i], w), c));
                else r[w] = pack_bf16x2(f.at(piece::get(held[i], 2 * w), c), f.at(piece::get(held[i], 2 * w + 1), c + 1));
            }
            to[at] = r;
        }
        if (blockIdx.y == 0) {
            const int ends = V - pieces * P;
            for (int e = lane; e < ends; e += lanes) {
                const int c = e < head ? e : pieces * P + e;
                store_value(out + c, f.at(value_of(row[c]), c));
            }
        }
    } else {                                             // rows that lie differently inside 16 bytes
        const int last = min(V, (int)(blockIdx.y + 1) * run * P);
        for (int c = blockIdx.y * run * P + lane; c < last; c += lanes) store_value(out + c, f.at(value_of(row[c]), c));
    }
}

static int logprobs_check(const char *who, int N, int V, long long stride, int dtype)
{
    MOE_REQUIRE(N >= 0 && V > 0, MOE_ERR_INVALID_ARG, "%s: N=%d V=%d out of range", who, N, V);
    MOE_REQUIRE(stride >= V, MOE_ERR_INVALID_ARG, "%s: rows of %d logits lie %lld apart", who, V, stride);
    MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
    MOE_REQUIRE(logprob_takes(N, V, dtype), MOE_ERR_UNSUPPORTED, "%s: N=%d V=%d too large (V <= %d)", who, N, V, LP_MAX_V);
    return MOE_OK;
}

}  // namespace moe

using namespace moe;

extern "C" size_t moe_token_logprobs_workspace_bytes(int N, int V, int k, int dtype)
{
    (void)k;
    if (N <= 0 || V <= 0 || (dtype != MOE_F32 && dtype != MOE_BF16) || !logprob_takes(N, V, dtype)) return 0;
    const LogprobShape g = logprob_shape(N, V, dtype);
    return g.parts > 1 ? (size_t)N * g.parts * LP_RECORD * sizeof(float) : 0;
}

template <class X>
static void logprobs_launch(const LogprobShape &g, const X *logits, size_t stride, const int32_t *target, int N, int V, int k, float *records,
                            const LogprobOut &out, hipStream_t st)
{
    if (g.lanes) {
        const bool pieces = ((uintptr_t)logits & 15) == 0 && stride * sizeof(X) % 16 == 0;
        const dim3 grid(ceil_div(N, LP_THREADS / g.lanes)), threads(LP_THREADS);
#define MOE_SHORT(L)                                                                                                                                \
    do {                                                                                                                                            \
        if (pieces) hipLaunchKernelGGL((token_logprobs_short_kernel<X, L, true>), grid, threads, 0, st, logits, stride, target, N, V, k, out);      \
        else hipLaunchKernelGGL((token_logprobs_short_kernel<X, L, false>), grid, threads, 0, st, logits, stride, target, N, V, k, out);            \
    } while (0)
        if (g.lanes == 4) MOE_SHORT(4);
        else if (g.lanes == 16) MOE_SHORT(16);
        else MOE_SHORT(64);
#undef MOE_SHORT
        return;
    }
    const dim3 grid(N, g.parts), threads(g.threads);
    if (g.parts == 1) {
        hipLaunchKernelGGL((token_logprobs_kernel<X, true>), grid, threads, 0, st, logits, stride, target, V, 1, g.part, k, g.threads, nullptr, out);
        return;
    }
    hipLaunchKernelGGL((token_logprobs_kernel<X, false>), grid, threads, 0, st, logits, stride, target, V, g.parts, g.part, k, g.threads, records,
                       out);
    hipLaunchKernelGGL(token_logprobs_join_kernel, dim3(N), dim3(WAVE), 0, st, records, target, V, g.parts, g.part, k, out);
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
    MOE_REQUIRE((uintptr_t)logits % (dtype == MOE_F32 ? 4 : 2) == 0, MOE_ERR_INVALID_ARG, "moe_token_logprobs: tensor misaligned");
    const LogprobShape g = logprob_shape(N, V, dtype);
    const size_t need = moe_token_logprobs_workspace_bytes(N, V, k, dtype);
    MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE,
                "moe_token_logprobs: workspace of %zu bytes given, %zu needed", ws ? ws_bytes : 0, need);
    const LogprobOut out = {logprob, entropy, lse, top_idx, top_logprob};
    if (dtype == MOE_BF16) logprobs_launch(g, (const bf16_t *)logits, (size_t)row_stride, target, N, V, k, (float *)ws, out, (hipStream_t)stream);
    else logprobs_launch(g, (const float *)logits, (size_t)row_stride, target, N, V, k, (float *)ws, out, (hipStream_t)stream);
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
    static_assert(LP_THREADS == 1 << LP_SLOPE_LG, "");
    const int size = dtype == MOE_F32 ? 4 : 2, pieces = logprob_slope_pieces(V, dtype), lg = logprob_slope_lanes(V, dtype);
    MOE_REQUIRE((uintptr_t)logits % size == 0 && (uintptr_t)dlogits % size == 0, MOE_ERR_INVALID_ARG, "moe_token_logprobs_backward: tensor misaligned");
    const dim3 grid(ceil_div(N, LP_THREADS >> lg), ceil_div(pieces, LP_SLOPE_PIECES << lg));
    hipStream_t st = (hipStream_t)stream;
    if (dtype == MOE_BF16)
        hipLaunchKernelGGL(token_logprobs_backward_kernel<bf16_t>, grid, dim3(LP_THREADS), 0, st, (const bf16_t *)logits, (size_t)row_stride,
                           target, lse, entropy, dlogprob, dentropy, N, V, lg, (bf16_t *)dlogits, (size_t)dlogits_stride);
    else
        hipLaunchKernelGGL(token_logprobs_backward_kernel<float>, grid, dim3(LP_THREADS), 0, st, (const float *)logits, (size_t)row_stride,
                           target, lse, entropy, dlogprob, dentropy, N, V, lg, (float *)dlogits, (size_t)dlogits_stride);
    MOE_CHECK_LAUNCH("moe_token_logprobs_backward");
    return MOE_OK;
}
