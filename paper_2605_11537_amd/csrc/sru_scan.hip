// sru_scan and its gradient: the recurrence of an SRU layer over pre-activations that lie in memory.
//
// c_t = f_t c_{t-1} + b_t composes: a run of steps is a pair (A, C), c_out = A c_in + C, and the pair of two runs is (A2 A1, A2 C1 + C2).
// The gradient dc_{t-1} = f_t (dc_t + e_t) is the same from the other end.  So a wavefront takes SCAN_STEPS steps of 64 lanes' channels with
// everything they read in registers, finds its pair from zero, and learns its start from the pairs of the wavefronts before it, through
// LDS: the wavefronts of a workgroup lie one behind the other on the sequence, and a round of them is read once and written once.
// Where sequences and channels alone are too few for the card, the sequence is cut into segments for several workgroups, whose pairs a launch
// before finds (it reads half of what the main one reads, again).
#include "scalar_math.h"
#include "sru_scan_rules.h"

namespace moe {

// A run's rows of a tensor as a buffer: the lane's offset in a register, the step's in a scalar one (addresses of 64 bits for every step and
// tensor spilled scalar registers into vector ones).  An offset from 2^31 on is outside: lanes without a channel ask for nothing and store nothing.
constexpr unsigned SCAN_NOWHERE = 0x80000000u;
typedef __amdgpu_buffer_rsrc_t scan_rows_t;

__device__ __forceinline__ scan_rows_t scan_rows(const void *first)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(first), 0, 0x7fffffff, 0x27000);
}
template <class T>
__device__ __forceinline__ T scan_get(scan_rows_t rows, unsigned lane_at, unsigned step_at)
{
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_raw_buffer_load_b16(rows, lane_at, step_at, 0);
    else return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(rows, lane_at, step_at, 0));
}
template <class T>
__device__ __forceinline__ void scan_put(float v, scan_rows_t rows, unsigned lane_at, unsigned step_at)
{
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(f32_to_bf16(v), rows, lane_at, step_at, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), rows, lane_at, step_at, 0);
}

// Where a workgroup stands: channels, sequence, segment.  Everything but the channel is the same for a whole wavefront.
template <class T>
struct ScanPlace {
    int b, seg, lane, wave, waves, n, first, last;     // first .. last-1: the segment's steps
    unsigned ch, col;                                  // this lane's channel; one that exists
    unsigned at, block;                                // its offset in a row of one block, and a block's length, in bytes
    bool on;
    __device__ __forceinline__ bool find(const ScanShape &g, const int32_t *lengths, int segments)
    {
        const unsigned wg = blockIdx.y * gridDim.x + blockIdx.x;
        const unsigned groups = g.groups, line = wg / groups;
        b = line / segments;
        seg = line - (unsigned)b * segments;
        if (b >= g.B) return false;
        lane = threadIdx.x % WAVE;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
        waves = blockDim.x / WAVE;
        ch = (wg - line * groups) * WAVE + lane;
        on = ch < (unsigned)g.H;
        col = on ? ch : 0;
        at = on ? ch * (unsigned)sizeof(T) : SCAN_NOWHERE;
        block = g.H * (unsigned)sizeof(T);
        n = lengths ? min(max(lengths[b], 0), g.L) : g.L;
        n = __builtin_amdgcn_readfirstlane(n);
        first = seg * g.seg_steps;
        last = min(g.L, first + g.seg_steps);
        return true;
    }
};

// A wavefront's steps are all inside the sequence (FULL: no step is asked for), or some are not.
struct ScanFull { static constexpr bool FULL = true; };
struct ScanPart { static constexpr bool FULL = false; };
template <bool FULL> __device__ __forceinline__ bool scan_in(int i, int count) { return FULL || i < count; }

// the steps of one column block, the first count of them
template <class T, bool FULL>
__device__ __forceinline__ void scan_load(T (&to)[SCAN_STEPS], scan_rows_t rows, unsigned lane_at, unsigned row_bytes, int count)
{
#pragma unroll
    for (int i = 0; i < SCAN_STEPS; ++i) {
        if (!FULL) to[i] = 0;
        if (scan_in<FULL>(i, count)) to[i] = scan_get<T>(rows, lane_at, i * row_bytes);
    }
}

// c_t from c_{t-1}: f c + (1 - f) z with both gates' own accuracy, or z + f (c - z) for bfloat16 results
template <bool PRECISE>
struct ScanForward {
    float f, in;
    __device__ __forceinline__ void make(float a, float bias, float z)
    {
        if (PRECISE) {
            float rest;
            gate_of<true>(a, bias, f, rest);
            in = rest * z;
        } else {
            f = gate_open<false>(a, bias);
            in = z;
        }
    }
    __device__ __forceinline__ float next(float c) const { return PRECISE ? fmaf(f, c, in) : fmaf(f, c - in, in); }
};

// the state that a pair list before this place leads to
__device__ __forceinline__ float scan_fold(float c, const float2 *pairs, size_t step, int count)
{
#pragma unroll 16
    for (int j = 0; j < count; ++j) {
        const float2 p = pairs[j * step];
        c = fmaf(p.x, c, p.y);
    }
    return c;
}

template <class T, bool HIGHWAY>
__global__ __launch_bounds__(SCAN_MAX_WAVES *WAVE) void sru_scan_kernel(ScanShape g, const T *__restrict__ u, const T *__restrict__ x,
                                                                       const float *__restrict__ b_f, const float *__restrict__ b_r,
                                                                       const float *c0, const int32_t *__restrict__ lengths,
                                                                       const float2 *__restrict__ pairs, T *__restrict__ h, float *c_last,
                                                                       float *__restrict__ states)
{
    constexpr bool PRECISE = sizeof(T) == 4;
    constexpr int K = HIGHWAY ? 3 : 4;
    __shared__ float2 sums[2][SCAN_MAX_WAVES][WAVE];
    ScanPlace<T> p;
    if (!p.find(g, lengths, g.segments)) return;
    const size_t H = g.H, row_len = K * H;
    const float bf = gate_bias<PRECISE>(b_f ? b_f[p.col] : 0.f), br = gate_bias<PRECISE>(b_r ? b_r[p.col] : 0.f);
    float c_in = c0 ? c0[(size_t)p.b * H + p.col] : 0.f;
    c_in = scan_fold(c_in, pairs + (size_t)p.b * (g.segments - 1) * H + p.col, H, p.seg);
    const int round = p.waves * SCAN_STEPS;
    for (int t = p.first, parity = 0; t < p.last; t += round, parity ^= 1) {
        const int t0 = t + p.wave * SCAN_STEPS, count = min(p.n - t0, SCAN_STEPS);    // this wavefront's steps inside the sequence
        auto steps = [&](auto how) {
            constexpr bool FULL = decltype(how)::FULL;
            const size_t row = (size_t)p.b * g.L + t0;
            const scan_rows_t ur = scan_rows(u + row * row_len), xr = HIGHWAY ? scan_rows(x + row * H) : ur, hr = scan_rows(h + row * H);
            T z[SCAN_STEPS], a[SCAN_STEPS], r[SCAN_STEPS], w[SCAN_STEPS];
            scan_load<T, FULL>(z, ur, p.at, K * p.block, count);
            scan_load<T, FULL>(a, ur, p.at + p.block, K * p.block, count);
            scan_load<T, FULL>(r, ur, p.at + 2 * p.block, K * p.block, count);
            if (HIGHWAY) scan_load<T, FULL>(w, xr, p.at, p.block, count);
            else scan_load<T, FULL>(w, ur, p.at + 3 * p.block, K * p.block, count);
            ScanForward<PRECISE> s[SCAN_STEPS];
            float A = 1.f, C = 0.f, c;
#pragma unroll
            for (int i = 0; i < SCAN_STEPS; ++i) {
                if (!scan_in<FULL>(i, count)) continue;
                s[i].make(value_of(a[i]), bf, value_of(z[i]));
                A *= s[i].f;
                C = s[i].next(C);
            }
            if (p.waves > 1) {
                sums[parity][p.wave][p.lane] = make_float2(A, C);
                barrier_anywhere();                    // a full and a partial wavefront wait for each other here
                c = c_in;
                for (int j = 0; j < p.waves; ++j) {
                    const float2 q = sums[parity][j][p.lane];
                    c_in = fmaf(q.x, c_in, q.y);
                    if (j + 1 == p.wave) c = c_in;
                }
            } else {
                c = c_in, c_in = fmaf(A, c_in, C);
            }
            if (states && (FULL || t0 < g.L) && p.on) states[((size_t)p.b * g.saved + t0 / SCAN_STEPS) * H + p.ch] = c;
#pragma unroll
            for (int i = 0; i < SCAN_STEPS; ++i) {
                if (!scan_in<FULL>(i, count)) {
                    if (t0 + i < p.last) scan_put<T>(0.f, hr, p.at, i * p.block);
                    continue;
                }
                c = s[i].next(c);
                const float wv = value_of(w[i]), t = tanh_of<PRECISE>(c);
                float out;
                if (PRECISE) {
                    float on, rest;
                    gate_of<true>(value_of(r[i]), br, on, rest);
                    out = fmaf(on, t, rest * wv);
                } else {
                    out = fmaf(gate_open<false>(value_of(r[i]), br), t - wv, wv);
                }
                scan_put<T>(out, hr, p.at, i * p.block);
            }
        };
        if (count >= SCAN_STEPS) steps(ScanFull());
        else steps(ScanPart());
    }
    if (c_last && p.seg == g.segments - 1 && p.wave == 0 && p.on) c_last[(size_t)p.b * H + p.ch] = c_in;
}

// The pairs of the first segments, [b][segment][channel]; a wavefront walks its own part of the segment from one end to the other.  Segment
// 0 lays c0 down beside them: c_last may be c0, and the main launch's last segment writes it while others still read.
template <class T>
__global__ __launch_bounds__(SCAN_MAX_WAVES *WAVE) void sru_scan_pairs_kernel(ScanShape g, const T *__restrict__ u, int blocks,
                                                                             const float *__restrict__ b_f, const float *__restrict__ c0,
                                                                             const int32_t *__restrict__ lengths, float2 *__restrict__ pairs,
                                                                             float *__restrict__ c0_copy)
{
    constexpr bool PRECISE = sizeof(T) == 4;
    __shared__ float2 sums[SCAN_MAX_WAVES][WAVE];
    ScanPlace<T> p;
    if (!p.find(g, lengths, g.segments - 1)) return;
    const size_t H = g.H, row_len = blocks * H;
    const float bf = gate_bias<PRECISE>(b_f ? b_f[p.col] : 0.f);
    float A = 1.f, C = 0.f;
    const int part = g.seg_steps / p.waves, from = p.first + p.wave * part, to = from + part;     // whole runs: seg_steps is whole rounds
    for (int t0 = from; t0 < to; t0 += SCAN_STEPS) {
        const int count = min(p.n - t0, SCAN_STEPS);
        const scan_rows_t ur = scan_rows(u + ((size_t)p.b * g.L + t0) * row_len);
        const unsigned row_bytes = blocks * p.block;
        auto steps = [&](auto how) {
            constexpr bool FULL = decltype(how)::FULL;
            T z[SCAN_STEPS], a[SCAN_STEPS];
            scan_load<T, FULL>(z, ur, p.at, row_bytes, count);
            scan_load<T, FULL>(a, ur, p.at + p.block, row_bytes, count);
#pragma unroll
            for (int i = 0; i < SCAN_STEPS; ++i) {
                if (!scan_in<FULL>(i, count)) continue;
                ScanForward<PRECISE> s;
                s.make(value_of(a[i]), bf, value_of(z[i]));
                A *= s.f;
                C = s.next(C);
            }
        };
        if (count >= SCAN_STEPS) steps(ScanFull());
        else steps(ScanPart());
    }
    sums[p.wave][p.lane] = make_float2(A, C);
    __syncthreads();
    if (p.wave != 0 || !p.on) return;
    for (int j = 1; j < p.waves; ++j) {
        const float2 q = sums[j][p.lane];
        C = fmaf(q.x, C, q.y);
        A *= q.x;
    }
    pairs[((size_t)p.b * (g.segments - 1) + p.seg) * H + p.ch] = make_float2(A, C);
    if (p.seg == 0) c0_copy[(size_t)p.b * H + p.ch] = c0 ? c0[(size_t)p.b * H + p.ch] : 0.f;
}

// what a step of the gradient needs of the forward, from the state before it: e and the factors of the outputs
template <bool PRECISE>
struct ScanStep {
    float f, rest, e, gap;       // gate, 1 - gate, dh r tanh'(c), (c_{t-1} - z) f (1 - f)
    float d_r, d_w;              // du2 and dw
    __device__ __forceinline__ void make(float &c, float z, float a, float bf, float r, float br, float w, float dh)
    {
        float s, off, slope;
        gate_of<PRECISE>(a, bf, f, rest);
        gate_of<PRECISE>(r, br, s, off);
        gap = (c - z) * (f * rest);
        c = fmaf(f, c, rest * z);
        const float t = tanh_of<PRECISE>(c, slope);
        e = dh * s * slope;
        d_w = dh * off;
        d_r = dh * (t - w) * (s * off);
    }
};

template <class T, bool HIGHWAY>
__global__ __launch_bounds__(SCAN_MAX_WAVES *WAVE) void sru_scan_backward_kernel(
    ScanShape g, const T *__restrict__ dh, const float *dc_last, const T *__restrict__ u, const T *__restrict__ x, const float *__restrict__ b_f,
    const float *__restrict__ b_r, const float *__restrict__ states, const int32_t *__restrict__ lengths, const float2 *__restrict__ pairs,
    T *__restrict__ du, T *__restrict__ dx, float *__restrict__ db, float *dc0)
{
    constexpr bool PRECISE = sizeof(T) == 4;
    constexpr int K = HIGHWAY ? 3 : 4;
    __shared__ float2 sums[2][SCAN_MAX_WAVES][WAVE];
    ScanPlace<T> p;
    if (!p.find(g, lengths, g.segments)) return;
    const size_t H = g.H, row_len = K * H;
    const float bf = gate_bias<PRECISE>(b_f ? b_f[p.col] : 0.f), br = gate_bias<PRECISE>(b_r ? b_r[p.col] : 0.f);
    float sum_f = 0.f, sum_r = 0.f, d_in = dc_last ? dc_last[(size_t)p.b * H + p.col] : 0.f;
    d_in = scan_fold(d_in, pairs + (size_t)p.b * (g.segments - 1) * H + p.col, H, g.segments - 1 - p.seg);
    const int round = p.waves * SCAN_STEPS, rounds = p.last > p.first ? (p.last - p.first + round - 1) / round : 0;
    for (int at = rounds - 1, parity = 0; at >= 0; --at, parity ^= 1) {
        const int t0 = p.first + at * round + p.wave * SCAN_STEPS, count = min(p.n - t0, SCAN_STEPS);
        const size_t row = (size_t)p.b * g.L + t0;
        const scan_rows_t ur = scan_rows(u + row * row_len), dr = scan_rows(dh + row * H), out = scan_rows(du + row * row_len);
        const scan_rows_t xr = HIGHWAY ? scan_rows(x + row * H) : ur, out_w = HIGHWAY ? scan_rows(dx + row * H) : out;
        const unsigned at_w = HIGHWAY ? p.at : p.at + 3 * p.block, row_bytes = K * p.block, w_bytes = HIGHWAY ? p.block : row_bytes;
        auto steps = [&](auto how) {
            constexpr bool FULL = decltype(how)::FULL;
            T z[SCAN_STEPS], a[SCAN_STEPS], r[SCAN_STEPS], w[SCAN_STEPS], d[SCAN_STEPS];
            scan_load<T, FULL>(z, ur, p.at, row_bytes, count);
            scan_load<T, FULL>(a, ur, p.at + p.block, row_bytes, count);
            scan_load<T, FULL>(r, ur, p.at + 2 * p.block, row_bytes, count);
            scan_load<T, FULL>(w, xr, at_w, w_bytes, count);
            scan_load<T, FULL>(d, dr, p.at, p.block, count);
            float f[SCAN_STEPS], rest[SCAN_STEPS], e[SCAN_STEPS], gap[SCAN_STEPS], A = 1.f, D = 0.f, dc;
            float c = FULL || count > 0 ? states[((size_t)p.b * g.saved + t0 / SCAN_STEPS) * H + p.col] : 0.f;
#pragma unroll
            for (int i = 0; i < SCAN_STEPS; ++i) {
                if (!scan_in<FULL>(i, count)) {
                    if (t0 + i < p.last) {
                        for (int k = 0; k < 3; ++k) scan_put<T>(0.f, out, p.at + k * p.block, i * row_bytes);
                        scan_put<T>(0.f, out_w, at_w, i * w_bytes);
                    }
                    continue;
                }
                ScanStep<PRECISE> s;
                s.make(c, value_of(z[i]), value_of(a[i]), bf, value_of(r[i]), br, value_of(w[i]), value_of(d[i]));
                f[i] = s.f, rest[i] = s.rest, e[i] = s.e, gap[i] = s.gap;
                sum_r += s.d_r;
                scan_put<T>(s.d_r, out, p.at + 2 * p.block, i * row_bytes);
                scan_put<T>(s.d_w, out_w, at_w, i * w_bytes);
            }
#pragma unroll
            for (int i = SCAN_STEPS - 1; i >= 0; --i) {
                if (!scan_in<FULL>(i, count)) continue;
                D = (D + e[i]) * f[i];
                A *= f[i];
            }
            if (p.waves > 1) {
                sums[parity][p.wave][p.lane] = make_float2(A, D);
                barrier_anywhere();
                dc = d_in;
                for (int j = p.waves - 1; j >= 0; --j) {
                    const float2 q = sums[parity][j][p.lane];
                    d_in = fmaf(q.x, d_in, q.y);
                    if (j - 1 == p.wave) dc = d_in;
                }
            } else {
                dc = d_in, d_in = fmaf(A, d_in, D);
            }
#pragma unroll
            for (int i = SCAN_STEPS - 1; i >= 0; --i) {
                if (!scan_in<FULL>(i, count)) continue;
                const float full = dc + e[i], d_f = full * gap[i];
                sum_f += d_f;
                dc = full * f[i];
                scan_put<T>(full * rest[i], out, p.at, i * row_bytes);
                scan_put<T>(d_f, out, p.at + p.block, i * row_bytes);
            }
        };
        if (count >= SCAN_STEPS) steps(ScanFull());
        else steps(ScanPart());
    }
    if (dc0 && p.seg == 0 && p.wave == 0 && p.on) dc0[(size_t)p.b * H + p.ch] = d_in;
    if (!db) return;
    // the wavefronts' sums in their order, a row of [2 H] for each sequence and segment
    __syncthreads();
    sums[0][p.wave][p.lane] = make_float2(sum_f, sum_r);
    __syncthreads();
    if (p.wave != 0 || !p.on) return;
    for (int j = 1; j < p.waves; ++j) {
        const float2 q = sums[0][j][p.lane];
        sum_f += q.x;
        sum_r += q.y;
    }
    float *to = db + ((size_t)p.b * g.segments + p.seg) * 2 * H + p.ch;
    to[0] = sum_f;
    to[H] = sum_r;
}

// The gradient's pairs of the last segments, [b][segments-1-segment][channel] (the order they are met in), and dc_last beside them, as above.
template <class T>
__global__ __launch_bounds__(SCAN_MAX_WAVES *WAVE) void sru_scan_backward_pairs_kernel(
    ScanShape g, const T *__restrict__ dh, const float *__restrict__ dc_last, const T *__restrict__ u, int blocks, const float *__restrict__ b_f,
    const float *__restrict__ b_r, const float *__restrict__ states, const int32_t *__restrict__ lengths, float2 *__restrict__ pairs,
    float *__restrict__ dc_copy)
{
    constexpr bool PRECISE = sizeof(T) == 4;
    __shared__ float2 sums[SCAN_MAX_WAVES][WAVE];
    ScanPlace<T> p;
    if (!p.find(g, lengths, g.segments - 1)) return;
    p.seg += 1, p.first += g.seg_steps;                // segment 0 has no one before it
    const size_t H = g.H, row_len = blocks * H;
    const float bf = gate_bias<PRECISE>(b_f ? b_f[p.col] : 0.f), br = gate_bias<PRECISE>(b_r ? b_r[p.col] : 0.f);
    float A = 1.f, D = 0.f;
    const int part = g.seg_steps / p.waves, from = p.first + p.wave * part;
    for (int t0 = from + part - SCAN_STEPS; t0 >= from; t0 -= SCAN_STEPS) {
        const int count = min(p.n - t0, SCAN_STEPS);
        if (count <= 0) continue;
        const size_t row = (size_t)p.b * g.L + t0;
        const scan_rows_t ur = scan_rows(u + row * row_len), dr = scan_rows(dh + row * H);
        const unsigned row_bytes = blocks * p.block;
        auto steps = [&](auto how) {
            constexpr bool FULL = decltype(how)::FULL;
            T z[SCAN_STEPS], a[SCAN_STEPS], r[SCAN_STEPS], d[SCAN_STEPS];
            scan_load<T, FULL>(z, ur, p.at, row_bytes, count);
            scan_load<T, FULL>(a, ur, p.at + p.block, row_bytes, count);
            scan_load<T, FULL>(r, ur, p.at + 2 * p.block, row_bytes, count);
            scan_load<T, FULL>(d, dr, p.at, p.block, count);
            float f[SCAN_STEPS], e[SCAN_STEPS], c = states[((size_t)p.b * g.saved + t0 / SCAN_STEPS) * H + p.col];
#pragma unroll
            for (int i = 0; i < SCAN_STEPS; ++i) {
                if (!scan_in<FULL>(i, count)) continue;
                ScanStep<PRECISE> s;
                s.make(c, value_of(z[i]), value_of(a[i]), bf, value_of(r[i]), br, 0.f, value_of(d[i]));
                f[i] = s.f, e[i] = s.e;
            }
#pragma unroll
            for (int i = SCAN_STEPS - 1; i >= 0; --i) {
                if (!scan_in<FULL>(i, count)) continue;
                D = (D + e[i]) * f[i];
                A *= f[i];
            }
        };
        if (count >= SCAN_STEPS) steps(ScanFull());
        else steps(ScanPart());
    }
    sums[p.wave][p.lane] = make_float2(A, D);
    __syncthreads();
    if (p.wave != p.waves - 1 || !p.on) return;
    for (int j = p.waves - 2; j >= 0; --j) {
        const float2 q = sums[j][p.lane];
        D = fmaf(q.x, D, q.y);
        A *= q.x;
    }
    pairs[((size_t)p.b * (g.segments - 1) + (g.segments - 1 - p.seg)) * H + p.ch] = make_float2(A, D);
    if (p.seg == g.segments - 1) dc_copy[(size_t)p.b * H + p.ch] = dc_last ? dc_last[(size_t)p.b * H + p.ch] : 0.f;
}

// db_f and db_r: 64 channels per workgroup; its wavefronts take the parts' sums in turn, and are added in their order
constexpr int BIAS_WAVES = 16;

__global__ __launch_bounds__(BIAS_WAVES *WAVE) void sru_scan_bias_kernel(const float *__restrict__ db, int parts, int H, float *__restrict__ db_f,
                                                                        float *__restrict__ db_r)
{
    __shared__ float sums[BIAS_WAVES][WAVE];
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const size_t col = (size_t)blockIdx.x * WAVE + lane, width = 2 * (size_t)H;
    float sum = 0.f;
    if (col < width) {
#pragma unroll 8
        for (int i = wave; i < parts; i += BIAS_WAVES) sum += db[i * width + col];
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || col >= width) return;
#pragma unroll
    for (int j = 1; j < BIAS_WAVES; ++j) sum += sums[j][lane];
    float *out = col < (size_t)H ? db_f : db_r;
    if (out) out[col < (size_t)H ? col : col - H] = sum;
}

static int scan_check(const char *who, int B, int L, int H, int n_blocks, int dtype, const void *x)
{
    MOE_REQUIRE(B >= 0 && L >= 0 && H > 0, MOE_ERR_INVALID_ARG, "%s: B=%d L=%d H=%d out of range", who, B, L, H);
    MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, dtype);
    MOE_REQUIRE(n_blocks == 3 || n_blocks == 4, MOE_ERR_INVALID_ARG, "%s: n_blocks=%d (3 with x, 4 without)", who, n_blocks);
    MOE_REQUIRE(n_blocks == 3 || !x, MOE_ERR_INVALID_ARG, "%s: x given beside a fourth block", who);
    MOE_REQUIRE(scan_takes(B, L, H), MOE_ERR_UNSUPPORTED, "%s: B=%d L=%d H=%d too large", who, B, L, H);
    return MOE_OK;
}

// pairs, then the copy of the state that the first workgroup starts from
static size_t scan_pairs_bytes(const ScanShape &g)
{
    return g.segments < 2 ? 0 : ((size_t)g.B * (g.segments - 1) * sizeof(float2) + (size_t)g.B * sizeof(float)) * g.H;
}

static dim3 scan_grid(const ScanShape &g, int segments)
{
    const long long n = (long long)g.B * segments * g.groups, across = n < (1 << 22) ? n : 1 << 22;
    return dim3((unsigned)across, (unsigned)((n + across - 1) / across));
}

}  // namespace moe

using namespace moe;

extern "C" size_t sru_scan_states_bytes(int B, int L, int H)
{
    if (B <= 0 || L <= 0 || H <= 0) return 0;
    return (size_t)B * ((L + SCAN_STEPS - 1) / SCAN_STEPS) * H * sizeof(float);
}

extern "C" size_t sru_scan_workspace_bytes(int B, int L, int H, int dtype)
{
    if (B <= 0 || L < 0 || H <= 0 || !scan_takes(B, L, H)) return 0;
    return scan_pairs_bytes(scan_shape(B, L, H));
}

extern "C" size_t sru_scan_backward_workspace_bytes(int B, int L, int H, int dtype)
{
    if (B <= 0 || L < 0 || H <= 0 || !scan_takes(B, L, H)) return 0;
    const ScanShape g = scan_shape(B, L, H);
    return scan_pairs_bytes(g) + (size_t)B * g.segments * 2 * H * sizeof(float);
}

// FORM(T): the build for a type
#define MOE_SCAN_FORMS(FORM)                    \
    do {                                        \
        if (dtype == MOE_F32) FORM(float);      \
        else FORM(bf16_t);                      \
    } while (0)

extern "C" int sru_scan(const void *u, const void *x, const float *b_f, const float *b_r, const float *c0, const int32_t *lengths, int B,
                        int L, int H, int n_blocks, int dtype, void *h, float *c_last, void *states, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = scan_check("sru_scan", B, L, H, n_blocks, dtype, x);
    if (rc != MOE_OK || B == 0) return rc;
    if (L > 0) {
        MOE_REQUIRE(u && h && (n_blocks == 4 || x), MOE_ERR_INVALID_ARG, "sru_scan: null pointer");
        MOE_REQUIRE(h != u && h != x, MOE_ERR_INVALID_ARG, "sru_scan: h aliases an input");
        MOE_REQUIRE(aligned16(u) && aligned16(x) && aligned16(h) && aligned16(states), MOE_ERR_INVALID_ARG, "sru_scan: tensor misaligned");
    }
    const ScanShape g = scan_shape(B, L, H);
    const size_t need = scan_pairs_bytes(g);
    MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE, "sru_scan: workspace of %zu bytes given, %zu needed",
                ws ? ws_bytes : 0, need);
    hipStream_t st = (hipStream_t)stream;
    float2 *pairs = (float2 *)ws;
    const dim3 threads(g.waves * WAVE);
    if (g.segments > 1) {
        float *copy = (float *)(pairs + (size_t)B * (g.segments - 1) * H);
#define MOE_PAIRS(T)                                                                                                                        \
    hipLaunchKernelGGL((sru_scan_pairs_kernel<T>), scan_grid(g, g.segments - 1), threads, 0, st, g, (const T *)u, n_blocks, b_f, c0, lengths, \
                       pairs, copy)
        MOE_SCAN_FORMS(MOE_PAIRS);
#undef MOE_PAIRS
        MOE_CHECK_LAUNCH("sru_scan");
        c0 = copy;
    }
#define MOE_SCAN(T, HW)                                                                                                                 \
    hipLaunchKernelGGL((sru_scan_kernel<T, HW>), scan_grid(g, g.segments), threads, 0, st, g, (const T *)u, (const T *)x, b_f, b_r, c0, lengths, \
                       pairs, (T *)h, c_last, (float *)states)
#define MOE_MAIN(T)                              \
    do {                                            \
        if (n_blocks == 3) MOE_SCAN(T, true);    \
        else MOE_SCAN(T, false);                 \
    } while (0)
    MOE_SCAN_FORMS(MOE_MAIN);
#undef MOE_MAIN
#undef MOE_SCAN
    MOE_CHECK_LAUNCH("sru_scan");
    return MOE_OK;
}

extern "C" int sru_scan_backward(const void *dh, const float *dc_last, const void *u, const void *x, const float *b_f, const float *b_r,
                                 const void *states, const int32_t *lengths, int B, int L, int H, int n_blocks, int dtype, void *du,
                                 void *dx, float *db_f, float *db_r, float *dc0, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = scan_check("sru_scan_backward", B, L, H, n_blocks, dtype, x);
    if (rc != MOE_OK) return rc;
    MOE_REQUIRE(n_blocks == 3 || !dx, MOE_ERR_INVALID_ARG, "sru_scan_backward: dx given beside a fourth block");
    if (B > 0 && L > 0) {
        MOE_REQUIRE(dh && u && states && du && (n_blocks == 4 || (x && dx)), MOE_ERR_INVALID_ARG, "sru_scan_backward: null pointer");
        MOE_REQUIRE(du != u && du != x && du != dh && (!dx || (dx != u && dx != x && dx != dh && dx != du)), MOE_ERR_INVALID_ARG,
                    "sru_scan_backward: an output aliases another tensor");
        MOE_REQUIRE(aligned16(dh) && aligned16(u) && aligned16(x) && aligned16(states) && aligned16(du) && aligned16(dx), MOE_ERR_INVALID_ARG,
                    "sru_scan_backward: tensor misaligned");
    }
    const size_t need = sru_scan_backward_workspace_bytes(B, L, H, dtype);
    MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE,
                "sru_scan_backward: workspace of %zu bytes given, %zu needed", ws ? ws_bytes : 0, need);
    hipStream_t st = (hipStream_t)stream;
    const ScanShape g = scan_shape(B, L, H);
    float2 *pairs = (float2 *)ws;
    float *db = db_f || db_r ? (float *)((char *)ws + scan_pairs_bytes(g)) : nullptr;
    if (B > 0) {
        const dim3 threads(g.waves * WAVE);
        if (g.segments > 1) {
            float *copy = (float *)(pairs + (size_t)B * (g.segments - 1) * H);
#define MOE_PAIRS(T)                                                                                                                       \
    hipLaunchKernelGGL((sru_scan_backward_pairs_kernel<T>), scan_grid(g, g.segments - 1), threads, 0, st, g, (const T *)dh, dc_last, (const T *)u, \
                       n_blocks, b_f, b_r, (const float *)states, lengths, pairs, copy)
            MOE_SCAN_FORMS(MOE_PAIRS);
#undef MOE_PAIRS
            MOE_CHECK_LAUNCH("sru_scan_backward");
            dc_last = copy;
        }
#define MOE_SCAN(T, HW)                                                                                                                    \
    hipLaunchKernelGGL((sru_scan_backward_kernel<T, HW>), scan_grid(g, g.segments), threads, 0, st, g, (const T *)dh, dc_last, (const T *)u, \
                       (const T *)x, b_f, b_r, (const float *)states, lengths, pairs, (T *)du, (T *)dx, db, dc0)
#define MOE_MAIN(T)                              \
    do {                                            \
        if (n_blocks == 3) MOE_SCAN(T, true);    \
        else MOE_SCAN(T, false);                 \
    } while (0)
        MOE_SCAN_FORMS(MOE_MAIN);
#undef MOE_MAIN
#undef MOE_SCAN
        MOE_CHECK_LAUNCH("sru_scan_backward");
    }
    if (db_f || db_r) {
        const unsigned across = (unsigned)((2 * (size_t)H + WAVE - 1) / WAVE);
        hipLaunchKernelGGL(sru_scan_bias_kernel, dim3(across), dim3(BIAS_WAVES * WAVE), 0, st, db, B * g.segments, H, db_f, db_r);
        MOE_CHECK_LAUNCH("sru_scan_backward");
    }
    return MOE_OK;
}
