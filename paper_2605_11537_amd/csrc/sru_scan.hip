// sru_scan and its gradient: the recurrence of an SRU layer over pre-activations that lie in memory.
//
// c_t = f_t c_{t-1} + b_t composes: a run of steps is a pair (A, C), c_out = A c_in + C, and the pair of two runs is (A2 A1, A2 C1 + C2).
// 1 - A goes along with its own accuracy (ScanRun): a channel that forgets little is all in it.
// The gradient dc_{t-1} = f_t (dc_t + e_t) is the same from the other end.  So a wavefront takes 8 or 16 steps of 64 lanes' channels with
// everything they read in registers, finds its pair from zero, and learns its start from the pairs of the wavefronts before it, through
// LDS: the wavefronts of a workgroup lie one behind the other on the sequence, and a round of them is read once and written once.
// Where sequences and channels alone are too few for the card, every round of a sequence is a workgroup of its own (a tile), and the pairs go
// from tile to tile through memory: see scan_look_back.
//
// Memory binds: 10 bytes a channel and step forward in bfloat16, 18 backward (and half a byte of saved states each), against some 30 and 50 vector
// operations, six of them transcendental.  Measured, bfloat16 with the highway: 64 x 512 x 768 forward 59 us (4.4 TB/s), gradient 107 us (4.3
// TB/s); 2 x 16384 x 768 in tiles 73 us (3.5 TB/s) and 125 us (3.7 TB/s); 1 x 300 x 256 8.4 and 13 us, two and three launches.
// One channel a lane: two (in bfloat16 a 4-byte load) took 65 and 124 us for the first, with half the workgroups and more registers.  The next
// round's rows asked for a round ahead: 70 us, with one workgroup less on a compute unit.  Outputs written past the caches: the calls 6 %
// faster, the products that read them slower by as much.
#include <float.h>

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

// Where a wavefront stands: channels and sequence (its line), for a tile which one, and its place among the line's wavefronts.  A workgroup has
// several lines where one or two wavefronts do for a line's steps.
template <class T>
struct ScanPlace {
    int b, tile, lane, wave, waves, base, n, first, last;   // base: the line's first wavefront in the workgroup; first .. last-1: its steps
    unsigned ch, col;                                       // this lane's channel; one that exists
    unsigned at, block;                                     // its offset in a row of one block, and a block's length, in bytes
    bool on;
    // WHOLE: a tile's eight wavefronts as a constant, where that is no slower (2 x 16384 x 768 bf16: gradient 128 -> 125 us; the forward of 16 steps 72 -> 80)
    template <bool TILES, bool WHOLE>
    __device__ __forceinline__ void find(const ScanShape &g, const int32_t *lengths, unsigned line, int which)
    {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
        waves = WHOLE ? SCAN_MAX_WAVES : g.waves;
        wave = TILES ? w : w & (waves - 1);
        base = w - wave;
        if (!TILES) line = line * g.pack + (w >> g.waves_lg);
        const bool live = TILES || line < (unsigned)g.B * g.groups;     // the last workgroup may have lines to spare
        if (!live) line = 0;
        b = line / (unsigned)g.groups;
        tile = which;
        lane = threadIdx.x % WAVE;
        ch = (line - b * (unsigned)g.groups) * WAVE + lane;
        on = live && ch < (unsigned)g.H;
        col = on ? ch : 0;
        at = on ? ch * (unsigned)sizeof(T) : SCAN_NOWHERE;
        block = g.H * (unsigned)sizeof(T);
        n = lengths ? min(max(lengths[b], 0), g.L) : g.L;
        n = __builtin_amdgcn_readfirstlane(n);
        first = TILES ? tile * waves * g.steps : 0;
        last = TILES ? min(g.L, first + waves * g.steps) : g.L;
    }
};

// A wavefront's steps are all inside the sequence (FULL: no step is asked for), or some are not.
struct ScanFull { static constexpr bool FULL = true; };
struct ScanPart { static constexpr bool FULL = false; };
template <bool FULL>
__device__ __forceinline__ bool scan_in(int i, int count)
{
    if (!FULL) asm("" : "+s"(count));                    // asked each time: sixteen answers kept would spill scalar registers
    return FULL || i < count;
}

// the steps of one column block, the first count of them
template <bool FULL, class T, int STEPS>
__device__ __forceinline__ void scan_load(T (&to)[STEPS], scan_rows_t rows, unsigned lane_at, unsigned row_bytes, int count)
{
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        if (!FULL) to[i] = 0;
        if (scan_in<FULL>(i, count)) to[i] = scan_get<T>(rows, lane_at, i * row_bytes);
    }
}

// c_t from c_{t-1}: f c + (1 - f) z with both gates' own accuracy.  A blend, z + f (c - z), is an operation shorter, but rounds by the larger of the two
// where the gate leaves little of it, and takes an infinity from itself.
template <bool PRECISE>
struct ScanForward {
    float f, in;
    __device__ __forceinline__ float make(float a, float bias, float z)     // -> 1 - f
    {
        float rest;
        gate_of<PRECISE>(a, bias, f, rest);
        in = rest * z;
        return rest;
    }
    __device__ __forceinline__ float next(float c) const { return fmaf(f, c, in); }
};

// What leads from the state before a run to the state behind it: c -> A c + C, R = 1 - A.  Gates near 1 are rounded by 2^-25 each, always the same way
// where they do not change, and a product of them has drifted by as much a step: held against R, whose sum of small shares has its own relative
// accuracy, a state would settle beside where its inputs are (1.1e-3 off after 10^5 steps of f = 1 - e^-9; with R 5e-7).
struct ScanRun {
    float A, R, C;
};
__device__ __forceinline__ ScanRun scan_none() { return {1.f, 0.f, 0.f}; }
// A product that underflows stays above 0: an infinite state times it is that state.
__device__ __forceinline__ float scan_kept(float a) { return fmaxf(a, FLT_TRUE_MIN); }
// a run of steps from its product, its shares and its state from zero
__device__ __forceinline__ ScanRun scan_run(float a, float r, float c) { return {r < 0.5f ? 1.f - r : scan_kept(a), r, c}; }
// a, then b, whose A is above 0
__device__ __forceinline__ ScanRun scan_then(ScanRun a, ScanRun b) { return {b.A * a.A, fmaf(b.R, a.A, a.R), fmaf(b.A, a.C, b.C)}; }
// The state behind it.  c + (C - R c) rounds once by c's last place, where A c + C would round A and the product; an infinite state would be taken from
// itself.
__device__ __forceinline__ float scan_through(ScanRun a, float c)
{
    const float slow = c + fmaf(-a.R, c, a.C), fast = fmaf(scan_kept(a.A), c, a.C);
    return a.R < 0.5f && fabsf(c) <= FLT_MAX ? slow : fast;
}
// In two words: minus R, which has the sign bit even at 0, or A.
__device__ __forceinline__ float2 scan_packed(ScanRun a) { return make_float2(a.R < 0.5f ? -a.R : scan_kept(a.A), a.C); }
__device__ __forceinline__ ScanRun scan_unpacked(float2 p)
{
    const float v = fabsf(p.x), w = 1.f - v;
    const bool r = __float_as_int(p.x) < 0;
    return {r ? w : v, r ? v : w, p.y};
}

// Pairs of tiles in memory: a scan in one pass by decoupled look-back, in an arrangement with runs and stretches of tiles.  A pair is one word of 64 bits, written and read whole by atomic operations of device scope (the eight L2 caches do
// not see each other's ordinary writes), and SCAN_UNKNOWN until then: the word is its own flag, so no order between two words is relied on.
// A workgroup draws its tile with a ticket, tile 0 of all chains first, and waits only for tiles whose tickets were drawn before its own: their
// workgroups run already, and publish their own pair before they wait themselves.  So the tile of the lowest unfinished ticket waits for no one,
// and every wait ends.  (A wait gives up after SCAN_PATIENCE looks, some seconds, and makes its outputs NaN: that takes a card that does not run
// what it has begun.)
// To find its start a tile takes the pairs of the tiles before it in its run of SCAN_RUN, the pairs of the whole runs before that one in its
// stretch of SCAN_RUN runs, and the state at the stretch's start: at most 15 + 15 + 1 words a channel however long the sequence, all in flight at
// once, and always folded in the same order.
struct ScanChain {
    unsigned long long *tiles, *runs, *stretches;       // of this chain, [place][lane]
    __device__ __forceinline__ void find(const ScanShape &g, unsigned long long *words, unsigned line)
    {
        const size_t runs_of = g.runs, stretches_of = g.stretches, chains = (size_t)g.B * g.groups;
        tiles = words + (size_t)line * g.tiles * WAVE;
        runs = words + (chains * g.tiles + line * runs_of) * WAVE;
        stretches = words + (chains * (g.tiles + runs_of) + line * stretches_of) * WAVE;
    }
};

__device__ __forceinline__ void scan_publish(unsigned long long *word, float2 pair)
{
    unsigned long long v = __builtin_bit_cast(unsigned long long, pair);
    if (v == SCAN_UNKNOWN) v = 0x7fc000007fc00000ull;    // two NaNs of that very pattern: two other NaNs
    __hip_atomic_store(word, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long scan_look(const unsigned long long *word)
{
    return __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 scan_await(const unsigned long long *word, unsigned long long v)
{
    for (int i = 0; i < SCAN_PATIENCE && __any(v == SCAN_UNKNOWN); ++i) {
        __builtin_amdgcn_s_sleep(1);
        v = scan_look(word);
    }
    return __builtin_bit_cast(float2, v);                // what never came is two NaNs
}
// the pairs of up to two neighbours, the first count of them
__device__ __forceinline__ ScanRun scan_await_two(const unsigned long long *words, unsigned long long v0, unsigned long long v1, int count)
{
    ScanRun a = scan_none();
    if (count > 0) a = scan_unpacked(scan_await(words, v0));
    if (count > 1) a = scan_then(a, scan_unpacked(scan_await(words + WAVE, v1)));
    a.A = scan_kept(a.A);
    return a;
}

// The state at the start of the tile at `at` (its place in the order of the recurrence), from the sequence's own start and the tile's pair, which
// every wavefront knows.  Each wavefront looks for two tiles and two runs.
__device__ float scan_look_back(const ScanChain &chain, int tiles, int at, int lane, int wave, ScanRun own, float start,
                                ScanRun (*of_tiles)[WAVE], ScanRun (*of_runs)[WAVE])
{
    own.A = scan_kept(own.A);
    const int run = at / SCAN_RUN, in_run = at % SCAN_RUN, stretch = run / SCAN_RUN, in_stretch = run % SCAN_RUN;
    const bool last = at + 1 == tiles;
    if (wave == 0 && !last && in_run + 1 < SCAN_RUN) scan_publish(chain.tiles + (size_t)at * WAVE + lane, scan_packed(own));
    const unsigned long long *t = chain.tiles + ((size_t)run * SCAN_RUN + 2 * wave) * WAVE + lane;
    const unsigned long long *r = chain.runs + ((size_t)stretch * SCAN_RUN + 2 * wave) * WAVE + lane;
    const unsigned long long *s = chain.stretches + (size_t)(stretch > 0 ? stretch - 1 : 0) * WAVE + lane;
    const int n_t = min(max(in_run - 2 * wave, 0), 2), n_r = min(max(in_stretch - 2 * wave, 0), 2);
    unsigned long long t0 = 0, t1 = 0, r0 = 0, r1 = 0, s0 = 0;
    if (n_t > 0) t0 = scan_look(t);
    if (n_t > 1) t1 = scan_look(t + WAVE);
    if (n_r > 0) r0 = scan_look(r);
    if (n_r > 1) r1 = scan_look(r + WAVE);
    if (stretch > 0) s0 = scan_look(s);
    of_tiles[wave][lane] = scan_await_two(t, t0, t1, n_t);
    __syncthreads();
    ScanRun before = scan_none();
    for (int w = 0; w < SCAN_MAX_WAVES; ++w) before = scan_then(before, of_tiles[w][lane]);
    const ScanRun whole = scan_then(before, own);        // a run's pair needs no other run's, and is out before one is waited for
    const bool ends = !last && in_run + 1 == SCAN_RUN, ends_stretch = ends && in_stretch + 1 == SCAN_RUN;
    if (wave == 0 && ends && !ends_stretch) scan_publish(chain.runs + (size_t)run * WAVE + lane, scan_packed(whole));
    of_runs[wave][lane] = scan_await_two(r, r0, r1, n_r);
    float c = stretch > 0 ? scan_await(s, s0).y : start;
    __syncthreads();
    ScanRun runs_before = scan_none();
    for (int w = 0; w < SCAN_MAX_WAVES; ++w) runs_before = scan_then(runs_before, of_runs[w][lane]);
    c = scan_through(runs_before, c);
    if (wave == 0 && ends_stretch) scan_publish(chain.stretches + (size_t)stretch * WAVE + lane, make_float2(0.f, scan_through(whole, c)));
    return scan_through(before, c);
}

// Before the tiles: every word unknown, no ticket drawn; the state at the start beside them, since c_last may be c0 and is written while others
// still read.
__global__ __launch_bounds__(SCAN_CLEAR_THREADS) void sru_scan_clear_kernel(unsigned long long *__restrict__ words, size_t count,
                                                                            const float *__restrict__ start, float *__restrict__ copy, size_t channels,
                                                                            unsigned *__restrict__ ticket, unsigned blocks)
{
    const size_t first = (size_t)blockIdx.x * SCAN_CLEAR_THREADS + threadIdx.x, step = (size_t)blocks * SCAN_CLEAR_THREADS;
    for (size_t i = first; i < count; i += step) words[i] = SCAN_UNKNOWN;
    for (size_t i = first; i < channels; i += step) copy[i] = start ? start[i] : 0.f;
    if (first == 0) *ticket = 0;
}

// the workgroup's number or, with tiles, its line and its place in the chain
template <bool TILES>
__device__ __forceinline__ bool scan_draw(const ScanShape &g, unsigned *ticket, unsigned *drawn, unsigned &line, int &at)
{
    if (!TILES) {
        line = blockIdx.y * g.across + blockIdx.x, at = 0;
        return line < (unsigned)g.workgroups;
    }
    const unsigned lines = (unsigned)g.B * g.groups;
    if (threadIdx.x == 0) *drawn = atomicAdd(ticket, 1u);
    __syncthreads();
    const unsigned t = __builtin_amdgcn_readfirstlane(*drawn);
    at = t / lines;
    line = t - at * lines;
    return at < g.tiles;
}

template <class T, bool HIGHWAY, bool TILES, int STEPS>
__global__ __launch_bounds__(SCAN_MAX_WAVES *WAVE, 4) void sru_scan_kernel(ScanShape g, const T *__restrict__ u, const T *__restrict__ x,
                                                                       const float *__restrict__ b_f, const float *__restrict__ b_r,
                                                                       const float *c0, const int32_t *__restrict__ lengths,
                                                                       unsigned *ticket, unsigned long long *words, T *__restrict__ h,
                                                                       float *c_last, float *__restrict__ states)
{
    constexpr bool PRECISE = sizeof(T) == 4;
    constexpr int K = HIGHWAY ? 3 : 4;
    __shared__ ScanRun sums[3][SCAN_MAX_WAVES][WAVE];
    __shared__ unsigned drawn;
    unsigned line;
    int at;
    if (!scan_draw<TILES>(g, ticket, &drawn, line, at)) return;
    ScanPlace<T> p;
    p.template find<TILES, TILES && STEPS == SCAN_SAVED>(g, lengths, line, at);
    ScanChain chain;
    if (TILES) chain.find(g, words, line);
    const size_t H = g.H, row_len = K * H;
    const float bf = gate_bias<PRECISE>(b_f ? b_f[p.col] : 0.f), br = gate_bias<PRECISE>(b_r ? b_r[p.col] : 0.f);
    float c_in = c0 ? c0[(size_t)p.b * H + p.col] : 0.f;
    const int round = p.waves * STEPS;
    for (int t = p.first, parity = 0; t < p.last; t += round, parity ^= 1) {
        const int t0 = t + p.wave * STEPS, count = min(p.n - t0, STEPS);    // this wavefront's steps inside the sequence
        const size_t row = (size_t)p.b * g.L + t0;
        T z[STEPS], a[STEPS], r[STEPS], w[STEPS];
        ScanForward<PRECISE> s[STEPS];
        float A = 1.f, R = 0.f, C = 0.f;
        auto gates = [&](auto how) {
            constexpr bool FULL = decltype(how)::FULL;
            const scan_rows_t ur = scan_rows(u + row * row_len), xr = HIGHWAY ? scan_rows(x + row * H) : ur;
            scan_load<FULL>(z, ur, p.at, K * p.block, count);
            scan_load<FULL>(a, ur, p.at + p.block, K * p.block, count);
            scan_load<FULL>(r, ur, p.at + 2 * p.block, K * p.block, count);
            if (HIGHWAY) scan_load<FULL>(w, xr, p.at, p.block, count);
            else scan_load<FULL>(w, ur, p.at + 3 * p.block, K * p.block, count);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if (!scan_in<FULL>(i, count)) continue;
                R = fmaf(s[i].make(value_of(a[i]), bf, value_of(z[i])), A, R);
                A *= s[i].f;
                C = s[i].next(C);
            }
        };
        if (count >= STEPS) gates(ScanFull());
        else gates(ScanPart());
        sums[parity][p.base + p.wave][p.lane] = scan_run(A, R, C);
        __syncthreads();
        ScanRun all = scan_none(), before = all;
        for (int j = 0; j < p.waves; ++j) {
            if (j == p.wave) before = all;
            all = scan_then(all, sums[parity][p.base + j][p.lane]);
        }
        if (TILES) c_in = scan_look_back(chain, g.tiles, at, p.lane, p.wave, all, c_in, sums[1], sums[2]);
        float c = scan_through(before, c_in);
        c_in = scan_through(all, c_in);
        auto outputs = [&](auto how) {
            constexpr bool FULL = decltype(how)::FULL;
            const scan_rows_t hr = scan_rows(h + row * H);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if (i % SCAN_SAVED == 0 && states && (FULL || t0 + i < g.L) && p.on)
                    states[((size_t)p.b * g.saved + (t0 + i) / SCAN_SAVED) * H + p.ch] = c;
                if (!scan_in<FULL>(i, count)) {
                    if (t0 + i < p.last) scan_put<T>(0.f, hr, p.at, i * p.block);
                    continue;
                }
                c = s[i].next(c);
                const float wv = value_of(w[i]), t = tanh_of<PRECISE>(c);
                float on, rest;
                gate_of<PRECISE>(value_of(r[i]), br, on, rest);
                scan_put<T>(fmaf(on, t, rest * wv), hr, p.at, i * p.block);
            }
        };
        if (count >= STEPS) outputs(ScanFull());
        else outputs(ScanPart());
    }
    if (c_last && p.tile == g.tiles - 1 && p.wave == 0 && p.on) c_last[(size_t)p.b * H + p.ch] = c_in;
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

template <class T, bool HIGHWAY, bool TILES, int STEPS>
__global__ __launch_bounds__(SCAN_MAX_WAVES *WAVE, 4) void sru_scan_backward_kernel(
    ScanShape g, const T *__restrict__ dh, const float *dc_last, const T *__restrict__ u, const T *__restrict__ x, const float *__restrict__ b_f,
    const float *__restrict__ b_r, const float *__restrict__ states, const int32_t *__restrict__ lengths, unsigned *ticket,
    unsigned long long *words, T *__restrict__ du, T *__restrict__ dx, float *__restrict__ db, float *dc0)
{
    constexpr bool PRECISE = sizeof(T) == 4;
    constexpr int K = HIGHWAY ? 3 : 4;
    __shared__ alignas(sizeof(float2)) ScanRun sums[3][SCAN_MAX_WAVES][WAVE];      // the biases' sums too, in pairs
    __shared__ unsigned drawn;
    unsigned line;
    int at;
    if (!scan_draw<TILES>(g, ticket, &drawn, line, at)) return;
    ScanPlace<T> p;
    p.template find<TILES, TILES && STEPS == SCAN_SAVED>(g, lengths, line, g.tiles - 1 - at);
    ScanChain chain;
    if (TILES) chain.find(g, words, line);
    const size_t H = g.H, row_len = K * H;
    const float bf = gate_bias<PRECISE>(b_f ? b_f[p.col] : 0.f), br = gate_bias<PRECISE>(b_r ? b_r[p.col] : 0.f);
    float sum_f = 0.f, sum_r = 0.f, d_in = dc_last ? dc_last[(size_t)p.b * H + p.col] : 0.f;
    const int round = p.waves * STEPS, rounds = p.last > p.first ? (p.last - p.first + round - 1) / round : 0;
    for (int back = rounds - 1, parity = 0; back >= 0; --back, parity ^= 1) {
        const int t0 = p.first + back * round + p.wave * STEPS, count = min(p.n - t0, STEPS);
        const size_t row = (size_t)p.b * g.L + t0;
        const scan_rows_t ur = scan_rows(u + row * row_len), dr = scan_rows(dh + row * H), out = scan_rows(du + row * row_len);
        const scan_rows_t xr = HIGHWAY ? scan_rows(x + row * H) : ur, out_w = HIGHWAY ? scan_rows(dx + row * H) : out;
        const unsigned at_w = HIGHWAY ? p.at : p.at + 3 * p.block, row_bytes = K * p.block, w_bytes = HIGHWAY ? p.block : row_bytes;
        float f[STEPS], rest[STEPS], e[STEPS], gap[STEPS], A = 1.f, R = 0.f, D = 0.f;
        auto forward = [&](auto how) {
            constexpr bool FULL = decltype(how)::FULL;
            T z[STEPS], a[STEPS], r[STEPS], w[STEPS], d[STEPS];
            scan_load<FULL>(z, ur, p.at, row_bytes, count);
            scan_load<FULL>(a, ur, p.at + p.block, row_bytes, count);
            scan_load<FULL>(r, ur, p.at + 2 * p.block, row_bytes, count);
            scan_load<FULL>(w, xr, at_w, w_bytes, count);
            scan_load<FULL>(d, dr, p.at, p.block, count);
            float c = FULL || count > 0 ? states[((size_t)p.b * g.saved + t0 / SCAN_SAVED) * H + p.col] : 0.f;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
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
            for (int i = STEPS - 1; i >= 0; --i) {
                if (!scan_in<FULL>(i, count)) continue;
                D = (D + e[i]) * f[i];
                R = fmaf(rest[i], A, R);
                A *= f[i];
            }
        };
        if (count >= STEPS) forward(ScanFull());
        else forward(ScanPart());
        sums[parity][p.base + p.wave][p.lane] = scan_run(A, R, D);
        __syncthreads();
        ScanRun all = scan_none(), before = all;
        for (int j = p.waves - 1; j >= 0; --j) {
            if (j == p.wave) before = all;
            all = scan_then(all, sums[parity][p.base + j][p.lane]);
        }
        if (TILES) d_in = scan_look_back(chain, g.tiles, at, p.lane, p.wave, all, d_in, sums[1], sums[2]);
        float dc = scan_through(before, d_in);
        d_in = scan_through(all, d_in);
        auto backward = [&](auto how) {
            constexpr bool FULL = decltype(how)::FULL;
#pragma unroll
            for (int i = STEPS - 1; i >= 0; --i) {
                if (!scan_in<FULL>(i, count)) continue;
                const float full = dc + e[i], d_f = full * gap[i];
                sum_f += d_f;
                dc = full * f[i];
                scan_put<T>(full * rest[i], out, p.at, i * row_bytes);
                scan_put<T>(d_f, out, p.at + p.block, i * row_bytes);
            }
        };
        if (count >= STEPS) backward(ScanFull());
        else backward(ScanPart());
    }
    if (dc0 && p.tile == 0 && p.wave == 0 && p.on) dc0[(size_t)p.b * H + p.ch] = d_in;
    if (!db) return;
    // the wavefronts' sums in their order, a row of [2 H] for each sequence and tile
    __syncthreads();
    float2 (*const biases)[WAVE] = reinterpret_cast<float2 (*)[WAVE]>(sums);
    biases[p.base + p.wave][p.lane] = make_float2(sum_f, sum_r);
    __syncthreads();
    if (p.wave != 0 || !p.on) return;
    for (int j = 1; j < p.waves; ++j) {
        const float2 q = biases[p.base + j][p.lane];
        sum_f += q.x;
        sum_r += q.y;
    }
    float *to = db + ((size_t)p.b * g.tiles + p.tile) * 2 * H + p.ch;
    to[0] = sum_f;
    to[H] = sum_r;
}

// db_f and db_r: 32 columns per workgroup; 32 groups of lanes take the parts' sums in turn and are added in their order
constexpr int BIAS_LANES = 32, BIAS_GROUPS = 32;

__global__ __launch_bounds__(BIAS_LANES *BIAS_GROUPS) void sru_scan_bias_kernel(const float *__restrict__ db, int parts, int H,
                                                                               float *__restrict__ db_f, float *__restrict__ db_r)
{
    __shared__ float sums[BIAS_GROUPS][BIAS_LANES];
    const int lane = threadIdx.x % BIAS_LANES, group = threadIdx.x / BIAS_LANES;
    const size_t col = (size_t)blockIdx.x * BIAS_LANES + lane, width = 2 * (size_t)H;
    float sum = 0.f;
    if (col < width) {
#pragma unroll 16
        for (int i = group; i < parts; i += BIAS_GROUPS) sum += db[i * width + col];
    }
    sums[group][lane] = sum;
    __syncthreads();
    if (group != 0 || col >= width) return;
#pragma unroll
    for (int j = 1; j < BIAS_GROUPS; ++j) sum += sums[j][lane];
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

// the workspace of tiles: words, the copy of the state at the start, the ticket
static size_t scan_words(const ScanShape &g) { return g.tiles == 1 ? 0 : (size_t)g.B * g.groups * (g.tiles + g.runs + g.stretches) * WAVE; }
static size_t scan_tiles_bytes(const ScanShape &g)
{
    return g.tiles == 1 ? 0 : align_up(scan_words(g) * sizeof(unsigned long long) + (size_t)g.B * g.H * sizeof(float) + sizeof(unsigned), 16);
}

struct ScanTiles {
    unsigned long long *words;
    float *copy;
    unsigned *ticket;
};
static ScanTiles scan_tiles(const ScanShape &g, void *ws)
{
    ScanTiles t = {(unsigned long long *)ws, nullptr, nullptr};
    t.copy = (float *)(t.words + scan_words(g));
    t.ticket = (unsigned *)(t.copy + (size_t)g.B * g.H);
    return t;
}
// prepares the tiles of a call; start becomes the copy
static int scan_clear(const ScanShape &g, const ScanTiles &t, const float *&start, hipStream_t st, const char *who)
{
    if (g.tiles == 1) return MOE_OK;
    const size_t words = scan_words(g), channels = (size_t)g.B * g.H, wanted = (words + SCAN_CLEAR_THREADS - 1) / SCAN_CLEAR_THREADS;
    const unsigned blocks = wanted < 2048 ? (unsigned)wanted : 2048;
    hipLaunchKernelGGL(sru_scan_clear_kernel, dim3(blocks), dim3(SCAN_CLEAR_THREADS), 0, st, t.words, words, start, t.copy, channels, t.ticket, blocks);
    MOE_CHECK_LAUNCH(who);
    start = t.copy;
    return MOE_OK;
}

static dim3 scan_grid(const ScanShape &g)
{
    return dim3((unsigned)g.across, (unsigned)((g.workgroups + g.across - 1) / g.across));
}

}  // namespace moe

using namespace moe;

extern "C" size_t sru_scan_states_bytes(int B, int L, int H)
{
    if (B <= 0 || L <= 0 || H <= 0) return 0;
    return (size_t)B * ((L + SCAN_SAVED - 1) / SCAN_SAVED) * H * sizeof(float);
}

extern "C" size_t sru_scan_workspace_bytes(int B, int L, int H, int dtype)
{
    if (B <= 0 || L < 0 || H <= 0 || !scan_takes(B, L, H)) return 0;
    return scan_tiles_bytes(scan_forward_shape(B, L, H));
}

extern "C" size_t sru_scan_backward_workspace_bytes(int B, int L, int H, int dtype)
{
    if (B <= 0 || L < 0 || H <= 0 || !scan_takes(B, L, H)) return 0;
    const ScanShape g = scan_backward_shape(B, L, H);
    return scan_tiles_bytes(g) + (size_t)B * g.tiles * 2 * H * sizeof(float);
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
    const ScanShape g = scan_forward_shape(B, L, H);
    const size_t need = scan_tiles_bytes(g);
    MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE, "sru_scan: workspace of %zu bytes given, %zu needed",
                ws ? ws_bytes : 0, need);
    hipStream_t st = (hipStream_t)stream;
    const ScanTiles tiles = scan_tiles(g, ws);
    const int cleared = scan_clear(g, tiles, c0, st, "sru_scan");
    if (cleared != MOE_OK) return cleared;
#define MOE_SCAN(T, HW)                                                                                                                          \
    hipLaunchKernelGGL((g.tiles > 1 ? (g.steps == SCAN_LONG ? sru_scan_kernel<T, HW, true, SCAN_LONG> : sru_scan_kernel<T, HW, true, SCAN_SAVED>) \
                        : g.steps == SCAN_LONG  ? sru_scan_kernel<T, HW, false, SCAN_LONG>                                                        \
                        : g.steps == SCAN_SAVED ? sru_scan_kernel<T, HW, false, SCAN_SAVED>                                                       \
                                                : sru_scan_kernel<T, HW, false, 1>),                                                              \
                       scan_grid(g), dim3(g.waves *g.pack *WAVE), 0, st, g, (const T *)u, (const T *)x, b_f, b_r, c0, lengths, tiles.ticket,      \
                       tiles.words, (T *)h, c_last, (float *)states)
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
    const ScanShape g = scan_backward_shape(B, L, H);
    const ScanTiles tiles = scan_tiles(g, ws);
    float *db = db_f || db_r ? (float *)((char *)ws + scan_tiles_bytes(g)) : nullptr;
    if (B > 0) {
        const int cleared = scan_clear(g, tiles, dc_last, st, "sru_scan_backward");
        if (cleared != MOE_OK) return cleared;
#define MOE_SCAN(T, HW)                                                                                                                             \
    hipLaunchKernelGGL((g.tiles > 1             ? sru_scan_backward_kernel<T, HW, true, SCAN_SAVED>                                                 \
                        : g.steps == SCAN_SAVED ? sru_scan_backward_kernel<T, HW, false, SCAN_SAVED>                                                \
                                                : sru_scan_backward_kernel<T, HW, false, 1>),                                                       \
                       scan_grid(g), dim3(g.waves *g.pack *WAVE), 0, st, g, (const T *)dh, dc_last, (const T *)u, (const T *)x, b_f, b_r,           \
                       (const float *)states, lengths, tiles.ticket, tiles.words, (T *)du, (T *)dx, db, dc0)
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
        const unsigned across = (unsigned)((2 * (size_t)H + BIAS_LANES - 1) / BIAS_LANES);
        hipLaunchKernelGGL(sru_scan_bias_kernel, dim3(across), dim3(BIAS_LANES * BIAS_GROUPS), 0, st, db, B * g.tiles, H, db_f, db_r);
        MOE_CHECK_LAUNCH("sru_scan_backward");
    }
    return MOE_OK;
}
