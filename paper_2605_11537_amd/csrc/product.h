// Tiles of matrix products whose operands lie in memory as their owners keep them: D[m][n] = sum over k of A(m, k) B(n, k), in bfloat16 or binary32,
// summed in binary32.  Each operand has k along its rows (ALONG_K: element (m, k) at m * ld + k) or rows along k (ACROSS_K: at k * ld + m), so that the
// products of a layer and of its gradient need no transposed copies.
//
// A stage is 128 bytes of k for every row of the two tiles (64 k of bfloat16, 32 of binary32), and goes from memory to LDS directly, 16 bytes a lane.  It
// lies there as the loads bring it, in the order of the operand in memory, its pieces permuted by an XOR so that the reads of a fragment meet no bank
// twice:
//   ALONG_K   row r's 16-byte piece p (of 8) lies at r * 8 + (p ^ (r >> 1 & 7)); a fragment is one 16-byte read a lane
//   ACROSS_K  bfloat16: the 32-byte piece q of step k lies at q ^ (k & 3 | k >> 1 & 4) of that step's row; a fragment is two reads that transpose 4 k x
//             16 rows among 16 lanes.  binary32: the 64-byte piece q lies at q ^ (k >> 2 & 3); a fragment is four reads of 4 bytes.  (Rows of less than
//             256 bytes have fewer pieces to permute.)
// The order of k inside a matrix instruction is free as long as both operands have the same: lane group g holds k = 8 g .. 8 g + 7 of 32 in bfloat16,
// and in binary32 instruction j takes k = 4 g + j of 16.
//
// Operands are read as buffers: what lies behind the last row of k or of the tile comes as zero.  ALONG_K the pieces behind the last k are sent out of
// the buffer's range.  Both operands are zero there, so that memory which holds a NaN does not reach a sum.
#pragma once
#include "common.h"

namespace moe {

typedef unsigned product_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned product_u32x2 __attribute__((ext_vector_type(2)));
typedef float product_f32x4 __attribute__((ext_vector_type(4)));
typedef short product_s16x4 __attribute__((ext_vector_type(4)));
typedef short product_s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 product_bf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char product_lds_t;
typedef __attribute__((address_space(3))) product_s16x4 product_lds_s16x4;

enum Order { ALONG_K, ACROSS_K };

template <class T>
struct Fragment;
template <>
struct Fragment<bf16_t> {
    typedef product_s16x8 type;
    static constexpr int K = 32;               // k of a step: two to a stage
};
template <>
struct Fragment<float> {
    typedef product_f32x4 type;
    static constexpr int K = 16;
};

__device__ __forceinline__ void product_mma(product_f32x4 &d, product_s16x8 b, product_s16x8 a)
{
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(product_bf16x8, b), __builtin_bit_cast(product_bf16x8, a), d, 0, 0, 0);
}
__device__ __forceinline__ void product_mma(product_f32x4 &d, product_f32x4 b, product_f32x4 a)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) d = __builtin_amdgcn_mfma_f32_16x16x4f32(b[j], a[j], d, 0, 0, 0);
}

// 1 KB from a buffer to LDS: lane l's 16 bytes at `at` go to lds + 16 l.  No register is written, so nothing has to wait but the readers of that LDS.
// Inline assembly: in front of every LDS read that the compiler sees it would wait for all such loads, those of later stages too.
// The assembler adds no waits by itself: m0 may be read one instruction after it is written, a buffer's registers five after a vector instruction has (as one
// that makes a value scalar, or brings a spilled register back).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(product_u32x4 buffer, unsigned at, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(at), "s"(buffer) : "m0");
}
#pragma clang diagnostic pop

// where one operand's tile begins in memory: its first row's (ALONG_K: first k's) address and how many rows (ALONG_K) or k (ACROSS_K) are there
struct Source {
    uint64_t base;
    unsigned records;                          // bytes from base that may be read
};

template <class T, Order ORDER, int ROWS, int WAVES>
struct Operand {
    static constexpr int ROW = 128;            // bytes of k that a stage holds for every row
    typedef typename Fragment<T>::type fragment;
    static constexpr int STAGE_K = ROW / (int)sizeof(T), STEPS = STAGE_K / Fragment<T>::K;
    static constexpr int BYTES = ROWS * ROW;
    static constexpr int LOADS = BYTES / 1024;
    static constexpr int MINE = LOADS >= WAVES ? LOADS / WAVES : 1;       // with fewer loads than wavefronts some are made twice, the same bytes
    static_assert(LOADS % WAVES == 0 || WAVES % LOADS == 0, "every wavefront has the same number of loads");
    static constexpr int PIECES = ROWS * (int)sizeof(T) / 16;             // ACROSS_K: 16-byte pieces of a step of k
    static_assert(ORDER == ALONG_K || ROWS >= 32, "what the XOR permutes");

    unsigned at[MINE];                         // byte offsets of this lane's pieces from the stage's base
    unsigned k_of[MINE];                       // ALONG_K: the piece's first k in its stage
    unsigned read_at[STEPS];                   // where this lane's fragment of row block 0 begins in a stage, for each of its steps
    unsigned swizzle;                          // ACROSS_K: this lane's XOR

    __device__ __forceinline__ static unsigned permute(unsigned k)
    {
        if (sizeof(T) == 4) return (k >> 2) & (ROWS >= 64 ? 3 : 1);
        if (ROWS >= 128) return (k & 3) | ((k >> 1) & 4);
        if (ROWS >= 64) return ((k >> 1) & 1) | ((k >> 2) & 2);            // rows of 128 bytes: neighbouring k alternate between the halves of the banks
        return (k >> 3) & 1;
    }

    // ALONG_K: the XOR of row r's pieces
    __device__ __forceinline__ static unsigned turn(unsigned r) { return (r >> 1) & 7; }

    // this wavefront's number among those that share the tile
    __device__ __forceinline__ static unsigned wave() { return WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

    // row: this wavefront's first row in the tile
    __device__ __forceinline__ void set_up(unsigned ld_bytes, int row)
    {
        const unsigned lane = threadIdx.x & 63, w = wave();
        const unsigned c = lane & 15, g = lane >> 4;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const unsigned q = ((w * MINE + i) % LOADS) * 64 + lane;
            if (ORDER == ALONG_K) {
                const unsigned r = q >> 3, p = (q & 7) ^ turn(r);
                at[i] = r * ld_bytes + p * 16;
                k_of[i] = p * (16 / sizeof(T));
            } else if (sizeof(T) == 2) {
                const unsigned k = q / PIECES, p = q % PIECES;
                at[i] = k * ld_bytes + (p ^ (permute(k) << 1)) * 16;
            } else {
                const unsigned k = q / PIECES, p = q % PIECES;
                at[i] = k * ld_bytes + (p ^ (permute(k) << 2)) * 16;
            }
        }
        if (ORDER == ALONG_K) {
#pragma unroll
            for (int ks = 0; ks < STEPS; ++ks) read_at[ks] = (row + c) * ROW + (((4 * ks + g) ^ turn(c)) << 4);
            swizzle = 0;
        } else if (sizeof(T) == 2) {
            const unsigned k = 8 * g + (c >> 2);
            swizzle = permute(k) * 32;
#pragma unroll
            for (int ks = 0; ks < STEPS; ++ks) read_at[ks] = (k + 32 * ks) * ROWS * 2 + (c & 3) * 8 + row * 2;
        } else {
            swizzle = permute(4 * g) * 64;
#pragma unroll
            for (int ks = 0; ks < STEPS; ++ks) read_at[ks] = (4 * g + 16 * ks) * ROWS * 4 + c * 4 + row * 4;
        }
    }

    // the buffer of a run's first stage, of k in all, and of the stage behind it with `left` k from there on
    __device__ __forceinline__ static unsigned records_of(Source s, int left, unsigned ld_bytes)
    {
        // ALONG_K every k of a row lies within the row.  ACROSS_K the columns in front of the tile are not in the buffer: the last row ends with the matrix
        return ORDER == ALONG_K ? s.records : ((unsigned)(left < STAGE_K ? left : STAGE_K) - 1) * ld_bytes + s.records;
    }
    __device__ __forceinline__ static product_u32x4 first_buffer(Source s, int k, unsigned ld_bytes)
    {
        product_u32x4 v = {(unsigned)s.base, (unsigned)(s.base >> 32), records_of(s, k, ld_bytes), 0x27000};
#pragma unroll
        for (int i = 0; i < 3; ++i) v[i] = __builtin_amdgcn_readfirstlane(v[i]);      // scalar, whatever the compiler has made of the job
        return v;
    }
    __device__ __forceinline__ static void next_buffer(product_u32x4 &v, int left, unsigned ld_bytes)
    {
        const unsigned by = ORDER == ALONG_K ? ROW : STAGE_K * ld_bytes;
        const uint64_t base = (((uint64_t)v[1] << 32) | v[0]) + by;
        v[0] = (unsigned)base;
        v[1] = (unsigned)(base >> 32);
        if (ORDER == ALONG_K) v[2] -= ROW;
        else if (left < STAGE_K) v[2] -= (STAGE_K - left) * ld_bytes;                 // the run's last
    }
    // this wavefront's load i of a stage; left: k from the stage's first on
    __device__ __forceinline__ void load(int i, product_u32x4 buffer, int left, unsigned lds) const
    {
        const unsigned w = wave();
        unsigned a = at[i];
        if (ORDER == ALONG_K) a = (int)k_of[i] < left ? a : 0x80000000u;
        load_to_lds(buffer, a, lds + ((w * MINE + i) % LOADS) * 1024);
    }

    // fragment of rows 16 rb .. 16 rb + 15 of this wavefront's, step ks of the stage at lds
    __device__ __forceinline__ fragment read(product_lds_t *lds, int rb, int ks) const
    {
        if constexpr (ORDER == ALONG_K) {
            return *reinterpret_cast<__attribute__((address_space(3))) fragment *>(lds + read_at[ks] + rb * 16 * ROW);
        } else if constexpr (sizeof(T) == 2) {
            // row is a multiple of 16 rows, so that the XOR meets the place of the 32-byte piece alone
            const unsigned a = (read_at[ks] + rb * 32) ^ swizzle;
            const product_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((product_lds_s16x4 *)(lds + a));
            const product_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((product_lds_s16x4 *)(lds + a + 4 * ROWS * 2));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            const unsigned a = (read_at[ks] + rb * 64) ^ swizzle;
            fragment f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<__attribute__((address_space(3))) float *>(lds + a + j * ROWS * 4);
            return f;
        }
    }
};

// four neighbouring values of a row, rounded once
__device__ __forceinline__ void store4(float *p, product_f32x4 v) { *reinterpret_cast<product_f32x4 *>(p) = v; }
__device__ __forceinline__ void store4(bf16_t *p, product_f32x4 v)
{
    uint2 two;
    two.x = pack_bf16x2(v[0], v[1]);
    two.y = pack_bf16x2(v[2], v[3]);
    *reinterpret_cast<uint2 *>(p) = two;
}

// What a workgroup computes next: a tile of D, from one or two runs of k (the second behind the first in the same sum).
struct Job {
    Source a[2], b[2];                         // of the runs; with two column halves b holds the halves' and there is one run
    int k, runs;                               // k of a run, 0 .. : D = 0 without
    int m0, n0, rows, columns;                 // the tile's origin in D and how much of it there is
    int group;                                 // expert, or part of a split sum
    size_t block;
};

__device__ __forceinline__ Source source_along(const void *p, size_t first_byte, unsigned ld_bytes, int rows, int most)
{
    return {reinterpret_cast<uint64_t>(p) + first_byte, (unsigned)(rows < most ? rows : most) * ld_bytes};
}
__device__ __forceinline__ Source source_across(const void *p, size_t first_byte, unsigned ld_bytes, unsigned column_bytes)
{
    return {reinterpret_cast<uint64_t>(p) + first_byte + column_bytes, ld_bytes - column_bytes};
}

// BM x BN of D by WM x WN wavefronts.  HALVES = 2: columns come from two operands of BN / 2 rows each, and a wavefront has the same columns of both.
// A ring of STAGES stages: the loop waits for a stage, asks for the one STAGES - 1 further on, which may be the next tile's, and
// multiplies, so that a tile's first stages land while the one before is written.
// BLOCK_K: A lies ALONG_K in blocks of so many k, j.block bytes from one to the next.
template <class T_, Order OA, Order OB, int BM_, int BN_, int WM, int WN, int HALVES_ = 1, int STAGES = 2, int BLOCK_K = 0>
struct Tile {
    typedef T_ T;
    static constexpr int BM = BM_, BN = BN_, HALVES = HALVES_, WAVES = WM * WN, THREADS = WAVES * WAVE;
    static constexpr int HALF_N = BN / HALVES, WAVE_M = BM / WM, WAVE_N = HALF_N / WN;       // rows and columns (of a half) of a wavefront
    static constexpr int MB = WAVE_M / 16, NB = WAVE_N / 16;                                 // blocks of 16
    static constexpr Order B_ORDER = OB;
    typedef Operand<T, OA, BM, WAVES> A;
    typedef Operand<T, OB, HALF_N, WAVES> B;
    static constexpr int STAGE_K = A::STAGE_K;
    static constexpr int STAGE = A::BYTES + HALVES * B::BYTES, LDS = STAGES * STAGE;
    static constexpr int LOADS = A::MINE + HALVES * B::MINE;                                 // of a wavefront for a stage

    typedef product_f32x4 Sums[HALVES][MB][NB];          // register i of [h][mb][nb]: row of_row(mb), column of_column(nb) + i of half h

    // binary32: sums of eight stages (256 k) are added up by themselves.  One sum over 5632 k was off by 1.1e-6 of the result, a library's by 6e-7.
    static constexpr int APART = sizeof(T) == 4 ? 8 : 0;
    template <class F>
    __device__ __forceinline__ static void each(Sums &x, F &&f, Sums &y)
    {
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) f(x[h][mb][nb], y[h][mb][nb]);
    }

    A a;
    B b;
    unsigned lda, ldb;
    int wm, wn;
    product_lds_t *lds;

    __device__ __forceinline__ Tile(product_lds_t *smem, unsigned lda_bytes, unsigned ldb_bytes) : lda(lda_bytes), ldb(ldb_bytes), lds(smem)
    {
        const int w = A::wave();
        wm = w / WN;
        wn = w % WN;
        a.set_up(lda, wm * WAVE_M);
        b.set_up(ldb, wn * WAVE_N);
    }
    __device__ __forceinline__ int of_row(int mb) const { return wm * WAVE_M + mb * 16 + (threadIdx.x & 15); }
    __device__ __forceinline__ int first_row() const { return wm * WAVE_M; }
    __device__ __forceinline__ int first_column() const { return wn * WAVE_N; }
    __device__ __forceinline__ int of_column(int nb) const { return wn * WAVE_N + nb * 16 + ((threadIdx.x & 63) >> 4) * 4; }

    __device__ __forceinline__ static int steps_of(const Job &j) { return (j.k + STAGE_K - 1) / STAGE_K * j.runs; }

    // the stage that is asked for next or was last: its operands' buffers, k from its first on, the ring's buffer it goes to
    struct Cursor {
        product_u32x4 a, b[HALVES];
        int left, runs;                        // runs behind this one
        unsigned lds;
    };
    __device__ __forceinline__ void begin(Cursor &c, const Job &j, bool second) const
    {
        c.left = __builtin_amdgcn_readfirstlane(j.k);
        c.runs = second ? 0 : __builtin_amdgcn_readfirstlane(j.runs) - 1;
        Source sa = j.a[0], sb = j.b[0];
        if (second) sa = j.a[1], sb = j.b[1];
        c.a = A::first_buffer(sa, c.left, lda);
        c.b[0] = B::first_buffer(sb, c.left, ldb);
        if (HALVES == 2) c.b[HALVES - 1] = B::first_buffer(j.b[1], c.left, ldb);
    }
    // whether there is a stage behind this one
    __device__ __forceinline__ bool advance(Cursor &c, const Job &j) const
    {
        c.left -= STAGE_K;
        if (c.left > 0) {
            A::next_buffer(c.a, c.left, lda);
            if (BLOCK_K > 0 && (j.k - c.left) % (BLOCK_K > 0 ? BLOCK_K : 1) == 0) {
                constexpr unsigned row = BLOCK_K * sizeof(T);
                const uint64_t base = (((uint64_t)c.a[1] << 32) | c.a[0]) + j.block - row;
                c.a[0] = (unsigned)base;
                c.a[1] = (unsigned)(base >> 32);
                c.a[2] += row;
            }
#pragma unroll
            for (int h = 0; h < HALVES; ++h) B::next_buffer(c.b[h], c.left, ldb);
            return true;
        }
        if (c.runs <= 0) return false;
        begin(c, j, true);
        return true;
    }
    // load i of the stage (there = false: the buffers have no records, and zeros go to LDS that nobody reads)
    __device__ __forceinline__ void load(const Cursor &c, int i) const
    {
        if (i < A::MINE) a.load(i, c.a, c.left, c.lds);
        else if (i < A::MINE + B::MINE) b.load(i - A::MINE, c.b[0], c.left, c.lds + A::BYTES);
        else b.load(i - A::MINE - B::MINE, c.b[HALVES - 1], c.left, c.lds + A::BYTES + B::BYTES);
    }

    // Groups of a fragment of A with all of B's: the reads of a group are two groups ahead of its products, the next step's fragments of B spread
    // over this step's groups, the loads of the stage asked for over the whole.
    __device__ __forceinline__ void multiply(Sums &sums, int buffer, const Cursor &st) const
    {
        product_lds_t *at = lds + buffer * STAGE;
        constexpr int S = A::STEPS, Q = S * MB, NBH = HALVES * NB, AHEAD = MB < 2 ? 1 : 2;
        typename A::fragment fa[S][MB];
        typename B::fragment fb[S][HALVES][NB];
#pragma unroll
        for (int i = 0; i < NBH; ++i) fb[0][i / NB][i % NB] = b.read(at + A::BYTES + i / NB * B::BYTES, i % NB, 0);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) fa[q / MB][q % MB] = a.read(at, q % MB, q / MB);
        int asked = 0, read = 0;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int ks = q / MB, mb = q % MB;
            if (q + AHEAD < Q) fa[(q + AHEAD) / MB][(q + AHEAD) % MB] = a.read(at, (q + AHEAD) % MB, (q + AHEAD) / MB);
            if (mb == 0) read = 0;
            if (ks + 1 < S) {
#pragma unroll
                for (; read < NBH * (mb + 1) / MB; ++read) fb[ks + 1][read / NB][read % NB] = b.read(at + A::BYTES + read / NB * B::BYTES, read % NB, ks + 1);
            }
#pragma unroll
            for (; asked < 4 * LOADS * (q + 1) / Q && asked < LOADS; ++asked) load(st, asked);
#pragma unroll
            for (int i = 0; i < NBH; ++i) product_mma(sums[i / NB][mb][i % NB], fb[ks][i / NB][i % NB], fa[ks][mb]);
            if (q + 1 < Q) __builtin_amdgcn_sched_barrier(0);
        }
    }

    // this wavefront's loads of the oldest of `pending` stages have landed (what was issued behind them only makes the wait longer) and its reads
    // of the stage before are done; behind the barrier everyone's
    // behind: a tile's STORES or more are younger than all of those loads
    template <int STORES>
    __device__ __forceinline__ static void wait(int pending, bool behind)
    {
        if (younger<STAGES - 2>(pending)) return;
        if (STORES > 0 && behind) landed<(STORES < 63 ? STORES : 63)>();
        else landed<0>();
    }
    // all but the newest N vector memory operations are done; a tile of one wavefront needs no barrier
    template <int N>
    __device__ __forceinline__ static void landed()
    {
        if constexpr (WAVES > 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    }
    // N or more stages are younger than the oldest
    template <int N>
    __device__ __forceinline__ static bool younger(int pending)
    {
        if constexpr (N > 0) {
            static_assert(N * LOADS < 64, "what the counter holds");
            if (pending <= N) return younger<N - 1>(pending);
            landed<N * LOADS>();
            return true;
        }
        return false;
    }

    // next(job) -> whether there is one; finish(job, sums) writes a tile.  Both are reached by the whole workgroup.
    // STORES: the fewest vector memory operations that finish issues.  Reads and writes complete in the order of their issue, so the first stage behind a
    // tile, which was asked for before its stores, has landed while they are on their way.
    template <int STORES, class Next, class Finish>
    __device__ __forceinline__ void run(Next &&next, Finish &&finish) const
    {
        Job job, then;
        if (!next(job)) return;
        bool more = next(then);
        int pending = 0, to = 0, from = 0;     // stages asked for and not multiplied yet; the ring's buffers for the next of either
        Cursor at;
        bool in_then = false, fresh = true;    // the cursor is in `then`; it stands on a stage that was not asked for yet
        begin(at, job, false);
        // moves the cursor to the next stage to ask for, if there is one
        auto following = [&] {
            if (!fresh && !advance(at, in_then ? then : job)) {
                at.left = 0;
                at.runs = 0;
            }
            fresh = false;
            if (at.left <= 0) {
                if (in_then || !more) return false;
                begin(at, then, false);
                in_then = true;
                if (at.left <= 0) return false;
            }
            at.lds = (unsigned)(uintptr_t)lds + to * STAGE;
            ++pending;
            to = to + 1 == STAGES ? 0 : to + 1;
            return true;
        };
        auto ask = [&](int most) {
            while (pending < most && following()) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) load(at, i);
            }
        };
        bool stored = false;
        ask(STAGES - 1);
        while (true) {
            const int steps = steps_of(job);
            Sums sums, part;                   // part: binary32's last stages, by themselves
            each(sums, [](product_f32x4 &v, product_f32x4 &) { v = product_f32x4{0.f, 0.f, 0.f, 0.f}; }, sums);
            if (APART) each(part, [](product_f32x4 &v, product_f32x4 &) { v = product_f32x4{0.f, 0.f, 0.f, 0.f}; }, part);
            for (int s = 0; s < steps; ++s) {
                wait<STORES>(pending, stored && s == 0);
                ask(STAGES - 1);
                if (!following()) {            // the buffer of the stage before this one is free
                    at.lds = (unsigned)(uintptr_t)lds + to * STAGE;
                    at.a[2] = 0;
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) at.b[h][2] = 0;
                }
                multiply(APART ? part : sums, from, at);
                if (APART && (s % APART == APART - 1 || s + 1 == steps))
                    each(sums, [](product_f32x4 &v, product_f32x4 &w) {
                        v += w;
                        w = product_f32x4{0.f, 0.f, 0.f, 0.f};
                    }, part);
                from = from + 1 == STAGES ? 0 : from + 1;
                --pending;
            }
            finish(job, sums);
            if (!more) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no load may reach LDS that others have by then
                break;
            }
            stored = pending > 0;
            job = then;
            if (!in_then) {
                begin(at, job, false);
                fresh = true;
            }
            in_then = false;
            more = next(then);
            // stages behind a tile without any: its buffers are free, everyone has passed the barrier of the last multiplied stage
            if (pending == 0) {
                landed<0>();
                ask(STAGES - 1);
            }
        }
    }
};

// SPLIT wavefronts with a tile of their own each (of one wavefront) share a job's k: this one's part of it.  A lies along k.
template <class TILE, int SPLIT>
__device__ __forceinline__ void share_k(Job &j, unsigned ldb)
{
    constexpr int STAGE_K = TILE::STAGE_K;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = ((j.k + SPLIT - 1) / SPLIT + STAGE_K - 1) / STAGE_K * STAGE_K;
    const int k0 = wave * part, along = k0 * (int)sizeof(typename TILE::T);
    for (int i = 0; i < 2; ++i) {
        j.a[i].base += along;
        j.a[i].records -= along;               // (of a part without k nothing is read)
        j.b[i].base += TILE::B_ORDER == ALONG_K ? (size_t)along : (size_t)k0 * ldb;
        if (TILE::B_ORDER == ALONG_K) j.b[i].records -= along;
    }
    j.k = j.k - k0 < part ? (j.k - k0 > 0 ? j.k - k0 : 0) : part;
}
template <class TILE, int SPLIT>
constexpr int SHARED_SUMS = (SPLIT - 1) * TILE::HALVES * TILE::MB * TILE::NB * 64;
// The first wavefront's sums become all of them together, in their order; -> whether this is the first.  By the whole workgroup.
template <class TILE, int SPLIT>
__device__ __forceinline__ bool join_sums(typename TILE::Sums &sums, product_f32x4 *shared)
{
    constexpr int N = TILE::HALVES * TILE::MB * TILE::NB;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    product_f32x4 *const mine = &sums[0][0][0];
    __syncthreads();                           // the sums of the tile before have been read
    if (wave > 0)
#pragma unroll
        for (int i = 0; i < N; ++i) shared[((wave - 1) * N + i) * 64 + lane] = mine[i];
    __syncthreads();
    if (wave > 0) return false;
#pragma unroll
    for (int w = 0; w < SPLIT - 1; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) mine[i] += shared[(w * N + i) * 64 + lane];
    return true;
}

// Where a tile's rows go, in U: row(mb, v) writes the columns `from` .. columns-1 of block row mb.  bfloat16: two blocks' lane groups exchange their halves,
// so that a lane has 16 bytes to write and a row's four lanes 64 in a run; every lane of the wavefront has to be there.  What is not in D goes to an offset
// behind the buffer's end, so that a row is always the same number of stores.
template <class TILE, class U>
struct Writer {
    static constexpr bool PAIRS = sizeof(U) == 2 && TILE::NB % 2 == 0;
    static constexpr int STEP = PAIRS ? 2 : 1, STORES = TILE::NB / STEP;     // of a row
    __amdgpu_buffer_rsrc_t to;
    unsigned at, ld;
    int row0, rows, column, from, columns;     // column: of this lane's first store in the tile

    // first: the tile's first element (of columns in front of `from` no address is used)
    __device__ __forceinline__ Writer(const TILE &tile, U *first, unsigned ld_bytes, int rows_, int columns_, int from_ = 0)
        : to(__builtin_amdgcn_make_buffer_rsrc(first, 0, 0x7fffffff, 0x27000)), ld(ld_bytes), row0(tile.of_row(0)), rows(rows_), from(from_), columns(columns_)
    {
        const int g = (threadIdx.x & 63) >> 4;
        column = tile.first_column() + (PAIRS ? (g & 1) * 16 + (g >> 1) * 8 : g * 4);
        at = (unsigned)row0 * ld + (unsigned)column * sizeof(U);
    }
    __device__ __forceinline__ void row(int mb, const product_f32x4 (&v)[TILE::NB]) const
    {
        const bool there = row0 + mb * 16 < rows;
#pragma unroll
        for (int nb = 0; nb < TILE::NB; nb += STEP) {
            const int c = column + nb * 16;
            // the whole offset in a vector register: behind a 16-byte store with a part of it in a scalar one the compiler takes the data's registers as free
            // one instruction later, and the last four lanes of sixteen were seen to write what came into them then
            const unsigned where = (there && c >= from && c < columns ? at + nb * 16 * (unsigned)sizeof(U) : 0x80000000u) + mb * 16 * ld;
            if constexpr (PAIRS) {
                const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16x2(v[nb][0], v[nb][1]), pack_bf16x2(v[nb + 1][0], v[nb + 1][1]), false, false);
                const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16x2(v[nb][2], v[nb][3]), pack_bf16x2(v[nb + 1][2], v[nb + 1][3]), false, false);
                __builtin_amdgcn_raw_buffer_store_b128(product_u32x4{lo[0], hi[0], lo[1], hi[1]}, to, where, 0, 0);
            } else if constexpr (sizeof(U) == 2) {
                __builtin_amdgcn_raw_buffer_store_b64(product_u32x2{pack_bf16x2(v[nb][0], v[nb][1]), pack_bf16x2(v[nb][2], v[nb][3])}, to, where, 0, 0);
            } else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(product_u32x4, v[nb]), to, where, 0, 0);
        }
    }
};

// Where the rows of groups and their tiles lie, from the caller's table `offset` [E + 1] (NULL: one group of all rows).  An entry that goes back, or past the
// rows there are, is taken for the nearest that does not, so that no row has two groups.
struct RowTiles {
    int *begin;                                // LDS, E + 1: first row of group e
    int *prefix;                               // LDS, E + 1: tiles in front of group e's, as many as its rows ask for
    int *blocks;                               // LDS, E + 1: blocks of 16 rows in front of group e's
    const int32_t *offset;
    int E, rows, tile;                         // rows of the matrix, of a tile

    __device__ __forceinline__ int first(int e) const { return begin[e]; }
    __device__ __forceinline__ int end(int e) const { return begin[e + 1]; }
    // by the first wavefront; the workgroup's barrier follows
    __device__ __forceinline__ void count() const
    {
        const int lane = threadIdx.x;
        if (lane < WAVE) {
            int last = 0, tiles_before = 0, blocks_before = 0;
            if (lane == 0) begin[0] = !offset ? 0 : clamped(offset[0]);
            last = !offset ? 0 : clamped(offset[0]);
            for (int e0 = 0; e0 < E; e0 += WAVE) {
                const int e = e0 + lane;
                int past = !offset ? rows : e < E ? clamped(offset[e + 1]) : 0;
                past = past > last ? past : last;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int before = __shfl_up(past, o, 64);
                    past = lane >= o && before > past ? before : past;
                }
                const int from = __shfl_up(past, 1, 64), n = past - (lane == 0 ? last : from);
                const int t = (n + tile - 1) / tile, t_upto = wave_scan_incl(t), b = (n + 15) / 16, b_upto = wave_scan_incl(b);
                if (e < E) {
                    begin[e + 1] = past;
                    prefix[e] = tiles_before + t_upto - t;
                    blocks[e] = blocks_before + b_upto - b;
                }
                last = __builtin_amdgcn_readlane(past, 63);
                tiles_before += __builtin_amdgcn_readlane(t_upto, 63);
                blocks_before += __builtin_amdgcn_readlane(b_upto, 63);
            }
            if (lane == 0) prefix[E] = tiles_before;
        }
        __syncthreads();
    }
    __device__ __forceinline__ int clamped(int v) const { return v < 0 ? 0 : v > rows ? rows : v; }
    // the group of row tile t and its rows
    __device__ __forceinline__ int find(int t, int &lo, int &hi) const
    {
        int e = 0, past = E;                   // prefix[e] <= t < prefix[past]
        while (past - e > 1) {
            const int mid = (e + past) >> 1;
            if (prefix[mid] <= t) e = mid;
            else past = mid;
        }
        e = __builtin_amdgcn_readfirstlane(e);
        lo = __builtin_amdgcn_readfirstlane(first(e) + (t - prefix[e]) * tile);
        hi = __builtin_amdgcn_readfirstlane(end(e));
        return e;
    }
};

// Unit u of n_m x n_n tiles: neighbours in groups of `tall` rows of tiles, column after column, so that the workgroups which run side by side on an XCD
// share the operands' tiles in its L2.
__device__ __forceinline__ void product_place(int u, int n_m, int n_n, int tall, int &m, int &n)
{
    const int per = tall * n_n, group = u / per, in = u - group * per;
    const int first = group * tall, h = n_m - first < tall ? n_m - first : tall;
    n = in / h;
    m = first + in - n * h;
}

// The units of a persistent workgroup: the ids that the hardware deals to one XCD take a contiguous range of them, side by side.
struct Units {
    int at, end, by;
    // the units from .. to-1 of an XCD's, for `slots` of its workgroups, of which this is number `slot`
    __device__ __forceinline__ Units(int total, int slot, int slots, int from, int to)
    {
        const int xcd = blockIdx.x & 7, per = (total + 7) >> 3, past = xcd * per + (to < per ? to : per);
        at = xcd * per + from + slot;
        end = past < total ? past : total;
        by = slots;
    }
    // all of them; grids are multiples of 8.  behind: of others, of which the first workgroups may have one more
    __device__ __forceinline__ explicit Units(int total, bool behind = false)
        : Units(total, behind ? (gridDim.x >> 3) - 1 - (blockIdx.x >> 3) : blockIdx.x >> 3, gridDim.x >> 3, 0, total)
    {
    }
    __device__ __forceinline__ bool take(int &u)
    {
        if (at >= end) return false;
        u = at;
        at += by;
        return true;
    }
};

// Two products in one launch.  Of an XCD's `slots` workgroups (2 .. 64) `mine` have the n1 units of the first, the others units of the second, of which they
// leave those from `rest` on to the first ones for when they are done: as brings all to the same end.  n: units of an XCD, cost: of a unit.  By all lanes of
// a wavefront, of which each tries a number.
struct Shares {
    int mine, rest;
    __device__ __forceinline__ Shares(int n1, float cost1, int n2, float cost2, int slots)
    {
        const int lane = threadIdx.x & 63, first = lane >= 1 && lane < slots ? lane : 1, second = slots - first;
        const float t1 = (float)((n1 + first - 1) / first) * cost1, even = (n2 * cost2 + first * t1) / slots;
        const float rounds = ceilf(even / cost2) * second;
        int m = even > t1 && rounds < (float)n2 ? (int)rounds : n2;
        const float t2 = (float)((m + second - 1) / second) * cost2, t3 = t1 + (float)((n2 - m + first - 1) / first) * cost2;
        float t = -fmaxf(t2, t3);
        int best = first;
        argmax_over<64>(t, best);
        mine = __builtin_amdgcn_readfirstlane(best);
        rest = __builtin_amdgcn_readfirstlane(__shfl(m, mine, 64));
        if (n1 == 0) mine = 0, rest = n2;
    }
};

// A product's tiles of the largest size in whole rounds over the compute units, and what is left over in tiles of a half down to a sixteenth of that size: a
// last round of a few large tiles would leave the other compute units without work for a whole tile's time.  bfloat16, one workgroup to a compute unit: as one
// round holds them (small tiles are bound by LDS).  binary32, whose matrix instructions take the longest, whatever the tile: by the time that the rounds take.
// run(tile type, first unit, past the last)
template <class SIZES, class Run>
__device__ __forceinline__ void in_rounds(int units, Run &&run)
{
    const int grid = gridDim.x, cus = grid < 256 ? grid : 256, rest = units % cus;
    int whole = units - rest, size;            // of the rest: a half, 2, ..
    if (SIZES::PER_CU == 1) {
        if (2 * rest > cus) whole = units;
        size = 4 * rest > cus ? 2 : 8 * rest > cus ? 4 : 16 * rest > cus ? 8 : 16;
    } else {
        // percent of a whole tile's time; alone on its compute unit a workgroup has nobody to fill its waits
        auto time = [&](int parts, int each) {
            const int rounds = (parts * rest + cus - 1) / cus;
            return (rounds * each + (rounds == 1 ? 15 : 0)) / parts;
        };
        const int t2 = time(2, 103), t4 = time(4, 108), t8 = time(8, 120);
        const int t = t2 < t4 ? t2 : t4;
        size = t8 < t ? 8 : t4 < t2 ? 4 : 2;
        if (t >= 100 && t8 >= 100) whole = units;
    }
    if (whole > 0) run(typename SIZES::Whole(), 0, whole);
    if (whole == units) return;
    if (whole > 0) __syncthreads();            // the buffers change their sizes
    if (size == 2) run(typename SIZES::Half(), whole, units);
    else if (size == 4) run(typename SIZES::Quarter(), whole, units);
    else if (size == 8) run(typename SIZES::Eighth(), whole, units);
    else run(typename SIZES::Sixteenth(), whole, units);
}
template <class TILE>
struct Sized {
    typedef TILE Type;
};
template <class T, Order A, Order B, int HALVES = 1>
struct Sizes;
template <Order A, Order B, int HALVES>
struct Sizes<bf16_t, A, B, HALVES> {
    typedef Sized<Tile<bf16_t, A, B, 256, 256, 2, 4, HALVES>> Whole;
    typedef Sized<Tile<bf16_t, A, B, 128, 256, 2, 4, HALVES, 3>> Half;
    typedef Sized<Tile<bf16_t, A, B, 128, 128, 2, 4, HALVES, 4>> Quarter;
    typedef Sized<Tile<bf16_t, A, B, 128, 64, 4, 2, HALVES, 6>> Eighth;
    typedef Sized<Tile<bf16_t, A, B, 64, 64, 4, 2, HALVES, 8>> Sixteenth;
    static constexpr int PER_CU = 1;
};
template <Order A, Order B, int HALVES>
struct Sizes<float, A, B, HALVES> {
    typedef Sized<Tile<float, A, B, 128, 128, 2, 2, HALVES>> Whole;
    typedef Sized<Tile<float, A, B, 64, 128, 2, 2, HALVES>> Half;
    typedef Sized<Tile<float, A, B, 64, 64, 2, 2, HALVES, 4>> Quarter;
    typedef Sized<Tile<float, A, B, 32, 64, 2, 2, HALVES, 5>> Eighth;
    typedef Eighth Sixteenth;
    static constexpr int PER_CU = 2;           // with 13 KB of tables beside 64 KB of stages
};
constexpr int larger(int a, int b) { return a > b ? a : b; }
template <class SIZES>
struct Whole {
    typedef typename SIZES::Whole::Type Tile;
    static constexpr int THREADS = Tile::THREADS;
    // of all sizes, which use the same LDS one after another
    static constexpr int LDS = larger(larger(larger(Tile::LDS, SIZES::Half::Type::LDS), larger(SIZES::Quarter::Type::LDS, SIZES::Eighth::Type::LDS)),
                                      SIZES::Sixteenth::Type::LDS);
    static_assert(SIZES::Half::Type::THREADS == THREADS && SIZES::Quarter::Type::THREADS == THREADS && SIZES::Eighth::Type::THREADS == THREADS &&
                      SIZES::Sixteenth::Type::THREADS == THREADS,
                  "one workgroup for all");
};

__host__ __device__ constexpr int tiles_of(int n, int tile) { return (n + tile - 1) / tile; }
constexpr int PRODUCT_CUS = 256, PRODUCT_PARTS = 16;
// workgroups for at most so many units of the largest size
static inline int product_grid(long long units, int resident)
{
    const long long n = units * PRODUCT_PARTS < resident ? units * PRODUCT_PARTS : resident;
    return (int)((n + 7) / 8 * 8);
}

}  // namespace moe
