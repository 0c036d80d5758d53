// How moe_token_logprobs cuts rows of logits: host rules.
#pragma once
#include "common.h"

namespace moe {

constexpr int LP_SMALL = 16;                  // logits of a lane that shares a short row
constexpr int LP_VECS = 8;                    // 16-byte pieces of a thread that shares a long one
constexpr int LP_MAX_THREADS = 1024;
constexpr int LP_MAX_PARTS = 64;              // of a row: one lane each where they are joined
constexpr int LP_MAX_V = 1 << 21;
constexpr int LP_RECORD = 4 + 2 * MOE_MAX_TOPK;   // floats of a part: maximum, sums, target's logit; the best logits and ids

struct LogprobShape {
    int lanes;                                // short rows: lanes of a row; 0: long ones
    int threads, parts, part;                 // long: threads of a workgroup, parts of a row, logits of a part
};

static inline LogprobShape logprob_shape(int N, int V, int dtype)
{
    LogprobShape g = {0, 0, 1, V};
    if (V <= WAVE * LP_SMALL) {
        g.lanes = V <= 4 * LP_SMALL ? 4 : V <= 16 * LP_SMALL ? 16 : WAVE;
        return g;
    }
    const int per = dtype == MOE_BF16 ? 8 : 4;                               // logits of a piece
    const int most = (LP_MAX_THREADS * LP_VECS - 1) * per;                   // one piece less: a row may begin inside one
    int parts = (V + most - 1) / most;
    // A row that one workgroup holds is not cut, however few there are: the join is a launch of its own (1 x 32000 bf16 6.7 us whole, 9.5 in
    // parts; 64 x 50257 8.0 and 9.1; 300 x 50257 15 and 18).  A longer one, in few rows: two workgroups for each compute unit, parts of
    // at least a piece for each lane of four wavefronts (3 x 131072: 12 us; two parts: 15).
    if (parts > 1) {
        const int want = N < 512 ? (512 + N - 1) / N : 1, room = V / (4 * WAVE * per), split = want < room ? want : room;
        if (split > parts) parts = split;
    }
    if (parts > LP_MAX_PARTS) parts = LP_MAX_PARTS;
    g.part = ((V + parts - 1) / parts + 63) / 64 * 64;                       // parts begin alike inside a piece
    g.parts = (V + g.part - 1) / g.part;
    const int pieces = (g.part < V ? g.part : V) / per + 1;
    // few workgroups: one or two pieces a thread; many: as few threads as hold the row
    const int each = (long long)N * g.parts < 2048 ? 2 : LP_VECS;
    g.threads = WAVE;
    while (g.threads < LP_MAX_THREADS && g.threads * each < pieces) g.threads *= 2;
    return g;
}

// The gradient: log2 of the threads that share a row, LP_SLOPE_PIECES pieces of 16 bytes each; what does not fit them goes to further workgroups.
constexpr int LP_SLOPE_PIECES = 4;
constexpr int LP_SLOPE_LG = 8;                // a workgroup of 256
static inline int logprob_slope_pieces(int V, int dtype) { return V / (dtype == MOE_BF16 ? 8 : 4) + 1; }
static inline int logprob_slope_lanes(int V, int dtype)
{
    int lg = 0;
    while (lg < LP_SLOPE_LG && (LP_SLOPE_PIECES << lg) < logprob_slope_pieces(V, dtype)) ++lg;
    return lg;
}

// a launch holds fewer than 2^32 threads in a dimension: short rows `lanes` each, long ones a workgroup each and their parts across the other
// dimension; the gradient's 2^lg
static inline bool logprob_takes(int N, int V, int dtype)
{
    if (V > LP_MAX_V) return false;
    const LogprobShape g = logprob_shape(N > 0 ? N : 1, V, dtype);
    const int each = g.lanes ? g.lanes : g.threads, slope = 1 << logprob_slope_lanes(V, dtype);
    return (long long)N * (each > slope ? each : slope) < (1ll << 32) - 1024;
}

}  // namespace moe
