// Sizes of the gated experts' calls: tiles by the number of rows, parts of the weights' sums, workspaces.
#pragma once
#include "common.h"

namespace moe {

constexpr int GATED_MAX_WIDTH = 1 << 20;       // byte offsets inside a tile's rows fit 31 bits

// The states' g and u: blocks of 16 rows (of an expert, from its first) x 16 columns, in the order of the matrix instructions' lanes, u's block behind g's.
// What a store or a load of a wavefront moves is then 1 KB in a run; in rows of 64 bytes they took 14 of a tile's 50 us (256 x 128 of F, d = 1024).
constexpr int GATED_BLOCK = 2 * 256;           // floats
__host__ __device__ constexpr int states_columns(int F) { return (F + 15) / 16; }
static inline size_t states_blocks(int R, int E) { return (size_t)R / 16 + (E < R ? E : R); }      // of rows, at most
static inline size_t hidden_bytes(int R, int F, int dtype) { return align_up((size_t)R * F * (dtype == MOE_F32 ? 4 : 2), 256); }

// The tile by the rows that an expert has if all have the same (the table is in device memory) and the columns of D.
//   TINY    16 rows x 32 columns, whose wavefronts share the sum: so few tiles that each has a compute unit to itself, where a stage's way from memory counts
//   SHARED  32 x 64 likewise
//   LOW     32 x 128, MID 64 x 128: bound by the stream of the weights
//   TALL    up to 256 x 256, by the matrix pipes; SMALL 64 x 64, where the sum is long and such tiles are few
// us, one way, the other.  Forward of 34 rows of 26 experts, 768 x 2048, MID 66, LOW 50; of 2181 of 128 MID 266, LOW 257.  With gradient, bfloat16, SHARED and what
// would be without: 30 rows of 1024 x 4096 83, 126 (LOW); 60 of 768 x 2048 58, 109 (MID); 200 69, 91 (TALL); 500 of 512 x 512 46, 59.  SMALL and TALL for y and dx:
// 700 rows of 1024 x 4096 154, 162; 1334 of 512 x 2048 112, 119; 2000 of 16 experts, 256 x 1376, 103, 114; with 756 tiles, 4000 rows of 768 x 2048, 229, 217.
// Binary32, whose sums take the longest, y and dx in SHARED with up to 256 tiles of LOW: 90 rows of 2048 x 512 137, 218; of 512 x 2048 93, 132; with some
// 500, 3000 rows of 64 experts, 512 x 1024, 495, 462.
enum GatedRows { GATED_TINY, GATED_SHARED, GATED_LOW, GATED_MID, GATED_SMALL, GATED_TALL };
// columns: of a SHARED tile.  long_sum: y's and dx's products
static inline GatedRows gated_rows_rule(int R, int E, int N, int columns, int dtype, bool long_sum)
{
    const long long experts = R < E ? R : E;
    if (R <= 16ll * E && experts * ceil_div(N, 128) <= 128) return GATED_TINY;
    if ((R / 32 + experts) * ceil_div(N, columns) <= 256) return GATED_SHARED;
    if (R / E >= 96) return dtype == MOE_BF16 && long_sum && (R / 64 + experts) * ceil_div(N, 64) <= 512 ? GATED_SMALL : GATED_TALL;
    if (dtype == MOE_F32 && long_sum && (R / 32 + experts / 2) * ceil_div(N, 128) <= 256) return GATED_SHARED;
    return R / E <= 32 ? GATED_LOW : GATED_MID;
}

// Parts of an expert's rows for the weights' gradients: where even an eighth of a tile each would leave compute units without work, and rows are many.
static inline int gated_parts(int R, int E, int d, int F, int dtype)
{
    const int big = dtype == MOE_F32 ? 128 : 256, slots = dtype == MOE_F32 ? 512 : 256;
    const long long tiles = (long long)E * ceil_div(d, big) * ceil_div(F, big);
    long long parts = slots / (4 * tiles);
    if (parts > R / E / 512) parts = R / E / 512;
    return parts < 2 ? 1 : parts > 16 ? 16 : (int)parts;
}

// Whether two products share a launch: tiles of rows (n1, of cost1 stages) and of weights.  One tile must not take longer than all of the work does.
static inline bool gated_pairs(int R, int E, int d, int F, int dtype, bool down)
{
    const int big = dtype == MOE_F32 ? 128 : 256, stage = dtype == MOE_F32 ? 32 : 64, slots = dtype == MOE_F32 ? 512 : 256;
    const double n1 = ((double)R / big + E / 2) * ceil_div(down ? F : d, big), cost1 = down ? d / stage + 20 : 2.0 * F / stage + 4;
    const double n2 = (double)E * ceil_div(d, big) * ceil_div(down ? F : 2 * F, big), cost2 = (double)R / E / stage + 5;
    return R / E >= 96 && n1 * cost1 + n2 * cost2 >= 0.95 * slots * (cost1 > cost2 ? cost1 : cost2);
}

}  // namespace moe
