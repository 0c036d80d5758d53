// Sizes of the head's calls: tiles by the number of rows, pieces of the vocabulary, parts of a sum.  Host code.
#pragma once
#include "common.h"

namespace moe {

constexpr int HEAD_MAX_WIDTH = 1 << 20;        // byte offsets inside a tile's rows fit 31 bits
constexpr int HEAD_MAX_IDS = 1 << 24, HEAD_MAX_ROWS = 1 << 24;
constexpr size_t HEAD_PIECE_BYTES = 1u << 30;    // of dz, and of the parts of dh's sum
// Backward: rows up to which the launch that would make rows again also prepares them and every workgroup of it looks at all of them for one that is far from
// zero; beyond, where that looking takes longer than a launch, another one does so first.  With gradient, us, one way, the other: 4096 x 256 x 128 43.9, 44.2 and,
// where it is waited for, 59, 62 to 70; 15009 x 256 x 256 68, 64; 777 x 320 x 5003 in binary32 157, 156, waited for 172, 174.
constexpr int HEAD_SCAN_ROWS = 4096;
constexpr int HEAD_DZ_ROW = 512;               // bytes of a row of dz in one of its blocks
constexpr int HEAD_FEW_COLUMNS = 128;          // of a tile of few rows

enum HeadRows { HEAD_FEW_TILES, HEAD_LOW_TILES, HEAD_FLAT_TILES, HEAD_TALL_TILES };      // of 16, 32, 64 rows and more
// (binary32 is bound by the matrix pipes, and rows behind the last cost as much as others: 192 rows are three tiles of 64, of 128 two with a quarter of
// nothing, and up to 32 rows of a last tile are a tile of 32: 20 x 704 x 45094 with gradient 160 us, in tiles of 64 220; 129 x 512 x 21296 174, 184)
static inline HeadRows head_rows(int N, int dtype)
{
    if (N <= 16) return HEAD_FEW_TILES;
    if (N > (dtype == MOE_F32 ? 192 : 128)) return HEAD_TALL_TILES;
    return dtype == MOE_F32 && (N - 1) % 64 < 32 ? HEAD_LOW_TILES : HEAD_FLAT_TILES;
}
static inline int head_tile_rows(int N, int dtype)
{
    const HeadRows r = head_rows(N, dtype);
    return r == HEAD_FEW_TILES ? 16 : r == HEAD_LOW_TILES ? 32 : r == HEAD_FLAT_TILES ? 64 : dtype == MOE_F32 ? 128 : 256;
}
static inline int head_tile_columns(int N, int dtype) { return head_rows(N, dtype) != HEAD_TALL_TILES ? HEAD_FEW_COLUMNS : dtype == MOE_F32 ? 128 : 256; }
// The logits, both ways: tiles of 16 rows x 32 columns where a compute unit has one of them at most.
constexpr int HEAD_TINY_ROWS = 16, HEAD_TINY_COLUMNS = 32, HEAD_TINY_TILES = 256;
static inline bool head_tiny(int N, int V) { return (long long)ceil_div(N, HEAD_TINY_ROWS) * ceil_div(V, HEAD_TINY_COLUMNS) <= HEAD_TINY_TILES; }
// forward: slots of maximum and sum that a row has, one for a tile's columns
static inline int head_row_slots(int N, int V, int dtype) { return ceil_div(V, head_tiny(N, V) ? HEAD_TINY_COLUMNS : head_tile_columns(N, dtype)); }
// the logits' maxima and sums, and the targets' logits in front of them
static inline size_t head_targets_bytes(int N) { return align_up((size_t)N * 4, 256); }
static inline size_t head_scores_bytes(int N, int V, int dtype) { return head_targets_bytes(N) + (size_t)N * head_row_slots(N, V, dtype) * 8; }
// backward: rows of a wavefront, for which the bias has a slot of partial sums
static inline int head_wave_rows(int N, int V, int dtype)
{
    if (head_tiny(N, V)) return HEAD_TINY_ROWS;
    return head_tile_rows(N, dtype) / (head_rows(N, dtype) == HEAD_TALL_TILES ? 2 : 1);
}

// The gradient's pieces and workspace.
struct HeadShape {
    int piece;                                 // ids of the vocabulary whose dz is in memory at a time
    int parts;                                 // of a piece's sum for dh
    int dw_parts;                              // of the rows in dW's sum (one piece only)
    bool paired;                               // dh and dW share a launch
    int db_rows;                               // rows of partial sums for db
    int n_again;                               // maxima and sums of a row made again, as dz is made from them: a row's tiles', up to 64, or one behind a join
    size_t again_at, rows_at, dz_at, dh_at, db_at, dw_at, bytes;
};
static inline HeadShape head_shape(int N, int d, int V, int dtype)
{
    HeadShape g;
    const int z = dtype == MOE_F32 ? 4 : 2;
    const size_t most = HEAD_PIECE_BYTES / ((size_t)N * z) / 256 * 256;
    const int fits = most < 256 ? 256 : most > (size_t)V ? V : (int)most;
    const int pieces = ceil_div(V, fits);
    g.piece = pieces == 1 ? V : (int)align_up(ceil_div(V, pieces), 256);
    // Parts of dh's sum.  A tile costs its k and some 384 beside, for its first stage and its writes; a part is written and read again.  Paired with dW, whose
    // tiles are as many as compute units, the parts fill what is left of the last round: about half a part's time is lost.  Alone: whole rounds.
    const int rows = head_tile_rows(N, dtype), columns = head_tile_columns(N, dtype), slots = dtype == MOE_F32 ? 512 : 256;
    const long long tiles = (long long)ceil_div(N, rows) * ceil_div(d, columns), of_dw = (long long)ceil_div(g.piece, rows) * ceil_div(d, columns);
    // (a tile of dW must not take longer than all of the work does)
    g.paired = head_rows(N, dtype) == HEAD_TALL_TILES && of_dw * (N + 256.0) + tiles * (g.piece + 384.0) >= slots * (N + 256.0);
    double best = 0;
    g.parts = 1;
    for (int s = 1; s <= 64; ++s) {
        if (s > 1 && (g.piece / s < 512 || (size_t)s * N * d * 4 > HEAD_PIECE_BYTES)) break;
        const double k = (double)g.piece / s + 384, traffic = 3e-5 * s * N * d;
        const double cost = traffic + (g.paired ? (double)tiles * s * k / slots + k / 2 : (double)((tiles * s + slots - 1) / slots) * k);
        if (s == 1 || cost < best * 0.99) {
            best = cost;
            g.parts = s;
        }
    }
    // dW alone: parts where even an eighth of a tile each would leave compute units without work, and rows are many
    long long dw_parts = pieces == 1 && !g.paired ? slots / (4 * of_dw) : 1;
    if (dw_parts > N / 512) dw_parts = N / 512;
    g.dw_parts = dw_parts < 2 ? 1 : dw_parts > 16 ? 16 : (int)dw_parts;
    g.db_rows = ceil_div(N, head_wave_rows(N, V, dtype));
    g.again_at = 256;
    g.n_again = head_row_slots(N, V, dtype) <= 64 ? head_row_slots(N, V, dtype) : 1;
    g.rows_at = g.again_at + align_up((size_t)N * g.n_again * 8, 256);
    g.dz_at = g.rows_at + align_up((size_t)N * d * z, 256);
    // before dz is written its place holds what summing the rows again takes
    const size_t dz = (size_t)N * align_up((size_t)g.piece * z, HEAD_DZ_ROW), scores = head_scores_bytes(N, V, dtype);
    g.dh_at = g.dz_at + align_up(dz > scores ? dz : scores, 256);
    g.db_at = g.dh_at + align_up((size_t)g.parts * N * d * 4, 256);
    g.dw_at = g.db_at + align_up((size_t)g.db_rows * V * 4, 256);
    g.bytes = g.dw_at + (g.dw_parts > 1 ? align_up((size_t)g.dw_parts * V * d * 4, 256) : 0);
    return g;
}

}  // namespace moe
