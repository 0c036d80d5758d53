// How sru_scan and sru_scan_backward cut their work: host rules.
#pragma once
#include "common.h"

namespace moe {

// Steps of a wavefront: 16 in the forward where there is work for the card (2 x 16384 x 768 bf16 72 us, with 8 93 us: more tiles to wait for), 8 in the
// gradient, whose registers hold more for each (126 us, with 16 133 us; 8 x 1000 x 768 43 and 61 us).
// States are saved every 8 steps: 5 % of the forward's bytes.
constexpr int SCAN_LONG = 16;
constexpr int SCAN_SAVED = 8;
constexpr int SCAN_MAX_WAVES = 8;      // wavefronts of a workgroup, one behind the other on the sequence
// Lines (sequences by 64 channels) from which on a sequence is walked by one workgroup instead of cut into tiles: 32 x 512 x 1024, 512 lines, 42 us
// walked, 50 us in tiles; 16 x 2048 x 1024, 256 lines, 87 and 94; 12 x 1024 x 1024 fp32, 192 lines, 65 and 63 (gradient 110 and 101).
constexpr int SCAN_ENOUGH = 256;
// Tiles below which the forward's are cut finer: 16 of them (1 x 200 x 512) 11 us, finer 8; 210 (5 x 777 x 321 fp32) 14 and 16.
constexpr int SCAN_FEW = 64;

// tiles (sru_scan.hip)
constexpr int SCAN_RUN = 16;           // tiles of a run, runs of a stretch: two for each wavefront to look for
constexpr unsigned long long SCAN_UNKNOWN = ~0ull;
constexpr int SCAN_PATIENCE = 1 << 22;
constexpr int SCAN_CLEAR_THREADS = 256;
static_assert(SCAN_RUN == 2 * SCAN_MAX_WAVES && SCAN_MAX_WAVES == 8, "");

struct ScanShape {
    int B, L, H;
    int groups;                        // of 64 channels, a lane each
    int waves, waves_lg, steps;        // of a line (and log2); of a wavefront
    int pack;                          // lines of a workgroup
    int tiles, runs, stretches;        // of a sequence; tiles = 1: one workgroup walks it round by round
    int saved;                         // saved states of a sequence
    long long workgroups;
    int across;                        // the grid's x
};

// sizes whose counts of workgroups and parts fit an int, and whose runs of SCAN_LONG rows of four blocks lie well within 2^31 bytes
static inline bool scan_takes(int B, int L, int H)
{
    return H <= (1 << 22) && L <= (1 << 30) && (long long)B * ((H + WAVE - 1) / WAVE) < (1 << 26);
}

static inline ScanShape scan_shape(int B, int L, int H, int steps)
{
    ScanShape g;
    g.B = B, g.L = L, g.H = H, g.steps = steps;
    g.groups = (H + WAVE - 1) / WAVE;
    g.waves_lg = 0;
    while (g.waves_lg < 3 && (steps << g.waves_lg) < L) ++g.waves_lg;
    g.waves = 1 << g.waves_lg;
    g.pack = g.waves < 4 ? 4 >> g.waves_lg : 1;
    const int round = g.waves * steps, rounds = L > 0 ? (L + round - 1) / round : 1;
    const long long lines = (long long)(B > 0 ? B : 1) * g.groups;
    g.tiles = lines < SCAN_ENOUGH ? rounds : 1;
    g.runs = (g.tiles + SCAN_RUN - 1) / SCAN_RUN;
    g.stretches = (g.runs + SCAN_RUN - 1) / SCAN_RUN;
    g.saved = L > 0 ? (L + SCAN_SAVED - 1) / SCAN_SAVED : 0;
    g.workgroups = (lines + g.pack - 1) / g.pack * g.tiles;
    g.across = (int)(g.workgroups < (1 << 22) ? g.workgroups : 1 << 22);
    return g;
}
// One token: builds of one step, which are small and take none for the others (1000 x 1 x 1024 bf16 21 us with sixteen, 9 with one).  Few steps or few
// tiles: eight (200 x 8 x 320 7 us with sixteen, 5 with eight; 1 x 300 x 256 11 and 8).
static inline ScanShape scan_forward_shape(int B, int L, int H)
{
    if (L <= 1) return scan_shape(B, L, H, 1);
    const ScanShape g = scan_shape(B, L, H, L <= SCAN_MAX_WAVES * SCAN_SAVED ? SCAN_SAVED : SCAN_LONG);
    return g.tiles > 1 && (long long)B * g.groups * g.tiles < SCAN_FEW ? scan_shape(B, L, H, SCAN_SAVED) : g;
}
static inline ScanShape scan_backward_shape(int B, int L, int H) { return scan_shape(B, L, H, L <= 1 ? 1 : SCAN_SAVED); }

}  // namespace moe
