// How sru_scan and sru_scan_backward cut their work: host rules.
#pragma once
#include "common.h"

namespace moe {

constexpr int SCAN_STEPS = 16;         // steps of a wavefront, and between saved states
constexpr int SCAN_MAX_WAVES = 8;      // wavefronts of a workgroup, one behind the other on the sequence
constexpr int SCAN_MAX_SEGMENTS = 64;
constexpr int SCAN_ENOUGH = 256;       // workgroups from which on no sequence is cut
constexpr int SCAN_WORKGROUPS = 768;   // that cut sequences give

struct ScanShape {
    int B, L, H;
    int groups;                        // of 64 channels, a lane each
    int waves, segments, seg_steps;    // seg_steps: whole rounds of the workgroup's wavefronts
    int saved;                         // saved states of a sequence
};

// sizes whose counts of workgroups and parts fit an int, and whose runs of SCAN_STEPS rows of four blocks lie within 2^31 bytes
static inline bool scan_takes(int B, int L, int H)
{
    return H <= (1 << 23) && L <= (1 << 30) && (long long)B * ((H + WAVE - 1) / WAVE) < (1 << 26);
}

static inline ScanShape scan_shape(int B, int L, int H)
{
    ScanShape g;
    g.B = B, g.L = L, g.H = H;
    g.groups = (H + WAVE - 1) / WAVE;
    g.waves = 1;
    while (g.waves < SCAN_MAX_WAVES && g.waves * SCAN_STEPS < L) g.waves *= 2;
    const int round = g.waves * SCAN_STEPS, rounds = L > 0 ? (L + round - 1) / round : 1;
    const long long have = (long long)(B > 0 ? B : 1) * g.groups;
    long long want = have >= SCAN_ENOUGH ? 1 : (SCAN_WORKGROUPS + have - 1) / have;
    if (want > SCAN_MAX_SEGMENTS) want = SCAN_MAX_SEGMENTS;
    if (want > rounds) want = rounds;
    const int per = (int)((rounds + want - 1) / want);
    g.seg_steps = per * round;
    g.segments = (rounds + per - 1) / per;
    g.saved = L > 0 ? (L + SCAN_STEPS - 1) / SCAN_STEPS : 0;
    return g;
}

}  // namespace moe
