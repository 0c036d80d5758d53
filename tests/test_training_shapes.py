"""How the scan and the scoring cut their work: the host rules, compiled from the library's headers, against what the kernels rely on."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = """
#include "sru_scan_rules.h"
#include "token_logprobs_rules.h"
#include "row_groups.h"
#include <stdio.h>
using namespace moe;
int main()
{
    char kind;
    int a, b, c;
    while (scanf(" %c %d %d %d", &kind, &a, &b, &c) == 4) {
        if (kind == 'f' || kind == 'b') {
            if (!scan_takes(a, b, c)) { printf("-1\\n"); continue; }
            const ScanShape g = kind == 'f' ? scan_forward_shape(a, b, c) : scan_backward_shape(a, b, c);
            printf("%d %d %d %d %d %d %d %d %d %d %d %lld\\n", g.groups, g.waves, g.steps, g.tiles, g.runs, g.stretches, g.saved, g.across, SCAN_RUN, SCAN_MAX_WAVES, g.pack, g.workgroups);
        } else if (kind == 'g') {
            const dim3 g = rows_grid(a, b);
            printf("%u %u %d\\n", g.x, g.y, ROWS_GRID_LG);
        } else {
            if (!logprob_takes(a, b, c)) { printf("-1\\n"); continue; }
            const LogprobShape g = logprob_shape(a, b, c);
            printf("%d %d %d %d %d %d\\n", g.lanes, g.threads, g.parts, g.part, LP_VECS, LP_SMALL);
        }
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("training_shapes")
    src, exe = str(d / "main.cpp"), str(d / "main")
    open(src, "w").write(MAIN)
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I",
                           os.path.join(ROOT, "paper_2605_11537_amd", "csrc"), src, "-o", exe])

    def run(rows):
        text = "\n".join(" ".join(str(v) for v in r) for r in rows)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [[int(v) for v in line.split()] for line in out.splitlines()]
    return run


def _log(rng, hi):
    return int(round(2 ** rng.uniform(0, hi)))


def test_scan_shapes(ask):
    rng = random.Random(1)
    rows = [(rng.choice("fb"), _log(rng, 12), rng.choice([0, _log(rng, 7), _log(rng, 20)]), _log(rng, 13)) for _ in range(4000)]
    rows += [(k, B, L, H) for k in "fb" for B in (1, 255, 256, 1 << 20) for L in (0, 1, 8, 16, 17, 128, 129, 1 << 30) for H in (1, 64, 65, 1 << 22)]
    for (kind, B, L, H), got in zip(rows, ask(rows)):
        lines = B * -(-H // 64)
        if got == [-1]:
            assert H > 1 << 22 or lines >= 1 << 26
            continue
        groups, waves, steps, tiles, runs, stretches, saved, across, RUN, MAX, pack, workgroups = got
        assert groups == -(-H // 64) and waves in (1, 2, 4, 8) and waves <= MAX
        assert steps in (8, 16) and (kind == "f" or steps == 8) if L > 1 else steps == 1
        round_ = waves * steps
        assert saved == -(-L // 8) and (steps % 8 == 0 or L <= 1)
        assert waves * pack in (4, 8) and (pack == 1 or tiles == 1) and waves * pack <= MAX
        if tiles > 1:
            # tiles are whole, the look-back has its eight wavefronts, and every list holds what indexes it
            assert waves == MAX and RUN == 2 * MAX and (tiles - 1) * round_ < L <= tiles * round_
            assert (tiles - 1) // RUN < runs and (runs - 1) // RUN < stretches
        else:
            assert lines >= 256 or L <= round_
        n = lines * tiles if pack == 1 else -(-lines // pack)
        assert n == workgroups
        assert across * 512 < 1 << 32 and -(-n // across) < 1 << 16
        assert 15 * 4 * H * 4 + 4 * H * 4 < 0x7fffffff              # the farthest step's row of binary32 in four blocks
    assert ask([("f", 1, 5, 1 << 23)]) == [[-1]]


def test_logprob_shapes(ask):
    rng = random.Random(2)
    rows = [("l", _log(rng, 20), _log(rng, 21), rng.randint(0, 1)) for _ in range(4000)]
    rows += [("l", N, V, t) for t in (0, 1) for N in (1, 511, 512, 4000000, (1 << 31) - 1)
             for V in (1, 64, 65, 256, 257, 1024, 1025, 32764, 32765, 32768, 65528, 65529, 65536, 131072, 1 << 21)]
    for (_, N, V, dtype), got in zip(rows, ask(rows)):
        if got == [-1]:
            assert N >= (1 << 22) - 8
            continue
        lanes, threads, parts, part, vecs, small = got
        if lanes:
            assert V <= 1024 and lanes in (4, 16, 64) and lanes * small >= V and N * lanes < 1 << 32
            continue
        per = 8 if dtype else 4
        assert threads in (64, 128, 256, 512, 1024) and 1 <= parts <= 64 and N * threads < 1 << 32
        assert (parts - 1) * part < V <= parts * part and (parts == 1 or part % 64 == 0)
        longest = min(part, V)
        for head in range(per):                                    # wherever a row begins inside a piece
            assert (longest - head) // per <= threads * vecs
            assert longest - (longest - head) // per * per <= threads   # single logits in front and behind: one a thread
    assert ask([("l", 1, (1 << 21) + 1, 1)]) == [[-1]]


def test_row_grids(ask):
    """Every row has its workgroup, numbered with a grid that is 2^22 wide when it has more than one row of workgroups."""
    rows = [("g", T, lg, 0) for T in (1, 255, 256, 1 << 20, (1 << 28) + 3, (1 << 31) - 1) for lg in (0, 2, 4, 5, 6, 8)]
    for (_, T, lg, _), (x, y, width) in zip(rows, ask(rows)):
        assert x * y * (256 >> lg) >= T and x * 256 < 1 << 32 and y < 1 << 16
        assert y == 1 or x == 1 << width
