"""How many rows of logits a call takes: the host rule, compiled from the library's header, against the launch limit and the documented sizes; and
numbers that do not fit the library's."""
import os
import subprocess

import pytest
import torch

import paper_2605_11537_amd as moe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = """
#include "token_logprobs_rules.h"
#include <stdio.h>
using namespace moe;
int main()
{
    int N, V, dtype;
    while (scanf("%d %d %d", &N, &V, &dtype) == 3) {
        const LogprobShape g = logprob_shape(N, V, dtype);
        printf("%d %d %d %d\\n", logprob_takes(N, V, dtype), g.lanes ? g.lanes : g.threads, 1 << logprob_slope_lanes(V, dtype),
               logprob_slope_pieces(V, dtype));
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("training_limits")
    src, exe = str(d / "main.cpp"), str(d / "main")
    open(src, "w").write(MAIN)
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I",
                           os.path.join(ROOT, "paper_2605_11537_amd", "csrc"), src, "-o", exe])

    def run(rows):
        out = subprocess.run([exe], input="\n".join(" ".join(map(str, r)) for r in rows), capture_output=True, text=True, check=True).stdout
        return [[int(v) for v in line.split()] for line in out.splitlines()]
    return run


def test_rows_are_refused_for_the_launch_only(ask):
    cases = [(N, V, t) for t in (0, 1) for V in (1, 8, 24, 25, 64, 65, 256, 257, 1024, 1025, 2000, 4096, 50257, 1 << 21)
             for N in (1, 1 << 16, 1 << 21, 1 << 22, 1 << 24, (1 << 24) + 37, 1 << 26, 1 << 28, 1 << 30, (1 << 31) - 1)]
    for (N, V, t), (takes, forward, slope, pieces) in zip(cases, ask(cases)):
        threads = N * max(forward, slope)
        assert bool(takes) == (threads < (1 << 32) - 1024), (N, V, t)
        assert slope == 256 or 4 * slope >= pieces
        assert -(-pieces // (4 * slope)) < 1 << 16                      # the grid's other dimension
        if not takes:
            continue
        for each in (forward, slope):                                  # the last workgroup's numbers, and what is computed on the way
            per = max(1, 256 // each) if each <= 256 else 1
            assert N + per < 1 << 31 and -(-N // per) * per <= 1 << 31


def test_the_documented_sizes_are_taken(ask):
    cases = [(N, V, t) for t in (0, 1) for N, top in ((1 << 28, 64), (1 << 26, 256), (1 << 24, 1024), (1 << 21, 1 << 21))
             for V in (1, 8, 64, 65, 100, 256, 257, 1000, 1024, 1025, 50257, 1 << 21) if V <= top]
    assert all(row[0] for row in ask(cases))


@pytest.mark.parametrize("k", [2 ** 32 + 3, 2 ** 31, -2 ** 31 - 1, 2 ** 64 + 1])
def test_a_number_of_alternatives_past_an_int_is_refused(k):
    """It was reduced to the int's width: 2^32 + 3 asked for 2^32 + 3 columns, of which 3 were written."""
    with pytest.raises(ValueError, match="does not fit an int"):
        moe.moe_token_logprobs(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), k)
