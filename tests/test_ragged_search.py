"""The search for a row's sequence in a ragged batch (csrc/qoq_ragged_search.h, the header that the kernels include), on the CPU:
64 lanes in a loop, for every number of sequences up to 5000 and next to where a round's candidates fill a wave, every answer."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2405_04532_amd", "csrc")

SRC = r'''
#include "qoq_ragged_search.h"
#include <cstdio>
#include <cstdlib>
// before(b) of b in 1 .. B holds up to b = number
static int check(int B, int number)
{
    qoq::LaneSearch s{0, B};
    int rounds = 0;
    for (; !s.near(B); ++rounds) {
        if (rounds > 4) return printf("%d of %d: no end\n", number, B), 1;
        int holds = 0;
        for (int lane = 0; lane < 64; ++lane) {
            if (!s.asks(lane)) continue;
            if (s.candidate(lane) < 1 || s.candidate(lane) > B) return printf("%d of %d: asks for %d\n", number, B, s.candidate(lane)), 1;
            holds += s.candidate(lane) <= number;
        }
        s.narrow(holds);
    }
    if (s.lo < 0 || s.lo > B) return printf("%d of %d: window at %d\n", number, B, s.lo), 1;
    const int held = B - s.lo < 64 ? B - s.lo : 64;
    int c = 0;
    for (int lane = 0; lane < held; ++lane) c += s.lo + lane + 1 <= number;
    // the callers: c lanes of `held` hold; c == held is the end of the batch and nothing else
    if (s.lo + c != number || (c == held) != (number == B)) return printf("%d of %d: %d + %d of %d\n", number, B, s.lo, c, held), 1;
    return 0;
}
int main(int argc, char** argv)
{
    const int from = atoi(argv[1]), to = atoi(argv[2]);
    for (int B = from; B <= to; ++B)
        for (int number = 0; number <= B; ++number)
            if (check(B, number)) return 1;
    return 0;
}
'''


@pytest.fixture(scope="module")
def search(tmp_path_factory):
    d = tmp_path_factory.mktemp("search")
    (d / "search.cpp").write_text(SRC)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-I", CSRC, str(d / "search.cpp"), "-o", str(d / "search")])
    return str(d / "search")


@pytest.mark.parametrize("first,last", [(0, 700), (701, 2600), (2601, 4000), (4001, 5000), (8190, 8260), (16380, 16400), (262143, 262146), (262208, 262210),
                                        (266303, 266306), (1 << 20, 1 << 20)])
def test_every_answer(search, first, last):
    run = subprocess.run([search, str(first), str(last)], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
