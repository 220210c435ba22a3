"""The bounded wait of the paged kernels, compiled for the host with a barrier and a clock of the test's own."""
import pathlib
import re
import subprocess

import pytest

SOURCE = pathlib.Path(__file__).parents[1] / "paper_2608_12703_gb300" / "csrc" / "paged.cuh"

FRAME = r"""
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#define __device__
#define __forceinline__ inline
static long long now = 1000, lands, step;
static int polls, reports;
enum { ST_WAIT_TIMEOUT = 1 };
static long long clock64() { return now; }
static long here_clock() { return (int32_t)now; }
#define clock here_clock
static bool mbar_try_wait(uint64_t*, uint32_t) { ++polls; now += step; return now >= lands; }
static void set_status(int* status, int bits) { ++reports; *status |= bits; }
%s
int main(int argc, char** argv) {
  // pairs of arguments: cycles until the barrier's phase ends, cycles of a look at it; one wait for each, one after another
  bool gave_up = false;
  int status = 0;
  uint64_t bar = 0;
  for (int i = 1; i + 1 < argc; i += 2) {
    const long long t0 = now;
    lands = now + atoll(argv[i]), step = atoll(argv[i + 1]), polls = reports = 0;
    bar_wait(&bar, 0, i == 1 && argc %% 4 == 1 ? nullptr : &status, gave_up);
    printf("%%lld %%d %%d %%d %%d\n", now - t0, (int)(now >= lands), (int)gave_up, status, reports);
  }
}
"""


@pytest.fixture(scope="module")
def waits(tmp_path_factory):
    at = tmp_path_factory.mktemp("bar_wait")
    body = re.search(r"__device__ __forceinline__ void bar_wait\(.*?\n\}\n", SOURCE.read_text(), re.S).group()
    (at / "wait.cpp").write_text(FRAME % body)
    subprocess.run(["g++", "-O1", "-std=c++17", "-o", str(at / "wait"), str(at / "wait.cpp")], check=True)

    def run(*pairs):
        out = subprocess.run([str(at / "wait"), *(str(x) for p in pairs for x in p)], check=True, capture_output=True, text=True, timeout=300)
        return [tuple(int(x) for x in line.split()) for line in out.stdout.splitlines()]
    return run


def test_a_phase_that_ends(waits):
    for took, landed, gave_up, status, reports in waits((0, 20), (10 ** 6, 20), (10 ** 9, 1000)):
        assert (landed, gave_up, status, reports) == (1, 0, 0, 0)


def test_a_phase_that_does_not_end(waits):
    """About 2^31 cycles, then the status word; later waits are short, and still wait for what comes in time."""
    end = 1 << 50
    first, copy, lost, again, there = waits((end, 1000), (10 ** 5, 100), (end, 100), (10 ** 5, 100), (0, 20))
    assert first[1:] == (0, 1, 1, 1) and 1 << 31 < first[0] < (1 << 31) + 10 ** 4
    assert copy[1] == again[1] == there[1] == 1 and copy[4] == again[4] == there[4] == 0
    assert lost[1] == 0 and 1 << 17 < lost[0] < (1 << 17) + 10 ** 4


def test_without_a_status_word(waits):
    first, second = waits((1 << 50, 1 << 20), (10, 100))
    assert first[1:3] == (0, 1) and first[3] == 0 and second[1] == 1
