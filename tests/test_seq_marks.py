"""The sequences of a tile's rows on the CPU: csrc/seq_marks.h compiled for the host with overflow trapped, against a walk over
the offsets.  However many sequences without rows touch a tile, few loads wait for one another, and bad offsets take no probe
out of the range."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

DRIVER = r"""
#include "seq_marks.h"
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

static int probes;

template <typename Begin>
static uint32_t find(uint32_t first, uint32_t count, int64_t row, Begin begin)
{
    probes = 0;
    const uint32_t s = fs::sequence_of_row(first, count, row, [&](uint32_t i) {
        ++probes;
        if (i <= first || i - first >= count) { std::printf("probe %u of %u .. + %u\n", i, first, count); std::exit(1); }
        return begin(i);
    });
    if (s < first || s - first >= count || probes > 31) { std::printf("%u of %u .. + %u after %d probes\n", s, first, count, probes); std::exit(1); }
    return s;
}

int main()
{
    std::mt19937 gen(7);
    for (int round = 0; round < 3000; ++round) {
        const int S = 1 + gen() % 400, empty = gen() % 100;
        std::vector<int64_t> off(S + 1, 0);
        for (int s = 0; s < S; ++s) off[s + 1] = off[s] + ((int)(gen() % 100) < empty ? 0 : 1 + gen() % 5);
        if (off[S] == 0) continue;
        // a tile of rows r0 .. r1 - 1 and the sequences that touch it
        const int64_t r0 = gen() % off[S], r1 = r0 + 1 + gen() % (off[S] - r0);
        uint32_t first = 0, last = 0;
        for (int s = 0; s < S; ++s) {
            if (off[s] < r0) first = s;
            if (off[s] < r1) last = s;
        }
        for (int64_t row = r0; row < r1; ++row) {
            const uint32_t s = find(first, last - first + 1, row, [&](uint32_t i) { return off[i]; });
            if (!(off[s] <= row && row < off[s + 1])) { std::printf("row %lld in sequence %u\n", (long long)row, s); return 1; }
        }
        std::vector<int64_t> bad(off);
        for (auto& v : bad) v = (int64_t)gen() % 1000 - 500;
        for (int64_t row = r0; row < r1; ++row) find(first, last - first + 1, row, [&](uint32_t i) { return bad[i]; });
    }
    // the most sequences that a call admits: offsets[s] = s, all in front of the row, all behind it
    const uint32_t all = 2147483647u;
    for (uint32_t first : {0u, 1u, 1000000u, all - 70u, all - 1u}) {
        const uint32_t count = all - first;
        for (uint32_t at : {0u, 1u, 63u, 64u, count / 3, count / 2, count - 2, count - 1}) {
            if (at >= count) continue;
            if (find(first, count, (int64_t)first + at, [](uint32_t i) { return (int64_t)i; }) != first + at) { std::printf("not %u\n", first + at); return 1; }
        }
        if (find(first, count, 5, [](uint32_t) { return (int64_t)0; }) != all - 1) return 1;
        if (find(first, count, 5, [](uint32_t) { return (int64_t)6; }) != first) return 1;
    }
    // rounds over the sequences behind the first 64: none for those, all of them covered, and the bisection's turn past the limit
    for (uint32_t count : {0u, 1u, 63u, 64u, 65u, 320u, 321u, 2112u, 2113u, 100000u, 1048576u, all}) {
        const uint64_t rounds = fs::mark_rounds(count), covered = fs::kWave + rounds * fs::kBlock;
        if (covered < count || (rounds > 0 && covered - fs::kBlock >= count)) { std::printf("%llu rounds for %u\n", (unsigned long long)rounds, count); return 1; }
    }
    if (fs::mark_rounds(64) != 0 || fs::mark_rounds(all) <= fs::kMostMarkRounds || fs::kMostMarkRounds > 32) return 1;
    std::printf("marks ok\n");
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")
def test_few_loads_find_a_rows_sequence(tmp_path):
    src, exe = tmp_path / "driver.cpp", tmp_path / "driver"
    src.write_text(DRIVER)
    built = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
                            "-I" + os.path.join(ROCM, "include"), "-I" + os.path.join(ROOT, "include"),
                            "-I" + os.path.join(ROOT, "paper_2301_02959_amd", "csrc"), str(src), "-o", str(exe)],
                           capture_output=True, text=True)
    assert built.returncode == 0, built.stderr[-2000:]
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "marks ok" in run.stdout, run.stdout + run.stderr
