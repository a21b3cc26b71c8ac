"""Which tokens a store copy moves (csrc/gkv_store_rows.h), compiled for the host with the checks for undefined arithmetic on: at the
ends of the range of first and count, with more tokens than rows, and everywhere near the borders."""
import subprocess
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent
PROGRAM = r"""
#include <stdio.h>
#include <vector>
#include "gkv_store_rows.h"
int main() {
    const int64_t lowest = INT32_MIN, highest = INT32_MAX;
    std::vector<int64_t> edge;
    for (int64_t base : {lowest, highest, (int64_t)0, (int64_t)100, (int64_t)-100, (int64_t)1 << 24, (int64_t)1 << 30, -((int64_t)1 << 30)})
        for (int64_t d : {-300, -257, -129, -65, -9, -8, -7, -1, 0, 1, 7, 8, 9, 64, 128, 257, 300})
            if (base + d >= lowest && base + d <= highest) edge.push_back(base + d);
    long runs = 0, moved = 0;
    for (int capacity : {1, 7, 8, 96, 100, 1 << 24})
        for (int n_tokens : {1, 8, 64, 65, 256, (1 << 24) + 300, (1 << 30) - 1})
            for (int64_t first : edge)
                for (int64_t count : edge)
                    for (int64_t at : {(int64_t)0, (int64_t)8, (int64_t)64, (int64_t)96, (int64_t)104, -first, capacity - first, count, (int64_t)n_tokens})
                        for (int64_t t = (at & ~(int64_t)7) - 8; t <= (at & ~(int64_t)7) + 8; t += 8) {
                            if (t < 0 || t > n_tokens + 64) continue;
                            const gkv::RunRows r = gkv::run_rows((int32_t)first, (int32_t)count, n_tokens, capacity, (int)t);
                            ++runs;
                            if (r.lo < 0 || r.lo > gkv::kRun || r.hi < 0 || r.hi > gkv::kRun) { printf("range\n"); return 1; }
                            for (int64_t i = 0; i < gkv::kRun; ++i) {
                                const bool is = i >= r.lo && i < r.hi;
                                const bool want = t + i < n_tokens && t + i < count && first + t + i >= 0 && first + t + i < capacity;
                                moved += is;
                                if (is != want) {
                                    printf("first %ld count %ld tokens %d capacity %d token %ld: %d\n", (long)first, (long)count, n_tokens, capacity, (long)(t + i), (int)is);
                                    return 1;
                                }
                            }
                        }
    printf("%ld %ld\n", runs, moved);
    return 0;
}
"""


def test_rows_of_a_run_over_the_whole_range(tmp_path):
    (tmp_path / "rows.cc").write_text(PROGRAM)
    exe = tmp_path / "rows"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                           str(ROOT / "paper_2512_00504_b200" / "csrc"), "-o", str(exe), str(tmp_path / "rows.cc")])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    runs, moved = (int(x) for x in r.stdout.split())
    assert runs > 100000 and moved > 10000
