"""Which of a block's tokens the rotation turns (csrc/gkv_store_rows.h), compiled for the host with the checks for undefined arithmetic
on: a count near the lower end of 32 bits is as good as 0 in every block, not only in the first."""
import subprocess
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent
PROGRAM = r"""
#include <initializer_list>
#include <stdio.h>
#include "gkv_store_rows.h"
int main() {
    const int64_t lowest = INT32_MIN, highest = INT32_MAX;
    long cases = 0, some = 0;
    for (int n_tokens : {1, 2, 33, 4097, (1 << 30) - 1})
        for (int per : {1, 2, 8, 64})
            for (int64_t base : {lowest, highest, (int64_t)0, (int64_t)n_tokens, -((int64_t)1 << 30), (int64_t)1 << 30})
                for (int64_t d = -70; d <= 70; ++d)
                    for (int64_t block : {(int64_t)0, (int64_t)1, (int64_t)2, (int64_t)n_tokens / per / 2, (int64_t)(n_tokens - 1) / per}) {
                        const int64_t count = base + d, t0 = block * per;
                        if (count < lowest || count > highest || t0 >= n_tokens) continue;
                        int64_t want = 0;
                        for (int64_t t = t0; t < t0 + per; ++t) want += t < count && t < n_tokens;
                        const int got = gkv::tokens_here((int32_t)count, n_tokens, (int)t0, per);
                        ++cases;
                        some += got > 0;
                        if (got != want) {
                            printf("count %ld of %d, block at %ld of %d: %d\n", (long)count, n_tokens, (long)t0, per, got);
                            return 1;
                        }
                    }
    printf("%ld %ld\n", cases, some);
    return 0;
}
"""


def test_tokens_of_a_block_over_the_whole_range(tmp_path):
    (tmp_path / "tokens.cc").write_text(PROGRAM)
    exe = tmp_path / "tokens"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                           str(ROOT / "paper_2512_00504_b200" / "csrc"), "-o", str(exe), str(tmp_path / "tokens.cc")])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    cases, some = (int(x) for x in r.stdout.split())
    assert cases > 5000 and some > 1000
