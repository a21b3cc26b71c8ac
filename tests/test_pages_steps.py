"""A warp's ring of copies in the paged attention (csrc/gkv_pages_steps.h), compiled for the host: a warp that gives up waits for exactly the
copies that are under way, whichever step it gives up at; and the arguments of the self-test that takes this path."""
import ctypes
import subprocess
from pathlib import Path

import paper_2512_00504_b200 as gkv
from test_pages_refusals import A, BAD, OK, pages, ref, table

ROOT = Path(__file__).resolve().parent.parent
PROGRAM = r"""
#include <stdio.h>
#include <vector>
#include "gkv_pages_steps.h"
struct Fill { int stage; uint32_t parity; };
// A warp of `steps` steps that gives up at `at` (from `steps` on: never), as the kernel goes through its ring.
template <int S>
int go(int steps, int at) {
    std::vector<Fill> fills;                                // of step s: what a ring of S barriers means by it
    for (int s = 0; s < steps; ++s) fills.push_back({s % S, (uint32_t)(s / S) & 1u});
    gkv::RingPlace<S> place;
    bool ok = true;
    int issued = steps < S ? steps : S, gave_up = 0;
    for (int step = 0; step < steps; ++step) {
        if (ok && (place.stage != fills[step].stage || place.parity != fills[step].parity)) return printf("step %d\n", step);
        if (ok && step >= at) { ok = false; gave_up = step; }
        if (issued < steps && ok) {
            if (fills[issued].stage != place.stage) return printf("issue %d\n", issued);
            ++issued;
        }
        if (ok) place.next();
    }
    if (ok) return 0;
    int next = gave_up;
    bool right = true;
    gkv::drain_ring(place, issued - gave_up, [&](int stage, uint32_t parity) {
        right = right && next < issued && fills[next].stage == stage && fills[next].parity == parity;
        ++next;
    });
    return right && next == issued ? 0 : printf("S %d steps %d at %d\n", S, steps, at);
}
int main() {
    for (int steps = 1; steps <= 14; ++steps)
        for (int at = 0; at <= steps; ++at)
            if (go<2>(steps, at) || go<3>(steps, at)) return 1;
    return 0;
}
"""


def test_copies_under_way_where_a_warp_gives_up(tmp_path):
    (tmp_path / "ring.cc").write_text(PROGRAM)
    exe = tmp_path / "ring"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                           str(ROOT / "paper_2512_00504_b200" / "csrc"), "-o", str(exe), str(tmp_path / "ring.cc")])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def test_selftest_arguments():
    gkv.build_library()
    L, none = gkv.lib(), ctypes.c_uint64()
    assert L.gkv_pages_attn_workspace(ref(pages()), 6, ref(none)) == OK

    def call(step, t=table(), q=A, ws_bytes=1 << 40):
        return L.gkv_selftest_pages_wait(step, ref(pages()), ref(t), A, 0, q, 1024, None, None, 0, None, None, A, None, A, ws_bytes, None)

    assert call(-1) == BAD and call(2 ** 31 - 1) == BAD and call(0, q=0) == BAD and call(0, ws_bytes=1000) == BAD and call(0, t=table(width=0)) == BAD
    assert call(0) == gkv.GKV_ERR_UNSUPPORTED                # 160 rows at most: no such waits
