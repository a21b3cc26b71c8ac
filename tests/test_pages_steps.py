"""A warp's ring of copies in the paged attention and the shape of its merge (csrc/gkv_pages_steps.h), compiled for the host: a warp that
gives up waits for exactly the copies that are under way, whichever step it gives up at; the merge fits the device that it is for; and the
arguments of the self-test that takes the first path."""
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


MERGE = r"""
#include <stdio.h>
#include "gkv_pages_steps.h"
int main() {
    for (int sms : {1, 16, 74, 132, 148, 160})
        for (int64_t units = 1; units <= 16384; ++units) {
            const gkv::MergeShape m = gkv::merge_shape(units, sms);
            const int64_t room = (m.few ? 2 : 8) * sms;      // CTAs that the device holds
            const int most = m.few ? 3 : 2;
            if (m.few != (units <= 2 * sms) || m.split < 0 || m.split > most) return printf("%d %ld\n", sms, (long)units);
            if (m.split > 0 && (units << m.split) > room) return printf("%d %ld: more than fit\n", sms, (long)units);
            if (m.split < most && (units << (m.split + 1)) <= room) return printf("%d %ld: room left\n", sms, (long)units);
        }
    return 0;
}
"""


def run(tmp_path, program):
    (tmp_path / "steps.cc").write_text("#include <initializer_list>\n" + program)
    exe = tmp_path / "steps"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                           str(ROOT / "paper_2512_00504_b200" / "csrc"), "-o", str(exe), str(tmp_path / "steps.cc")])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def test_copies_under_way_where_a_warp_gives_up(tmp_path):
    run(tmp_path, PROGRAM)


def test_the_merge_fits_the_device(tmp_path):
    run(tmp_path, MERGE)


def test_selftest_arguments():
    gkv.build_library()
    L, none = gkv.lib(), ctypes.c_uint64()
    assert L.gkv_pages_attn_workspace(ref(pages()), 6, ref(none)) == OK

    def call(step, t=table(), q=A, ws_bytes=1 << 40):
        return L.gkv_selftest_pages_wait(step, ref(pages()), ref(t), A, 0, q, 1024, None, None, 0, None, None, A, None, A, ws_bytes, None)

    assert call(-1) == BAD and call(2 ** 31 - 1) == BAD and call(0, q=0) == BAD and call(0, ws_bytes=1000) == BAD and call(0, t=table(width=0)) == BAD
    assert call(0) == gkv.GKV_ERR_UNSUPPORTED                # 160 rows at most: no such waits
