"""cos and sin of the rotation (csrc/gkv_rotary_series.h), compiled for the host, over the whole range of angles and both ends of what an
angle that was cut may have been: within the error that the source states."""
import subprocess
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent
PROGRAM = r"""
#include <stdio.h>
#include "gkv_rotary_series.h"
int main() {
    const double step = 2 * 3.14159265358979323846 / 4294967296.0;
    double most_c = 0, most_s = 0;
    for (int64_t rest = -(1ll << 29); rest <= (1ll << 29); rest += rest < -(1ll << 29) + 100000 || rest >= (1ll << 29) - 100000 ? 1 : 97) {
        float c, s;
        gkv::small_cos_sin((int32_t)rest, &c, &s);
        const double C = cos(rest * step), S = sin(rest * step);
        most_c = fmax(most_c, fmax(fabs(c - C), fabs(c - (C - step * S))));      // the angle, and one 2^-32 of a turn further on
        most_s = fmax(most_s, fmax(fabs(s - S), fabs(s - (S + step * C))));
    }
    printf("%.3f %.3f\n", most_c * 16777216, most_s * 16777216);
    return 0;
}
"""


def test_cos_and_sin_over_all_angles(tmp_path):
    (tmp_path / "series.cc").write_text(PROGRAM)
    exe = tmp_path / "series"
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-I", str(ROOT / "paper_2512_00504_b200" / "csrc"), "-o", str(exe),
                           str(tmp_path / "series.cc")])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    cos, sin = (float(x) for x in r.stdout.split())
    # what the source states; and a sweep that finds less than a rounding's half has looked at nothing
    assert 1.0 < cos <= 1.73 and 1.0 < sin <= 1.53
