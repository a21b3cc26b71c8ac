"""The other configurations in the benchmark's line: shorter, and nothing lost but digits behind the sixth (no GPU needed)."""
import json
import math
import sys
from pathlib import Path

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
import bench  # noqa: E402


def cell(i):
    return {"b": 256 * (1 + i % 4), "batch": 64, "ms": {"score": 0.029904000461101532 * (i + 1), "fused": 0.03 / 7 * (i + 1)},
            "fused_bytes": 121611264.0 + i, "score_bound": "hbm", "fused_frac": 1 / 3 + i, "cpu_baseline": {"value": 1e6 / 7, "sample": f"{i} of 64"}}


def test_records_become_a_table_and_come_back():
    cells = [cell(i) for i in range(16)]
    configs = {"cfg0": {"cell": cells[0], "clocks": {"reasons": [], "samples": 1}, "note": None}, "cfg3": {"cells": cells, "min": 1 / 3}}
    got = json.loads(json.dumps(bench.short(configs)))
    table = got["cfg3"]["cells"]
    assert table["same"] == {"batch": 64, "score_bound": "hbm", "cpu_baseline.value": 142857} and len(table["rows"]) == 16
    for row, want in zip(table["rows"], cells):
        have, want = {**table["same"], **dict(zip(table["columns"], row))}, bench.flatten(want)
        assert have.keys() == want.keys()
        for k, v in want.items():
            assert have[k] == v if not isinstance(v, float) else math.isclose(have[k], v, rel_tol=5.1e-6), k
    assert [r[table["columns"].index("fused_bytes")] for r in table["rows"]] == [121611264 + i for i in range(16)]     # counts stay whole
    assert got["cfg0"]["clocks"] == {"reasons": [], "samples": 1} and got["cfg0"]["note"] is None and got["cfg0"]["cell"]["ms"]["score"] == 0.029904
    assert 2 * len(json.dumps(got)) < 1.5 * len(json.dumps(configs))


def test_lists_of_other_things_stay():
    x = {"a": [1, 2.5, "x"], "one": [{"b": 1.0 / 3}], "mixed": [{"b": 1}, {"c": 2}], "inf": math.inf}
    assert bench.short(x) == {"a": [1, 2.5, "x"], "one": [{"b": 0.333333}], "mixed": [{"b": 1}, {"c": 2}], "inf": math.inf}
