"""Which sources the committed counter readings of bench.py go by (no GPU)."""
import importlib.util
import json
import os
import shutil

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def bench(tmp_path, monkeypatch):
    spec = importlib.util.spec_from_file_location("bench", os.path.join(ROOT, "bench.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    shutil.copytree(os.path.join(ROOT, "paper_1807_06629_amd", "csrc"), tmp_path / "paper_1807_06629_amd" / "csrc")
    os.mkdir(tmp_path / "profiles")
    monkeypatch.setattr(m, "ROOT", str(tmp_path))
    m.csrc = tmp_path / "paper_1807_06629_amd" / "csrc"
    with open(tmp_path / "profiles" / "hbm_traffic.json", "w") as f:
        json.dump({"c5": {"gemm_bwd": {"source_sha256": m.kernel_source_digest(), "traffic_bytes_per_launch": 5.0, "counters": {"a": 1}}}}, f)
    return m


def _change(path):
    with open(path, "a") as f:
        f.write("// changed\n")


@pytest.mark.parametrize("name", ["kernels_norm.hip", "kernels_orth.hip", "kernels_square.hip", "orth_rows.h", "prsgd_ops_api.hip",
                                  "prsgd_ops_internal.h"])
def test_the_operators_sources_leave_the_methods_readings_valid(bench, name):
    _change(bench.csrc / name)
    assert bench.measured_traffic("c5", "gemm_bwd") == 5.0 and bench.measured_counters("c5", "gemm_bwd") == {"a": 1}


def test_the_methods_own_sources_do_not(bench):
    own = sorted(p.name for p in bench.csrc.iterdir() if p.suffix in (".hip", ".h") and p.name not in bench.OPERATOR_SOURCES)
    assert "kernels_gemm.hip" in own or any(n.startswith("kernels_") for n in own)
    digests = {bench.kernel_source_digest()}
    for name in own:
        _change(bench.csrc / name)
        digests.add(bench.kernel_source_digest())
        assert bench.measured_traffic("c5", "gemm_bwd") is None
    assert len(digests) == len(own) + 1
