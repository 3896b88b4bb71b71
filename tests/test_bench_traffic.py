"""The benchmark quotes a stored traffic figure for the kernels that it was measured on, whatever changes beside them."""
import os
import shutil

import pytest

import bench

SERVING = ("paged", "beam")  # operators that no workload of the benchmark runs


@pytest.fixture
def csrc(tmp_path, monkeypatch):
    copy = tmp_path / "csrc"
    shutil.copytree(bench.CSRC, copy)
    monkeypatch.setattr(bench, "CSRC", str(copy))
    return copy


def test_serving_operators_leave_the_hash_alone(csrc):
    before = bench.sources_sha256()
    changed = [n for n in os.listdir(csrc) if n.startswith(SERVING)]
    assert len(changed) >= 10
    for name in changed:
        (csrc / name).write_text("// changed\n")
    assert bench.sources_sha256() == before


@pytest.mark.parametrize("name", ["mfma_fwd.hip", "common.h", "launch.h", "select.hip"])
def test_the_workloads_kernels_do_not(csrc, name):
    before = bench.sources_sha256()
    (csrc / name).write_text((csrc / name).read_text() + "// changed\n")
    assert bench.sources_sha256() != before
