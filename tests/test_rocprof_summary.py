"""Which source changes void counter figures taken on the layer's kernels."""
import shutil

import pytest

from paper_2311_10770_amd import rocprof_summary


@pytest.fixture
def sources(tmp_path, monkeypatch):
    shutil.copytree(rocprof_summary.PKG / "csrc", tmp_path / "csrc")
    monkeypatch.setattr(rocprof_summary, "PKG", tmp_path)
    return tmp_path / "csrc"


@pytest.mark.parametrize("name", ["fff_norm.hip", "fff_group.hip", "fff_grouped.hip", "fff_grouped_grad.hip",
                                  "fff_grouped.hpp", "fff_rows.hpp", "fff_operators.hpp", "fff_api.cpp"])
def test_other_kernels_leave_the_hash(sources, name):
    before = [rocprof_summary.kernel_source_hash(b) for b in (False, True)]
    with open(sources / name, "a") as f:
        f.write("\n// changed\n")
    assert [rocprof_summary.kernel_source_hash(b) for b in (False, True)] == before


@pytest.mark.parametrize("name,forward,backward", [
    ("fff_kernels.hip", True, False), ("fff_dense.hip", True, False), ("fff_masked.hip", True, False),
    ("fff_gemm.hip", True, False), ("fff_subtree.hip", True, False), ("fff_wide.hip", True, False),
    ("fff_backward.hip", False, True), ("fff_internal.hpp", True, True), ("fff_device.hpp", True, True),
    ("fff_common.hpp", True, True)])
def test_the_layers_kernels_change_the_hash(sources, name, forward, backward):
    before = [rocprof_summary.kernel_source_hash(b) for b in (False, True)]
    with open(sources / name, "a") as f:
        f.write("\n// changed\n")
    after = [rocprof_summary.kernel_source_hash(b) for b in (False, True)]
    assert [a != b for a, b in zip(after, before)] == [forward, backward]
