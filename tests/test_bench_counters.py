"""Which sources the counters of profiles/counters.json are tied to."""
import shutil

import pytest

import bench


@pytest.mark.parametrize("name,counts", [("select.hip", True), ("grad.hip", True), ("devutil.h", True), ("engine.hip", True), ("products.hip", False),
                                         ("norm.hip", False), ("preference.hip", False), ("layers.h", False)])
def test_counters_hold_until_a_source_of_the_step_changes(name, counts, tmp_path, monkeypatch):
    """engine.hip decides which of the step's kernels are launched, and for which sizes; the operators of other models take no part in it."""
    shutil.copytree(bench.CSRC, tmp_path / "csrc")
    monkeypatch.setattr(bench, "CSRC", str(tmp_path / "csrc"))
    before = bench.kernel_sources_digest()
    with open(tmp_path / "csrc" / name, "a") as f:
        f.write("// another line\n")
    assert (bench.kernel_sources_digest() != before) == counts
