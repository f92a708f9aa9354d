"""Counter summaries are quoted for the sources they were taken on: of the kernel that they describe, and of no other."""
import shutil

import pytest

import bench


@pytest.fixture
def sources(tmp_path, monkeypatch):
    shutil.copytree(bench.CSRC, tmp_path / "csrc")
    monkeypatch.setattr(bench, "CSRC", str(tmp_path / "csrc"))
    return tmp_path / "csrc"


@pytest.mark.parametrize("name, its", [
    ("lychee_layer.hip", True), ("lychee_api.hip", True), ("lychee_select.h", True), ("lychee_stream.h", True), ("lychee_device.h", True),
    ("lychee_internal.h", True), ("lychee_plan.h", True), ("lychee_context.h", True),
    ("lychee_prompt.hip", False), ("lychee_prompt_device.h", False), ("lychee_q4.hip", False), ("lychee_units.hip", False),
    ("lychee_another.hip", False), ("lychee_another.h", False)])
def test_the_stamp_is_of_the_kernels_own_sources(sources, name, its):
    before = bench.source_stamp()
    with open(sources / name, "a") as f:
        f.write("// another line\n")
    assert (bench.source_stamp() != before) == its


def test_the_layer_launch_has_its_measured_traffic():
    """The committed counters are of the committed sources; bench.py says null otherwise."""
    assert bench.measured_traffic() is not None, "take profiles/lychee_layer_kernel_c3_pmc.txt again: stamp %s" % bench.source_stamp()
