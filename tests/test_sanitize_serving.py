"""AddressSanitizer / UndefinedBehaviorSanitizer run of the serving entry points' host-only argument checks and workspace carving."""
import os

from tests.test_sanitize_host import ROOT, _build_and_run


def test_serving_validation_and_workspace_carving_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "seq_layout_check.cc")],
                         ["-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2506_16640_amd", "csrc")])
    assert int(out.split()[1]) > 1000
