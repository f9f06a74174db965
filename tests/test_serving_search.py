"""The threshold search of the tiled serving kernel, run on the CPU under sanitizers: how close it comes, and in how many sweeps."""
import os

from tests.test_sanitize_host import ROOT, _build_and_run


def test_threshold_search(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "seq_search_check.cc")],
                         ["-std=c++17", "-I", os.path.join(ROOT, "paper_2506_16640_amd", "csrc")])
    assert int(out.splitlines()[-1].split()[1]) > 20000
