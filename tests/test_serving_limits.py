"""Sizes and layouts that the serving entry points refuse or take at their limits, before anything reaches a GPU."""
import os

import pytest

from tests.test_sanitize_host import ROOT, _build_and_run
from tests.test_serving_refusals import app, b, call_append, call_packed, call_paged, packed, seq  # noqa: F401


def test_append_checks_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "append_check.cc")],
                         ["-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2506_16640_amd", "csrc")])
    assert int(out.split()[1]) > 1000


@pytest.mark.parametrize("Hkv", [4097, 1 << 24, (1 << 31) - 1])
def test_many_key_heads_without_queries(b, Hkv):  # noqa: F811
    # (with queries, their number is bounded as well)
    assert call_append(b, app(b, Hq=0, Hkv=Hkv)) == -2


def test_append_of_more_tokens_than_a_launch_holds(b):  # noqa: F811
    assert call_append(b, app(b, T=1 << 26)) == -2
