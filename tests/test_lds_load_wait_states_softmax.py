"""The softmax attention's tiles of whole rows go from global memory straight to LDS with an address that the kernel makes itself; the wait states of these
loads, as in test_lds_load_wait_states.py."""
import os
import re
import subprocess

import pytest

from paper_2506_16640_amd import build
from tests.test_lds_load_wait_states import _registers, _wait_states

SOURCE = """
#include <hip/hip_runtime.h>
#include "softmax.hip.h"
namespace entmax { template __global__ void softmax_tiled_kernel<bf16_t, %d, false>(SoftmaxArgs); }
"""


@pytest.mark.parametrize("D", [64, 128])
def test_tiles_of_the_softmax_attention_keep_the_hazard_rules(tmp_path, D):
    src, asm = tmp_path / "k.hip", tmp_path / "k.s"
    src.write_text(SOURCE % D)
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + build.HIPCC_FLAGS + [
        "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S", str(src), "-o", str(asm)]
    subprocess.run(cmd, check=True, capture_output=True)
    lines = [re.sub(r";.*", "", l).strip() for l in asm.read_text().splitlines()]
    lines = [l for l in lines if l and not l.startswith(".") and not l.endswith(":")]
    loads = [n for n, l in enumerate(lines) if l.startswith("global_load_lds_dwordx4")]
    places = [lines[n].split(",")[1].strip() for n in loads]
    assert loads and all(x.startswith("s[") or x == "off" for x in places)
    for n, place in zip(loads, places):
        address = _registers(place) if place != "off" else set()
        states, m0_seen = 0, False
        for l in reversed(lines[:n]):
            op, _, args = l.partition(" ")
            dst = args.split(",")[0].strip()
            if dst == "m0" and not m0_seen:
                m0_seen = True
                assert states >= 1, "no wait state between the write of m0 and the load that reads it"
            if op.startswith("v_readfirstlane") and dst in address:
                assert states >= 5, "fewer than five wait states between a vector write of the address and the load"
            if states >= 5 and m0_seen:
                break
            states += _wait_states(l)
        assert m0_seen
