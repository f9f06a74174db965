"""The 64-bit exponential of the sampling kernels as it is compiled: its argument is bounded before it is taken apart.  Otherwise the compiler forms argument minus whole part
from the unrounded product: beyond 2^53 that is no fraction but a number of any size, whose polynomial overflows."""
import os
import re
import subprocess

from paper_2506_16640_amd import build

SOURCE = """
#include <hip/hip_runtime.h>
#include "sample.hip"
__global__ void weights(const float* x, const float* m, const double* scale, double* out) {
  RowAsk ask;
  ask.scale = scale[0];
  out[threadIdx.x] = ask.weight(x[threadIdx.x], m[0]);
}
"""


def test_exponents_are_bounded(tmp_path):
    src, asm = tmp_path / "w.hip", tmp_path / "w.s"
    src.write_text(SOURCE)
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + build.HIPCC_FLAGS + [
        "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S", str(src), "-o", str(asm)]
    subprocess.run(cmd, check=True, capture_output=True)
    written, seen = {}, 0
    for line in asm.read_text().splitlines():
        m = re.match(r"\s+(v_\w+)\s+(v\[\d+:\d+\]),\s*(.*)", line)
        if not m:
            continue
        op, to, args = m.groups()
        if op.startswith("v_rndne_f64"):
            seen += 1
            assert written.get(args.strip(), "").startswith("v_max_f64"), (args, written.get(args.strip()))
        written[to] = op
    assert seen > 0
