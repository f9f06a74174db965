"""Tiles of paged and packed keys go from global memory straight to LDS, whole ones with a scalar address, ragged ones with an address for every lane; the
wait states of both, as in test_lds_load_wait_states.py."""
import os
import re
import subprocess

import pytest

from paper_2506_16640_amd import build
from tests.test_lds_load_wait_states import _registers, _wait_states

SOURCE = """
#include <hip/hip_runtime.h>
#include "seq.hip.h"
using namespace entmax;
using Tile = SeqTile<%s, %d, 64, %s>;
__global__ void k(SeqGeom g, SeqView v, const char* src, uint4* out) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  SeqKeys keys;
  keys.init(g, v, src, blockIdx.x, false, sizeof(%s));
  Tile::Pages pg;
  pg.ask(keys, blockIdx.y * 64, v.L, wave);
  Tile::load(keys, pg, blockIdx.y * 64, v.L, (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem, wave, lane);
  lds_loads_wait<0>();
  __syncthreads();
  out[threadIdx.x] = reinterpret_cast<uint4*>(smem)[threadIdx.x ^ 1];
}
"""


@pytest.mark.parametrize("values", ["false", "true"])
@pytest.mark.parametrize("ctype,D", [("bf16_t", 64), ("bf16_t", 128), ("float", 64)])
def test_tiles_of_sequences_keep_the_hazard_rules(tmp_path, ctype, D, values):
    src, asm = tmp_path / "k.hip", tmp_path / "k.s"
    src.write_text(SOURCE % (ctype, D, values, ctype))
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + build.HIPCC_FLAGS + [
        "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "--cuda-device-only", "-S", str(src), "-o", str(asm)]
    subprocess.run(cmd, check=True, capture_output=True)
    lines = [re.sub(r";.*", "", l).strip() for l in asm.read_text().splitlines()]
    lines = [l for l in lines if l and not l.startswith(".") and not l.endswith(":")]
    loads = [n for n, l in enumerate(lines) if l.startswith("global_load_lds_dwordx4")]
    whole = [n for n in loads if lines[n].split(",")[1].strip().startswith("s[")]
    ragged = [n for n in loads if lines[n].split(",")[1].strip() == "off"]
    assert whole and ragged and len(whole) + len(ragged) == len(loads)
    for n in loads:
        address = _registers(lines[n].split(",")[1].strip()) if n in whole else set()
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
