"""The plan of a serving step with its kernels run on the CPU, lane by lane, and a workgroup's waves in the orders that depend most on its barriers (tests/emulate)."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

from tests.step_util import plain_plan
from tests.test_gpu_cache_plan import DECODE, MIXED, _problem
from tests.test_sanitize_host import ROOT


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("emulate") / "plan_emulated.so")
    here = os.path.join(ROOT, "tests", "emulate")
    clang = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++")
    subprocess.run([clang, "-x", "c++", "-std=c++17", "-O1", "-fPIC", "-shared", "-w", "-I", here, "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2506_16640_amd", "csrc"), os.path.join(here, "plan_emulated.cc"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.entmax_cache_plan.argtypes = [ctypes.c_char_p] + [ctypes.c_void_p] * 13 + [ctypes.c_size_t, ctypes.c_void_p]
    lib.emulate_end.restype = ctypes.c_char_p
    return lib


def check(lib, order, new, kv, table, free, count, page, rows, release=None, in_place=False):
    from paper_2506_16640_amd import binding
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    nseq, columns = len(new), len(table[0])
    p = binding._plan_bytes.pack(nseq, rows, page, len(free), columns)
    t_new, t_kv, t_table, t_free, t_count = i32(new), i32(kv), i32(table), i32(free), i32([count])
    t_release = None if release is None else i32(release)
    kv_out, count_out = (t_kv, t_count) if in_place else (i32([77] * nseq), i32([77]))
    cu, positions, sequences = i32([77] * (nseq + 1)), i32([77] * rows), i32([77] * rows)
    slots = torch.full((rows,), 77, dtype=torch.int64)
    ws = torch.full((512 + 4 * nseq + 1024,), 255, dtype=torch.uint8)
    lib.emulate_begin(order)
    rc = lib.entmax_cache_plan(p, *[None if t is None or t.numel() == 0 else t.data_ptr() for t in
                                    (t_new, t_release, t_kv, t_count, t_table, t_free, kv_out, count_out, cu, slots, positions, sequences)],
                               (ws.data_ptr() + 255) // 256 * 256, ws.numel() - 256, None)
    assert rc == 0
    error = lib.emulate_end().decode()
    assert not error, error
    want_cu, left, want_slots, want_positions, want_sequences = plain_plan(new, kv, table, free, count, page, rows, release)
    assert cu.tolist() == want_cu and kv_out.tolist() == kv and count_out.tolist() == [left]
    assert positions.tolist() == want_positions and sequences.tolist() == want_sequences and slots.tolist() == want_slots
    assert t_table.tolist() == table and t_free.tolist() == free


@pytest.mark.parametrize("order", [0, 1, 2])
@pytest.mark.parametrize("nseq,rows", [(1, None), (64, 64), (65, None), (200, 256), (300, None), (2048, 4000), (2049, None), (4100, 2000)])
@pytest.mark.parametrize("new", [DECODE, MIXED], ids=["decode", "mixed"])
def test_steps(lib, order, nseq, rows, new):
    rng = random.Random(nseq)
    for share in (0.0, 0.3, 1.0):
        n, kv, table, free, count, release = _problem(rng, nseq, 16, 40, nseq // 2 + 4, new, 600, released=share)
        check(lib, order, n, kv, table, free, count, 16, sum(n) + 1 if rows is None else rows, release if share else None, in_place=share > 0.5)


@pytest.mark.parametrize("order", [0, 1])
def test_numbers_that_make_no_sense(lib, order):
    big = 2 ** 31 - 1
    new = [1, -5, big, 3, 20, 1, big, 2]
    kv = [15, 4, 10, -7, 16, 64, big, 0]
    table = [[5, 1, 2, 3], [0, 9, 9, 9], [6, 9, 9, 9], [9] * 4, [-2, 9, 9, 9], [9] * 4, [7, 8, -1, 12], [9] * 4]
    for release in (None, [0, 0, 0, 1, 0, 0, 1, 1]):
        for count in (10, -4, 99):
            free = [10, 11, -6, 3, 99, 4, 2, 1, 0, 13]
            check(lib, order, list(new), list(kv), [list(r) for r in table], free, count, 16, 40, release)
