"""GPU tests of the plan of a serving step: whole numbers, equal to those of a loop over sequences and tokens."""
import random

import pytest
import torch

from tests.step_util import plain_plan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2506_16640_amd import binding as b
    return b


def _problem(rng, nseq, page, columns, spare, new, cached, released=0.0):
    kv = [rng.randint(0, cached) for _ in range(nseq)]
    per = [-(-L // page) for L in kv]
    perm = list(range(sum(per) + spare))
    rng.shuffle(perm)
    table, at = [], 0
    for n in per:
        table.append((perm[at:at + n] + [-9] * columns)[:columns])
        at += n
    free = perm[at:] + [-3] * at
    release = [int(rng.random() < released) * rng.choice([1, 5, -1]) for _ in range(nseq)]
    return [new(rng) for _ in range(nseq)], kv, table, free, spare, release


def _check(binding, new, kv, table, free, count, page, rows, release=None, in_place=False):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    nseq, columns = len(new), len(table[0]) if table else 4
    plan = binding.new_plan(nseq, rows)
    for t in plan[:-1]:
        t.fill_(77)
    t_new, t_kv, t_free, t_count = i32(new), i32(kv), i32(free), i32([count])
    t_table = i32(table).reshape(nseq, columns)
    t_release = None if release is None else i32(release)
    if in_place:
        plan = plan._replace(kv_len=t_kv, free_count=t_count)
    binding.cache_plan(t_new, t_kv, t_table, t_free, t_count, page, plan, release=t_release)
    torch.cuda.synchronize()
    cu, left, slots, positions, sequences = plain_plan(new, kv, table, free, count, page, rows, release)
    assert plan.cu_seqlens.tolist() == cu
    assert plan.kv_len.tolist() == kv
    assert plan.free_count.tolist() == [left]
    assert plan.positions.tolist() == positions and plan.sequences.tolist() == sequences
    assert plan.slots.tolist() == slots
    assert t_table.tolist() == table and t_free.tolist() == free


DECODE = lambda rng: 1  # noqa: E731
MIXED = lambda rng: rng.choice([0, 1, 1, 1, rng.randint(2, 90)])  # noqa: E731


@pytest.mark.parametrize("nseq", [1, 2, 63, 64, 65, 1000, 1024, 1025, 2048, 2049, 5000])
@pytest.mark.parametrize("new", [DECODE, MIXED], ids=["decode", "mixed"])
def test_sequences(binding, nseq, new):
    rng = random.Random(nseq)
    n, kv, table, free, count, _ = _problem(rng, nseq, 16, 12, 3 * nseq + 5, new, 60)
    _check(binding, n, kv, table, free, count, 16, sum(n) + 3)


@pytest.mark.parametrize("page", [16, 64, 512, 65536])
def test_page_sizes(binding, page):
    rng = random.Random(page)
    n, kv, table, free, count, _ = _problem(rng, 37, page, 5, 200, lambda r: r.choice([0, 1, 2, min(page + 1, 700)]), 3 * page)
    _check(binding, n, kv, table, free, count, page, sum(n))


@pytest.mark.parametrize("rows", [0, 1, 500, 4096, 4097, 20000])
def test_rows_that_do_not_suffice(binding, rows):
    rng = random.Random(rows)
    n, kv, table, free, count, _ = _problem(rng, 300, 16, 40, 3000, MIXED, 300)
    _check(binding, n, kv, table, free, count, 16, rows)


@pytest.mark.parametrize("count", [0, 1, 40, 150])
@pytest.mark.parametrize("nseq", [100, 3000])
def test_pages_that_do_not_suffice(binding, count, nseq):
    """Those that need no page go on; of the others the first ones are served."""
    rng = random.Random(count)
    n, kv, table, free, _, _ = _problem(rng, nseq, 16, 12, 150, MIXED, 60)
    _check(binding, n, kv, table, free, count, 16, sum(n))


@pytest.mark.parametrize("nseq", [1, 30, 1500, 4000])
@pytest.mark.parametrize("share", [0.1, 0.6, 1.0])
@pytest.mark.parametrize("in_place", [False, True])
def test_release(binding, nseq, share, in_place):
    """Ended sequences give their pages back, some begin again in the same step with pages that have just come back."""
    rng = random.Random(nseq)
    n, kv, table, free, count, release = _problem(rng, nseq, 16, 70, 4, MIXED, 1100, released=share)
    _check(binding, n, kv, table, free, count, 16, sum(n) + 1, release, in_place)


def test_numbers_that_make_no_sense(binding):
    """Negative and huge lengths, entries that are no page, a count beyond the list: nothing outside the arrays is touched, and the others are served."""
    big = 2 ** 31 - 1
    new = [1, -5, big, 3, 20, 1, big, 2]
    kv = [15, 4, 10, -7, 16, 64, big, 0]
    table = [[5, 1, 2, 3], [0, 9, 9, 9], [6, 9, 9, 9], [9] * 4, [-2, 9, 9, 9], [9] * 4, [7, 8, -1, 12], [9] * 4]
    for release in (None, [0, 0, 0, 1, 0, 0, 1, 1]):
        for count in (10, -4, 99):
            free = [10, 11, -6, 3, 99, 4, 2, 1, 0, 13]
            _check(binding, list(new), list(kv), [list(r) for r in table], free, count, 16, 40, release)


def test_a_list_that_is_full_takes_no_more(binding):
    table = [[0, 1, 2, 0], [1, 1, 1, 1]]
    _check(binding, [0, 0], [64, 50], table, [0, 1, 2], 2, 16, 4, [1, 1])


def test_no_sequences(binding):
    plan = binding.new_plan(0, 5)
    free, count = torch.arange(4, dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda")
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    plan.cu_seqlens.fill_(9)
    binding.cache_plan(empty, empty, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), free, count, 16, plan)
    assert plan.cu_seqlens.tolist() == [0] and plan.free_count.tolist() == [3] and plan.slots.tolist() == [-1] * 5


@pytest.mark.parametrize("missing", [("slots",), ("positions", "sequences"), ("slots", "positions")])
def test_outputs_that_are_not_wanted(binding, missing):
    rng = random.Random(8)
    for nseq in (20, 3000):
        n, kv, table, free, count, _ = _problem(rng, nseq, 16, 12, 3 * nseq, MIXED, 60)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        plan = binding.new_plan(nseq, sum(n) + 2)._replace(**{m: None for m in missing})
        t_table = i32(table)
        binding.cache_plan(i32(n), i32(kv), t_table, i32(free), i32([count]), 16, plan)
        cu, left, slots, positions, sequences = plain_plan(n, kv, table, free, count, 16, sum(n) + 2)
        assert plan.cu_seqlens.tolist() == cu and t_table.tolist() == table
        for name, want in (("slots", slots), ("positions", positions), ("sequences", sequences)):
            assert name in missing or getattr(plan, name).tolist() == want


def test_long_cache_slots(binding):
    """Places beyond 32 bits."""
    page, pages = 65536, 40000
    free = torch.arange(pages, dtype=torch.int32, device="cuda")
    plan = binding.new_plan(2, 3)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.full((2, 3), 39990, dtype=torch.int32, device="cuda")
    binding.cache_plan(i32([1, 2]), i32([65536, 70000]), table, free, i32([pages]), page, plan)
    assert plan.slots.tolist() == [39999 * page, 39990 * page + 4464, 39990 * page + 4465]
    assert table[0].tolist() == [39990, 39999, 39990]


def test_many_steps_in_place(binding):
    """A captured step replayed with other numbers: pages wander between the list and the sequences, none is lost or given twice."""
    rng = random.Random(3)
    nseq, page, columns, pages, rows = 40, 16, 10, 120, 64
    dev = "cuda"
    new, release = (torch.zeros(nseq, dtype=torch.int32, device=dev) for _ in range(2))
    table = torch.full((nseq, columns), -1, dtype=torch.int32, device=dev)
    free = torch.arange(pages, dtype=torch.int32, device=dev)
    plan = binding.new_plan(nseq, rows)
    plan.free_count.fill_(pages)
    binding.cache_plan(new, plan.kv_len, table, free, plan.free_count, page, plan, release=release)  # (no tokens: nothing changes)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.cache_plan(new, plan.kv_len, table, free, plan.free_count, page, plan, release=release)
    kv, t, f, count = [0] * nseq, [[-1] * columns for _ in range(nseq)], list(range(pages)), pages
    for _ in range(60):
        n = [rng.choice([0, 1, 1, 7, 30]) for _ in range(nseq)]
        r = [int(rng.random() < 0.1) for _ in range(nseq)]
        new.copy_(torch.tensor(n, dtype=torch.int32))
        release.copy_(torch.tensor(r, dtype=torch.int32))
        graph.replay()
        cu, count, slots, positions, sequences = plain_plan(n, kv, t, f, count, page, rows, r)
        assert plan.cu_seqlens.tolist() == cu and plan.kv_len.tolist() == kv and plan.free_count.tolist() == [count]
        assert plan.slots.tolist() == slots and table.tolist() == t and free.tolist() == f
        used = [t[s][e] for s in range(nseq) for e in range(-(-kv[s] // page))]
        assert sorted(used + f[:count]) == list(range(pages))
