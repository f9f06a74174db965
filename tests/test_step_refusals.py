"""What the entry points of a decode step (plan, softmax attention, sampling) refuse, before anything reaches a GPU."""
import ctypes
import os
import re

import pytest
import torch

from tests.test_sanitize_host import ROOT, _build_and_run
from tests.test_serving_refusals import BAD, FAKE, NULL, ODD, SEQ_BAD, _tensors, b, packed, seq  # noqa: F401

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses must not reach a GPU")


def fields(cls, base, kw):
    p = cls()
    for k, v in dict(base, **kw).items():
        setattr(p, k, v)
    return p


def soft(b, **kw):  # noqa: F811
    return seq(b, **dict(dict(alpha=1.0), **kw))


def call_softmax(b, p, cap=0.0, size=1 << 40, **kw):  # noqa: F811
    names = ("Q", "K", "V", "cu", "kv_len", "table", "beta", "gamma", "slopes", "O", "lse", "ws")
    a = [kw.get(n, NULL if n in ("beta", "gamma", "slopes", "lse") else FAKE) for n in names]
    return b._lib.entmax_paged_softmax_fwd(ctypes.byref(p) if p is not None else None, ctypes.c_float(cap), *a, ctypes.c_size_t(size), NULL)


def plan(b, **kw):  # noqa: F811
    return fields(b.PlanParams, dict(nseq=3, T=100, page_size=16, num_pages=50, max_pages=10), kw)


PLAN_ARRAYS = ("new_len", "release", "kv_len", "free_count", "table", "free", "kv_out", "free_out", "cu", "slots", "positions", "sequences", "ws")


def call_plan(b, p, size=1 << 40, **kw):  # noqa: F811
    a = [kw.get(n, ctypes.c_void_p((i + 1) << 24)) for i, n in enumerate(PLAN_ARRAYS)]
    return b._lib.entmax_cache_plan(ctypes.byref(p) if p is not None else None, *a, ctypes.c_size_t(size), NULL)


def samp(b, **kw):  # noqa: F811
    return fields(b.SampleParams, dict(rows=5, vocab=1000, dtype=0, stride=1000), kw)


SAMPLE_ARRAYS = ("logits", "uniform", "temperature", "top_k", "top_p", "min_p", "token", "logprob", "ws")


def call_sample(b, p, size=1 << 40, **kw):  # noqa: F811
    a = [kw.get(n, ctypes.c_void_p((i + 1) << 24)) for i, n in enumerate(SAMPLE_ARRAYS)]
    return b._lib.entmax_sample(ctypes.byref(p) if p is not None else None, *a, ctypes.c_size_t(size), NULL)


def test_every_declared_entry_point_is_there(b):  # noqa: F811
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "entmax_attn.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(entmax_[a-z_]+)\s*\(", text))
    assert {"entmax_cache_plan", "entmax_plan_workspace_bytes", "entmax_paged_softmax_fwd", "entmax_softmax_workspace_bytes", "entmax_sample",
            "entmax_sample_workspace_bytes"} <= names
    for n in names:
        assert hasattr(b._lib, n), n


def test_checks_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "step_layout_check.cc")],
                         ["-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2506_16640_amd", "csrc")])
    assert int(out.split()[1]) > 1000


# ------------------------------------------------------------------------------------------- softmax attention

@pytest.mark.parametrize("kw,code", [x for x in SEQ_BAD if "alpha" not in x[0]] +
                         [(dict(alpha=a), -1) for a in (0.0, 1.5, 2.0, float("nan"))] + [(dict(path=1), -1), (dict(page_size=0), -2), (dict(page_size=8), -2),
                          (dict(page_size=48), -2), (dict(num_pages=-1), -1), (dict(max_pages=-1), -1), (dict(max_keys=161), -1)])
def test_softmax_parameters(b, kw, code):  # noqa: F811
    assert call_softmax(b, soft(b, **kw), size=0) == code
    assert b._lib.entmax_softmax_workspace_bytes(ctypes.byref(soft(b, **kw))) == 0


def test_softmax_pointers(b):  # noqa: F811
    p = soft(b)
    need = b._lib.entmax_softmax_workspace_bytes(ctypes.byref(p))
    assert need > 0 and call_softmax(b, p, size=need - 1) == -4
    for cap in (-1.0, float("inf"), float("nan")):
        assert call_softmax(b, p, cap=cap, size=0) == -1
    for n in ("Q", "K", "V", "cu", "kv_len", "table", "O", "ws"):
        assert call_softmax(b, p, size=0, **{n: NULL}) == -1, n
        assert call_softmax(b, p, size=0, **{n: BAD if n in ("Q", "K", "V", "O", "ws") else ODD}) == -3, n
    for layout in (1, 2):
        assert call_softmax(b, soft(b, scale_layout=layout), beta=FAKE, size=0) == -1
        assert call_softmax(b, soft(b, scale_layout=layout), gamma=FAKE, size=0) == -1
    for n in ("beta", "gamma", "slopes", "lse"):
        assert call_softmax(b, p, size=0, **{n: ODD}) == -3, n
    assert call_softmax(b, soft(b, num_pages=0), size=0) == -1
    assert call_softmax(b, packed(b, alpha=1.0), size=0) == -1  # (no pages)
    assert call_softmax(b, None) == -1 and b._lib.entmax_softmax_workspace_bytes(None) == 0
    for kw in (dict(nseq=0), dict(T=0), dict(max_new=0)):
        assert call_softmax(b, soft(b, **kw), size=0, Q=NULL, K=NULL, cu=NULL, ws=NULL) == 0


@no_gpu
def test_softmax_outputs_that_meet(b):  # noqa: F811
    at = lambda x: ctypes.c_void_p((1 << 32) + x)  # noqa: E731
    far = dict(Q=at(0), K=at(1 << 24), V=at(2 << 24), O=at(3 << 24), lse=at(4 << 24))
    assert call_softmax(b, soft(b), **far) not in (-1, -2, -3, -4)  # (without a GPU the launch fails)
    for x in (0, 1024, 99 * 1024, (1 << 24) + 64, 2 << 24):
        assert call_softmax(b, soft(b), **dict(far, O=at(x))) == -1
        assert call_softmax(b, soft(b), **dict(far, lse=at(x))) == -1
    for x in (0, 99 * 1024 + 1020, -4):
        assert call_softmax(b, soft(b), **dict(far, lse=at((3 << 24) + x))) == -1


def test_binding_of_softmax(b):  # noqa: F811
    q, kc, cu, kv, table = _tensors()
    ok = (q, kc, kc, cu, kv, table)

    def refused(err, *args, **kw):
        with pytest.raises(err):
            b.paged_softmax_fwd(*args, **kw)
    refused(ValueError, *ok)  # (no GPU here: the last check)
    refused(TypeError, q.half(), *ok[1:])
    refused(ValueError, q[0], *ok[1:])
    refused(TypeError, q, kc.float(), kc.float(), cu, kv, table)
    refused(ValueError, q, kc, kc[:4], cu, kv, table)
    refused(ValueError, q[:, :3], *ok[1:])
    refused(ValueError, q, kc, kc, cu[:2], kv, table)
    refused(ValueError, q, kc, kc, cu, kv.long(), table)
    refused(ValueError, q, kc, kc, cu, kv, table[:, ::2])
    refused(ValueError, *ok, beta=torch.ones(4))
    refused(ValueError, *ok, out=q[:5])
    refused(TypeError, *ok, out=q.float())
    for lse in (torch.zeros(6, 4), torch.zeros(4, 6).double(), torch.zeros(4, 12)[:, ::2], torch.zeros(4, 5)):
        refused(ValueError, *ok, lse=lse)


# ------------------------------------------------------------------------------------------- plan

@pytest.mark.parametrize("kw,code", [(dict(nseq=-1), -1), (dict(T=-1), -1), (dict(page_size=0), -2), (dict(page_size=8), -2), (dict(page_size=48), -2),
                                     (dict(page_size=1 << 17), -2), (dict(num_pages=-1), -1), (dict(max_pages=-1), -1), (dict(nseq=(1 << 20) + 1), -2),
                                     (dict(T=(1 << 26) + 1), -2), (dict(page_size=65536, max_pages=1 << 15), -2)])
def test_plan_parameters(b, kw, code):  # noqa: F811
    assert call_plan(b, plan(b, **kw), size=0) == code
    assert b._lib.entmax_plan_workspace_bytes(ctypes.byref(plan(b, **kw))) == 0


def test_plan_pointers(b):  # noqa: F811
    p = plan(b)
    need = b._lib.entmax_plan_workspace_bytes(ctypes.byref(p))
    assert need > 0 and call_plan(b, p, size=need - 1) == -4
    for i, n in enumerate(PLAN_ARRAYS):
        if n not in ("release", "slots", "positions", "sequences"):
            assert call_plan(b, p, size=0, **{n: NULL}) == -1, n
        assert call_plan(b, p, size=0, **{n: ctypes.c_void_p(((i + 1) << 24) + 2)}) == -3, n
    assert call_plan(b, p, size=0, slots=ctypes.c_void_p((10 << 24) + 4)) == -3
    assert call_plan(b, None) == -1 and b._lib.entmax_plan_workspace_bytes(None) == 0


@no_gpu
def test_plan_arrays_that_meet(b):  # noqa: F811
    at = {n: (i + 1) << 24 for i, n in enumerate(PLAN_ARRAYS)}
    length = dict(new_len=12, release=12, kv_len=12, free_count=4, table=120, free=200, kv_out=12, free_out=4, cu=16, slots=800, positions=400, sequences=400)
    written = PLAN_ARRAYS[4:]
    launched = lambda rc: rc not in (-1, -2, -3, -4)  # noqa: E731
    assert launched(call_plan(b, plan(b)))
    # the next lengths and count in the place of the last
    assert launched(call_plan(b, plan(b), kv_out=ctypes.c_void_p(at["kv_len"]), free_out=ctypes.c_void_p(at["free_count"])))
    for n in written:
        for m in PLAN_ARRAYS[:-1]:
            if n == m:
                continue
            for x in (0, length[m] - 4):
                if (n, m) in (("kv_out", "kv_len"), ("free_out", "free_count")) and x == 0:
                    continue
                x = x // 16 * 16 if n == "ws" else x // 8 * 8 if n == "slots" else x
                assert call_plan(b, plan(b), **{n: ctypes.c_void_p(at[m] + x)}) == -1 or (n, m, x) == ("kv_out", "kv_len", 0), (n, m, x)
    assert call_plan(b, plan(b), kv_out=ctypes.c_void_p(at["kv_len"] + 4)) == -1


def test_binding_of_plan(b):  # noqa: F811
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    p = b.new_plan(3, 10, "cpu")
    args = dict(new_len=ints(3), kv_len=ints(3), page_table=ints(3, 4), free_pages=ints(20), free_count=ints(1), page_size=16, plan=p)

    def refused(**kw):
        with pytest.raises(ValueError):
            b.cache_plan(**dict(args, **kw))
    refused()  # (no GPU here: the last check)
    for name, n in (("new_len", 3), ("kv_len", 3), ("free_count", 1), ("release", 3)):
        refused(**{name: ints(n + 1)})
        refused(**{name: ints(n).long()})
        refused(**{name: ints(n, 1)})
        refused(**{name: ints(2 * n)[::2]} if n > 1 else {name: ints(0)})
    refused(page_table=ints(3, 4).long())
    refused(page_table=ints(4, 3).t())
    refused(free_pages=ints(20, 1))
    refused(free_pages=ints(20).float())
    for field, bad in (("cu_seqlens", ints(3)), ("kv_len", ints(4)), ("free_count", ints(2)), ("slots", ints(10)), ("positions", ints(9)),
                       ("sequences", ints(11)), ("workspace", ints(64))):
        refused(plan=p._replace(**{field: bad}))
    refused(plan=p._replace(slots=None, positions=None, sequences=None))


# ------------------------------------------------------------------------------------------- sampling

@pytest.mark.parametrize("kw,code", [(dict(rows=-1), -1), (dict(vocab=0), -1), (dict(vocab=-5), -1), (dict(stride=999), -1), (dict(dtype=2), -1),
                                     (dict(dtype=-1), -1), (dict(rows=(1 << 20) + 1), -2), (dict(vocab=(1 << 22) + 1, stride=1 << 23), -2),
                                     (dict(stride=1 << 50), -2), (dict(rows=1 << 20, vocab=1 << 20, stride=1 << 20), -2)])
def test_sample_parameters(b, kw, code):  # noqa: F811
    assert call_sample(b, samp(b, **kw), size=0) == code
    assert b._lib.entmax_sample_workspace_bytes(ctypes.byref(samp(b, **kw))) == 0


def test_sample_pointers(b):  # noqa: F811
    for dtype in (0, 1):
        p = samp(b, dtype=dtype)
        need = b._lib.entmax_sample_workspace_bytes(ctypes.byref(p))
        assert need > 0 and call_sample(b, p, size=need - 1) == -4
        for i, n in enumerate(SAMPLE_ARRAYS):
            if n in ("logits", "uniform", "token", "ws"):
                assert call_sample(b, p, size=0, **{n: NULL}) == -1, n
            assert call_sample(b, p, size=0, **{n: ctypes.c_void_p(((i + 1) << 24) + 1)}) == -3, n
    assert call_sample(b, samp(b, dtype=1), size=0, logits=ctypes.c_void_p((1 << 24) + 2)) == -3
    assert call_sample(b, samp(b, rows=0), size=0, logits=NULL, ws=NULL) == 0
    assert call_sample(b, None) == -1 and b._lib.entmax_sample_workspace_bytes(None) == 0


@no_gpu
def test_sample_arrays_that_meet(b):  # noqa: F811
    at = {n: (i + 1) << 24 for i, n in enumerate(SAMPLE_ARRAYS)}
    assert call_sample(b, samp(b)) not in (-1, -2, -3, -4)
    # (the rows of a wider tensor: its other columns are nobody's)
    assert call_sample(b, samp(b, stride=2000), token=ctypes.c_void_p(at["logits"] + 2000)) not in (-1, -2, -3, -4)
    assert call_sample(b, samp(b, stride=2000), token=ctypes.c_void_p(at["logits"] + 4 * 4000)) == -1
    for n in ("token", "logprob", "ws"):
        for m in SAMPLE_ARRAYS[:-1]:
            if n != m:
                assert call_sample(b, samp(b), **{n: ctypes.c_void_p(at[m])}) == -1, (n, m)


def test_binding_of_sample(b):  # noqa: F811
    x, u = torch.zeros(4, 50), torch.zeros(4)

    def refused(err, *args, **kw):
        with pytest.raises(err):
            b.sample(*args, **kw)
    refused(ValueError, x, u)  # (no GPU here: the last check)
    refused(TypeError, x.half(), u)
    refused(TypeError, x.double(), u)
    refused(ValueError, x[0], u)
    refused(ValueError, x.t().contiguous().t(), u)
    refused(ValueError, x, u[:3])
    refused(ValueError, x, u.double())
    refused(ValueError, x, u[:, None])
    for name in ("temperature", "top_p", "min_p", "logprob"):
        refused(ValueError, x, u, **{name: torch.zeros(5)})
        refused(ValueError, x, u, **{name: torch.zeros(4).bfloat16()})
    for name in ("top_k", "token"):
        refused(ValueError, x, u, **{name: torch.zeros(4)})
        refused(ValueError, x, u, **{name: torch.zeros(4, dtype=torch.int64)})
        refused(ValueError, x, u, **{name: torch.zeros(8, dtype=torch.int32)[::2]})
