"""Sizes and layouts that the serving entry points refuse or take at their limits, before anything reaches a GPU."""
import ctypes
import os

import pytest
import torch

from tests.test_sanitize_host import ROOT, _build_and_run
from tests.test_serving_refusals import NULL, app, b, call_append, call_packed, call_paged, packed, seq  # noqa: F401


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


def test_overlap_check_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "overlap_check.cc")],
                         ["-std=c++17", "-I", os.path.join(ROOT, "paper_2506_16640_amd", "csrc")])
    assert int(out.split()[1]) > 1000


no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses must not reach a GPU")
AT = 1 << 32  # (addresses that nothing looks at before a GPU is asked for)


def _at(x):
    return ctypes.c_void_p(AT + x)


def _refused(rc):
    assert rc == -1


def _passed(rc):  # the checks; without a GPU the launch fails
    assert rc not in (-1, -2, -3, -4)


@no_gpu
def test_outputs_that_meet_what_is_read(b):  # noqa: F811
    far = dict(Q=_at(0), K=_at(1 << 24), V=_at(2 << 24), O=_at(3 << 24))
    T, token = 100, 512 * 2
    # the queries, a token or a head further, their last row
    for x in (0, token, 64 * 2, (T - 1) * token):
        _refused(call_paged(b, seq(b), **dict(far, O=_at(x))))
        _refused(call_packed(b, packed(b), **dict(far, O=_at(x))))
    for name, base in (("K", 1), ("V", 2)):
        _refused(call_paged(b, seq(b), **dict(far, O=_at((base << 24) + 64))))
        _refused(call_packed(b, packed(b), **dict(far, O=_at(base << 24))))
    # rows of O on top of each other
    _refused(call_paged(b, seq(b, o_stride_t=64, o_stride_h=64), **far))
    _refused(call_paged(b, seq(b, o_stride_t=512, o_stride_h=512), **far))


@no_gpu
def test_outputs_beside_what_is_read(b):  # noqa: F811
    far = dict(Q=_at(0), K=_at(1 << 24), V=_at(2 << 24), O=_at(3 << 24))
    _passed(call_paged(b, seq(b), **far))
    _passed(call_packed(b, packed(b), **far))
    _passed(call_paged(b, seq(b), **dict(far, O=_at(100 * 1024))))
    # queries and output side by side in rows of one tensor, head by head in one tensor, halves of every row of one
    for st, sh, off in ((1024, 64, 512), (64, 64 * 200, 64 * 100), (1024, 128, 64)):
        p = seq(b, q_stride_t=st, o_stride_t=st, q_stride_h=sh, o_stride_h=sh)
        _passed(call_paged(b, p, **dict(far, O=_at(2 * off))))
        _refused(call_paged(b, p, **dict(far, O=_at(2 * (off - 8)))))
    # queries, keys, values and output of a packed call in one tensor [T, 8 + 2 + 2 + 8, 64]
    p = packed(b, q_stride_t=1280, o_stride_t=1280, k_stride_n=1280, v_stride_n=1280)
    _passed(call_packed(b, p, Q=_at(0), K=_at(8 * 128), V=_at(10 * 128), O=_at(12 * 128)))
    _refused(call_packed(b, p, Q=_at(0), K=_at(8 * 128), V=_at(10 * 128), O=_at(11 * 128)))


def _append_at(**kw):
    base = dict(Q=_at(0), K=_at(1 << 24), V=_at(2 << 24), Qo=_at(3 << 24), Kc=_at(4 << 24), Vc=_at(5 << 24))
    return dict(base, **{k: _at(x) for k, x in kw.items()})


@no_gpu
def test_appends_on_top_of_something(b):  # noqa: F811
    cases = [({}, dict(Qo=128)), ({}, dict(Qo=1 << 24)), ({}, dict(Qo=2 << 24)), ({}, dict(Qo=4 << 24)), ({}, dict(Kc=5 << 24)), ({}, dict(Kc=0)),
             ({}, dict(Vc=1 << 24)), ({}, dict(Kc=1 << 24)), ({}, dict(Vc=(4 << 24) + 4096)),
             (dict(qo_stride_t=576), dict(Qo=0)),  # the queries' place, but other strides
             (dict(kc_stride_p=0), {}), (dict(kc_stride_h=0), {}), (dict(vc_stride_h=512), {}), (dict(qo_stride_t=64), {})]
    for kw, at in cases:
        _refused(call_append(b, app(b, **kw), **_append_at(**at)))


@no_gpu
def test_appends_beside_something(b):  # noqa: F811
    _passed(call_append(b, app(b), **_append_at()))
    _passed(call_append(b, app(b), **_append_at(Qo=0)))
    # a fused projection rotated in place: [T, 8 + 2 + 2, 64]
    p = app(b, q_stride_t=768, qo_stride_t=768, k_stride_t=768, v_stride_t=768)
    _passed(call_append(b, p, **_append_at(Q=0, Qo=0, K=8 * 128, V=10 * 128)))
    _refused(call_append(b, p, **_append_at(Q=0, Qo=128, K=8 * 128, V=10 * 128)))
    # keys and values of a page together: [pages, 2, 2, 16, 64]; token by token: [pages, 16, 2, 2, 64]
    _passed(call_append(b, app(b, kc_stride_p=4096, vc_stride_p=4096), **_append_at(Vc=(4 << 24) + 4096)))
    p = app(b, kc_stride_p=4096, vc_stride_p=4096, kc_stride_n=256, vc_stride_n=256, kc_stride_h=64, vc_stride_h=64)
    _passed(call_append(b, p, **_append_at(Vc=(4 << 24) + 256)))
    _passed(call_append(b, app(b, num_pages=1, kc_stride_p=0, vc_stride_p=0), **_append_at()))
    _passed(call_append(b, app(b, Hq=0), **dict(_append_at(), Q=NULL, Qo=NULL)))


@no_gpu
def test_a_cache_without_keys(b):  # noqa: F811
    far = dict(Q=_at(0), O=_at(3 << 24))
    p = seq(b, max_pages=0, max_keys=0)
    _passed(call_paged(b, p, table=NULL, **far))
    _passed(call_paged(b, seq(b, num_pages=0, max_pages=0, max_keys=0), table=NULL, K=NULL, V=NULL, **far))
    _refused(call_paged(b, seq(b, max_keys=16), table=NULL, **far))


def test_a_page_table_wider_than_any_call(b):  # noqa: F811
    q, cache = torch.zeros(1, 1, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 65536, 64, dtype=torch.bfloat16)
    table = torch.zeros(1, 40000, dtype=torch.int32)  # 2.6e9 places
    cu, kv = torch.tensor([0, 1], dtype=torch.int32), torch.tensor([5], dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):  # (no GPU here: the last check)
        b.paged_attn_fwd(q, cache, cache, cu, kv, table)
    assert b._lib.entmax_seq_workspace_bytes(b._paged_params(q, cache, cache, table, None, None, *b._DEFAULTS)[1]) == 0


def test_overlap_of_ranges_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "overlap_ranges_check.cc")],
                         ["-std=c++17", "-I", os.path.join(ROOT, "paper_2506_16640_amd", "csrc")])
    assert int(out.split()[3]) > 1000


@no_gpu
def test_outputs_in_the_gaps_of_a_pool(b):  # noqa: F811
    # pages of 4096 elements of keys (and values behind them) in blocks of 1 MB, the output between two of them
    far = dict(Q=_at(1 << 28), K=_at(0), V=_at(8192))
    p = seq(b, k_stride_p=1 << 19, v_stride_p=1 << 19)
    _passed(call_paged(b, p, **dict(far, O=_at((3 << 20) + (1 << 16)))))
    _refused(call_paged(b, p, **dict(far, O=_at((4 << 20) - (1 << 16)))))
    p = app(b, kc_stride_p=1 << 19, vc_stride_p=1 << 19)
    at = dict(_append_at(), Kc=_at(0), Vc=_at(8192), Q=_at(1 << 28))
    _passed(call_append(b, p, **dict(at, Qo=_at((3 << 20) + (1 << 16)), K=_at((5 << 20) + (1 << 16)), V=_at((7 << 20) + (1 << 16)))))
    _refused(call_append(b, p, **dict(at, Qo=_at((4 << 20) - (1 << 16)), K=_at((5 << 20) + (1 << 16)), V=_at((7 << 20) + (1 << 16)))))
