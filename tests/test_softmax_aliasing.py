"""Outputs and workspace of the softmax attention on top of anything that the call reads."""
import ctypes

import pytest

from tests.test_serving_refusals import b  # noqa: F401
from tests.test_step_refusals import call_softmax, no_gpu, soft

NAMES = ("Q", "K", "V", "cu", "kv_len", "table", "beta", "gamma", "slopes", "O", "lse", "ws")
AT = {n: (1 << 32) + (k << 24) for k, n in enumerate(NAMES)}


def _call(b, p, **moved):  # noqa: F811
    return call_softmax(b, p, **{n: ctypes.c_void_p(moved.get(n, AT[n])) for n in NAMES})


def _bytes(layout):
    """T 100, 8 query heads and 2 of keys, 64 features of bf16, 50 pages of 16, 3 sequences of at most 10 pages."""
    return dict(Q=100 * 1024, K=50 * 4096, V=50 * 4096, cu=16, kv_len=12, table=120, beta=32 if layout == 1 else 3200, gamma=32 if layout == 1 else 3200,
                slopes=32, O=100 * 1024, lse=3200)


def launched(rc):
    return rc not in (-1, -2, -3, -4)  # (without a GPU the launch fails)


@no_gpu
@pytest.mark.parametrize("layout", [1, 2])
def test_outputs_on_top_of_what_is_read(b, layout):  # noqa: F811
    p = soft(b, scale_layout=layout)
    size = _bytes(layout)
    assert launched(_call(b, p))
    for out, step in (("O", 16), ("lse", 4)):
        for n in NAMES[:9]:
            for at in (AT[n], AT[n] + (size[n] - 4) // step * step, AT[n] - size[out] + 16):
                assert _call(b, p, **{out: at}) == -1, (out, n, at - AT[n])
            for at in (AT[n] + (size[n] + 15) // 16 * 16, AT[n] - size[out]):
                assert launched(_call(b, p, **{out: at})), (out, n, at - AT[n])


@no_gpu
def test_workspace_on_top_of_tensors(b):  # noqa: F811
    p = soft(b, scale_layout=1)
    need = b._lib.entmax_softmax_workspace_bytes(ctypes.byref(p))
    size = _bytes(1)
    for n in ("Q", "K", "V", "beta", "gamma", "slopes", "O", "lse"):
        for at in (AT[n], AT[n] + (size[n] - 1) // 256 * 256, AT[n] - need + 256):
            assert _call(b, p, ws=at) == -1, (n, at - AT[n])
        for at in (AT[n] + (size[n] + 255) // 256 * 256, AT[n] - need):
            assert launched(_call(b, p, ws=at)), (n, at - AT[n])


@no_gpu
def test_what_is_not_read_may_lie_anywhere(b):  # noqa: F811
    """beta and gamma of a call without scales; a table without columns."""
    p = soft(b, scale_layout=0)
    assert launched(_call(b, p, O=AT["beta"])) and launched(_call(b, p, lse=AT["gamma"]))
    assert launched(_call(b, soft(b, max_pages=0, max_keys=0), lse=AT["table"]))
