"""Thin ctypes binding of the C ABI in include/entmax_attn.h.

Argument marshalling only: torch supplies device memory and the stream, every
step of the computation runs in the HIP kernels of lib/libentmax_attn.so.
There is no fallback: if the library is missing, importing this module fails.
"""
import collections
import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libentmax_attn.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "libentmax_attn.so is not built: run `python -m paper_2506_16640_amd.build` "
        "(or __graft_entry__.build()) first; there is no CPU fallback")

_lib = ctypes.CDLL(LIB_PATH)

NUM_STATS = 24
STAT_NAMES = {
    "fwd_tiles_visible": 0, "fwd_qk_max": 1, "fwd_qk_solve": 2, "fwd_qk_pv": 3, "fwd_pv_tiles": 4,
    "fwd_solve_sweeps": 5, "fwd_blocks": 6, "fwd_eval_tiles": 7,
    "bwd_tiles_visible": 8, "bwd_qk_mask": 9, "bwd_active_tiles": 10, "bwd_dq_tiles": 11, "bwd_dkv_tiles": 12,
    "fwd_cand_tiles": 13, "fwd_candidates": 14, "fwd_support": 15, "fwd_sparse_blocks": 16, "fwd_list_qk": 17, "bwd_list_qk": 18, "bwd_support": 19,
    "fwd_window_skipped": 20,
}
FWD_NUM_PHASES = 5
BWD_NUM_PHASES = 8
FWD_PHASES = ("prepare", "lists", "finish", "transpose", "tiled")
BWD_PHASES = ("lists", "rows", "transpose", "mask", "dq", "dkv", "keys", "scale_grad")


class Params(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Nq", ctypes.c_int32), ("Nk", ctypes.c_int32),
        ("D", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("scale_layout", ctypes.c_int32), ("logn_mode", ctypes.c_int32), ("bias_mode", ctypes.c_int32),
        ("path", ctypes.c_int32),
        ("alpha", ctypes.c_float), ("delta", ctypes.c_float),
        ("q_stride_b", ctypes.c_int64), ("q_stride_h", ctypes.c_int64), ("q_stride_n", ctypes.c_int64),
        ("kv_stride_b", ctypes.c_int64), ("kv_stride_h", ctypes.c_int64), ("kv_stride_n", ctypes.c_int64),
    ]


_vp = ctypes.c_void_p
_lib.entmax_attn_fwd.restype = ctypes.c_int
_lib.entmax_attn_fwd.argtypes = [ctypes.POINTER(Params)] + [_vp] * 9 + [ctypes.c_size_t, _vp, _vp, ctypes.c_size_t, _vp,
                                                                     _vp]
_lib.entmax_attn_bwd.restype = ctypes.c_int
_lib.entmax_attn_bwd.argtypes = ([ctypes.POINTER(Params)] + [_vp] * 7 + [ctypes.c_size_t] + [_vp] * 10 +
                                 [ctypes.c_size_t, _vp, _vp])
_lib.entmax_attn_workspace_bytes.restype = ctypes.c_size_t
_lib.entmax_attn_workspace_bytes.argtypes = [ctypes.POINTER(Params), ctypes.c_int]
_lib.entmax_attn_saved_bytes.restype = ctypes.c_size_t
_lib.entmax_attn_saved_bytes.argtypes = [ctypes.POINTER(Params)]
_lib.entmax_attn_check_params.restype = ctypes.c_int
_lib.entmax_attn_check_params.argtypes = [ctypes.POINTER(Params)]
_lib.entmax_attn_fwd_noalloc.restype = ctypes.c_int
_lib.entmax_attn_fwd_noalloc.argtypes = [ctypes.POINTER(Params)] + [_vp] * 10
_lib.entmax_attn_noalloc_init.restype = ctypes.c_int
_lib.entmax_attn_noalloc_init.argtypes = []
_lib.entmax_attn_noalloc_scratch_bytes.restype = ctypes.c_size_t
_lib.entmax_attn_noalloc_scratch_bytes.argtypes = []
_lib.entmax_attn_mfma_probe.restype = ctypes.c_int
_lib.entmax_attn_mfma_probe.argtypes = [ctypes.c_int, ctypes.c_int, _vp, _vp]


class ProjParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("E", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("gamma_scale", ctypes.c_float)]


_lib.entmax_scale_proj_fwd.restype = ctypes.c_int
_lib.entmax_scale_proj_fwd.argtypes = [ctypes.POINTER(ProjParams)] + [_vp] * 6
_lib.entmax_scale_proj_bwd.restype = ctypes.c_int
_lib.entmax_scale_proj_bwd.argtypes = [ctypes.POINTER(ProjParams)] + [_vp] * 11 + [ctypes.c_size_t, _vp]
_lib.entmax_scale_proj_workspace_bytes.restype = ctypes.c_size_t
_lib.entmax_scale_proj_workspace_bytes.argtypes = [ctypes.POINTER(ProjParams)]
_lib.entmax_attn_strerror.restype = ctypes.c_char_p
_lib.entmax_attn_strerror.argtypes = [ctypes.c_int]


class EntmaxAttnError(RuntimeError):
    def __init__(self, code):
        self.code = code
        super().__init__("entmax_attn: %s (%d)" % (_lib.entmax_attn_strerror(code).decode(), code))


def strerror(code):
    return _lib.entmax_attn_strerror(int(code)).decode()


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def make_params(q, k, alpha, delta, causal, beta, logn_mode, path=0, bias_mode=0):
    if q.dim() != 4 or k.dim() != 4 or q.shape[:2] != k.shape[:2] or q.shape[3] != k.shape[3]:
        raise ValueError("Q must be [B,H,Nq,D] and K [B,H,Nk,D]")
    B, H, Nq, D = q.shape
    Nk = k.shape[2]
    if q.dtype == torch.bfloat16:
        dt = 0
    elif q.dtype == torch.float32:
        dt = 1
    else:
        raise TypeError("Q must be bfloat16 or float32")
    layout = 0 if beta is None else (1 if beta.dim() == 1 else 2)
    p = Params(B, H, Nq, Nk, D, dt, int(bool(causal)), layout, int(logn_mode), int(bias_mode), int(path), float(alpha), float(delta),
               0, 0, 0, 0, 0, 0)
    if not q.is_contiguous():
        if q.stride(3) != 1:
            raise ValueError("the last dimension of Q must be contiguous")
        p.q_stride_b, p.q_stride_h, p.q_stride_n = q.stride(0), q.stride(1), q.stride(2)
    if not k.is_contiguous():
        if k.stride(3) != 1:
            raise ValueError("the last dimension of K must be contiguous")
        p.kv_stride_b, p.kv_stride_h, p.kv_stride_n = k.stride(0), k.stride(1), k.stride(2)
    return p


def _check_like(name, t, ref):
    """t must have ref's shape, strides, dtype and device (the ABI passes one set of strides per tensor family)."""
    if t.shape != ref.shape or t.stride() != ref.stride():
        raise ValueError("%s must have the shape and strides of its reference tensor" % name)
    if t.dtype != ref.dtype or t.device != ref.device:
        raise TypeError("%s must have the dtype and device of Q" % name)


def _check_scale(p, q, beta, gamma):
    if (beta is None) != (gamma is None):
        raise ValueError("beta and gamma come together")
    if beta is None:
        return
    want = (p.H,) if p.scale_layout == 1 else (p.B, p.H, p.Nq)
    for name, t in (("beta", beta), ("gamma", gamma)):
        if t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != want or t.device != q.device:
            raise ValueError("%s must be a contiguous float32 tensor of shape %s on Q's device" % (name, want))


def _check_slopes(p, q, slopes):
    if slopes is None:
        return
    if slopes.dtype != torch.float32 or not slopes.is_contiguous() or tuple(slopes.shape) != (p.H,) or slopes.device != q.device:
        raise ValueError("alibi_slopes must be a contiguous float32 tensor of shape (%d,) on Q's device" % p.H)


def _check_aux(p, stats, saved, workspace, is_bwd):
    if stats is not None and (stats.numel() < NUM_STATS or stats.element_size() != 8 or not stats.is_contiguous()):
        raise ValueError("stats must be a contiguous 64-bit integer tensor with at least %d entries" % NUM_STATS)
    if saved is not None and (saved.dtype != torch.uint8 or not saved.is_contiguous()):
        raise ValueError("saved must be a contiguous uint8 tensor")
    if workspace is not None and (workspace.dtype != torch.uint8 or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor")


def workspace_bytes(params, is_bwd):
    return int(_lib.entmax_attn_workspace_bytes(ctypes.byref(params), int(is_bwd)))


def saved_bytes(params):
    return int(_lib.entmax_attn_saved_bytes(ctypes.byref(params)))


def new_saved(params, device="cuda"):
    """Buffer that carries the forward's lists to the backward (pass it to both as `saved`), of the size the library
    asks for; a larger uint8 tensor holds longer lists."""
    return torch.empty(max(saved_bytes(params), 256), dtype=torch.uint8, device=device)


def check_params(params):
    return int(_lib.entmax_attn_check_params(ctypes.byref(params)))


def _events_arg(events, n):
    if events is None:
        return None
    if len(events) != n + 1:
        raise ValueError("phase_events needs %d handles" % (n + 1))
    arr = (ctypes.c_void_p * (n + 1))(*[ctypes.c_void_p(e) for e in events])
    return arr


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def entmax_attn_fwd(q, k, v, alpha=1.5, beta=None, gamma=None, delta=1.0, causal=True, logn_mode=0, path=0,
                    out=None, tau=None, stats=None, workspace=None, phase_events=None, saved=None, alibi_slopes=None,
                    bias_mode=0):
    """O, tau = entmax attention forward.  q [B,H,Nq,D], k,v [B,H,Nk,D] on the GPU, bf16 or fp32;
    beta,gamma fp32 [H] or [B,H,Nq] or None.  stats: optional uint64/int64 device tensor [NUM_STATS] (added to).
    path: 0 automatic, 1 tiled kernel only.  phase_events: optional list of FWD_NUM_PHASES + 1 hipEvent_t handles.
    saved: optional uint8 device tensor of at least saved_bytes(params) bytes, filled for the backward.
    alibi_slopes: optional fp32 [H] slopes of the linear distance bias (0 = head without bias); bias_mode 0 puts the
    bias inside the ASEntmax scale, 1 outside."""
    p = make_params(q, k, alpha, delta, causal, beta, logn_mode, path, bias_mode)
    _check_slopes(p, q, alibi_slopes)
    if k.dtype != q.dtype or k.device != q.device:
        raise TypeError("K must have the dtype and device of Q")
    _check_like("V", v, k)
    _check_scale(p, q, beta, gamma)
    _check_aux(p, stats, saved, workspace, False)
    if out is None:
        out = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device)
    else:
        _check_like("out", out, q)
    if tau is None:
        tau = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    elif tau.dtype != torch.float32 or not tau.is_contiguous() or tau.shape != q.shape[:3]:
        raise ValueError("tau must be a contiguous float32 tensor [B,H,Nq]")
    need = workspace_bytes(p, 0)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    ev = _events_arg(phase_events, FWD_NUM_PHASES)
    rc = _lib.entmax_attn_fwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(gamma),
                              _ptr(alibi_slopes), _ptr(out), _ptr(tau), _ptr(saved),
                              0 if saved is None else saved.numel(), _ptr(stats),
                              _ptr(workspace), workspace.numel(), _stream(), ev)
    if rc != 0:
        raise EntmaxAttnError(rc)
    return out, tau


def mfma_probe(iters, blocks, sink):
    """Enqueue the matrix-pipeline probe; returns the flops it issues (the caller times it)."""
    rc = _lib.entmax_attn_mfma_probe(int(iters), int(blocks), _ptr(sink), _stream())
    if rc != 0:
        raise EntmaxAttnError(rc)
    return float(blocks) * 4 * iters * 4 * 2 * 32 * 32 * 16


def noalloc_scratch_bytes():
    return int(_lib.entmax_attn_noalloc_scratch_bytes())


def noalloc_init():
    rc = _lib.entmax_attn_noalloc_init()
    if rc != 0:
        raise EntmaxAttnError(rc)


def entmax_attn_fwd_noalloc(q, k, v, out, tau, alpha=1.5, beta=None, gamma=None, delta=1.0, causal=True, logn_mode=0,
                            path=0, stats=None, alibi_slopes=None, bias_mode=0):
    """Forward through the entry point that allocates nothing: the caller brings `out` and `tau`, the scratch is
    the library's built-in buffer (noalloc_scratch_bytes()).  Raises EntmaxAttnError(-6) for problems beyond it."""
    p = make_params(q, k, alpha, delta, causal, beta, logn_mode, path, bias_mode)
    _check_slopes(p, q, alibi_slopes)
    if k.dtype != q.dtype or k.device != q.device:
        raise TypeError("K must have the dtype and device of Q")
    _check_like("V", v, k)
    _check_like("out", out, q)
    _check_scale(p, q, beta, gamma)
    _check_aux(p, stats, None, None, False)
    if tau.dtype != torch.float32 or not tau.is_contiguous() or tau.shape != q.shape[:3]:
        raise ValueError("tau must be a contiguous float32 tensor [B,H,Nq]")
    rc = _lib.entmax_attn_fwd_noalloc(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(gamma),
                                      _ptr(alibi_slopes), _ptr(out), _ptr(tau), _ptr(stats), _stream())
    if rc != 0:
        raise EntmaxAttnError(rc)
    return out, tau


def entmax_attn_bwd(q, k, v, o, do, tau, alpha=1.5, beta=None, gamma=None, delta=1.0, causal=True, logn_mode=0, path=0,
                    stats=None, workspace=None, phase_events=None, saved=None, alibi_slopes=None, bias_mode=0):
    """dQ, dK, dV, dbeta, dgamma = entmax attention backward (dbeta/dgamma None without scale parameters).
    saved: the buffer the forward filled for the same inputs, or None.  alibi_slopes, bias_mode: as in the forward."""
    p = make_params(q, k, alpha, delta, causal, beta, logn_mode, path, bias_mode)
    _check_slopes(p, q, alibi_slopes)
    if k.dtype != q.dtype or k.device != q.device:
        raise TypeError("K must have the dtype and device of Q")
    _check_like("V", v, k)
    _check_like("dO", do, q)
    _check_scale(p, q, beta, gamma)
    _check_aux(p, stats, saved, workspace, True)
    if tau.dtype != torch.float32 or not tau.is_contiguous() or tau.shape != q.shape[:3]:
        raise ValueError("tau must be a contiguous float32 tensor [B,H,Nq]")
    dq = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device)
    dk = torch.empty_strided(k.shape, k.stride(), dtype=k.dtype, device=k.device)
    dv = torch.empty_strided(v.shape, v.stride(), dtype=v.dtype, device=v.device)
    dbeta = torch.empty_like(beta) if beta is not None else None
    dgamma = torch.empty_like(gamma) if gamma is not None else None
    need = workspace_bytes(p, 1)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    ev = _events_arg(phase_events, BWD_NUM_PHASES)
    rc = _lib.entmax_attn_bwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(do), _ptr(tau), _ptr(saved),
                              0 if saved is None else saved.numel(), _ptr(beta), _ptr(gamma),
                              _ptr(alibi_slopes), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dbeta), _ptr(dgamma), _ptr(stats),
                              _ptr(workspace), workspace.numel(), _stream(), ev)
    if rc != 0:
        raise EntmaxAttnError(rc)
    return dq, dk, dv, dbeta, dgamma


def new_stats(device="cuda"):
    return torch.zeros(NUM_STATS, dtype=torch.int64, device=device)


def stats_dict(stats):
    vals = stats.cpu().tolist()
    return {name: int(vals[i]) for name, i in STAT_NAMES.items()}


def _proj_params(x, wb, wg, gamma_scale):
    if x.dim() != 3 or not x.is_contiguous():
        raise ValueError("X must be a contiguous [B,N,E] tensor")
    if x.dtype == torch.bfloat16:
        dt = 0
    elif x.dtype == torch.float32:
        dt = 1
    else:
        raise TypeError("X must be bfloat16 or float32")
    B, N, E = x.shape
    for name, w in (("Wb", wb), ("Wg", wg)):
        if w.dtype != torch.float32 or not w.is_contiguous() or w.dim() != 2 or w.shape[1] != E or w.device != x.device:
            raise ValueError("%s must be a contiguous float32 [H,E] tensor on X's device" % name)
    if wb.shape != wg.shape:
        raise ValueError("Wb and Wg must have the same shape")
    return ProjParams(B, wb.shape[0], N, E, dt, float(gamma_scale))


def scale_proj_fwd(x, wb, wg, gamma_scale=1.0):
    """beta, gamma [B,H,N] fp32 = softplus(X Wb^T), gamma_scale * tanh(X Wg^T), in the attention's per-query layout."""
    p = _proj_params(x, wb, wg, gamma_scale)
    beta = torch.empty(p.B, p.H, p.N, dtype=torch.float32, device=x.device)
    gamma = torch.empty_like(beta)
    rc = _lib.entmax_scale_proj_fwd(ctypes.byref(p), _ptr(x), _ptr(wb), _ptr(wg), _ptr(beta), _ptr(gamma), _stream())
    if rc != 0:
        raise EntmaxAttnError(rc)
    return beta, gamma


def scale_proj_bwd(x, wb, wg, beta, gamma, dbeta, dgamma, gamma_scale=1.0, workspace=None):
    """dX [B,N,E] (X's dtype), dWb, dWg [H,E] fp32 from the attention backward's d beta, d gamma."""
    p = _proj_params(x, wb, wg, gamma_scale)
    for name, t in (("beta", beta), ("gamma", gamma), ("dbeta", dbeta), ("dgamma", dgamma)):
        if t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != (p.B, p.H, p.N) or t.device != x.device:
            raise ValueError("%s must be a contiguous float32 [B,H,N] tensor on X's device" % name)
    need = int(_lib.entmax_scale_proj_workspace_bytes(ctypes.byref(p)))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor")
    dx = torch.empty_like(x)
    dwb, dwg = torch.empty_like(wb), torch.empty_like(wg)
    rc = _lib.entmax_scale_proj_bwd(ctypes.byref(p), _ptr(x), _ptr(wb), _ptr(wg), _ptr(beta), _ptr(gamma), _ptr(dbeta),
                                    _ptr(dgamma), _ptr(dx), _ptr(dwb), _ptr(dwg), _ptr(workspace), workspace.numel(),
                                    _stream())
    if rc != 0:
        raise EntmaxAttnError(rc)
    return dx, dwb, dwg


# ------------------------------------------------- serving: packed sequences, paged cache
# (A decode step is a few microseconds of GPU work: these functions look at every tensor once, and hand parameters over as packed bytes.)

class SeqParams(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("nseq", "T", "Hq", "Hkv", "D", "dtype", "causal", "scale_layout", "logn_mode",
                                               "bias_mode", "path", "page_size", "num_pages", "max_pages", "max_new", "max_keys")] +
                [("alpha", ctypes.c_float), ("delta", ctypes.c_float)] +
                [(n, ctypes.c_int64) for n in ("q_stride_t", "q_stride_h", "o_stride_t", "o_stride_h", "k_stride_p", "k_stride_h",
                                               "k_stride_n", "v_stride_p", "v_stride_h", "v_stride_n")])


class AppendParams(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("nseq", "T", "Hq", "Hkv", "D", "dtype", "page_size", "num_pages", "max_pages", "rot",
                                               "interleaved")] +
                [(n, ctypes.c_int64) for n in ("q_stride_t", "q_stride_h", "qo_stride_t", "qo_stride_h", "k_stride_t", "k_stride_h",
                                               "v_stride_t", "v_stride_h", "kc_stride_p", "kc_stride_h", "kc_stride_n", "vc_stride_p",
                                               "vc_stride_h", "vc_stride_n")])


_seq_bytes = struct.Struct("@16i2f10q")
_append_bytes = struct.Struct("@11i4x14q")
assert _seq_bytes.size == ctypes.sizeof(SeqParams) and _append_bytes.size == ctypes.sizeof(AppendParams)

_lib.entmax_paged_attn_fwd.restype = ctypes.c_int
_lib.entmax_paged_attn_fwd.argtypes = [_vp] * 12 + [ctypes.c_size_t, _vp]
_lib.entmax_packed_attn_fwd.restype = ctypes.c_int
_lib.entmax_packed_attn_fwd.argtypes = [_vp] * 10 + [ctypes.c_size_t, _vp]
_lib.entmax_seq_workspace_bytes.restype = ctypes.c_size_t
_lib.entmax_seq_workspace_bytes.argtypes = [_vp]
_lib.entmax_cache_append.restype = ctypes.c_int
_lib.entmax_cache_append.argtypes = [_vp] * 12

_DTYPES = {torch.bfloat16: 0, torch.float32: 1}
_INT32_MOST = 2 ** 31 - 1  # (more keys than any call takes: refused like other large bounds)


def _rows_of(name, t):
    """Shape and (token, head) strides of a [T,H,D] tensor.  Strides of dimensions of size one or of empty tensors do not matter: valid ones."""
    shape = t.shape
    if len(shape) != 3:
        raise ValueError("%s must be [T,H,D]" % name)
    T, H, D = shape
    if t.dtype not in _DTYPES:
        raise TypeError("%s must be bfloat16 or float32" % name)
    if T == 0 or H == 0 or D == 0:
        return T, H, D, H * D, D
    st, sh, sd = t.stride()
    if sd != 1:
        raise ValueError("the last dimension of %s must be contiguous" % name)
    if H == 1:
        sh = D
    if T == 1:
        st = (H - 1) * sh + D
    return T, H, D, st, sh


def _like(name, t, ref, T, H, D, t_T, t_H, t_D):
    if t.dtype != ref.dtype or t.get_device() != ref.get_device():
        raise TypeError("%s must have the dtype and device of the others" % name)
    if t_T != T or t_H != H or t_D != D:
        raise ValueError("%s must be [%d,%d,%d]" % (name, T, H, D))


def _cache_of(name, t, ref, D):
    """Shape and (page, head, token) strides of a cache [num_pages,Hkv,page_size,D]."""
    shape = t.shape
    if len(shape) != 4 or shape[3] != D:
        raise ValueError("%s must be [num_pages,Hkv,page_size,D]" % name)
    if t.dtype != ref.dtype or t.get_device() != ref.get_device():
        raise TypeError("%s must have the dtype and device of the others" % name)
    P, H, n, _ = shape
    if P == 0 or H == 0 or n == 0 or D == 0:
        return shape, (H * n * D, n * D, D)
    sp, sh, sn, sd = t.stride()
    if sd != 1:
        raise ValueError("the last dimension of %s must be contiguous" % name)
    if n == 1:
        sn = D
    if H == 1:
        sh = n * sn
    return shape, (H * n * D if P == 1 else sp, sh, sn)


def _int_array(name, t, ref, want):
    """want: elements, None if any number will do."""
    if t.dtype != torch.int32 or not t.is_contiguous() or t.get_device() != ref.get_device() or t.dim() != 1 or (want is not None and t.shape[0] != want):
        raise ValueError("%s must be a contiguous int32 tensor%s on the device of the others" % (name, "" if want is None else " of %d elements" % want))


def _page_table(t, ref):
    if t.dtype != torch.int32 or not t.is_contiguous() or t.dim() != 2 or t.get_device() != ref.get_device():
        raise ValueError("page_table must be a contiguous int32 tensor [nseq,max_pages] on the device of the others")
    return t.shape


def _floats(name, t, ref, want):
    if t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != want or t.get_device() != ref.get_device():
        raise ValueError("%s must be a contiguous float32 tensor of shape %s on the device of the others" % (name, want))


def _at(t):
    return None if t is None else t.data_ptr()


def _arrays(ref, dtype, *named):
    """named: (name, tensor or None, elements) of contiguous tensors of one dimension on ref's device."""
    device = ref.get_device()
    for name, t, want in named:
        if t is not None and (t.dtype is not dtype or t.dim() != 1 or t.numel() != want or not t.is_contiguous() or t.get_device() != device):
            raise ValueError("%s must be a contiguous %s tensor of %d elements on the device of the others" % (name, str(dtype)[6:], want))


class _DeviceOf:
    """The GPU of a tensor as the current one, for calls from another one."""

    def __init__(self, t):
        if not t.is_cuda:
            raise ValueError("the tensors must be on a GPU")
        self.index = t.get_device()
        self.guard = None if torch._C._cuda_getDevice() == self.index else torch.cuda.device(self.index)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return torch._C._cuda_getCurrentRawStream(self.index)

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _seq_params(q, rows, Hkv, nseq, pages, max_new, max_keys, k_strides, v_strides, alpha, beta, gamma, delta, causal, logn_mode, alibi_slopes,
                bias_mode, path, out):
    T, Hq, D, q_st, q_sh = rows
    if Hkv < 1 or Hq < 1 or Hq % Hkv:
        raise ValueError("the query heads must be a multiple of the key/value heads")
    layout = 0
    if beta is not None or gamma is not None:
        if beta is None or gamma is None:
            raise ValueError("beta and gamma come together")
        layout = 1 if beta.dim() == 1 else 2
        want = (Hq,) if layout == 1 else (Hq, T)
        _floats("beta", beta, q, want)
        _floats("gamma", gamma, q, want)
    if alibi_slopes is not None:
        _floats("alibi_slopes", alibi_slopes, q, (Hq,))
    o_st, o_sh = Hq * D, D
    if out is not None:
        oT, oH, oD, o_st, o_sh = _rows_of("out", out)
        _like("out", out, q, T, Hq, D, oT, oH, oD)
    page_size, num_pages, max_pages = pages
    return _seq_bytes.pack(nseq, T, Hq, Hkv, D, _DTYPES[q.dtype], 1 if causal else 0, layout, logn_mode, bias_mode, path, page_size, num_pages,
                           max_pages, max_new, max_keys, alpha, delta, q_st, q_sh, o_st, o_sh, *k_strides, *v_strides)


def _paged_params(q, k_cache, v_cache, page_table, max_new, max_keys, *args):
    rows = _rows_of("q", q)
    shape, k_strides = _cache_of("k_cache", k_cache, q, rows[2])
    v_strides = k_strides
    if v_cache is not k_cache:
        v_shape, v_strides = _cache_of("v_cache", v_cache, q, rows[2])
        if v_shape != shape:
            raise ValueError("v_cache must have the shape of k_cache")
    nseq, max_pages = _page_table(page_table, q)
    return nseq, _seq_params(q, rows, shape[1], nseq, (shape[2], shape[0], max_pages), rows[0] if max_new is None else max_new,
                             min(max_pages * shape[2], _INT32_MOST) if max_keys is None else max_keys, k_strides, v_strides, *args)


def _packed_params(q, k, v, nseq, max_len, *args):
    rows = _rows_of("q", q)
    T, Hkv, D, k_st, k_sh = _rows_of("k", k)
    _like("k", k, q, rows[0], Hkv, rows[2], T, Hkv, D)
    v_st, v_sh = k_st, k_sh
    if v is not k:
        vT, vH, vD, v_st, v_sh = _rows_of("v", v)
        _like("v", v, q, T, Hkv, D, vT, vH, vD)
    most = T if max_len is None else max_len
    return _seq_params(q, rows, Hkv, nseq, (0, 0, 0), most, most, (0, k_sh, k_st), (0, v_sh, v_st), *args)


def _seq_workspace(params, device):
    return torch.empty(max(int(_lib.entmax_seq_workspace_bytes(params)), 256), dtype=torch.uint8, device=device)


_DEFAULTS = (1.5, None, None, 1.0, True, 0, None, 0, 0, None)


def new_paged_workspace(q, k_cache, page_table, max_new=None, max_keys=None):
    """Workspace for paged_attn_fwd calls of these shapes and bounds, whatever their other arguments."""
    return _seq_workspace(_paged_params(q, k_cache, k_cache, page_table, max_new, max_keys, *_DEFAULTS)[1], q.device)


def new_packed_workspace(q, k, cu_seqlens, max_len=None):
    """Workspace for packed_attn_fwd calls of these shapes and bounds, whatever their other arguments."""
    return _seq_workspace(_packed_params(q, k, k, cu_seqlens.shape[0] - 1, max_len, *_DEFAULTS), q.device)


def _outputs(q, params, out, workspace):
    if out is None:
        out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)  # (rows that no sequence owns)
    if workspace is None:
        workspace = _seq_workspace(params, q.device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.get_device() != q.get_device():
        raise ValueError("workspace must be a contiguous uint8 tensor on the device of q")
    return out, workspace


def paged_attn_fwd(q, k_cache, v_cache, cu_seqlens, kv_len, page_table, max_new=None, max_keys=None, alpha=1.5, beta=None, gamma=None,
                   delta=1.0, causal=True, logn_mode=0, alibi_slopes=None, bias_mode=0, path=0, out=None, workspace=None):
    """Entmax attention of new tokens over a paged cache that holds their keys and values already (cache_append).
    q [T,Hq,D]: the new tokens of all sequences, rows cu_seqlens[s] .. cu_seqlens[s+1]-1 those of sequence s; k_cache, v_cache
    [num_pages,Hkv,page_size,D]; kv_len [nseq]: keys of each sequence, new ones included; page_table [nseq,max_pages]; all int32 on the GPU.
    max_new, max_keys: bounds that no sequence passes (default: those of the shapes; close ones save workspace and launches).
    beta, gamma: fp32 [Hq] or [Hq,T] or None; alibi_slopes: fp32 [Hq] or None.  Returns out [T,Hq,D], which must not share
    memory with q or the cache; rows that no sequence owns are left as they are (zero in a tensor made here)."""
    nseq, p = _paged_params(q, k_cache, v_cache, page_table, max_new, max_keys, alpha, beta, gamma, delta, causal, logn_mode, alibi_slopes,
                            bias_mode, path, out)
    _int_array("cu_seqlens", cu_seqlens, q, nseq + 1)
    _int_array("kv_len", kv_len, q, nseq)
    with _DeviceOf(q) as stream:
        out, workspace = _outputs(q, p, out, workspace)
        rc = _lib.entmax_paged_attn_fwd(p, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), cu_seqlens.data_ptr(), kv_len.data_ptr(),
                                        page_table.data_ptr(), _at(beta), _at(gamma), _at(alibi_slopes), out.data_ptr(), workspace.data_ptr(),
                                        workspace.numel(), stream)
    if rc != 0:
        raise EntmaxAttnError(rc)
    return out


def packed_attn_fwd(q, k, v, cu_seqlens, max_len=None, alpha=1.5, beta=None, gamma=None, delta=1.0, causal=True, logn_mode=0,
                    alibi_slopes=None, bias_mode=0, path=0, out=None, workspace=None):
    """Entmax attention of whole prompts: q [T,Hq,D], k, v [T,Hkv,D], sequence s in rows cu_seqlens[s] .. cu_seqlens[s+1]-1.
    max_len: no sequence is longer (default: T).  The other arguments and the result as in paged_attn_fwd."""
    _int_array("cu_seqlens", cu_seqlens, q, None)
    nseq = cu_seqlens.shape[0] - 1
    if nseq < 0:
        raise ValueError("cu_seqlens must be [nseq + 1]")
    p = _packed_params(q, k, v, nseq, max_len, alpha, beta, gamma, delta, causal, logn_mode, alibi_slopes, bias_mode, path, out)
    with _DeviceOf(q) as stream:
        out, workspace = _outputs(q, p, out, workspace)
        rc = _lib.entmax_packed_attn_fwd(p, q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(), _at(beta), _at(gamma),
                                         _at(alibi_slopes), out.data_ptr(), workspace.data_ptr(), workspace.numel(), stream)
    if rc != 0:
        raise EntmaxAttnError(rc)
    return out


def cache_append(k, v, k_cache, v_cache, cu_seqlens, kv_len, page_table, q=None, q_out=None, inv_freq=None, interleaved=False):
    """Writes the new tokens' keys and values (k, v [T,Hkv,D]) to their places in the cache, keys rotated by their positions, and
    returns the queries q [T,Hq,D] rotated likewise (q_out, which may be q; None without q).
    inv_freq: fp32 [rot / 2], the angle per position of each pair of features; None: no rotation.  interleaved: pairs are neighbouring
    features, else features i and i + rot / 2.  kv_len counts the new tokens.  Other arguments as in paged_attn_fwd."""
    T, Hkv, D, k_st, k_sh = _rows_of("k", k)
    vT, vH, vD, v_st, v_sh = _rows_of("v", v)
    _like("v", v, k, T, Hkv, D, vT, vH, vD)
    shape, kc_strides = _cache_of("k_cache", k_cache, k, D)
    v_shape, vc_strides = _cache_of("v_cache", v_cache, k, D)
    if v_shape != shape or shape[1] != Hkv:
        raise ValueError("k_cache and v_cache must be [num_pages,Hkv,page_size,D] with the heads of k")
    nseq, max_pages = _page_table(page_table, k)
    _int_array("cu_seqlens", cu_seqlens, k, nseq + 1)
    _int_array("kv_len", kv_len, k, nseq)
    Hq, q_st, q_sh, qo_st, qo_sh, rot = 0, 0, 0, 0, 0, 0
    if q is not None:
        qT, Hq, qD, q_st, q_sh = _rows_of("q", q)
        _like("q", q, k, T, Hq, D, qT, Hq, qD)
        qo_st, qo_sh = Hq * D, D
        if q_out is not None:
            oT, oH, oD, qo_st, qo_sh = _rows_of("q_out", q_out)
            _like("q_out", q_out, q, T, Hq, D, oT, oH, oD)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if inv_freq is not None:
        if inv_freq.dtype != torch.float32 or not inv_freq.is_contiguous() or inv_freq.dim() != 1 or inv_freq.get_device() != k.get_device():
            raise ValueError("inv_freq must be a contiguous float32 tensor [rot / 2] on the device of the others")
        rot = 2 * inv_freq.shape[0]
    p = _append_bytes.pack(nseq, T, Hq, Hkv, D, _DTYPES[k.dtype], shape[2], shape[0], max_pages, rot, 1 if interleaved else 0, q_st, q_sh, qo_st,
                           qo_sh, k_st, k_sh, v_st, v_sh, *kc_strides, *vc_strides)
    with _DeviceOf(k) as stream:
        if q is not None and q_out is None:
            q_out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)  # (rows that no sequence owns)
        rc = _lib.entmax_cache_append(p, _at(q), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(),
                                      _at(inv_freq), _at(q_out), k_cache.data_ptr(), v_cache.data_ptr(), stream)
    if rc != 0:
        raise EntmaxAttnError(rc)
    return q_out


# ------------------------------------------------- serving: the plan of a step, softmax attention, sampling

class PlanParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("nseq", "T", "page_size", "num_pages", "max_pages")]


class SampleParams(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("stride", ctypes.c_int64)]


_plan_bytes = struct.Struct("@5i")
_sample_bytes = struct.Struct("@3i4xq")
assert _plan_bytes.size == ctypes.sizeof(PlanParams) and _sample_bytes.size == ctypes.sizeof(SampleParams)

_lib.entmax_cache_plan.restype = ctypes.c_int
_lib.entmax_cache_plan.argtypes = [_vp] * 14 + [ctypes.c_size_t, _vp]
_lib.entmax_plan_workspace_bytes.restype = ctypes.c_size_t
_lib.entmax_plan_workspace_bytes.argtypes = [_vp]
_lib.entmax_paged_softmax_fwd.restype = ctypes.c_int
_lib.entmax_paged_softmax_fwd.argtypes = [_vp, ctypes.c_float] + [_vp] * 12 + [ctypes.c_size_t, _vp]
_lib.entmax_softmax_workspace_bytes.restype = ctypes.c_size_t
_lib.entmax_softmax_workspace_bytes.argtypes = [_vp]
_lib.entmax_sample.restype = ctypes.c_int
_lib.entmax_sample.argtypes = [_vp] * 10 + [ctypes.c_size_t, _vp]
_lib.entmax_sample_workspace_bytes.restype = ctypes.c_size_t
_lib.entmax_sample_workspace_bytes.argtypes = [_vp]

# What cache_plan makes: cu_seqlens [nseq + 1], kv_len [nseq], free_count [1], and for each row of the step slots (int64), positions and sequences
Plan = collections.namedtuple("Plan", "cu_seqlens kv_len free_count slots positions sequences workspace")


def new_plan(nseq, rows, device="cuda"):
    """Outputs and workspace of cache_plan for steps of `rows` rows; kv_len and free_count begin at zero."""
    ints = lambda n: torch.zeros(n, dtype=torch.int32, device=device)  # noqa: E731
    need = int(_lib.entmax_plan_workspace_bytes(_plan_bytes.pack(nseq, rows, 16, 0, 0)))
    return Plan(ints(nseq + 1), ints(nseq), ints(1), torch.zeros(rows, dtype=torch.int64, device=device), ints(rows), ints(rows),
                torch.empty(max(need, 256), dtype=torch.uint8, device=device))


def cache_plan(new_len, kv_len, page_table, free_pages, free_count, page_size, plan, release=None):
    """Pages and places in the cache for the new tokens of a step; fills and returns `plan` (new_plan; slots, positions, sequences may be None in it).
    new_len, kv_len [nseq]: new tokens and cached keys of each sequence; release [nseq] or None: sequences with a number other than 0 have ended and
    give their pages back first.  page_table [nseq,max_pages] and free_pages [num_pages], whose first free_count [1] entries are the free pages, are
    updated.  kv_len and free_count may be the plan's own: the next step goes on from there.  All int32 on the GPU.  A sequence that does not
    get its pages (or whose tokens do not fit the plan's rows) gets no rows; those behind the last sequence have -1 everywhere."""
    nseq, max_pages = _page_table(page_table, new_len)
    i32 = torch.int32
    cu_seqlens, slots, positions, sequences = plan.cu_seqlens, plan.slots, plan.positions, plan.sequences
    rows = slots if slots is not None else positions if positions is not None else sequences
    if rows is None:
        raise ValueError("the plan needs slots, positions or sequences: their length is the number of rows")
    rows = rows.numel()
    _arrays(new_len, i32, ("new_len", new_len, nseq), ("kv_len", kv_len, nseq), ("release", release, nseq), ("free_count", free_count, 1),
            ("free_pages", free_pages, free_pages.numel()), ("plan.cu_seqlens", cu_seqlens, nseq + 1), ("plan.kv_len", plan.kv_len, nseq),
            ("plan.free_count", plan.free_count, 1), ("plan.positions", positions, rows), ("plan.sequences", sequences, rows))
    _arrays(new_len, torch.int64, ("plan.slots", slots, rows))
    w = plan.workspace
    if w.dtype != torch.uint8 or not w.is_contiguous() or w.get_device() != new_len.get_device():
        raise ValueError("plan.workspace must be a contiguous uint8 tensor on the device of the others")
    p = _plan_bytes.pack(nseq, rows, page_size, free_pages.numel(), max_pages)
    with _DeviceOf(new_len) as stream:
        rc = _lib.entmax_cache_plan(p, new_len.data_ptr(), _at(release), kv_len.data_ptr(), free_count.data_ptr(), page_table.data_ptr(),
                                    free_pages.data_ptr(), plan.kv_len.data_ptr(), plan.free_count.data_ptr(), cu_seqlens.data_ptr(),
                                    _at(slots), _at(positions), _at(sequences), w.data_ptr(), w.numel(), stream)
    if rc != 0:
        raise EntmaxAttnError(rc)
    return plan


_SOFTMAX_DEFAULTS = (1.0,) + _DEFAULTS[1:]


def _softmax_workspace(params, device):
    return torch.empty(max(int(_lib.entmax_softmax_workspace_bytes(params)), 256), dtype=torch.uint8, device=device)


def new_softmax_workspace(q, k_cache, page_table, max_new=None, max_keys=None):
    """Workspace for paged_softmax_fwd calls of these shapes and bounds, whatever their other arguments."""
    return _softmax_workspace(_paged_params(q, k_cache, k_cache, page_table, max_new, max_keys, *_SOFTMAX_DEFAULTS)[1], q.device)


def paged_softmax_fwd(q, k_cache, v_cache, cu_seqlens, kv_len, page_table, max_new=None, max_keys=None, cap=0.0, beta=None, gamma=None,
                      delta=1.0, causal=True, logn_mode=0, alibi_slopes=None, bias_mode=0, out=None, lse=None, workspace=None):
    """Softmax attention of new tokens over a paged cache: paged_attn_fwd in the limit alpha -> 1, with the same arguments and result.
    cap: 0, or c > 0 for scores c tanh(s / c).  lse: optional fp32 [Hq,T] tensor that receives the logarithm of each row's sum of exponentials."""
    nseq, p = _paged_params(q, k_cache, v_cache, page_table, max_new, max_keys, 1.0, beta, gamma, delta, causal, logn_mode, alibi_slopes,
                            bias_mode, 0, out)
    _int_array("cu_seqlens", cu_seqlens, q, nseq + 1)
    _int_array("kv_len", kv_len, q, nseq)
    if lse is not None:
        _floats("lse", lse, q, (q.shape[1], q.shape[0]))
    with _DeviceOf(q) as stream:
        if out is None:
            out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)  # (rows that no sequence owns)
        if workspace is None:
            workspace = _softmax_workspace(p, q.device)
        elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.get_device() != q.get_device():
            raise ValueError("workspace must be a contiguous uint8 tensor on the device of q")
        rc = _lib.entmax_paged_softmax_fwd(p, cap, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), cu_seqlens.data_ptr(), kv_len.data_ptr(),
                                           page_table.data_ptr(), _at(beta), _at(gamma), _at(alibi_slopes), out.data_ptr(), _at(lse),
                                           workspace.data_ptr(), workspace.numel(), stream)
    if rc != 0:
        raise EntmaxAttnError(rc)
    return out


def _sample_params(logits):
    if logits.dim() != 2:
        raise ValueError("logits must be [rows,vocab]")
    if logits.dtype not in _DTYPES:
        raise TypeError("logits must be bfloat16 or float32")
    rows, vocab = logits.shape
    stride = vocab
    if rows and vocab:
        if vocab > 1 and logits.stride(1) != 1:
            raise ValueError("the last dimension of logits must be contiguous")
        if rows > 1:
            stride = logits.stride(0)
    return rows, _sample_bytes.pack(rows, vocab, _DTYPES[logits.dtype], stride)


def _sample_workspace(params, device):
    return torch.empty(max(int(_lib.entmax_sample_workspace_bytes(params)), 256), dtype=torch.uint8, device=device)


def new_sample_workspace(logits):
    """Workspace for sample calls with logits of this shape and type."""
    return _sample_workspace(_sample_params(logits)[1], logits.device)


def sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, token=None, logprob=None, workspace=None):
    """One token of each row of logits [rows,vocab] (bf16 or fp32, rows any stride apart) as int32 [rows], drawn with the random numbers uniform
    (fp32 [rows] in [0,1)) after temperature, top_k, top_p and min_p in this order.  temperature, top_p, min_p: fp32 [rows], top_k: int32 [rows]; None, or a
    row's top_k <= 0, top_p >= 1, min_p <= 0: not wanted; temperature <= 0: the largest logit.  Of equal logits the first is the larger.
    logprob: optional fp32 [rows] tensor that receives the log of the probability with which the token was drawn.  -1 for rows without a token to
    draw (all -infinity or NaN)."""
    rows, p = _sample_params(logits)
    f32, i32 = torch.float32, torch.int32
    _arrays(logits, f32, ("uniform", uniform, rows), ("temperature", temperature, rows), ("top_p", top_p, rows), ("min_p", min_p, rows),
            ("logprob", logprob, rows))
    _arrays(logits, i32, ("top_k", top_k, rows), ("token", token, rows))
    with _DeviceOf(logits) as stream:
        if token is None:
            token = torch.empty(rows, dtype=i32, device=logits.device)
        if workspace is None:
            workspace = _sample_workspace(p, logits.device)
        elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.get_device() != logits.get_device():
            raise ValueError("workspace must be a contiguous uint8 tensor on the device of logits")
        rc = _lib.entmax_sample(p, logits.data_ptr(), uniform.data_ptr(), _at(temperature), _at(top_k), _at(top_p), _at(min_p), token.data_ptr(),
                                _at(logprob), workspace.data_ptr(), workspace.numel(), stream)
    if rc != 0:
        raise EntmaxAttnError(rc)
    return token
