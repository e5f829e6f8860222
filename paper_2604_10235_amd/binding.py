"""ctypes binding of libcodecomp.so: argument marshalling only.

Every step of the path runs in the library's HIP kernels; nothing here computes.  Tensors are
torch CUDA(ROCm) tensors used as device memory, the stream is torch's current stream.  The
library must have been built in-tree (paper_2604_10235_amd/build.py); loading fails loudly
otherwise - there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# CODECOMP_LIB selects another build of the same library (experiments); the default is the in-tree one
LIB_PATH = os.environ.get("CODECOMP_LIB") or os.path.join(_HERE, "libcodecomp.so")

STATUS = {
    0: "CODECOMP_OK", -1: "CODECOMP_EINVAL_NULL", -2: "CODECOMP_EINVAL_SHAPE", -3: "CODECOMP_EINVAL_WINDOW",
    -4: "CODECOMP_EINVAL_BUDGET", -5: "CODECOMP_EINVAL_POOL", -6: "CODECOMP_EINVAL_HEADS",
    -7: "CODECOMP_EINVAL_HEADDIM", -8: "CODECOMP_EINVAL_SEQLENS", -9: "CODECOMP_EINVAL_WORKSPACE",
    -10: "CODECOMP_EINVAL_PRIOR", -11: "CODECOMP_EINVAL_MODE", -12: "CODECOMP_EINVAL_PAGES",
}


class codecomp_params(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("window", C.c_int32), ("pool_kernel", C.c_int32), ("prior_weight", C.c_float), ("softmax_scale", C.c_float),
        ("n_seqs", C.c_int32), ("select_mode", C.c_int32),
        ("cu_seqlens_host", C.c_void_p), ("cu_seqlens_dev", C.c_void_p),
        ("cu_budgets_host", C.c_void_p), ("cu_budgets_dev", C.c_void_p),
        ("q_stride_layer", C.c_int64), ("q_stride_seq", C.c_int64), ("q_stride_head", C.c_int64),
        ("q_stride_tok", C.c_int64),
        ("kv_stride_layer", C.c_int64), ("kv_stride_head", C.c_int64), ("kv_stride_tok", C.c_int64),
        ("out_stride_layer", C.c_int64), ("out_stride_head", C.c_int64), ("out_stride_tok", C.c_int64),
        ("span_budget_ratio", C.c_float), ("span_budget_min", C.c_int32),
        ("score_variant", C.c_int32), ("kv_dtype", C.c_int32),
        ("score_workgroups", C.c_int32), ("score_lead_tiles", C.c_int32),
    ]


class codecomp_pages(C.Structure):
    _fields_ = [
        ("k", C.c_void_p), ("v", C.c_void_p), ("n_layers", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32),
        ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("kv_dtype", C.c_int32),
        ("stride_layer", C.c_int64), ("stride_page", C.c_int64), ("stride_head", C.c_int64), ("stride_tok", C.c_int64),
        ("k_scale", C.c_float), ("v_scale", C.c_float),
    ]


class codecomp_batch(C.Structure):
    _fields_ = [
        ("n_seqs", C.c_int32), ("n_q_heads", C.c_int32), ("table_width", C.c_int32), ("max_kv_len", C.c_int32), ("causal", C.c_int32),
        ("softmax_scale", C.c_float), ("cu_q_host", C.c_void_p), ("cu_q_dev", C.c_void_p), ("kv_lens_dev", C.c_void_p), ("table_dev", C.c_void_p),
        ("q_stride_tok", C.c_int64), ("q_stride_head", C.c_int64), ("new_stride_tok", C.c_int64), ("new_stride_head", C.c_int64),
        ("out_stride_tok", C.c_int64), ("out_stride_head", C.c_int64),
    ]


class codecomp_rotary(C.Structure):
    _fields_ = [("dim", C.c_int32), ("interleaved", C.c_int32), ("inverse", C.c_int32), ("magnitude", C.c_float), ("freq", C.c_double * 64)]


class CodecompError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({STATUS.get(status, 'hipError_t' if status > 0 else '?')}): "
                         f"{status_string(status)}")


_lib = None


def lib() -> C.CDLL:
    """The loaded library.  Raises if it has not been built: the HIP path has no substitute."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2604_10235_amd.build)")
        # The device memory and the streams that this binding hands to the library come from torch, which ships
        # its own HIP runtime.  Loaded first, that runtime is the one the library binds to; the other way round
        # the process ends up with two runtimes and every launch fails with hipErrorNoDevice.
        import torch  # noqa: F401
        l = C.CDLL(LIB_PATH)
        P = C.POINTER(codecomp_params)
        l.codecomp_workspace_bytes.restype = C.c_size_t
        l.codecomp_workspace_bytes.argtypes = [P]
        l.codecomp_validate.restype = C.c_int
        l.codecomp_validate.argtypes = [P]
        l.codecomp_score_layout.restype = C.c_int
        l.codecomp_score_layout.argtypes = [P, C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                            C.POINTER(C.c_uint32)]
        IP = C.POINTER(C.c_int32)
        l.codecomp_score_route.restype = C.c_int
        l.codecomp_score_route.argtypes = [P, IP, IP, IP]
        l.codecomp_score_teams.restype = C.c_int
        l.codecomp_score_teams.argtypes = [P, IP]
        l.codecomp_score.restype = C.c_int
        l.codecomp_score.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, P, C.c_void_p, C.c_void_p, C.c_size_t,
                                     C.c_void_p]
        l.codecomp_score_stages.restype = C.c_int
        l.codecomp_score_stages.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, P, C.c_void_p, C.c_void_p, C.c_size_t,
                                            C.c_uint, C.c_void_p]
        l.codecomp_select.restype = C.c_int
        l.codecomp_select.argtypes = [C.c_void_p, P, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        l.codecomp_select_two_stage.restype = C.c_int
        l.codecomp_select_two_stage.argtypes = [C.c_void_p, C.c_void_p, P, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        l.codecomp_gather.restype = C.c_int
        l.codecomp_gather.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, P, C.c_void_p, C.c_void_p, C.c_void_p]
        l.codecomp_compress.restype = C.c_int
        l.codecomp_compress.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, P, C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        l.codecomp_compress_static.restype = C.c_int
        l.codecomp_compress_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, P, C.c_void_p, C.c_void_p,
                                               C.c_void_p, C.c_void_p, C.c_void_p]
        l.codecomp_structure_score.restype = C.c_int
        l.codecomp_structure_score.argtypes = [C.c_void_p, C.c_void_p, P, C.c_void_p, C.c_void_p]
        DP = C.POINTER(C.c_double)
        l.codecomp_chunk_structure_scores.restype = C.c_int
        l.codecomp_chunk_structure_scores.argtypes = [DP, DP, DP, C.c_int32, C.c_int32, DP]
        l.codecomp_chunk_budgets.restype = C.c_int
        l.codecomp_chunk_budgets.argtypes = [DP, IP, C.c_int32, C.c_double, C.c_double, C.c_double, C.c_double,
                                             C.c_double, C.c_int32, IP]
        PP, BP, RP, V = C.POINTER(codecomp_pages), C.POINTER(codecomp_batch), C.POINTER(codecomp_rotary), C.c_void_p
        for name, args in {
            "rotary_init": [RP, C.c_int32, C.c_int32, C.c_double, C.c_int32] + [C.c_double] * 4,
            "rotate": [V, V, RP, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_int64, V, C.c_int64, C.c_int64, V],
            "append": [V, V, V, V, RP, BP, PP, C.c_int32, V, V],
            "pages_store": [V, V, V, P, PP, V, C.c_int32, V, V],
            "pages_load": [PP, V, C.c_int32, V, V, P, V, V, V],
            "pages_compact": [PP, V, C.c_int32, V, V, P, PP, V, C.c_int32, V, V],
            "pages_copy": [PP, V, C.c_int32, V],
            "attend_validate": [BP, PP],
            "attend": [V, BP, PP, C.c_int32, V, V, V, C.c_size_t, V],
        }.items():
            f = getattr(l, "codecomp_" + name)
            f.restype, f.argtypes = C.c_int, args
        l.codecomp_attend_workspace_bytes.restype = C.c_size_t
        l.codecomp_attend_workspace_bytes.argtypes = [BP, PP]
        l.codecomp_status_string.restype = C.c_char_p
        l.codecomp_status_string.argtypes = [C.c_int]
        l.codecomp_version.restype = C.c_int
        l.codecomp_version.argtypes = []
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().codecomp_status_string(int(status)).decode()


def version() -> int:
    return lib().codecomp_version()


def make_params(*, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, window: int, pool_kernel: int,
                prior_weight: float, cu_seqlens_host: np.ndarray, cu_budgets_host: np.ndarray,
                cu_seqlens_dev: int = 0, cu_budgets_dev: int = 0, softmax_scale: float = 0.0, **strides):
    """Fills a codecomp_params.  The host arrays are kept alive on the returned object; the device
    pointers are plain integers (tensor.data_ptr())."""
    csl = np.ascontiguousarray(cu_seqlens_host, dtype=np.int32)
    cbl = np.ascontiguousarray(cu_budgets_host, dtype=np.int32)
    p = codecomp_params()
    p.n_layers, p.n_q_heads, p.n_kv_heads, p.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
    p.window, p.pool_kernel, p.prior_weight, p.softmax_scale = window, pool_kernel, prior_weight, softmax_scale
    p.n_seqs = len(csl) - 1
    p.cu_seqlens_host = csl.ctypes.data
    p.cu_budgets_host = cbl.ctypes.data
    p.cu_seqlens_dev = cu_seqlens_dev
    p.cu_budgets_dev = cu_budgets_dev
    for name, val in strides.items():      # strides, select_mode, span_budget_*, score_variant, kv_dtype, score_workgroups ...
        setattr(p, name, val)
    p._keep = (csl, cbl)
    return p


def codecomp_validate(params: codecomp_params) -> int:
    return lib().codecomp_validate(C.byref(params))


def codecomp_score_layout(params: codecomp_params):
    """(status, row_splits, row_blocks, waves, wave_desc[8]) of the score passes for these parameters."""
    rs, rb, nw = C.c_int32(0), C.c_int32(0), C.c_int32(0)
    desc = (C.c_uint32 * 8)()
    rc = lib().codecomp_score_layout(C.byref(params), C.byref(rs), C.byref(rb), C.byref(nw), desc)
    return rc, rs.value, rb.value, nw.value, list(desc)


ROUTE_TWO_PASSES, ROUTE_ONE_PASS, ROUTE_FEW_ROWS = 0, 1, 2


def codecomp_score_route(params: codecomp_params):
    """(route per request (ROUTE_*), row chunks of a one-pass request, how many of them a workgroup takes in turn)."""
    route, chunks, turn = (C.c_int32 * max(1, params.n_seqs))(), C.c_int32(0), C.c_int32(0)
    _check(lib().codecomp_score_route(C.byref(params), route, C.byref(chunks), C.byref(turn)), "codecomp_score_route")
    return np.ctypeslib.as_array(route).copy(), chunks.value, turn.value


def codecomp_score_teams(params: codecomp_params) -> int:
    """Workgroups of the largest team where the ROUTE_TWO_PASSES requests are given to teams, which form every logit once; else 0."""
    members = C.c_int32(0)
    _check(lib().codecomp_score_teams(C.byref(params), C.byref(members)), "codecomp_score_teams")
    return members.value


def codecomp_workspace_bytes(params: codecomp_params) -> int:
    return lib().codecomp_workspace_bytes(C.byref(params))


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _stream() -> int:
    import torch
    return int(torch.cuda.current_stream().cuda_stream)


def _check(rc: int, where: str):
    if rc != 0:
        raise CodecompError(rc, where)


def codecomp_score(q_obs, k, prior, params, scores, workspace) -> None:
    _check(lib().codecomp_score(_ptr(q_obs), _ptr(k), _ptr(prior), C.byref(params), _ptr(scores), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream()), "codecomp_score")


STAGE_ROW_STATS, STAGE_ROW_MERGE, STAGE_MASS, STAGE_FINISH, STAGE_ALL = 1, 2, 4, 8, 15
VARIANT_GROUP_SUM, VARIANT_GROUP_MAX, VARIANT_POOL_MAX, VARIANT_SOFTMAX_PREFIX, VARIANT_POOL_PREFIX = 1, 2, 4, 8, 16
VARIANT_NO_TEAMS, VARIANT_TEAMS_APART = 256, 512
KV_BF16, KV_FP8_E4M3 = 0, 1


def codecomp_score_stages(q_obs, k, prior, params, scores, workspace, stages: int) -> None:
    _check(lib().codecomp_score_stages(_ptr(q_obs), _ptr(k), _ptr(prior), C.byref(params), _ptr(scores),
                                       _ptr(workspace), workspace.numel() * workspace.element_size(), int(stages),
                                       _stream()), "codecomp_score_stages")


def codecomp_select(scores, params, idx, workspace) -> None:
    _check(lib().codecomp_select(_ptr(scores), C.byref(params), _ptr(idx), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream()), "codecomp_select")


def codecomp_select_two_stage(scores, prior, params, idx, workspace) -> None:
    _check(lib().codecomp_select_two_stage(_ptr(scores), _ptr(prior), C.byref(params), _ptr(idx), _ptr(workspace),
                                           workspace.numel() * workspace.element_size(), _stream()),
           "codecomp_select_two_stage")


def codecomp_gather(k, v, idx, params, k_out, v_out) -> None:
    _check(lib().codecomp_gather(_ptr(k), _ptr(v), _ptr(idx), C.byref(params), _ptr(k_out), _ptr(v_out), _stream()),
           "codecomp_gather")


def codecomp_compress(q_obs, k, v, prior, params, scores, idx, k_out, v_out, workspace) -> None:
    _check(lib().codecomp_compress(_ptr(q_obs), _ptr(k), _ptr(v), _ptr(prior), C.byref(params), _ptr(scores),
                                   _ptr(idx), _ptr(k_out), _ptr(v_out), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream()), "codecomp_compress")


STATIC_SCRATCH_BYTES = 32 * 1024 * 1024


def codecomp_compress_static(q_obs, k, v, prior, params, scores, idx, k_out, v_out) -> None:
    _check(lib().codecomp_compress_static(_ptr(q_obs), _ptr(k), _ptr(v), _ptr(prior), C.byref(params), _ptr(scores),
                                          _ptr(idx), _ptr(k_out), _ptr(v_out), _stream()), "codecomp_compress_static")


def codecomp_structure_score(idx, prior, params, retained) -> None:
    _check(lib().codecomp_structure_score(_ptr(idx), _ptr(prior), C.byref(params), _ptr(retained), _stream()),
           "codecomp_structure_score")


def _dp(a):
    return a.ctypes.data_as(C.POINTER(C.c_double))


def codecomp_chunk_structure_scores(features, tau, weights) -> np.ndarray:
    f = np.ascontiguousarray(features, dtype=np.float64)
    t = np.ascontiguousarray(tau, dtype=np.float64)
    w = np.ascontiguousarray(weights, dtype=np.float64)
    out = np.empty(f.shape[0], dtype=np.float64)
    _check(lib().codecomp_chunk_structure_scores(_dp(f), _dp(t), _dp(w), f.shape[0], f.shape[1], _dp(out)),
           "codecomp_chunk_structure_scores")
    return out


def codecomp_chunk_budgets(sigma, chunk_len, *, ratio, m_min, m_max, r_max, eps, window) -> np.ndarray:
    s = np.ascontiguousarray(sigma, dtype=np.float64)
    ln = np.ascontiguousarray(chunk_len, dtype=np.int32)
    out = np.empty(len(s), dtype=np.int32)
    ip = C.POINTER(C.c_int32)
    _check(lib().codecomp_chunk_budgets(_dp(s), ln.ctypes.data_as(ip), len(s), ratio, m_min, m_max, r_max, eps, window,
                                        out.ctypes.data_as(ip)), "codecomp_chunk_budgets")
    return out


# ---- serving from a compressed cache (codecomp_cache.h).  Sizes and strides come from the tensors' shapes, so that a call cannot
# reach outside of them; tensors of another type, shape or device than the call needs are refused with ValueError.

_torch_module = None


def _torch():
    """torch, imported by the first call that is given tensors (a global is looked up several times faster than an import statement runs)."""
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_WAVELENGTH, ROTARY_RAMP = 0, 1, 2, 3, 4
ROTARY_SCALINGS = {"plain": ROTARY_PLAIN, "linear": ROTARY_LINEAR, "base": ROTARY_BASE, "wavelength": ROTARY_WAVELENGTH, "ramp": ROTARY_RAMP}


def make_rotary(dim: int, *, base: float = 10000.0, interleaved: bool = False, inverse: bool = False, scaling: int = ROTARY_PLAIN,
                factor: float = 1.0, context: float = 0.0, low: float = 1.0, high: float = 4.0, magnitude: float = 1.0) -> codecomp_rotary:
    """Frequencies by codecomp_rotary_init (the meaning of factor, context, low and high per scaling stands there); `freq` may be overwritten."""
    r = codecomp_rotary()
    _check(lib().codecomp_rotary_init(C.byref(r), dim, int(interleaved), base, scaling, factor, context, low, high), "codecomp_rotary_init")
    r.inverse, r.magnitude = int(inverse), magnitude
    return r


def _own_strides(t, what: str):
    """Strides for the library: 0 (dense) where there is one place only; a stride of 0 between several would be taken for dense."""
    if any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride())):
        raise ValueError(f"{what} must not be a broadcast tensor (strides {t.stride()})")
    return [s if n > 1 else 0 for n, s in zip(t.shape, t.stride())]


def make_pages(k, v, *, k_scale: float = 1.0, v_scale: float = 1.0) -> codecomp_pages:
    """A pool over two tensors [layers, pages, KV heads, page size, head_dim] with the same strides, bf16 or 8-bit (float8_e4m3fn, or codes as uint8)."""
    torch = _torch()
    if k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device:
        raise ValueError("k and v must be tensors [layers, pages, KV heads, page size, head_dim] of the same shape, strides, type and device")
    if k.dtype not in (torch.bfloat16, torch.uint8, torch.float8_e4m3fn):
        raise ValueError(f"a cache holds bfloat16 or 8-bit (float8_e4m3fn, uint8) elements, not {k.dtype}")
    if k.stride(4) != 1:
        raise ValueError("the elements of a row must be contiguous")
    strides = _own_strides(k, "a pool")
    p = codecomp_pages()
    p.k, p.v = k.data_ptr(), v.data_ptr()
    p.n_layers, p.n_pages, p.n_kv_heads, p.page_size, p.head_dim = k.shape
    p.kv_dtype = KV_BF16 if k.dtype == torch.bfloat16 else KV_FP8_E4M3
    p.stride_layer, p.stride_page, p.stride_head, p.stride_tok = strides[:4]
    p.k_scale, p.v_scale = k_scale, v_scale
    p._keep, p._at = (k, v), k.get_device()
    return p


def _int32(t, shape, what: str):
    if t.dtype is not (_torch_module or _torch()).int32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous int32 tensor of shape {shape}, not {t.dtype} {tuple(t.shape)}")


def make_batch(*, n_q_heads: int, cu_q_host: np.ndarray, cu_q, kv_lens, table, max_kv_len: int, causal: bool = True, softmax_scale: float = 0.0,
               **strides) -> codecomp_batch:
    """New tokens of n_seqs requests over their caches.  cu_q, kv_lens, table: device int32 tensors [n_seqs + 1], [n_seqs], [n_seqs, width]; the host
    array cu_q_host (same values as cu_q; copied) sizes the launches.  Strides of q, of new k and v, and of what comes out: 0 or left out = dense."""
    host = np.array(cu_q_host, dtype=np.int32, order="C")        # a copy: calls read it, long after the tensors were checked against it
    n = len(host) - 1
    _int32(cu_q, (n + 1,), "cu_q")
    _int32(kv_lens, (n,), "kv_lens")
    _int32(table, (n, table.shape[-1]), "table")
    if len({t.device for t in (cu_q, kv_lens, table)}) > 1:
        raise ValueError("cu_q, kv_lens and table must be on the same device")
    b = codecomp_batch()
    b.n_seqs, b.n_q_heads, b.table_width, b.max_kv_len, b.causal, b.softmax_scale = n, n_q_heads, table.shape[1], max_kv_len, int(causal), softmax_scale
    b.cu_q_host, b.cu_q_dev, b.kv_lens_dev, b.table_dev = host.ctypes.data, cu_q.data_ptr(), kv_lens.data_ptr(), table.data_ptr()
    for name, val in strides.items():
        if "_stride_" not in name or not hasattr(b, name):
            raise TypeError(f"codecomp_batch has no stride {name}")
        setattr(b, name, val)
    b._keep, b._tokens, b._at = (host, cu_q, kv_lens, table), int(host[-1]), cu_q.get_device()
    return b


def _launch_stream(*at: int) -> int:
    """torch's current stream on the current device, where everything has to be (`at`: device numbers, -1 for the CPU): the library launches there."""
    c = (_torch_module or _torch())._C
    device = c._cuda_getDevice()
    for i in at:
        if i != device:
            raise ValueError(f"a tensor is on {'the CPU' if i < 0 else f'cuda:{i}'}, the current device is cuda:{device}")
    return c._cuda_getCurrentRawStream(device)


def _at(t, otherwise: int) -> int:
    return otherwise if t is None else t.get_device()


def _vectors(t, what: str, shape, stride_tok: int, stride_head: int) -> int:
    """bf16 [tokens, heads, head_dim] with the strides that the call will use (0 = dense)."""
    if t.dtype is not (_torch_module or _torch()).bfloat16 or t.shape != shape:
        raise ValueError(f"{what} must be bfloat16 {shape}, not {t.dtype} {tuple(t.shape)}")
    if not shape[0] or (not stride_tok and not stride_head and t.is_contiguous()):          # strides of nothing say nothing
        return t.data_ptr()
    want = (stride_tok or shape[1] * shape[2], stride_head or shape[2], 1)
    if t.stride() != want and any(n > 1 and s != w for n, s, w in zip(shape, t.stride(), want)):
        raise ValueError(f"{what} has strides {t.stride()}, the call goes by {want}")
    return t.data_ptr()


def _row_strides(t, what: str):
    """Of tokens and heads, for vectors that are not dense."""
    tok, head, one = t.stride()
    if one != 1 and t.shape[2] > 1:
        raise ValueError(f"{what} must have contiguous heads (strides {t.stride()})")
    if (tok == 0 and t.shape[0] > 1) or (head == 0 and t.shape[1] > 1):
        raise ValueError(f"{what} must not be a broadcast tensor (strides {t.stride()})")
    return tok if t.shape[0] > 1 else 0, head if t.shape[1] > 1 else 0


def codecomp_rotate(x, positions, rotary: codecomp_rotary, out) -> None:
    """x, out: bf16 [tokens, heads, head_dim], any strides of tokens and heads."""
    bf16 = (_torch_module or _torch()).bfloat16
    shape = x.shape
    if len(shape) != 3 or shape != out.shape or x.dtype is not bf16 or out.dtype is not bf16:
        raise ValueError("x and out must be bfloat16 [tokens, heads, head_dim]")
    T, H, d = shape
    _int32(positions, (T,), "positions")
    x_tok, x_head = (0, 0) if x.is_contiguous() else _row_strides(x, "x")
    o_tok, o_head = (0, 0) if out.is_contiguous() else _row_strides(out, "out")
    stream = _launch_stream(x.get_device(), positions.get_device(), out.get_device())
    _check(lib().codecomp_rotate(x.data_ptr(), positions.data_ptr(), C.byref(rotary), T, H, d, x_tok, x_head, out.data_ptr(), o_tok, o_head, stream),
           "codecomp_rotate")


def codecomp_append(q, k, v, positions, rotary: Optional[codecomp_rotary], batch: codecomp_batch, pages: codecomp_pages, layer: int, q_out) -> None:
    T, d = batch._tokens, pages.head_dim
    kv = (T, pages.n_kv_heads, d)
    kp, vp = _vectors(k, "k", kv, batch.new_stride_tok, batch.new_stride_head), _vectors(v, "v", kv, batch.new_stride_tok, batch.new_stride_head)
    qp = op = 0
    if q is not None:
        qp = _vectors(q, "q", (T, batch.n_q_heads, d), batch.q_stride_tok, batch.q_stride_head)
    if q_out is not None:
        op = _vectors(q_out, "q_out", (T, batch.n_q_heads, d), batch.out_stride_tok, batch.out_stride_head)
    if positions is not None:
        _int32(positions, (T,), "positions")
    at = pages._at
    stream = _launch_stream(at, batch._at, k.get_device(), v.get_device(), _at(q, at), _at(q_out, at), _at(positions, at))
    _check(lib().codecomp_append(qp, kp, vp, _ptr(positions), None if rotary is None else C.byref(rotary), C.byref(batch), C.byref(pages), layer, op,
                                 stream), "codecomp_append")


def _rows(t, params, what: str, total: int, strides) -> int:
    """Dense rows [layers, KV heads, total, head_dim] in the cache's type with the strides that `params` says."""
    torch = _torch()
    fp8 = params.kv_dtype == KV_FP8_E4M3
    shape = (params.n_layers, params.n_kv_heads, total, params.head_dim)
    if (t.dtype not in (torch.uint8, torch.float8_e4m3fn) if fp8 else t.dtype != torch.bfloat16) or t.shape != shape:
        raise ValueError(f"{what} must be {'8-bit' if fp8 else 'bfloat16'} {shape}, not {t.dtype} {tuple(t.shape)}")
    want = (strides[0] or shape[1] * shape[2] * shape[3], strides[1] or shape[2] * shape[3], strides[2] or shape[3], 1)
    if any(n > 1 and s != w for n, s, w in zip(t.shape, t.stride(), want)):
        raise ValueError(f"{what} has strides {t.stride()}, the call goes by {want}")
    return t.data_ptr()


def _side(params, compact: bool):
    if compact:
        return int(params._keep[1][-1]), (params.out_stride_layer, params.out_stride_head, params.out_stride_tok)
    return int(params._keep[0][-1]), (params.kv_stride_layer, params.kv_stride_head, params.kv_stride_tok)


def _table(table, first, params):
    _int32(table, (params.n_seqs, table.shape[-1]), "table")
    if first is not None:
        _int32(first, (params.n_seqs,), "first")


def _idx(idx, params):
    _int32(idx, (params.n_layers, params.n_kv_heads, int(params._keep[1][-1])), "idx")


def codecomp_pages_store(k, v, idx, params, pages, table, first=None) -> None:
    """idx None: the compact k, v [L, H_kv, TB, d] into pages; else rows idx [L, H_kv, TB] of the cache k, v [L, H_kv, T, d]."""
    total, strides = _side(params, idx is None)
    _table(table, first, params)
    if idx is not None:
        _idx(idx, params)
    kp, vp = _rows(k, params, "k", total, strides), _rows(v, params, "v", total, strides)
    at = pages._at
    stream = _launch_stream(at, k.get_device(), v.get_device(), table.get_device(), _at(idx, at), _at(first, at))
    _check(lib().codecomp_pages_store(kp, vp, _ptr(idx), C.byref(params), C.byref(pages), table.data_ptr(), table.shape[1], _ptr(first), stream),
           "codecomp_pages_store")


def codecomp_pages_load(pages, table, first, idx, params, k, v) -> None:
    """idx None: all rows of the requests into k, v [L, H_kv, T, d]; else rows idx into k, v [L, H_kv, TB, d]."""
    total, strides = _side(params, idx is not None)
    _table(table, first, params)
    if idx is not None:
        _idx(idx, params)
    kp, vp = _rows(k, params, "k", total, strides), _rows(v, params, "v", total, strides)
    at = pages._at
    stream = _launch_stream(at, k.get_device(), v.get_device(), table.get_device(), _at(idx, at), _at(first, at))
    _check(lib().codecomp_pages_load(C.byref(pages), table.data_ptr(), table.shape[1], _ptr(first), _ptr(idx), C.byref(params), kp, vp, stream),
           "codecomp_pages_load")


def codecomp_pages_compact(pages, table, first, idx, params, to, to_table, to_first=None) -> None:
    _table(table, first, params)
    _table(to_table, to_first, params)
    _idx(idx, params)
    at = pages._at
    stream = _launch_stream(at, to._at, table.get_device(), to_table.get_device(), idx.get_device(), _at(first, at), _at(to_first, at))
    _check(lib().codecomp_pages_compact(C.byref(pages), table.data_ptr(), table.shape[1], _ptr(first), idx.data_ptr(), C.byref(params), C.byref(to),
                                        to_table.data_ptr(), to_table.shape[1], _ptr(to_first), stream), "codecomp_pages_compact")


def codecomp_pages_copy(pages, pairs) -> None:
    """pairs: device int32 [n, 2], (source page, target page)."""
    _int32(pairs, (pairs.shape[0], 2), "pairs")
    stream = _launch_stream(pages._at, pairs.get_device())
    _check(lib().codecomp_pages_copy(C.byref(pages), pairs.data_ptr(), pairs.shape[0], stream), "codecomp_pages_copy")


def codecomp_attend_workspace_bytes(batch, pages) -> int:
    _check(lib().codecomp_attend_validate(C.byref(batch), C.byref(pages)), "codecomp_attend_validate")
    return lib().codecomp_attend_workspace_bytes(C.byref(batch), C.byref(pages))


def codecomp_attend(q, batch: codecomp_batch, pages: codecomp_pages, layer: int, out, workspace, lse=None) -> None:
    torch = _torch_module or _torch()
    shape = (batch._tokens, batch.n_q_heads, pages.head_dim)
    qp, op = _vectors(q, "q", shape, batch.q_stride_tok, batch.q_stride_head), _vectors(out, "out", shape, batch.out_stride_tok, batch.out_stride_head)
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != shape[:2] or not lse.is_contiguous()):
        raise ValueError(f"lse must be a contiguous float32 tensor {shape[:2]}, not {lse.dtype} {tuple(lse.shape)}")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    at = pages._at
    stream = _launch_stream(at, batch._at, q.get_device(), out.get_device(), _at(lse, at), _at(workspace, at))
    size = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().codecomp_attend(qp, C.byref(batch), C.byref(pages), layer, op, _ptr(lse), _ptr(workspace), size, stream), "codecomp_attend")


class DeviceProblem:
    """Device buffers of one workload: inputs uploaded from the host arrays of the workload
    generator, outputs and workspace allocated with torch.  Plumbing only.  k_bits / v_bits of dtype
    uint8 are an FP8 E4M3 cache (kv_dtype = KV_FP8_E4M3), uint16 a bf16 one."""

    def __init__(self, w, q_bits: np.ndarray, k_bits: np.ndarray, v_bits: Optional[np.ndarray], prior: np.ndarray,
                 device: str = "cuda:0", select_mode: int = 0, span_budget_ratio: float = 0.5,
                 span_budget_min: int = 0, score_variant: int = 0, score_workgroups: int = 0, score_lead_tiles: int = 0):
        import torch
        self.w = w
        dev = torch.device(device)

        def up_bits(x):
            return torch.from_numpy(x.view(np.int16)).to(dev).view(torch.bfloat16)

        fp8 = k_bits.dtype == np.uint8
        if v_bits is not None and v_bits.dtype != k_bits.dtype:
            raise ValueError("k and v must have the same storage type")

        def up_kv(x):
            return torch.from_numpy(x).to(dev) if fp8 else up_bits(x)

        self.q = up_bits(q_bits)
        self.k = up_kv(k_bits)
        self.v = up_kv(v_bits) if v_bits is not None else None
        self.prior = torch.from_numpy(prior).to(dev)
        self.n_layers = int(k_bits.shape[0])
        self.cu_seqlens = torch.from_numpy(w.cu_seqlens()).to(dev)
        self.cu_budgets = torch.from_numpy(w.cu_budgets()).to(dev)
        self.params = make_params(n_layers=self.n_layers, n_q_heads=w.n_q_heads, n_kv_heads=w.n_kv_heads,
                                  head_dim=w.head_dim, window=w.window, pool_kernel=w.pool_kernel,
                                  prior_weight=w.prior_weight, cu_seqlens_host=w.cu_seqlens(),
                                  cu_budgets_host=w.cu_budgets(), cu_seqlens_dev=_ptr(self.cu_seqlens),
                                  cu_budgets_dev=_ptr(self.cu_budgets), select_mode=select_mode,
                                  span_budget_ratio=span_budget_ratio, span_budget_min=span_budget_min,
                                  score_variant=score_variant, kv_dtype=KV_FP8_E4M3 if fp8 else KV_BF16,
                                  score_workgroups=score_workgroups, score_lead_tiles=score_lead_tiles)
        rc = codecomp_validate(self.params)
        _check(rc, "codecomp_validate")
        T, TB = w.total_tokens, w.total_budget
        self.scores = torch.empty((self.n_layers, w.n_kv_heads, T), dtype=torch.float32, device=dev)
        self.idx = torch.empty((self.n_layers, w.n_kv_heads, TB), dtype=torch.int32, device=dev)
        self.k_out = torch.empty((self.n_layers, w.n_kv_heads, TB, w.head_dim),
                                 dtype=torch.uint8 if fp8 else torch.bfloat16, device=dev)
        self.v_out = torch.empty_like(self.k_out)
        self.workspace = torch.empty(max(256, codecomp_workspace_bytes(self.params)), dtype=torch.uint8, device=dev)

    def score(self):
        codecomp_score(self.q, self.k, self.prior, self.params, self.scores, self.workspace)

    def score_stages(self, stages: int):
        codecomp_score_stages(self.q, self.k, self.prior, self.params, self.scores, self.workspace, stages)

    def select(self):
        if self.params.select_mode == 1:
            codecomp_select_two_stage(self.scores, self.prior, self.params, self.idx, self.workspace)
        else:
            codecomp_select(self.scores, self.params, self.idx, self.workspace)

    def gather(self):
        codecomp_gather(self.k, self.v, self.idx, self.params, self.k_out, self.v_out)

    def compress(self):
        codecomp_compress(self.q, self.k, self.v, self.prior, self.params, self.scores, self.idx, self.k_out,
                          self.v_out, self.workspace)

    def compress_static(self):
        codecomp_compress_static(self.q, self.k, self.v, self.prior, self.params, self.scores, self.idx, self.k_out,
                                 self.v_out)

    @staticmethod
    def bits(t) -> np.ndarray:
        """bf16 tensor -> host uint16 bit patterns (a uint8 tensor of FP8 codes comes back as it is)."""
        import torch
        if t.dtype == torch.uint8:
            return t.cpu().numpy()
        return t.view(torch.int16).cpu().numpy().view(np.uint16)
