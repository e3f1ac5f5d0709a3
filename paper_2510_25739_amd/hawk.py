"""ctypes binding of libhawk.so: argument marshalling only, same call names as the C ABI."""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libhawk.so")
_lib = None

HAWK_FP32, HAWK_BF16, HAWK_FP16 = 0, 1, 2


class HawkError(RuntimeError):
    def __init__(self, code: int, where: str, text: str = ""):
        super().__init__(f"{where} failed with code {code}: {text}")
        self.code = code


class HawkConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_layers", "d_model", "n_heads", "d_mlp", "vocab", "samp_lo", "samp_n", "max_cond",
        "max_grid_h", "max_grid_w", "max_batch", "k_max", "dtype", "use_cfg")] + [
        ("rms_eps", C.c_float), ("rope_theta", C.c_float)]

    @classmethod
    def from_shape(cls, s, *, batch: Optional[int] = None, k_max: Optional[int] = None):
        """From a synth.HawkShape-like object (duck typed: only attributes are read)."""
        return cls(n_layers=s.n_layers, d_model=s.d_model, n_heads=s.n_heads, d_mlp=s.d_mlp, vocab=s.vocab,
                   samp_lo=s.samp_lo, samp_n=s.samp_n, max_cond=s.n_cond, max_grid_h=s.grid_h,
                   max_grid_w=s.grid_w, max_batch=s.batch if batch is None else batch,
                   k_max=s.k if k_max is None else k_max, dtype=HAWK_FP32 if s.dtype == "fp32" else HAWK_BF16,
                   use_cfg=int(s.cfg_scale != 1.0), rms_eps=s.rms_eps, rope_theta=s.rope_theta)


class HawkStats(C.Structure):
    _fields_ = [("steps", C.c_int64), ("accepted", C.c_int64), ("tokens", C.c_int64), ("iters", C.c_int64),
                ("ms_prefill", C.c_float), ("ms_decode", C.c_float)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class HawkPagedCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("page_stride", C.c_int64),
                ("head_stride", C.c_int64), ("entry_stride", C.c_int64), ("table", C.c_void_p), ("table_stride", C.c_int64)] + [
        (n, C.c_int32) for n in ("dtype", "n_layers", "n_pages", "page_size", "n_heads", "head_dim", "n_seq", "max_pages")]


class HawkPagedRows(C.Structure):
    _fields_ = [("row_start", C.c_void_p), ("n_past", C.c_void_p), ("rows", C.c_int32)]


class HawkHeads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("n_heads", C.c_int32),
                ("dtype", C.c_int32)]


class HawkAdapters(C.Structure):
    _fields_ = [("a", C.c_void_p), ("b", C.c_void_p)] + [(n, C.c_int64) for n in (
        "a_adapter_stride", "a_row_stride", "b_adapter_stride", "b_row_stride")] + [("scale", C.c_void_p)] + [
        (n, C.c_int32) for n in ("dtype", "n_adapters", "rank", "d_in", "d_out")]


class HawkMatrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("dtype", C.c_int32)]


EXPORTS = {
    "hawk_workspace_bytes": (C.c_size_t, [C.POINTER(HawkConfig)]),
    "hawk_plan_info": (C.c_int, [C.POINTER(HawkConfig), C.POINTER(C.c_int64)]),
    "hawk_create": (C.c_int, [C.POINTER(HawkConfig), C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_void_p)]),
    "hawk_destroy": (None, [C.c_void_p]),
    "hawk_last_error": (C.c_char_p, [C.c_void_p]),
    "hawk_load": (C.c_int, [C.c_void_p, C.c_void_p, C.c_size_t]),
    "hawk_prefill": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_float,
                               C.c_int, C.c_float, C.c_void_p]),
    "hawk_draft": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]),
    "hawk_draft_forced": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_int]),
    "hawk_verify": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hawk_generate": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                C.c_float, C.c_int, C.c_float, C.c_uint64, C.c_void_p, C.c_void_p,
                                C.POINTER(HawkStats)]),
    "hawk_run_steps": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_uint64, C.c_int, C.POINTER(C.c_float),
                                 C.POINTER(C.c_float), C.POINTER(C.c_float)]),
    "hawk_set_replay": (C.c_int, [C.c_void_p, C.c_void_p]),
    "hawk_get_stats": (C.c_int, [C.c_void_p, C.POINTER(HawkStats)]),
    "hawk_force": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int]),
    "hawk_get_n": (C.c_int, [C.c_void_p, C.c_void_p]),
    "hawk_get_grid": (C.c_int, [C.c_void_p, C.c_void_p]),
    "hawk_get_logits": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int]),
    "hawk_get_draft_logits": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int]),
    "hawk_set_path": (C.c_int, [C.c_void_p, C.c_int]),
    "hawk_last_path": (C.c_int, [C.c_void_p]),
    "hawk_last_kernel": (C.c_int, [C.c_void_p]),
    "hawk_debug_raise_timeout": (C.c_int, [C.c_void_p]),
    "hawk_phase_trace": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_size_t]),
    "hawk_tree_layout": (C.c_int, [C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hawk_verify_tree": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_void_p, C.c_void_p]),
    "hawk_get_tree_logits": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int]),
    "hawk_get_tree_path": (C.c_int, [C.c_void_p, C.c_void_p]),
    "hawk_last_hidden": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "hawk_multi_verify_workspace_bytes": (C.c_size_t, [C.c_int, C.c_int]),
    "hawk_multi_verify": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                    C.c_int, C.c_int, C.c_float, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_size_t, C.c_void_p]),
    "hawk_multi_verify_static": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_int, C.c_int, C.c_int, C.c_float, C.c_int, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_void_p]),
    "hawk_spatial_heads_workspace_bytes": (C.c_size_t, [C.c_int, C.c_int, C.c_int]),
    "hawk_spatial_heads": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hawk_spec_cache_bytes": (C.c_size_t, [C.c_int, C.c_int, C.c_int]),
    "hawk_spec_cache_slot": (C.c_int, [C.c_int, C.c_int, C.c_int, C.c_int]),
    "hawk_spec_cache_reset": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p]),
    "hawk_spec_cache_push": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                       C.c_size_t, C.c_int, C.c_void_p]),
    "hawk_spec_pool": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_size_t,
                                 C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hawk_sample_rows": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_float, C.c_int,
                                   C.c_void_p, C.c_void_p]),
    "hawk_rotary_table": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_double, C.c_void_p]),
    "hawk_paged_append": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_float, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hawk_paged_attention_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int, C.c_int, C.c_int]),
    "hawk_paged_attention": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_int, C.c_void_p,
                                       C.c_void_p, C.c_size_t, C.c_void_p]),
    "hawk_paged_keep": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]),
    "hawk_paged_entry": (C.c_int64, [C.c_void_p, C.c_void_p, C.c_int, C.c_int64]),
    "hawk_paged_pages_workspace_bytes": (C.c_size_t, [C.c_void_p]),
    "hawk_paged_fork": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]),
    "hawk_paged_take": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hawk_paged_trim": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hawk_paged_compact": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hawk_paged_copy": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]),
    "hawk_adapter_plan_bytes": (C.c_size_t, [C.c_int, C.c_int]),
    "hawk_adapter_plan": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hawk_adapter_apply_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int]),
    "hawk_adapter_apply": (C.c_int, [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hawk_sample_filtered_workspace_bytes": (C.c_size_t, [C.c_int, C.c_int]),
    "hawk_sample_filtered": (C.c_int, [C.c_void_p, C.c_int, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                       C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hawk_verify_chains_workspace_bytes": (C.c_size_t, [C.c_int, C.c_int, C.c_int]),
    "hawk_verify_chains": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_int, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_float, C.c_int,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hawk_generate_spatial_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int, C.c_int, C.c_int]),
    "hawk_generate_spatial": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_float, C.c_int, C.c_void_p,
                                        C.c_void_p, C.c_int, C.c_int, C.c_uint64, C.c_void_p, C.c_size_t, C.c_void_p,
                                        C.c_void_p]),
}


def lib_path() -> str:
    return _LIB_PATH


def load_library() -> C.CDLL:
    """Loads the built HIP library; never falls back to anything else."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise HawkError(-4, "load_library", f"{_LIB_PATH} is missing: run `python __graft_entry__.py` "
                                                "(or paper_2510_25739_amd/build.py) first")
        L = C.CDLL(_LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def workspace_bytes(cfg: HawkConfig) -> int:
    return int(load_library().hawk_workspace_bytes(C.byref(cfg)))


def plan_info(cfg: HawkConfig) -> dict:
    out = (C.c_int64 * 8)()
    rc = load_library().hawk_plan_info(C.byref(cfg), out)
    if rc != 0:
        raise HawkError(rc, "hawk_plan_info")
    keys = ("supported", "layer_tiles", "total_tiles", "min_wg_tiles", "max_wg_tiles", "lm_rounds", "tables_ok", "workgroups")
    return dict(zip(keys, [int(v) for v in out]))


def _f32(a):
    return np.ascontiguousarray(a, dtype=np.float32)


def _i32(a):
    return np.ascontiguousarray(a, dtype=np.int32)


def _p(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def multi_verify_workspace_bytes(rows: int, m: int) -> int:
    return int(load_library().hawk_multi_verify_workspace_bytes(rows, m))


def multi_verify(p_logits, q_logits, cand, u_acc, u_final, temperature: float, top_k: int, want_resid: bool = False,
                 workspace=None, m_rows=None):
    """hawk_multi_verify on device tensors (torch, on the GPU): p_logits [rows, n] fp32, q_logits
    [rows, m, n] fp32, cand [rows, m] int32, u_acc [rows, m] fp32, u_final [rows] fp32.
    workspace: None, or a device uint8 tensor of at least multi_verify_workspace_bytes(rows, m) bytes.
    m_rows: None, or a device int32 tensor [rows] with each position's own number of candidates.
    Returns device tensors (index [rows] int32, token [rows] int32[, residual masses [rows, m] fp64]);
    the launch is asynchronous on torch's current stream."""
    import torch  # device memory and stream only
    rows, m, n = q_logits.shape
    for t, shape, dt in ((p_logits, (rows, n), torch.float32), (q_logits, (rows, m, n), torch.float32),
                         (cand, (rows, m), torch.int32), (u_acc, (rows, m), torch.float32),
                         (u_final, (rows,), torch.float32)) + (
                                 ((m_rows, (rows,), torch.int32),) if m_rows is not None else ()):
        if not (t.is_cuda and t.is_contiguous() and t.dtype == dt and tuple(t.shape) == shape):
            raise HawkError(-1, "hawk_multi_verify", "arguments must be contiguous device tensors of the documented shapes")
    idx = torch.empty(rows, dtype=torch.int32, device=p_logits.device)
    tok = torch.empty(rows, dtype=torch.int32, device=p_logits.device)
    resid = torch.empty((rows, m), dtype=torch.float64, device=p_logits.device) if want_resid else None
    rc = load_library().hawk_multi_verify(p_logits.data_ptr(), q_logits.data_ptr(), cand.data_ptr(), u_acc.data_ptr(),
                                          u_final.data_ptr(), m_rows.data_ptr() if m_rows is not None else None,
                                          rows, m, n, float(temperature), int(top_k),
                                          idx.data_ptr(), tok.data_ptr(), resid.data_ptr() if want_resid else None,
                                          workspace.data_ptr() if workspace is not None else None,
                                          workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                          torch.cuda.current_stream(p_logits.device).cuda_stream)
    if rc != 0:
        raise HawkError(rc, "hawk_multi_verify")
    return (idx, tok, resid) if want_resid else (idx, tok)


def multi_verify_static(p_logits, q_logits, cand, u_acc, u_final, temperature: float, top_k: int, out_index, out_token,
                        out_resid=None, m_rows=None):
    """hawk_multi_verify_static: hawk_multi_verify without any allocation - the caller passes the output
    tensors too (out_index, out_token int32 [rows]; out_resid None or fp64 [rows, m]); the statistics go
    to the library's fixed device array.  At most 4096 logit rows (rows * (m + 1)) per call."""
    import torch  # stream handle only
    rows, m, n = q_logits.shape
    rc = load_library().hawk_multi_verify_static(p_logits.data_ptr(), q_logits.data_ptr(), cand.data_ptr(), u_acc.data_ptr(),
                                                 u_final.data_ptr(), m_rows.data_ptr() if m_rows is not None else None,
                                                 rows, m, n, float(temperature), int(top_k), out_index.data_ptr(),
                                                 out_token.data_ptr(), out_resid.data_ptr() if out_resid is not None else None,
                                                 torch.cuda.current_stream(p_logits.device).cuda_stream)
    if rc != 0:
        raise HawkError(rc, "hawk_multi_verify_static")


def tree_layout(m_depth):
    """hawk_tree_layout: (parent, depth, candidate, ancestors) arrays of the candidate tree's nodes."""
    md = _i32(m_depth)
    parent, depth, cand = (np.zeros(64, dtype=np.int32) for _ in range(3))
    anc = np.zeros(64, dtype=np.uint64)
    n = load_library().hawk_tree_layout(len(md), _p(md), _p(parent), _p(depth), _p(cand), _p(anc))
    if n < 0:
        raise HawkError(-1, "hawk_tree_layout", "bad tree shape")
    return parent[:n], depth[:n], cand[:n], anc[:n]


def _int32():
    import torch
    return torch.int32


def _int64():
    import torch
    return torch.int64


def _float32():
    import torch
    return torch.float32


def _empty_like():
    import torch  # device memory and stream only
    return torch.empty_like


def _uint8():
    import torch
    return torch.uint8


def _stream_of(t):
    import torch  # device memory and stream only
    return torch.cuda.current_stream(t.device).cuda_stream


def _dev_ok(t, dtype, shape=None):
    return t.is_cuda and t.is_contiguous() and t.dtype == dtype and (shape is None or tuple(t.shape) == tuple(shape))


def spatial_heads(h, W_heads, W_out, want_g: bool = False):
    """hawk_spatial_heads on device tensors: h [rows, d] fp32, W_heads [n_heads, d, d] bf16, W_out
    [V_s, d] bf16.  Returns q_logits [rows, n_heads, V_s] fp32 (and g [rows, n_heads, d] fp32)."""
    import torch  # device memory and stream only
    rows, d = h.shape
    n_heads, v_s = W_heads.shape[0], W_out.shape[0]
    if not (_dev_ok(h, torch.float32) and _dev_ok(W_heads, torch.bfloat16, (n_heads, d, d))
            and _dev_ok(W_out, torch.bfloat16, (v_s, d))):
        raise HawkError(-1, "hawk_spatial_heads", "arguments must be contiguous device tensors of the documented shapes")
    L = load_library()
    nws = int(L.hawk_spatial_heads_workspace_bytes(rows, n_heads, d))
    ws = torch.empty(max(nws, 16), dtype=torch.uint8, device=h.device)
    q = torch.empty((rows, n_heads, v_s), dtype=torch.float32, device=h.device)
    g = torch.empty((rows, n_heads, d), dtype=torch.float32, device=h.device) if want_g else None
    rc = L.hawk_spatial_heads(h.data_ptr(), W_heads.data_ptr(), W_out.data_ptr(), rows, n_heads, d, v_s, q.data_ptr(),
                              g.data_ptr() if want_g else None, ws.data_ptr(), nws, _stream_of(h))
    if rc != 0:
        raise HawkError(rc, "hawk_spatial_heads")
    return (q, g) if want_g else q


def spec_cache_bytes(IW: int, VSD: int, v_s: int) -> int:
    return int(load_library().hawk_spec_cache_bytes(IW, VSD, v_s))


def spec_cache_slot(IW: int, VSD: int, pos: int, depth: int) -> int:
    return int(load_library().hawk_spec_cache_slot(IW, VSD, pos, depth))


class SpecCache:
    """The speculation cache of one image in device memory (a torch uint8 tensor) and its calls."""

    def __init__(self, IW: int, IH: int, VSD: int, v_s: int, device: str = "cuda:0"):
        import torch  # device memory and stream only
        self._torch = torch
        self.IW, self.IH, self.VSD, self.v_s = IW, IH, VSD, v_s
        self._L = load_library()
        nbytes = spec_cache_bytes(IW, VSD, v_s)
        if nbytes == 0:
            raise HawkError(-1, "hawk_spec_cache_bytes", "invalid cache shape")
        self.mem = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.reset()

    def reset(self):
        rc = self._L.hawk_spec_cache_reset(self.mem.data_ptr(), self.IW, self.VSD, self.v_s, _stream_of(self.mem))
        if rc != 0:
            raise HawkError(rc, "hawk_spec_cache_reset")

    def push(self, pos, q_vert, row_stride: int):
        """pos [rows] int32; q_vert: a device fp32 tensor whose row r starts r * row_stride floats in."""
        torch = self._torch
        rows = pos.numel()
        if not (_dev_ok(pos, torch.int32) and q_vert.is_cuda and q_vert.dtype == torch.float32
                and q_vert.numel() >= (rows - 1) * row_stride + self.VSD * self.v_s):
            raise HawkError(-1, "hawk_spec_cache_push", "bad arguments")
        rc = self._L.hawk_spec_cache_push(self.mem.data_ptr(), self.IW, self.IH, self.VSD, self.v_s, pos.data_ptr(),
                                          q_vert.data_ptr(), row_stride, rows, _stream_of(self.mem))
        if rc != 0:
            raise HawkError(rc, "hawk_spec_cache_push")

    def pool(self, target, q_horiz, horiz_stride: int):
        """target [n] int32; q_horiz: device fp32 tensor, item i's horizontal logits i * horiz_stride
        floats in.  Returns pool_logits [n, VSD + 1, V_s], pool_m [n], pool_delta [n, VSD + 1]."""
        torch = self._torch
        n = target.numel()
        if not (_dev_ok(target, torch.int32) and q_horiz.is_cuda and q_horiz.dtype == torch.float32
                and q_horiz.numel() >= (n - 1) * horiz_stride + self.v_s):
            raise HawkError(-1, "hawk_spec_pool", "bad arguments")
        dev = self.mem.device
        logits = torch.empty((n, self.VSD + 1, self.v_s), dtype=torch.float32, device=dev)   # rows beyond the count stay unwritten
        m = torch.empty(n, dtype=torch.int32, device=dev)
        delta = torch.empty((n, self.VSD + 1), dtype=torch.int32, device=dev)
        rc = self._L.hawk_spec_pool(self.mem.data_ptr(), self.IW, self.IH, self.VSD, self.v_s, target.data_ptr(),
                                    q_horiz.data_ptr(), horiz_stride, n, logits.data_ptr(), m.data_ptr(),
                                    delta.data_ptr(), _stream_of(self.mem))
        if rc != 0:
            raise HawkError(rc, "hawk_spec_pool")
        return logits, m, delta


def sample_rows(logits, u, temperature: float, top_k: int, skip=None):
    """hawk_sample_rows on device tensors: logits [rows, n] fp32, u [rows] fp32, skip None or [rows] int32."""
    import torch  # device memory and stream only
    rows, n = logits.shape
    if not (_dev_ok(logits, torch.float32) and _dev_ok(u, torch.float32, (rows,))
            and (skip is None or _dev_ok(skip, torch.int32, (rows,)))):
        raise HawkError(-1, "hawk_sample_rows", "arguments must be contiguous device tensors of the documented shapes")
    out = torch.empty(rows, dtype=torch.int32, device=logits.device)
    rc = load_library().hawk_sample_rows(logits.data_ptr(), skip.data_ptr() if skip is not None else None, u.data_ptr(),
                                         rows, n, float(temperature), int(top_k), out.data_ptr(), _stream_of(logits))
    if rc != 0:
        raise HawkError(rc, "hawk_sample_rows")
    return out

_DTYPES = None   # torch dtype -> HAWK_*
_PACK_HEADS = struct.Struct("@Pqqii").pack     # HawkHeads, HawkPagedRows as bytes: a third of a structure object's cost
_PACK_ROWS = struct.Struct("@PPi4x").pack
_PACK_ADAPTERS = struct.Struct("@PPqqqqP5i4x").pack
_PACK_MATRIX = struct.Struct("@Pqi4x").pack


def _dtype_of(t):
    global _DTYPES
    if _DTYPES is None:
        import torch
        _DTYPES = {torch.float32: HAWK_FP32, torch.bfloat16: HAWK_BF16, torch.float16: HAWK_FP16}
    return _DTYPES.get(t.dtype, -1)


_torch = None


def _call_on(index, fn, *args):
    """fn(*args, stream) with device `index` current - launches go to the current device, whatever stream they are given - on
    torch's current stream of that device."""
    global _torch
    if _torch is None:
        import torch  # device memory and stream only
        _torch = torch
    stream = _torch._C._cuda_getCurrentRawStream(index)
    if _torch._C._cuda_getDevice() == index:
        return fn(*args, stream)
    with _torch.cuda.device(index):
        return fn(*args, stream)


def _call_at(index, stream, fn, *args):
    """_call_on where torch's current stream of device `index` is known already (_raw_stream)."""
    if _torch._C._cuda_getDevice() == index:
        return fn(*args, stream)
    with _torch.cuda.device(index):
        return fn(*args, stream)


def _raw_stream():
    global _torch
    import torch  # device memory and stream only
    _torch = torch
    return torch._C._cuda_getCurrentRawStream


def rotary_table(n_pos: int, rot_dim: int, theta: float = 10000.0, device: str = "cuda:0"):
    """hawk_rotary_table: fp32 device tensor [n_pos, rot_dim // 2, 2] of cos and sin of position * theta^(-2 j / rot_dim)."""
    import torch  # device memory and stream only
    out = torch.empty((max(n_pos, 0), max(rot_dim, 0) // 2, 2), dtype=torch.float32, device=device)
    if not out.is_cuda:
        raise HawkError(-1, "hawk_rotary_table", "the table is a device tensor")
    rc = _call_on(out.get_device(), load_library().hawk_rotary_table, out.data_ptr(), n_pos, rot_dim, float(theta))
    if rc != 0:
        raise HawkError(rc, "hawk_rotary_table")
    return out


class PagedCache:
    """Keys and values of many sequences in pages (hawk_paged_cache) and the calls on them.

    k, v: device tensors [n_layers, n_pages, n_heads, page_size, head_dim] (or without the first axis) of the same strides,
    fp32, bf16 or fp16, the last axis contiguous - any other order of the axes is a permuted view.  table [n_seq, max_pages]
    int32: the pages of every sequence.  The tensors stay the caller's: their contents may change between calls (new pages
    in the table), and `table` may be replaced by another tensor (a captured graph goes on reading the one it was captured with,
    which the caller then keeps).
    Calls launch on torch's current stream of the cache's device.  `row_start` [n_seq + 1] and `n_past` [n_seq] are int32 device
    tensors: rows row_start[s] .. row_start[s + 1] - 1 of a call belong to sequence s, which has n_past[s] committed entries."""

    def __init__(self, k, v, table):
        if k.dim() == 4:
            k, v = k.unsqueeze(0), v.unsqueeze(0)
        if not (k.is_cuda and v.device == k.device and k.dim() == 5 and v.shape == k.shape and v.dtype == k.dtype
                and _dtype_of(k) >= 0 and k.stride() == v.stride() and k.stride(4) == 1):
            raise HawkError(-1, "PagedCache", "k and v must be device tensors [layers, pages, heads, page_size, head_dim] of one type and one layout")
        self._L = load_library()
        self.k, self.v = k, v
        self.device = k.device
        n_layers, n_pages, n_heads, page_size, head_dim = k.shape
        sl, sp, sh, se, _ = k.stride()
        # the stride of an axis of one is not used
        sp, sh, se = (st if n > 1 else max(st, head_dim) for st, n in ((sp, n_pages), (sh, n_heads), (se, page_size)))
        self._c = HawkPagedCache(k=k.data_ptr(), v=v.data_ptr(), layer_stride=sl if n_layers > 1 else 0, page_stride=(sp + 7) // 8 * 8 if n_pages == 1 else sp,
                                 head_stride=(sh + 7) // 8 * 8 if n_heads == 1 else sh,
                                 entry_stride=(se + 7) // 8 * 8 if page_size == 1 else se, dtype=_dtype_of(k), n_layers=n_layers,
                                 n_pages=n_pages, page_size=page_size, n_heads=n_heads, head_dim=head_dim)
        self._ref = C.byref(self._c)
        self._dev, self._hd, self._kv = k.get_device(), head_dim, n_heads
        self._dtype, self._f32, self._i32, self._i64 = k.dtype, _float32(), _int32(), _int64()
        self._room = {}     # workspace of an attention by (rows, q heads, max_len)
        self._refs_shape = (n_pages,)
        self._like = _empty_like()
        self.table = table

    @property
    def table(self):
        return self._table

    @table.setter
    def table(self, t):
        if not (_dev_ok(t, _int32()) and t.dim() == 2 and t.device == self.device):
            raise HawkError(-1, "PagedCache", "table must be a contiguous int32 tensor [n_seq, max_pages] on the cache's device")
        self._table = t
        self._c.table, self._c.table_stride = t.data_ptr(), max(t.shape[1], 1)
        self._c.n_seq, self._c.max_pages = t.shape
        self._n_seq = t.shape[0]
        self._past_shape, self._start_shape = (self._n_seq,), (self._n_seq + 1,)
        self._room.clear()
        self._pages_room = None

    def _rows(self, where, rows, row_start, n_past):
        i32, dev = self._i32, self._dev
        if not (row_start.dtype is i32 and n_past.dtype is i32 and row_start.get_device() == dev and n_past.get_device() == dev
                and row_start.shape == self._start_shape and n_past.shape == self._past_shape and row_start.is_contiguous() and n_past.is_contiguous()):
            raise HawkError(-1, where, "row_start [n_seq + 1] and n_past [n_seq] must be contiguous int32 tensors on the cache's device")
        return _PACK_ROWS(row_start.data_ptr(), n_past.data_ptr(), rows)

    def _heads(self, where, t, rows=None, heads=None):
        """HawkHeads of a tensor [rows, heads, head_dim] (strides of axes of one are not used), its rows and heads."""
        if t.dim() == 3 and t.get_device() == self._dev:
            r, h, d = t.shape
            rs, hs, es = t.stride()
            if d == self._hd and (es == 1 or r == 0) and h > 0 and (rows is None or r == rows) and (heads is None or h == heads):
                return _PACK_HEADS(t.data_ptr(), rs if r > 1 else h * d, hs if h > 1 else d, h, _DTYPES.get(t.dtype, -1)), r, h
        raise HawkError(-1, where, "vectors must be tensors [rows, heads, head_dim] on the cache's device, the last axis contiguous, of the same rows "
                                   "(keys and values: of the cache's heads; results: of the queries')")

    def _result(self, like, rows, heads, dtype):
        """A new tensor [rows, heads, head_dim] and its HawkHeads."""
        t = like.new_empty((rows, heads, self._hd), dtype=dtype)
        return t, _PACK_HEADS(t.data_ptr(), heads * self._hd, self._hd, heads, _DTYPES[dtype])

    def _fits(self, where, what, t, dtype, shape):
        if not (t.dtype is dtype and t.get_device() == self._dev and t.shape == shape and t.is_contiguous()):
            raise HawkError(-1, where, what)

    def append(self, k, v, row_start, n_past, q=None, rot=None, halves: bool = False, pos=None, q_gain=None, k_gain=None,
               eps: float = 1e-5, q_out=None, layer: int = 0):
        """hawk_paged_append: k, v [rows, n_heads, head_dim] become entries of layer `layer`, q [rows, q heads, head_dim] (or None)
        comes back normalised and rotated in the cache's type (q_out: where, q itself allowed; None: a new tensor, whose
        rows of no sequence are not written).  rot: a table [n_pos, rot_dim // 2, 2] (rotary_table) or None;
        halves: pairs (j, j + rot_dim / 2) instead of (2 j, 2 j + 1); pos [rows] int32: positions other than the entries' own;
        q_gain, k_gain [head_dim] fp32: RMS norm per head with eps."""
        where = "hawk_paged_append"
        hk, rows, _ = self._heads(where, k, None, self._kv)
        hv, _, _ = self._heads(where, v, rows, self._kv)
        r = self._rows(where, rows, row_start, n_past)
        hq = ho = None
        if q is not None:
            hq, _, n_heads = self._heads(where, q, rows)
            if q_out is None:
                q_out, ho = self._result(q, rows, n_heads, self._dtype)
            else:
                ho, _, _ = self._heads(where, q_out, rows, n_heads)
        elif q_out is not None:
            raise HawkError(-1, where, "q_out without q")
        gq = gk = table = at = None
        n_pos = rot_dim = 0
        if q_gain is not None:
            self._fits(where, "gains must be fp32 tensors [head_dim] on the cache's device", q_gain, self._f32, (self._hd,))
            gq = q_gain.data_ptr()
        if k_gain is not None:
            self._fits(where, "gains must be fp32 tensors [head_dim] on the cache's device", k_gain, self._f32, (self._hd,))
            gk = k_gain.data_ptr()
        if rot is not None:
            if rot.dim() != 3:
                raise HawkError(-1, where, "rot must be a tensor [n_pos, rot_dim / 2, 2]")
            n_pos, half, _ = rot.shape
            rot_dim = 2 * half
            self._fits(where, "rot must be a contiguous fp32 tensor [n_pos, rot_dim / 2, 2] on the cache's device", rot, self._f32, (n_pos, half, 2))
            table = rot.data_ptr()
        if pos is not None:
            self._fits(where, "pos must be a contiguous int32 tensor [rows] on the cache's device", pos, self._i32, (rows,))
            at = pos.data_ptr()
        rc = _call_on(self._dev, self._L.hawk_paged_append, self._ref, layer, r, hq, hk, hv, gq, gk, eps, table, n_pos, rot_dim, 1 if halves else 0,
                      at, ho)
        if rc != 0:
            raise HawkError(rc, where)
        return q_out

    def attend(self, q, row_start, n_past, max_len: int = 0, scale: Optional[float] = None, tree=None, out=None, layer: int = 0):
        """hawk_paged_attention: q [rows, q heads, head_dim] of the cache's type, the step's entries appended already.  max_len: the
        longest n_past + rows of a sequence, if the caller knows it (it chooses the kernel, nothing else).  scale None:
        1 / sqrt(head_dim).  tree [rows] int64: which of the first 64 rows of its sequence a row sees besides itself
        (hawk_tree_layout's ancestors); None: those up to itself.  out: where the result goes, any of the three types (None: a new tensor of
        q's type, whose rows of no sequence are not written)."""
        where = "hawk_paged_attention"
        hq, rows, heads = self._heads(where, q)
        r = self._rows(where, rows, row_start, n_past)
        if out is None:
            out, ho = self._result(q, rows, heads, self._dtype)
        else:
            ho, _, _ = self._heads(where, out, rows, heads)
        bits = None
        if tree is not None:
            self._fits(where, "tree must be a contiguous int64 tensor [rows] on the cache's device", tree, self._i64, (rows,))
            bits = tree.data_ptr()
        key = (rows, heads, max_len)
        nws = self._room.get(key)
        if nws is None:
            if len(self._room) > 4096:
                self._room.clear()
            nws = self._room[key] = self._L.hawk_paged_attention_workspace_bytes(self._ref, rows, heads, max_len)
        ws = q.new_empty((nws,), dtype=_uint8()) if nws else None
        rc = _call_on(self._dev, self._L.hawk_paged_attention, self._ref, layer, r, hq, bits, scale if scale is not None else self._hd ** -0.5, max_len,
                      ho, ws.data_ptr() if nws else None, nws)
        if rc != 0:
            raise HawkError(rc, where)
        return out

    def keep(self, n_past, path, n_keep):
        """hawk_paged_keep: the accepted path of a tree step, path [n_seq, depth] int32 of node numbers of which the first n_keep
        [n_seq] count, goes to the entries behind n_past's, in every layer."""
        where, i32, n = "hawk_paged_keep", self._i32, self._n_seq
        what = "path [n_seq, depth], n_past and n_keep [n_seq] must be contiguous int32 tensors on the cache's device"
        self._fits(where, what, n_past, i32, (n,))
        self._fits(where, what, n_keep, i32, (n,))
        depth = path.shape[1] if path.dim() == 2 else 0
        self._fits(where, what, path, i32, (n, depth))
        rc = _call_on(self._dev, self._L.hawk_paged_keep, self._ref, n_past.data_ptr(), path.data_ptr(), n_keep.data_ptr(), depth)
        if rc != 0:
            raise HawkError(rc, where)

    def _refs(self, where, refs):
        self._fits(where, "refs must be a contiguous int32 tensor [n_pages] on the cache's device", refs, self._i32, self._refs_shape)
        return refs.data_ptr()

    def _pages_workspace(self, like):
        """Workspace of a take or compact, from an int32 tensor's memory, and its bytes."""
        n = self._pages_room
        if n is None:
            n = self._pages_room = max(self._L.hawk_paged_pages_workspace_bytes(self._ref), 16)
        return like.new_empty((n // 4,)), n

    def fork(self, refs, n_past, src, dst):
        """hawk_paged_fork: sequences dst [n] int32 share from now on the pages of the entries that sequences src [n] have committed; the
        table, refs [n_pages] and n_past [n_seq] change in place."""
        where, i32, dev, shape = "hawk_paged_fork", self._i32, self._dev, src.shape
        if not (src.dtype is i32 and dst.dtype is i32 and n_past.dtype is i32 and src.get_device() == dev and dst.get_device() == dev
                and n_past.get_device() == dev and len(shape) == 1 and dst.shape == shape and n_past.shape == self._past_shape
                and src.is_contiguous() and dst.is_contiguous() and n_past.is_contiguous()):
            raise HawkError(-1, where, "src and dst must be contiguous int32 tensors [n], n_past [n_seq], on the cache's device")
        rc = _call_on(dev, self._L.hawk_paged_fork, self._ref, self._refs(where, refs), n_past.data_ptr(), src.data_ptr(), dst.data_ptr(), shape[0])
        if rc != 0:
            raise HawkError(rc, where)

    def take(self, refs, n_past, n_new, short_by=None):
        """hawk_paged_take: pages for the next n_new [n_seq] int32 entries of every sequence, shared ones copied first; the table and refs change
        in place.  Returns short_by [n_seq] int32: 0, or how many pages a sequence needs that was left as it was because there were too few."""
        where, i32, dev, shape = "hawk_paged_take", self._i32, self._dev, self._past_shape
        what = "n_past, n_new and short_by must be contiguous int32 tensors [n_seq] on the cache's device"
        if not (n_past.dtype is i32 and n_new.dtype is i32 and n_past.get_device() == dev and n_new.get_device() == dev and n_past.shape == shape
                and n_new.shape == shape and n_past.is_contiguous() and n_new.is_contiguous()):
            raise HawkError(-1, where, what)
        if short_by is None:
            short_by = self._like(n_past)
        else:
            self._fits(where, what, short_by, i32, shape)
        at = self._refs(where, refs)
        ws, n = self._pages_workspace(n_past)
        rc = _call_on(dev, self._L.hawk_paged_take, self._ref, at, n_past.data_ptr(), n_new.data_ptr(), short_by.data_ptr(), ws.data_ptr(), n)
        if rc != 0:
            raise HawkError(rc, where)
        return short_by

    def trim(self, refs, n_past):
        """hawk_paged_trim: the pages behind every sequence's first n_past entries are free again (as far as nobody else holds them); the table
        and refs change in place."""
        where = "hawk_paged_trim"
        self._fits(where, "n_past must be a contiguous int32 tensor [n_seq] on the cache's device", n_past, self._i32, self._past_shape)
        rc = _call_on(self._dev, self._L.hawk_paged_trim, self._ref, self._refs(where, refs), n_past.data_ptr())
        if rc != 0:
            raise HawkError(rc, where)

    def compact(self, refs, table=None, refs_out=None, n_used=None):
        """hawk_paged_compact: the pages in use move to the front of the pool.  Returns (table, refs, n_used): the table and the counts as they
        are then and the number of pages in use [1], int32 device tensors (new ones, or those given: table [n_seq, max_pages], the cache's own
        or another, refs_out [n_pages], refs itself or another).  The cache goes on with the new table once it is set: cache.table = table."""
        where, i32 = "hawk_paged_compact", self._i32
        ptr = self._refs(where, refs)
        if table is None:
            table = refs.new_empty(self._table.shape)
        else:
            self._fits(where, "table must be a contiguous int32 tensor [n_seq, max_pages] on the cache's device", table, i32, self._table.shape)
        if refs_out is None:
            refs_out = refs.new_empty(refs.shape)
        if n_used is None:
            n_used = refs.new_empty((1,))
        else:
            self._fits(where, "n_used must be an int32 tensor [1] on the cache's device", n_used, i32, (1,))
        to = self._refs(where, refs_out)
        ws, n = self._pages_workspace(refs)
        rc = _call_on(self._dev, self._L.hawk_paged_compact, self._ref, ptr, table.data_ptr(), self._c.table_stride, to, n_used.data_ptr(), ws.data_ptr(), n)
        if rc != 0:
            raise HawkError(rc, where)
        return table, refs_out, n_used

    def copy_pages(self, src, dst, to=None):
        """hawk_paged_copy: pages src [n] int32, all layers, go to pages dst [n] of the cache `to` (None: this one), which has the same shape."""
        where, i32 = "hawk_paged_copy", self._i32
        to = self if to is None else to
        what = "src and dst must be contiguous int32 tensors [n], and both pools on one device"
        n = src.shape[0] if src.dim() == 1 else -1
        self._fits(where, what, src, i32, (n,))
        self._fits(where, what, dst, i32, (n,))
        if to._dev != self._dev:
            raise HawkError(-1, where, what)
        rc = _call_on(self._dev, self._L.hawk_paged_copy, self._ref, to._ref, src.data_ptr(), dst.data_ptr(), n)
        if rc != 0:
            raise HawkError(rc, where)

    def entry(self, table_row, e: int, layer: int = 0) -> int:
        """hawk_paged_entry: elements from k's (v's) start to entry e, head 0, of a sequence with the pages table_row (host); -1: none."""
        t = _i32(table_row)
        if t.shape != (self._c.max_pages,):
            raise HawkError(-1, "hawk_paged_entry", "table_row must have max_pages entries")
        return int(self._L.hawk_paged_entry(self._ref, _p(t), layer, e))


class AdapterPlan:
    """Which rows of a step have which low-rank adapter (hawk_adapter_plan): rows row_start[s] .. row_start[s + 1] - 1 of sequence s,
    adapter[s] (-1: none), int32 device tensors [n_seq + 1] and [n_seq].  Made once a step and used for every projection of every layer
    (apply), on any stream that waits for the one it was made on; update lays out another step of as many rows and adapters in the same
    memory, in a captured graph as well."""

    def __init__(self, row_start, adapter, rows: int, n_adapters: int):
        self._L = load_library()
        self.rows, self.n_adapters = int(rows), int(n_adapters)
        n = self._L.hawk_adapter_plan_bytes(self.rows, self.n_adapters)
        if n == 0:
            raise HawkError(-1, "hawk_adapter_plan_bytes", "rows or n_adapters out of range")
        self._dev, self._i32, self._f32 = row_start.get_device(), _int32(), _float32()
        self._plan = row_start.new_empty((n,), dtype=_uint8())
        self._now, self._apply = _raw_stream(), self._L.hawk_adapter_apply
        self._streams = {self._now(self._dev) if self._dev >= 0 else 0}
        self._ptr, self._n = self._plan.data_ptr(), n
        self._room = {}     # workspace of an apply by (rank, d_in, d_out, type)
        self._like = _empty_like()
        self.update(row_start, adapter)

    def _note_stream(self, stream):
        """The plan's memory belongs to the stream it was made on; another one that works with it is noted, so that the memory is not given to
        others before that work is done, whenever the plan is dropped."""
        self._plan.record_stream(_torch.cuda.current_stream(self._dev))
        self._streams.add(stream)

    def update(self, row_start, adapter):
        where, n = "hawk_adapter_plan", adapter.shape[0] if adapter.dim() == 1 else -1
        for t, shape in ((row_start, (n + 1,)), (adapter, (n,))):
            if self._dev < 0 or t.dtype is not self._i32 or t.get_device() != self._dev or t.shape != shape or not t.is_contiguous():
                raise HawkError(-1, where, "row_start [n_seq + 1] and adapter [n_seq] must be contiguous int32 tensors on one device")
        stream = self._now(self._dev)
        if stream not in self._streams:
            self._note_stream(stream)
        rc = _call_at(self._dev, stream, self._L.hawk_adapter_plan, row_start.data_ptr(), adapter.data_ptr(), n, self.rows, self.n_adapters, self._ptr, self._n)
        if rc != 0:
            raise HawkError(rc, where)

    def _matrix(self, what, t, width):
        st = t.stride()
        if t.get_device() != self._dev or t.shape != (self.rows, width) or (st[1] != 1 and self.rows):
            raise HawkError(-1, "hawk_adapter_apply", f"{what} must be a tensor [rows, {width}] on the plan's device, the last axis contiguous")
        return _PACK_MATRIX(t.data_ptr(), st[0] if self.rows > 1 else (width + 7) // 8 * 8, _DTYPES.get(t.dtype, -1))

    def apply(self, x, a, b, base=None, scale=None, out=None, dtype=None):
        """hawk_adapter_apply: base + scale[i] * B_i (A_i x) of every row, i its adapter.  x [rows, d_in], a [n_adapters, rank, d_in],
        b [n_adapters, d_out, rank] of one type; base [rows, d_out] (None: zero) and out of one type; scale [n_adapters] fp32 (None: 1).
        out: where the result goes, base itself allowed, nothing that lies over x or over part of base (None: a new tensor of base's
        type, or of `dtype`, or of x's, whose rows of no sequence are not written)."""
        where, dev, n = "hawk_adapter_apply", self._dev, self.n_adapters
        if a.dim() != 3 or b.dim() != 3 or a.get_device() != dev or b.get_device() != dev or a.dtype is not b.dtype:
            raise HawkError(-1, where, "a [n_adapters, rank, d_in] and b [n_adapters, d_out, rank] must be tensors of one type on the plan's device")
        na, rank, d_in = a.shape
        nb, d_out, rank_b = b.shape
        (sa, ja, ia), (sb, jb, ib) = a.stride(), b.stride()
        if na != n or nb != n or rank_b != rank or ((ia != 1 or ib != 1) and n):
            raise HawkError(-1, where, "a [n_adapters, rank, d_in] and b [n_adapters, d_out, rank] must have the plan's adapters and last axes that are contiguous")
        s = 0
        if scale is not None:
            if scale.dtype is not self._f32 or scale.get_device() != dev or scale.shape != (n,) or not scale.is_contiguous():
                raise HawkError(-1, where, "scale must be a contiguous fp32 tensor [n_adapters] on the plan's device")
            s = scale.data_ptr()
        kind = _dtype_of(a)
        hx = self._matrix("x", x, d_in)
        hb = self._matrix("base", base, d_out) if base is not None else None
        if out is None:
            if dtype is None and base is not None and base.is_contiguous():
                out = self._like(base)               # (0.3 us less than new_empty)
            else:
                out = x.new_empty((self.rows, d_out), dtype=dtype if dtype is not None else (base.dtype if base is not None else x.dtype))
            ho = _PACK_MATRIX(out.data_ptr(), d_out, _DTYPES.get(out.dtype, -1))
        else:
            ho = self._matrix("out", out, d_out)
        w = _PACK_ADAPTERS(a.data_ptr(), b.data_ptr(), sa if n > 1 else 0, ja, sb if n > 1 else 0, jb, s, kind, n, rank, d_in, d_out)
        key = (rank, d_in, d_out, kind)                  # (all that the size is made of: it is 0 where they are refused)
        nws = self._room.get(key)
        if nws is None:
            nws = self._room[key] = self._L.hawk_adapter_apply_workspace_bytes(w, self.rows)
        ws = x.new_empty((nws,), dtype=_uint8()) if nws else None
        stream = self._now(dev)
        if stream not in self._streams:
            self._note_stream(stream)
        rc = _call_at(dev, stream, self._apply, w, self._ptr, self._n, self.rows, hx, hb, ho, ws.data_ptr() if nws else None, nws)
        if rc != 0:
            raise HawkError(rc, where)
        return out


_FILTER_ROOM = {}    # workspace of sample_filtered by (rows, n)


def sample_filtered(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, skip=None):
    """hawk_sample_filtered on device tensors: one draw a row of logits [rows, n] (any of the three types, rows may be strided) with u [rows] fp32,
    each row with parameters of its own: temperature, top_p, min_p [rows] fp32, top_k [rows] int32 (None: 1, 1, 0, all); skip [rows] int32:
    rows with a negative entry are not read.  Returns device tensors (token int32, probability fp32, entries kept int32), each [rows]."""
    where = "hawk_sample_filtered"
    dev = logits.get_device()
    if dev < 0 or logits.dim() != 2 or _dtype_of(logits) < 0:
        raise HawkError(-1, where, "logits must be a device tensor [rows, n] of fp32, bf16 or fp16")
    rows, n = logits.shape
    row, each = logits.stride()
    if each != 1 and n > 1:
        raise HawkError(-1, where, "the last axis of logits must be contiguous")
    f32, i32 = _float32(), _int32()
    ptr = []
    for t, dt in ((skip, i32), (u, f32), (temperature, f32), (top_k, i32), (top_p, f32), (min_p, f32)):
        if t is None:
            ptr.append(None)
        elif t.dtype is dt and t.get_device() == dev and t.shape == (rows,) and t.is_contiguous():
            ptr.append(t.data_ptr())
        else:
            raise HawkError(-1, where, "u, temperature, top_p, min_p (fp32) and top_k, skip (int32) must be contiguous tensors [rows] on the logits' device")
    L = load_library()
    nws = _FILTER_ROOM.get((rows, n))
    if nws is None:
        if len(_FILTER_ROOM) > 4096:
            _FILTER_ROOM.clear()
        nws = _FILTER_ROOM[rows, n] = L.hawk_sample_filtered_workspace_bytes(rows, n)
    ws = logits.new_empty((nws,), dtype=_uint8()) if nws else None
    token, kept, prob = logits.new_empty((rows,), dtype=i32), logits.new_empty((rows,), dtype=i32), logits.new_empty((rows,), dtype=f32)
    rc = _call_on(dev, L.hawk_sample_filtered, logits.data_ptr(), _dtype_of(logits), row if rows > 1 else n, *ptr, rows, n, token.data_ptr(),
                  prob.data_ptr(), kept.data_ptr(), ws.data_ptr() if nws else None, nws)
    if rc != 0:
        raise HawkError(rc, where)
    return token, prob, kept


_CHAIN_ROOM = {}     # workspace of verify_chains by (n_seq, k, n)


def verify_chains(p_logits, q_logits, draft, u_acc, u_final, temperature: float, top_k: int, n_draft=None, p_start=None):
    """hawk_verify_chains on device tensors: p_logits fp32 [p_rows, n] (rows may be strided), the k + 1 target rows of sequence s
    from row p_start[s] (int32 [n_seq]; None: s * (k + 1)); q_logits fp32 [n_seq, k, n] (strided) or None (the drafts are
    certain); draft [n_seq, k] int32; u_acc [n_seq, k], u_final [n_seq] fp32; n_draft None or int32 [n_seq].
    Returns device tensors (accepted [n_seq], tokens [n_seq, k + 1]) int32."""
    where, f32, i32 = "hawk_verify_chains", _float32(), _int32()
    dev = p_logits.get_device()
    n_seq, k = draft.shape if draft.dim() == 2 else (-1, -1)
    small = [(draft, i32, (n_seq, k)), (u_acc, f32, (n_seq, k)), (u_final, f32, (n_seq,))]
    if n_draft is not None:
        small.append((n_draft, i32, (n_seq,)))
    if p_start is not None:
        small.append((p_start, i32, (n_seq,)))
    if dev < 0 or p_logits.dim() != 2 or p_logits.dtype is not f32 or any(
            t.dtype is not dt or t.get_device() != dev or t.shape != shape or not t.is_contiguous() for t, dt, shape in small):
        raise HawkError(-1, where, "arguments must be device tensors of the documented shapes and types")
    p_rows, n = p_logits.shape
    ps, es = p_logits.stride()
    if es != 1 and n > 1:
        raise HawkError(-1, where, "the last axis of p_logits must be contiguous")
    q, qs, qr = None, 0, n
    if q_logits is not None:
        if q_logits.dtype is not f32 or q_logits.get_device() != dev or q_logits.shape != (n_seq, k, n) or (q_logits.stride(2) != 1 and n > 1):
            raise HawkError(-1, where, "q_logits must be a device fp32 tensor [n_seq, k, n], the last axis contiguous")
        q, qs, qr = q_logits.data_ptr(), q_logits.stride(0) if n_seq > 1 else 0, q_logits.stride(1) if k > 1 else n
    if p_start is None and p_rows < n_seq * (k + 1):
        raise HawkError(-1, where, "p_logits has fewer rows than n_seq * (k + 1)")
    L = load_library()
    nws = _CHAIN_ROOM.get((n_seq, k, n))
    if nws is None:
        if len(_CHAIN_ROOM) > 4096:
            _CHAIN_ROOM.clear()
        nws = _CHAIN_ROOM[n_seq, k, n] = L.hawk_verify_chains_workspace_bytes(n_seq, k, n)
    ws = p_logits.new_empty((max(nws, 16),), dtype=_uint8())
    count, toks = draft.new_empty((n_seq,)), draft.new_empty((n_seq, k + 1))
    rc = _call_on(dev, L.hawk_verify_chains, p_logits.data_ptr(), ps if p_rows > 1 else n, p_start.data_ptr() if p_start is not None else None, p_rows,
                  q, qs, qr, draft.data_ptr(), n_draft.data_ptr() if n_draft is not None else None, u_acc.data_ptr(), u_final.data_ptr(),
                  n_seq, k, n, temperature, top_k, count.data_ptr(), toks.data_ptr(), ws.data_ptr(), nws)
    if rc != 0:
        raise HawkError(rc, where)
    return count, toks


class Hawk:
    """One context: device workspace (a torch uint8 tensor) + the C handle."""

    def __init__(self, cfg: HawkConfig, device: str = "cuda:0", stream=None):
        import torch  # device memory and stream only
        self._L = load_library()
        self.cfg = cfg
        nbytes = workspace_bytes(cfg)
        if nbytes == 0:
            raise HawkError(-1, "hawk_workspace_bytes", "invalid configuration")
        if not torch.cuda.is_available():
            raise HawkError(-4, "Hawk", "no GPU visible: the HIP path has no CPU fallback")
        self._torch = torch
        self._dev = torch.device(device)
        with torch.cuda.device(self._dev):
            self._ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=self._dev)
            self._stream = stream if stream is not None else torch.cuda.current_stream(self._dev)
        base = self._ws.data_ptr()
        self._ws_ptr = (base + 255) & ~255
        h = C.c_void_p()
        rc = self._L.hawk_create(C.byref(cfg), C.c_void_p(self._ws_ptr), nbytes, C.c_void_p(self._stream.cuda_stream),
                                 C.byref(h))
        if rc != 0:
            raise HawkError(rc, "hawk_create")
        self._h = h
        self.v_s = cfg.samp_n if cfg.samp_n else cfg.vocab
        self.batch = 0
        self.n_img = 0

    # -- plumbing
    def _chk(self, rc, where):
        if rc != 0:
            raise HawkError(rc, where, self._L.hawk_last_error(self._h).decode())

    def close(self):
        if getattr(self, "_h", None):
            self._L.hawk_destroy(self._h)
            self._h = None
            self._ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def stream_handle(self) -> int:
        return int(self._stream.cuda_stream)

    # -- the C calls
    def set_path(self, path: int):
        self._chk(self._L.hawk_set_path(self._h, path), "hawk_set_path")

    def last_path(self) -> int:
        return int(self._L.hawk_last_path(self._h))

    def last_kernel(self) -> int:
        """0: one kernel per operation, 1: grid-barrier persistent kernel, 2: the kernel laid out on the XCDs."""
        return int(self._L.hawk_last_kernel(self._h))

    def debug_raise_timeout(self):
        """Test hook: sets the persistent kernels' error word from the host."""
        self._chk(self._L.hawk_debug_raise_timeout(self._h), "hawk_debug_raise_timeout")

    def phase_trace(self, enable: bool, n_stages: int = 0):
        """Switches the streaming kernel's stage time stamps; returns [4, n_stages, 8] uint64 if asked."""
        if n_stages <= 0:
            self._chk(self._L.hawk_phase_trace(self._h, int(enable), None, 0), "hawk_phase_trace")
            return None
        out = np.zeros(4 * 4096 * 8 + 2 * 256 * 256, dtype=np.uint64)
        self._chk(self._L.hawk_phase_trace(self._h, int(enable), _p(out), out.size), "hawk_phase_trace")
        self.last_arrivals = out[4 * 4096 * 8:].reshape(2, 256, 256)   # [arrive | release seen][stage][workgroup]
        return out[:4 * 4096 * 8].reshape(4, 4096, 8)[:, :n_stages]

    def load(self, blob: np.ndarray):
        blob = np.ascontiguousarray(blob, dtype=np.uint8)
        self._chk(self._L.hawk_load(self._h, _p(blob), blob.nbytes), "hawk_load")

    def prefill(self, cond, uncond, grid_h, grid_w, temperature, top_k, cfg_scale, u_first):
        cond = _f32(cond)
        unc = None if uncond is None else _f32(uncond)
        self.batch, self.n_img = cond.shape[0], grid_h * grid_w
        self._chk(self._L.hawk_prefill(self._h, _p(cond), _p(unc), cond.shape[0], cond.shape[1], grid_h, grid_w,
                                       temperature, top_k, cfg_scale, _p(_f32(u_first))), "hawk_prefill")

    def draft(self, k, u_draft, want=True):
        u = _f32(u_draft) if k > 0 else None
        out = np.full((self.batch, max(k, 1)), -1, dtype=np.int32) if want else None
        self._chk(self._L.hawk_draft(self._h, k, _p(u), _p(out) if (want and k > 0) else None), "hawk_draft")
        return None if out is None else out[:, :k]

    def draft_forced(self, k, tokens, point_mass):
        t = _i32(tokens) if k > 0 else None
        self._chk(self._L.hawk_draft_forced(self._h, k, _p(t), int(point_mass)), "hawk_draft_forced")

    def verify(self, k, u_acc, u_final, want=True):
        ua = _f32(u_acc) if k > 0 else None
        na = np.zeros(self.batch, dtype=np.int32) if want else None
        toks = np.zeros((self.batch, k + 1), dtype=np.int32) if want else None
        self._chk(self._L.hawk_verify(self._h, k, _p(ua), _p(_f32(u_final)), _p(na), _p(toks)), "hawk_verify")
        return na, toks

    def verify_tree(self, m_depth, cand, q_logits, u_acc, u_final):
        """hawk_verify_tree: m_depth [D]; cand [D, batch, m_max] int32 (host); q_logits a device fp32
        tensor [D, batch, m_max, V_s]; u_acc [D, batch, m_max], u_final [D + 1, batch] (host).
        Returns (accepted [batch], tokens [batch, D + 1])."""
        md = _i32(m_depth)
        D, m_max = len(md), int(md.max())
        cand, ua, uf = _i32(cand), _f32(u_acc), _f32(u_final)
        if cand.shape != (D, self.batch, m_max) or ua.shape != cand.shape or uf.shape != (D + 1, self.batch):
            raise HawkError(-1, "hawk_verify_tree", "host arrays do not have the documented shapes")
        if not (q_logits.is_cuda and q_logits.is_contiguous() and q_logits.dtype == self._torch.float32
                and tuple(q_logits.shape) == (D, self.batch, m_max, self.v_s)):
            raise HawkError(-1, "hawk_verify_tree", "q_logits must be a contiguous device fp32 tensor [D, batch, m_max, V_s]")
        na = np.zeros(self.batch, dtype=np.int32)
        toks = np.zeros((self.batch, D + 1), dtype=np.int32)
        self._chk(self._L.hawk_verify_tree(self._h, D, _p(md), _p(cand), C.c_void_p(q_logits.data_ptr()), _p(ua), _p(uf),
                                           _p(na), _p(toks)), "hawk_verify_tree")
        return na, toks

    def generate_spatial(self, cond, grid_h, grid_w, temperature, top_k, W_heads, W_out, HD, VSD, seed):
        """hawk_generate_spatial: the whole drafting and verification scheme over one image.  cond [1, n_cond, d]
        (host); W_heads [HD + VSD, d, d], W_out [V_s, d]: contiguous device bf16 tensors.  Returns (grid [1, N],
        dict(passes, accepted, tail_steps, tokens))."""
        torch = self._torch
        cond = _f32(cond)
        self.batch, self.n_img = 1, grid_h * grid_w
        d = self.cfg.d_model
        if not (W_heads.is_cuda and W_heads.is_contiguous() and W_heads.dtype == torch.bfloat16
                and tuple(W_heads.shape) == (HD + VSD, d, d) and W_out.is_cuda and W_out.is_contiguous()
                and W_out.dtype == torch.bfloat16 and tuple(W_out.shape) == (self.v_s, d)):
            raise HawkError(-1, "hawk_generate_spatial", "head weights must be contiguous device bf16 tensors [HD + VSD, d, d] and [V_s, d]")
        nbytes = int(self._L.hawk_generate_spatial_workspace_bytes(C.byref(self.cfg), grid_w, HD, VSD))
        if nbytes == 0:
            raise HawkError(-1, "hawk_generate_spatial_workspace_bytes", "bad arguments")
        ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=W_heads.device)
        base = (ws.data_ptr() + 255) & ~255
        grid = np.zeros((1, self.n_img), dtype=np.int32)
        stats = np.zeros(4, dtype=np.int64)
        self._chk(self._L.hawk_generate_spatial(self._h, _p(cond), cond.shape[1], grid_h, grid_w, float(temperature), int(top_k),
                                                C.c_void_p(W_heads.data_ptr()), C.c_void_p(W_out.data_ptr()), HD, VSD,
                                                C.c_uint64(seed), C.c_void_p(base), nbytes, _p(grid), _p(stats)),
                  "hawk_generate_spatial")
        return grid, dict(passes=int(stats[0]), accepted=int(stats[1]), tail_steps=int(stats[2]), tokens=int(stats[3]))

    def tree_path(self):
        out = np.zeros((self.batch, 8), dtype=np.int32)
        self._chk(self._L.hawk_get_tree_path(self._h, _p(out)), "hawk_get_tree_path")
        return out

    def last_hidden(self, rows_per_seq: int):
        """The hidden states of the last pass's rows as a device tensor view [sequences * rows_per_seq, d]
        (fp32 in the bf16 configurations, fp64 in the fp32 one) into the workspace: read only."""
        ptr, eb = C.c_void_p(), C.c_int()
        self._chk(self._L.hawk_last_hidden(self._h, C.byref(ptr), C.byref(eb)), "hawk_last_hidden")
        torch = self._torch
        n_seq = self.batch * (2 if self.cfg.use_cfg else 1)
        off = ptr.value - self._ws.data_ptr()
        nbytes = n_seq * rows_per_seq * self.cfg.d_model * eb.value
        return self._ws[off:off + nbytes].view(torch.float32 if eb.value == 4 else torch.float64).view(
            n_seq * rows_per_seq, self.cfg.d_model)

    def tree_logits(self, n_nodes):
        out = np.zeros((self.batch, n_nodes, self.v_s), dtype=np.float32)
        self._chk(self._L.hawk_get_tree_logits(self._h, _p(out), n_nodes), "hawk_get_tree_logits")
        return out

    def generate(self, cond, uncond, grid_h, grid_w, k, temperature, top_k, cfg_scale, seed, replay=None):
        cond = _f32(cond)
        unc = None if uncond is None else _f32(uncond)
        self.batch, self.n_img = cond.shape[0], grid_h * grid_w
        grid = np.zeros((self.batch, self.n_img), dtype=np.int32)
        rp = None if replay is None else _i32(replay)
        st = HawkStats()
        self._chk(self._L.hawk_generate(self._h, _p(cond), _p(unc), cond.shape[0], cond.shape[1], grid_h, grid_w, k,
                                        temperature, top_k, cfg_scale, seed, _p(rp), _p(grid), C.byref(st)),
                  "hawk_generate")
        return grid, st.as_dict()

    def run_steps(self, k, n_steps, seed, replay=False, timed=False):
        """Enqueues n_steps steps; with timed=True returns (ms_draft, ms_verify, ms_kernel) summed over them."""
        if timed:
            a, b, k_ = C.c_float(), C.c_float(), C.c_float()
            self._chk(self._L.hawk_run_steps(self._h, k, n_steps, seed, int(replay), C.byref(a), C.byref(b),
                                             C.byref(k_)), "hawk_run_steps")
            return a.value, b.value, k_.value
        self._chk(self._L.hawk_run_steps(self._h, k, n_steps, seed, int(replay), None, None, None), "hawk_run_steps")
        return None

    def set_replay(self, tokens):
        self._chk(self._L.hawk_set_replay(self._h, _p(_i32(tokens))), "hawk_set_replay")

    def stats(self):
        st = HawkStats()
        self._chk(self._L.hawk_get_stats(self._h, C.byref(st)), "hawk_get_stats")
        return st.as_dict()

    def synchronize(self):
        self._stream.synchronize()

    def force(self, n_from, tokens):
        t = _i32(tokens).reshape(self.batch, -1)
        self._chk(self._L.hawk_force(self._h, _p(_i32(n_from)), _p(t), t.shape[1]), "hawk_force")

    def n(self):
        out = np.zeros(self.batch, dtype=np.int32)
        self._chk(self._L.hawk_get_n(self._h, _p(out)), "hawk_get_n")
        return out

    def grid(self):
        out = np.zeros((self.batch, self.n_img), dtype=np.int32)
        self._chk(self._L.hawk_get_grid(self._h, _p(out)), "hawk_get_grid")
        return out

    def logits(self, rows):
        out = np.zeros((self.batch, rows, self.v_s), dtype=np.float32)
        self._chk(self._L.hawk_get_logits(self._h, _p(out), rows), "hawk_get_logits")
        return out

    def draft_logits(self, k):
        out = np.zeros((self.batch, k, self.v_s), dtype=np.float32)
        self._chk(self._L.hawk_get_draft_logits(self._h, _p(out), k), "hawk_get_draft_logits")
        return out
