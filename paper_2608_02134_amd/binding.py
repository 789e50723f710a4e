"""ctypes binding of libgmc.so: the C-ABI entry points under the same names,
plus a thin tensor-level wrapper (argument marshalling only).

Every step of the operator runs inside the HIP library.  If the library has
not been built, ``lib()`` raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgmc.so")

GMC_OK, GMC_ERR_ARG, GMC_ERR_CAPACITY, GMC_ERR_STATE, GMC_ERR_HIP = 0, -1, -2, -3, -4
GMC_ERR_DEVICE, GMC_ERR_NONFINITE = -5, -6
GMC_STATUS_SELECT_TIMEOUT, GMC_STATUS_BANK_TIMEOUT, GMC_STATUS_NONFINITE = 1, 2, 4
GMC_DIAG_CERT, GMC_DIAG_FINITE = 1, 2
GMC_CERT_MAX_ROUNDS = 64
GMC_STATIC_SCRATCH_BYTES = 64 << 20
GMC_F32, GMC_BF16 = 0, 1
GMC_STATS = 15
GMC_MAX_HIST_VIEWS = 3
GMC_MAX_IMAGES = 64
GMC_AUDIT_ROW, GMC_AUDIT_OUT = 8, 8
GMC_STATUS_INPUT = 8
GMC_MAX_GATHER_TENSORS = 64
GMC_CACHE_MAX_HEADS = 256

_i32, _f32, _i64, _vp = ctypes.c_int32, ctypes.c_float, ctypes.c_int64, ctypes.c_void_p


class GmcConfig(ctypes.Structure):
    """Mirror of ``gmc_config`` in include/gmc.h (same field order)."""
    _fields_ = [
        ("d", _i32), ("n_q_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32),
        ("probe_rank", _i32), ("dtype", _i32), ("max_batch", _i32), ("max_n", _i32),
        ("max_t", _i32), ("max_k", _i32),
        ("value_probe", _vp), ("app_projection", _vp),
        ("lambda_mass", _f32), ("eps_mass", _f32),
        ("beta_msg", _f32), ("beta_app", _f32), ("beta_spa", _f32),
        ("tau_v", _f32), ("tau_s", _f32),
        ("landmarks", _i32),
        ("batch_b", _i32), ("pool_mult", _i32),
        ("tau_r", _f32), ("resp_eps", _f32),
        ("spatial_w", _f32), ("gate_t", _f32), ("gate_p", _f32),
        ("amb_margin", _f32), ("amb_p", _f32),
        ("g_form", _i32),
        ("pop_strength", _f32), ("tau_j", _f32),
        ("max_head_clusters", _i32),
        ("disp_eps", _f32), ("terminal_q_weight", _f32),
        ("rms_eps", _f32), ("norm_eps", _f32), ("restore_eps", _f32),
        ("bounded_threshold_n", _i32),
        ("app_rank", _i32), ("app_max_clients", _i32),
        ("batch_b_bounded", _i32),
        ("value_probe_bias", _vp),
        ("max_hist_views", _i32), ("hist_mass", _f32),
        ("value_probe_hist", _vp), ("value_probe_bias_hist", _vp),
        ("max_images", _i32),
    ]


class GmcTrace(ctypes.Structure):
    """Mirror of ``gmc_trace``: optional device output pointers."""
    _fields_ = [("round_pool", _vp), ("round_batch", _vp), ("assign", _vp), ("omega", _vp),
                ("ebar", _vp), ("client", _vp), ("stats", _vp), ("round_gains", _vp),
                ("round_scores", _vp)]


class GmcView(ctypes.Structure):
    """Mirror of ``gmc_view``: one historical message view's device tensors."""
    _fields_ = [("hidden", _vp), ("text_q", _vp), ("vis_k", _vp), ("nonvis_lse", _vp)]


class GmcDiag(ctypes.Structure):
    """Mirror of ``gmc_diag``: host-side diagnostics of the last call."""
    _fields_ = [("status", ctypes.c_uint32), ("identity", _i32), ("has_certificate", _i32),
                ("k", _i32), ("rounds", _i32), ("m_rows", _i32), ("n_discarded", _i32),
                ("s_x", _f32), ("dbar", _f32), ("f_s", _f32), ("f_v", _f32),
                ("f_bank_s", _f32 * 3), ("f_bank_v", _f32 * 3), ("c_b", _f32),
                ("max_rounds", _i32),
                ("u_top", ctypes.POINTER(_f32)), ("gain", ctypes.POINTER(_f32)),
                ("q", ctypes.POINTER(_f32)), ("pool_margin", ctypes.POINTER(_f32)),
                ("batch_margin", ctypes.POINTER(_f32))]


class GmcCache(ctypes.Structure):
    """Mirror of ``gmc_cache``: one layer's paged K/V cache."""
    _fields_ = [("dtype", _i32), ("n_q_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32),
                ("page_size", _i32), ("max_pages", _i32), ("n_pages", _i64), ("n_seq", _i64),
                ("k_pages", _vp), ("v_pages", _vp), ("page_table", _vp), ("lens", _vp), ("seen", _vp),
                ("slot_pos", _vp), ("weights", _vp)]


class GmcRotary(ctypes.Structure):
    """Mirror of ``gmc_rotary``: the table of a rotary position encoding."""
    _fields_ = [("cos", _vp), ("sin", _vp), ("n_pos", _i64), ("rot_dim", _i32), ("interleaved", _i32),
                ("sections", _i32 * 3)]


class GmcCache4(ctypes.Structure):
    """Mirror of ``gmc_cache4``: one layer's paged K/V cache in 4 bits."""
    _fields_ = [("dtype", _i32), ("n_q_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32),
                ("page_size", _i32), ("max_pages", _i32), ("n_pages", _i64), ("n_seq", _i64),
                ("k_codes", _vp), ("v_codes", _vp), ("k_scales", _vp), ("v_scales", _vp), ("page_table", _vp),
                ("lens", _vp)]


# name -> (restype, argtypes) of every symbol include/gmc.h declares
SIGNATURES = {
    "gmc_config_default": (None, [ctypes.POINTER(GmcConfig)]),
    "gmc_init": (ctypes.c_int, [ctypes.POINTER(GmcConfig)]),
    "gmc_set_stream": (ctypes.c_int, [_vp]),
    "gmc_prune": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "gmc_prune_ex": (ctypes.c_int, [_i64, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp,
                                    ctypes.POINTER(GmcTrace)]),
    "gmc_prune_views": (ctypes.c_int, [_i64, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i64,
                                       ctypes.POINTER(GmcView), ctypes.POINTER(GmcTrace)]),
    "gmc_prune_full": (ctypes.c_int, [_i64, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp,
                                      _i64, ctypes.POINTER(GmcView), ctypes.POINTER(GmcTrace)]),
    "gmc_realized_budget": (_i64, [_i64, _i64, _i64]),
    "gmc_audit_message": (ctypes.c_int, [_i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                         _vp]),
    "gmc_trace_dims_full": (ctypes.c_int, [_i64, _i64, _i64, _i64, _i64, ctypes.POINTER(_i64), ctypes.POINTER(_i64),
                                           ctypes.POINTER(_i64), ctypes.POINTER(_i64)]),
    "gmc_realized_k": (_i64, [_i64, _i64]),
    "gmc_trace_dims": (ctypes.c_int, [_i64, _i64, _i64, ctypes.POINTER(_i64), ctypes.POINTER(_i64),
                                      ctypes.POINTER(_i64), ctypes.POINTER(_i64)]),
    "gmc_compact_sequence": (ctypes.c_int, [_i64, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _i64,
                                            _vp, _vp]),
    "gmc_gather_rows": (ctypes.c_int, [_i64, ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i64, _i64, _i64, _i64,
                                       _i64, _vp]),
    "gmc_set_diag": (ctypes.c_int, [_i32]),
    "gmc_get_diag": (ctypes.c_int, [_i64, ctypes.POINTER(GmcDiag)]),
    "gmc_prune_static": (ctypes.c_int, [ctypes.POINTER(GmcConfig), _i64, _vp, _vp, _vp, _vp, _i64, _i64, _i64,
                                        _vp, _vp, _vp, _vp, _vp]),
    "gmc_cache_append": (ctypes.c_int, [ctypes.POINTER(GmcCache), _vp, _vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp]),
    "gmc_cache_prefill_bytes": (_i64, [ctypes.POINTER(GmcCache), _i64]),
    "gmc_cache_prefill": (ctypes.c_int, [ctypes.POINTER(GmcCache), _vp, _i64, _i64, _vp, _i64, _f32, _i64, _i64, _vp,
                                         _vp, _vp, _i64, _vp]),
    "gmc_cache_decode_bytes": (_i64, [ctypes.POINTER(GmcCache), _i32]),
    "gmc_cache_decode": (ctypes.c_int, [ctypes.POINTER(GmcCache), _vp, _i64, _f32, _i64, _i64, _i32, _vp, _vp, _vp,
                                        _i64, _vp]),
    "gmc_cache_evict_bytes": (_i64, [ctypes.POINTER(GmcCache), _i64]),
    "gmc_cache_evict": (ctypes.c_int, [ctypes.POINTER(GmcCache), _i64, _i64, _i64, _vp, _i64, _vp]),
    "gmc_cache_append_rotary": (ctypes.c_int, [ctypes.POINTER(GmcCache), ctypes.POINTER(GmcRotary), _vp, _vp, _i64,
                                               _i64, _i64, _vp, _vp, _i64, _vp, _vp, _i64, _vp, _vp]),
    "gmc_cache4_append": (ctypes.c_int, [ctypes.POINTER(GmcCache4), ctypes.POINTER(GmcRotary), _vp, _vp, _i64, _i64,
                                         _i64, _vp, _vp, _i64, _vp, _vp, _i64, _vp, _vp]),
    "gmc_cache4_read": (ctypes.c_int, [ctypes.POINTER(GmcCache4), _i64, _vp, _i64, _vp, _vp, _vp]),
    "gmc_cache4_prefill_bytes": (_i64, [ctypes.POINTER(GmcCache4), _i64]),
    "gmc_cache4_prefill": (ctypes.c_int, [ctypes.POINTER(GmcCache4), _vp, _i64, _i64, _vp, _i64, _f32, _i64, _i64,
                                          _vp, _vp, _vp, _i64, _vp]),
    "gmc_cache4_decode_bytes": (_i64, [ctypes.POINTER(GmcCache4)]),
    "gmc_cache4_decode": (ctypes.c_int, [ctypes.POINTER(GmcCache4), _vp, _i64, _f32, _i64, _i64, _vp, _vp, _vp, _i64,
                                         _vp]),
    "gmc_workspace_bytes": (_i64, []),
    "gmc_last_error": (ctypes.c_char_p, []),
    "gmc_free": (None, []),
}

_LIB = None


def lib():
    """Load libgmc.so (raises if it has not been built)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -c 'import __graft_entry__ as g; g.build()'`")
        so = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(so, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = so
    return _LIB


class GmcError(RuntimeError):
    def __init__(self, code: int, where: str):
        msg = lib().gmc_last_error().decode(errors="replace")
        super().__init__(f"{where} failed ({code}): {msg}")
        self.code = code


def _check(code: int, where: str):
    if code != GMC_OK:
        raise GmcError(code, where)


# --- C-ABI entry points under their own names ------------------------------
def gmc_config_default() -> GmcConfig:
    cfg = GmcConfig()
    lib().gmc_config_default(ctypes.byref(cfg))
    return cfg


def gmc_init(cfg: GmcConfig) -> int:
    return lib().gmc_init(ctypes.byref(cfg))


def gmc_set_stream(stream: int) -> int:
    return lib().gmc_set_stream(_vp(stream))


def gmc_prune(hidden, text_q, vis_k, pos3d, n, t, k, out_hidden, out_pos, out_idx) -> int:
    return lib().gmc_prune(hidden, text_q, vis_k, pos3d, n, t, k, out_hidden, out_pos, out_idx)


def gmc_prune_ex(b, hidden, text_q, vis_k, pos3d, n, t, k, out_hidden, out_pos, out_idx,
                 nonvis_lse=None, trace: Optional[GmcTrace] = None) -> int:
    tr = ctypes.byref(trace) if trace is not None else None
    return lib().gmc_prune_ex(b, hidden, text_q, vis_k, pos3d, n, t, k, out_hidden, out_pos,
                              out_idx, nonvis_lse, tr)


def gmc_prune_views(b, hidden, text_q, vis_k, pos3d, n, t, k, out_hidden, out_pos, out_idx, nonvis_lse,
                    hist_views, trace: Optional[GmcTrace] = None) -> int:
    """hist_views: a sequence of GmcView."""
    nh = len(hist_views)
    arr = (GmcView * max(nh, 1))(*hist_views)
    tr = ctypes.byref(trace) if trace is not None else None
    return lib().gmc_prune_views(b, hidden, text_q, vis_k, pos3d, n, t, k, out_hidden, out_pos, out_idx,
                                 nonvis_lse, nh, arr, tr)


def gmc_prune_full(b, hidden, text_q, vis_k, pos3d, image_id, n_images, n, t, k, out_hidden, out_pos, out_idx,
                   nonvis_lse=None, hist_views=(), trace: Optional[GmcTrace] = None) -> int:
    nh = len(hist_views)
    arr = (GmcView * max(nh, 1))(*hist_views)
    tr = ctypes.byref(trace) if trace is not None else None
    return lib().gmc_prune_full(b, hidden, text_q, vis_k, pos3d, image_id, n_images, n, t, k, out_hidden,
                                out_pos, out_idx, nonvis_lse, nh, arr, tr)


def gmc_audit_message(b, n, t, k, text_q, vis_k, vis_v, comp_k, comp_v, carrier, weights, nonvis_lse, rows_out,
                      vec_out, out) -> int:
    return lib().gmc_audit_message(b, n, t, k, text_q, vis_k, vis_v, comp_k, comp_v, carrier, weights, nonvis_lse,
                                   rows_out, vec_out, out)


def gmc_realized_budget(n: int, k_req: int, n_images: int) -> int:
    return int(lib().gmc_realized_budget(n, k_req, n_images))


def gmc_trace_dims_full(n: int, t: int, k: int, n_hist: int, n_images: int):
    vals = [_i64() for _ in range(4)]
    code = lib().gmc_trace_dims_full(n, t, k, n_hist, n_images, *[ctypes.byref(v) for v in vals])
    _check(code, "gmc_trace_dims_full")
    return tuple(int(v.value) for v in vals)


def gmc_realized_k(n: int, k_req: int) -> int:
    return int(lib().gmc_realized_k(n, k_req))


def gmc_trace_dims(n: int, t: int, k: int):
    vals = [_i64() for _ in range(4)]
    code = lib().gmc_trace_dims(n, t, k, *[ctypes.byref(v) for v in vals])
    _check(code, "gmc_trace_dims")
    return tuple(int(v.value) for v in vals)


def gmc_compact_sequence(b, seq_len, vis_start, n, k, out_idx, iota, keep, seq_rows, vis_rows, out_rows,
                         row_bytes, seq_pos, out_pos) -> int:
    return lib().gmc_compact_sequence(b, seq_len, vis_start, n, k, out_idx, iota, keep, seq_rows, vis_rows,
                                      out_rows, row_bytes, seq_pos, out_pos)


def gmc_gather_rows(src_ptrs, dst_ptrs, n_seq, seqs_per_keep, seq_len, seq_len2, row_bytes, keep) -> int:
    n = len(src_ptrs)
    src = (_vp * max(n, 1))(*src_ptrs)
    dst = (_vp * max(len(dst_ptrs), 1))(*dst_ptrs)
    return lib().gmc_gather_rows(n, src, dst, n_seq, seqs_per_keep, seq_len, seq_len2, row_bytes, keep)


def check_prune_inputs(cfg: GmcConfig, dtype, hidden, text_q, vis_k, pos3d, nonvis_lse=None):
    """Shapes, dtypes and devices of a pruning call's tensors against the
    context's configuration (the library itself sees raw pointers only).
    Returns (B, N, T); raises ValueError."""
    import torch
    if hidden.dim() != 3 or hidden.shape[2] != cfg.d:
        raise ValueError(f"hidden must be [B][N][{cfg.d}], got {tuple(hidden.shape)}")
    b, n, _ = hidden.shape
    hd = cfg.n_q_heads * cfg.head_dim
    if text_q.dim() < 3 or text_q.shape[0] != b or int(np.prod(text_q.shape[2:])) != hd:
        raise ValueError(f"text_q must be [B][T][{cfg.n_q_heads}][{cfg.head_dim}] (or [B][T][Hq*dh]), "
                         f"got {tuple(text_q.shape)}")
    t = text_q.shape[1]
    if vis_k.dim() < 3 or vis_k.shape[0] != b or vis_k.shape[1] != n or \
            int(np.prod(vis_k.shape[2:])) != cfg.n_kv_heads * cfg.head_dim:
        raise ValueError(f"vis_k must be [B][N][{cfg.n_kv_heads}][{cfg.head_dim}] (or [B][N][Hkv*dh]), "
                         f"got {tuple(vis_k.shape)}")
    if tuple(pos3d.shape) != (b, n, 3) or pos3d.dtype != torch.int32:
        raise ValueError(f"pos3d must be int32 [B][N][3] = ({b}, {n}, 3), got {pos3d.dtype} {tuple(pos3d.shape)}")
    for name, x in (("hidden", hidden), ("text_q", text_q), ("vis_k", vis_k)):
        if x.dtype != dtype:
            raise ValueError(f"{name} has dtype {x.dtype}, the context computes in {dtype}")
    tensors = [("hidden", hidden), ("text_q", text_q), ("vis_k", vis_k), ("pos3d", pos3d)]
    if nonvis_lse is not None:
        if nonvis_lse.dtype != torch.float32 or tuple(nonvis_lse.shape) != (b, cfg.n_q_heads, t):
            raise ValueError(f"nonvis_lse must be float32 [B][Hq][T] = ({b}, {cfg.n_q_heads}, {t}), "
                             f"got {nonvis_lse.dtype} {tuple(nonvis_lse.shape)}")
        tensors.append(("nonvis_lse", nonvis_lse))
    for name, x in tensors:
        if not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    dev = hidden.device
    for name, x in tensors:
        if x.device.type != "cuda" or x.device != dev:
            raise ValueError(f"{name} must be on the GPU, on hidden's device; got {x.device}")
    return b, n, t


def check_gather_inputs(caches, keep, seqs_per_keep):
    """Every cache contiguous with the same [n_seq][L] leading shape and row
    bytes, on keep's device; keep int32 [n_seq / seqs_per_keep][L2].  Raises
    ValueError."""
    import torch
    if not caches:
        raise ValueError("gather_rows needs at least one cache")
    c0 = caches[0]
    if c0.dim() < 2:
        raise ValueError("caches must be [n_seq][L][...]")
    n_seq, seq_len = c0.shape[:2]
    row_bytes = (c0.numel() // max(n_seq * seq_len, 1)) * c0.element_size()
    for i, c in enumerate(caches):
        if c.dim() < 2 or tuple(c.shape[:2]) != (n_seq, seq_len):
            raise ValueError(f"cache {i} has leading shape {tuple(c.shape[:2])}, expected {(n_seq, seq_len)}")
        if (c.numel() // max(n_seq * seq_len, 1)) * c.element_size() != row_bytes:
            raise ValueError(f"cache {i} rows are not {row_bytes} bytes")
        if not c.is_contiguous():
            raise ValueError(f"cache {i} must be contiguous")
    if keep.dtype != torch.int32 or keep.dim() != 2 or not keep.is_contiguous():
        raise ValueError("keep must be a contiguous int32 [n_seq / seqs_per_keep][L2] tensor")
    if seqs_per_keep < 1 or keep.shape[0] * seqs_per_keep != n_seq:
        raise ValueError(f"keep has {keep.shape[0]} lists; {n_seq} sequences need {n_seq} / seqs_per_keep")
    for i, c in enumerate(caches):
        if c.device.type != "cuda" or c.device != keep.device:
            raise ValueError(f"cache {i} must be on the GPU, on keep's device; got {c.device}")
    return n_seq, seq_len, row_bytes


def check_compact_inputs(out_idx, n, seq_rows, vis_rows, seq_pos, seq_len):
    """out_idx int32 [B][K]; seq_rows [B][L][...] and vis_rows [B][K][...] of one
    dtype and row size; seq_pos int32 [B][L][3]; all on out_idx's device.
    Raises ValueError."""
    import torch
    if out_idx.dtype != torch.int32 or out_idx.dim() != 2 or not out_idx.is_contiguous():
        raise ValueError("out_idx must be a contiguous int32 [B][K] tensor")
    b, k = out_idx.shape
    if not 1 <= k <= n:
        raise ValueError(f"need 1 <= K <= N, got K={k}, N={n}")
    tensors = [("out_idx", out_idx)]
    if (seq_rows is None) != (vis_rows is None):
        raise ValueError("seq_rows and vis_rows must be given together")
    if seq_rows is not None:
        if seq_rows.shape[0] != b or seq_rows.shape[1] != seq_len or vis_rows.shape[0] != b or vis_rows.shape[1] != k:
            raise ValueError(f"seq_rows must be [B][L][...] and vis_rows [B][K][...] with B={b}, L={seq_len}, K={k}")
        if seq_rows.dtype != vis_rows.dtype or seq_rows[0, 0].numel() != vis_rows[0, 0].numel():
            raise ValueError("seq_rows and vis_rows must share dtype and row size")
        tensors += [("seq_rows", seq_rows), ("vis_rows", vis_rows)]
    if seq_pos is not None:
        if seq_pos.dtype != torch.int32 or tuple(seq_pos.shape) != (b, seq_len, 3):
            raise ValueError(f"seq_pos must be int32 [B][L][3] = ({b}, {seq_len}, 3)")
        tensors.append(("seq_pos", seq_pos))
    for name, x in tensors:
        if not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    for name, x in tensors:
        if x.device.type != "cuda" or x.device != out_idx.device:
            raise ValueError(f"{name} must be on the GPU, on out_idx's device; got {x.device}")


def compact_sequence(out_idx, vis_start, n, seq_rows=None, vis_rows=None, seq_pos=None, seq_len=None):
    """Tensor-level sequence compaction on torch's current stream (argument
    marshalling only): out_idx [B][K] int32 device; seq_rows [B][L][...] and
    vis_rows [B][K][...] of one dtype; seq_pos [B][L][3] int32.  Returns
    (iota [B][L], keep [B][L2], out_rows or None, out_pos or None)."""
    import torch
    b, k = out_idx.shape
    if seq_len is None:
        seq_len = seq_rows.shape[1] if seq_rows is not None else seq_pos.shape[1]
    check_compact_inputs(out_idx, n, seq_rows, vis_rows, seq_pos, seq_len)
    l2 = seq_len - n + k
    dev = out_idx.device
    iota = torch.empty((b, seq_len), dtype=torch.int32, device=dev)
    keep = torch.empty((b, l2), dtype=torch.int32, device=dev)
    out_rows = out_pos = None
    row_bytes = 0
    if seq_rows is not None:
        out_rows = torch.empty((b, l2) + tuple(seq_rows.shape[2:]), dtype=seq_rows.dtype, device=dev)
        row_bytes = seq_rows[0, 0].numel() * seq_rows.element_size()
    if seq_pos is not None:
        out_pos = torch.empty((b, l2, 3), dtype=torch.int32, device=dev)
    _check(gmc_set_stream(torch.cuda.current_stream(dev).cuda_stream), "gmc_set_stream")
    ptr = (lambda t: None if t is None else t.data_ptr())
    _check(gmc_compact_sequence(b, seq_len, vis_start, n, k, out_idx.data_ptr(), iota.data_ptr(), keep.data_ptr(),
                                ptr(seq_rows), ptr(vis_rows), ptr(out_rows), row_bytes, ptr(seq_pos), ptr(out_pos)),
           "gmc_compact_sequence")
    return iota, keep, out_rows, out_pos


def gather_rows(caches, keep, seqs_per_keep=1):
    """Tensor-level row gather on torch's current stream: each cache is
    [n_seq][L][...] (contiguous), keep [n_seq / seqs_per_keep][L2] int32;
    returns the gathered [n_seq][L2][...] caches."""
    import torch
    n_seq, seq_len, row_bytes = check_gather_inputs(caches, keep, seqs_per_keep)
    l2 = keep.shape[1]
    outs = [torch.empty((n_seq, l2) + tuple(c.shape[2:]), dtype=c.dtype, device=c.device) for c in caches]
    _check(gmc_set_stream(torch.cuda.current_stream(caches[0].device).cuda_stream), "gmc_set_stream")
    for i in range(0, len(caches), GMC_MAX_GATHER_TENSORS):
        part = slice(i, i + GMC_MAX_GATHER_TENSORS)
        _check(gmc_gather_rows([c.data_ptr() for c in caches[part]], [o.data_ptr() for o in outs[part]], n_seq,
                               seqs_per_keep, seq_len, l2, row_bytes, keep.data_ptr()), "gmc_gather_rows")
    return outs


def gmc_set_diag(flags: int) -> int:
    return lib().gmc_set_diag(flags)


def gmc_get_diag(problem: int = 0, max_rounds: int = GMC_CERT_MAX_ROUNDS):
    """Diagnostics of the last pruning call for one problem (synchronises).
    Returns (code, dict); the per-round arrays hold `rounds` entries."""
    arrs = {k: (_f32 * max(max_rounds, 1))() for k in ("u_top", "gain", "q", "pool_margin", "batch_margin")}
    d = GmcDiag()
    d.max_rounds = max_rounds
    for k, a in arrs.items():
        setattr(d, k, ctypes.cast(a, ctypes.POINTER(_f32)))
    code = lib().gmc_get_diag(problem, ctypes.byref(d))
    out = {k: getattr(d, k) for k in ("status", "identity", "has_certificate", "k", "rounds", "m_rows",
                                       "n_discarded", "s_x", "dbar", "f_s", "f_v", "c_b")}
    out["f_bank_s"] = list(d.f_bank_s)
    out["f_bank_v"] = list(d.f_bank_v)
    nr = min(d.rounds, max_rounds) if d.has_certificate else 0
    for k, a in arrs.items():
        out[k] = [a[i] for i in range(nr)]
    return code, out


def gmc_prune_static(cfg: GmcConfig, b, hidden, text_q, vis_k, pos3d, n, t, k, out_hidden, out_pos, out_idx,
                     nonvis_lse=None, stream=None) -> int:
    return lib().gmc_prune_static(ctypes.byref(cfg), b, hidden, text_q, vis_k, pos3d, n, t, k, out_hidden,
                                  out_pos, out_idx, nonvis_lse, stream)


def gmc_cache_append(cache: GmcCache, k, v, k_stride, v_stride, rows, starts, src, max_new, stream=None) -> int:
    return lib().gmc_cache_append(ctypes.byref(cache), k, v, k_stride, v_stride, rows, starts, src, max_new, stream)


def gmc_cache_prefill_bytes(cache: GmcCache, max_new: int) -> int:
    return lib().gmc_cache_prefill_bytes(ctypes.byref(cache), max_new)


def gmc_cache_prefill(cache: GmcCache, q, q_stride, rows, starts, max_new, scale, window, sinks, out, lse, workspace,
                      workspace_bytes, stream=None) -> int:
    return lib().gmc_cache_prefill(ctypes.byref(cache), q, q_stride, rows, starts, max_new, scale, window, sinks, out,
                                   lse, workspace, workspace_bytes, stream)


def gmc_cache_decode_bytes(cache: GmcCache, accumulate: bool) -> int:
    return lib().gmc_cache_decode_bytes(ctypes.byref(cache), int(accumulate))


def gmc_cache_decode(cache: GmcCache, q, q_stride, scale, window, sinks, accumulate, out, lse, workspace,
                     workspace_bytes, stream=None) -> int:
    return lib().gmc_cache_decode(ctypes.byref(cache), q, q_stride, scale, window, sinks, int(accumulate), out, lse,
                                  workspace, workspace_bytes, stream)


def gmc_cache_evict_bytes(cache: GmcCache, budget: int) -> int:
    return lib().gmc_cache_evict_bytes(ctypes.byref(cache), budget)


def gmc_cache_evict(cache: GmcCache, budget, sinks, recent, workspace, workspace_bytes, stream=None) -> int:
    return lib().gmc_cache_evict(ctypes.byref(cache), budget, sinks, recent, workspace, workspace_bytes, stream)


def gmc_cache_append_rotary(cache: GmcCache, rotary: GmcRotary, k, v, k_stride, v_stride, rows, starts, src, max_new,
                            pos, q, q_stride, q_out, stream=None) -> int:
    return lib().gmc_cache_append_rotary(ctypes.byref(cache), ctypes.byref(rotary), k, v, k_stride, v_stride, rows,
                                         starts, src, max_new, pos, q, q_stride, q_out, stream)


def gmc_cache4_append(cache: GmcCache4, rotary, k, v, k_stride, v_stride, rows, starts, src, max_new, pos, q,
                      q_stride, q_out, stream=None) -> int:
    return lib().gmc_cache4_append(ctypes.byref(cache), None if rotary is None else ctypes.byref(rotary), k, v,
                                   k_stride, v_stride, rows, starts, src, max_new, pos, q, q_stride, q_out, stream)


def gmc_cache4_read(cache: GmcCache4, rows, starts, max_new, k_out, v_out, stream=None) -> int:
    return lib().gmc_cache4_read(ctypes.byref(cache), rows, starts, max_new, k_out, v_out, stream)


def gmc_cache4_prefill_bytes(cache: GmcCache4, max_new: int) -> int:
    return lib().gmc_cache4_prefill_bytes(ctypes.byref(cache), max_new)


def gmc_cache4_prefill(cache: GmcCache4, q, q_stride, rows, starts, max_new, scale, window, sinks, out, lse, workspace,
                       workspace_bytes, stream=None) -> int:
    return lib().gmc_cache4_prefill(ctypes.byref(cache), q, q_stride, rows, starts, max_new, scale, window, sinks, out,
                                    lse, workspace, workspace_bytes, stream)


def gmc_cache4_decode_bytes(cache: GmcCache4) -> int:
    return lib().gmc_cache4_decode_bytes(ctypes.byref(cache))


def gmc_cache4_decode(cache: GmcCache4, q, q_stride, scale, window, sinks, out, lse, workspace, workspace_bytes,
                      stream=None) -> int:
    return lib().gmc_cache4_decode(ctypes.byref(cache), q, q_stride, scale, window, sinks, out, lse, workspace,
                                   workspace_bytes, stream)


def gmc_workspace_bytes() -> int:
    return int(lib().gmc_workspace_bytes())


def gmc_last_error() -> str:
    return lib().gmc_last_error().decode(errors="replace")


def gmc_free() -> None:
    lib().gmc_free()


# --- tensor-level wrapper ----------------------------------------------------
class Pruner:
    """Owns one library context for a model shape and capacity.

    ``probe`` [Hq][r][d] and ``app_projection`` [app_rank][d] are device
    tensors in the operator dtype, ``probe_bias`` [Hq][r] an optional fp32
    device tensor; the wrapper keeps them alive.  ``prune``
    allocates outputs with torch and calls gmc_prune_ex on torch's current
    stream.
    """

    def __init__(self, *, d, n_q_heads, n_kv_heads, head_dim, probe, dtype, max_batch, max_n,
                 max_t, max_k=0, app_projection=None, probe_bias=None, probe_hist=None, **overrides):
        import torch
        self.torch = torch
        cfg = gmc_config_default()
        cfg.d, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim = d, n_q_heads, n_kv_heads, head_dim
        cfg.probe_rank = probe.shape[1]
        cfg.dtype = GMC_BF16 if dtype == torch.bfloat16 else GMC_F32
        cfg.max_batch, cfg.max_n, cfg.max_t, cfg.max_k = max_batch, max_n, max_t, max_k
        for key, val in overrides.items():
            setattr(cfg, key, val)
        self.probe = probe.contiguous()
        self.app_projection = None if app_projection is None else app_projection.contiguous()
        cfg.value_probe = self.probe.data_ptr()
        cfg.app_projection = 0 if self.app_projection is None else self.app_projection.data_ptr()
        self.probe_bias = None if probe_bias is None else probe_bias.contiguous()
        if self.probe_bias is not None and (self.probe_bias.dtype != torch.float32 or
                                            tuple(self.probe_bias.shape) != (n_q_heads, cfg.probe_rank)):
            raise ValueError("probe_bias must be a float32 [n_q_heads][probe_rank] tensor")
        cfg.value_probe_bias = 0 if self.probe_bias is None else self.probe_bias.data_ptr()
        # probes of the historical message views [n_hist][Hq][r][d]
        self.probe_hist = None if probe_hist is None else probe_hist.contiguous()
        if self.probe_hist is not None:
            if self.probe_hist.dim() != 4 or tuple(self.probe_hist.shape[1:]) != tuple(self.probe.shape) or \
                    self.probe_hist.dtype != self.probe.dtype:
                raise ValueError("probe_hist must be [n_hist] x the probe's shape and dtype")
            cfg.max_hist_views = self.probe_hist.shape[0]
            cfg.value_probe_hist = self.probe_hist.data_ptr()
        self.cfg = cfg
        self.dtype = dtype
        _check(gmc_init(cfg), "gmc_init")

    def trace_dims(self, n, t, k):
        return gmc_trace_dims(n, t, k)

    def prune(self, hidden, text_q, vis_k, pos3d, k, nonvis_lse=None, trace: bool = False, hist=None,
              image_id=None, n_images: int = 1):
        """hist: optional list of historical views, each (hidden, text_q,
        vis_k[, nonvis_lse]) shaped like the current view's tensors;
        image_id: optional int32 [B][N] device tensor of image ids in
        [0, n_images) for a multi-image prompt."""
        torch = self.torch
        b, n, t = check_prune_inputs(self.cfg, self.dtype, hidden, text_q, vis_k, pos3d, nonvis_lse)
        hist = list(hist or [])
        views = []
        for i, hv in enumerate(hist):
            hv = tuple(hv) + (None,) * (4 - len(hv))
            try:
                check_prune_inputs(self.cfg, self.dtype, hv[0], hv[1], hv[2], pos3d, hv[3])
                if hv[0].shape != hidden.shape or hv[1].shape != text_q.shape:
                    raise ValueError("shapes differ from the current view's")
                if hv[0].device != hidden.device:
                    raise ValueError("not on hidden's device")
            except ValueError as e:
                raise ValueError(f"historical view {i}: {e}") from None
            views.append(GmcView(hv[0].data_ptr(), hv[1].data_ptr(), hv[2].data_ptr(),
                                 None if hv[3] is None else hv[3].data_ptr()))
        if image_id is not None:
            if image_id.dtype != torch.int32 or tuple(image_id.shape) != (b, n) or not image_id.is_contiguous() \
                    or image_id.device != hidden.device:
                raise ValueError(f"image_id must be a contiguous int32 [B][N] = ({b}, {n}) tensor on hidden's device")
        multi = image_id is not None and n_images > 1
        d = hidden.shape[2]
        kk = gmc_realized_budget(n, k, n_images if image_id is not None else 1)
        dev = hidden.device
        out_h = torch.empty((b, kk, d), dtype=hidden.dtype, device=dev)
        out_p = torch.empty((b, kk, 3), dtype=torch.int32, device=dev)
        out_i = torch.empty((b, kk), dtype=torch.int32, device=dev)
        tr, bufs = None, {}
        if trace:
            rounds, pool_cap, bcap, m_rows = gmc_trace_dims_full(n, t, k, len(views),
                                                                 n_images if multi else 1)
            hq = self.cfg.n_q_heads
            r1 = max(rounds, 1)
            bufs = dict(
                round_pool=torch.full((b, r1, pool_cap), -1, dtype=torch.int32, device=dev),
                round_batch=torch.full((b, r1, bcap), -1, dtype=torch.int32, device=dev),
                assign=torch.full((b, n), -1, dtype=torch.int32, device=dev),
                omega=torch.zeros((b, hq), dtype=torch.float32, device=dev),
                ebar=torch.zeros((b, n), dtype=torch.float32, device=dev),
                client=torch.zeros((b, m_rows, n), dtype=torch.float32, device=dev),
                stats=torch.zeros((b, GMC_STATS), dtype=torch.float32, device=dev),
                round_gains=torch.full((b, r1, n), -1.0, dtype=torch.float32, device=dev),
                round_scores=torch.full((b, r1, pool_cap), -1.0, dtype=torch.float32, device=dev))
            tr = GmcTrace(**{key: v.data_ptr() for key, v in bufs.items()})
        _check(gmc_set_stream(torch.cuda.current_stream(dev).cuda_stream), "gmc_set_stream")
        nv = None if nonvis_lse is None else nonvis_lse.data_ptr()
        if multi:
            code = gmc_prune_full(b, hidden.data_ptr(), text_q.data_ptr() if t > 0 else None,
                                  vis_k.data_ptr(), pos3d.data_ptr(), image_id.data_ptr(), n_images, n, t, k,
                                  out_h.data_ptr(), out_p.data_ptr(), out_i.data_ptr(), nv, views, tr)
            _check(code, "gmc_prune_full")
        elif views:
            code = gmc_prune_views(b, hidden.data_ptr(), text_q.data_ptr() if t > 0 else None,
                                   vis_k.data_ptr(), pos3d.data_ptr(), n, t, k, out_h.data_ptr(),
                                   out_p.data_ptr(), out_i.data_ptr(), nv, views, tr)
            _check(code, "gmc_prune_views")
        else:
            code = gmc_prune_ex(b, hidden.data_ptr(), text_q.data_ptr() if t > 0 else None,
                                vis_k.data_ptr(), pos3d.data_ptr(), n, t, k, out_h.data_ptr(),
                                out_p.data_ptr(), out_i.data_ptr(), nv, tr)
            _check(code, "gmc_prune_ex")
        if trace:
            return out_h, out_p, out_i, bufs
        return out_h, out_p, out_i

    def audit(self, text_q, vis_k, vis_v, comp_k, comp_v, carrier, weights=None, nonvis_lse=None,
              rows: bool = False, vectors: bool = False):
        """gmc_audit_message on torch's current stream: text_q [B][T][Hq][dh],
        vis_k / vis_v [B][N][Hkv][dh], comp_k / comp_v [B][K][Hkv][dh] in the
        context dtype, carrier [B][N] int32 slots, weights / nonvis_lse
        [B][Hq][T] fp32 or None.  Returns (out [B][8], rows [B][Hq][T][8] or
        None, vectors [B][Hq][T][4][dh] or None)."""
        torch = self.torch
        cfg = self.cfg
        b, t = text_q.shape[:2]
        n, k = vis_k.shape[1], comp_k.shape[1]
        hd = (cfg.n_kv_heads, cfg.head_dim)
        for name, x, lead in (("vis_k", vis_k, (b, n)), ("vis_v", vis_v, (b, n)), ("comp_k", comp_k, (b, k)),
                              ("comp_v", comp_v, (b, k))):
            if tuple(x.shape) != lead + hd or x.dtype != self.dtype or not x.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {self.dtype} {lead + hd} tensor")
        if tuple(text_q.shape) != (b, t, cfg.n_q_heads, cfg.head_dim) or text_q.dtype != self.dtype:
            raise ValueError("text_q must be [B][T][Hq][dh] in the context dtype")
        if tuple(carrier.shape) != (b, n) or carrier.dtype != torch.int32 or not carrier.is_contiguous():
            raise ValueError("carrier must be a contiguous int32 [B][N] tensor")
        for name, x in (("weights", weights), ("nonvis_lse", nonvis_lse)):
            if x is not None and (tuple(x.shape) != (b, cfg.n_q_heads, t) or x.dtype != torch.float32):
                raise ValueError(f"{name} must be float32 [B][Hq][T]")
        dev = text_q.device
        out = torch.zeros((b, GMC_AUDIT_OUT), dtype=torch.float32, device=dev)
        ro = torch.zeros((b, cfg.n_q_heads, t, GMC_AUDIT_ROW), dtype=torch.float32, device=dev) if rows else None
        vo = torch.zeros((b, cfg.n_q_heads, t, 4, cfg.head_dim), dtype=torch.float32, device=dev) if vectors else None
        _check(gmc_set_stream(torch.cuda.current_stream(dev).cuda_stream), "gmc_set_stream")
        ptr = (lambda x: None if x is None else x.contiguous().data_ptr())
        _check(gmc_audit_message(b, n, t, k, text_q.data_ptr(), vis_k.data_ptr(), vis_v.data_ptr(), comp_k.data_ptr(),
                                 comp_v.data_ptr(), carrier.data_ptr(), ptr(weights), ptr(nonvis_lse), ptr(ro),
                                 ptr(vo), out.data_ptr()), "gmc_audit_message")
        return out, ro, vo

    def set_diag(self, flags: int):
        _check(gmc_set_diag(flags), "gmc_set_diag")

    def diag(self, problem: int = 0):
        """(code, dict) of gmc_get_diag for the last call (synchronises)."""
        return gmc_get_diag(problem)

    def close(self):
        gmc_free()


def check_cache_tensors(k_pages, v_pages, page_table, lens, n_q_heads, slot_pos=None, seen=None, weights=None):
    """Shapes, dtypes and devices of a cache's tensors (see gmc_cache).  Raises
    ValueError."""
    import torch
    if k_pages.dim() != 4 or k_pages.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("k_pages must be [n_pages][n_kv_heads][page_size][head_dim] in float32 or bfloat16, got "
                         f"{k_pages.dtype} {tuple(k_pages.shape)}")
    if v_pages.shape != k_pages.shape or v_pages.dtype != k_pages.dtype:
        raise ValueError("v_pages must have k_pages' shape and dtype")
    if page_table.dim() != 2 or page_table.dtype != torch.int32:
        raise ValueError("page_table must be int32 [n_seq][max_pages]")
    if k_pages.numel() == 0 or page_table.numel() == 0:
        raise ValueError(f"k_pages {tuple(k_pages.shape)} and page_table {tuple(page_table.shape)} must not be empty")
    b, slots = page_table.shape[0], page_table.shape[1] * k_pages.shape[2]
    if n_q_heads < 1 or n_q_heads % max(k_pages.shape[1], 1) != 0:
        raise ValueError(f"n_q_heads={n_q_heads} must be a multiple of the cache's {k_pages.shape[1]} kv heads")
    tensors = [("k_pages", k_pages), ("v_pages", v_pages), ("page_table", page_table)]
    for name, x in (("lens", lens), ("seen", seen)):
        if x is not None:
            if tuple(x.shape) != (b,) or x.dtype != torch.int32:
                raise ValueError(f"{name} must be int32 [n_seq] = ({b},)")
            tensors.append((name, x))
    for name, x, dt in (("slot_pos", slot_pos, torch.int32), ("weights", weights, torch.float32)):
        if x is not None:
            if tuple(x.shape) != (b, k_pages.shape[1], slots) or x.dtype != dt:
                raise ValueError(f"{name} must be {dt} [n_seq][n_kv_heads][slots] = ({b}, {k_pages.shape[1]}, {slots})")
            tensors.append((name, x))
    if slot_pos is not None and seen is None:
        raise ValueError("slot_pos needs seen")
    for name, x in tensors:
        if not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    for name, x in tensors:
        if x.device.type != "cuda" or x.device != k_pages.device:
            raise ValueError(f"{name} must be on the GPU, on k_pages' device; got {x.device}")


class Rotary:
    """The table of a rotary position encoding (gmc_rotary), which it keeps alive.

    ``cos`` / ``sin`` [n_pos][rot_dim / 2] float32 on the GPU: of the angle of each
    pair at each position.  ``interleaved``: a pair is two neighbouring elements,
    not one of each half.  ``sections`` (t, h, w): how many pairs, in this order,
    turn by each of a token's three positions.
    """

    def __init__(self, cos, sin, *, interleaved=False, sections=None):
        import torch
        if cos.dim() != 2 or cos.dtype != torch.float32 or cos.shape != sin.shape or sin.dtype != torch.float32:
            raise ValueError("cos and sin must be float32 [n_pos][rot_dim / 2] of one shape, got "
                             f"{cos.dtype} {tuple(cos.shape)} and {sin.dtype} {tuple(sin.shape)}")
        if cos.shape[0] < 1 or cos.shape[1] < 8 or cos.shape[1] % 8 != 0:
            raise ValueError(f"rot_dim={2 * cos.shape[1]} must be a positive multiple of 16, with at least one position")
        if not cos.is_contiguous() or not sin.is_contiguous():
            raise ValueError("cos and sin must be contiguous")
        if cos.device.type != "cuda" or sin.device != cos.device:
            raise ValueError(f"cos and sin must be on one GPU; got {cos.device} and {sin.device}")
        if sections is not None:
            sections = tuple(int(n) for n in sections)
            if len(sections) != 3 or any(n < 0 or n % 4 for n in sections) or sum(sections) != cos.shape[1]:
                raise ValueError(f"sections={sections} must be three multiples of 4 that hold {cos.shape[1]} pairs")
        self.cos, self.sin, self.sections, self.device = cos, sin, sections, cos.device
        self.desc = GmcRotary(cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], int(bool(interleaved)),
                              (_i32 * 3)(*(sections or (0, 0, 0))))
        self._ref = ctypes.byref(self.desc)

    @classmethod
    def create(cls, n_pos, rot_dim, *, base=10000.0, device="cuda", **more):
        """The angles position * base ** (-2 j / rot_dim) of pairs j, formed in
        64 bits (in 32 their rounding alone is up to 4e-3 from 2^16 on, which
        the second pair's reaches at position 10^5)."""
        import torch
        if n_pos < 1 or rot_dim < 16 or rot_dim % 16 != 0:
            raise ValueError(f"n_pos={n_pos} must be at least 1 and rot_dim={rot_dim} a positive multiple of 16")
        f = float(base) ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
        angle = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * f
        return cls(torch.cos(angle).float(), torch.sin(angle).float(), **more)


class KvCache:
    """One layer's paged K/V cache of a batch of sequences (gmc_cache): the
    tensors, which the wrapper keeps alive, and the calls on them on torch's
    current stream.  Needs no Pruner.

    ``k_pages`` / ``v_pages`` [n_pages][n_kv_heads][page_size][head_dim],
    ``page_table`` [n_seq][max_pages] int32, ``lens`` [n_seq] int32; for a cache
    that evicts also ``seen`` [n_seq] int32, ``slot_pos``
    [n_seq][n_kv_heads][slots] int32 and ``weights`` of the same shape, float32.
    The calls work on these very tensors: change them in place.
    Sequences may share pages that are only read, not those that are appended to
    or evicted from.
    """

    def __init__(self, k_pages, v_pages, page_table, lens, *, n_q_heads, slot_pos=None, seen=None, weights=None):
        check_cache_tensors(k_pages, v_pages, page_table, lens, n_q_heads, slot_pos, seen, weights)
        self.k_pages, self.v_pages = k_pages, v_pages
        self.slot_pos, self.seen, self.weights = slot_pos, seen, weights
        n_pages, hkv, page, dh = k_pages.shape
        ptr = (lambda t: None if t is None else t.data_ptr())
        self._start(k_pages.device, k_pages.dtype, page_table, lens, n_q_heads, hkv, page, dh)
        self.desc = GmcCache(GMC_BF16 if self.dtype == self.torch.bfloat16 else GMC_F32, n_q_heads, hkv, dh, page,
                             page_table.shape[1], n_pages, self.n_seq, ptr(k_pages), ptr(v_pages), ptr(page_table),
                             ptr(lens), ptr(seen), ptr(slot_pos), ptr(weights))
        self._ref = ctypes.byref(self.desc)

    _kind = "gmc_cache_"    # what the names of its entry points begin with

    def _start(self, device, dtype, page_table, lens, n_q_heads, hkv, page, dh):
        import torch
        self.torch, self.device, self.dtype, self.page_table, self.lens = torch, device, dtype, page_table, lens
        self.n_seq, self.slots = page_table.shape[0], page_table.shape[1] * page
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, hkv, dh
        self._scale = dh ** -0.5
        self._index_of_device = self.device.index
        self._current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        # (the address alone: a Stream object takes longer than the call)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda i: torch.cuda.current_stream(i).cuda_stream)
        self._entry = {n: getattr(lib(), n) for n in SIGNATURES if n.startswith(self._kind)}
        self._need = {}

    @classmethod
    def create(cls, *, n_seq, slots, n_q_heads, n_kv_heads, head_dim, dtype, device="cuda", page_size=64,
               evicts=False):
        """An empty cache of `slots` slots a sequence (rounded up to whole
        pages), its pages in order; ``evicts`` adds positions and weights."""
        import torch
        if n_seq < 1 or slots < 1 or page_size < 1:
            raise ValueError(f"n_seq={n_seq}, slots={slots} and page_size={page_size} must be at least 1")
        per = -(-slots // page_size)
        pages = [torch.zeros((n_seq * per, n_kv_heads, page_size, head_dim), dtype=dtype, device=device) for _ in "kv"]
        table = torch.arange(n_seq * per, dtype=torch.int32, device=device).view(n_seq, per)
        lens = torch.zeros(n_seq, dtype=torch.int32, device=device)
        more = {}
        if evicts:
            shape = (n_seq, n_kv_heads, per * page_size)
            more = dict(seen=torch.zeros_like(lens), slot_pos=torch.zeros(shape, dtype=torch.int32, device=device),
                        weights=torch.zeros(shape, dtype=torch.float32, device=device))
        return cls(*pages, table, lens, n_q_heads=n_q_heads, **more)

    def _call(self, name, *args):
        """The entry point on the current stream of the cache's device, which is
        the current device almost always."""
        if self._current_device() == self._index_of_device:
            code = self._entry[name](self._ref, *args, self._raw_stream(self._index_of_device))
        else:
            with self.torch.cuda.device(self.device):
                code = self._entry[name](self._ref, *args, self._raw_stream(self._index_of_device))
        if code != GMC_OK:
            _check(code, name)

    def _scratch(self, name, *what):
        """(tensor or None, its address, its bytes) for a call; sizes are asked for
        once for each `what`, the memory is torch's, of the call's own."""
        need = self._need.get((name, what))
        if need is None:
            need = self._entry[name + "_bytes"](self._ref, *what)
            if need < 0:
                _check(int(need), name)
            self._need[name, what] = need
        if need == 0:
            return None, None, 0
        x = self.torch.empty(need, dtype=self.torch.uint8, device=self.device)
        return x, x.data_ptr(), need

    def _rows(self, name, x, heads):
        """Tokens x heads x head_dim in the cache's dtype, each token's heads in
        one run; returns the tokens' stride."""
        shape, strides, row = x.shape, x.stride(), heads * self.head_dim
        if len(shape) != 3 or shape[1] != heads or shape[2] != self.head_dim or x.dtype != self.dtype:
            raise ValueError(f"{name} must be {self.dtype} [tokens][{heads}][{self.head_dim}], got {x.dtype} "
                             f"{tuple(shape)}")
        if x.device != self.device:
            raise ValueError(f"{name} must be on the cache's device {self.device}; got {x.device}")
        stride = strides[0] if shape[0] > 1 else row
        if strides[2] != 1 or (heads > 1 and strides[1] != self.head_dim) or stride < row:
            raise ValueError(f"{name} must hold each token's heads in one run, got strides {strides}")
        return stride

    def _index(self, name, x, shape):
        if x.dtype != self.torch.int32 or tuple(x.shape) != shape or not x.is_contiguous() or x.device != self.device:
            raise ValueError(f"{name} must be a contiguous int32 {shape} tensor on the cache's device")
        return x.data_ptr()

    def _new(self, rows, starts, max_new):
        if starts is not None:
            if max_new is None:
                raise ValueError("starts needs max_new, the most new tokens of a sequence")
            return self._index("starts", starts, (self.n_seq + 1,)), max_new
        if rows % self.n_seq != 0 or (max_new is not None and max_new * self.n_seq != rows):
            raise ValueError(f"without starts the {rows} rows must be the same number for each of {self.n_seq} sequences")
        return None, rows // self.n_seq

    def append(self, k, v, *, starts=None, max_new=None, src=None):
        """gmc_cache_append: k, v [tokens][n_kv_heads][head_dim] (tokens may be
        strided); ``starts`` [n_seq + 1] int32 with ``max_new`` for ragged
        rows, or ``src`` [n_seq][n] int32, the rows of each sequence to take."""
        self._call("gmc_cache_append", *self._appended(k, v, starts, max_new, src))

    def _appended(self, k, v, starts, max_new, src):
        """Addresses of k and v, their strides, rows, addresses of starts and src, max_new."""
        sk, sv = self._rows("k", k, self.n_kv_heads), self._rows("v", v, self.n_kv_heads)
        rows = k.shape[0]
        if v.shape[0] != rows:
            raise ValueError(f"k and v hold {rows} and {v.shape[0]} tokens")
        if src is not None:
            if starts is not None:
                raise ValueError("src and starts must not both be given")
            n = src.shape[1] if src.dim() == 2 else 0
            if max_new is not None and max_new != n:
                raise ValueError(f"max_new={max_new} must be the {n} columns of src, or not be given")
            first, max_new, taken = None, n, self._index("src", src, (self.n_seq, n))
        else:
            (first, max_new), taken = self._new(rows, starts, max_new), None
        return k.data_ptr(), v.data_ptr(), sk, sv, rows, first, taken, max_new

    def append_rotary(self, k, v, rotary, *, pos=None, q=None, starts=None, max_new=None, src=None, out=None):
        """gmc_cache_append_rotary: append with k rotated by ``rotary`` (a Rotary)
        on the way.  ``pos`` int32 [tokens], or [tokens][3] where the rotary has
        sections; None: the slots' positions, which are not those of an answer to a
        pruned prompt (see gmc_cache_append_rotary).  ``q`` [tokens][n_q_heads][head_dim]:
        the tokens' queries; their rotated ones are returned (in ``out`` if given,
        which without src may be q), [n_seq * n][n_q_heads][head_dim] with src."""
        rows = self._appended(k, v, starts, max_new, src)
        tokens = rows[4]
        if rotary.device != self.device:
            raise ValueError(f"rotary must be on the cache's device {self.device}; got {rotary.device}")
        p = None if pos is None else self._index("pos", pos, (tokens, 3) if rotary.sections else (tokens,))
        if q is None:
            if out is not None:
                raise ValueError("out needs q")
            self._call(self._turned, rotary._ref, *rows, p, None, 0, None)
            return None
        stride = self._rows("q", q, self.n_q_heads)
        if q.shape[0] != tokens:
            raise ValueError(f"q and k hold {q.shape[0]} and {tokens} tokens")
        shape = (tokens if src is None else self.n_seq * rows[7], self.n_q_heads, self.head_dim)
        if out is None:
            out = q.new_empty(shape)
        elif tuple(out.shape) != shape or out.dtype != self.dtype or not out.is_contiguous() or out.device != self.device:
            raise ValueError(f"out must be a contiguous {self.dtype} {shape} tensor on the cache's device")
        self._call(self._turned, rotary._ref, *rows, p, q.data_ptr(), stride, out.data_ptr())
        return out

    _turned = "gmc_cache_append_rotary"

    def _outputs(self, q, out, lse):
        torch = self.torch
        shape = (q.shape[0], self.n_q_heads, self.head_dim)
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)   # (q has been checked)
        elif tuple(out.shape) != shape or out.dtype != self.dtype or not out.is_contiguous() or out.device != self.device:
            raise ValueError(f"out must be a contiguous {self.dtype} {shape} tensor on the cache's device")
        if lse is True:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=self.device)
        elif lse is False:
            lse = None
        elif lse is not None and (tuple(lse.shape) != shape[:2] or lse.dtype != torch.float32 or
                                  not lse.is_contiguous() or lse.device != self.device):
            raise ValueError(f"lse must be a contiguous float32 {shape[:2]} tensor on the cache's device")
        return out, lse

    def prefill(self, q, *, starts=None, max_new=None, window=0, sinks=0, scale=None, lse=False, out=None):
        """gmc_cache_prefill: q [tokens][n_q_heads][head_dim] of the newest
        tokens (appended before), the same number for every sequence or ragged by
        ``starts`` / ``max_new``.  Returns out, or (out, lse) with ``lse`` True or
        a tensor to fill.  Rows of no sequence are left as ``out`` holds them."""
        stride = self._rows("q", q, self.n_q_heads)
        first, max_new = self._new(q.shape[0], starts, max_new)
        out, ls = self._outputs(q, out, lse)
        ws, at, size = self._scratch(self._kind + "prefill", max_new)
        self._call(self._kind + "prefill", q.data_ptr(), stride, q.shape[0], first, max_new,
                   self._scale if scale is None else scale, window, sinks, out.data_ptr(),
                   None if ls is None else ls.data_ptr(), at, size)
        return out if ls is None else (out, ls)

    def decode(self, q, *, window=0, sinks=0, scale=None, accumulate=False, lse=False, out=None):
        """gmc_cache_decode: q [n_seq][n_q_heads][head_dim], one token a
        sequence (appended before).  ``accumulate`` adds its attention weights to
        ``weights``.  Returns as prefill."""
        stride = self._rows("q", q, self.n_q_heads)
        if q.shape[0] != self.n_seq:
            raise ValueError(f"q must hold one token for each of {self.n_seq} sequences, got {q.shape[0]}")
        out, ls = self._outputs(q, out, lse)
        ws, at, size = self._scratch("gmc_cache_decode", 1 if accumulate else 0)
        self._call("gmc_cache_decode", q.data_ptr(), stride, self._scale if scale is None else scale, window, sinks,
                   1 if accumulate else 0, out.data_ptr(), None if ls is None else ls.data_ptr(), at, size)
        return out if ls is None else (out, ls)

    def evict(self, budget, *, sinks=0, recent=0):
        """gmc_cache_evict: every sequence keeps at most ``budget`` rows a kv
        head, the first ``sinks`` and last ``recent`` positions among them."""
        ws, at, size = self._scratch("gmc_cache_evict", budget)
        self._call("gmc_cache_evict", budget, sinks, recent, at, size)


def check_cache4_tensors(k_codes, v_codes, k_scales, v_scales, page_table, lens, n_q_heads, dtype):
    """Shapes, dtypes and devices of the tensors of a cache of 4 bits (see
    gmc_cache4).  Raises ValueError."""
    import torch
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"dtype must be float32 or bfloat16, got {dtype}")
    if k_codes.dim() != 4 or k_codes.dtype != torch.uint8 or k_codes.shape[3] < 16 or k_codes.shape[3] % 16 != 0:
        raise ValueError("k_codes must be uint8 [n_pages][n_kv_heads][page_size][head_dim / 2], head_dim a multiple of "
                         f"32, got {k_codes.dtype} {tuple(k_codes.shape)}")
    if v_codes.shape != k_codes.shape or v_codes.dtype != torch.uint8:
        raise ValueError("v_codes must have k_codes' shape and dtype")
    want = tuple(k_codes.shape[:3]) + (cache4_scale_bytes(2 * k_codes.shape[3]),)
    for name, x in (("k_scales", k_scales), ("v_scales", v_scales)):
        if tuple(x.shape) != want or x.dtype != torch.uint8:
            raise ValueError(f"{name} must be uint8 {want}, got {x.dtype} {tuple(x.shape)}")
    if page_table.dim() != 2 or page_table.dtype != torch.int32:
        raise ValueError("page_table must be int32 [n_seq][max_pages]")
    if k_codes.numel() == 0 or page_table.numel() == 0:
        raise ValueError(f"k_codes {tuple(k_codes.shape)} and page_table {tuple(page_table.shape)} must not be empty")
    if n_q_heads < 1 or n_q_heads % k_codes.shape[1] != 0:
        raise ValueError(f"n_q_heads={n_q_heads} must be a multiple of the cache's {k_codes.shape[1]} kv heads")
    if tuple(lens.shape) != (page_table.shape[0],) or lens.dtype != torch.int32:
        raise ValueError(f"lens must be int32 [n_seq] = ({page_table.shape[0]},)")
    tensors = [("k_codes", k_codes), ("v_codes", v_codes), ("k_scales", k_scales), ("v_scales", v_scales),
               ("page_table", page_table), ("lens", lens)]
    for name, x in tensors:
        if not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    for name, x in tensors:
        if x.device.type != "cuda" or x.device != k_codes.device:
            raise ValueError(f"{name} must be on the GPU, on k_codes' device; got {x.device}")


def cache4_scale_bytes(head_dim):
    """Bytes of the scales of a row of a cache of 4 bits."""
    return 1 << (head_dim // 32 - 1).bit_length()


class KvCache4(KvCache):
    """One layer's paged K/V cache of a batch of sequences in 4 bits, 4.25 with
    the scales (gmc_cache4): KvCache's calls but evict, and read.

    ``k_codes`` / ``v_codes`` [n_pages][n_kv_heads][page_size][head_dim / 2] uint8,
    ``k_scales`` / ``v_scales`` [n_pages][n_kv_heads][page_size][head_dim / 32,
    rounded up to a power of two] uint8, ``page_table`` and ``lens`` as KvCache's;
    ``dtype`` is that of k, v, q and the outputs.  Sharing pages as with KvCache.
    """

    def __init__(self, k_codes, v_codes, k_scales, v_scales, page_table, lens, *, n_q_heads, dtype):
        check_cache4_tensors(k_codes, v_codes, k_scales, v_scales, page_table, lens, n_q_heads, dtype)
        self.k_codes, self.v_codes, self.k_scales, self.v_scales = k_codes, v_codes, k_scales, v_scales
        n_pages, hkv, page, half = k_codes.shape
        self._start(k_codes.device, dtype, page_table, lens, n_q_heads, hkv, page, 2 * half)
        self.desc = GmcCache4(GMC_BF16 if dtype == self.torch.bfloat16 else GMC_F32, n_q_heads, hkv, 2 * half, page,
                              page_table.shape[1], n_pages, self.n_seq,
                              *(x.data_ptr() for x in (k_codes, v_codes, k_scales, v_scales, page_table, lens)))
        self._ref = ctypes.byref(self.desc)

    _kind = "gmc_cache4_"
    _turned = "gmc_cache4_append"

    @classmethod
    def create(cls, *, n_seq, slots, n_q_heads, n_kv_heads, head_dim, dtype, device="cuda", page_size=64):
        """An empty cache of `slots` slots a sequence (rounded up to whole
        pages), its pages in order."""
        import torch
        if n_seq < 1 or slots < 1 or page_size < 1:
            raise ValueError(f"n_seq={n_seq}, slots={slots} and page_size={page_size} must be at least 1")
        if head_dim < 32 or head_dim % 32 != 0:
            raise ValueError(f"head_dim={head_dim} must be a positive multiple of 32")
        per = -(-slots // page_size)
        rows = (n_seq * per, n_kv_heads, page_size)
        new = [torch.zeros(rows + (n,), dtype=torch.uint8, device=device)
               for n in (head_dim // 2, head_dim // 2, cache4_scale_bytes(head_dim), cache4_scale_bytes(head_dim))]
        table = torch.arange(n_seq * per, dtype=torch.int32, device=device).view(n_seq, per)
        lens = torch.zeros(n_seq, dtype=torch.int32, device=device)
        return cls(*new, table, lens, n_q_heads=n_q_heads, dtype=dtype)

    def append(self, k, v, *, starts=None, max_new=None, src=None):
        """gmc_cache4_append without rotation: as KvCache.append, each block of 32
        elements to the nearest values of 4 bits and a power of two."""
        self._call("gmc_cache4_append", None, *self._appended(k, v, starts, max_new, src), None, None, 0, None)

    def read(self, rows=None, *, starts=None, max_new=None):
        """gmc_cache4_read: the newest slots' values as (k, v) [tokens][n_kv_heads]
        [head_dim], ``max_new`` of each sequence, or ragged by ``starts`` in
        tensors of ``rows`` rows (those of no sequence are not written)."""
        if starts is None:
            if max_new is None or (rows is not None and rows != self.n_seq * max_new):
                raise ValueError(f"without starts read needs max_new, and rows={rows} must be n_seq * max_new or not given")
            rows = self.n_seq * max_new
        elif rows is None:
            raise ValueError("starts needs rows, the rows of the outputs")
        if rows < 1:
            raise ValueError(f"rows={rows} must be at least 1")
        first, max_new = self._new(rows, starts, max_new)
        k, v = self.torch.empty((2, rows, self.n_kv_heads, self.head_dim), dtype=self.dtype, device=self.device).unbind()
        self._call("gmc_cache4_read", rows, first, max_new, k.data_ptr(), v.data_ptr())
        return k, v

    def decode(self, q, *, window=0, sinks=0, scale=None, lse=False, out=None):
        """gmc_cache4_decode: as KvCache.decode; no weights are accumulated."""
        stride = self._rows("q", q, self.n_q_heads)
        if q.shape[0] != self.n_seq:
            raise ValueError(f"q must hold one token for each of {self.n_seq} sequences, got {q.shape[0]}")
        out, ls = self._outputs(q, out, lse)
        ws, at, size = self._scratch("gmc_cache4_decode")
        self._call("gmc_cache4_decode", q.data_ptr(), stride, self._scale if scale is None else scale, window, sinks,
                   out.data_ptr(), None if ls is None else ls.data_ptr(), at, size)
        return out if ls is None else (out, ls)

    def evict(self, budget, *, sinks=0, recent=0):
        raise TypeError("a cache of 4 bits keeps its rows: slots have no weights and positions to evict by")


def gmc_timing_enable(enable: bool) -> int:
    return lib().gmc_timing_enable(1 if enable else 0)


def gmc_timing_read():
    """Per-stage (total ms, span count) since the last read (syncs the stream)."""
    n = GMC_TIMERS
    ms = (ctypes.c_double * n)()
    cnt = (_i64 * n)()
    _check(lib().gmc_timing_read(ms, cnt, n), "gmc_timing_read")
    return list(ms), list(cnt)


GMC_TIMERS = 13
STAGE_NAMES = ["probe", "logits", "heads", "appearance", "spatial", "cov", "gains", "resp",
               "objective", "assign", "transport", "init", "select"]
SIGNATURES["gmc_timing_enable"] = (ctypes.c_int, [ctypes.c_int])
SIGNATURES["gmc_timing_read"] = (ctypes.c_int, [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_i64),
                                                ctypes.c_int32])


# --- host <-> device marshalling of seeded workloads --------------------------
def to_device(a, dtype: str, torch):
    """A float32 numpy array holding exact values of `dtype` ("f32" or
    "bf16") as a contiguous device tensor of that dtype."""
    from . import synth
    if dtype == "bf16":
        bits = synth.bf16_bits(a).view(np.int16)
        return torch.from_numpy(np.ascontiguousarray(bits)).view(torch.bfloat16).cuda()
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def from_device(t, torch) -> np.ndarray:
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def make_pruner(prob, torch, max_k=0, probe_bias=None, hist=None, **overrides) -> Pruner:
    """A Pruner sized for a seeded workload (synth.Problem): its shape, dtype,
    batch and token capacity, probe and bounded-bank projection, and the
    probes of its historical views (synth.HistView list) when given."""
    w = prob.workload
    tdt = torch.bfloat16 if w.dtype == "bf16" else torch.float32
    probe = to_device(prob.probe, w.dtype, torch)
    proj = None if prob.app_proj is None else to_device(prob.app_proj, w.dtype, torch)
    bias = None if probe_bias is None else torch.from_numpy(np.ascontiguousarray(probe_bias, np.float32)).cuda()
    ph = None if not hist else to_device(np.stack([v.probe for v in hist]), w.dtype, torch)
    return Pruner(d=w.d, n_q_heads=w.hq, n_kv_heads=w.hkv, head_dim=w.dh, probe=probe, dtype=tdt,
                  max_batch=w.batch, max_n=w.n, max_t=max(w.t, 1), max_k=max_k, app_projection=proj,
                  probe_bias=bias, probe_hist=ph, **overrides)
