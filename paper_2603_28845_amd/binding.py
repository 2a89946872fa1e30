"""ctypes binding of libonecomp.so: argument marshalling only.

Each function has the name of the C entry point it calls (include/onecomp.h) and
takes torch tensors that live on the GPU; torch supplies device memory and the
current HIP stream, every step of the computation runs in the library's kernels.
There is no CPU fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
from typing import Optional, Sequence, Tuple

import torch  # imported before the library so that both share one HIP runtime

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libonecomp.so")

ONECOMP_OK = 0
ONECOMP_F32 = 0
ONECOMP_BF16 = 1
ONECOMP_GRID_MINMAX = 0
ONECOMP_GRID_SYMMETRIC = 1
ONECOMP_GRID_MINMAX_MSE = 2
ONECOMP_GRID_SYMMETRIC_MSE = 3
_GRIDS = {"minmax": ONECOMP_GRID_MINMAX, "symmetric": ONECOMP_GRID_SYMMETRIC, "minmax_mse": ONECOMP_GRID_MINMAX_MSE,
          "symmetric_mse": ONECOMP_GRID_SYMMETRIC_MSE}
ONECOMP_FACTOR_INVERSE = 0
ONECOMP_FACTOR_BLOCK = 1

EXPORTED_SYMBOLS = (
    "onecomp_hessian_accumulate",
    "onecomp_hessian_factor",
    "onecomp_quantize_layer",
    "onecomp_quantize_layer_grid",
    "onecomp_hessian_factor_form",
    "onecomp_hessian_accumulate_ws",
    "onecomp_accumulate_workspace_bytes",
    "onecomp_accumulate_describe",
    "onecomp_mfma_rate_probe",
    "onecomp_quantize_layer_form",
    "onecomp_factor_workspace_bytes",
    "onecomp_quantize_workspace_bytes",
    "onecomp_crossgram_accumulate",
    "onecomp_qep_target",
    "onecomp_qep_workspace_bytes",
    "onecomp_rtn_sensitivity",
    "onecomp_sensitivity_workspace_bytes",
    "onecomp_rtn_sensitivity_static",
    "onecomp_jointq_refine",
    "onecomp_jointq_workspace_bytes",
    "onecomp_attention_forward",
    "onecomp_attention_workspace_bytes",
    "onecomp_attention_backward",
    "onecomp_attention_backward_workspace_bytes",
    "onecomp_block_norm_forward",
    "onecomp_block_norm_backward",
    "onecomp_block_norm_workspace_bytes",
    "onecomp_clip_gradients",
    "onecomp_clip_workspace_bytes",
    "onecomp_status_string",
    "onecomp_version",
)

_lib = None


class Heads(ctypes.Structure):
    """onecomp_heads"""
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class AttentionShape(ctypes.Structure):
    """onecomp_attention_shape"""
    _fields_ = [("dtype", ctypes.c_int), ("n_heads", ctypes.c_int), ("n_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("n_seqs", ctypes.c_int), ("causal", ctypes.c_int), ("scale", ctypes.c_float), ("total_q", ctypes.c_int64),
                ("total_k", ctypes.c_int64), ("max_q", ctypes.c_int64), ("max_k", ctypes.c_int64), ("cu_q", ctypes.c_void_p),
                ("cu_k", ctypes.c_void_p), ("len_k", ctypes.c_void_p)]


class Rows(ctypes.Structure):
    """onecomp_rows"""
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64)]


class NormShape(ctypes.Structure):
    """onecomp_norm_shape"""
    _fields_ = [("dtype", ctypes.c_int), ("w_dtype", ctypes.c_int), ("kind", ctypes.c_int), ("gate_kind", ctypes.c_int),
                ("post_norm", ctypes.c_int), ("rows", ctypes.c_int64), ("width", ctypes.c_int64), ("residual_scale", ctypes.c_float),
                ("eps", ctypes.c_float)]


class NormGradients(ctypes.Structure):
    """onecomp_norm_gradients"""
    _fields_ = [("dh", ctypes.POINTER(Rows)), ("dy", ctypes.POINTER(Rows)), ("dgate", ctypes.POINTER(Rows)), ("dweight", ctypes.c_void_p),
                ("dbias", ctypes.c_void_p), ("dpost_weight", ctypes.c_void_p), ("dpost_bias", ctypes.c_void_p),
                ("dgate_channel", ctypes.c_void_p)]


class Gradient(ctypes.Structure):
    """onecomp_gradient"""
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("numel", ctypes.c_int64), ("dtype", ctypes.c_int)]


class OnecompError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (status {code})")


def load_library() -> ctypes.CDLL:
    """Load libonecomp.so (once) and declare its prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2603_28845_amd.build` "
            "(or __graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, f32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.onecomp_hessian_accumulate.argtypes = [vp, i32, i64, i64, i64, vp, vp]
    lib.onecomp_hessian_accumulate.restype = i32
    lib.onecomp_hessian_factor.argtypes = [vp, i64, f32, i32, vp, vp, vp, vp, sz, vp]
    lib.onecomp_hessian_factor.restype = i32
    lib.onecomp_hessian_accumulate_ws.argtypes = [vp, i32, i64, i64, i64, vp, vp, sz, vp]
    lib.onecomp_hessian_accumulate_ws.restype = i32
    lib.onecomp_accumulate_workspace_bytes.argtypes = [i32, i64]
    lib.onecomp_accumulate_workspace_bytes.restype = sz
    lib.onecomp_accumulate_describe.argtypes = [i32, i64, i64, i64, sz, vp]
    lib.onecomp_accumulate_describe.restype = i32
    lib.onecomp_mfma_rate_probe.argtypes = [i32, i32, i32, i64, vp, vp, vp]
    lib.onecomp_mfma_rate_probe.restype = i32
    lib.onecomp_hessian_factor_form.argtypes = [vp, i64, f32, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.onecomp_hessian_factor_form.restype = i32
    lib.onecomp_quantize_layer_form.argtypes = [vp, i32, i64, i64, vp, i32, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp,
                                                vp, sz, vp]
    lib.onecomp_quantize_layer_form.restype = i32
    lib.onecomp_quantize_layer.argtypes = [vp, i32, i64, i64, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.onecomp_quantize_layer.restype = i32
    lib.onecomp_quantize_layer_grid.argtypes = [vp, i32, i64, i64, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz,
                                                vp]
    lib.onecomp_quantize_layer_grid.restype = i32
    lib.onecomp_factor_workspace_bytes.argtypes = [i64]
    lib.onecomp_factor_workspace_bytes.restype = sz
    lib.onecomp_quantize_workspace_bytes.argtypes = [i64, i64, i32]
    lib.onecomp_quantize_workspace_bytes.restype = sz
    lib.onecomp_crossgram_accumulate.argtypes = [vp, vp, i32, i64, i64, i64, i64, vp, vp]
    lib.onecomp_crossgram_accumulate.restype = i32
    lib.onecomp_qep_target.argtypes = [vp, i32, i64, i64, vp, vp, vp, vp, f32, vp, vp, sz, vp]
    lib.onecomp_qep_target.restype = i32
    lib.onecomp_qep_workspace_bytes.argtypes = [i64, i64]
    lib.onecomp_qep_workspace_bytes.restype = sz
    lib.onecomp_rtn_sensitivity.argtypes = [vp, i32, i64, i64, vp, vp, i32, i32, i32, vp, vp, sz, vp]
    lib.onecomp_rtn_sensitivity.restype = i32
    lib.onecomp_rtn_sensitivity_static.argtypes = [vp, i32, i64, i64, vp, vp, i32, i32, i32, vp, vp]
    lib.onecomp_rtn_sensitivity_static.restype = i32
    lib.onecomp_sensitivity_workspace_bytes.argtypes = []
    lib.onecomp_sensitivity_workspace_bytes.restype = sz
    lib.onecomp_jointq_refine.argtypes = [vp, i32, i64, i64, vp, vp, f32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp,
                                          vp, sz, vp]
    lib.onecomp_jointq_refine.restype = i32
    lib.onecomp_jointq_workspace_bytes.argtypes = [i64, i64, i32]
    lib.onecomp_jointq_workspace_bytes.restype = sz
    # structures go by address: an int, or ctypes.byref of the classes above
    lib.onecomp_attention_forward.argtypes = [vp] * 7 + [sz, vp]
    lib.onecomp_attention_forward.restype = i32
    lib.onecomp_attention_workspace_bytes.argtypes = [vp]
    lib.onecomp_attention_workspace_bytes.restype = sz
    lib.onecomp_attention_backward.argtypes = [vp] * 11 + [sz, vp]
    lib.onecomp_attention_backward.restype = i32
    lib.onecomp_attention_backward_workspace_bytes.argtypes = [vp]
    lib.onecomp_attention_backward_workspace_bytes.restype = sz
    lib.onecomp_block_norm_forward.argtypes = [vp] * 11
    lib.onecomp_block_norm_forward.restype = i32
    lib.onecomp_block_norm_backward.argtypes = [vp] * 11 + [sz, vp]
    lib.onecomp_block_norm_backward.restype = i32
    lib.onecomp_block_norm_workspace_bytes.argtypes = [vp]
    lib.onecomp_block_norm_workspace_bytes.restype = sz
    lib.onecomp_clip_gradients.argtypes = [vp, i32, f32, vp, vp, sz, vp]
    lib.onecomp_clip_gradients.restype = i32
    lib.onecomp_clip_workspace_bytes.argtypes = []
    lib.onecomp_clip_workspace_bytes.restype = sz
    lib.onecomp_status_string.argtypes = [i32]
    lib.onecomp_status_string.restype = ctypes.c_char_p
    lib.onecomp_version.argtypes = []
    lib.onecomp_version.restype = i32
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load_library().onecomp_status_string(int(code)).decode()


def onecomp_version() -> int:
    return int(load_library().onecomp_version())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return ONECOMP_F32
    if t.dtype == torch.bfloat16:
        return ONECOMP_BF16
    raise TypeError(f"unsupported dtype {t.dtype}: float32 or bfloat16 expected")


def _dev(t: torch.Tensor, name: str, dtype=None, contiguous=True):
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t: Optional[torch.Tensor]):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)


def onecomp_factor_workspace_bytes(d_in: int) -> int:
    return int(load_library().onecomp_factor_workspace_bytes(int(d_in)))


def onecomp_quantize_workspace_bytes(d_out: int, d_in: int, block_size: int = 128) -> int:
    return int(load_library().onecomp_quantize_workspace_bytes(int(d_out), int(d_in), int(block_size)))


def onecomp_accumulate_workspace_bytes(dtype: torch.dtype, d_in: int) -> int:
    code = ONECOMP_BF16 if dtype == torch.bfloat16 else ONECOMP_F32
    return int(load_library().onecomp_accumulate_workspace_bytes(code, int(d_in)))


def onecomp_accumulate_describe(dtype: torch.dtype, n_tokens: int, d_in: int, workspace_bytes: int = 0,
                                ldx: Optional[int] = None) -> dict:
    """How an accumulate call of this size would run: tile shape of its main kernel and launches of it per call."""
    code = ONECOMP_BF16 if dtype == torch.bfloat16 else ONECOMP_F32
    out = (ctypes.c_int32 * 3)()
    rc = load_library().onecomp_accumulate_describe(code, int(n_tokens), int(d_in), int(d_in if ldx is None else ldx),
                                                    int(workspace_bytes), ctypes.cast(out, ctypes.c_void_p))
    if rc != 0:
        raise OnecompError(rc, "onecomp_accumulate_describe")
    return {"tile_rows": int(out[0]), "tile_cols": int(out[1]), "launches": int(out[2])}


def onecomp_mfma_rate_probe(kind: str, waves_per_simd: int, iters: int, sink: torch.Tensor,
                            random_operands: bool = True) -> float:
    """Enqueues the register-only MFMA loop (kind "bf16" or "f64") on the current stream; returns its flop count."""
    flops = ctypes.c_double(0.0)
    rc = load_library().onecomp_mfma_rate_probe({"bf16": 0, "f64": 1}[kind], int(waves_per_simd),
                                                int(bool(random_operands)), int(iters),
                                                _ptr(sink), ctypes.cast(ctypes.byref(flops), ctypes.c_void_p),
                                                _stream())
    if rc != 0:
        raise OnecompError(rc, "onecomp_mfma_rate_probe")
    return float(flops.value)


def onecomp_hessian_accumulate(X: torch.Tensor, H: torch.Tensor, workspace: Optional[torch.Tensor] = None) -> None:
    """H += 2 X^T X.  X: [n_tokens, d_in] fp32/bf16 (rows may be strided), H: [d_in, d_in] fp32.
    workspace (uint8 device tensor, see onecomp_accumulate_workspace_bytes) selects onecomp_hessian_accumulate_ws."""
    lib = load_library()
    if X.dim() != 2 or H.dim() != 2 or H.shape[0] != H.shape[1] or H.shape[0] != X.shape[1]:
        raise ValueError("shapes: X [n_tokens, d_in], H [d_in, d_in]")
    if X.shape[0] > 0 and X.stride(1) != 1:
        raise ValueError("X rows must be dense")
    _dev(X, "X", contiguous=False)
    ldx = X.stride(0) if X.shape[0] > 1 else X.shape[1]
    if workspace is None:
        rc = lib.onecomp_hessian_accumulate(_ptr(X), _dtype_code(X), X.shape[0], X.shape[1], ldx,
                                            _dev(H, "H", torch.float32), _stream())
    else:
        rc = lib.onecomp_hessian_accumulate_ws(_ptr(X), _dtype_code(X), X.shape[0], X.shape[1], ldx,
                                               _dev(H, "H", torch.float32), _dev(workspace, "workspace", torch.uint8),
                                               workspace.numel(), _stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_hessian_accumulate")


def onecomp_hessian_factor(H: torch.Tensor, damp: float, act_order: bool = False,
                           U: Optional[torch.Tensor] = None, perm_out: Optional[torch.Tensor] = None,
                           info: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                           form: str = "inverse") -> Tuple[torch.Tensor, Optional[torch.Tensor], torch.Tensor]:
    """Returns (U, perm, info) as device tensors; perm is None when act_order is False and no perm_out was given.
    form = "inverse" calls onecomp_hessian_factor, "block" onecomp_hessian_factor_form with ONECOMP_FACTOR_BLOCK
    (the matrix returned is then meant for onecomp_quantize_layer(..., form="block") only)."""
    lib = load_library()
    d = H.shape[0]
    if U is None:
        U = torch.empty((d, d), dtype=torch.float32, device=H.device)
    if info is None:
        info = torch.zeros(1, dtype=torch.int32, device=H.device)
    if act_order and perm_out is None:
        perm_out = torch.empty(d, dtype=torch.int32, device=H.device)
    need = onecomp_factor_workspace_bytes(d)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=H.device)
    tail = (_ptr(perm_out), _dev(U, "U", torch.float32), _dev(info, "info", torch.int32),
            _dev(workspace, "workspace", torch.uint8), workspace.numel(), _stream())
    if form == "inverse":
        rc = lib.onecomp_hessian_factor(_dev(H, "H", torch.float32), d, float(damp), int(bool(act_order)), *tail)
    elif form == "block":
        rc = lib.onecomp_hessian_factor_form(_dev(H, "H", torch.float32), d, float(damp), int(bool(act_order)),
                                             ONECOMP_FACTOR_BLOCK, *tail)
    else:
        raise ValueError("form must be 'inverse' or 'block'")
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_hessian_factor")
    return U, perm_out, info


def onecomp_quantize_layer(W: torch.Tensor, U: torch.Tensor, bits: int, group_size: int,
                           perm: Optional[torch.Tensor] = None, block_size: int = 128, want_w_hat: bool = True,
                           workspace: Optional[torch.Tensor] = None, out: Optional[dict] = None,
                           grid: str = "minmax", form: str = "inverse") -> dict:
    """Returns dict(Q_codes uint8, scales, zeros, W_hat (or None), loss) of device tensors.
    grid = "minmax" calls onecomp_quantize_layer, "symmetric" onecomp_quantize_layer_grid with that grid;
    "minmax_mse" / "symmetric_mse" (the grid with the scale search) call onecomp_quantize_layer_form;
    form = "block" (U from onecomp_hessian_factor(..., form="block")) calls onecomp_quantize_layer_form."""
    lib = load_library()
    d_out, d_in = W.shape
    dev = W.device
    if out is None:
        n_g = d_in // group_size if group_size > 0 and d_in % group_size == 0 else 1
        out = {
            "Q_codes": torch.empty((d_out, d_in), dtype=torch.uint8, device=dev),
            "scales": torch.empty((d_out, n_g), dtype=torch.float32, device=dev),
            "zeros": torch.empty((d_out, n_g), dtype=torch.float32, device=dev),
            "W_hat": torch.empty((d_out, d_in), dtype=torch.float32, device=dev) if want_w_hat else None,
            "loss": torch.zeros(1, dtype=torch.float32, device=dev),
        }
    need = onecomp_quantize_workspace_bytes(d_out, d_in, block_size)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    if perm is not None:
        _dev(perm, "perm", torch.int32)
    head = (_dev(W, "W"), _dtype_code(W), d_out, d_in, _dev(U, "U", torch.float32), _ptr(perm), int(bits),
            int(group_size), int(block_size))
    tail = (_dev(out["Q_codes"], "Q_codes", torch.uint8), _dev(out["scales"], "scales", torch.float32),
            _dev(out["zeros"], "zeros", torch.float32), _ptr(out["W_hat"]), _dev(out["loss"], "loss", torch.float32),
            _dev(workspace, "workspace", torch.uint8), workspace.numel(), _stream())
    if grid not in _GRIDS:
        raise ValueError("grid must be one of " + ", ".join(sorted(_GRIDS)))
    if form not in ("inverse", "block"):
        raise ValueError("form must be 'inverse' or 'block'")
    if form == "block" or grid.endswith("_mse"):
        rc = lib.onecomp_quantize_layer_form(*head[:5], ONECOMP_FACTOR_BLOCK if form == "block" else ONECOMP_FACTOR_INVERSE,
                                             *head[5:], _GRIDS[grid], *tail)
    elif grid == "minmax":
        rc = lib.onecomp_quantize_layer(*head, *tail)
    else:
        rc = lib.onecomp_quantize_layer_grid(*head, ONECOMP_GRID_SYMMETRIC, *tail)
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_quantize_layer")
    return out


def onecomp_qep_workspace_bytes(d_out: int, d_in: int) -> int:
    return int(load_library().onecomp_qep_workspace_bytes(int(d_out), int(d_in)))


def onecomp_crossgram_accumulate(X_hat: torch.Tensor, X: torch.Tensor, G: torch.Tensor) -> None:
    """G += 2 X_hat^T X.  X_hat, X: [n_tokens, d_in] bf16 (rows may be strided), G: [d_in, d_in] fp32."""
    lib = load_library()
    if X.dim() != 2 or X_hat.shape != X.shape or G.dim() != 2 or G.shape[0] != G.shape[1] or G.shape[0] != X.shape[1]:
        raise ValueError("shapes: X_hat, X [n_tokens, d_in], G [d_in, d_in]")
    if X.shape[0] > 0 and (X.stride(1) != 1 or X_hat.stride(1) != 1):
        raise ValueError("rows of X_hat and X must be dense")
    if X_hat.dtype != X.dtype:
        raise TypeError("X_hat and X must have the same dtype")
    _dev(X, "X", contiguous=False)
    _dev(X_hat, "X_hat", contiguous=False)
    ldx = X.stride(0) if X.shape[0] > 1 else X.shape[1]
    ldxh = X_hat.stride(0) if X_hat.shape[0] > 1 else X_hat.shape[1]
    rc = lib.onecomp_crossgram_accumulate(_ptr(X_hat), _ptr(X), _dtype_code(X), X.shape[0], X.shape[1], ldxh, ldx,
                                          _dev(G, "G", torch.float32), _stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_crossgram_accumulate")


def onecomp_qep_target(W: torch.Tensor, G: torch.Tensor, H: torch.Tensor, U: torch.Tensor, alpha: float,
                       perm: Optional[torch.Tensor] = None, W_star: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Returns W* = W + alpha W (G - H)^T (H + lambda I)^-1 as an fp32 device tensor (U, perm from the factor call)."""
    lib = load_library()
    d_out, d_in = W.shape
    if W_star is None:
        W_star = torch.empty((d_out, d_in), dtype=torch.float32, device=W.device)
    need = onecomp_qep_workspace_bytes(d_out, d_in)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=W.device)
    if perm is not None:
        _dev(perm, "perm", torch.int32)
    rc = lib.onecomp_qep_target(_dev(W, "W"), _dtype_code(W), d_out, d_in, _dev(G, "G", torch.float32),
                                _dev(H, "H", torch.float32), _dev(U, "U", torch.float32), _ptr(perm), float(alpha),
                                _dev(W_star, "W_star", torch.float32), _dev(workspace, "workspace", torch.uint8),
                                workspace.numel(), _stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_qep_target")
    return W_star


def onecomp_rtn_sensitivity(W: torch.Tensor, a_diag: torch.Tensor, bits: int, group_size: int,
                            b_diag: Optional[torch.Tensor] = None, grid: str = "minmax",
                            err: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """err = 1/2 sum_r sum_c b_r a_c (RTN(W) - W)_rc^2 as a device fp32 scalar tensor."""
    lib = load_library()
    d_out, d_in = W.shape
    if err is None:
        err = torch.zeros(1, dtype=torch.float32, device=W.device)
    if workspace is None:
        workspace = torch.empty(max(int(lib.onecomp_sensitivity_workspace_bytes()), 256), dtype=torch.uint8,
                                device=W.device)
    if grid not in ("minmax", "symmetric"):
        raise ValueError("grid must be 'minmax' or 'symmetric'")
    rc = lib.onecomp_rtn_sensitivity(_dev(W, "W"), _dtype_code(W), d_out, d_in, _dev(a_diag, "a_diag", torch.float32),
                                     _ptr(b_diag), int(bits), int(group_size),
                                     ONECOMP_GRID_SYMMETRIC if grid == "symmetric" else ONECOMP_GRID_MINMAX,
                                     _dev(err, "err", torch.float32), _dev(workspace, "workspace", torch.uint8),
                                     workspace.numel(), _stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_rtn_sensitivity")
    return err


def onecomp_rtn_sensitivity_static(W: torch.Tensor, a_diag: torch.Tensor, bits: int, group_size: int,
                                   b_diag: Optional[torch.Tensor] = None, grid: str = "minmax",
                                   err: Optional[torch.Tensor] = None) -> torch.Tensor:
    """onecomp_rtn_sensitivity without a workspace (the library's built-in scratch).  Pass `err` (device fp32[1]) to keep
    this wrapper from allocating as well."""
    lib = load_library()
    d_out, d_in = W.shape
    if err is None:
        err = torch.zeros(1, dtype=torch.float32, device=W.device)
    if grid not in ("minmax", "symmetric"):
        raise ValueError("grid must be 'minmax' or 'symmetric'")
    rc = lib.onecomp_rtn_sensitivity_static(_dev(W, "W"), _dtype_code(W), d_out, d_in,
                                            _dev(a_diag, "a_diag", torch.float32), _ptr(b_diag), int(bits), int(group_size),
                                            ONECOMP_GRID_SYMMETRIC if grid == "symmetric" else ONECOMP_GRID_MINMAX,
                                            _dev(err, "err", torch.float32), _stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_rtn_sensitivity_static")
    return err


def onecomp_jointq_workspace_bytes(d_out: int, d_in: int, group_size: int) -> int:
    return int(load_library().onecomp_jointq_workspace_bytes(int(d_out), int(d_in), int(group_size)))


def onecomp_jointq_refine(W: torch.Tensor, H: torch.Tensor, Q_codes: torch.Tensor, scales: torch.Tensor,
                          zeros: torch.Tensor, bits: int, group_size: int, grid: str = "minmax", lam: float = 0.0,
                          n_pass: int = 1, max_scans: int = 4, want_w_hat: bool = True,
                          workspace: Optional[torch.Tensor] = None, out: Optional[dict] = None,
                          perm: Optional[torch.Tensor] = None) -> dict:
    """Refines Q_codes and scales IN PLACE; returns dict(Q_codes, scales, W_hat (or None), objective [2] = row
    objective summed over the layer before and after, n_moves) of device tensors.  out: optional dict with
    preallocated "W_hat" (or None), "objective" (fp32[2]) and "n_moves" (int32[1])."""
    lib = load_library()
    d_out, d_in = W.shape
    dev = W.device
    if grid not in _GRIDS:
        raise ValueError("grid must be one of " + ", ".join(sorted(_GRIDS)))
    if workspace is None:
        workspace = torch.empty(max(onecomp_jointq_workspace_bytes(d_out, d_in, group_size), 256), dtype=torch.uint8,
                                device=dev)
    if out is not None:
        W_hat, objective, n_moves = out.get("W_hat"), out["objective"], out["n_moves"]
    else:
        W_hat = torch.empty((d_out, d_in), dtype=torch.float32, device=dev) if want_w_hat else None
        objective = torch.zeros(2, dtype=torch.float32, device=dev)
        n_moves = torch.zeros(1, dtype=torch.int32, device=dev)
    if perm is not None:
        _dev(perm, "perm", torch.int32)
    rc = lib.onecomp_jointq_refine(_dev(W, "W"), _dtype_code(W), d_out, d_in, _dev(H, "H", torch.float32), _ptr(perm),
                                   float(lam),
                                   int(bits), int(group_size), _GRIDS[grid], int(n_pass), int(max_scans),
                                   _dev(Q_codes, "Q_codes", torch.uint8), _dev(scales, "scales", torch.float32),
                                   _dev(zeros, "zeros", torch.float32), _ptr(W_hat),
                                   _dev(objective, "objective", torch.float32), _dev(n_moves, "n_moves", torch.int32),
                                   _dev(workspace, "workspace", torch.uint8), workspace.numel(), _stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_jointq_refine")
    return {"Q_codes": Q_codes, "scales": scales, "W_hat": W_hat, "objective": objective, "n_moves": n_moves}


# ---- the block around the linear layers ----------------------------------------------------------------------------
# These calls are made for single tokens too, where they take less time than ctypes needs to build a structure per tensor.
# Their structures are packed into one buffer per thread (the library reads them before it returns) and go by address.
_DTYPE_CODES = {torch.float32: ONECOMP_F32, torch.bfloat16: ONECOMP_BF16}
_SHAPE = struct.Struct("iiiiiifqqqqPPP")          # onecomp_attention_shape
_NORM_SHAPE = struct.Struct("iiiiiqqff")          # onecomp_norm_shape
_GRAD_FIELDS = 4                                  # words of onecomp_gradient


class _Buffer(threading.local):
    def __init__(self):
        self.data = ctypes.create_string_buffer(1024)
        self.at = ctypes.addressof(self.data)


_buffer = _Buffer()


def _like(t: torch.Tensor) -> torch.Tensor:
    """A dense tensor of t's shape, dtype and device (1.3 us; torch.empty takes 2.2)."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _raw_stream() -> int:
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _head_fields(t: torch.Tensor, name: str, dtype: torch.dtype, device: int, shape) -> Tuple[int, int, int]:
    """(address, token stride, head stride) of a [tokens, heads, dim] tensor."""
    if t.shape != shape:
        raise ValueError(f"{name} must be [tokens, heads, dim], here {list(shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} must live on GPU {device}")
    token, head, one = t.stride()
    n, h, d = shape
    if one != 1 and d > 1 and n > 0:
        raise ValueError(f"rows of {name} must be dense")
    return t.data_ptr(), token if n > 1 else h * d, head if h > 1 else d


def _index_address(t: Optional[torch.Tensor], name: str, device: int, n: int) -> int:
    if t is None:
        return 0
    if t.dtype is not torch.int32:
        raise TypeError(f"{name} must be torch.int32, got {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} must live on GPU {device}")
    if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must have {n} entries (cu_q and cu_k: the starts of the sequences and the end)")
    return t.data_ptr()


def _attention_shape(q, k, cu_q, cu_k, max_q, max_k, causal, scale, len_k) -> int:
    """Packs onecomp_attention_shape to the start of the buffer; returns the device."""
    if not q.is_cuda:
        raise ValueError("q must live on the GPU")
    code = _DTYPE_CODES.get(q.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {q.dtype}: float32 or bfloat16 expected")
    if q.dim() != 3 or k.dim() != 3 or q.shape[2] != k.shape[2]:
        raise ValueError("shapes: q [tokens, heads, dim], k and v [tokens, key heads, dim]")
    device, n = q.get_device(), cu_q.numel() - 1
    if n < 0:
        raise ValueError("cu_q and cu_k hold one start per sequence and the end")
    tokens, heads, dim = q.shape
    _SHAPE.pack_into(_buffer.data, 0, code, heads, k.shape[1], dim, n, 1 if causal else 0, dim ** -0.5 if scale is None else scale, tokens,
                     k.shape[0], max_q, max_k, _index_address(cu_q, "cu_q", device, n + 1), _index_address(cu_k, "cu_k", device, n + 1),
                     _index_address(len_k, "len_k", device, n))
    return device


def _scratch(workspace: Optional[torch.Tensor], need: int, device) -> Tuple[int, int, Optional[torch.Tensor]]:
    """Address, size and owner of a call's workspace; allocated here where the caller brought none."""
    if workspace is None:
        if need == 0:
            return 0, 0, None
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        return workspace.data_ptr(), need, workspace
    return _dev(workspace, "workspace", torch.uint8).value or 0, workspace.numel(), workspace


def _lse_address(lse: torch.Tensor, q: torch.Tensor) -> int:
    if lse.dtype is not torch.float32 or lse.get_device() != q.get_device() or not lse.is_contiguous() or lse.shape != (q.shape[1], q.shape[0]):
        raise ValueError("lse must be dense float32 [heads, total_q] on the GPU of q")
    return lse.data_ptr()


def onecomp_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: torch.Tensor,
                              max_q: int, max_k: int, causal: bool = True, scale: Optional[float] = None,
                              len_k: Optional[torch.Tensor] = None, want_lse: bool = True, out: Optional[torch.Tensor] = None,
                              lse: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Attention of packed sequences.  q: [total_q, heads, dim], k, v: [total_k, key heads, dim] bf16/fp32 (any strides with
    dense rows); cu_q, cu_k: int32 starts of the sequences and the end; len_k: int32 keys of each, where its room in k holds
    more; scale: 1 / sqrt(dim) unless given.  Returns (out [total_q, heads, dim], lse [heads, total_q] fp32 or None)."""
    lib = _lib or load_library()
    device = _attention_shape(q, k, cu_q, cu_k, max_q, max_k, causal, scale, len_k)
    dtype, shape, k_shape = q.dtype, q.shape, k.shape
    if out is None:
        out = _like(q)
    if lse is None and want_lse:
        lse = torch.empty((shape[1], shape[0]), dtype=torch.float32, device=q.device)
    at, base = _SHAPE.size, _buffer.at
    struct.pack_into("Pqq" * 4, _buffer.data, at, *_head_fields(q, "q", dtype, device, shape), *_head_fields(k, "k", dtype, device, k_shape),
                     *_head_fields(v, "v", dtype, device, k_shape), *_head_fields(out, "out", dtype, device, shape))
    ws, ws_bytes, _keep = _scratch(workspace, lib.onecomp_attention_workspace_bytes(base), q.device)
    at += base
    rc = lib.onecomp_attention_forward(base, at, at + 24, at + 48, at + 72, _lse_address(lse, q) if lse is not None else 0, ws, ws_bytes,
                                       _raw_stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_attention_forward")
    return out, lse


def onecomp_attention_backward(d_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                               lse: torch.Tensor, cu_q: torch.Tensor, cu_k: torch.Tensor, max_q: int, max_k: int,
                               causal: bool = True, scale: Optional[float] = None, len_k: Optional[torch.Tensor] = None,
                               dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                               dv: Optional[torch.Tensor] = None,
                               workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Returns (dq, dk, dv) from the gradient of the forward call's output and from what that call took and returned."""
    lib = _lib or load_library()
    device = _attention_shape(q, k, cu_q, cu_k, max_q, max_k, causal, scale, len_k)
    dtype, shape, k_shape, dev = q.dtype, q.shape, k.shape, q.device
    dq = _like(q) if dq is None else dq
    dk = _like(k) if dk is None else dk
    dv = _like(v) if dv is None else dv
    at, base = _SHAPE.size, _buffer.at
    struct.pack_into("Pqq" * 8, _buffer.data, at, *_head_fields(q, "q", dtype, device, shape), *_head_fields(k, "k", dtype, device, k_shape),
                     *_head_fields(v, "v", dtype, device, k_shape), *_head_fields(out, "out", dtype, device, shape),
                     *_head_fields(d_out, "d_out", dtype, device, shape), *_head_fields(dq, "dq", dtype, device, shape),
                     *_head_fields(dk, "dk", dtype, device, k_shape), *_head_fields(dv, "dv", dtype, device, k_shape))
    ws, ws_bytes, _keep = _scratch(workspace, lib.onecomp_attention_backward_workspace_bytes(base), dev)
    at += base
    rc = lib.onecomp_attention_backward(base, at, at + 24, at + 48, at + 72, _lse_address(lse, q), at + 96, at + 120, at + 144, at + 168, ws,
                                        ws_bytes, _raw_stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_attention_backward")
    return dq, dk, dv


_NORMS = {"rms": 0, "layer": 1}


def _row_fields(t: Optional[torch.Tensor], name: str, like: torch.Tensor) -> Tuple[int, int]:
    """(address, row stride) of a [rows, width] tensor; zeros for None."""
    if t is None:
        return 0, 0
    if t.shape != like.shape:
        raise ValueError(f"{name} must be [rows, width], here {list(like.shape)}")
    if t.dtype is not like.dtype:
        raise TypeError(f"{name} must be {like.dtype}, got {t.dtype}")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} must live on {like.device}")
    row, one = t.stride()
    rows, width = t.shape
    if one != 1 and width > 1 and rows > 0:
        raise ValueError(f"rows of {name} must be dense")
    return t.data_ptr(), row if rows > 1 else width


def _param_address(t: Optional[torch.Tensor], name: str, like: torch.Tensor, dtype: Optional[torch.dtype]) -> int:
    if t is None:
        return 0
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 1 or t.shape[0] != like.shape[1] or not t.is_contiguous():
        raise ValueError(f"{name} must have {like.shape[1]} dense entries")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} must live on {like.device}")
    return t.data_ptr()


def _norm_shape(h, weight, bias, post_weight, post_bias, gate, residual_scale, eps, kind, post_norm):
    """Packs onecomp_norm_shape to the start of the buffer; returns (dtype of the parameters, gate as (address, stride))."""
    if not h.is_cuda:
        raise ValueError("h must live on the GPU")
    code = _DTYPE_CODES.get(h.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {h.dtype}: float32 or bfloat16 expected")
    if h.dim() != 2:
        raise ValueError("h must be [rows, width]")
    if kind not in _NORMS:
        raise ValueError("kind must be 'rms' or 'layer'")
    channel = gate is not None and gate.dim() == 1
    first = next((t for t in (weight, bias, post_weight, post_bias, gate if channel else None) if t is not None), h)
    w_dtype = first.dtype
    w_code = _DTYPE_CODES.get(w_dtype)
    if w_code is None:
        raise TypeError(f"unsupported dtype {w_dtype} of the parameters: float32 or bfloat16 expected")
    if post_norm is None:
        post_norm = post_weight is not None or post_bias is not None
    rows, width = h.shape
    _NORM_SHAPE.pack_into(_buffer.data, 0, code, w_code, _NORMS[kind], 0 if gate is None else 1 if channel else 2, 1 if post_norm else 0, rows, width,
                          residual_scale, eps)
    return w_dtype, (_param_address(gate, "gate", h, w_dtype), 0) if channel else _row_fields(gate, "gate", h)


def onecomp_block_norm_forward(h: torch.Tensor, y: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                               bias: Optional[torch.Tensor] = None, post_weight: Optional[torch.Tensor] = None,
                               post_bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                               residual_scale: float = 1.0, eps: float = 1e-6, kind: str = "rms", post_norm: Optional[bool] = None,
                               want_n: bool = True, h_out: Optional[torch.Tensor] = None,
                               n: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """h' = residual_scale h + gate u with u = y, or norm(y) (post_norm: whether; by default where post_weight or post_bias is
    given), and n = norm(h').  h, y: [rows, width] bf16/fp32 (rows may be strided); weights, biases: [width] of one dtype; gate:
    [width] of that dtype or [rows, width].  Without y h' is h.  Returns (h', n); h_out may be h."""
    lib = _lib or load_library()
    w_dtype, gate_fields = _norm_shape(h, weight, bias, post_weight, post_bias, gate, residual_scale, eps, kind, post_norm)
    if y is None:
        if h_out is not None:
            raise ValueError("h_out goes with y: without it h' is h")
    elif h_out is None:
        h_out = _like(h)
    if n is None and want_n:
        n = _like(h)
    at, base = _NORM_SHAPE.size, _buffer.at
    struct.pack_into("Pq" * 5, _buffer.data, at, *_row_fields(h, "h", h), *_row_fields(y, "y", h), *gate_fields, *_row_fields(h_out, "h_out", h),
                     *_row_fields(n, "n", h))
    at += base
    rc = lib.onecomp_block_norm_forward(base, at, at + 16 if y is not None else 0, _param_address(weight, "weight", h, w_dtype),
                                        _param_address(bias, "bias", h, w_dtype), _param_address(post_weight, "post_weight", h, w_dtype),
                                        _param_address(post_bias, "post_bias", h, w_dtype), at + 32 if gate is not None else 0,
                                        at + 48 if h_out is not None else 0, at + 64 if n is not None else 0, _raw_stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_block_norm_forward")
    return (h if y is None else h_out), n


def onecomp_block_norm_backward(dn: Optional[torch.Tensor], dh_out: Optional[torch.Tensor], h: torch.Tensor,
                                y: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                                bias: Optional[torch.Tensor] = None, post_weight: Optional[torch.Tensor] = None,
                                post_bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                                residual_scale: float = 1.0, eps: float = 1e-6, kind: str = "rms", post_norm: Optional[bool] = None,
                                out: Optional[dict] = None, workspace: Optional[torch.Tensor] = None) -> dict:
    """Gradients of onecomp_block_norm_forward from those of n and of h' (either None if there is none); h is the h' that it
    returned.  Returns dict(h, y, weight, bias, post_weight, post_bias, gate), None for what was not given; out: optional dict of
    preallocated tensors of these names."""
    lib = _lib or load_library()
    w_dtype, gate_fields = _norm_shape(h, weight, bias, post_weight, post_bias, gate, residual_scale, eps, kind, post_norm)
    res = {"weight": weight, "bias": bias, "post_weight": post_weight, "post_bias": post_bias, "h": h, "y": y, "gate": gate}
    if out is None:
        for name, t in res.items():
            if t is not None:
                res[name] = _like(t)
    else:
        for name, t in res.items():
            if t is not None:
                res[name] = out.get(name)
    if dn is None:
        res["weight"] = res["bias"] = None
    d_gate = res["gate"]
    channel = gate is not None and gate.dim() == 1
    rows = (dn, dh_out, h, y, res["h"], res["y"], None if channel else d_gate)
    fields = [x for t, name in zip(rows, ("dn", "dh_out", "h", "y", "gradient of h", "gradient of y", "gradient of gate")) for x in _row_fields(t, name, h)]
    at, base = _NORM_SHAPE.size, _buffer.at
    at += base
    # behind the shape: seven tensors, the gate, onecomp_norm_gradients
    struct.pack_into("Pq" * 8 + "8P", _buffer.data, at - base, *fields, *gate_fields,
                     at + 64 if rows[4] is not None else 0, at + 80 if rows[5] is not None else 0, at + 96 if rows[6] is not None else 0,
                     *(_param_address(res[name], "gradient of " + name, h, w_dtype) for name in ("weight", "bias", "post_weight", "post_bias")),
                     _param_address(d_gate, "gradient of gate", h, w_dtype) if channel else 0)
    ws, ws_bytes, _keep = _scratch(workspace, lib.onecomp_block_norm_workspace_bytes(base), h.device)
    rc = lib.onecomp_block_norm_backward(base, at if dn is not None else 0, at + 16 if dh_out is not None else 0, at + 32,
                                         at + 48 if y is not None else 0, _param_address(weight, "weight", h, w_dtype),
                                         _param_address(post_weight, "post_weight", h, w_dtype), _param_address(post_bias, "post_bias", h, w_dtype),
                                         at + 112 if gate is not None else 0, at + 128, ws, ws_bytes, _raw_stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_block_norm_backward")
    return res


def onecomp_clip_gradients(grads: Sequence[torch.Tensor], max_norm: float, out: Optional[Sequence[torch.Tensor]] = None,
                           norm: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None) -> Tuple[Sequence[torch.Tensor], torch.Tensor]:
    """Scales the gradients (dense fp32/bf16 tensors, in any mixture) by min(1, max_norm / (norm + 1e-6)), norm that of all of them
    together: into `out`, or in place.  Returns (out or grads, norm as a device fp32 scalar)."""
    lib = _lib or load_library()
    to, n = grads if out is None else out, len(grads)
    if len(to) != n:
        raise ValueError("out must have one tensor per gradient")
    if n == 0 and norm is None:
        raise ValueError("no gradients: pass norm, so that it is known where it belongs")
    if norm is None:
        norm = torch.empty((), dtype=torch.float32, device=grads[0].device)
    norm_at = _dev(norm, "norm", torch.float32)
    device = norm.get_device()
    table = []
    for g, o in zip(grads, to):
        dtype, size, address = g.dtype, g.numel(), g.data_ptr()
        if g.get_device() != device or not g.is_contiguous() or dtype not in _DTYPE_CODES:
            raise ValueError(f"gradient {len(table) // _GRAD_FIELDS} must be dense float32 or bfloat16 on {norm.device}")
        if o is g:
            table += (address, address, size, _DTYPE_CODES[dtype])
        else:
            if o.dtype is not dtype or o.numel() != size or o.get_device() != device or not o.is_contiguous():
                raise ValueError(f"out {len(table) // _GRAD_FIELDS} must be dense, of the dtype, size and device of its gradient")
            table += (address, o.data_ptr(), size, _DTYPE_CODES[dtype])
    ws, ws_bytes, _keep = _scratch(workspace, lib.onecomp_clip_workspace_bytes(), norm.device)
    rc = lib.onecomp_clip_gradients(struct.pack("q" * len(table), *table), n, max_norm, norm_at, ws, ws_bytes, _raw_stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_clip_gradients")
    return to, norm
