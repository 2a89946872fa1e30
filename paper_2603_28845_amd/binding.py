"""ctypes binding of libonecomp.so: argument marshalling only.

Each function has the name of the C entry point it calls (include/onecomp.h) and
takes torch tensors that live on the GPU; torch supplies device memory and the
current HIP stream, every step of the computation runs in the library's kernels.
There is no CPU fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
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
    shape, heads = ctypes.POINTER(AttentionShape), ctypes.POINTER(Heads)
    lib.onecomp_attention_forward.argtypes = [shape, heads, heads, heads, heads, vp, vp, sz, vp]
    lib.onecomp_attention_forward.restype = i32
    lib.onecomp_attention_workspace_bytes.argtypes = [shape]
    lib.onecomp_attention_workspace_bytes.restype = sz
    lib.onecomp_attention_backward.argtypes = [shape, heads, heads, heads, heads, vp, heads, heads, heads, heads, vp, sz, vp]
    lib.onecomp_attention_backward.restype = i32
    lib.onecomp_attention_backward_workspace_bytes.argtypes = [shape]
    lib.onecomp_attention_backward_workspace_bytes.restype = sz
    rows = ctypes.POINTER(Rows)
    lib.onecomp_block_norm_forward.argtypes = [ctypes.POINTER(NormShape), rows, rows, vp, vp, vp, vp, rows, rows, rows, vp]
    lib.onecomp_block_norm_forward.restype = i32
    lib.onecomp_block_norm_backward.argtypes = [ctypes.POINTER(NormShape), rows, rows, rows, rows, vp, vp, vp, rows,
                                                ctypes.POINTER(NormGradients), vp, sz, vp]
    lib.onecomp_block_norm_backward.restype = i32
    lib.onecomp_block_norm_workspace_bytes.argtypes = [ctypes.POINTER(NormShape)]
    lib.onecomp_block_norm_workspace_bytes.restype = sz
    lib.onecomp_clip_gradients.argtypes = [ctypes.POINTER(Gradient), i32, f32, vp, vp, sz, vp]
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


def _heads(t: torch.Tensor, name: str, like: torch.Tensor, shape: Optional[tuple] = None) -> Heads:
    if t.dim() != 3 or (shape is not None and tuple(t.shape) != shape):
        raise ValueError(f"{name} must be [tokens, heads, dim]" + (f", here {list(shape)}" if shape is not None else ""))
    if t.dtype != like.dtype:
        raise TypeError(f"{name} must be {like.dtype}, got {t.dtype}")
    if t.device != like.device:
        raise ValueError(f"{name} must live on {like.device}")
    if t.numel() > 0 and t.stride(2) != 1 and t.shape[2] > 1:
        raise ValueError(f"rows of {name} must be dense")
    token = t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]
    return Heads(t.data_ptr(), token, t.stride(1) if t.shape[1] > 1 else t.shape[2])


def _attention_shape(q, k, v, cu_q, cu_k, max_q, max_k, causal, scale, len_k) -> AttentionShape:
    _dev(q, "q", contiguous=False)
    if q.dim() != 3 or k.dim() != 3 or q.shape[2] != k.shape[2]:
        raise ValueError("shapes: q [tokens, heads, dim], k and v [tokens, key heads, dim]")
    for t, name in ((cu_q, "cu_q"), (cu_k, "cu_k"), (len_k, "len_k")):
        if t is not None:
            _dev(t, name, torch.int32)
            if t.device != q.device:
                raise ValueError(f"{name} must live on {q.device}")
    n = cu_q.numel() - 1
    if n < 0 or cu_k.numel() != n + 1 or (len_k is not None and len_k.numel() != n):
        raise ValueError("cu_q and cu_k hold one start per sequence and the end, len_k one length per sequence")
    return AttentionShape(_dtype_code(q), q.shape[1], k.shape[1], q.shape[2], n, int(bool(causal)),
                          q.shape[2] ** -0.5 if scale is None else float(scale), q.shape[0], k.shape[0], int(max_q), int(max_k),
                          cu_q.data_ptr(), cu_k.data_ptr(), len_k.data_ptr() if len_k is not None else None)


def _scratch(workspace: Optional[torch.Tensor], need: int, device) -> Tuple[ctypes.c_void_p, int, Optional[torch.Tensor]]:
    """Address, size and owner of a call's workspace; allocated here where the caller brought none."""
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    if workspace is None:
        return ctypes.c_void_p(0), 0, None
    return _dev(workspace, "workspace", torch.uint8), workspace.numel(), workspace


def onecomp_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: torch.Tensor,
                              max_q: int, max_k: int, causal: bool = True, scale: Optional[float] = None,
                              len_k: Optional[torch.Tensor] = None, want_lse: bool = True, out: Optional[torch.Tensor] = None,
                              lse: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Attention of packed sequences.  q: [total_q, heads, dim], k, v: [total_k, key heads, dim] bf16/fp32 (any strides with
    dense rows); cu_q, cu_k: int32 starts of the sequences and the end; len_k: int32 keys of each, where its room in k holds
    more; scale: 1 / sqrt(dim) unless given.  Returns (out [total_q, heads, dim], lse [heads, total_q] fp32 or None)."""
    lib = load_library()
    s = _attention_shape(q, k, v, cu_q, cu_k, max_q, max_k, causal, scale, len_k)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None and want_lse:
        lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device)
    if lse is not None and tuple(lse.shape) != (q.shape[1], q.shape[0]):
        raise ValueError("lse must be [heads, total_q]")
    ws, ws_bytes, _keep = _scratch(workspace, int(lib.onecomp_attention_workspace_bytes(ctypes.byref(s))), q.device)
    rc = lib.onecomp_attention_forward(ctypes.byref(s), ctypes.byref(_heads(q, "q", q)), ctypes.byref(_heads(k, "k", q)),
                                       ctypes.byref(_heads(v, "v", q, tuple(k.shape))),
                                       ctypes.byref(_heads(out, "out", q, tuple(q.shape))),
                                       _dev(lse, "lse", torch.float32) if lse is not None else _ptr(None), ws, ws_bytes, _stream())
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
    lib = load_library()
    s = _attention_shape(q, k, v, cu_q, cu_k, max_q, max_k, causal, scale, len_k)
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=q.dtype, device=q.device) if dk is None else dk
    dv = torch.empty(v.shape, dtype=q.dtype, device=q.device) if dv is None else dv
    if tuple(lse.shape) != (q.shape[1], q.shape[0]):
        raise ValueError("lse must be [heads, total_q]")
    ws, ws_bytes, _keep = _scratch(workspace, int(lib.onecomp_attention_backward_workspace_bytes(ctypes.byref(s))), q.device)
    rows = [ctypes.byref(_heads(t, name, q, tuple(like.shape))) for t, name, like in
            ((q, "q", q), (k, "k", k), (v, "v", k), (out, "out", q), (d_out, "d_out", q), (dq, "dq", q), (dk, "dk", k), (dv, "dv", k))]
    rc = lib.onecomp_attention_backward(ctypes.byref(s), *rows[:4], _dev(lse, "lse", torch.float32), *rows[4:], ws, ws_bytes, _stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_attention_backward")
    return dq, dk, dv


_NORMS = {"rms": 0, "layer": 1}
_GATES = {"none": 0, "channel": 1, "rows": 2}


def _row_view(t: Optional[torch.Tensor], name: str, like: torch.Tensor):
    """onecomp_rows of a [rows, width] tensor (None stays None)."""
    if t is None:
        return None
    if t.dim() != 2 or t.shape != like.shape:
        raise ValueError(f"{name} must be [rows, width], here {list(like.shape)}")
    if t.dtype != like.dtype:
        raise TypeError(f"{name} must be {like.dtype}, got {t.dtype}")
    if t.device != like.device:
        raise ValueError(f"{name} must live on {like.device}")
    if t.numel() > 0 and t.stride(1) != 1 and t.shape[1] > 1:
        raise ValueError(f"rows of {name} must be dense")
    return Rows(t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1])


def _param(t: Optional[torch.Tensor], name: str, like: torch.Tensor, dtype: torch.dtype) -> ctypes.c_void_p:
    if t is None:
        return ctypes.c_void_p(0)
    if t.numel() != like.shape[1]:
        raise ValueError(f"{name} must have {like.shape[1]} entries")
    if t.device != like.device:
        raise ValueError(f"{name} must live on {like.device}")
    return _dev(t, name, dtype)


def _norm_shape(h, y, params, gate, residual_scale, eps, kind, post_norm):
    """(shape, dtype of the parameters, gate as rows or None); params: dict of the weights and biases."""
    _dev(h, "h", contiguous=False)
    if h.dim() != 2:
        raise ValueError("h must be [rows, width]")
    if kind not in _NORMS:
        raise ValueError("kind must be 'rms' or 'layer'")
    channel = gate is not None and gate.dim() == 1
    given = [t for t in list(params.values()) + ([gate] if channel else []) if t is not None]
    w_dtype = given[0].dtype if given else h.dtype
    gate_kind = "none" if gate is None else "channel" if channel else "rows"
    if post_norm is None:
        post_norm = params["post_weight"] is not None or params["post_bias"] is not None
    shape = NormShape(_dtype_code(h), ONECOMP_BF16 if w_dtype == torch.bfloat16 else ONECOMP_F32, _NORMS[kind], _GATES[gate_kind], int(bool(post_norm)),
                      h.shape[0], h.shape[1], float(residual_scale), float(eps))
    if channel:
        gate_rows = Rows(_param(gate, "gate", h, w_dtype).value, 0)
    else:
        gate_rows = _row_view(gate, "gate", h)
    return shape, w_dtype, gate_rows


def _ref(struct):
    return ctypes.byref(struct) if struct is not None else None


def onecomp_block_norm_forward(h: torch.Tensor, y: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                               bias: Optional[torch.Tensor] = None, post_weight: Optional[torch.Tensor] = None,
                               post_bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                               residual_scale: float = 1.0, eps: float = 1e-6, kind: str = "rms", post_norm: Optional[bool] = None,
                               want_n: bool = True, h_out: Optional[torch.Tensor] = None,
                               n: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """h' = residual_scale h + gate u with u = y, or norm(y) (post_norm: whether; by default where post_weight or post_bias is
    given), and n = norm(h').  h, y: [rows, width] bf16/fp32 (rows may be strided); weights, biases: [width] of one dtype; gate:
    [width] of that dtype or [rows, width].  Without y h' is h.  Returns (h', n); h_out may be h."""
    lib = load_library()
    params = {"weight": weight, "bias": bias, "post_weight": post_weight, "post_bias": post_bias}
    shape, w_dtype, gate_rows = _norm_shape(h, y, params, gate, residual_scale, eps, kind, post_norm)
    if y is None:
        if h_out is not None:
            raise ValueError("h_out goes with y: without it h' is h")
    elif h_out is None:
        h_out = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    if n is None and want_n:
        n = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    views = [_row_view(t, name, h) for t, name in ((h, "h"), (y, "y"), (h_out, "h_out"), (n, "n"))]
    rc = lib.onecomp_block_norm_forward(ctypes.byref(shape), _ref(views[0]), _ref(views[1]),
                                        *(_param(t, name, h, w_dtype) for name, t in params.items()), _ref(gate_rows), _ref(views[2]),
                                        _ref(views[3]), _stream())
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
    lib = load_library()
    params = {"weight": weight, "bias": bias, "post_weight": post_weight, "post_bias": post_bias}
    shape, w_dtype, gate_rows = _norm_shape(h, y, params, gate, residual_scale, eps, kind, post_norm)
    given = dict(params, h=h, y=y, gate=gate)
    res = {name: None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device) if out is None else out.get(name)
           for name, t in given.items()}
    if dn is None:
        res["weight"] = res["bias"] = None
    channel = gate is not None and gate.dim() == 1
    views = {name: _row_view(t, name, h) for name, t in (("dn", dn), ("dh_out", dh_out), ("h", h), ("y", y), ("dh", res["h"]),
                                                         ("dy", res["y"]), ("dgate", None if channel else res["gate"]))}
    grads = NormGradients(*(ctypes.pointer(views[name]) if views[name] is not None else None for name in ("dh", "dy", "dgate")),
                          *(_param(res[name], "gradient of " + name, h, w_dtype) for name in params),
                          _param(res["gate"] if channel else None, "gradient of gate", h, w_dtype))
    ws, ws_bytes, _keep = _scratch(workspace, int(lib.onecomp_block_norm_workspace_bytes(ctypes.byref(shape))), h.device)
    rc = lib.onecomp_block_norm_backward(ctypes.byref(shape), _ref(views["dn"]), _ref(views["dh_out"]), _ref(views["h"]), _ref(views["y"]),
                                         *(_param(params[name], name, h, w_dtype) for name in ("weight", "post_weight", "post_bias")),
                                         _ref(gate_rows), ctypes.byref(grads), ws, ws_bytes, _stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_block_norm_backward")
    return res


def onecomp_clip_gradients(grads: Sequence[torch.Tensor], max_norm: float, out: Optional[Sequence[torch.Tensor]] = None,
                           norm: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None) -> Tuple[Sequence[torch.Tensor], torch.Tensor]:
    """Scales the gradients (dense fp32/bf16 tensors, in any mixture) by min(1, max_norm / (norm + 1e-6)), norm that of all of them
    together: into `out`, or in place.  Returns (out or grads, norm as a device fp32 scalar)."""
    lib = load_library()
    to = grads if out is None else out
    if len(to) != len(grads):
        raise ValueError("out must have one tensor per gradient")
    if not grads and norm is None:
        raise ValueError("no gradients: pass norm, so that it is known where it belongs")
    device = norm.device if norm is not None else grads[0].device
    table = (Gradient * max(1, len(grads)))()
    for i, (g, o) in enumerate(zip(grads, to)):
        if o is not g and (o.dtype != g.dtype or o.numel() != g.numel()):
            raise ValueError(f"out {i} must have the dtype and size of its gradient")
        if g.device != device or o.device != device:
            raise ValueError(f"gradient {i} must live on {device}")
        table[i] = Gradient(_dev(g, f"gradient {i}").value, _dev(o, f"out {i}").value, g.numel(), _dtype_code(g))
    if norm is None:
        norm = torch.empty((), dtype=torch.float32, device=device)
    ws, ws_bytes, _keep = _scratch(workspace, int(lib.onecomp_clip_workspace_bytes()), device)
    rc = lib.onecomp_clip_gradients(table, len(grads), float(max_norm), _dev(norm, "norm", torch.float32), ws, ws_bytes, _stream())
    if rc != ONECOMP_OK:
        raise OnecompError(rc, "onecomp_clip_gradients")
    return to, norm
