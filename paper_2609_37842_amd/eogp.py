"""Python binding of the EOGP C ABI (include/eogp.h).

Argument marshalling only: every step of the hot path runs in the HIP kernels of
libeogp.so. torch supplies device memory (tensors) and the current HIP stream.
The functions carry the same names as the C entry points. If the library is
missing the import of any entry point raises; there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libeogp.so")

F32, BF16, F16 = 0, 1, 2
PREC_FAST, PREC_ACCURATE, PREC_F16 = 0, 1, 2

_DTYPE_CODE = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

c_i64 = ctypes.c_int64
c_i32 = ctypes.c_int32
c_vp = ctypes.c_void_p
c_sz = ctypes.c_size_t


class EogpError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"eogp status {status}: {msg}")
        self.status = status


class PlanInfo(ctypes.Structure):
    _fields_ = [("d_out", c_i64), ("d_in", c_i64), ("m", c_i64), ("damping", ctypes.c_double),
                ("n_rows", c_i64), ("n_cols", c_i64), ("n_tiles", c_i64),
                ("retained_flat", c_vp), ("retained_weight", c_vp)]


class Heads(ctypes.Structure):
    """A tensor of heads [N, T, heads, D] by its address and strides (eogp_heads)."""
    _fields_ = [("data", c_vp), ("heads", c_i64), ("ld_example", c_i64), ("ld_token", c_i64), ("ld_head", c_i64)]


_lib = None

EXPORTED = (
    "eogp_plan_create", "eogp_plan_destroy", "eogp_plan_get_info", "eogp_plan_copy_retained",
    "eogp_plan_set_input_exponents",
    "eogp_rotate_retain_workspace_size", "eogp_rotate_retain_planned",
    "eogp_compact_tokens_workspace_size", "eogp_compact_tokens", "eogp_rotate_retain_compacted",
    "eogp_rotate_retain_oneshot_workspace_size", "eogp_rotate_retain",
    "eogp_pca_project_workspace_size", "eogp_pca_project",
    "eogp_sign_pack", "eogp_sign_pack_tiled", "eogp_srht_project_workspace_size",
    "eogp_srht_project",
    "eogp_pca_fit_workspace_size", "eogp_pca_fit",
    "eogp_ekfac_workspace_size", "eogp_ekfac_eigenvalues",
    "eogp_score_topk_workspace_size", "eogp_score_topk", "eogp_score_topk_tiled",
    "eogp_score_topk_noalloc",
    "eogp_embed_tokens", "eogp_embed_backward_workspace_size", "eogp_embed_backward",
    "eogp_layer_norm", "eogp_layer_norm_backward_workspace_size", "eogp_layer_norm_backward",
    "eogp_softmax_xent", "eogp_sample_tokens",
    "eogp_rotary_table", "eogp_rotate_heads", "eogp_rotate_heads_backward_workspace_size",
    "eogp_rotate_heads_backward", "eogp_attention_workspace_size", "eogp_attention",
    "eogp_attention_backward_workspace_size", "eogp_attention_backward",
    "eogp_timing_enable", "eogp_timing_read",
    "eogp_status_string", "eogp_last_error", "eogp_version",
)


def load(path: str | None = None):
    """Load libeogp.so once and declare the C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"{path} not found; build it with "
                           "`python -m paper_2609_37842_amd.build`")
    L = ctypes.CDLL(path)
    sig = {
        "eogp_plan_create": (c_i32, [c_vp, c_i64, c_i64, ctypes.c_double, c_i64, c_vp, c_vp, c_vp,
                                     ctypes.POINTER(c_vp)]),
        "eogp_plan_destroy": (None, [c_vp]),
        "eogp_plan_get_info": (c_i32, [c_vp, ctypes.POINTER(PlanInfo)]),
        "eogp_plan_copy_retained": (c_i32, [c_vp, c_vp, c_vp, c_vp]),
        "eogp_plan_set_input_exponents": (c_i32, [c_vp, c_i32, c_i32]),
        "eogp_rotate_retain_workspace_size": (c_sz, [c_vp, c_i64, c_i64]),
        "eogp_rotate_retain_planned": (c_i32, [c_vp, c_vp, c_i64, c_vp, c_i64, c_i32, c_vp, c_i64,
                                               c_i64, c_vp, c_i32, c_i64, c_i32, c_vp, c_sz, c_vp]),
        "eogp_compact_tokens_workspace_size": (c_sz, [c_i64, c_i64]),
        "eogp_compact_tokens": (c_i32, [c_vp, c_i64, c_i64, c_i32, c_vp, c_sz, c_vp]),
        "eogp_rotate_retain_compacted": (c_i32, [c_vp, c_vp, c_i64, c_vp, c_i64, c_i32, c_i64, c_i64,
                                                 c_vp, c_i32, c_i64, c_i32, c_vp, c_sz, c_vp]),
        "eogp_rotate_retain_oneshot_workspace_size": (c_sz, [c_i64, c_i64, c_i64, c_i64, c_i64]),
        "eogp_rotate_retain": (c_i32, [c_vp, c_i64, c_vp, c_i64, c_i32, c_vp, c_i64, c_i64, c_i64,
                                       c_i64, c_vp, c_vp, c_vp, ctypes.c_double, c_i64, c_vp, c_i64,
                                       c_i32, c_vp, c_sz, c_vp]),
        "eogp_pca_project_workspace_size": (c_sz, [c_i64, c_i64, c_i64, c_i32, c_i32]),
        "eogp_pca_project": (c_i32, [c_vp, c_i32, c_i64, c_i64, c_i64, c_vp, c_i32, c_i64, c_i64,
                                     c_vp, c_i64, c_i32, c_vp, c_sz, c_vp]),
        "eogp_sign_pack": (c_i32, [c_vp, c_i64, c_i64, c_i64, c_vp, c_i64, c_vp, c_i64, c_vp]),
        "eogp_sign_pack_tiled": (c_i32, [c_vp, c_i64, c_i64, c_i64, c_i64, c_vp, c_i64, c_i64, c_vp,
                                         c_i64, c_vp]),
        "eogp_ekfac_workspace_size": (c_sz, [c_i64, c_i64, c_i64, c_i64]),
        "eogp_ekfac_eigenvalues": (c_i32, [c_vp, c_i64, c_vp, c_i64, c_i32, c_vp, c_i64, c_i64,
                                           c_i64, c_i64, c_vp, c_vp, c_i32, c_i32, c_i32, c_vp,
                                           c_i32, c_vp, c_sz, c_vp]),
        "eogp_srht_project_workspace_size": (c_sz, [c_i64, c_i64]),
        "eogp_srht_project": (c_i32, [c_vp, c_i64, c_i64, c_i64, c_vp, c_vp, c_i64, c_vp, c_i64,
                                      c_vp, c_sz, c_vp]),
        "eogp_pca_fit_workspace_size": (c_sz, [c_i64, c_i64, c_i64]),
        "eogp_pca_fit": (c_i32, [c_vp, c_i64, c_i64, c_i64, c_i64, c_vp, c_i64, c_vp, c_vp, c_sz,
                                 c_vp]),
        "eogp_score_topk_workspace_size": (c_sz, [c_i64, c_i64, c_i32, ctypes.POINTER(c_i64),
                                                  c_i32]),
        "eogp_score_topk": (c_i32, [c_vp, c_i64, c_vp, c_i64, c_i32, ctypes.POINTER(c_i64), c_vp,
                                    c_i64, c_i64, c_i32, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]),
        "eogp_score_topk_tiled": (c_i32, [c_vp, c_vp, c_i64, c_i32, ctypes.POINTER(c_i64), c_vp,
                                          c_i64, c_i64, c_i32, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]),
        "eogp_score_topk_noalloc": (c_i32, [c_vp, c_i64, c_vp, c_i64, c_i32, ctypes.POINTER(c_i64),
                                            c_vp, c_i64, c_i64, c_i32, c_vp, c_vp, c_vp, c_vp]),
        "eogp_embed_tokens": (c_i32, [c_vp, c_i32, c_i64, c_i64, c_i64, c_vp, c_vp, c_i64,
                                      ctypes.c_float, c_i32, c_vp, c_i32, c_i64, c_vp]),
        "eogp_embed_backward_workspace_size": (c_sz, [c_i64, c_i64, c_i64]),
        "eogp_embed_backward": (c_i32, [c_vp, c_i32, c_i64, c_vp, c_vp, c_i64, c_i64, c_i64,
                                        ctypes.c_float, c_i32, c_vp, c_i64, c_vp, c_sz, c_vp]),
        "eogp_layer_norm": (c_i32, [c_vp, c_i32, c_i64, c_vp, c_vp, c_i32, ctypes.c_float, c_vp,
                                    c_i64, c_i64, c_vp, c_i32, c_i64, c_i32, c_vp, c_vp, c_vp]),
        "eogp_layer_norm_backward_workspace_size": (c_sz, [c_i64, c_i64, c_i64, c_i32]),
        "eogp_layer_norm_backward": (c_i32, [c_vp, c_i64, c_vp, c_i64, c_i32, c_vp, c_i32, c_vp,
                                             c_vp, c_vp, c_vp, c_i64, c_i64, c_i64, c_i64, c_vp,
                                             c_i64, c_vp, c_vp, c_vp, c_sz, c_vp]),
        "eogp_softmax_xent": (c_i32, [c_vp, c_i32, c_i64, c_vp, c_vp, c_i64, c_i64, ctypes.c_float,
                                      c_vp, c_vp, c_i64, c_vp]),
        "eogp_sample_tokens": (c_i32, [c_vp, c_i32, c_i64, c_i64, c_i64, c_vp, c_vp,
                                       ctypes.c_double, c_i64, ctypes.c_double, ctypes.c_double,
                                       c_vp, c_vp]),
        "eogp_rotary_table": (c_i32, [c_i64, c_i64] + [ctypes.c_double] * 6 + [c_vp, c_vp]),
        "eogp_rotate_heads": (c_i32, [c_vp, c_vp, c_i32, c_i64, c_i64, c_i64, c_i32, c_vp, c_vp, c_i32, ctypes.c_float,
                                      c_vp, c_i64, c_i64, c_i32, c_vp, c_vp, c_vp, c_vp, c_vp]),
        "eogp_rotate_heads_backward_workspace_size": (c_sz, [c_i64] * 5 + [c_i32, c_i32, c_i64, c_i32]),
        "eogp_rotate_heads_backward": (c_i32, [c_vp] * 4 + [c_i32, c_i64, c_i64, c_i64, c_i32, c_vp, c_vp, c_i32,
                                               ctypes.c_float, c_vp, c_i64, c_i64, c_i32, c_vp, c_vp, c_i32, c_vp,
                                               c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]),
        "eogp_attention_workspace_size": (c_sz, [c_i64] * 6 + [c_i32]),
        "eogp_attention": (c_i32, [c_vp] * 3 + [c_i32] + [c_i64] * 4 + [ctypes.c_float, c_i32, c_i64, c_i64, c_vp, c_vp,
                                                                       c_vp, c_vp, c_i32, c_vp, c_vp, c_sz, c_vp]),
        "eogp_attention_backward_workspace_size": (c_sz, [c_i64] * 6 + [c_i32]),
        "eogp_attention_backward": (c_i32, [c_vp] * 4 + [c_i32] + [c_i64] * 4 +
                                    [ctypes.c_float, c_i32, c_i64, c_i64, c_vp, c_vp, c_vp, c_vp, c_i32, c_vp, c_vp,
                                     c_vp, c_vp, c_vp, c_sz, c_vp]),
        "eogp_timing_enable": (c_i32, [c_i32]),
        "eogp_timing_read": (c_i32, [c_i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(c_i64)]),
        "eogp_status_string": (ctypes.c_char_p, [c_i32]),
        "eogp_last_error": (ctypes.c_char_p, []),
        "eogp_version": (c_i32, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        L = load()
        raise EogpError(status, L.eogp_last_error().decode())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _need_cuda(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda):
            raise ValueError("EOGP arguments must be device tensors")


def _check_workspace(status: int, need: int):
    """For calls that run in less than the size reported: the library decides."""
    if status == -4:                             # EOGP_ERR_WORKSPACE
        raise ValueError(f"workspace needs {need} bytes")
    _check(status)


def _workspace(nbytes: int, device, ws=None, less_ok=False):
    if nbytes == 0:
        return None, 0
    if ws is not None:
        if not less_ok and ws.numel() * ws.element_size() < nbytes:
            raise ValueError(f"workspace needs {nbytes} bytes")
        return ws, ws.numel() * ws.element_size()
    return torch.empty(nbytes, dtype=torch.uint8, device=device), nbytes


# ---------------------------------------------------------------------------
# Plans (fitting shared projections)
# ---------------------------------------------------------------------------
class eogp_plan:
    """Retained-axis plan of one module; see eogp_plan_create in eogp.h."""

    def __init__(self, eigvals, damping: float, m: int, Q_A, Q_S, stream=None):
        L = load()
        _need_cuda(eigvals, Q_A, Q_S)
        for t in (eigvals, Q_A, Q_S):
            if t.dtype != torch.float32 or not t.is_contiguous():
                raise ValueError("eigvals, Q_A, Q_S must be contiguous float32")
        d_out, d_in = eigvals.shape
        if tuple(Q_A.shape) != (d_in, d_in) or tuple(Q_S.shape) != (d_out, d_out):
            raise ValueError("Q_A must be [d_in, d_in] and Q_S [d_out, d_out]")
        h = c_vp()
        _check(L.eogp_plan_create(_ptr(eigvals), d_out, d_in, float(damping), int(m), _ptr(Q_A),
                                  _ptr(Q_S), _stream(stream), ctypes.byref(h)))
        self._h = h
        self.device = eigvals.device
        info = PlanInfo()
        _check(L.eogp_plan_get_info(h, ctypes.byref(info)))
        self.d_out, self.d_in, self.m = int(info.d_out), int(info.d_in), int(info.m)
        self.damping = float(info.damping)
        self.n_rows, self.n_cols, self.n_tiles = int(info.n_rows), int(info.n_cols), int(info.n_tiles)
        self._flat_ptr, self._w_ptr = info.retained_flat, info.retained_weight

    def retained(self):
        """(flat index int32 [m], weight float32 [m]) copied to new device tensors."""
        flat = torch.empty(self.m, dtype=torch.int32, device=self.device)
        w = torch.empty(self.m, dtype=torch.float32, device=self.device)
        _check(load().eogp_plan_copy_retained(self._h, _ptr(flat), _ptr(w), _stream()))
        return flat, w

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            load().eogp_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def eogp_plan_create(eigvals, damping, m, Q_A, Q_S, stream=None) -> eogp_plan:
    return eogp_plan(eigvals, damping, m, Q_A, Q_S, stream)


def eogp_plan_set_input_exponents(plan: eogp_plan, e_acts: int, e_grads: int) -> None:
    """Power-of-two input scaling of the plan's fp16 first stage (see eogp.h)."""
    _check(load().eogp_plan_set_input_exponents(plan._h, int(e_acts), int(e_grads)))


# ---------------------------------------------------------------------------
# First stage
# ---------------------------------------------------------------------------
def _token_stride(x, name):
    """Row stride (elements) of a [N, T, d] token tensor whose tokens are laid
    out at a constant stride, e.g. a column slice of a wider padded buffer."""
    if x.dim() != 3 or x.stride(2) != 1 or x.stride(0) != x.shape[1] * x.stride(1):
        raise ValueError(f"{name} must be [N, T, d] with unit column stride and tokens at a "
                         "constant row stride")
    return x.stride(1)


def _acts_dtype(acts, out_grads):
    if acts.dtype != out_grads.dtype or acts.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("acts and out_grads must both be float32 or both bfloat16")
    return _DTYPE_CODE[acts.dtype]


def eogp_rotate_retain_workspace_size(plan: eogp_plan, N: int, T: int) -> int:
    return int(load().eogp_rotate_retain_workspace_size(plan._h, N, T))


def _first_stage_args(plan, acts, out_grads, Z):
    """Checks shared by the planned first-stage calls; returns (N, T, ld_a, ld_g, Z)."""
    _need_cuda(acts, out_grads, Z)
    N, T, d_in = acts.shape
    if tuple(out_grads.shape) != (N, T, plan.d_out) or d_in != plan.d_in:
        raise ValueError("acts [N,T,d_in] / out_grads [N,T,d_out] do not match the plan")
    ld_a, ld_g = _token_stride(acts, "acts"), _token_stride(out_grads, "out_grads")
    if Z is None:
        Z = torch.empty((N, plan.m), dtype=torch.float32, device=acts.device)
    if (Z.dtype not in (torch.float32, torch.float16) or Z.dim() != 2 or Z.stride(1) != 1
            or Z.shape[0] != N):
        raise ValueError("Z must be float32 or float16 [N, >= m] with unit column stride")
    return N, T, ld_a, ld_g, Z


def eogp_rotate_retain_planned(plan: eogp_plan, acts, out_grads, token_mask=None, Z=None,
                               prec=PREC_ACCURATE, ws=None, stream=None):
    """Z [N, m] (float32) of the batch; see eogp_rotate_retain_planned in eogp.h."""
    L = load()
    _need_cuda(token_mask)
    N, T, ld_a, ld_g, Z = _first_stage_args(plan, acts, out_grads, Z)
    if token_mask is not None and (token_mask.dtype != torch.uint8 or tuple(token_mask.shape) != (N, T)
                                   or not token_mask.is_contiguous()):
        raise ValueError("token_mask must be contiguous uint8 [N, T]")
    need = eogp_rotate_retain_workspace_size(plan, N, T)
    ws, wsb = _workspace(need, acts.device, ws)
    _check(L.eogp_rotate_retain_planned(plan._h, _ptr(acts), ld_a, _ptr(out_grads), ld_g,
                                        _acts_dtype(acts, out_grads), _ptr(token_mask), N, T,
                                        _ptr(Z), _DTYPE_CODE[Z.dtype], Z.stride(0), prec, _ptr(ws),
                                        wsb, _stream(stream)))
    return Z


def eogp_compact_tokens_workspace_size(N: int, T: int) -> int:
    return int(load().eogp_compact_tokens_workspace_size(N, T))


def eogp_compact_tokens(token_mask, N: int, T: int, prec, ws, stream=None):
    """Valid-token list of (token_mask, N, T) into the head of the first-stage
    workspace `ws` (a uint8 device tensor); see eogp_compact_tokens in eogp.h."""
    L = load()
    if ws is None:
        raise ValueError("eogp_compact_tokens writes into a caller's first-stage workspace")
    _need_cuda(token_mask, ws)
    if token_mask is not None and (token_mask.dtype != torch.uint8 or tuple(token_mask.shape) != (N, T)
                                   or not token_mask.is_contiguous()):
        raise ValueError("token_mask must be contiguous uint8 [N, T]")
    ws, wsb = _workspace(eogp_compact_tokens_workspace_size(N, T), ws.device, ws)
    _check(L.eogp_compact_tokens(_ptr(token_mask), N, T, prec, _ptr(ws), wsb, _stream(stream)))


def eogp_rotate_retain_compacted(plan: eogp_plan, acts, out_grads, ws, Z=None, prec=PREC_ACCURATE,
                                 stream=None):
    """The planned first stage with the token list already in `ws` (written by
    eogp_compact_tokens for the same N, T and precision layout)."""
    L = load()
    if ws is None:
        raise ValueError("the compacted first stage reads the token list from ws")
    _need_cuda(ws)
    N, T, ld_a, ld_g, Z = _first_stage_args(plan, acts, out_grads, Z)
    ws, wsb = _workspace(eogp_rotate_retain_workspace_size(plan, N, T), acts.device, ws)
    _check(L.eogp_rotate_retain_compacted(plan._h, _ptr(acts), ld_a, _ptr(out_grads), ld_g,
                                          _acts_dtype(acts, out_grads), N, T, _ptr(Z),
                                          _DTYPE_CODE[Z.dtype], Z.stride(0), prec, _ptr(ws), wsb,
                                          _stream(stream)))
    return Z


def eogp_rotate_retain(acts, out_grads, token_mask, Q_A, Q_S, eigvals, damping, m, Z=None,
                       prec=PREC_ACCURATE, ws=None, stream=None):
    """One-shot first stage with the paper's arguments (builds and frees a plan)."""
    L = load()
    _need_cuda(acts, out_grads, token_mask, Q_A, Q_S, eigvals, Z)
    N, T, d_in = acts.shape
    d_out = out_grads.shape[2]
    ld_a, ld_g = _token_stride(acts, "acts"), _token_stride(out_grads, "out_grads")
    if Z is None:
        Z = torch.empty((N, m), dtype=torch.float32, device=acts.device)
    need = int(L.eogp_rotate_retain_oneshot_workspace_size(N, T, d_in, d_out, int(m)))
    ws, wsb = _workspace(need, acts.device, ws)
    _check(L.eogp_rotate_retain(_ptr(acts), ld_a, _ptr(out_grads), ld_g, _acts_dtype(acts, out_grads),
                                _ptr(token_mask), N, T, d_in, d_out, _ptr(Q_A), _ptr(Q_S),
                                _ptr(eigvals), float(damping), int(m), _ptr(Z), Z.stride(0), prec,
                                _ptr(ws), wsb, _stream(stream)))
    return Z


# ---------------------------------------------------------------------------
# Second stage, encoding, scoring
# ---------------------------------------------------------------------------
def eogp_pca_project_workspace_size(N: int, m: int, k: int, p_dtype: int, prec: int) -> int:
    """Bytes of workspace eogp_pca_project needs for these sizes."""
    return int(load().eogp_pca_project_workspace_size(N, m, k, p_dtype, prec))


def eogp_pca_project(Z, Pt, X=None, prec=PREC_FAST, ws=None, stream=None):
    """X [N, k] = Z [N, m] @ P, with P given as Pt [k, m] (each direction
    contiguous, i.e. P column-major) in float16, bfloat16 or float32; Z in
    float32, or in P's own 16-bit type."""
    L = load()
    _need_cuda(Z, Pt, X)
    N, m = Z.shape
    k, m2 = Pt.shape
    if m2 != m or Pt.stride(1) != 1 or Z.stride(1) != 1:
        raise ValueError("Pt must be [k, m] with unit column stride; Z [N, m]")
    if Z.dtype not in (torch.float32, torch.float16, torch.bfloat16):
        raise ValueError("Z must be float32, float16 or bfloat16")
    if X is None:
        X = torch.empty((N, k), dtype=torch.float32, device=Z.device)
    pd = _DTYPE_CODE[Pt.dtype]
    need = int(L.eogp_pca_project_workspace_size(N, m, k, pd, prec))
    ws, wsb = _workspace(need, Z.device, ws)
    _check(L.eogp_pca_project(_ptr(Z), _DTYPE_CODE[Z.dtype], Z.stride(0), N, m, _ptr(Pt), pd,
                              Pt.stride(0), k, _ptr(X), X.stride(0), prec, _ptr(ws), wsb,
                              _stream(stream)))
    return X


def eogp_ekfac_workspace_size(N: int, T: int, d_in: int, d_out: int) -> int:
    """Bytes of workspace eogp_ekfac_eigenvalues needs for these sizes."""
    return int(load().eogp_ekfac_workspace_size(N, T, d_in, d_out))


def eogp_ekfac_eigenvalues(acts, out_grads, token_mask, Q_A, Q_S, sq_sum=None, accumulate=False,
                           prec=PREC_ACCURATE, exponents=(0, 0), ws=None, stream=None):
    """Sum over the batch of the squared rotated gradients (Q_S^T G_i Q_A)^2,
    [d_out, d_in] float32 (divide by the total number of examples for the
    corrected eigenvalues). exponents = (e_acts, e_grads), the power-of-two
    input scaling of the fp16 mode; see eogp_ekfac_eigenvalues in eogp.h."""
    L = load()
    _need_cuda(acts, out_grads, token_mask, Q_A, Q_S, sq_sum)
    N, T, d_in = acts.shape
    d_out = out_grads.shape[2]
    ld_a, ld_g = _token_stride(acts, "acts"), _token_stride(out_grads, "out_grads")
    if sq_sum is None:
        sq_sum = torch.empty((d_out, d_in), dtype=torch.float32, device=acts.device)
        accumulate = False
    if sq_sum.dtype != torch.float32 or tuple(sq_sum.shape) != (d_out, d_in) or not sq_sum.is_contiguous():
        raise ValueError("sq_sum must be contiguous float32 [d_out, d_in]")
    need = int(L.eogp_ekfac_workspace_size(N, T, d_in, d_out))
    ws, wsb = _workspace(need, acts.device, ws, less_ok=True)
    status = L.eogp_ekfac_eigenvalues(_ptr(acts), ld_a, _ptr(out_grads), ld_g,
                                      _acts_dtype(acts, out_grads), _ptr(token_mask), N, T, d_in,
                                      d_out, _ptr(Q_A), _ptr(Q_S), prec, int(exponents[0]),
                                      int(exponents[1]), _ptr(sq_sum), 1 if accumulate else 0,
                                      _ptr(ws), wsb, _stream(stream))
    _check_workspace(status, need)
    return sq_sum


def eogp_srht_project_workspace_size(N: int, m: int) -> int:
    return int(load().eogp_srht_project_workspace_size(N, m))


def eogp_srht_project(Z, signs, rows, X=None, ws=None, stream=None):
    """X [N, k] = the SRHT of each row of Z [N, m] (float32) with random signs
    [m] (int8) and kept rows [k] (int32); see eogp_srht_project in eogp.h."""
    L = load()
    _need_cuda(Z, signs, rows, X)
    N, m = Z.shape
    k = rows.shape[0]
    if Z.dtype != torch.float32 or (Z.numel() > 0 and Z.stride(1) != 1):
        raise ValueError("Z must be float32 [N, m] with unit column stride")
    if signs.dtype != torch.int8 or signs.shape[0] != m or not signs.is_contiguous():
        raise ValueError("signs must be contiguous int8 [m]")
    if rows.dtype != torch.int32 or not rows.is_contiguous():
        raise ValueError("rows must be contiguous int32 [k]")
    if X is None:
        X = torch.empty((N, k), dtype=torch.float32, device=Z.device)
    ws, wsb = _workspace(int(L.eogp_srht_project_workspace_size(N, m)), Z.device, ws)
    _check(L.eogp_srht_project(_ptr(Z), max(Z.stride(0), m), N, m, _ptr(signs), _ptr(rows), k,
                               _ptr(X), max(X.stride(0), k), _ptr(ws), wsb, _stream(stream)))
    return X


def eogp_pca_fit_workspace_size(n: int, m: int, k: int) -> int:
    return int(load().eogp_pca_fit_workspace_size(n, m, k))


def eogp_pca_fit(Z, k, Pt=None, mu=None, ws=None, stream=None):
    """Fit the PCA projection from first-stage coordinates Z [n, m] (float32):
    returns (Pt [k, m] float32, mu [k] float32); see eogp_pca_fit in eogp.h.
    Synchronises the stream."""
    L = load()
    _need_cuda(Z, Pt, mu)
    n, m = Z.shape
    if Z.dtype != torch.float32 or Z.stride(1) != 1:
        raise ValueError("Z must be float32 [n, m] with unit column stride")
    if Pt is None:
        Pt = torch.empty((k, m), dtype=torch.float32, device=Z.device)
    if mu is None:
        mu = torch.empty((k,), dtype=torch.float32, device=Z.device)
    need = int(L.eogp_pca_fit_workspace_size(n, m, k))
    if need == 0:
        bad_sizes = not (1 <= k <= min(n, m))
        raise EogpError(-1 if bad_sizes else -3, L.eogp_last_error().decode())
    ws, wsb = _workspace(need, Z.device, ws)
    _check(L.eogp_pca_fit(_ptr(Z), max(Z.stride(0), m), n, m, k, _ptr(Pt), Pt.stride(0), _ptr(mu),
                          _ptr(ws), wsb, _stream(stream)))
    return Pt, mu


def eogp_sign_pack(X, codes=None, scales=None, stream=None):
    """Packed sign bits [N, ceil(k/8)] (uint8) and fp16 scales [N] (uint16 bits)."""
    L = load()
    _need_cuda(X, codes, scales)
    N, k = X.shape
    if codes is None:
        codes = torch.empty((N, (k + 7) // 8), dtype=torch.uint8, device=X.device)
    if scales is None:
        scales = torch.empty((N, 1), dtype=torch.int16, device=X.device)
    sstride = scales.stride(0) if scales.dim() == 2 else 1
    _check(L.eogp_sign_pack(_ptr(X), X.stride(0), N, k, _ptr(codes), codes.stride(0),
                            _ptr(scales), sstride, _stream(stream)))
    return codes, scales


def tiled_store_bytes(N: int, k_per_module) -> int:
    """Bytes of a tiled store of N rows (see eogp_sign_pack_tiled in eogp.h)."""
    steps = sum(int(k) for k in k_per_module) // 512
    return -(-int(N) // 32) * steps * 2048


def eogp_sign_pack_tiled(X, codes, row0, steps_per_row, step0, scales, stream=None):
    """Sign bits of X [N, k] into rows row0 .. row0+N-1 of a tiled store
    (uint8, tiled_store_bytes long) at the module's first step step0, and
    the fp16 scales into scales (int16 [N] or a column of an [N, U] array)."""
    L = load()
    _need_cuda(X, codes, scales)
    N, k = X.shape
    if codes.dtype != torch.uint8 or not codes.is_contiguous():
        raise ValueError("codes must be a contiguous uint8 tiled store")
    need = -(-(int(row0) + N) // 32) * int(steps_per_row) * 2048
    if N > 0 and codes.numel() < need:
        raise ValueError(f"the tiled store needs at least {need} bytes for these rows")
    sstride = scales.stride(0) if scales.dim() == 2 else 1
    _check(L.eogp_sign_pack_tiled(_ptr(X), X.stride(0), N, k, int(row0), _ptr(codes),
                                  int(steps_per_row), int(step0), _ptr(scales), sstride,
                                  _stream(stream)))
    return codes, scales


def eogp_score_topk_tiled(codes, scales, N, k_per_module, Y, topk, full_scores=False,
                          out_idx=None, out_score=None, ws=None, stream=None):
    """eogp_score_topk over a tiled store of N rows (codes: the uint8 store)."""
    L = load()
    U = len(k_per_module)
    if codes.dtype != torch.uint8 or not codes.is_contiguous():
        raise ValueError("codes must be a contiguous uint8 tiled store")
    if N > 0 and codes.numel() < tiled_store_bytes(N, k_per_module):
        raise ValueError("the tiled store is too small for N rows")
    if scales.dtype not in (torch.int16, torch.float16) or not scales.is_contiguous() or \
            scales.numel() != N * U:
        raise ValueError("scales must be contiguous fp16 bits [N, U]")
    if Y.dtype != torch.float32 or Y.dim() != 2 or (Y.shape[0] > 0 and Y.stride(1) != 1):
        raise ValueError("Y must be float32 [Q, sum k_u] with unit column stride")
    _need_cuda(codes, scales, Y)
    Q = Y.shape[0]
    ks = (c_i64 * U)(*[int(k) for k in k_per_module])
    if out_idx is None:
        out_idx = torch.empty((Q, topk), dtype=torch.int64, device=Y.device)
    if out_score is None:
        out_score = torch.empty((Q, topk), dtype=torch.float32, device=Y.device)
    full = torch.empty((Q, N), dtype=torch.float32, device=Y.device) if full_scores else None
    need = int(L.eogp_score_topk_workspace_size(N, Q, U, ks, topk))
    ws, wsb = _workspace(need, Y.device, ws, less_ok=True)
    ldy = Y.stride(0) if Q > 0 else sum(int(k) for k in k_per_module)
    status = L.eogp_score_topk_tiled(_ptr(codes), _ptr(scales), N, U, ks, _ptr(Y), ldy, Q, topk,
                                     _ptr(out_idx), _ptr(out_score), _ptr(full), _ptr(ws), wsb,
                                     _stream(stream))
    _check_workspace(status, need)
    return out_idx, out_score, full


def eogp_score_topk_workspace_size(N, Q, k_per_module, topk) -> int:
    ks = (c_i64 * len(k_per_module))(*[int(k) for k in k_per_module])
    return int(load().eogp_score_topk_workspace_size(N, Q, len(k_per_module), ks, topk))


def _score_layout(codes, scales, k_per_module, Y):
    U = len(k_per_module)
    if codes.dtype != torch.uint8 or codes.dim() != 2 or (codes.shape[0] > 0 and codes.stride(1) != 1):
        raise ValueError("codes must be uint8 [N, row bytes] with unit column stride")
    N = codes.shape[0]
    if scales.dtype not in (torch.int16, torch.float16):
        raise ValueError("scales must hold fp16 bit patterns (int16 or float16)")
    if not ((scales.dim() == 2 and tuple(scales.shape) == (N, U)) or
            (scales.dim() == 1 and U == 1 and scales.shape[0] == N)) or not scales.is_contiguous():
        raise ValueError("scales must be contiguous [N, U] (or [N] for one module)")
    if Y.dtype != torch.float32 or Y.dim() != 2 or (Y.shape[0] > 0 and Y.stride(1) != 1):
        raise ValueError("Y must be float32 [Q, sum k_u] with unit column stride")
    _need_cuda(codes, scales, Y)
    ksum = sum(int(k) for k in k_per_module)
    # an empty tensor may report stride 0; with no rows any valid stride will do
    cstride = codes.stride(0) if N > 0 else ksum // 8
    ldy = Y.stride(0) if Y.shape[0] > 0 else ksum
    return N, Y.shape[0], U, cstride, ldy


def eogp_score_topk_noalloc(codes, scales, k_per_module, Y, topk, out_idx, out_score,
                            full_scores=None, stream=None):
    """eogp_score_topk without a workspace (see eogp_score_topk_noalloc in
    eogp.h): the library's per-GPU scratch array serves as workspace, so the
    call allocates nothing; outputs are the caller's (index int64 [Q, topk],
    score float32 [Q, topk], optionally every score float32 [Q, N])."""
    L = load()
    N, Q, U, cstride, ldy = _score_layout(codes, scales, k_per_module, Y)
    _need_cuda(out_idx, out_score, full_scores)
    if (out_idx.dtype != torch.int64 or tuple(out_idx.shape) != (Q, topk) or not out_idx.is_contiguous()
            or out_score.dtype != torch.float32 or tuple(out_score.shape) != (Q, topk)
            or not out_score.is_contiguous()):
        raise ValueError("out_idx / out_score must be contiguous int64 / float32 [Q, topk]")
    if full_scores is not None and (full_scores.dtype != torch.float32 or
                                    tuple(full_scores.shape) != (Q, N) or
                                    not full_scores.is_contiguous()):
        raise ValueError("full_scores must be contiguous float32 [Q, N]")
    ks = (c_i64 * U)(*[int(k) for k in k_per_module])
    _check(L.eogp_score_topk_noalloc(_ptr(codes), cstride, _ptr(scales), N, U, ks, _ptr(Y), ldy, Q,
                                     topk, _ptr(out_idx), _ptr(out_score), _ptr(full_scores),
                                     _stream(stream)))
    return out_idx, out_score, full_scores


def eogp_score_topk(codes, scales, k_per_module, Y, topk, full_scores=False, out_idx=None,
                    out_score=None, ws=None, stream=None):
    """Per-query top-k (index int64 [Q, topk], score float32 [Q, topk]) and
    optionally every score (float32 [Q, N])."""
    L = load()
    N, Q, U, cstride, ldy = _score_layout(codes, scales, k_per_module, Y)
    ks = (c_i64 * U)(*[int(k) for k in k_per_module])
    if out_idx is None:
        out_idx = torch.empty((Q, topk), dtype=torch.int64, device=Y.device)
    if out_score is None:
        out_score = torch.empty((Q, topk), dtype=torch.float32, device=Y.device)
    full = torch.empty((Q, N), dtype=torch.float32, device=Y.device) if full_scores else None
    need = int(L.eogp_score_topk_workspace_size(N, Q, U, ks, topk))
    ws, wsb = _workspace(need, Y.device, ws, less_ok=True)
    status = L.eogp_score_topk(_ptr(codes), cstride, _ptr(scales), N, U, ks, _ptr(Y), ldy, Q,
                               topk, _ptr(out_idx), _ptr(out_score), _ptr(full), _ptr(ws), wsb,
                               _stream(stream))
    _check_workspace(status, need)
    return out_idx, out_score, full


# ---------------------------------------------------------------------------
# The ends of a language model: embedding, layer norm, cross-entropy, sampling
# ---------------------------------------------------------------------------
def _empty(shape, dtype, device, stream):
    """A new tensor that belongs to the stream the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


# The stream and the addresses as plain integers: calls of a few microseconds (a decoding step's
# norm, a short query) are as long as their marshalling, and a Stream object alone costs 2.8 us.
_raw_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(stream, device):
    if stream is not None:
        return stream.cuda_stream
    if _raw_current_stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    return _raw_current_stream(device.index)


def _at(t):
    return None if t is None else t.data_ptr()


# The device that kernels are launched on. (Asked for after a device tensor has been seen, so the
# runtime is there; torch.cuda.current_device() would look for that again.)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _need_here(stream, first, *ts):
    """Device tensors, and a stream if there is one, of the device that kernels are launched on."""
    here = first.get_device()
    if here >= 0 and here != _current_device():
        _refuse_device(_current_device(), here)
    for t in ts:
        if t is not None and t.get_device() != here:
            _refuse_device(here, t.get_device())
    if here < 0:
        _refuse_device(here, here)
    if stream is not None and stream.device_index != here:
        raise ValueError(f"stream must belong to the current device cuda:{here}, not cuda:{stream.device_index}")


def _refuse_device(here, there):
    if min(here, there) < 0:
        raise ValueError("EOGP arguments must be device tensors")
    raise ValueError(f"EOGP arguments must be on the current device cuda:{here}, not cuda:{there}")


def _scratch(need, device, ws, stream):
    """The caller's workspace, or a new one that belongs to the stream the call runs on."""
    if ws is None:
        return (_empty((need,), torch.uint8, device, stream), need) if need else (None, 0)
    if not ws.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return _workspace(need, device, ws)


def _rows_of(x, name):
    """(rows, width, row stride) of a [n, d] or [N, T, d] tensor whose rows have
    unit column stride and lie at one constant stride."""
    if x.dim() not in (2, 3):
        raise ValueError(f"{name} must be [n, d] or [N, T, d]")
    d = x.shape[-1]
    if d > 0 and x.is_contiguous():
        return x.numel() // d, d, d
    if x.dim() == 2:
        n, T = x.shape[0], 1
        ld = x.stride(0)
    else:
        N, T = x.shape[0], x.shape[1]
        n = N * T
        ld = x.stride(1) if T > 1 else x.stride(0)
        if N > 1 and T > 1 and x.stride(0) != T * ld:
            raise ValueError(f"{name} must have its rows at a constant row stride")
    if d > 1 and x.stride(-1) != 1:
        raise ValueError(f"{name} must have unit column stride")
    if n > 1 and ld < d:
        raise ValueError(f"{name} must not have overlapping rows")
    return n, d, (ld if n > 1 else max(ld, d))


def _model_dtype(x, name):
    code = _DTYPE_CODE.get(x.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16")
    return code


def _per_row(x, lead, dtype, name):
    """A contiguous tensor with one element per row, or None."""
    if x is not None and (x.dtype != dtype or x.shape != lead or not x.is_contiguous()):
        raise ValueError(f"{name} must be contiguous {str(dtype)[6:]} {list(lead)}")


def _weight(w, d, x, name):
    if w is not None and (w.dim() != 1 or w.shape[0] != d or not w.is_contiguous()
                          or (w.dtype != x.dtype and w.dtype != torch.float32)):
        raise ValueError(f"{name} must be contiguous [{d}] of the rows' type or float32")


def _same_shape(x, like, name):
    if x.shape != like.shape or x.dtype != like.dtype:
        raise ValueError(f"{name} must have the shape and type of its counterpart")


def eogp_embed_tokens(table, tokens, scale=1.0, token_mask=None, out=None, accumulate=False,
                      stream=None):
    """out [*tokens.shape, d] = scale * table[tokens] (table [V, d]; tokens int64 [n]
    or [N, T]), added to `out` if accumulate; see eogp_embed_tokens in eogp.h."""
    L = load()
    _need_here(stream, table, tokens, token_mask, out)
    V, d, ldt = _rows_of(table, "table")
    if table.dim() != 2 or tokens.dim() not in (1, 2):
        raise ValueError("table must be [V, d] and tokens [n] or [N, T]")
    lead = tokens.shape
    _per_row(tokens, lead, torch.int64, "tokens")
    _per_row(token_mask, lead, torch.uint8, "token_mask")
    if out is None:
        if accumulate:
            raise ValueError("accumulate adds to a caller's out")
        out = _empty((*lead, d), table.dtype, table.device, stream)
    if tuple(out.shape) != (*lead, d) or out.dtype not in (table.dtype, torch.float32):
        raise ValueError("out must be [*tokens.shape, d] of the table's type or float32")
    n, _, ldo = _rows_of(out, "out")
    _check(L.eogp_embed_tokens(_at(table), _model_dtype(table, "table"), ldt, V, d, _at(tokens),
                               _at(token_mask), n, float(scale), 1 if accumulate else 0, _at(out),
                               _DTYPE_CODE[out.dtype], ldo, _stream_handle(stream, out.device)))
    return out


def eogp_embed_backward_workspace_size(n: int, V: int, d: int) -> int:
    return int(load().eogp_embed_backward_workspace_size(n, V, d))


def eogp_embed_backward(d_out, tokens, V, scale=1.0, token_mask=None, dtable=None, accumulate=False,
                        ws=None, stream=None):
    """dtable [V, d] (float32) = scale * sum of d_out's rows by token, added to
    `dtable` if accumulate; see eogp_embed_backward in eogp.h."""
    L = load()
    _need_here(stream, d_out, tokens, token_mask, dtable, ws)
    n, d, ldd = _rows_of(d_out, "d_out")
    lead = d_out.shape[:-1]
    _per_row(tokens, lead, torch.int64, "tokens")
    _per_row(token_mask, lead, torch.uint8, "token_mask")
    if dtable is None:
        if accumulate:
            raise ValueError("accumulate adds to a caller's dtable")
        dtable = _empty((V, d), torch.float32, d_out.device, stream)
    if dtable.dtype != torch.float32 or tuple(dtable.shape) != (V, d):
        raise ValueError("dtable must be float32 [V, d]")
    _, _, ldt = _rows_of(dtable, "dtable")
    need = eogp_embed_backward_workspace_size(n, V, d)
    ws, wsb = _scratch(need, d_out.device, ws, stream)
    _check(L.eogp_embed_backward(_at(d_out), _model_dtype(d_out, "d_out"), ldd, _at(tokens),
                                 _at(token_mask), n, V, d, float(scale), 1 if accumulate else 0,
                                 _at(dtable), ldt, _at(ws), wsb,
                                 _stream_handle(stream, dtable.device)))
    return dtable


def eogp_layer_norm(x, gamma=None, beta=None, eps=1e-5, token_mask=None, ones_column=False, out=None,
                    mean=None, rstd=None, stream=None):
    """(y, mean, rstd) of x [n, d] or [N, T, d]; with ones_column y has d + 1
    columns, the last 1 in valid rows (a new y then has rows of a multiple of 16
    elements); see eogp_layer_norm in eogp.h."""
    L = load()
    _need_here(stream, x, gamma, beta, token_mask, out, mean, rstd)
    n, d, ldx = _rows_of(x, "x")
    lead, width = x.shape[:-1], d + (1 if ones_column else 0)
    _per_row(token_mask, lead, torch.uint8, "token_mask")
    _weight(gamma, d, x, "gamma")
    _weight(beta, d, x, "beta")
    if gamma is not None and beta is not None and gamma.dtype != beta.dtype:
        raise ValueError("gamma and beta must have one type")
    if out is None:
        ld = -(-width // 16) * 16 if ones_column else width
        out = _empty((*lead, ld), x.dtype, x.device, stream)[..., :width]
    if tuple(out.shape) != (*lead, width) or out.dtype not in (x.dtype, torch.float32):
        raise ValueError("out must be [..., d (+ 1 with ones_column)] of x's type or float32")
    _, _, ldy = _rows_of(out, "out")
    if mean is None:
        mean = _empty(lead, torch.float32, x.device, stream)
    if rstd is None:
        rstd = _empty(lead, torch.float32, x.device, stream)
    _per_row(mean, lead, torch.float32, "mean")
    _per_row(rstd, lead, torch.float32, "rstd")
    w = gamma if gamma is not None else beta
    _check(L.eogp_layer_norm(_at(x), _model_dtype(x, "x"), ldx, _at(gamma), _at(beta),
                             F32 if w is None else _DTYPE_CODE[w.dtype], float(eps), _at(token_mask), n,
                             d, _at(out), _DTYPE_CODE[out.dtype], ldy, 1 if ones_column else 0,
                             _at(mean), _at(rstd), _stream_handle(stream, x.device)))
    return out, mean, rstd


def eogp_layer_norm_backward_workspace_size(groups: int, rows: int, d: int, dtype: int) -> int:
    return int(load().eogp_layer_norm_backward_workspace_size(groups, rows, d, dtype))


def eogp_layer_norm_backward(dy, x, gamma, mean, rstd, token_mask=None, residual=None,
                             per_example=False, dx=None, dgamma=None, dbeta=None, ws=None, stream=None):
    """(dx, dgamma, dbeta): gradient at x (plus `residual`), and the weight and bias
    gradients, float32 [d] or with per_example [N, d] (x [N, T, d]); see
    eogp_layer_norm_backward in eogp.h."""
    L = load()
    _need_here(stream, dy, x, gamma, mean, rstd, token_mask, residual, dx, dgamma, dbeta, ws)
    n, d, ldx = _rows_of(x, "x")
    lead = x.shape[:-1]
    _same_shape(dy, x, "dy")
    _, _, lddy = _rows_of(dy, "dy")
    _weight(gamma, d, x, "gamma")
    _per_row(token_mask, lead, torch.uint8, "token_mask")
    for t, name in ((mean, "mean"), (rstd, "rstd")):
        if t is None:
            raise ValueError(f"the backward pass reads the forward pass's {name}")
        _per_row(t, lead, torch.float32, name)
    ldr = 0
    if residual is not None:
        _same_shape(residual, x, "residual")
        _, _, ldr = _rows_of(residual, "residual")
    if dx is None:
        dx = _empty(tuple(x.shape), x.dtype, x.device, stream)
    _same_shape(dx, x, "dx")
    _, _, lddx = _rows_of(dx, "dx")
    if per_example and x.dim() != 3:
        raise ValueError("per-example gradients need x [N, T, d]")
    groups = x.shape[0] if per_example else 1
    rows = x.shape[1] if per_example else n
    shape = (groups, d) if per_example else (d,)
    if dgamma is None:
        dgamma = _empty(shape, torch.float32, x.device, stream)
    if dbeta is None:
        dbeta = _empty(shape, torch.float32, x.device, stream)
    _per_row(dgamma, shape, torch.float32, "dgamma")
    _per_row(dbeta, shape, torch.float32, "dbeta")
    code = _model_dtype(x, "x")
    need = eogp_layer_norm_backward_workspace_size(groups, rows, d, code)
    ws, wsb = _scratch(need, x.device, ws, stream)
    _check(L.eogp_layer_norm_backward(_at(dy), lddy, _at(x), ldx, code, _at(gamma),
                                      F32 if gamma is None else _DTYPE_CODE[gamma.dtype], _at(mean),
                                      _at(rstd), _at(token_mask), _at(residual), ldr, groups, rows, d,
                                      _at(dx), lddx, _at(dgamma), _at(dbeta), _at(ws), wsb,
                                      _stream_handle(stream, x.device)))
    return dx, dgamma, dbeta


def eogp_softmax_xent(logits, labels, token_mask=None, grad_scale=1.0, grad=True, loss=None,
                      dlogits=None, stream=None):
    """(loss float32, dlogits) of logits [n, V] or [N, T, V] and labels int64 [n] or
    [N, T]; grad=False leaves dlogits out (None); dlogits may be the logits; see
    eogp_softmax_xent in eogp.h."""
    L = load()
    _need_here(stream, logits, labels, token_mask, loss, dlogits)
    n, V, ldl = _rows_of(logits, "logits")
    lead = logits.shape[:-1]
    _per_row(labels, lead, torch.int64, "labels")
    _per_row(token_mask, lead, torch.uint8, "token_mask")
    if loss is None:
        loss = _empty(lead, torch.float32, logits.device, stream)
    _per_row(loss, lead, torch.float32, "loss")
    if not grad and dlogits is not None:
        raise ValueError("dlogits without grad")
    ldd = 0
    if grad:
        if dlogits is None:
            dlogits = _empty(tuple(logits.shape), logits.dtype, logits.device, stream)
        _same_shape(dlogits, logits, "dlogits")
        _, _, ldd = _rows_of(dlogits, "dlogits")
    _check(L.eogp_softmax_xent(_at(logits), _model_dtype(logits, "logits"), ldl, _at(labels),
                               _at(token_mask), n, V, float(grad_scale), _at(loss), _at(dlogits), ldd,
                               _stream_handle(stream, logits.device)))
    return loss, dlogits


def eogp_sample_tokens(logits, uniforms=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
                       token_mask=None, out=None, stream=None):
    """Tokens int64 drawn from logits [n, V] or [N, T, V] with uniforms float32 [n] or
    [N, T] in [0, 1); see eogp_sample_tokens in eogp.h."""
    L = load()
    _need_here(stream, logits, uniforms, token_mask, out)
    n, V, ldl = _rows_of(logits, "logits")
    lead = logits.shape[:-1]
    _per_row(uniforms, lead, torch.float32, "uniforms")
    _per_row(token_mask, lead, torch.uint8, "token_mask")
    if out is None:
        out = _empty(lead, torch.int64, logits.device, stream)
    _per_row(out, lead, torch.int64, "out")
    _check(L.eogp_sample_tokens(_at(logits), _model_dtype(logits, "logits"), ldl, n, V, _at(uniforms),
                                _at(token_mask), float(temperature), int(top_k), float(top_p),
                                float(min_p), _at(out), _stream_handle(stream, logits.device)))
    return out


# ---------------------------------------------------------------------------
# The middle of a block: rotary positions, norms of queries and keys, attention
# ---------------------------------------------------------------------------
NORMS = {"none": 0, "head": 1, "row": 2}


def _heads_of(x, name):
    """[N, T, heads, D] with unit stride in its last dimension, as the library takes it."""
    s = x.stride()
    if len(s) != 4:
        raise ValueError(f"{name} must be [N, T, heads, D]")
    if s[3] != 1 and x.shape[3] > 1:
        if x.numel():
            raise ValueError(f"{name} must have unit stride within a head")
        s = (0, 0, 0)
    return Heads(x.data_ptr(), x.shape[2], s[0], s[1], s[2])


def _heads_like(x, like, shape, name):
    """The same of a tensor with the shape and type of `like`."""
    if x is not like and (x.shape != shape or x.dtype != like.dtype):
        raise ValueError(f"{name} must have the shape and type of its counterpart")
    return _heads_of(x, name)


def _norm_weights(norm, weight, x, shape, name):
    if weight is None:
        return
    if norm == 0:
        raise ValueError(f"{name} without a norm")
    _weight(weight, shape[3] if norm == 1 else shape[2] * shape[3], x, name)


def _table_shape(table):
    """(positions, width) of a rotary table, (0, 0) without one."""
    if table is None:
        return 0, 0
    if table.dim() != 3 or table.shape[2] != 2 or table.dtype != torch.float32 or not table.is_contiguous():
        raise ValueError("table must be contiguous float32 [positions, width / 2, 2]")
    return table.shape[0], 2 * table.shape[1]


def eogp_rotary_table(positions, width, base=10000.0, factor=1.0, original=0, low=1.0, high=32.0, magnitude=1.0,
                      out=None, device=None, stream=None):
    """(cos, sin) of positions 0 .. positions - 1 times each pair's frequency, float32 [positions, width / 2, 2];
    `factor`, `original`, `low` and `high` scale frequencies for long contexts; see eogp_rotary_table in eogp.h."""
    L = load()
    if positions < 0 or width < 2 or width % 2:
        raise ValueError("a table needs positions >= 0 and an even width >= 2")
    if out is None:
        device = torch.device("cuda", _current_device()) if device is None else torch.device(device)
        out = _empty((positions, width // 2, 2), torch.float32, device, stream)
    _need_here(stream, out)
    if out.dtype != torch.float32 or tuple(out.shape) != (positions, width // 2, 2) or not out.is_contiguous():
        raise ValueError("out must be contiguous float32 [positions, width / 2, 2]")
    _check(L.eogp_rotary_table(positions, width, float(base), float(factor), float(original), float(low), float(high),
                               float(magnitude), _at(out), _stream_handle(stream, out.device)))
    return out


def eogp_rotate_heads(q, k=None, table=None, positions=None, norm="none", q_weight=None, k_weight=None, eps=1e-6,
                      interleaved=False, token_mask=None, q_out=None, k_out=None, stream=None):
    """(q_out, k_out) of queries [N, T, heads, D] and keys [N, T, key heads, D] or None: normed (norm "head", "row" or
    "none") and turned by their positions; see eogp_rotate_heads in eogp.h."""
    L = load()
    _need_here(stream, q, k, table, positions, q_weight, k_weight, token_mask, q_out, k_out)
    code = _model_dtype(q, "q")
    qh, kh, ok = _heads_of(q, "q"), None, None
    shape = q.shape
    N, T, _, D = shape
    if norm not in NORMS:
        raise ValueError(f"norm must be one of {', '.join(NORMS)}")
    nc = NORMS[norm]
    _norm_weights(nc, q_weight, q, shape, "q_weight")
    P, width = _table_shape(table)
    lead = (N, T)
    _per_row(positions, lead, torch.int64, "positions")
    _per_row(token_mask, lead, torch.uint8, "token_mask")
    if q_out is None:
        q_out = _empty(tuple(shape), q.dtype, q.device, stream)
    oq = _heads_like(q_out, q, shape, "q_out")
    if k is not None:
        ks = k.shape
        if len(ks) != 4 or ks[0] != N or ks[1] != T or ks[3] != D or k.dtype != q.dtype:
            raise ValueError("k must be [N, T, key heads, D] of q's type")
        kh = _heads_of(k, "k")
        _norm_weights(nc, k_weight, k, ks, "k_weight")
        if q_weight is not None and k_weight is not None and q_weight.dtype != k_weight.dtype:
            raise ValueError("q_weight and k_weight must have one type")
        if k_out is None:
            k_out = _empty(tuple(ks), k.dtype, k.device, stream)
        ok = _heads_like(k_out, k, ks, "k_out")
    elif k_out is not None or k_weight is not None:
        raise ValueError(f"{'k_weight' if k_out is None else 'k_out'} without k")
    w = q_weight if q_weight is not None else k_weight
    _check(L.eogp_rotate_heads(ctypes.byref(qh), kh and ctypes.byref(kh), code, N, T, D, nc, _at(q_weight), _at(k_weight),
                               F32 if w is None else _DTYPE_CODE[w.dtype], float(eps), _at(table), P, width,
                               1 if interleaved else 0, _at(positions), _at(token_mask), ctypes.byref(oq),
                               ok and ctypes.byref(ok), _stream_handle(stream, q.device)))
    return q_out, k_out


def eogp_rotate_heads_backward_workspace_size(N, T, q_heads, k_heads, D, dtype, norm="none", width=0,
                                              per_example=False) -> int:
    return int(load().eogp_rotate_heads_backward_workspace_size(N, T, q_heads, k_heads, D, dtype, NORMS[norm], width,
                                                                1 if per_example else 0))


def eogp_rotate_heads_backward(dq, dk=None, q=None, k=None, table=None, positions=None, norm="none", q_weight=None,
                               k_weight=None, eps=1e-6, interleaved=False, token_mask=None, per_example=False, dq_in=None,
                               dk_in=None, dq_weight=None, dk_weight=None, ws=None, stream=None):
    """(dq_in, dk_in, dq_weight, dk_weight): gradients at the inputs q, k (read only with a norm) of eogp_rotate_heads
    from those of its outputs, and with a norm those of the weights, float32 [weight] or with per_example
    [N, weight]; see eogp_rotate_heads_backward in eogp.h."""
    L = load()
    _need_here(stream, dq, dk, q, k, table, positions, q_weight, k_weight, token_mask, dq_in, dk_in, dq_weight, dk_weight, ws)
    code = _model_dtype(dq, "dq")
    gq, gk, xq, xk, ok = _heads_of(dq, "dq"), None, None, None, None
    shape = dq.shape
    N, T, Hq, D = shape
    if norm not in NORMS:
        raise ValueError(f"norm must be one of {', '.join(NORMS)}")
    nc = NORMS[norm]
    if nc:
        if q is None or (dk is not None and k is None):
            raise ValueError("a norm's backward pass reads the forward pass's inputs")
        xq = _heads_like(q, dq, shape, "q")
    _norm_weights(nc, q_weight, dq, shape, "q_weight")
    P, width = _table_shape(table)
    lead = (N, T)
    _per_row(positions, lead, torch.int64, "positions")
    _per_row(token_mask, lead, torch.uint8, "token_mask")
    if dq_in is None:
        dq_in = _empty(tuple(shape), dq.dtype, dq.device, stream)
    oq = _heads_like(dq_in, dq, shape, "dq_in")
    if dk is not None:
        ks = dk.shape
        if len(ks) != 4 or ks[0] != N or ks[1] != T or ks[3] != D or dk.dtype != dq.dtype:
            raise ValueError("dk must be [N, T, key heads, D] of dq's type")
        gk = _heads_of(dk, "dk")
        if nc:
            xk = _heads_like(k, dk, ks, "k")
        _norm_weights(nc, k_weight, dk, ks, "k_weight")
        if q_weight is not None and k_weight is not None and q_weight.dtype != k_weight.dtype:
            raise ValueError("q_weight and k_weight must have one type")
        if dk_in is None:
            dk_in = _empty(tuple(ks), dk.dtype, dk.device, stream)
        ok = _heads_like(dk_in, dk, ks, "dk_in")
    elif dk_in is not None or dk_weight is not None or k_weight is not None:
        raise ValueError("dk_in, dk_weight and k_weight need dk")
    if nc:
        lead = (N,) if per_example else ()
        size = (*lead, D if nc == 1 else Hq * D)
        if dq_weight is None:
            dq_weight = _empty(size, torch.float32, dq.device, stream)
        _per_row(dq_weight, size, torch.float32, "dq_weight")
        if dk is not None:
            size = (*lead, D if nc == 1 else ks[2] * D)
            if dk_weight is None:
                dk_weight = _empty(size, torch.float32, dk.device, stream)
            _per_row(dk_weight, size, torch.float32, "dk_weight")
    elif dq_weight is not None or dk_weight is not None:
        raise ValueError("weight gradients without a norm")
    need = int(L.eogp_rotate_heads_backward_workspace_size(N, T, Hq, 0 if dk is None else dk.shape[2], D, code, nc, width,
                                                           1 if per_example else 0)) if nc else 0
    ws, wsb = _scratch(need, dq.device, ws, stream)
    w = q_weight if q_weight is not None else k_weight
    ref = lambda x: x and ctypes.byref(x)                              # noqa: E731
    _check(L.eogp_rotate_heads_backward(ref(gq), ref(gk), ref(xq), ref(xk), code, N, T, D, nc, _at(q_weight),
                                        _at(k_weight), F32 if w is None else _DTYPE_CODE[w.dtype], float(eps), _at(table),
                                        P, width, 1 if interleaved else 0, _at(positions), _at(token_mask),
                                        1 if per_example else 0, ref(oq), ref(ok), _at(dq_weight), _at(dk_weight), _at(ws),
                                        wsb, _stream_handle(stream, dq.device)))
    return dq_in, dk_in, dq_weight, dk_weight


def _attention_shapes(q, k, v, q_start, q_mask, k_mask):
    """Sizes (N, Tq, Tk, Hq, Hkv, D) of queries [N, Tq, Hq, D], keys and values [N, Tk, Hkv, D]."""
    qs, ks = q.shape, k.shape
    if len(qs) != 4 or len(ks) != 4:
        raise ValueError("q must be [N, Tq, heads, D], k and v [N, Tk, key heads, D]")
    N, Tq, Hq, D = qs
    _, Tk, Hkv, _ = ks
    if ks[0] != N or ks[3] != D or v.shape != ks or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("k and v must be [N, Tk, key heads, D] of q's type")
    _per_row(q_start, (N,), torch.int64, "q_start")
    _per_row(q_mask, (N, Tq), torch.uint8, "q_mask")
    _per_row(k_mask, (N, Tk), torch.uint8, "k_mask")
    return N, Tq, Tk, Hq, Hkv, D


def eogp_attention_workspace_size(N, Tq, Tk, q_heads, k_heads, D, dtype) -> int:
    return int(load().eogp_attention_workspace_size(N, Tq, Tk, q_heads, k_heads, D, dtype))


def eogp_attention(q, k, v, scale=None, causal=True, window=0, sinks=0, q_start=None, q_mask=None, k_mask=None,
                   out=None, lse=None, stats=True, ws=None, stream=None):
    """(out, lse): softmax attention of queries [N, Tq, heads, D] over keys and values [N, Tk, key heads, D], and the
    rows' log-sum-exp, float32 [N, Tq, heads] (stats=False: left out, None). scale is D^-1/2 unless given; see
    eogp_attention in eogp.h."""
    L = load()
    _need_here(stream, q, k, v, q_start, q_mask, k_mask, out, lse, ws)
    code = _model_dtype(q, "q")
    N, Tq, Tk, Hq, Hkv, D = _attention_shapes(q, k, v, q_start, q_mask, k_mask)
    if out is None:
        out = _empty((N, Tq, Hq, D), q.dtype, q.device, stream)
    if out.shape != q.shape or out.dtype not in (q.dtype, torch.float32):
        raise ValueError("out must be [N, Tq, heads, D] of q's type or float32")
    if stats and lse is None:
        lse = _empty((N, Tq, Hq), torch.float32, q.device, stream)
    if not stats and lse is not None:
        raise ValueError("lse without stats")
    _per_row(lse, (N, Tq, Hq), torch.float32, "lse")
    need = int(L.eogp_attention_workspace_size(N, Tq, Tk, Hq, Hkv, D, code))
    ws, wsb = _scratch(need, q.device, ws, stream)
    ref = ctypes.byref
    _check(L.eogp_attention(ref(_heads_of(q, "q")), ref(_heads_of(k, "k")), ref(_heads_of(v, "v")), code, N, Tq, Tk, D,
                            D ** -0.5 if scale is None and D else float(scale or 0), 1 if causal else 0, int(window),
                            int(sinks), _at(q_start), _at(q_mask), _at(k_mask), ref(_heads_of(out, "out")),
                            _DTYPE_CODE[out.dtype], _at(lse), _at(ws), wsb, _stream_handle(stream, q.device)))
    return out, lse


def eogp_attention_backward_workspace_size(N, Tq, Tk, q_heads, k_heads, D, dtype) -> int:
    return int(load().eogp_attention_backward_workspace_size(N, Tq, Tk, q_heads, k_heads, D, dtype))


def eogp_attention_backward(dout, q, k, v, out, lse, scale=None, causal=True, window=0, sinks=0, q_start=None,
                            q_mask=None, k_mask=None, dq=None, dk=None, dv=None, ws=None, stream=None):
    """(dq, dk, dv) from the gradient of eogp_attention's out, with its out and lse and the same other arguments; see
    eogp_attention_backward in eogp.h."""
    L = load()
    _need_here(stream, dout, q, k, v, out, lse, q_start, q_mask, k_mask, dq, dk, dv, ws)
    code = _model_dtype(q, "q")
    N, Tq, Tk, Hq, Hkv, D = _attention_shapes(q, k, v, q_start, q_mask, k_mask)
    if out.shape != q.shape or out.dtype not in (q.dtype, torch.float32):
        raise ValueError("out must be [N, Tq, heads, D] of q's type or float32")
    if lse is None:
        raise ValueError("the backward pass reads the forward pass's lse")
    _per_row(lse, (N, Tq, Hq), torch.float32, "lse")
    dq = _empty(tuple(q.shape), q.dtype, q.device, stream) if dq is None else dq
    dk = _empty(tuple(k.shape), k.dtype, k.device, stream) if dk is None else dk
    dv = _empty(tuple(v.shape), v.dtype, v.device, stream) if dv is None else dv
    need = int(L.eogp_attention_backward_workspace_size(N, Tq, Tk, Hq, Hkv, D, code))
    ws, wsb = _scratch(need, q.device, ws, stream)
    ref = ctypes.byref
    _check(L.eogp_attention_backward(ref(_heads_like(dout, q, q.shape, "dout")), ref(_heads_of(q, "q")), ref(_heads_of(k, "k")),
                                     ref(_heads_of(v, "v")), code, N, Tq, Tk, D,
                                     D ** -0.5 if scale is None and D else float(scale or 0), 1 if causal else 0,
                                     int(window), int(sinks), _at(q_start), _at(q_mask), _at(k_mask),
                                     ref(_heads_of(out, "out")), _DTYPE_CODE[out.dtype], _at(lse),
                                     ref(_heads_like(dq, q, q.shape, "dq")), ref(_heads_like(dk, k, k.shape, "dk")),
                                     ref(_heads_like(dv, v, k.shape, "dv")), _at(ws), wsb, _stream_handle(stream, q.device)))
    return dq, dk, dv


def eogp_version() -> int:
    return int(load().eogp_version())


# ---------------------------------------------------------------------------
# Kernel timing (measurement harnesses)
# ---------------------------------------------------------------------------
KT_ROTATION_GEMM, KT_RETAINED, KT_PCA_GEMM, KT_SIGN_PACK = 0, 1, 2, 3
KT_SCORE_PASS, KT_SCORE_MERGE, KT_SCORE_PREP, KT_COMPACTION = 4, 5, 6, 7
KT_SRHT, KT_EKFAC, KT_PCA_FIT = 8, 9, 10
KT_EMBED, KT_LAYER_NORM, KT_XENT, KT_SAMPLE = 11, 12, 13, 14
KT_ROTARY, KT_ATTENTION = 15, 16
KERNEL_CLASSES = {"rotation_gemm": 0, "retained": 1, "pca_gemm": 2, "sign_pack": 3,
                  "score_pass": 4, "score_merge": 5, "score_prep": 6, "compaction": 7,
                  "srht": 8, "ekfac": 9, "pca_fit": 10, "embed": 11, "layer_norm": 12,
                  "xent": 13, "sample": 14, "rotary": 15, "attention": 16}


def eogp_timing_enable(on: bool = True):
    _check(load().eogp_timing_enable(1 if on else 0))


def eogp_timing_read(kernel_class: int):
    """(total milliseconds, launches) of one kernel class since the last read."""
    ms = ctypes.c_double()
    n = c_i64()
    _check(load().eogp_timing_read(int(kernel_class), ctypes.byref(ms), ctypes.byref(n)))
    return float(ms.value), int(n.value)
