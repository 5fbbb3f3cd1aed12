"""MI355X (gfx950) BitsMoE spectral quantizer: Python binding of libbitsmoe.

Thin ctypes marshalling over the C ABI declared in ``include/bitsmoe.h``.
Every step runs in the library (HIP kernels on the device, LAPACK and the
exact ILP on the host); torch is used only to allocate device memory and to
name the current stream.  There is no fallback: if the library is not built,
importing the functions raises.

Steps, in order (one projection type of one MoE layer):

    H      = gram(X)                         # X^T X / n
    M      = gram_experts(W)                 # sum_e W_e W_e^T (fp64)
    Ut, ev = shared_basis(M, r)              # top-r eigenvectors (host)
    C      = project(Ut, W)                  # C_e = U^T W_e, [E*r][d_in]
    L      = score(C, H, bits, group)        # delta H delta^T per (unit, width)
    b, obj = allocate(L, bits, budget)       # exact ILP (host)
    off    = pack_layout(b, d)
    codes, params = pack(C, b, off, group)

An MoE layer whose experts are held in microscaled 4-bit floats (MX4):

    codes, scales = mx4_quantize(W)          # once, [E][N][K/2] and [E][N][K/32]
    r = route(logits, k)                     # experts, weights, expert order, losses
    z = mx4_product(codes, scales, x, offsets=r.offsets, rows=r.rows)
    y = combine(z, r.slots, r.weights)
    (route_grad, mx4_product_grad, combine_grad: the gradients)
"""
from __future__ import annotations

import ctypes
import glob
import os
from typing import NamedTuple, Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# BITSMOE_LIB selects another build of the same library (e.g. the
# host-sanitized libbitsmoe_san.so of ``build --sanitize``)
LIB_PATH = os.environ.get("BITSMOE_LIB") or os.path.join(_HERE, "libbitsmoe.so")

OK = 0
_STATUS = {0: "OK", 1: "ERR_ARG", 2: "ERR_SHAPE", 3: "ERR_DTYPE", 4: "ERR_DEVICE",
           5: "ERR_NOMEM", 6: "ERR_NUMERIC", 7: "ERR_INFEASIBLE", 8: "ERR_UNAVAILABLE"}
F32, BF16 = 0, 1

EXPORTS = [
    "bitsmoe_gram", "bitsmoe_gram_experts", "bitsmoe_shared_basis", "bitsmoe_project",
    "bitsmoe_score", "bitsmoe_allocate", "bitsmoe_allocate_ex", "bitsmoe_pack_layout",
    "bitsmoe_pack", "bitsmoe_unpack", "bitsmoe_set_lapack", "bitsmoe_last_error",
    "bitsmoe_release", "bitsmoe_version", "bitsmoe_timing", "bitsmoe_timing_only",
    "bitsmoe_kernel_time",
    "bitsmoe_surrogate", "bitsmoe_surrogate_budget", "bitsmoe_gram_experts_in",
    "bitsmoe_project_in", "bitsmoe_basis_importance", "bitsmoe_score_diag",
    "bitsmoe_gram_routed", "bitsmoe_score_routed", "bitsmoe_moe_decode",
    "bitsmoe_moe_decode_topk", "bitsmoe_shared_basis_gpu", "bitsmoe_moe_decode_in",
    "bitsmoe_moe_decode_topk_noalloc", "bitsmoe_route", "bitsmoe_route_ws", "bitsmoe_route_workspace",
    "bitsmoe_route_grad",
    "bitsmoe_mx4_quantize", "bitsmoe_mx4_dequantize", "bitsmoe_mx4_product",
    "bitsmoe_mx4_product_q", "bitsmoe_mx4_product_grad", "bitsmoe_combine",
    "bitsmoe_combine_grad", "bitsmoe_combine_grad_all",
]
# Candidate widths of the surrogate table, in column order.
SURROGATE_WIDTHS = (0, 1, 2, 3, 4, 6, 8, 16)
_COMBINE_SCAN = 16384  # BITSMOE_COMBINE_SCAN


class BitsmoeError(RuntimeError):
    def __init__(self, status: int, where: str, msg: str):
        self.status = status
        self.code = _STATUS.get(status, str(status))
        super().__init__(f"{where}: {self.code}: {msg}")


_lib = None


def _find_lapack() -> Optional[str]:
    """A LAPACK shared library for the host eigensolve: the one bundled with
    numpy/scipy (OpenBLAS), else the system one."""
    import numpy
    cands = []
    for mod_dir in (os.path.dirname(numpy.__file__),):
        parent = os.path.dirname(mod_dir)
        cands += sorted(glob.glob(os.path.join(parent, "numpy.libs", "libscipy_openblas*.so")))
        cands += sorted(glob.glob(os.path.join(parent, "scipy.libs", "libscipy_openblas*.so")))
    cands += ["liblapack.so.3"]
    return cands[0] if cands else None


def lib() -> ctypes.CDLL:
    """Loads libbitsmoe.so (built by ``paper_2606_00079_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2606_00079_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    L.bitsmoe_gram.argtypes = [vp, i32, i64, i64, vp, vp]
    L.bitsmoe_gram_experts.argtypes = [vp, i32, i64, i64, i64, vp, vp]
    L.bitsmoe_shared_basis.argtypes = [vp, i64, i64, vp, vp, vp, vp]
    L.bitsmoe_project.argtypes = [vp, vp, i32, i64, i64, i64, i64, vp, vp]
    L.bitsmoe_score.argtypes = [vp, i64, i64, vp, vp, i32, i32, vp, vp]
    L.bitsmoe_allocate.argtypes = [vp, i64, vp, i32, i64, vp, vp]
    L.bitsmoe_allocate_ex.argtypes = [vp, i64, vp, i32, i64, vp, vp, i64, vp]
    L.bitsmoe_pack_layout.argtypes = [vp, i64, i64, vp]
    L.bitsmoe_pack.argtypes = [vp, i64, i64, i32, vp, vp, i64, vp, vp, vp]
    L.bitsmoe_unpack.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, vp, vp]
    L.bitsmoe_surrogate.argtypes = [vp, i64, i64, vp, ctypes.c_double, vp, vp, vp, vp]
    L.bitsmoe_surrogate_budget.argtypes = [i64, i64, i64, i64, ctypes.c_double, vp]
    L.bitsmoe_gram_experts_in.argtypes = [vp, i32, i64, i64, i64, vp, vp]
    L.bitsmoe_project_in.argtypes = [vp, vp, i32, i64, i64, i64, i64, vp, vp]
    L.bitsmoe_basis_importance.argtypes = [vp, i64, i64, vp, vp, vp]
    L.bitsmoe_score_diag.argtypes = [vp, i64, i64, vp, i64, vp, i32, i32, vp, vp]
    L.bitsmoe_gram_routed.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp]
    L.bitsmoe_score_routed.argtypes = [vp, i64, i64, vp, i64, vp, i32, i32, vp, vp]
    L.bitsmoe_moe_decode.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i32, vp, i64, vp, i64,
                                     vp, vp, vp, vp, vp]
    L.bitsmoe_shared_basis_gpu.argtypes = [vp, i64, i64, vp, vp, vp, vp]
    L.bitsmoe_moe_decode_in.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i32, vp, i64, vp, i64,
                                        vp, vp, vp, vp, vp]
    L.bitsmoe_moe_decode_topk.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i32, vp, i64, vp,
                                          i64, i64, vp, vp, vp, vp]
    L.bitsmoe_moe_decode_topk_noalloc.argtypes = L.bitsmoe_moe_decode_topk.argtypes
    L.bitsmoe_route.argtypes = [vp, i32, i64, i64, i64, i64, vp, i32] + [vp] * 9
    L.bitsmoe_route_ws.argtypes = [vp, i32, i64, i64, i64, i64, vp, i32] + [vp] * 9 + [i64, vp]
    L.bitsmoe_route_workspace.argtypes = [i64, i64]
    L.bitsmoe_route_grad.argtypes = [vp, i32, i64, i64, i64, i64, i32] + [vp] * 8
    L.bitsmoe_mx4_quantize.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp]
    L.bitsmoe_mx4_dequantize.argtypes = [vp, vp, i64, i64, vp, i32, vp]
    L.bitsmoe_mx4_product.argtypes = [vp, vp, i64, i64, i64, vp, i32, i64, i64, vp, vp, i64, i32,
                                      vp, i32, i64, vp]
    L.bitsmoe_mx4_product_q.argtypes = [vp, vp, i64, i64, i64, vp, vp, i64, vp, vp, i64, i32, vp,
                                        i32, i64, vp]
    L.bitsmoe_mx4_product_grad.argtypes = [vp, vp, i64, i64, i64, vp, i32, i64, vp, i64, vp, i32,
                                           i64, vp]
    L.bitsmoe_combine.argtypes = [vp, i32, i64, vp, vp, i64, i64, i64, vp, vp]
    L.bitsmoe_combine_grad.argtypes = [vp, i32, i64, vp, vp, vp, i64, i64, i64, vp, vp, vp]
    L.bitsmoe_combine_grad_all.argtypes = [vp, i32, i64, vp, vp, vp, i64, i64, i64, vp, vp, vp, vp]
    L.bitsmoe_set_lapack.argtypes = [ctypes.c_char_p]
    L.bitsmoe_timing.argtypes = [i32]
    L.bitsmoe_timing_only.argtypes = [ctypes.c_char_p]
    L.bitsmoe_kernel_time.argtypes = [ctypes.c_char_p, vp, vp]
    L.bitsmoe_last_error.restype = ctypes.c_char_p
    L.bitsmoe_version.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name not in ("bitsmoe_last_error", "bitsmoe_version", "bitsmoe_release", "bitsmoe_route_workspace"):
            getattr(L, name).restype = ctypes.c_int
    L.bitsmoe_release.restype = None
    L.bitsmoe_route_workspace.restype = i64
    lp = _find_lapack()
    if lp and os.environ.get("BITSMOE_LAPACK") is None:
        L.bitsmoe_set_lapack(lp.encode())
    _lib = L
    return L


def _check(st: int, where: str) -> None:
    if st != OK:
        raise BitsmoeError(st, where, lib().bitsmoe_last_error().decode())


# ---------------------------------------------------------------------------
# torch glue (device memory and streams only)
# ---------------------------------------------------------------------------
def _torch():
    import torch
    return torch


def _stream():
    return ctypes.c_void_p(_torch().cuda.current_stream().cuda_stream)


def _dev(t, name: str):
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _dtype_code(t, name: str) -> int:
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"{name} must be bfloat16 or float32")


def _bits_arr(bits: Sequence[int]):
    a = np.ascontiguousarray(np.asarray(bits, dtype=np.int32))
    return a, a.ctypes.data_as(ctypes.c_void_p)


def gram(X, out=None):
    """H = X^T X / n for calibration rows X [n][d] (bf16 or fp32) -> fp32 [d][d]."""
    torch = _torch()
    n, d = X.shape
    if out is None:
        out = torch.empty((d, d), dtype=torch.float32, device=X.device)
    _check(lib().bitsmoe_gram(_dev(X, "X"), _dtype_code(X, "X"), n, d, _dev(out, "H"), _stream()),
           "gram")
    return out


def gram_experts(W, out=None):
    """M = sum_e W_e W_e^T for W [E][d_out][d_in] -> fp64 [d_out][d_out]."""
    torch = _torch()
    E, d_out, d_in = W.shape
    if out is None:
        out = torch.empty((d_out, d_out), dtype=torch.float64, device=W.device)
    _check(lib().bitsmoe_gram_experts(_dev(W, "W"), _dtype_code(W, "W"), E, d_out, d_in,
                                      _dev(out, "M"), _stream()), "gram_experts")
    return out


def shared_basis(M, r: int, out=None) -> Tuple[object, np.ndarray, float]:
    """Top-r eigenvectors of M (host LAPACK). Returns (Ut [r][d_out] fp32, eigvals, host_ms)."""
    torch = _torch()
    d = M.shape[0]
    if M.dtype != torch.float64:
        raise TypeError("M must be float64")
    if out is None:
        out = torch.empty((r, d), dtype=torch.float32, device=M.device)
    ev = np.zeros(r, dtype=np.float64)
    ms = ctypes.c_double(0.0)
    _check(lib().bitsmoe_shared_basis(_dev(M, "M"), d, r, _dev(out, "Ut"),
                                      ev.ctypes.data_as(ctypes.c_void_p), ctypes.byref(ms),
                                      _stream()), "shared_basis")
    return out, ev, ms.value


def shared_basis_gpu(M, r: int, out=None) -> Tuple[object, np.ndarray, float]:
    """Top-r eigenvectors of M, tridiagonal reduction on the device.
    Returns (Ut [r][d_out] fp32, eigvals, wall ms of the call)."""
    torch = _torch()
    d = M.shape[0]
    if M.dtype != torch.float64:
        raise TypeError("M must be float64")
    if out is None:
        out = torch.empty((r, d), dtype=torch.float32, device=M.device)
    ev = np.zeros(r, dtype=np.float64)
    ms = ctypes.c_double(0.0)
    _check(lib().bitsmoe_shared_basis_gpu(_dev(M, "M"), d, r, _dev(out, "Ut"),
                                          ev.ctypes.data_as(ctypes.c_void_p), ctypes.byref(ms),
                                          _stream()), "shared_basis_gpu")
    return out, ev, ms.value


def project(Ut, W, out=None):
    """C_e = U^T W_e -> fp32 [E*r][d_in] (unit u = e*r + k)."""
    torch = _torch()
    r, d_out = Ut.shape
    E, d_out2, d_in = W.shape
    if d_out2 != d_out:
        raise ValueError("Ut and W disagree on d_out")
    if Ut.dtype != torch.float32:
        raise TypeError("Ut must be float32")
    if out is None:
        out = torch.empty((E * r, d_in), dtype=torch.float32, device=W.device)
    _check(lib().bitsmoe_project(_dev(Ut, "Ut"), _dev(W, "W"), _dtype_code(W, "W"), E, d_out, d_in,
                                 r, _dev(out, "C"), _stream()), "project")
    return out


def score(C, H, bits: Sequence[int], group: int, out=None):
    """L[u][j] = delta H delta^T for every unit and width -> fp32 [units][len(bits)]."""
    torch = _torch()
    units, d = C.shape
    if C.dtype != torch.float32 or H.dtype != torch.float32:
        raise TypeError("C and H must be float32")
    if tuple(H.shape) != (d, d):
        raise ValueError("H must be [d][d]")
    b, bp = _bits_arr(bits)
    if out is None:
        out = torch.empty((units, len(b)), dtype=torch.float32, device=C.device)
    _check(lib().bitsmoe_score(_dev(C, "C"), units, d, _dev(H, "H"), bp, len(b), group,
                               _dev(out, "L"), _stream()), "score")
    return out


def gram_experts_in(W, out=None):
    """M_in = sum_e W_e^T W_e for W [E][d_out][d_in] -> fp64 [d_in][d_in] (input-space basis)."""
    torch = _torch()
    E, d_out, d_in = W.shape
    if out is None:
        out = torch.empty((d_in, d_in), dtype=torch.float64, device=W.device)
    _check(lib().bitsmoe_gram_experts_in(_dev(W, "W"), _dtype_code(W, "W"), E, d_out, d_in,
                                         _dev(out, "M_in"), _stream()), "gram_experts_in")
    return out


def project_in(Vt, W, out=None):
    """C_e = Phi_r^T W_e^T -> fp32 [E*r][d_out] (unit u = e*r + k is the column W_e phi_k)."""
    torch = _torch()
    r, d_in = Vt.shape
    E, d_out, d_in2 = W.shape
    if d_in2 != d_in:
        raise ValueError("Vt and W disagree on d_in")
    if Vt.dtype != torch.float32:
        raise TypeError("Vt must be float32")
    if out is None:
        out = torch.empty((E * r, d_out), dtype=torch.float32, device=W.device)
    _check(lib().bitsmoe_project_in(_dev(Vt, "Vt"), _dev(W, "W"), _dtype_code(W, "W"), E, d_out,
                                    d_in, r, _dev(out, "C"), _stream()), "project_in")
    return out


def basis_importance(Vt, H, out=None):
    """beta_k = phi_k^T H phi_k for the rows of Vt -> fp32 [r]."""
    torch = _torch()
    r, d = Vt.shape
    if Vt.dtype != torch.float32 or H.dtype != torch.float32:
        raise TypeError("Vt and H must be float32")
    if tuple(H.shape) != (d, d):
        raise ValueError("H must be [d][d]")
    if out is None:
        out = torch.empty((r,), dtype=torch.float32, device=Vt.device)
    _check(lib().bitsmoe_basis_importance(_dev(Vt, "Vt"), r, d, _dev(H, "H"), _dev(out, "beta"),
                                          _stream()), "basis_importance")
    return out


def score_diag(C, beta, bits: Sequence[int], group: int, out=None):
    """L[u][j] = beta[u % r] ||c_u - Q_{bits[j]}(c_u)||^2 -> fp32 [units][len(bits)]."""
    torch = _torch()
    units, d = C.shape
    if C.dtype != torch.float32 or beta.dtype != torch.float32:
        raise TypeError("C and beta must be float32")
    b, bp = _bits_arr(bits)
    if out is None:
        out = torch.empty((units, len(b)), dtype=torch.float32, device=C.device)
    _check(lib().bitsmoe_score_diag(_dev(C, "C"), units, d, _dev(beta, "beta"), beta.shape[0], bp,
                                    len(b), group, _dev(out, "L"), _stream()), "score_diag")
    return out


def gram_routed(X, offsets, rows, weights, out=None):
    """Per-expert routed Grams H_e = (1/n) sum w x x^T -> fp32 [E][d][d]; the
    routing tables (offsets [E+1], rows [nnz], weights [nnz]) are host arrays."""
    torch = _torch()
    n, d = X.shape
    off = np.ascontiguousarray(np.asarray(offsets, dtype=np.int64))
    rw = np.ascontiguousarray(np.asarray(rows, dtype=np.int32))
    wt = np.ascontiguousarray(np.asarray(weights, dtype=np.float32))
    E = off.shape[0] - 1
    if rw.shape[0] < off[-1] or wt.shape[0] < off[-1]:
        raise ValueError("rows and weights need offsets[-1] entries")
    if out is None:
        out = torch.empty((E, d, d), dtype=torch.float32, device=X.device)
    _check(lib().bitsmoe_gram_routed(_dev(X, "X"), _dtype_code(X, "X"), n, d, E,
                                     off.ctypes.data_as(ctypes.c_void_p),
                                     rw.ctypes.data_as(ctypes.c_void_p),
                                     wt.ctypes.data_as(ctypes.c_void_p), _dev(out, "H"),
                                     _stream()), "gram_routed")
    return out


def score_routed(C, Hs, units_per_h: int, bits: Sequence[int], group: int, out=None):
    """Loss table with one H per block of units_per_h units -> fp32 [units][len(bits)]."""
    torch = _torch()
    units, d = C.shape
    if C.dtype != torch.float32 or Hs.dtype != torch.float32:
        raise TypeError("C and H must be float32")
    if Hs.dim() != 3 or tuple(Hs.shape[1:]) != (d, d) or Hs.shape[0] * units_per_h != units:
        raise ValueError("Hs must be [units / units_per_h][d][d]")
    b, bp = _bits_arr(bits)
    if out is None:
        out = torch.empty((units, len(b)), dtype=torch.float32, device=C.device)
    _check(lib().bitsmoe_score_routed(_dev(C, "C"), units, d, _dev(Hs, "H"), units_per_h, bp, len(b),
                                      group, _dev(out, "L"), _stream()), "score_routed")
    return out


def moe_decode(codes, params, bits_dev, offsets_dev, total_words: int, E: int, r: int, d_in: int,
               group: int, Ut, X, routing, out=None):
    """y = U sum_j g_j C^_e x for every token of X [B][d_in] (fp32) from the packed
    units; routing = (offsets [E+1], tokens, weights) host arrays -> fp32 [B][d_out]."""
    torch = _torch()
    B = X.shape[0]
    d_out = Ut.shape[1]
    if X.dtype != torch.float32 or Ut.dtype != torch.float32:
        raise TypeError("X and Ut must be float32")
    if X.dim() != 2 or X.shape[1] != d_in or Ut.dim() != 2 or Ut.shape[0] != r:
        raise ValueError("X must be [B][d_in] and Ut [r][d_out]")
    off = np.ascontiguousarray(np.asarray(routing[0], dtype=np.int64))
    tok = np.ascontiguousarray(np.asarray(routing[1], dtype=np.int32))
    wt = np.ascontiguousarray(np.asarray(routing[2], dtype=np.float32))
    if off.shape[0] != E + 1 or tok.shape[0] < off[-1] or wt.shape[0] < off[-1]:
        raise ValueError("routing tables do not match E")
    if out is None:
        out = torch.empty((B, d_out), dtype=torch.float32, device=X.device)
    _check(lib().bitsmoe_moe_decode(_dev(codes, "codes"), _dev(params, "params"),
                                    _dev(bits_dev, "bits"), _dev(offsets_dev, "offsets"),
                                    int(total_words), E, r, d_in, group, _dev(Ut, "Ut"), d_out,
                                    _dev(X, "X"), B, off.ctypes.data_as(ctypes.c_void_p),
                                    tok.ctypes.data_as(ctypes.c_void_p),
                                    wt.ctypes.data_as(ctypes.c_void_p), _dev(out, "Y"), _stream()),
           "moe_decode")
    return out


def moe_decode_in(codes, params, bits_dev, offsets_dev, total_words: int, E: int, r: int,
                  d_out: int, group: int, Vt, X, routing, out=None):
    """Input-space (gate/up) decode: y = sum_j g_j C^_e^T (Vt x) for every token
    of X [B][d_in] (fp32); Vt [r][d_in] fp32; units of length d_out ->
    fp32 [B][d_out]."""
    torch = _torch()
    B = X.shape[0]
    if X.dtype != torch.float32 or Vt.dtype != torch.float32:
        raise TypeError("X and Vt must be float32")
    if X.dim() != 2 or Vt.dim() != 2 or Vt.shape[0] != r or Vt.shape[1] != X.shape[1]:
        raise ValueError("Vt must be [r][d_in] and X [B][d_in]")
    off = np.ascontiguousarray(np.asarray(routing[0], dtype=np.int64))
    tok = np.ascontiguousarray(np.asarray(routing[1], dtype=np.int32))
    wt = np.ascontiguousarray(np.asarray(routing[2], dtype=np.float32))
    if off.shape[0] != E + 1 or tok.shape[0] < off[-1] or wt.shape[0] < off[-1]:
        raise ValueError("routing tables do not match E")
    if out is None:
        out = torch.empty((B, d_out), dtype=torch.float32, device=X.device)
    _check(lib().bitsmoe_moe_decode_in(_dev(codes, "codes"), _dev(params, "params"),
                                       _dev(bits_dev, "bits"), _dev(offsets_dev, "offsets"),
                                       int(total_words), E, r, d_out, group, _dev(Vt, "Vt"),
                                       X.shape[1], _dev(X, "X"), B,
                                       off.ctypes.data_as(ctypes.c_void_p),
                                       tok.ctypes.data_as(ctypes.c_void_p),
                                       wt.ctypes.data_as(ctypes.c_void_p), _dev(out, "Y"), _stream()),
           "moe_decode_in")
    return out


def moe_decode_topk(codes, params, bits_dev, offsets_dev, total_words: int, E: int, r: int,
                    d_in: int, group: int, Ut, X, topk_experts, topk_weights, out=None,
                    noalloc: bool = False):
    """moe_decode from the router's device top-k table: topk_experts int32
    [B][k], topk_weights fp32 [B][k] (both on the device) -> fp32 [B][d_out].
    noalloc=True calls bitsmoe_moe_decode_topk_noalloc (no device allocation
    in the library; pass ``out`` to allocate nothing here either)."""
    torch = _torch()
    B = X.shape[0]
    d_out = Ut.shape[1]
    if X.dtype != torch.float32 or Ut.dtype != torch.float32 or topk_weights.dtype != torch.float32:
        raise TypeError("X, Ut and topk_weights must be float32")
    if topk_experts.dtype != torch.int32:
        raise TypeError("topk_experts must be int32")
    if X.dim() != 2 or X.shape[1] != d_in or Ut.dim() != 2 or Ut.shape[0] != r:
        raise ValueError("X must be [B][d_in] and Ut [r][d_out]")
    if topk_experts.dim() != 2 or topk_experts.shape[0] != B or \
            tuple(topk_weights.shape) != tuple(topk_experts.shape):
        raise ValueError("topk_experts and topk_weights must both be [B][k]")
    k = topk_experts.shape[1]
    if out is None:
        out = torch.empty((B, d_out), dtype=torch.float32, device=X.device)
    fn = lib().bitsmoe_moe_decode_topk_noalloc if noalloc else lib().bitsmoe_moe_decode_topk
    _check(fn(_dev(codes, "codes"), _dev(params, "params"), _dev(bits_dev, "bits"),
              _dev(offsets_dev, "offsets"), int(total_words), E, r, d_in, group, _dev(Ut, "Ut"),
              d_out, _dev(X, "X"), B, k, _dev(topk_experts, "topk_experts"),
              _dev(topk_weights, "topk_weights"), _dev(out, "Y"), _stream()),
           "moe_decode_topk_noalloc" if noalloc else "moe_decode_topk")
    return out


def surrogate(C, H, gamma: float, kappa: Sequence[float], out=None, stats=None):
    """The paper's surrogate costs alpha^2 beta^gamma E(b) for the widths
    SURROGATE_WIDTHS -> fp32 [units][8]; ``stats`` (optional, [units][4]) gets
    {alpha^2, beta, rho, cos theta}."""
    torch = _torch()
    units, d = C.shape
    if C.dtype != torch.float32 or H.dtype != torch.float32:
        raise TypeError("C and H must be float32")
    if tuple(H.shape) != (d, d):
        raise ValueError("H must be [d][d]")
    k = np.ascontiguousarray(np.asarray(kappa, dtype=np.float64))
    if k.shape != (3,):
        raise ValueError("kappa holds the coefficients of widths 2, 3, 4")
    if out is None:
        out = torch.empty((units, len(SURROGATE_WIDTHS)), dtype=torch.float32, device=C.device)
    sp = _dev(stats, "stats") if stats is not None else None
    _check(lib().bitsmoe_surrogate(_dev(C, "C"), units, d, _dev(H, "H"), float(gamma),
                                   k.ctypes.data_as(ctypes.c_void_p), _dev(out, "L"), sp,
                                   _stream()), "surrogate")
    return out


def surrogate_budget(E: int, n_out: int, m: int, r: int, b_eq: float) -> int:
    """Equivalent-bit ILP budget of one projection (host)."""
    b = ctypes.c_int64(0)
    _check(lib().bitsmoe_surrogate_budget(E, n_out, m, r, float(b_eq), ctypes.byref(b)),
           "surrogate_budget")
    return b.value


def allocate(L, bits: Sequence[int], budget: int, full_dp_limit: int = -1,
             return_core: bool = False):
    """Exact ILP on the host. L: host array [units][len(bits)] fp32."""
    Lh = np.ascontiguousarray(np.asarray(L, dtype=np.float32))
    units = Lh.shape[0]
    b, bp = _bits_arr(bits)
    out = np.zeros(units, dtype=np.uint8)
    obj = ctypes.c_double(0.0)
    core = ctypes.c_int64(0)
    _check(lib().bitsmoe_allocate_ex(Lh.ctypes.data_as(ctypes.c_void_p), units, bp, len(b),
                                     int(budget), out.ctypes.data_as(ctypes.c_void_p),
                                     ctypes.byref(obj), int(full_dp_limit),
                                     ctypes.byref(core)),
           "allocate")
    if return_core:
        return out, obj.value, core.value
    return out, obj.value


def pack_layout(bits_u, d: int) -> np.ndarray:
    bu = np.ascontiguousarray(np.asarray(bits_u, dtype=np.uint8))
    off = np.zeros(bu.shape[0] + 1, dtype=np.int64)
    _check(lib().bitsmoe_pack_layout(bu.ctypes.data_as(ctypes.c_void_p), bu.shape[0], d,
                                     off.ctypes.data_as(ctypes.c_void_p)), "pack_layout")
    return off


def pack(C, bits_dev, offsets_dev, group: int, total_words: int, codes=None, params=None):
    """Bit-plane codes (uint64 words, as int64 tensor) and fp16 params (as int16 [units][d/G][2])."""
    torch = _torch()
    units, d = C.shape
    if codes is None:
        codes = torch.empty((max(int(total_words), 1),), dtype=torch.int64, device=C.device)
    if params is None:
        params = torch.empty((units, d // group, 2), dtype=torch.int16, device=C.device)
    _check(lib().bitsmoe_pack(_dev(C, "C"), units, d, group, _dev(bits_dev, "bits"),
                              _dev(offsets_dev, "offsets"), int(total_words), _dev(codes, "codes"),
                              _dev(params, "params"), _stream()), "pack")
    return codes, params


def unpack(codes, params, bits_dev, offsets_dev, units: int, d: int, group: int,
           total_words: int, out=None):
    torch = _torch()
    if out is None:
        out = torch.empty((units, d), dtype=torch.float32, device=codes.device)
    _check(lib().bitsmoe_unpack(_dev(codes, "codes"), _dev(params, "params"), _dev(bits_dev, "bits"),
                                _dev(offsets_dev, "offsets"), int(total_words), units, d, group,
                                _dev(out, "Chat"), _stream()), "unpack")
    return out


# ---------------------------------------------------------------------------
# an MoE layer with experts in MX4
# ---------------------------------------------------------------------------
# (These calls are short enough for their marshalling to count: addresses go
# as plain ints, and the stream is asked for by its number.)
def _place(t, name: str):
    """(torch, the stream to run on) for calls whose first tensor is t."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    dev = t.get_device()
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"{name} must be on the current device")
    return torch, torch._C._cuda_getCurrentRawStream(dev)


def _code(t, name: str, torch):
    dt = t.dtype
    if dt is torch.bfloat16:
        return BF16
    if dt is torch.float32:
        return F32
    raise TypeError(f"{name} must be bfloat16 or float32")


def _in(t, name: str, like, dtype, shape=None):
    """Address of a contiguous tensor (None: none) on the device of `like`."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {str(dtype).replace('torch.', '')}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}")
    if t.get_device() != like.get_device():
        raise TypeError(f"{name} must be on the same CUDA (HIP) device")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _rows(t, name: str):
    """(address, row stride) of a matrix whose rows may be apart."""
    if t.is_contiguous():
        return t.data_ptr(), t.shape[-1]
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must have contiguous rows")
    return t.data_ptr(), (t.stride(0) if t.shape[0] > 1 else t.shape[1])


def _out(out, shape, dtype, like, torch):
    """The output tensor, new or given."""
    if out is None:
        return like.new_empty(shape, dtype=dtype)
    _in(out, "out", like, dtype, shape)
    return out


class Routing(NamedTuple):
    """What ``route`` gives for T rows and E experts."""
    experts: object  # int32 [T][k], -1 for a slot without an expert
    weights: object  # fp32 [T][k]
    counts: object   # int32 [E+1]: slots of every expert, then the rows that count
    offsets: object  # int32 [E+1]: where each expert's slots begin in expert order
    rows: object     # int32 [T*k]: the row of each slot in expert order
    slots: object    # int32 [T][k]: the place of each slot in expert order
    lse: object      # fp32 [T]
    losses: object   # fp32 [2]: balance, z


def route(logits, k: int, valid=None, renorm: bool = True) -> Routing:
    """Top-k experts of every row of logits [T][E] (bf16 or fp32), their softmax
    weights, the slots in expert order, and the balance and z losses; rows with
    valid[t] = 0 (bool or uint8) do not count."""
    torch, stream = _place(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be [T][E]")
    T, E = logits.shape
    k = int(k)
    if valid is not None and valid.dtype is torch.bool:
        valid = valid.view(torch.uint8)
    vp = _in(valid, "valid", logits, torch.uint8, (T,))
    lp, ld = _rows(logits, "logits")
    n, w = max(T * k, 0), max(k, 0)
    # one allocation for the whole numbers and one for the others, their parts 16 bytes aligned; after the whole numbers
    # a workspace of the call's own (of many rows an eighth of fp32 logits or less), so that calls may overlap and be
    # captured
    n4, e4, t4 = (n + 3) // 4 * 4, (E + 4) // 4 * 4, (T + 3) // 4 * 4
    L = lib()
    room = L.bitsmoe_route_workspace(T, E) if T > 16 else 0
    ints = logits.new_empty((3 * n4 + 2 * e4 + (room + 3) // 4,), dtype=torch.int32)
    floats = logits.new_empty((n4 + t4 + 4,), dtype=torch.float32)
    ip, fp = ints.data_ptr(), floats.data_ptr()
    ex, co, of, ro, sl = ip, ip + 12 * n4, ip + 12 * n4 + 4 * e4, ip + 4 * n4, ip + 8 * n4
    we, ls, lo = fp, fp + 4 * n4, fp + 4 * (n4 + t4)
    _check(L.bitsmoe_route_ws(lp, _code(logits, "logits", torch), T, E, ld, k, vp, int(renorm), ex, we, co, of,
                              ro, sl, ls, lo, ip + 12 * n4 + 8 * e4 if room else None, room, stream), "route")
    return Routing(ints.as_strided((T, w), (w, 1), 0), floats.as_strided((T, w), (w, 1), 0),
                   ints.as_strided((E + 1,), (1,), 3 * n4), ints.as_strided((E + 1,), (1,), 3 * n4 + e4),
                   ints.as_strided((n,), (1,), n4), ints.as_strided((T, w), (w, 1), 2 * n4),
                   floats.as_strided((T,), (1,), n4), floats.as_strided((2,), (1,), n4 + t4))


def route_grad(logits, routing: Routing, dweights=None, dlosses=None, renorm: bool = True, out=None):
    """Gradient of the logits from those of the weights [T][k] and of the losses
    [2] (fp32, on the device) -> [T][E] of the logits' type."""
    torch, stream = _place(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be [T][E]")
    T, E = logits.shape
    k = routing.experts.shape[1]
    out = _out(out, (T, E), logits.dtype, logits, torch)
    lp, ld = _rows(logits, "logits")
    i32, f32 = torch.int32, torch.float32
    _check(lib().bitsmoe_route_grad(
        lp, _code(logits, "logits", torch), T, E, ld, k, int(renorm),
        _in(routing.experts, "experts", logits, i32, (T, k)),
        _in(routing.weights, "weights", logits, f32, (T, k)),
        _in(routing.counts, "counts", logits, i32, (E + 1,)),
        _in(routing.lse, "lse", logits, f32, (T,)),
        _in(dweights, "dweights", logits, f32, (T, k)),
        _in(dlosses, "dlosses", logits, f32, (2,)), out.data_ptr(), stream), "route_grad")
    return out


def mx4_quantize(X):
    """Rows of X [..][cols] (bf16 or fp32) to MX4: codes uint8 [..][cols/2] and
    scales uint8 [..][cols/32]."""
    torch, stream = _place(X, "X")
    lead, cols = X.shape[:-1], X.shape[-1]
    if cols % 32 != 0 or cols == 0:
        raise ValueError("cols must be a multiple of 32")
    xp, ld = _rows(X, "X")
    codes = X.new_empty((*lead, cols // 2), dtype=torch.uint8)
    scales = X.new_empty((*lead, cols // 32), dtype=torch.uint8)
    _check(lib().bitsmoe_mx4_quantize(xp, _code(X, "X", torch), X.numel() // cols, cols, ld,
                                      codes.data_ptr(), scales.data_ptr(), stream), "mx4_quantize")
    return codes, scales


def _mx4(codes, scales, name: str, like, torch, dims: int = 0):
    """Addresses of MX4 rows."""
    if (dims and codes.dim() != dims) or codes.shape[:-1] != scales.shape[:-1] or \
            codes.shape[-1] != 16 * scales.shape[-1]:
        raise ValueError(f"{name}'s codes must be [..][K/2] and its scales [..][K/32]")
    return (_in(codes, f"{name}'s codes", like, torch.uint8),
            _in(scales, f"{name}'s scales", like, torch.uint8))


def mx4_dequantize(codes, scales, dtype=None, out=None):
    """What MX4 rows stand for -> [..][cols] (bf16 unless ``dtype`` says fp32)."""
    torch, stream = _place(codes, "X's codes")
    cp, sp = _mx4(codes, scales, "X", codes, torch)
    cols = 2 * codes.shape[-1]
    out = _out(out, (*codes.shape[:-1], cols), dtype or torch.bfloat16, codes, torch)
    _check(lib().bitsmoe_mx4_dequantize(cp, sp, codes.numel() * 2 // max(cols, 1), cols, out.data_ptr(),
                                        _code(out, "out", torch), stream), "mx4_dequantize")
    return out


def _experts(codes, scales, offsets, like, torch, glu: bool = False):
    cp, sp = _mx4(codes, scales, "W", like, torch, 3)
    E, N, K = codes.shape[0], codes.shape[1], 2 * codes.shape[2]
    if glu:
        if N % 2:
            raise ValueError("glu takes as many gate as up rows")
        N //= 2
    return cp, sp, E, N, K, _in(offsets, "offsets", like, torch.int32, (E + 1,))


def mx4_product(codes, scales, X, offsets=None, rows=None, glu: bool = False, dtype=None, out=None):
    """y_s = W_e x_{rows[s]} for the slots in expert order (offsets int32 [E+1],
    rows int32 [S]; without rows slot s reads row s): W in MX4 as codes
    [E][N][K/2] and scales [E][N][K/32], X bf16 [rows][K] -> [S][N], bf16 unless
    ``dtype`` says fp32.  glu: W holds gate rows, then up rows, and
    y = silu(gate) * up -> [S][N/2]."""
    torch, stream = _place(X, "X")
    if X.dim() != 2:
        raise ValueError("X must be [rows][K]")
    S = X.shape[0] if rows is None else rows.shape[0]
    cp, sp, E, N, K, op = _experts(codes, scales, offsets, X, torch, glu)
    if X.shape[1] != K:
        raise ValueError("X and W disagree on K")
    xp, ldx = _rows(X, "X")
    out = _out(out, (S, N), dtype or torch.bfloat16, X, torch)
    _check(lib().bitsmoe_mx4_product(cp, sp, E, N, K, xp, _code(X, "X", torch), X.shape[0], ldx, op,
                                     _in(rows, "rows", X, torch.int32, (S,)), S, int(glu),
                                     out.data_ptr(), _code(out, "out", torch), N, stream),
           "mx4_product")
    return out


def mx4_product_q(codes, scales, xcodes, xscales, offsets=None, rows=None, glu: bool = False,
                  dtype=None, out=None):
    """mx4_product with the tokens in MX4 too (``mx4_quantize`` of X)."""
    torch, stream = _place(xcodes, "X's codes")
    xcp, xsp = _mx4(xcodes, xscales, "X", xcodes, torch, 2)
    S = xcodes.shape[0] if rows is None else rows.shape[0]
    cp, sp, E, N, K, op = _experts(codes, scales, offsets, xcodes, torch, glu)
    if 2 * xcodes.shape[1] != K:
        raise ValueError("X and W disagree on K")
    out = _out(out, (S, N), dtype or torch.bfloat16, xcodes, torch)
    _check(lib().bitsmoe_mx4_product_q(cp, sp, E, N, K, xcp, xsp, xcodes.shape[0], op,
                                       _in(rows, "rows", xcodes, torch.int32, (S,)), S, int(glu),
                                       out.data_ptr(), _code(out, "out", torch), N, stream),
           "mx4_product_q")
    return out


def mx4_product_grad(codes, scales, dY, offsets=None, dtype=None, out=None):
    """dx_s = W_e^T dy_s for the slots in expert order: dY bf16 [S][N] ->
    [S][K], bf16 unless ``dtype`` says fp32."""
    torch, stream = _place(dY, "dY")
    if dY.dim() != 2:
        raise ValueError("dY must be [S][N]")
    S = dY.shape[0]
    cp, sp, E, N, K, op = _experts(codes, scales, offsets, dY, torch)
    if dY.shape[1] != N:
        raise ValueError("dY and W disagree on N")
    yp, ldy = _rows(dY, "dY")
    out = _out(out, (S, K), dtype or torch.bfloat16, dY, torch)
    _check(lib().bitsmoe_mx4_product_grad(cp, sp, E, N, K, yp, _code(dY, "dY", torch), ldy, op, S,
                                          out.data_ptr(), _code(out, "out", torch), K, stream),
           "mx4_product_grad")
    return out


def combine(Z, slots, weights=None, out=None):
    """y_t = sum_j weights[t][j] Z[slots[t][j]] (weights None: all 1) for Z [S][d]
    (bf16 or fp32), slots int32 [T][k], weights fp32 [T][k] -> [T][d] of Z's type."""
    torch, stream = _place(Z, "Z")
    if Z.dim() != 2 or slots.dim() != 2:
        raise ValueError("Z must be [S][d] and slots [T][k]")
    (S, d), (T, k) = Z.shape, slots.shape
    out = _out(out, (T, d), Z.dtype, Z, torch)
    _check(lib().bitsmoe_combine(_in(Z, "Z", Z, Z.dtype), _code(Z, "Z", torch), S,
                                 _in(slots, "slots", Z, torch.int32),
                                 _in(weights, "weights", Z, torch.float32, (T, k)), T, k, d,
                                 out.data_ptr(), stream), "combine")
    return out


def combine_grad(Z, slots, weights, dY):
    """Gradients of ``combine``: (dZ [S][d], dweights fp32 [T][k]).  A row of Z that
    no slot names has gradient 0; none may be named twice."""
    torch, stream = _place(Z, "Z")
    if Z.dim() != 2 or slots.dim() != 2:
        raise ValueError("Z must be [S][d] and slots [T][k]")
    (S, d), (T, k) = Z.shape, slots.shape
    zp = _in(Z, "Z", Z, Z.dtype)
    dZ = Z.new_empty((S, d), dtype=Z.dtype)
    dw = Z.new_empty((T, k), dtype=torch.float32)
    work = Z.new_empty((S,), dtype=torch.int32) if T * k > _COMBINE_SCAN else None
    _check(lib().bitsmoe_combine_grad_all(zp, _code(Z, "Z", torch), S, _in(slots, "slots", Z, torch.int32),
                                          _in(weights, "weights", Z, torch.float32, (T, k)),
                                          _in(dY, "dY", Z, Z.dtype, (T, d)), T, k, d, dZ.data_ptr(), dw.data_ptr(),
                                          None if work is None else work.data_ptr(), stream), "combine_grad")
    return dZ, dw


def timing(enable: bool, only: Optional[str] = None) -> None:
    """Records HIP events around every main kernel while enabled (``only``:
    just around the kernels timed under that name)."""
    _check(lib().bitsmoe_timing_only((only or "").encode()), "timing")
    _check(lib().bitsmoe_timing(1 if enable else 0), "timing")


def kernel_time(name: str) -> Tuple[float, int]:
    """(summed ms, launches) of the kernel ``name`` since it was last read."""
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    _check(lib().bitsmoe_kernel_time(name.encode(), ctypes.byref(ms), ctypes.byref(n)), "kernel_time")
    return ms.value, n.value


def release() -> None:
    lib().bitsmoe_release()


def version() -> str:
    return lib().bitsmoe_version().decode()


def last_error() -> str:
    return lib().bitsmoe_last_error().decode()
