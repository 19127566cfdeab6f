"""ctypes binding of libregot.so: argument marshalling only.

Each function has the name of the C entry point it calls (see include/regot.h).
PyTorch is used for device memory and for the current stream; every step of the
computation runs in the HIP kernels.  There is no fallback: if the library is not
built, the first call raises.
"""
import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libregot.so")

SYMBOLS = (
    "regot_status_string",
    "regot_workspace_bytes",
    "regot_plan_geometry",
    "regot_dual_eval",
    "regot_dual_eval_noalloc",
    "regot_sparsify_csr",
    "regot_dual_eval_sparsify",
    "regot_sinkhorn_half_step",
    "regot_sinkhorn_sweeps",
    "regot_topk_workspace_bytes",
    "regot_topk_threshold",
    "regot_pattern_values",
    "regot_pattern_transpose_workspace_bytes",
    "regot_pattern_transpose",
    "regot_hessian_matvec",
    "regot_hessian_workspace_bytes",
    "regot_hessian_lower_csc",
    "regot_dual_metrics",
    "regot_choose_candidate",
    "regot_pcg_workspace_bytes",
    "regot_refresh_candidate_capacity",
    "regot_dual_eval_sparsify_topk",
    "regot_pcg_solve",
    "regot_pcg_solve2",
    "regot_pcg_solve_reduced",
    "regot_pcg_solve2_reduced",
    "regot_splr_direction",
    "regot_row_logprob_workspace_bytes",
    "regot_row_logprob",
    "regot_row_logprob_grad",
    "regot_row_distill_workspace_bytes",
    "regot_row_distill",
    "regot_row_route",
    "regot_row_route_grad",
    "regot_expert_order_workspace_bytes",
    "regot_expert_order",
    "regot_expert_product",
    "regot_expert_weight_grad_workspace_bytes",
    "regot_expert_weight_grad",
    "regot_expert_combine",
    "regot_expert_combine_grad",
    "regot_grad_norm_workspace_bytes",
    "regot_grad_norm",
    "regot_grad_clip",
    "regot_profile_stage1",
    "regot_sweep_patience",
    "regot_stream_read_probe",
    "regot_placement_probe",
)

_lib = None


class RegotError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


def load():
    """Open libregot.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2605_08793_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    i64, dbl, p, sz = ctypes.c_int64, ctypes.c_double, ctypes.c_void_p, ctypes.c_size_t
    lib.regot_status_string.argtypes = [ctypes.c_int]
    lib.regot_status_string.restype = ctypes.c_char_p
    lib.regot_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
    lib.regot_plan_geometry.argtypes = [i64, i64, i64, ctypes.POINTER(i64)]
    lib.regot_dual_eval.argtypes = [i64, i64, p, i64, p, p, p, p, dbl, p, p, p, p, p, p, sz, p]
    lib.regot_dual_eval_noalloc.argtypes = [i64, i64, p, i64, p, p, p, p, dbl, p, p, p, p, p, p]
    lib.regot_sparsify_csr.argtypes = [i64, i64, p, i64, p, p, dbl, dbl, p, p, p, i64, p, p, sz, p]
    lib.regot_dual_eval_sparsify.argtypes = [i64, i64, p, i64, p, p, p, p, dbl, p, p, p, p, p,
                                             dbl, p, p, p, i64, p, p, sz, p]
    lib.regot_sinkhorn_half_step.argtypes = [i64, i64, p, i64, p, p, p, dbl, ctypes.c_int, p, p, sz, p]
    lib.regot_sinkhorn_sweeps.argtypes = [i64, i64, p, i64, p, p, p, p, dbl, ctypes.c_int, p, sz, p]
    lib.regot_topk_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
    lib.regot_topk_threshold.argtypes = [i64, i64, p, i64, p, p, dbl, i64, p, p, p, p, sz, p]
    lib.regot_pattern_values.argtypes = [i64, i64, p, i64, p, p, dbl, p, p, p, i64, p, p, p]
    lib.regot_pattern_transpose_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
    lib.regot_pattern_transpose.argtypes = [i64, i64, i64, p, p, p, p, p, p, sz, p]
    lib.regot_hessian_matvec.argtypes = [i64, i64, dbl, dbl, p, p, p, p, p, p, i64, p, p, p, p, p]
    lib.regot_hessian_workspace_bytes.argtypes = [i64, i64, ctypes.POINTER(sz)]
    lib.regot_hessian_lower_csc.argtypes = [i64, i64, dbl, dbl, p, p, p, i64, p, p, p, p, p, i64, p, ctypes.c_int,
                                            p, sz, p]
    lib.regot_dual_metrics.argtypes = [i64, i64, p, p, p, p, dbl, p, p, p, p, sz, p]
    lib.regot_choose_candidate.argtypes = [i64, i64, p, p, p, p, p, p, p, p, p, p]
    lib.regot_refresh_candidate_capacity.argtypes = [i64, i64, i64, ctypes.POINTER(i64)]
    lib.regot_dual_eval_sparsify_topk.argtypes = [i64, i64, p, i64, p, p, p, p, dbl, i64, p, p, p, p, p, p, p, p, p, i64, p,
                                                  p, sz, p, sz, p]
    lib.regot_pcg_workspace_bytes.argtypes = [i64, i64, ctypes.POINTER(sz)]
    lib.regot_pcg_solve.argtypes = [i64, i64, dbl, dbl, p, p, p, p, p, p, i64, p, p, p, p, dbl, ctypes.c_int, ctypes.c_int,
                                    p, p, sz, p]
    lib.regot_pcg_solve_reduced.argtypes = lib.regot_pcg_solve.argtypes
    lib.regot_pcg_solve2.argtypes = [i64, i64, dbl, dbl, p, p, p, p, p, p, i64, p, p, p, p, p, p, dbl, ctypes.c_int,
                                     ctypes.c_int, p, p, sz, p]
    lib.regot_pcg_solve2_reduced.argtypes = lib.regot_pcg_solve2.argtypes
    lib.regot_splr_direction.argtypes = [i64, i64, p, p, p, p, p, p, p, p, sz, p]
    c_int = ctypes.c_int
    lib.regot_row_logprob_workspace_bytes.argtypes = [i64, i64, c_int, ctypes.POINTER(sz)]
    lib.regot_row_logprob.argtypes = [i64, i64, p, c_int, i64, p, dbl, p, c_int, c_int, p, p, p, p, p, p, sz, p]
    lib.regot_row_logprob_grad.argtypes = [i64, i64, p, c_int, i64, p, dbl, p, c_int, p, p, p, p, p, i64, p]
    lib.regot_row_distill_workspace_bytes.argtypes = [i64, i64, c_int, ctypes.POINTER(sz)]
    lib.regot_row_distill.argtypes = [i64, i64, p, c_int, i64, dbl, p, p, c_int, p, p, p, i64, p, sz, p]
    lib.regot_row_route.argtypes = [i64, i64, p, c_int, i64, p, c_int, c_int, c_int, c_int, c_int, c_int, c_int, dbl, p, p, p]
    lib.regot_row_route_grad.argtypes = [i64, i64, p, c_int, i64, c_int, p, c_int, c_int, dbl, p, p, i64, p]
    lib.regot_expert_order_workspace_bytes.argtypes = [i64, c_int, i64, ctypes.POINTER(sz)]
    lib.regot_expert_order.argtypes = [i64, c_int, i64, p, p, p, p, p, sz, p]
    lib.regot_expert_product.argtypes = [i64, i64, i64, i64, p, p, c_int, i64, i64, p, c_int, p, c_int, i64, i64, c_int, p, i64, p, i64, p]
    lib.regot_expert_weight_grad_workspace_bytes.argtypes = [i64, i64, i64, i64, ctypes.POINTER(sz)]
    lib.regot_expert_weight_grad.argtypes = [i64, i64, i64, i64, p, p, c_int, i64, p, i64, i64, p, c_int, p, c_int, i64, i64, p, sz, p]
    lib.regot_expert_combine.argtypes = [i64, c_int, i64, i64, p, c_int, i64, p, p, p, i64, p]
    lib.regot_expert_combine_grad.argtypes = [i64, c_int, i64, i64, p, c_int, i64, p, i64, p, p, p, i64, p, p]
    lib.regot_grad_norm_workspace_bytes.argtypes = [i64, p, ctypes.POINTER(sz)]
    lib.regot_grad_norm.argtypes = [i64, p, p, p, sz, p]
    lib.regot_grad_clip.argtypes = [i64, p, dbl, p, p, p, sz, p]
    lib.regot_profile_stage1.argtypes = [p, p]
    lib.regot_sweep_patience.argtypes = [ctypes.c_int]
    lib.regot_stream_read_probe.argtypes = [i64, i64, p, i64, p, p, sz, p]
    lib.regot_placement_probe.argtypes = [ctypes.c_int, p, p]
    for name in SYMBOLS[1:]:
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().regot_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise RegotError(status, where)


def _p(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _ws(workspace: torch.Tensor):
    """(pointer, bytes) of a workspace; it has to live on the device, a host pointer would fault in the kernels."""
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous CUDA tensor")
    return ctypes.c_void_p(workspace.data_ptr()), workspace.numel() * workspace.element_size()


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _matrix(M: torch.Tensor):
    if not isinstance(M, torch.Tensor) or not M.is_cuda:
        raise TypeError("M must be a 2-D float64 CUDA tensor")
    return _matrix_layout(M)


def _matrix_layout(M: torch.Tensor):
    """(n, m, ldM) of a row-major float64 matrix, after checking that n rows of m elements at that
    leading dimension lie inside its storage (the kernels read exactly those)."""
    if M.dtype != torch.float64 or M.dim() != 2:
        raise TypeError("M must be a 2-D float64 CUDA tensor")
    n, m = M.shape
    if n > 0 and m > 0 and M.stride(1) != 1:
        raise TypeError("M must be row-major (unit stride along columns)")
    if n > 1 and m > 0 and M.stride(0) < m:
        # an expanded or overlapping view: the kernels would read n dense rows from a storage that
        # need not hold them
        raise TypeError(f"M must have a row stride of at least m = {m} elements (got {M.stride(0)})")
    ld = M.stride(0) if (n > 1 and m > 0) else max(m, 1)
    if n > 0 and m > 0:
        have = M.untyped_storage().nbytes() // M.element_size()
        if M.storage_offset() + (n - 1) * ld + m > have:
            raise TypeError("M reaches beyond its storage")
    return n, m, ld


def _vector(v: Optional[torch.Tensor], length: int, name: str, dtype=torch.float64, optional=False):
    if v is None:
        if optional:
            return None
        raise TypeError(f"{name} is required")
    if v.dtype != dtype or not v.is_cuda or v.dim() != 1 or v.numel() != length or (length > 1 and v.stride(0) != 1):
        raise TypeError(f"{name} must be a contiguous 1-D {dtype} CUDA tensor of length {length}")
    return v


def regot_workspace_bytes(n: int, m: int, csr_capacity: int = -1) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_workspace_bytes(int(n), int(m), int(csr_capacity), ctypes.byref(out)),
           "regot_workspace_bytes")
    return int(out.value)


def regot_plan_geometry(n: int, m: int, csr_capacity: int = -1):
    """(g_r, g_c, rounds, rows of the tallest chunk, strip workgroups) of the dense calls' decomposition."""
    out = (ctypes.c_int64 * 5)()
    _check(load().regot_plan_geometry(int(n), int(m), int(csr_capacity), out), "regot_plan_geometry")
    return tuple(int(x) for x in out)


def new_workspace(n: int, m: int, csr_capacity: int = -1, device="cuda") -> torch.Tensor:
    """A device buffer of the size regot_workspace_bytes() asks for (torch allocations are 256-byte aligned)."""
    return torch.empty(max(regot_workspace_bytes(n, m, csr_capacity), 256), dtype=torch.uint8, device=device)


def regot_dual_eval(M, a, b, alpha, beta, eta, obj, grad_alpha, grad_beta, row_sum=None, col_sum=None, *,
                    workspace, stream=None) -> None:
    n, m, ld = _matrix(M)
    _check(load().regot_dual_eval(
        n, m, _p(M), ld, _p(_vector(a, n, "a")), _p(_vector(b, m, "b")),
        _p(_vector(alpha, n, "alpha")), _p(_vector(beta, m, "beta")), float(eta),
        _p(_vector(obj, 1, "obj")), _p(_vector(grad_alpha, n, "grad_alpha")), _p(_vector(grad_beta, m, "grad_beta")),
        _p(_vector(row_sum, n, "row_sum", optional=True)), _p(_vector(col_sum, m, "col_sum", optional=True)),
        *_ws(workspace), _stream(stream)), "regot_dual_eval")


def regot_dual_eval_noalloc(M, a, b, alpha, beta, eta, obj, grad_alpha, grad_beta, row_sum=None, col_sum=None, *,
                            stream=None) -> None:
    n, m, ld = _matrix(M)
    _check(load().regot_dual_eval_noalloc(
        n, m, _p(M), ld, _p(_vector(a, n, "a")), _p(_vector(b, m, "b")),
        _p(_vector(alpha, n, "alpha")), _p(_vector(beta, m, "beta")), float(eta),
        _p(_vector(obj, 1, "obj")), _p(_vector(grad_alpha, n, "grad_alpha")), _p(_vector(grad_beta, m, "grad_beta")),
        _p(_vector(row_sum, n, "row_sum", optional=True)), _p(_vector(col_sum, m, "col_sum", optional=True)),
        _stream(stream)), "regot_dual_eval_noalloc")


def regot_sparsify_csr(M, alpha, beta, eta, delta, row_ptr, col_idx, val, info, *, workspace, stream=None) -> None:
    n, m, ld = _matrix(M)
    capacity = int(col_idx.numel())
    _vector(val, capacity, "val")
    _vector(col_idx, capacity, "col_idx", torch.int32)
    _check(load().regot_sparsify_csr(
        n, m, _p(M), ld, _p(_vector(alpha, n, "alpha")), _p(_vector(beta, m, "beta")), float(eta), float(delta),
        _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)), _p(col_idx), _p(val), capacity,
        _p(_vector(info, 2, "info", torch.int64)),
        *_ws(workspace), _stream(stream)), "regot_sparsify_csr")


def regot_dual_eval_sparsify(M, a, b, alpha, beta, eta, obj, grad_alpha, grad_beta, row_sum, col_sum,
                             delta, row_ptr, col_idx, val, info, *, workspace, stream=None) -> None:
    n, m, ld = _matrix(M)
    capacity = int(col_idx.numel())
    _vector(val, capacity, "val")
    _vector(col_idx, capacity, "col_idx", torch.int32)
    _check(load().regot_dual_eval_sparsify(
        n, m, _p(M), ld, _p(_vector(a, n, "a")), _p(_vector(b, m, "b")),
        _p(_vector(alpha, n, "alpha")), _p(_vector(beta, m, "beta")), float(eta),
        _p(_vector(obj, 1, "obj")), _p(_vector(grad_alpha, n, "grad_alpha")), _p(_vector(grad_beta, m, "grad_beta")),
        _p(_vector(row_sum, n, "row_sum", optional=True)), _p(_vector(col_sum, m, "col_sum", optional=True)),
        float(delta), _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)), _p(col_idx), _p(val), capacity,
        _p(_vector(info, 2, "info", torch.int64)),
        *_ws(workspace), _stream(stream)), "regot_dual_eval_sparsify")


def regot_refresh_candidate_capacity(n: int, m: int, k: int) -> int:
    out = ctypes.c_int64(0)
    _check(load().regot_refresh_candidate_capacity(int(n), int(m), int(k), ctypes.byref(out)),
           "regot_refresh_candidate_capacity")
    return int(out.value)


def regot_dual_eval_sparsify_topk(M, a, b, alpha, beta, eta, k, obj, grad_alpha, grad_beta, row_sum, col_sum, delta,
                                  row_ptr, col_idx, val, info, *, workspace, topk_workspace, stream=None) -> None:
    n, m, ld = _matrix(M)
    capacity = int(col_idx.numel())
    _vector(val, capacity, "val")
    _vector(col_idx, capacity, "col_idx", torch.int32)
    _check(load().regot_dual_eval_sparsify_topk(
        n, m, _p(M), ld, _p(_vector(a, n, "a")), _p(_vector(b, m, "b")),
        _p(_vector(alpha, n, "alpha")), _p(_vector(beta, m, "beta")), float(eta), int(k),
        _p(_vector(obj, 1, "obj")), _p(_vector(grad_alpha, n, "grad_alpha")), _p(_vector(grad_beta, m, "grad_beta")),
        _p(_vector(row_sum, n, "row_sum", optional=True)), _p(_vector(col_sum, m, "col_sum", optional=True)),
        _p(_vector(delta, 1, "delta")), _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)), _p(col_idx), _p(val),
        capacity, _p(_vector(info, 2, "info", torch.int64)), *_ws(workspace), *_ws(topk_workspace), _stream(stream)),
        "regot_dual_eval_sparsify_topk")


def regot_sinkhorn_half_step(M, marginal, alpha, beta, eta, which, out, *, workspace, stream=None) -> None:
    n, m, ld = _matrix(M)
    length = n if which == 0 else m
    _check(load().regot_sinkhorn_half_step(
        n, m, _p(M), ld, _p(_vector(marginal, length, "marginal")),
        _p(_vector(alpha, n, "alpha", optional=(which == 0))), _p(_vector(beta, m, "beta", optional=(which == 1))),
        float(eta), int(which), _p(_vector(out, length, "out")),
        *_ws(workspace), _stream(stream)), "regot_sinkhorn_half_step")


def regot_sinkhorn_sweeps(M, a, b, alpha, beta, eta, sweeps, *, workspace, stream=None) -> None:
    n, m, ld = _matrix(M)
    _check(load().regot_sinkhorn_sweeps(
        n, m, _p(M), ld, _p(_vector(a, n, "a")), _p(_vector(b, m, "b")), _p(_vector(alpha, n, "alpha")),
        _p(_vector(beta, m, "beta")), float(eta), int(sweeps), *_ws(workspace), _stream(stream)), "regot_sinkhorn_sweeps")


def regot_topk_workspace_bytes(n: int, m: int, k: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_topk_workspace_bytes(int(n), int(m), int(k), ctypes.byref(out)),
           "regot_topk_workspace_bytes")
    return int(out.value)


def new_topk_workspace(n: int, m: int, k: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(regot_topk_workspace_bytes(n, m, k), 256), dtype=torch.uint8, device=device)


def regot_topk_threshold(M, alpha, beta, eta, k, delta, s_k, info, *, workspace, stream=None) -> None:
    n, m, ld = _matrix(M)
    _check(load().regot_topk_threshold(
        n, m, _p(M), ld, _p(_vector(alpha, n, "alpha")), _p(_vector(beta, m, "beta")), float(eta), int(k),
        _p(_vector(delta, 1, "delta")), _p(_vector(s_k, 1, "s_k", optional=True)),
        _p(_vector(info, 2, "info", torch.int64)),
        *_ws(workspace), _stream(stream)), "regot_topk_threshold")


def _entries(t, name, dtype, capacity, optional=False):
    """An entry array of a pattern: 1-D, contiguous, at least `capacity` long."""
    if t is None:
        if optional:
            return None
        raise TypeError(f"{name} is required")
    if t.dtype != dtype or not t.is_cuda or t.dim() != 1 or t.numel() < capacity or (t.numel() > 1 and t.stride(0) != 1):
        raise TypeError(f"{name} must be a contiguous 1-D {dtype} CUDA tensor with at least {capacity} entries")
    return t


def regot_pattern_values(M, alpha, beta, eta, row_ptr, col_idx, csc_pos, val, val_csc, *, stream=None) -> None:
    n, m, ld = _matrix(M)
    capacity = int(col_idx.numel())
    _check(load().regot_pattern_values(
        n, m, _p(M), ld, _p(_vector(alpha, n, "alpha")), _p(_vector(beta, m, "beta")), float(eta),
        _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)), _p(_entries(col_idx, "col_idx", torch.int32, capacity)),
        _p(_entries(csc_pos, "csc_pos", torch.int64, capacity, optional=True)), capacity,
        _p(_entries(val, "val", torch.float64, capacity)),
        _p(_entries(val_csc, "val_csc", torch.float64, capacity, optional=True)), _stream(stream)),
        "regot_pattern_values")


def regot_pattern_transpose_workspace_bytes(n: int, m: int, nnz: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_pattern_transpose_workspace_bytes(int(n), int(m), int(nnz), ctypes.byref(out)),
           "regot_pattern_transpose_workspace_bytes")
    return int(out.value)


def regot_pattern_transpose(n, m, nnz, row_ptr, col_idx, col_ptr, row_idx, csc_pos, *, workspace, stream=None) -> None:
    nnz = int(nnz)
    _check(load().regot_pattern_transpose(
        int(n), int(m), nnz, _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)),
        _p(_entries(col_idx, "col_idx", torch.int32, nnz)), _p(_vector(col_ptr, m + 1, "col_ptr", torch.int64)),
        _p(_entries(row_idx, "row_idx", torch.int32, nnz)), _p(_entries(csc_pos, "csc_pos", torch.int64, nnz)),
        *_ws(workspace), _stream(stream)), "regot_pattern_transpose")


def regot_hessian_matvec(n, m, eta, tau, row_ptr, col_idx, val, col_ptr, row_idx, val_csc, row_sum, col_sum, x, y, *,
                         stream=None) -> None:
    capacity = int(col_idx.numel())
    _check(load().regot_hessian_matvec(
        int(n), int(m), float(eta), float(tau), _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)),
        _p(_entries(col_idx, "col_idx", torch.int32, capacity)), _p(_entries(val, "val", torch.float64, capacity)),
        _p(_vector(col_ptr, m + 1, "col_ptr", torch.int64)), _p(_entries(row_idx, "row_idx", torch.int32, capacity)),
        _p(_entries(val_csc, "val_csc", torch.float64, capacity)), capacity,
        _p(_vector(row_sum, n, "row_sum")), _p(_vector(col_sum, m, "col_sum")),
        _p(_vector(x, n + m - 1, "x")), _p(_vector(y, n + m - 1, "y")), _stream(stream)), "regot_hessian_matvec")


def regot_hessian_workspace_bytes(n: int, m: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_hessian_workspace_bytes(int(n), int(m), ctypes.byref(out)), "regot_hessian_workspace_bytes")
    return int(out.value)


def regot_hessian_lower_csc(n, m, eta, tau, row_ptr, col_idx, val, row_sum, col_sum, h_col_ptr, h_row_idx, h_val, info,
                            values_only=False, *, workspace, stream=None) -> None:
    capacity = int(col_idx.numel())
    h_capacity = int(h_row_idx.numel())
    _check(load().regot_hessian_lower_csc(
        int(n), int(m), float(eta), float(tau), _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)),
        _p(_entries(col_idx, "col_idx", torch.int32, capacity)), _p(_entries(val, "val", torch.float64, capacity)),
        capacity, _p(_vector(row_sum, n, "row_sum")), _p(_vector(col_sum, m, "col_sum")),
        _p(_vector(h_col_ptr, n + m, "h_col_ptr", torch.int64)),
        _p(_entries(h_row_idx, "h_row_idx", torch.int32, h_capacity)),
        _p(_entries(h_val, "h_val", torch.float64, h_capacity)), h_capacity,
        _p(_vector(info, 2, "info", torch.int64)), 1 if values_only else 0,
        *_ws(workspace), _stream(stream)), "regot_hessian_lower_csc")


def regot_dual_metrics(a, b, alpha, beta, eta, row_sum, col_sum, metrics, *, workspace, stream=None) -> None:
    n, m = int(a.numel()), int(b.numel())
    _check(load().regot_dual_metrics(
        n, m, _p(_vector(a, n, "a")), _p(_vector(b, m, "b")), _p(_vector(alpha, n, "alpha")),
        _p(_vector(beta, m, "beta")), float(eta), _p(_vector(row_sum, n, "row_sum")), _p(_vector(col_sum, m, "col_sum")),
        _p(_vector(metrics, 4, "metrics")), *_ws(workspace),
        _stream(stream)), "regot_dual_metrics")


def regot_choose_candidate(obj_q, obj_s, alpha_q, beta_q, alpha_s, beta_s, alpha_out, beta_out, choice, *,
                           stream=None) -> None:
    n, m = int(alpha_q.numel()), int(beta_q.numel())
    _check(load().regot_choose_candidate(
        n, m, _p(_vector(obj_q, 1, "obj_q")), _p(_vector(obj_s, 1, "obj_s")),
        _p(_vector(alpha_q, n, "alpha_q")), _p(_vector(beta_q, m, "beta_q")),
        _p(_vector(alpha_s, n, "alpha_s")), _p(_vector(beta_s, m, "beta_s")),
        _p(_vector(alpha_out, n, "alpha_out")), _p(_vector(beta_out, m, "beta_out")),
        _p(_vector(choice, 1, "choice", torch.int64)), _stream(stream)), "regot_choose_candidate")


def regot_pcg_workspace_bytes(n: int, m: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_pcg_workspace_bytes(int(n), int(m), ctypes.byref(out)), "regot_pcg_workspace_bytes")
    return int(out.value)


def regot_pcg_solve(n, m, eta, tau, row_ptr, col_idx, val, col_ptr, row_idx, val_csc, row_sum, col_sum, rhs, x, rtol,
                    iterations, restart, info, *, workspace, stream=None) -> None:
    capacity = int(col_idx.numel())
    N = n + m - 1
    _check(load().regot_pcg_solve(
        int(n), int(m), float(eta), float(tau), _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)),
        _p(_entries(col_idx, "col_idx", torch.int32, capacity)), _p(_entries(val, "val", torch.float64, capacity)),
        _p(_vector(col_ptr, m + 1, "col_ptr", torch.int64)), _p(_entries(row_idx, "row_idx", torch.int32, capacity)),
        _p(_entries(val_csc, "val_csc", torch.float64, capacity)), capacity,
        _p(_vector(row_sum, n, "row_sum")), _p(_vector(col_sum, m, "col_sum")),
        _p(_vector(rhs, N, "rhs")), _p(_vector(x, N, "x")), float(rtol), int(iterations), 1 if restart else 0,
        _p(_vector(info, 4, "info")), *_ws(workspace), _stream(stream)),
        "regot_pcg_solve")


def regot_pcg_solve_reduced(n, m, eta, tau, row_ptr, col_idx, val, col_ptr, row_idx, val_csc, row_sum, col_sum, rhs, x,
                            rtol, iterations, restart, info, *, workspace, stream=None) -> None:
    capacity = int(col_idx.numel())
    N = n + m - 1
    _check(load().regot_pcg_solve_reduced(
        int(n), int(m), float(eta), float(tau), _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)),
        _p(_entries(col_idx, "col_idx", torch.int32, capacity)), _p(_entries(val, "val", torch.float64, capacity)),
        _p(_vector(col_ptr, m + 1, "col_ptr", torch.int64)), _p(_entries(row_idx, "row_idx", torch.int32, capacity)),
        _p(_entries(val_csc, "val_csc", torch.float64, capacity)), capacity,
        _p(_vector(row_sum, n, "row_sum")), _p(_vector(col_sum, m, "col_sum")),
        _p(_vector(rhs, N, "rhs")), _p(_vector(x, N, "x")), float(rtol), int(iterations), 1 if restart else 0,
        _p(_vector(info, 4, "info")), *_ws(workspace), _stream(stream)),
        "regot_pcg_solve_reduced")


def regot_pcg_solve2(n, m, eta, tau, row_ptr, col_idx, val, col_ptr, row_idx, val_csc, row_sum, col_sum, rhs_a, rhs_b,
                     x_a, x_b, rtol, iterations, restart, info, *, workspace, stream=None) -> None:
    capacity = int(col_idx.numel())
    N = n + m - 1
    _check(load().regot_pcg_solve2(
        int(n), int(m), float(eta), float(tau), _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)),
        _p(_entries(col_idx, "col_idx", torch.int32, capacity)), _p(_entries(val, "val", torch.float64, capacity)),
        _p(_vector(col_ptr, m + 1, "col_ptr", torch.int64)), _p(_entries(row_idx, "row_idx", torch.int32, capacity)),
        _p(_entries(val_csc, "val_csc", torch.float64, capacity)), capacity,
        _p(_vector(row_sum, n, "row_sum")), _p(_vector(col_sum, m, "col_sum")),
        _p(_vector(rhs_a, N, "rhs_a")), _p(_vector(rhs_b, N, "rhs_b")), _p(_vector(x_a, N, "x_a")),
        _p(_vector(x_b, N, "x_b")), float(rtol), int(iterations), 1 if restart else 0,
        _p(_vector(info, 8, "info")), *_ws(workspace), _stream(stream)),
        "regot_pcg_solve2")


def regot_pcg_solve2_reduced(n, m, eta, tau, row_ptr, col_idx, val, col_ptr, row_idx, val_csc, row_sum, col_sum, rhs_a,
                             rhs_b, x_a, x_b, rtol, iterations, restart, info, *, workspace, stream=None) -> None:
    capacity = int(col_idx.numel())
    N = n + m - 1
    _check(load().regot_pcg_solve2_reduced(
        int(n), int(m), float(eta), float(tau), _p(_vector(row_ptr, n + 1, "row_ptr", torch.int64)),
        _p(_entries(col_idx, "col_idx", torch.int32, capacity)), _p(_entries(val, "val", torch.float64, capacity)),
        _p(_vector(col_ptr, m + 1, "col_ptr", torch.int64)), _p(_entries(row_idx, "row_idx", torch.int32, capacity)),
        _p(_entries(val_csc, "val_csc", torch.float64, capacity)), capacity,
        _p(_vector(row_sum, n, "row_sum")), _p(_vector(col_sum, m, "col_sum")),
        _p(_vector(rhs_a, N, "rhs_a")), _p(_vector(rhs_b, N, "rhs_b")), _p(_vector(x_a, N, "x_a")),
        _p(_vector(x_b, N, "x_b")), float(rtol), int(iterations), 1 if restart else 0,
        _p(_vector(info, 8, "info")), *_ws(workspace), _stream(stream)),
        "regot_pcg_solve2_reduced")


def regot_splr_direction(n, m, p, q, s_prev, y_prev, v, d, info, *, workspace, stream=None) -> None:
    N = n + m - 1
    _check(load().regot_splr_direction(
        int(n), int(m), _p(_vector(p, N, "p")), _p(_vector(q, N, "q", optional=True)),
        _p(_vector(s_prev, N, "s_prev", optional=True)), _p(_vector(y_prev, N, "y_prev", optional=True)),
        _p(_vector(v, N, "v", optional=True)), _p(_vector(d, N, "d")), _p(_vector(info, 2, "info")),
        *_ws(workspace), _stream(stream)), "regot_splr_direction")


# ---- rows of scores (fp32, bf16 or fp16) -----------------------------------------------------------------------------

SCORE_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
SCORE_KINDS = {"softmax": 0, "sigmoid": 1}
BIAS_ON = {None: 0, "score": 0, "logit": 1}
GROUP_BY = {"max": 0, "top2": 1}


def _scores(S: torch.Tensor, name="S"):
    """(n, m, type, ldS, address) of a matrix of scores.  Its rows may lie apart (a view of some of a wider matrix's columns),
    but its columns may not, and rows may not share memory."""
    if not isinstance(S, torch.Tensor) or not S.is_cuda or S.dim() != 2 or S.dtype not in SCORE_TYPES:
        raise TypeError(f"{name} must be a 2-D float32, bfloat16 or float16 CUDA tensor")
    n, m = S.shape
    ld, unit = S.stride()
    if n <= 1 or m == 0:
        ld = max(m, 1)
    if (m > 1 and unit != 1) or ld < m:
        raise TypeError(f"{name} must be row-major (unit stride along columns, a row stride of at least m = {m})")
    return n, m, SCORE_TYPES[S.dtype], ld, S.data_ptr()


def _list(v: Optional[torch.Tensor], n: int, width: int, name: str, dtype=torch.float32, optional=False):
    """The address of n rows of `width` numbers without gaps, 1-D or 2-D; 0 for None."""
    if v is None:
        if optional:
            return 0
        raise TypeError(f"{name} is required")
    if not isinstance(v, torch.Tensor) or v.dtype != dtype or not v.is_cuda or v.numel() != n * width or not v.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} CUDA tensor of {n} x {width} elements")
    return v.data_ptr()


def _width(v: Optional[torch.Tensor], n: int, name: str) -> int:
    """Entries per row of an n-row list given as (n, width) or, for one a row, (n,)."""
    if v is None:
        return 0
    if v.dim() not in (1, 2) or v.shape[0] != n:
        raise TypeError(f"{name} must have {n} rows")
    return 1 if v.dim() == 1 else v.shape[1]


def _same_scores(dS: torch.Tensor, S: torch.Tensor, name="dS"):
    """(leading dimension, address) of an output of S's shape and type."""
    if not isinstance(dS, torch.Tensor) or dS.dtype != S.dtype or dS.shape != S.shape:
        raise TypeError(f"{name} must have the shape and type of S")
    return _scores(dS, name)[3:]


def _row_stream(S: torch.Tensor, stream):
    """The stream of a call on S: the given one, or the current one of S's device, which has to be the current device.  (The raw
    handle: the object that torch.cuda.current_stream makes costs 2.7 us, as much as a small call's launch.)"""
    if stream is not None:
        return _stream(stream)
    device = S.get_device()
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"S is on device {device}, which is not the current one")
    return torch._C._cuda_getCurrentRawStream(device)


def regot_row_logprob_workspace_bytes(n: int, m: int, k: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_row_logprob_workspace_bytes(int(n), int(m), int(k), ctypes.byref(out)), "regot_row_logprob_workspace_bytes")
    return int(out.value)


def regot_row_distill_workspace_bytes(n: int, m: int, k: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_row_distill_workspace_bytes(int(n), int(m), int(k), ctypes.byref(out)), "regot_row_distill_workspace_bytes")
    return int(out.value)


def regot_row_logprob(S, target, eta, logprob, entropy, stats, top_idx, top_logprob, *, bias=None, workspace, stream=None) -> None:
    """target, logprob: (n, targets) or None; entropy (n), stats (n, 2): or None; top_idx, top_logprob: (n, k) or None."""
    n, m, kind, ld, at = _scores(S)
    targets, k = _width(target, n, "target"), _width(top_idx, n, "top_idx")
    _check(load().regot_row_logprob(
        n, m, at, kind, ld, _list(bias, 1, m, "bias", optional=True), float(eta),
        _list(target, n, targets, "target", torch.int32, optional=True), targets, k,
        _list(logprob, n, targets, "logprob", optional=targets == 0), _list(entropy, n, 1, "entropy", optional=True),
        _list(stats, n, 2, "stats", optional=True), _list(top_idx, n, k, "top_idx", torch.int32, optional=True),
        _list(top_logprob, n, k, "top_logprob", optional=k == 0), *_ws(workspace), _row_stream(S, stream)), "regot_row_logprob")


def regot_row_logprob_grad(S, target, eta, stats, entropy, g_logprob, g_entropy, dS, *, bias=None, stream=None) -> None:
    """g_logprob (n, targets) with target, or both None; g_entropy (n) with entropy, or both None."""
    n, m, kind, ld, at = _scores(S)
    targets = _width(target, n, "target")
    ldD, to = _same_scores(dS, S)
    _check(load().regot_row_logprob_grad(
        n, m, at, kind, ld, _list(bias, 1, m, "bias", optional=True), float(eta),
        _list(target, n, targets, "target", torch.int32, optional=True), targets, _list(stats, n, 2, "stats"),
        _list(entropy, n, 1, "entropy", optional=g_entropy is None), _list(g_logprob, n, targets, "g_logprob", optional=targets == 0),
        _list(g_entropy, n, 1, "g_entropy", optional=True), to, ldD, _row_stream(S, stream)), "regot_row_logprob_grad")


def regot_row_distill(S, t_idx, t_score, eta, loss, dS=None, *, row_weight=None, workspace, stream=None) -> None:
    """t_idx (int32), t_score: (n, k); dS None: the loss alone."""
    n, m, kind, ld, at = _scores(S)
    k = _width(t_idx, n, "t_idx")
    ldD, to = (m, 0) if dS is None else _same_scores(dS, S)
    _check(load().regot_row_distill(
        n, m, at, kind, ld, float(eta), _list(t_idx, n, k, "t_idx", torch.int32), _list(t_score, n, k, "t_score"), k,
        _list(row_weight, n, 1, "row_weight", optional=True), _list(loss, n, 1, "loss"), to, ldD, *_ws(workspace),
        _row_stream(S, stream)), "regot_row_distill")


def regot_row_route(S, idx, weight, *, bias=None, bias_on="score", score="softmax", groups=1, groups_kept=1, group_by="max",
                    renormalise=True, scale=1.0, stream=None) -> None:
    """idx (int32), weight: (n, k)."""
    n, m, kind, ld, at = _scores(S)
    k = _width(idx, n, "idx")
    _check(load().regot_row_route(
        n, m, at, kind, ld, _list(bias, 1, m, "bias", optional=True), BIAS_ON[bias_on], SCORE_KINDS[score], int(groups),
        int(groups_kept), GROUP_BY[group_by], k, int(bool(renormalise)), float(scale), _list(idx, n, k, "idx", torch.int32),
        _list(weight, n, k, "weight"), _row_stream(S, stream)), "regot_row_route")


def regot_row_route_grad(S, idx, g_weight, dS, *, score="softmax", renormalise=True, scale=1.0, stream=None) -> None:
    n, m, kind, ld, at = _scores(S)
    k = _width(idx, n, "idx")
    ldD, to = _same_scores(dS, S)
    _check(load().regot_row_route_grad(
        n, m, at, kind, ld, SCORE_KINDS[score], _list(idx, n, k, "idx", torch.int32), k, int(bool(renormalise)), float(scale),
        _list(g_weight, n, k, "g_weight"), to, ldD, _row_stream(S, stream)), "regot_row_route_grad")


# ---- what follows a router's choices ---------------------------------------------------------------------------------

ACTS = {None: 0, "gate": 1, "gate_grad": 2}


def _weights(W: torch.Tensor, name="W"):
    """(experts, outputs, inputs, w_by, ldW, strideW, address) of (experts, outputs, inputs) weights, of which either the inputs or
    the outputs are neighbours in memory (W, or W.transpose(1, 2) of one that lies the other way)."""
    if not isinstance(W, torch.Tensor) or not W.is_cuda or W.dim() != 3 or W.dtype not in SCORE_TYPES:
        raise TypeError(f"{name} must be a 3-D float32, bfloat16 or float16 CUDA tensor")
    experts, outputs, inputs = W.shape
    stride, by_output, by_input = W.stride()
    if by_input == 1 or inputs <= 1:
        by, ld, least, single = 0, by_output, inputs, outputs <= 1
    elif by_output == 1 or outputs <= 1:
        by, ld, least, single = 1, by_input, outputs, inputs <= 1
    else:
        raise TypeError(f"{name}: the numbers of an output, or those of an input, must be neighbours")
    if single or W.numel() == 0:
        ld = max(least, 1)
    if ld < least:
        raise TypeError(f"{name} must have a distance of at least {least} between neighbouring rows")
    return experts, outputs, inputs, by, ld, stride, W.data_ptr()


def _one_device(*tensors):
    if len({t.get_device() for t in tensors if isinstance(t, torch.Tensor)}) > 1:
        raise TypeError("the tensors of a call must be on one device")


def regot_expert_order_workspace_bytes(n: int, k: int, experts: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_expert_order_workspace_bytes(int(n), int(k), int(experts), ctypes.byref(out)), "regot_expert_order_workspace_bytes")
    return int(out.value)


def regot_expert_order(idx, start, order, place, *, workspace, stream=None) -> None:
    """idx, place (n, k), order (n * k): int32; start (experts + 1): int64."""
    _one_device(idx, start, order, place, workspace)
    if not isinstance(idx, torch.Tensor) or idx.dim() not in (1, 2):
        raise TypeError("idx must be a 1-D or 2-D int32 CUDA tensor")
    n, k = idx.shape[0], _width(idx, idx.shape[0], "idx")
    experts = start.numel() - 1
    _check(load().regot_expert_order(
        n, k, experts, _list(idx, n, k, "idx", torch.int32), _list(start, experts + 1, 1, "start", torch.int64),
        _list(order, n, k, "order", torch.int32), _list(place, n, k, "place", torch.int32), *_ws(workspace), _row_stream(idx, stream)),
        "regot_expert_order")


def regot_expert_product(X, W, start, Y, *, order=None, k=1, act=None, saved=None, stream=None) -> None:
    """X (x_rows, d), W (experts, m or 2 m, d), Y (rows, m or 2 m), saved (rows, 2 m): one type; order (rows): int32, start: int64."""
    _one_device(X, W, start, Y, order, saved)
    x_rows, d, kind, ldX, at = _scores(X, "X")
    experts, wide, inputs, by, ldW, stride, w_at = _weights(W)
    rows, out, _, ldY, to = _scores(Y, "Y")
    m = wide // 2 if act == "gate" else wide
    if inputs != d or out != (2 * m if act == "gate_grad" else m) or (act == "gate" and wide % 2):
        raise TypeError("W must be (experts, outputs, inputs) of X's inputs and Y's outputs")
    ldS, s_at = 2 * m, 0
    if saved is not None:
        s_rows, s_cols, _, ldS, s_at = _scores(saved, "saved")
        if s_rows != rows or s_cols != 2 * m:
            raise TypeError(f"saved must be {rows} x {2 * m}")
    if any(t is not None and t.dtype != X.dtype for t in (W, Y, saved)):
        raise TypeError("X, W, Y and saved must be of one type")
    _check(load().regot_expert_product(
        rows, m, d, experts, _list(start, experts + 1, 1, "start", torch.int64), at, kind, ldX, x_rows,
        _list(order, rows, 1, "order", torch.int32, optional=True), int(k), w_at, by, ldW, stride, ACTS[act], to, ldY, s_at, ldS,
        _row_stream(X, stream)), "regot_expert_product")


def regot_expert_weight_grad_workspace_bytes(rows: int, m: int, d: int, experts: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_expert_weight_grad_workspace_bytes(int(rows), int(m), int(d), int(experts), ctypes.byref(out)),
           "regot_expert_weight_grad_workspace_bytes")
    return int(out.value)


def regot_expert_weight_grad(dY, X, start, dW, *, order=None, k=1, workspace, stream=None) -> None:
    """dY (rows, m) and X (x_rows, d) of one type, dW (experts, m, d) of that type or float32, the numbers of its last dimension neighbours."""
    _one_device(dY, X, start, dW, order, workspace)
    rows, m, kind, ldY, g_at = _scores(dY, "dY")
    x_rows, d, _, ldX, at = _scores(X, "X")
    experts, outputs, inputs, by, ldW, stride, to = _weights(dW, "dW")
    if (outputs, inputs) != (m, d) or (by != 0 and dW.numel()) or X.dtype != dY.dtype:
        raise TypeError(f"dW must be (experts, {m}, {d}) with rows of neighbours, dY and X of one type")
    _check(load().regot_expert_weight_grad(
        rows, m, d, experts, _list(start, experts + 1, 1, "start", torch.int64), g_at, kind, ldY, at, ldX, x_rows,
        _list(order, rows, 1, "order", torch.int32, optional=True), int(k), to, SCORE_TYPES[dW.dtype], ldW, stride, *_ws(workspace),
        _row_stream(X, stream)), "regot_expert_weight_grad")


def regot_expert_combine(Y, place, weight, out, *, stream=None) -> None:
    """Y (rows, m), out (n, m); place (n, k) int32, weight (n, k) or None."""
    _one_device(Y, place, weight, out)
    rows, m, kind, ldY, at = _scores(Y, "Y")
    n, cols, _, ldO, to = _scores(out, "out")
    if cols != m or out.dtype != Y.dtype:
        raise TypeError("out must have the columns and the type of Y")
    k = _width(place, n, "place")
    _check(load().regot_expert_combine(
        n, k, m, rows, at, kind, ldY, _list(place, n, k, "place", torch.int32), _list(weight, n, k, "weight", optional=True), to, ldO,
        _row_stream(Y, stream)), "regot_expert_combine")


def regot_expert_combine_grad(g_out, Y, place, weight, dY, g_weight=None, *, stream=None) -> None:
    """g_out (n, m), dY (rows, m); Y (rows, m) and g_weight (n, k), or both None."""
    _one_device(g_out, Y, place, weight, dY, g_weight)
    n, m, kind, ldG, g_at = _scores(g_out, "g_out")
    rows, cols, _, ldD, to = _scores(dY, "dY")
    if cols != m or dY.dtype != g_out.dtype:
        raise TypeError("dY must have the columns and the type of g_out")
    ldY, at = (m, 0) if Y is None else _same_scores(Y, dY, "Y")
    k = _width(place, n, "place")
    _check(load().regot_expert_combine_grad(
        n, k, m, rows, g_at, kind, ldG, at, ldY, _list(place, n, k, "place", torch.int32), _list(weight, n, k, "weight", optional=True),
        to, ldD, _list(g_weight, n, k, "g_weight", optional=True), _row_stream(g_out, stream)), "regot_expert_combine_grad")


class _Tensor(ctypes.Structure):
    """regot_tensor"""
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_int64), ("type", ctypes.c_int32)]


def _tensors(tensors, out=None):
    """A host list of tensors without gaps, all on one device, and of what they become (themselves where out is None)."""
    out = tensors if out is None else out
    if len(out) != len(tensors):
        raise TypeError("there must be an output for each tensor")
    made = (_Tensor * max(len(tensors), 1))()
    for i, (t, o) in enumerate(zip(tensors, out)):
        for v in (t, o):
            if not isinstance(v, torch.Tensor) or not v.is_cuda or v.dtype not in SCORE_TYPES or not v.is_contiguous() or v.device != tensors[0].device:
                raise TypeError("tensors must be contiguous float32, bfloat16 or float16 CUDA tensors on one device")
        if o.dtype != t.dtype or o.shape != t.shape:
            raise TypeError("an output must have the shape and type of its tensor")
        made[i] = _Tensor(t.data_ptr(), o.data_ptr(), t.numel(), SCORE_TYPES[t.dtype])
    return made


def _list_stream(tensors, stream):
    return _row_stream(tensors[0], stream) if len(tensors) else _stream(stream)


def regot_grad_norm_workspace_bytes(tensors) -> int:
    out = ctypes.c_size_t(0)
    _check(load().regot_grad_norm_workspace_bytes(len(tensors), _tensors(tensors), ctypes.byref(out)), "regot_grad_norm_workspace_bytes")
    return int(out.value)


def regot_grad_norm(tensors, norm, *, workspace, stream=None) -> None:
    _one_device(*tensors, norm, workspace)
    _check(load().regot_grad_norm(len(tensors), _tensors(tensors), _list(norm, 1, 1, "norm"), *_ws(workspace), _list_stream(tensors, stream)),
           "regot_grad_norm")


def regot_grad_clip(tensors, max_norm, norm, factor, out=None, *, workspace, stream=None) -> None:
    _one_device(*tensors, norm, factor, workspace)
    _check(load().regot_grad_clip(
        len(tensors), _tensors(tensors, out), float(max_norm), _list(norm, 1, 1, "norm"), _list(factor, 1, 1, "factor"), *_ws(workspace),
        _list_stream(tensors, stream)), "regot_grad_clip")


def regot_profile_stage1(start_event, stop_event) -> None:
    """start_event / stop_event: raw hipEvent_t handles (ints) or None; see include/regot.h."""
    _check(load().regot_profile_stage1(ctypes.c_void_p(start_event) if start_event else None,
                                       ctypes.c_void_p(stop_event) if stop_event else None),
           "regot_profile_stage1")


def regot_stream_read_probe(M, total, *, workspace, stream=None) -> None:
    """total[0] = sum of all entries of M, by a pass with the tiling of the dense calls (a bandwidth probe)."""
    n, m, ld = _matrix(M)
    _check(load().regot_stream_read_probe(n, m, _p(M), ld, _p(_vector(total, 1, "total")), *_ws(workspace), _stream(stream)),
           "regot_stream_read_probe")


def regot_placement_probe(ids, *, stream=None) -> None:
    """ids: int32 CUDA tensor [2 * grid]: hardware-id and die-id registers of every workgroup of a grid launched like the fused pass."""
    if ids.dtype != torch.int32 or not ids.is_cuda or ids.dim() != 1 or ids.numel() % 2 or not ids.is_contiguous():
        raise TypeError("ids must be a contiguous 1-D int32 CUDA tensor of even length")
    _check(load().regot_placement_probe(ids.numel() // 2, _p(ids), _stream(stream)), "regot_placement_probe")


def regot_sweep_patience(looks: int) -> None:
    """For tests: how often the next single-read sweeps look for other workgroups' numbers before computing them."""
    _check(load().regot_sweep_patience(int(looks)), "regot_sweep_patience")
