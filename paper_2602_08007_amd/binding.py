"""ctypes binding of include/tsr.h.  Argument marshalling only.

Functions keep the C names.  Tensors are torch CUDA tensors (PyTorch supplies device
memory and the stream, nothing else); sizes and leading dimensions are taken from them.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

import torch

__all__ = [
    "TSR_F32", "TSR_BF16", "TSR_PREC_SPLIT", "TSR_PREC_BF16", "TsrError", "lib", "lib_path",
    "tsr_status_string", "tsr_device_count",
    "tsr_stream_scale", "tsr_project_workspace_bytes", "tsr_project_core", "tsr_project_core_static",
    "TSR_PROJECT_STATIC_SCRATCH_BYTES", "tsr_core_average", "tsr_adam_core", "tsr_sgd_core",
    "tsr_backproject_workspace_bytes", "tsr_backproject_apply",
    "tsr_refresh_workspace_bytes", "tsr_refresh_rsvd", "tsr_refresh_workers_workspace_bytes", "tsr_refresh_rsvd_workers",
    "tsr_realign_workspace_bytes", "tsr_realign_moment",
    "tsr_one_sided_workspace_bytes", "tsr_project_one_sided", "tsr_backproject_one_sided",
    "tsr_refresh_exact_workspace_bytes", "tsr_refresh_exact_svd",
    "tsr_matrix_desc", "tsr_hyper", "Plan", "workspace",
    "TSR_E4M3", "TSR_E5M2", "TSR_STATE_F32", "TSR_STATE_8BIT", "TSR_STATE_BLOCK", "tsr_tensor_desc", "TensorSet",
    "tsr_adamw_batched", "tsr_grad_norm_workspace_bytes", "tsr_grad_norm_batched",
    "tsr_fp8_matrix", "fp8_matrix", "tsr_fp8_quantize", "tsr_fp8_matmul_workspace_bytes", "tsr_fp8_matmul",
]

TSR_F32, TSR_BF16, TSR_E4M3, TSR_E5M2 = 0, 1, 2, 3
TSR_STATE_F32, TSR_STATE_8BIT, TSR_STATE_BLOCK = 0, 1, 256
TSR_PREC_SPLIT, TSR_PREC_BF16 = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
lib_path = os.path.join(_HERE, "libtsr.so")
if not os.path.exists(lib_path):
    # nothing built yet: compile the library in-tree (hipcc, gfx950); there is no other code path
    import importlib.util as _ilu
    _spec = _ilu.spec_from_file_location("_tsr_lib_build", os.path.join(_HERE, "build.py"))
    _mod = _ilu.module_from_spec(_spec)
    try:
        _spec.loader.exec_module(_mod)
        _mod.build()
    except Exception as e:  # noqa: BLE001
        raise ImportError(
            "libtsr.so is not built and building it failed (%s): run `python -c 'import __graft_entry__ as g; g.build()'`; "
            "there is no fallback path" % e)
lib = ctypes.CDLL(lib_path)

_vp, _i, _ll, _f, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float, ctypes.c_size_t


class tsr_matrix_desc(ctypes.Structure):
    _fields_ = [("G", _vp), ("g_dtype", _i), ("m", _i), ("n", _i), ("r", _i), ("ldg", _ll), ("g_stride", _ll),
                ("W", _vp), ("ldw", _ll), ("U", _vp), ("V", _vp), ("M", _vp), ("Vm", _vp), ("C", _vp), ("D", _vp)]


class tsr_hyper(ctypes.Structure):
    _fields_ = [("lr", _f), ("wd", _f), ("beta1", _f), ("beta2", _f), ("eps", _f), ("scale", _f)]


class tsr_tensor_desc(ctypes.Structure):
    _fields_ = [("p", _vp), ("g", _vp), ("m", _vp), ("v", _vp), ("m_scale", _vp), ("v_scale", _vp), ("p16", _vp),
                ("count", _ll), ("p_dtype", _i), ("g_dtype", _i), ("state", _i), ("wd_scale", _f)]


class tsr_fp8_matrix(ctypes.Structure):
    _fields_ = [("q", _vp), ("scale", _vp), ("ld", _ll), ("ld_scale", _ll), ("dtype", _i), ("block_rows", _i)]


def _sig(name, restype, *argtypes):
    fn = getattr(lib, name)
    fn.restype = restype
    fn.argtypes = list(argtypes)
    return fn


_status_string = _sig("tsr_status_string", ctypes.c_char_p, _i)
_last_hip = _sig("tsr_last_hip_error", _i)
_device_count = _sig("tsr_device_count", _i)
_project_ws = _sig("tsr_project_workspace_bytes", _sz, _i, _i, _i)
_project = _sig("tsr_project_core", _i, _vp, _i, _i, _i, _ll, _vp, _vp, _i, _f, _i, _vp, _i, _vp, _sz, _vp)
_project_static = _sig("tsr_project_core_static", _i, _vp, _i, _i, _i, _ll, _vp, _vp, _i, _f, _i, _vp, _i, _vp)
_average = _sig("tsr_core_average", _i, _vp, _i, _i, _vp, _vp)
_stream_scale = _sig("tsr_stream_scale", _i, _vp, _vp, _ll, _f, _vp)
_adam = _sig("tsr_adam_core", _i, _vp, _vp, _vp, _vp, _ll, _i, _f, _f, _f, _vp)
_sgd = _sig("tsr_sgd_core", _i, _vp, _vp, _vp, _ll, _f, _vp)
_lift_ws = _sig("tsr_backproject_workspace_bytes", _sz, _i, _i, _i)
_lift = _sig("tsr_backproject_apply", _i, _vp, _i, _i, _ll, _vp, _vp, _vp, _i, _f, _f, _f, _i, _vp, _sz, _vp)
_refresh_ws = _sig("tsr_refresh_workspace_bytes", _sz, _i, _i, _i, _i)
_refresh = _sig("tsr_refresh_rsvd", _i, _vp, _i, _i, _i, _ll, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp)
_realign_ws = _sig("tsr_realign_workspace_bytes", _sz, _i, _i, _i)
_realign = _sig("tsr_realign_moment", _i, _vp, _vp, _vp, _vp, _i, _i, _i, _vp, _vp, _sz, _vp)
_one_sided_ws = _sig("tsr_one_sided_workspace_bytes", _sz, _i, _i, _i)
_project_one = _sig("tsr_project_one_sided", _i, _vp, _i, _i, _i, _ll, _vp, _i, _f, _i, _vp, _i, _vp, _sz, _vp)
_lift_one = _sig("tsr_backproject_one_sided", _i, _vp, _i, _i, _ll, _vp, _vp, _i, _f, _f, _f, _i, _vp, _sz, _vp)
_exact_ws = _sig("tsr_refresh_exact_workspace_bytes", _sz, _i, _i, _i)
_exact = _sig("tsr_refresh_exact_svd", _i, _vp, _i, _i, _i, _ll, _i, _vp, _vp, _vp, _vp, _sz, _vp)
_refresh_workers_ws = _sig("tsr_refresh_workers_workspace_bytes", _sz, _i, _i, _i, _i, _i)
_refresh_workers = _sig("tsr_refresh_rsvd_workers", _i, _vp, _i, _i, _i, _ll, _ll, _i, _vp, _i, _i, _i, _vp, _vp, _vp, _vp,
                        _sz, _vp)
_plan_ws = _sig("tsr_plan_workspace_bytes", _sz, ctypes.POINTER(tsr_matrix_desc), _i, _i, _i, _i, _i)
_bases_changed = _sig("tsr_plan_bases_changed", _i, _vp)
_kernel_path = _sig("tsr_plan_kernel_path", _i, _vp)
_plan_create = _sig("tsr_plan_create", _i, ctypes.POINTER(tsr_matrix_desc), _i, _i, _i, _i, _i, _vp, _sz, _vp,
                    ctypes.POINTER(_vp))
_plan_destroy = _sig("tsr_plan_destroy", None, _vp)
_step_batched = _sig("tsr_step_batched", _i, _vp, _i, ctypes.POINTER(tsr_hyper), _vp)
_refresh_batched = _sig("tsr_refresh_batched", _i, _vp, ctypes.POINTER(_vp), _i, _vp)
_prof_begin = _sig("tsr_plan_profile_begin", _i, _vp)
_prof_end = _sig("tsr_plan_profile_end", _i, _vp, _vp, ctypes.POINTER(_f), ctypes.POINTER(_i))
_payload = _sig("tsr_plan_payload_bytes", None, _vp, _i, ctypes.POINTER(_ll), ctypes.POINTER(_ll))


_adamw = _sig("tsr_adamw_batched", _i, ctypes.POINTER(tsr_tensor_desc), _i, _i, ctypes.POINTER(tsr_hyper), ctypes.c_ulonglong,
              _vp, _vp)
_norm_ws = _sig("tsr_grad_norm_workspace_bytes", _sz, ctypes.POINTER(tsr_tensor_desc), _i)
_norm = _sig("tsr_grad_norm_batched", _i, ctypes.POINTER(tsr_tensor_desc), _i, _f, _vp, _vp, _vp, _sz, _vp)
_quantize = _sig("tsr_fp8_quantize", _i, _vp, _i, _i, _i, _ll, _i, _i, _vp, _ll, _vp, _ll, _vp, _ll, _vp, _ll, _vp)
_matmul_ws = _sig("tsr_fp8_matmul_workspace_bytes", _sz, _i, _i, _i)
_matmul = _sig("tsr_fp8_matmul", _i, ctypes.POINTER(tsr_fp8_matrix), ctypes.POINTER(tsr_fp8_matrix), _i, _i, _i, _vp, _ll, _vp, _sz, _vp)


class TsrError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        msg = _status_string(status).decode()
        if status == -5:
            msg += " (hipError %d)" % _last_hip()
        super().__init__("tsr: %s" % msg)


def _check(status: int) -> None:
    if status != 0:
        raise TsrError(status)


def tsr_status_string(status: int) -> str:
    return _status_string(status).decode()


def tsr_device_count() -> int:
    return int(_device_count())


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _gdtype(G: torch.Tensor) -> int:
    if G.dtype == torch.float32:
        return TSR_F32
    if G.dtype == torch.bfloat16:
        return TSR_BF16
    raise TypeError("G must be float32 or bfloat16")


def _f32c(*ts):
    for t in ts:
        if t is not None and (t.dtype != torch.float32 or not t.is_contiguous()):
            raise TypeError("expected contiguous float32 tensors")


def _ld(t: torch.Tensor) -> int:
    if t.dim() != 2 or t.stride(1) != 1:
        raise TypeError("expected a row-major 2-D tensor (unit column stride)")
    return t.stride(0)


def workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """A 256-byte aligned device buffer of at least nbytes (torch allocations are 512-byte aligned)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _temp_workspace(nbytes: int, device, stream) -> torch.Tensor:
    """Workspace for a one-shot call that did not bring its own.  It is dropped when the call returns, while the kernels
    may still be queued.  The caching allocator hands a block on in the order of the stream on which it was taken, so it is
    taken on the one that uses it: a block of another stream's could still be in use by what is queued there."""
    if stream is None:
        return workspace(nbytes, device)
    if not isinstance(stream, torch.cuda.Stream):
        raise ValueError("pass a torch.cuda.Stream, or an explicit ws together with a raw stream handle")
    with torch.cuda.stream(stream):
        return workspace(nbytes, device)


def tsr_project_workspace_bytes(m: int, n: int, r: int) -> int:
    return int(_project_ws(m, n, r))


def tsr_project_core(G, U, V, C, alpha=1.0, accumulate=False, precision=TSR_PREC_SPLIT, ws=None, stream=None):
    m, n = G.shape
    r = U.shape[1]
    _f32c(U, V, C)
    if ws is None:
        ws = _temp_workspace(tsr_project_workspace_bytes(m, n, r), G.device, stream)
    _check(_project(_ptr(G), _gdtype(G), m, n, _ld(G), _ptr(U), _ptr(V), r, alpha, int(bool(accumulate)), _ptr(C),
                    precision, _ptr(ws), ws.numel(), _stream(stream)))
    return C


TSR_PROJECT_STATIC_SCRATCH_BYTES = 16 << 20


def tsr_project_core_static(G, U, V, C, alpha=1.0, accumulate=False, precision=TSR_PREC_SPLIT, stream=None):
    """tsr_project_core on the library's built-in scratch: nothing is allocated, here or there."""
    m, n = G.shape
    r = U.shape[1]
    _f32c(U, V, C)
    _check(_project_static(_ptr(G), _gdtype(G), m, n, _ld(G), _ptr(U), _ptr(V), r, alpha, int(bool(accumulate)), _ptr(C),
                           precision, _stream(stream)))
    return C


def tsr_core_average(Cs, Cbar, stream=None):
    _f32c(Cs, Cbar)
    K, r = Cs.shape[0], Cs.shape[1]
    _check(_average(_ptr(Cs), K, r, _ptr(Cbar), _stream(stream)))
    return Cbar


def tsr_stream_scale(dst, src, scale=1.0, stream=None):
    _f32c(dst, src)
    _check(_stream_scale(_ptr(dst), _ptr(src), src.numel(), scale, _stream(stream)))
    return dst


def tsr_adam_core(C, M, Vm, D, t, beta1=0.9, beta2=0.999, eps=1e-8, stream=None):
    _f32c(C, M, Vm, D)
    _check(_adam(_ptr(C), _ptr(M), _ptr(Vm), _ptr(D), C.numel(), t, beta1, beta2, eps, _stream(stream)))
    return D


def tsr_sgd_core(C, M, D, beta=0.9, stream=None):
    _f32c(C, M, D)
    _check(_sgd(_ptr(C), _ptr(M), _ptr(D), C.numel(), beta, _stream(stream)))
    return D


def tsr_backproject_workspace_bytes(m: int, n: int, r: int) -> int:
    return int(_lift_ws(m, n, r))


def tsr_backproject_apply(W, U, V, D, lr, wd=0.0, scale=1.0, precision=TSR_PREC_SPLIT, ws=None, stream=None):
    m, n = W.shape
    r = U.shape[1]
    _f32c(U, V, D)
    if W.dtype != torch.float32:
        raise TypeError("W must be float32")
    if ws is None:
        ws = _temp_workspace(tsr_backproject_workspace_bytes(m, n, r), W.device, stream)
    _check(_lift(_ptr(W), m, n, _ld(W), _ptr(U), _ptr(V), _ptr(D), r, lr, wd, scale, precision, _ptr(ws), ws.numel(),
                 _stream(stream)))
    return W


def tsr_refresh_workspace_bytes(m: int, n: int, r: int, p: int) -> int:
    return int(_refresh_ws(m, n, r, p))


def tsr_refresh_rsvd(G, Omega, r, p, q, U, V, sigma=None, ws=None, stream=None):
    m, n = G.shape
    _f32c(Omega, U, V, sigma)
    if tuple(Omega.shape) != (n, r + p):
        raise ValueError("Omega must be n x (r+p)")
    if ws is None:
        ws = _temp_workspace(tsr_refresh_workspace_bytes(m, n, r, p), G.device, stream)
    _check(_refresh(_ptr(G), _gdtype(G), m, n, _ld(G), _ptr(Omega), r, p, q, _ptr(U), _ptr(V), _ptr(sigma), _ptr(ws),
                    ws.numel(), _stream(stream)))
    return U, V


def tsr_refresh_workers_workspace_bytes(m: int, n: int, r: int, p: int, n_workers: int) -> int:
    return int(_refresh_workers_ws(m, n, r, p, n_workers))


def tsr_refresh_rsvd_workers(G, Omega, r, p, q, U, V, sigma=None, ws=None, stream=None):
    """G: the workers' gradients stacked as [workers, m, n] (contiguous)."""
    if G.dim() != 3 or not G.is_contiguous():
        raise ValueError("G must be a contiguous [workers, m, n] tensor")
    K, m, n = G.shape
    _f32c(Omega, U, V, sigma)
    if tuple(Omega.shape) != (n, r + p):
        raise ValueError("Omega must be n x (r+p)")
    if ws is None:
        ws = _temp_workspace(tsr_refresh_workers_workspace_bytes(m, n, r, p, K), G.device, stream)
    _check(_refresh_workers(_ptr(G), _gdtype(G), m, n, n, m * n, K, _ptr(Omega), r, p, q, _ptr(U), _ptr(V), _ptr(sigma),
                            _ptr(ws), ws.numel(), _stream(stream)))
    return U, V


def tsr_realign_workspace_bytes(m: int, n: int, r: int) -> int:
    return int(_realign_ws(m, n, r))


def tsr_realign_moment(U_old, V_old, U_new, V_new, M, ws=None, stream=None):
    m, r = U_old.shape
    n = V_old.shape[0]
    _f32c(U_old, V_old, U_new, V_new, M)
    if tuple(U_new.shape) != (m, r) or tuple(V_old.shape) != (n, r) or tuple(V_new.shape) != (n, r) or tuple(M.shape) != (r, r):
        raise ValueError("shape mismatch")
    if ws is None:
        ws = _temp_workspace(tsr_realign_workspace_bytes(m, n, r), M.device, stream)
    _check(_realign(_ptr(U_old), _ptr(V_old), _ptr(U_new), _ptr(V_new), m, n, r, _ptr(M), _ptr(ws), ws.numel(),
                    _stream(stream)))
    return M


def tsr_one_sided_workspace_bytes(m: int, n: int, r: int) -> int:
    return int(_one_sided_ws(m, n, r))


def tsr_project_one_sided(G, U, Ct, alpha=1.0, accumulate=False, precision=TSR_PREC_SPLIT, ws=None, stream=None):
    """Ct (n x r) <- alpha G^T U (+ Ct): the one-sided object U^T G, held transposed."""
    m, n = G.shape
    r = U.shape[1]
    _f32c(U, Ct)
    if tuple(Ct.shape) != (n, r):
        raise ValueError("Ct must be n x r")
    if ws is None:
        ws = _temp_workspace(tsr_one_sided_workspace_bytes(m, n, r), G.device, stream)
    _check(_project_one(_ptr(G), _gdtype(G), m, n, _ld(G), _ptr(U), r, alpha, int(bool(accumulate)), _ptr(Ct), precision,
                        _ptr(ws), ws.numel(), _stream(stream)))
    return Ct


def tsr_backproject_one_sided(W, U, Dt, lr, wd=0.0, scale=1.0, precision=TSR_PREC_SPLIT, ws=None, stream=None):
    """W <- W - lr (scale U Dt^T + wd W) with the transposed one-sided update Dt (n x r)."""
    m, n = W.shape
    r = U.shape[1]
    _f32c(U, Dt)
    if W.dtype != torch.float32 or tuple(Dt.shape) != (n, r):
        raise TypeError("W must be float32 and Dt n x r")
    if ws is None:
        ws = _temp_workspace(tsr_one_sided_workspace_bytes(m, n, r), W.device, stream)
    _check(_lift_one(_ptr(W), m, n, _ld(W), _ptr(U), _ptr(Dt), r, lr, wd, scale, precision, _ptr(ws), ws.numel(),
                     _stream(stream)))
    return W


def tsr_refresh_exact_workspace_bytes(m: int, n: int, r: int) -> int:
    return int(_exact_ws(m, n, r))


def tsr_refresh_exact_svd(G, r, U, V, sigma=None, ws=None, stream=None):
    m, n = G.shape
    _f32c(U, V, sigma)
    if ws is None:
        nbytes = tsr_refresh_exact_workspace_bytes(m, n, r)
        if nbytes == 0:
            raise TsrError(-2)
        ws = _temp_workspace(nbytes, G.device, stream)
    _check(_exact(_ptr(G), _gdtype(G), m, n, _ld(G), r, _ptr(U), _ptr(V), _ptr(sigma), _ptr(ws), ws.numel(), _stream(stream)))
    return U, V


class Plan:
    """Batched all-layers plan (tsr_plan_* / tsr_step_batched / tsr_refresh_batched).

    blocks: sequence of dicts with tensors G (n_workers stacked as [workers, m, ld] or a single
    [m, ld] matrix), W, U, V, M, Vm, C, D.  The plan's workspace is a torch buffer owned here."""

    def __init__(self, blocks: Sequence[dict], n_workers=1, precision=TSR_PREC_SPLIT, with_refresh=False, p=0,
                 stream=None):
        self._handle = _vp()
        self.count = len(blocks)
        self.n_workers = n_workers
        self._keep = list(blocks)
        arr = (tsr_matrix_desc * self.count)()
        for d, b in zip(arr, blocks):
            G, W, U = b["G"], b["W"], b["U"]
            g2 = G[0] if G.dim() == 3 else G
            if (G.dim() == 3) != (n_workers > 1) and not (G.dim() == 3 and G.shape[0] == 1):
                raise ValueError("G must be [workers, m, n] when n_workers > 1")
            m, n = W.shape
            _f32c(U, b["V"], b["M"], b["Vm"], b["C"], b["D"])
            d.G = _ptr(G); d.g_dtype = _gdtype(G); d.m = m; d.n = n; d.r = U.shape[1]
            d.ldg = _ld(g2); d.g_stride = G.stride(0) if G.dim() == 3 else 0
            d.W = _ptr(W); d.ldw = _ld(W)
            d.U = _ptr(U); d.V = _ptr(b["V"]); d.M = _ptr(b["M"]); d.Vm = _ptr(b["Vm"]); d.C = _ptr(b["C"]); d.D = _ptr(b["D"])
        self._descs = arr
        nbytes = int(_plan_ws(arr, self.count, n_workers, precision, int(with_refresh), p))
        if nbytes == 0:
            raise TsrError(-2)
        self.ws = workspace(nbytes, blocks[0]["W"].device)
        _check(_plan_create(arr, self.count, n_workers, precision, int(with_refresh), p, _ptr(self.ws), self.ws.numel(),
                            _stream(stream), ctypes.byref(self._handle)))

    def tsr_step_batched(self, t, lr, wd=0.0, beta1=0.9, beta2=0.999, eps=1e-8, scale=1.0, stream=None):
        h = tsr_hyper(lr, wd, beta1, beta2, eps, scale)
        _check(_step_batched(self._handle, t, ctypes.byref(h), _stream(stream)))

    def tsr_plan_kernel_path(self):
        return _kernel_path(self._handle)

    def tsr_plan_bases_changed(self):
        _check(_bases_changed(self._handle))

    def tsr_refresh_batched(self, omegas: List[torch.Tensor], q, stream=None):
        _f32c(*omegas)
        arr = (_vp * self.count)(*[_ptr(o) for o in omegas])
        _check(_refresh_batched(self._handle, arr, q, _stream(stream)))

    PROF_KINDS = ("gv", "utp", "adam", "ud", "tvt", "sketch_gemm", "orth_gemm", "chol", "jacobi", "basis_gemm")

    def tsr_plan_profile_begin(self):
        _check(_prof_begin(self._handle))

    def tsr_plan_profile_end(self, stream=None):
        """{kind: (milliseconds, stages)} summed since tsr_plan_profile_begin; synchronizes."""
        n = len(self.PROF_KINDS)
        ms = (_f * n)()
        cnt = (_i * n)()
        _check(_prof_end(self._handle, _stream(stream), ms, cnt))
        return {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(self.PROF_KINDS)}

    def payload_bytes(self, bytes_per_dense_element=4):
        c, d = _ll(), _ll()
        _payload(self._handle, bytes_per_dense_element, ctypes.byref(c), ctypes.byref(d))
        return int(c.value), int(d.value)

    def close(self):
        if self._handle:
            _plan_destroy(self._handle)
            self._handle = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ------------------------------------------------------------------ parameters that are kept dense
_FP8 = {torch.float8_e4m3fn: TSR_E4M3, torch.float8_e5m2: TSR_E5M2}


def _device_of(*tensors) -> torch.device:
    """The one GPU that all tensors (those that are not None) lie on."""
    first, at = None, -1
    for t in tensors:
        if t is None:
            continue
        if first is None:
            first, at = t, t.get_device()
        elif t.get_device() != at:
            raise ValueError("tensors on different devices: %s and %s" % (first.device, t.device))
    if at < 0:
        raise TypeError("expected GPU tensors")
    return first.device


def _int(n: int) -> int:
    """n for a C int, of which ctypes would take the low 32 bits without a word."""
    if not -0x80000000 <= n <= 0x7fffffff:
        raise OverflowError("%d does not fit 32 bits" % n)
    return n


def _launch(dev: torch.device, stream, fn, *args) -> None:
    """fn(*args, stream) with the tensors' device current; the stream is that device's current one unless given."""
    at = dev.index
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(at)      # current_stream(at).cuda_stream without the object, 0.8 us
    else:
        if isinstance(stream, torch.cuda.Stream) and stream.device != dev:
            raise ValueError("the stream belongs to another device than the tensors")
        handle = _stream(stream)
    if at == torch._C._cuda_getDevice():
        status = fn(*args, handle)
    else:
        with torch.cuda.device(dev):
            status = fn(*args, handle)
    if status:
        raise TsrError(status)


class TensorSet:
    """The tensors of tsr_adamw_batched and tsr_grad_norm_batched, as the array the library takes.

    tensors: sequence of dicts with p, g, m, v (m and v float32, or float8_e4m3fn and float8_e5m2 with m_scale, v_scale
    uint8 of a value for each 256 elements), optionally p16 (bfloat16) and wd_scale (1 by default).  For the norm alone, g
    is enough.  All contiguous, all on one device; the set keeps them alive and describes their storage as it is now.

    Building one takes the host some 2 microseconds a tensor, more than the step of small tensors does: build it once, keep the
    gradients where they are (zero_grad(set_to_none=False)), and build it again when they are allocated anew."""

    def __init__(self, tensors: Sequence[dict]):
        self._keep = [dict(t) for t in tensors]
        self.count = len(self._keep)
        if not self.count:
            raise ValueError("no tensors")
        self.only_g = any("p" not in t for t in self._keep)
        self.descs = (tsr_tensor_desc * self.count)()
        self.device = _device_of(*(x for t in self._keep for x in t.values() if isinstance(x, torch.Tensor)))
        for d, t in zip(self.descs, self._keep):
            g = t["g"]
            for x in t.values():
                if isinstance(x, torch.Tensor) and not x.is_contiguous():
                    raise TypeError("expected contiguous tensors")
            d.g, d.g_dtype, d.count = _ptr(g), _gdtype(g), g.numel()
            d.wd_scale = t.get("wd_scale", 1.0)
            if "p" not in t:
                continue
            p, m, v = t["p"], t["m"], t["v"]
            if p.numel() != d.count or m.numel() != d.count or v.numel() != d.count:
                raise ValueError("p, g, m and v must have as many elements")
            d.p, d.p_dtype, d.m, d.v = _ptr(p), _gdtype(p), _ptr(m), _ptr(v)
            if m.dtype == torch.float32 and v.dtype == torch.float32:
                d.state = TSR_STATE_F32
            elif m.dtype == torch.float8_e4m3fn and v.dtype == torch.float8_e5m2:
                d.state = TSR_STATE_8BIT
                blocks = -(-d.count // TSR_STATE_BLOCK)
                for x in (t["m_scale"], t["v_scale"]):
                    if x.dtype != torch.uint8 or x.numel() < blocks:
                        raise ValueError("m_scale and v_scale must be uint8, a value for each %d elements" % TSR_STATE_BLOCK)
                d.m_scale, d.v_scale = _ptr(t["m_scale"]), _ptr(t["v_scale"])
            else:
                raise TypeError("m and v must be float32, or float8_e4m3fn and float8_e5m2")
            p16 = t.get("p16")
            if p16 is not None:
                if p16.dtype != torch.bfloat16 or p16.numel() != d.count:
                    raise TypeError("p16 must be bfloat16 with as many elements as p")
                d.p16 = _ptr(p16)


def _tensor_set(tensors) -> TensorSet:
    return tensors if isinstance(tensors, TensorSet) else TensorSet(tensors)


def _scalar(t: Optional[torch.Tensor], name: str) -> None:
    if t is not None and (t.dtype != torch.float32 or t.numel() != 1):
        raise TypeError("%s must be one float32 value" % name)


def tsr_adamw_batched(tensors, t, lr, wd=0.0, beta1=0.9, beta2=0.999, eps=1e-8, scale=1.0, g_scale=None, seed=0, stream=None):
    """One AdamW step of all tensors (a TensorSet, or the dicts it is made of)."""
    s = _tensor_set(tensors)
    if s.only_g:
        raise ValueError("every tensor needs p, g, m and v")
    _scalar(g_scale, "g_scale")
    if g_scale is not None and g_scale.device != s.device:
        raise ValueError("g_scale must lie on the tensors' device")
    h = tsr_hyper(lr, wd, beta1, beta2, eps, scale)
    _launch(s.device, stream, _adamw, s.descs, s.count, _int(t), ctypes.byref(h), seed, _ptr(g_scale))


def tsr_grad_norm_workspace_bytes(tensors) -> int:
    s = _tensor_set(tensors)
    return int(_norm_ws(s.descs, s.count))


def tsr_grad_norm_batched(tensors, max_norm, norm, coef=None, ws=None, stream=None):
    """norm (one float32 value) <- the norm of all g; coef <- what brings it to max_norm at most."""
    s = _tensor_set(tensors)
    _scalar(norm, "norm")
    _scalar(coef, "coef")
    dev = _device_of(norm, coef, ws)
    if dev != s.device:
        raise ValueError("norm, coef and ws must lie on the tensors' device")
    if ws is None:
        ws = _temp_workspace(tsr_grad_norm_workspace_bytes(s), dev, stream)
    _launch(dev, stream, _norm, s.descs, s.count, max_norm, _ptr(norm), _ptr(coef), _ptr(ws), ws.numel())
    return norm


# ------------------------------------------------------------------ 8-bit matrices
def fp8_matrix(rows: int, cols: int, dtype=torch.float8_e4m3fn, block_rows=1, device="cuda"):
    """Place for an 8-bit matrix as the calls below take it: (q, scale), q rows x cols of a float8 type with rows padded to 16
    bytes, scale uint8 ceil(rows / block_rows) x ceil(cols / 128) with rows padded to 4."""
    q = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=device).view(dtype)[:, :cols]
    s = torch.empty(-(-rows // block_rows), -(-cols // 512) * 4, dtype=torch.uint8, device=device)[:, :-(-cols // 128)]
    return q, s


def _fp8(q: torch.Tensor) -> int:
    if q.dtype not in _FP8:
        raise TypeError("expected float8_e4m3fn or float8_e5m2")
    return _FP8[q.dtype]


def _fp8_place(q, s, rows, cols, block_rows, name):
    """(pointer, ld, scale pointer, ld) of an output of the quantiser, or four empty places."""
    if q is None:
        return None, 0, None, 0
    if s is None or tuple(q.shape) != (rows, cols) or s.dtype != torch.uint8 or tuple(s.shape) != (-(-rows // block_rows), -(-cols // 128)):
        raise ValueError("%s must be %d x %d with a uint8 scale for each %d x 128 of it" % (name, rows, cols, block_rows))
    return _ptr(q), _rows_ld(q), _ptr(s), _rows_ld(s)


def _rows_ld(t: torch.Tensor) -> int:
    """Leading dimension.  What torch says of a single row's pitch or a single column's stride may be anything and is not
    looked at; the pitch of a single row is made one that holds it."""
    ld, one = t.stride()
    if one != 1 and t.size(1) > 1:
        raise TypeError("expected a row-major 2-D tensor (unit column stride)")
    return ld if t.size(0) > 1 else -(-t.size(1) // 16) * 16


def tsr_fp8_quantize(X, Q=None, S=None, Qt=None, St=None, block_rows=1, stream=None):
    """X (float32 or bfloat16) into Q with scales S, and / or transposed into Qt with St (fp8_matrix makes such pairs)."""
    m, n = X.shape
    dev = _device_of(X, Q, S, Qt, St)
    some = Q if Q is not None else Qt
    if some is None or (Q is not None and Qt is not None and Q.dtype != Qt.dtype):
        raise ValueError("give Q, Qt or both, of one type")
    q, ldq, s, lds = _fp8_place(Q, S, m, n, block_rows, "Q")
    qt, ldqt, st, ldst = _fp8_place(Qt, St, n, m, block_rows, "Qt")
    _launch(dev, stream, _quantize, _ptr(X), _gdtype(X), _int(m), _int(n), _rows_ld(X), block_rows, _fp8(some), q, ldq, s, lds, qt, ldqt, st, ldst)


def _fp8_operand(q, s, rows, k, name) -> tsr_fp8_matrix:
    srows, scols = s.shape
    dtype = _FP8.get(q.dtype)
    if dtype is None:
        raise TypeError("%s must be float8_e4m3fn or float8_e5m2" % name)
    if s.dtype != torch.uint8 or scols != -(-k // 128) or srows not in (rows, -(-rows // 128)):
        raise ValueError("the scales of %s must be uint8, one for each 128 values of a row or of 128 rows" % name)
    return tsr_fp8_matrix(q.data_ptr(), s.data_ptr(), _rows_ld(q), _rows_ld(s), dtype, 1 if srows == rows else 128)


def tsr_fp8_matmul_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(_matmul_ws(_int(m), _int(n), _int(k)))


def tsr_fp8_matmul(A, SA, B, SB, C, ws=None, stream=None):
    """C (m x n, bfloat16) <- A B^T, A (m x k) and B (n x k) 8-bit with scales SA and SB."""
    m, k = A.shape
    n, kb = B.shape
    dev = _device_of(A, SA, B, SB, C, ws)
    if kb != k or C.shape != (m, n):
        raise ValueError("A m x k, B n x k and C m x n do not fit")
    if C.dtype != torch.bfloat16:
        raise TypeError("C must be bfloat16")
    if ws is None:
        nbytes = tsr_fp8_matmul_workspace_bytes(m, n, k)
        ws = _temp_workspace(nbytes, dev, stream) if nbytes else None
    a, b = _fp8_operand(A, SA, m, k, "A"), _fp8_operand(B, SB, n, k, "B")
    _launch(dev, stream, _matmul, ctypes.byref(a), ctypes.byref(b), _int(m), _int(n), _int(k), _ptr(C), _rows_ld(C), _ptr(ws),
            0 if ws is None else ws.numel())
    return C
