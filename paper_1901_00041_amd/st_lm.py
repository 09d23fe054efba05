"""Thin ctypes binding of the operators of language models (include/st_lm.h): same names as the C ABI, argument marshalling only.
They live in libst_conv.so beside the convolutions; status codes, errors and streams are those of st_conv."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

from . import st_conv as sc
from .st_conv import DTYPE_CODE, ST_EPI_RELU, ST_EPI_RESIDUAL, StError, _check, _ptr, _stream, plan_opts, st_plan_opts  # noqa: F401

ST_EPI_BIAS, ST_EPI_GELU, ST_EPI_GELU_TANH, ST_EPI_SILU, ST_EPI_RESIDUAL_LAST = 4, 8, 16, 32, 64


class st_matmul_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("M", "N", "K", "in_dtype", "out_dtype")] + [("epilogue", ctypes.c_uint32)] + \
               [(n, ctypes.c_int64) for n in ("ldx", "ldw", "ldy", "ldr")] + [(n, ctypes.c_void_p) for n in ("x", "w", "bias", "y", "residual")]


class st_matmul_plan_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_tenants", "host_only", "launches", "reserved")] + \
               [(n, ctypes.c_int64) for n in ("n_items", "flops", "bytes", "workspace_bytes")]


class st_matmul_tenant_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tile_cfg", "MT", "NT", "tiles_m", "tiles_n", "split_k")] + [("item_count", ctypes.c_int64)]


_bound = False


def lib() -> ctypes.CDLL:
    """The loaded shared library (see st_conv.lib), with this header's signatures."""
    global _bound
    L = sc.lib()
    if not _bound:
        vp, i32, P = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER
        for name, args in (("st_matmul_plan", [P(st_matmul_desc), i32, P(st_plan_opts), P(vp)]), ("st_matmul_run", [vp, vp]),
                           ("st_matmul_rebind_all", [vp, P(st_matmul_desc), i32, vp]), ("st_matmul_get_info", [vp, P(st_matmul_plan_info)]),
                           ("st_matmul_get_tenant_info", [vp, i32, P(st_matmul_tenant_info)]), ("st_matmul_tile_shape", [i32, P(i32), P(i32)]),
                           ("st_matmul_tile_count", [])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, i32
        for name in ("st_matmul_destroy",):
            getattr(L, name).argtypes, getattr(L, name).restype = [vp], None
        _bound = True
    return L


class _Owned:
    """Owns a plan handle; keeps the tensors it borrows alive."""
    _destroy = ""

    def __init__(self, handle: int, keep):
        self.handle, self._keep = handle, keep

    def destroy(self):
        if getattr(self, "handle", None) and sc._lib is not None:
            try:
                getattr(sc._lib, self._destroy)(self.handle)
            except Exception:      # interpreter shutdown
                pass
            self.handle = None

    def __del__(self):
        self.destroy()


class MatmulPlan(_Owned):
    _destroy = "st_matmul_destroy"


def _run(name: str, plan: _Owned, stream) -> None:
    # the stream and the status are looked at here: a decoding step makes several of these calls, each a few microseconds long
    try:
        st = getattr(lib(), name)(plan.handle, stream if stream is None or type(stream) is int else stream.cuda_stream)
    except (AttributeError, ctypes.ArgumentError):
        st = getattr(lib(), name)(plan.handle, _stream(stream))
    if st != sc.ST_OK:
        raise StError(st, name)


def _array(kind, descs):
    return (kind * max(len(descs), 1))(*descs), len(descs)


# ---- matrix products ----------------------------------------------------------------------------------------------
def make_matmul_desc(M, N, K, in_dtype, out_dtype, x, w, y, bias=None, residual=None, epilogue=0, ldx=0, ldw=0, ldy=0, ldr=0) -> st_matmul_desc:
    d = st_matmul_desc()
    d.M, d.N, d.K = M, N, K
    d.in_dtype, d.out_dtype = DTYPE_CODE.get(in_dtype, in_dtype), DTYPE_CODE.get(out_dtype, out_dtype)
    d.epilogue = epilogue
    d.ldx, d.ldw, d.ldy, d.ldr = ldx, ldw, ldy, ldr
    d.x, d.w, d.bias, d.y, d.residual = _ptr(x), _ptr(w), _ptr(bias), _ptr(y), _ptr(residual)
    return d


def st_matmul_plan(descs: Sequence[st_matmul_desc], opts: Optional[st_plan_opts] = None, keep=None) -> MatmulPlan:
    arr, n = _array(st_matmul_desc, descs)
    out = ctypes.c_void_p()
    _check(lib().st_matmul_plan(arr, n, ctypes.byref(opts) if opts is not None else None, ctypes.byref(out)), "st_matmul_plan")
    return MatmulPlan(out.value, keep)


def st_matmul_run(plan: MatmulPlan, stream=None) -> None:
    _run("st_matmul_run", plan, stream)


def st_matmul_rebind_all(plan: MatmulPlan, descs: Sequence[st_matmul_desc], stream=None, keep=None) -> None:
    arr, n = _array(st_matmul_desc, descs)
    _check(lib().st_matmul_rebind_all(plan.handle, arr, n, _stream(stream)), "st_matmul_rebind_all")
    if keep is not None:
        plan._keep = (plan._keep, keep)


def st_matmul_get_info(plan: MatmulPlan) -> st_matmul_plan_info:
    out = st_matmul_plan_info()
    _check(lib().st_matmul_get_info(plan.handle, ctypes.byref(out)), "st_matmul_get_info")
    return out


def st_matmul_get_tenant_info(plan: MatmulPlan, tenant: int) -> st_matmul_tenant_info:
    out = st_matmul_tenant_info()
    _check(lib().st_matmul_get_tenant_info(plan.handle, tenant, ctypes.byref(out)), "st_matmul_get_tenant_info")
    return out


def st_matmul_tile_shape(index: int):
    mt, nt = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().st_matmul_tile_shape(index, ctypes.byref(mt), ctypes.byref(nt)), "st_matmul_tile_shape")
    return mt.value, nt.value


def st_matmul_tile_count() -> int:
    return lib().st_matmul_tile_count()
