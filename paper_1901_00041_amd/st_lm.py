"""Thin ctypes binding of the operators of language models (include/st_lm.h): same names as the C ABI, argument marshalling only.
They live in libst_conv.so beside the convolutions; status codes, errors and streams are those of st_conv."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

from . import st_conv as sc
from .st_conv import DTYPE_CODE, ST_EPI_RELU, ST_EPI_RESIDUAL, StError, _check, _ptr, _stream, plan_opts, st_plan_opts  # noqa: F401

ST_EPI_BIAS, ST_EPI_GELU, ST_EPI_GELU_TANH, ST_EPI_SILU, ST_EPI_RESIDUAL_LAST = 4, 8, 16, 32, 64
ST_ATTN_CAUSAL = 1
ST_ATTN_BAD_PAGE, ST_ATTN_BAD_LENGTH = 1, 2


class st_matmul_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("M", "N", "K", "in_dtype", "out_dtype")] + [("epilogue", ctypes.c_uint32)] + \
               [(n, ctypes.c_int64) for n in ("ldx", "ldw", "ldy", "ldr")] + [(n, ctypes.c_void_p) for n in ("x", "w", "bias", "y", "residual")]


class st_matmul_plan_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_tenants", "host_only", "launches", "reserved")] + \
               [(n, ctypes.c_int64) for n in ("n_items", "flops", "bytes", "workspace_bytes")]


class st_matmul_tenant_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tile_cfg", "MT", "NT", "tiles_m", "tiles_n", "split_k")] + [("item_count", ctypes.c_int64)]


class st_attn_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("heads", "kv_heads", "head_dim", "dtype", "n_seqs", "max_tokens", "max_new", "n_pages", "page_tokens",
                                              "table_pages", "window")] + \
               [("flags", ctypes.c_uint32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)] + \
               [(n, ctypes.c_int64) for n in ("ldq", "ldk", "ldv", "ldo")] + \
               [(n, ctypes.c_void_p) for n in ("q", "k", "v", "out", "k_out", "v_out", "pages", "table", "first", "length")]


class st_attn_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_tenants", "host_only", "launches", "reserved")] + [(n, ctypes.c_int64) for n in ("n_items", "workspace_bytes")]


_bound = False


def lib() -> ctypes.CDLL:
    """The loaded shared library (see st_conv.lib), with this header's signatures."""
    global _bound
    L = sc.lib()
    if not _bound:
        vp, i32, i64, P = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.POINTER
        for name, args in (("st_matmul_plan", [P(st_matmul_desc), i32, P(st_plan_opts), P(vp)]), ("st_matmul_run", [vp, vp]),
                           ("st_matmul_rebind_all", [vp, P(st_matmul_desc), i32, vp]), ("st_matmul_get_info", [vp, P(st_matmul_plan_info)]),
                           ("st_matmul_get_tenant_info", [vp, i32, P(st_matmul_tenant_info)]), ("st_matmul_tile_shape", [i32, P(i32), P(i32)]),
                           ("st_matmul_tile_count", []),
                           ("st_attn_plan", [P(st_attn_desc), i32, P(st_plan_opts), P(vp)]), ("st_attn_append", [vp, vp]), ("st_attn_read", [vp, vp]),
                           ("st_attn_run", [vp, vp]), ("st_attn_rebind_all", [vp, P(st_attn_desc), i32, vp]), ("st_attn_status", [vp, P(i32)]),
                           ("st_attn_get_info", [vp, P(st_attn_info)])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, i32
        L.st_attn_page_bytes.argtypes, L.st_attn_page_bytes.restype = [P(st_attn_desc)], i64
        for name in ("st_matmul_destroy", "st_attn_destroy"):
            getattr(L, name).argtypes, getattr(L, name).restype = [vp], None
        _bound = True
    return L


class _Owned:
    """Owns a plan handle and keeps alive what it borrows: every object that was given as `keep`, when the plan was made and at each rebinding, until
    release() or destroy().  A program that rebinds to new tensors again and again calls release() now and then, or holds its tensors itself."""
    _destroy = ""

    def __init__(self, handle: int, keep):
        self.handle, self._held = handle, {}
        self._hold(keep)

    def _hold(self, keep):
        if keep is not None:
            self._held[id(keep)] = keep

    @property
    def kept(self) -> list:
        return list(self._held.values())

    def release(self, keep=None) -> None:
        """Lets go of all but `keep`, which has to cover what the plan is bound to now.  To be called when the runs that used the rest have ended, and
        no graph will run them again."""
        self._held = {}
        self._hold(keep)

    def destroy(self):
        if getattr(self, "handle", None):
            try:
                getattr(sc._lib, self._destroy)(self.handle)
            except Exception:      # interpreter shutdown
                pass
            self.handle = None
            self._held = {}

    def __del__(self):
        self.destroy()


class MatmulPlan(_Owned):
    _destroy = "st_matmul_destroy"


class AttnPlan(_Owned):
    _destroy = "st_attn_destroy"


def _run(name: str, plan: _Owned, stream) -> None:
    # the stream and the status are looked at here: a decoding step makes several of these calls, each a few microseconds long
    try:
        st = getattr(sc._lib if _bound else lib(), name)(plan.handle, stream if stream is None or type(stream) is int else stream.cuda_stream)
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
    plan._hold(keep)


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


# ---- attention over a paged cache in 4 bits -----------------------------------------------------------------------
def make_attn_desc(heads, kv_heads, head_dim, dtype, n_seqs, max_tokens, max_new, n_pages, page_tokens, table_pages, pages=None, table=None, first=None,
                   length=None, q=None, k=None, v=None, out=None, k_out=None, v_out=None, scale=1.0, window=0, flags=0, ldq=0, ldk=0, ldv=0,
                   ldo=0) -> st_attn_desc:
    d = st_attn_desc()
    d.heads, d.kv_heads, d.head_dim, d.dtype = heads, kv_heads, head_dim, DTYPE_CODE.get(dtype, dtype)
    d.n_seqs, d.max_tokens, d.max_new = n_seqs, max_tokens, max_new
    d.n_pages, d.page_tokens, d.table_pages = n_pages, page_tokens, table_pages
    d.window, d.flags, d.scale, d.reserved = window, flags, scale, 0
    d.ldq, d.ldk, d.ldv, d.ldo = ldq, ldk, ldv, ldo
    d.q, d.k, d.v, d.out, d.k_out, d.v_out = (_ptr(t) for t in (q, k, v, out, k_out, v_out))
    d.pages, d.table, d.first, d.length = (_ptr(t) for t in (pages, table, first, length))
    return d


def st_attn_page_bytes(desc: st_attn_desc) -> int:
    return int(lib().st_attn_page_bytes(ctypes.byref(desc)))


def st_attn_plan(descs: Sequence[st_attn_desc], opts: Optional[st_plan_opts] = None, keep=None) -> AttnPlan:
    arr, n = _array(st_attn_desc, descs)
    out = ctypes.c_void_p()
    _check(lib().st_attn_plan(arr, n, ctypes.byref(opts) if opts is not None else None, ctypes.byref(out)), "st_attn_plan")
    return AttnPlan(out.value, keep)


def st_attn_append(plan: AttnPlan, stream=None) -> None:
    _run("st_attn_append", plan, stream)


def st_attn_read(plan: AttnPlan, stream=None) -> None:
    _run("st_attn_read", plan, stream)


def st_attn_run(plan: AttnPlan, stream=None) -> None:
    _run("st_attn_run", plan, stream)


def st_attn_rebind_all(plan: AttnPlan, descs: Sequence[st_attn_desc], stream=None, keep=None) -> None:
    arr, n = _array(st_attn_desc, descs)
    _check(lib().st_attn_rebind_all(plan.handle, arr, n, _stream(stream)), "st_attn_rebind_all")
    plan._hold(keep)


def st_attn_status(plan: AttnPlan) -> int:
    out = ctypes.c_int32()
    _check(lib().st_attn_status(plan.handle, ctypes.byref(out)), "st_attn_status")
    return out.value


def st_attn_get_info(plan: AttnPlan) -> st_attn_info:
    out = st_attn_info()
    _check(lib().st_attn_get_info(plan.handle, ctypes.byref(out)), "st_attn_get_info")
    return out
