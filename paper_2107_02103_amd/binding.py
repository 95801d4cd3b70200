"""ctypes binding of libdpc.so (see include/dpc.h).

Argument marshalling only: every computation happens in the library (host
table builder and HIP kernels).  Functions keep the C names; device arrays are
torch tensors on a ROCm device (their data pointers are passed), host arrays
are numpy arrays.  A missing library is an ImportError: there is no fallback.
"""
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libdpc.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"libdpc.so not found at {LIB_PATH}; build it with "
        "`python -m paper_2107_02103_amd.build` (or __graft_entry__.build())")
# PyTorch-ROCm ships its own HIP runtime with the same SONAME as the system one
# (libamdhip64.so.7).  Loading torch first makes the dynamic linker bind
# libdpc.so to that already-loaded runtime, so that the library, torch's
# allocator and torch's streams share one HIP runtime in the process.
try:
    import torch  # noqa: F401
except ImportError:  # the C library can be used without torch
    torch = None
_lib = C.CDLL(LIB_PATH)

DPC_OK, DPC_EINVAL, DPC_ERANGE, DPC_EHIP, DPC_ENOTSUP, DPC_EOVERFLOW = 0, -1, -2, -3, -4, -5
DPC_F64, DPC_F32, DPC_F32_ACC64 = 0, 1, 2
DPC_MAX_TYPES, DPC_MAX_M1 = 8, 256
DPC_NLIST_NOALLOC_MAX_ATOMS = 524288
DPC_ELEM_F64, DPC_ELEM_F32, DPC_ELEM_F16, DPC_ELEM_BF16 = 0, 1, 2, 3
DPC_MAX_EXPERTS, DPC_MAX_TOPK, DPC_MAX_I8_COLS = 1024, 64, 131071
EXPORTED = ("dpc_strerror", "dpc_last_hip_error", "dpc_version", "dpc_table_layout", "dpc_build_table",
            "dpc_se_a_tab_fwd", "dpc_se_a_tab_bwd", "dpc_descriptor_bwd", "dpc_env_mat_a",
            "dpc_nlist_reverse", "dpc_force_a", "dpc_fitting_workspace_bytes", "dpc_fitting_fwd_bwd",
            "dpc_nlist_workspace_bytes", "dpc_nlist_build", "dpc_nlist_build_noalloc",
            "dpc_se_a_tab_bwd_from_dD", "dpc_route_workspace_bytes", "dpc_route_plan", "dpc_route_gather",
            "dpc_route_combine", "dpc_route_combine_bwd", "dpc_quant_rows", "dpc_matmul_i8",
            "dpc_linear_i8_workspace_bytes", "dpc_linear_i8")


class dpc_range(C.Structure):
    _fields_ = [("lo", C.c_double), ("d1", C.c_double), ("d2", C.c_double),
                ("L1", C.c_int64), ("L2", C.c_int64), ("offset", C.c_int64)]


class dpc_net(C.Structure):
    _fields_ = [("n_layers", C.c_int), ("widths", C.POINTER(C.c_int)),
                ("W", C.POINTER(C.POINTER(C.c_double))), ("b", C.POINTER(C.POINTER(C.c_double)))]


_lib.dpc_strerror.restype = C.c_char_p
_lib.dpc_strerror.argtypes = [C.c_int]
_lib.dpc_version.restype = C.c_int
_lib.dpc_last_hip_error.restype = C.c_char_p
_lib.dpc_table_layout.restype = C.c_int
_lib.dpc_table_layout.argtypes = [C.c_int, C.c_int, C.POINTER(dpc_range), C.c_int,
                                  C.POINTER(C.c_size_t)]
_lib.dpc_build_table.restype = C.c_int
_lib.dpc_build_table.argtypes = [C.POINTER(dpc_net), C.POINTER(dpc_range), C.c_int, C.c_void_p]
_lib.dpc_se_a_tab_fwd.restype = C.c_int
_lib.dpc_se_a_tab_fwd.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int),
                                  C.c_int, C.c_int, C.POINTER(dpc_range), C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.dpc_se_a_tab_bwd.restype = C.c_int
_lib.dpc_se_a_tab_bwd.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int),
                                  C.c_int, C.POINTER(dpc_range), C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.dpc_se_a_tab_bwd_from_dD.restype = C.c_int
_lib.dpc_se_a_tab_bwd_from_dD.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int),
                                          C.c_int, C.c_int, C.POINTER(dpc_range), C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]


class dpc_fitting_net(C.Structure):
    _fields_ = [("n_in", C.c_int), ("width", C.c_int), ("W", C.c_void_p * 3), ("b", C.c_void_p * 3),
                ("w_out", C.c_void_p), ("b_out", C.c_double)]


_lib.dpc_fitting_workspace_bytes.restype = C.c_size_t
_lib.dpc_fitting_workspace_bytes.argtypes = [C.c_int, C.c_int]
_lib.dpc_fitting_fwd_bwd.restype = C.c_int
_lib.dpc_fitting_fwd_bwd.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.POINTER(dpc_fitting_net),
                                     C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
_D = C.c_double
_lib.dpc_env_mat_a.restype = C.c_int
_lib.dpc_env_mat_a.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, _D, _D, _D,
                               C.POINTER(_D), C.POINTER(_D), C.POINTER(_D), C.c_void_p, C.c_void_p,
                               C.c_void_p, C.c_void_p]
_lib.dpc_nlist_reverse.restype = C.c_int
_lib.dpc_nlist_reverse.argtypes = [C.c_void_p, C.c_int, C.c_int, C.POINTER(C.c_int), _D, C.c_void_p,
                                   C.c_void_p, C.c_void_p, C.c_void_p]
_lib.dpc_force_a.restype = C.c_int
_lib.dpc_force_a.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, _D, _D, _D,
                             C.POINTER(_D), C.POINTER(_D), C.c_void_p, C.c_void_p, C.c_void_p,
                             C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.dpc_nlist_workspace_bytes.restype = C.c_size_t
_lib.dpc_nlist_workspace_bytes.argtypes = [C.c_int, _D, _D]
_lib.dpc_nlist_build.restype = C.c_int
_lib.dpc_nlist_build.argtypes = [C.c_void_p, C.c_int, C.c_int, C.POINTER(C.c_int), _D, _D, C.c_void_p,
                                 C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_int)]
_lib.dpc_nlist_build_noalloc.restype = C.c_int
_lib.dpc_nlist_build_noalloc.argtypes = [C.c_void_p, C.c_int, C.c_int, C.POINTER(C.c_int), _D, _D,
                                         C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
_lib.dpc_descriptor_bwd.restype = C.c_int
_lib.dpc_descriptor_bwd.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p,
                                    C.c_void_p, C.c_void_p]
_P, _I, _L, _Z = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
_lib.dpc_route_workspace_bytes.restype = _Z
_lib.dpc_route_workspace_bytes.argtypes = [_I, _I, _I]
_lib.dpc_route_plan.restype = _I
_lib.dpc_route_plan.argtypes = [_P, _I, _I, _I, _P, _P, _Z, _P, _P, _P]
_lib.dpc_route_gather.restype = _I
_lib.dpc_route_gather.argtypes = [_P, _I, _I, _I, _I, _P, _L, _P, _P, _P, _P, _L]
_lib.dpc_route_combine.restype = _I
_lib.dpc_route_combine.argtypes = [_P, _I, _I, _I, _I, _P, _L, _P, _P, _P, _L]
_lib.dpc_route_combine_bwd.restype = _I
_lib.dpc_route_combine_bwd.argtypes = [_P, _I, _I, _I, _I, _P, _L, _P, _P, _P, _P, _L, _P, _L, _P]
_lib.dpc_quant_rows.restype = _I
_lib.dpc_quant_rows.argtypes = [_P, _I, _I, _I, _P, _L, _P, _P]
_lib.dpc_matmul_i8.restype = _I
_lib.dpc_matmul_i8.argtypes = [_P, _I, _I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _L]
_lib.dpc_linear_i8_workspace_bytes.restype = _Z
_lib.dpc_linear_i8_workspace_bytes.argtypes = [_I, _I]
_lib.dpc_linear_i8.restype = _I
_lib.dpc_linear_i8.argtypes = [_P, _I, _I, _I, _I, _I, _I, _I, _P, _L, _P, _P, _P, _P, _P, _P, _Z, _P, _L]


class DpcError(RuntimeError):
    def __init__(self, status, where=""):
        self.status = status
        msg = f"{where}: {dpc_strerror(status)} ({status})"
        if status == DPC_EHIP:
            msg += ": " + dpc_last_hip_error()
        super().__init__(msg)


def _check(status, where):
    if status != DPC_OK:
        raise DpcError(status, where)


def dpc_strerror(status):
    return _lib.dpc_strerror(int(status)).decode()


def dpc_last_hip_error():
    return _lib.dpc_last_hip_error().decode()


def dpc_version():
    return int(_lib.dpc_version())


def table_ld(m1):
    """Row stride of the coefficient table (DPC_TABLE_LD in dpc.h)."""
    return (int(m1) + 3) // 4 * 4


def unpack_table(buf, n_intervals, ld):
    """View of one pair's coefficients as [interval][power q][channel]
    (the buffer holds [interval][q // 2][channel][q % 2], DPC_TABLE_AT in dpc.h)."""
    a = np.asarray(buf).reshape(n_intervals, 3, ld, 2)
    return a.transpose(0, 1, 3, 2).reshape(n_intervals, 6, ld)


def make_ranges(lo, d1, L1, d2, L2):
    """ctypes array of dpc_range from per-pair sequences."""
    n = len(lo)
    arr = (dpc_range * n)()
    for p in range(n):
        arr[p].lo, arr[p].d1, arr[p].d2 = float(lo[p]), float(d1[p]), float(d2[p])
        arr[p].L1, arr[p].L2, arr[p].offset = int(L1[p]), int(L2[p]), 0
    return arr


def dpc_table_layout(ranges, m1, dtype):
    """Fills ranges[p].offset; returns the coefficient buffer size in bytes."""
    total = C.c_size_t(0)
    _check(_lib.dpc_table_layout(len(ranges), int(m1), ranges, int(dtype), C.byref(total)),
           "dpc_table_layout")
    return int(total.value)


def _net_struct(net):
    W = [np.ascontiguousarray(w, np.float64) for w in net["W"]]
    b = [np.ascontiguousarray(v, np.float64) for v in net["b"]]
    widths = [W[0].shape[0]] + [w.shape[1] for w in W]
    keep = (W, b)
    s = dpc_net()
    s.n_layers = len(W)
    s.widths = (C.c_int * len(widths))(*widths)
    s.W = (C.POINTER(C.c_double) * len(W))(*[w.ctypes.data_as(C.POINTER(C.c_double)) for w in W])
    s.b = (C.POINTER(C.c_double) * len(b))(*[v.ctypes.data_as(C.POINTER(C.c_double)) for v in b])
    return s, keep


def dpc_build_table(net, rng, dtype, host_out):
    """Tabulate one net (dict of W, b lists) over one dpc_range into host_out
    (a numpy array with room for (L1 + L2) * 6 * table_ld(m1) coefficients)."""
    s, keep = _net_struct(net)
    m1 = keep[0][-1].shape[1]
    need = (rng.L1 + rng.L2) * 6 * table_ld(m1)
    want = np.float64 if dtype == DPC_F64 else np.float32
    if host_out.dtype != want or host_out.size < need or not host_out.flags.c_contiguous:
        raise ValueError("host_out has the wrong dtype, size or layout")
    _check(_lib.dpc_build_table(C.byref(s), C.byref(rng), int(dtype),
                                host_out.ctypes.data_as(C.c_void_p)), "dpc_build_table")
    return host_out


def build_tables(nets, ranges, dtype):
    """All pairs' tables in one host buffer laid out by dpc_table_layout."""
    m1 = np.asarray(nets[0]["W"][-1]).shape[1]
    nbytes = dpc_table_layout(ranges, m1, dtype)
    want = np.float64 if dtype == DPC_F64 else np.float32
    buf = np.zeros(nbytes // np.dtype(want).itemsize, want)
    for p, net in enumerate(nets):
        r = ranges[p]
        n = (r.L1 + r.L2) * 6 * table_ld(m1)
        dpc_build_table(net, r, dtype, buf[r.offset:r.offset + n])
    return buf


def _ptr(x, dtype=None, name="?"):
    """Device pointer of a contiguous torch tensor on a GPU (or an int
    address, taken as is).  A tensor in host memory is refused: its address
    would reach the kernels as a device address."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not getattr(x, "is_cuda", False):
        raise ValueError(f"{name} must be a tensor on a GPU device, not {getattr(x, 'device', type(x))}")
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and x.dtype != dtype:
        raise TypeError(f"{name} has dtype {x.dtype}, expected {dtype}")
    return x.data_ptr()


def _one_device(stream, **tensors):
    """Every tensor argument (and a torch stream) must be on one GPU."""
    devs = {k: v.device for k, v in tensors.items() if v is not None and not isinstance(v, int)}
    for k, v in tensors.items():
        if v is not None and not isinstance(v, int):
            _ptr(v, name=k)
    if stream is not None and not isinstance(stream, int) and hasattr(stream, "device"):
        devs["stream"] = stream.device
    idx = {(d.type, d.index) for d in devs.values()}
    if len(idx) > 1:
        raise ValueError("arguments on different devices: "
                         + ", ".join(f"{k}={d}" for k, d in devs.items()))


def _sel(sel):
    return (C.c_int * len(sel))(*[int(s) for s in sel])


def _need(x, count, esize, name):
    """A tensor argument must hold at least `count` elements of `esize`
    bytes: the library cannot see the size of a device buffer, so an
    undersized one is refused here, before anything is launched."""
    if x is None or isinstance(x, int):
        return
    have = x.numel() * x.element_size()
    if have < int(count) * esize:
        raise ValueError(f"{name} holds {have} bytes, needs {int(count) * esize}")


def _io_sizes(dtype):
    """(input element bytes, output element bytes) of a dtype mode."""
    return {DPC_F64: (8, 8), DPC_F32: (4, 4), DPC_F32_ACC64: (4, 8)}.get(int(dtype), (8, 8))


def _stream(stream):
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def dpc_se_a_tab_fwd(stream, dtype, nloc, ntypes, sel, m1, m2, ranges, coeff, atype, nlist, em,
                     T, D):
    nnei, (ei, eo) = sum(int(v) for v in sel), _io_sizes(dtype)
    _need(atype, nloc, 4, "atype"); _need(nlist, nloc * nnei, 4, "nlist")
    _need(em, nloc * nnei * 4, ei, "em"); _need(T, nloc * m1 * 4, eo, "T"); _need(D, nloc * m1 * m2, eo, "D")
    _one_device(stream, coeff=coeff, atype=atype, nlist=nlist, em=em, T=T, D=D)
    _check(_lib.dpc_se_a_tab_fwd(_stream(stream), int(dtype), int(nloc), int(ntypes), _sel(sel),
                                 int(m1), int(m2), ranges, _ptr(coeff, name="coeff"),
                                 _ptr(atype, name="atype"), _ptr(nlist, name="nlist"),
                                 _ptr(em, name="em"), _ptr(T, name="T"), _ptr(D, name="D")),
           "dpc_se_a_tab_fwd")


def dpc_se_a_tab_bwd(stream, dtype, nloc, ntypes, sel, m1, ranges, coeff, atype, nlist, em,
                     dE_dT, dE_dem):
    nnei, (ei, eo) = sum(int(v) for v in sel), _io_sizes(dtype)
    _need(atype, nloc, 4, "atype"); _need(nlist, nloc * nnei, 4, "nlist")
    _need(em, nloc * nnei * 4, ei, "em"); _need(dE_dT, nloc * m1 * 4, ei, "dE_dT")
    _need(dE_dem, nloc * nnei * 4, eo, "dE_dem")
    _one_device(stream, coeff=coeff, atype=atype, nlist=nlist, em=em, dE_dT=dE_dT, dE_dem=dE_dem)
    _check(_lib.dpc_se_a_tab_bwd(_stream(stream), int(dtype), int(nloc), int(ntypes), _sel(sel),
                                 int(m1), ranges, _ptr(coeff, name="coeff"),
                                 _ptr(atype, name="atype"), _ptr(nlist, name="nlist"),
                                 _ptr(em, name="em"), _ptr(dE_dT, name="dE_dT"),
                                 _ptr(dE_dem, name="dE_dem")),
           "dpc_se_a_tab_bwd")


def dpc_se_a_tab_bwd_from_dD(stream, dtype, nloc, ntypes, sel, m1, m2, ranges, coeff, atype, nlist,
                             em, T, dE_dD, dE_dem):
    nnei = sum(int(v) for v in sel)
    _need(atype, nloc, 4, "atype"); _need(nlist, nloc * nnei, 4, "nlist")
    _need(em, nloc * nnei * 4, 8, "em"); _need(T, nloc * m1 * 4, 8, "T")
    _need(dE_dD, nloc * m1 * m2, 8, "dE_dD"); _need(dE_dem, nloc * nnei * 4, 8, "dE_dem")
    _one_device(stream, coeff=coeff, atype=atype, nlist=nlist, em=em, T=T, dE_dD=dE_dD, dE_dem=dE_dem)
    _check(_lib.dpc_se_a_tab_bwd_from_dD(_stream(stream), int(dtype), int(nloc), int(ntypes), _sel(sel),
                                         int(m1), int(m2), ranges, _ptr(coeff, name="coeff"),
                                         _ptr(atype, name="atype"), _ptr(nlist, name="nlist"),
                                         _ptr(em, name="em"), _ptr(T, name="T"), _ptr(dE_dD, name="dE_dD"),
                                         _ptr(dE_dem, name="dE_dem")),
           "dpc_se_a_tab_bwd_from_dD")


def dpc_descriptor_bwd(stream, dtype, nloc, m1, m2, T, dE_dD, dE_dT):
    ei = 4 if int(dtype) == DPC_F32 else 8
    eo = 8 if int(dtype) == DPC_F64 else 4
    _need(T, nloc * m1 * 4, ei, "T"); _need(dE_dD, nloc * m1 * m2, ei, "dE_dD")
    _need(dE_dT, nloc * m1 * 4, eo, "dE_dT")
    _one_device(stream, T=T, dE_dD=dE_dD, dE_dT=dE_dT)
    _check(_lib.dpc_descriptor_bwd(_stream(stream), int(dtype), int(nloc), int(m1), int(m2),
                                   _ptr(T, name="T"), _ptr(dE_dD, name="dE_dD"),
                                   _ptr(dE_dT, name="dE_dT")),
           "dpc_descriptor_bwd")


def _dvec(v, n, name):
    a = np.ascontiguousarray(v, dtype=np.float64).ravel()
    if a.size < n:
        raise ValueError(f"{name} needs {n} values")
    return a.ctypes.data_as(C.POINTER(C.c_double)), a


def dpc_env_mat_a(stream, dtype, nloc, ntypes, nnei, box, rc, rcs, mean, sigma, sigma_all, coord,
                  atype, nlist, em):
    pm, km = _dvec(mean, ntypes, "mean")
    ps, ks = _dvec(sigma, ntypes, "sigma")
    pa, ka = _dvec(sigma_all, ntypes, "sigma_all")
    _need(coord, nloc * 3, 8, "coord"); _need(atype, nloc, 4, "atype")
    _need(nlist, nloc * nnei, 4, "nlist"); _need(em, nloc * nnei * 4, 8 if int(dtype) == DPC_F64 else 4, "em")
    _one_device(stream, coord=coord, atype=atype, nlist=nlist, em=em)
    _check(_lib.dpc_env_mat_a(_stream(stream), int(dtype), int(nloc), int(ntypes), int(nnei),
                              float(box), float(rc), float(rcs), pm, ps, pa, _ptr(coord, name="coord"),
                              _ptr(atype, name="atype"), _ptr(nlist, name="nlist"), _ptr(em, name="em")),
           "dpc_env_mat_a")


def dpc_nlist_reverse(stream, nloc, ntypes, sel, box, coord, atype, nlist, rev):
    nnei = sum(int(v) for v in sel)
    _need(coord, nloc * 3, 8, "coord"); _need(atype, nloc, 4, "atype")
    _need(nlist, nloc * nnei, 4, "nlist"); _need(rev, nloc * nnei, 4, "rev")
    _one_device(stream, coord=coord, atype=atype, nlist=nlist, rev=rev)
    _check(_lib.dpc_nlist_reverse(_stream(stream), int(nloc), int(ntypes), _sel(sel), float(box),
                                  _ptr(coord, name="coord"), _ptr(atype, name="atype"),
                                  _ptr(nlist, name="nlist"), _ptr(rev, name="rev")),
           "dpc_nlist_reverse")


def dpc_force_a(stream, dtype, nloc, ntypes, nnei, box, rc, rcs, sigma, sigma_all, coord, atype,
                nlist, rev, dE_dem, force, virial=None):
    ps, ks = _dvec(sigma, ntypes, "sigma")
    pa, ka = _dvec(sigma_all, ntypes, "sigma_all")
    _need(coord, nloc * 3, 8, "coord"); _need(atype, nloc, 4, "atype")
    _need(nlist, nloc * nnei, 4, "nlist"); _need(rev, nloc * nnei, 4, "rev")
    _need(dE_dem, nloc * nnei * 4, 4 if int(dtype) == DPC_F32 else 8, "dE_dem")
    _need(force, nloc * 3, 8, "force"); _need(virial, nloc * 9, 8, "virial")
    _one_device(stream, coord=coord, atype=atype, nlist=nlist, rev=rev, dE_dem=dE_dem, force=force,
                virial=virial)
    _check(_lib.dpc_force_a(_stream(stream), int(dtype), int(nloc), int(ntypes), int(nnei),
                            float(box), float(rc), float(rcs), ps, pa, _ptr(coord, name="coord"),
                            _ptr(atype, name="atype"), _ptr(nlist, name="nlist"),
                            _ptr(rev, name="rev"), _ptr(dE_dem, name="dE_dem"),
                            _ptr(force, name="force"), _ptr(virial, name="virial")),
           "dpc_force_a")


def dpc_nlist_workspace_bytes(nloc, box, rc):
    return int(_lib.dpc_nlist_workspace_bytes(int(nloc), float(box), float(rc)))


def dpc_nlist_build(stream, nloc, ntypes, sel, box, rc, coord, atype, workspace, workspace_bytes, nlist,
                    wait=True):
    """Neighbour list into ``nlist``.  With ``wait`` the call synchronises and
    returns the two status counters (truncated lists, lists over capacity),
    raising DpcError for either; without, it returns None."""
    nnei = sum(int(v) for v in sel)
    _need(coord, nloc * 3, 8, "coord"); _need(atype, nloc, 4, "atype")
    _need(workspace, workspace_bytes, 1, "workspace"); _need(nlist, nloc * nnei, 4, "nlist")
    _one_device(stream, coord=coord, atype=atype, workspace=workspace, nlist=nlist)
    st = (C.c_int * 2)(0, 0) if wait else None
    _check(_lib.dpc_nlist_build(_stream(stream), int(nloc), int(ntypes), _sel(sel), float(box), float(rc),
                                _ptr(coord, name="coord"), _ptr(atype, name="atype"),
                                _ptr(workspace, name="workspace"), int(workspace_bytes),
                                _ptr(nlist, name="nlist"), st), "dpc_nlist_build")
    return (st[0], st[1]) if wait else None


def dpc_nlist_build_noalloc(stream, nloc, ntypes, sel, box, rc, coord, atype, nlist, status=None):
    """dpc_nlist_build with the library's static cell list (no allocation,
    asynchronous); ``status``: a device int32 tensor of 2 for the counters."""
    nnei = sum(int(v) for v in sel)
    _need(coord, nloc * 3, 8, "coord"); _need(atype, nloc, 4, "atype")
    _need(nlist, nloc * nnei, 4, "nlist"); _need(status, 2, 4, "status")
    _one_device(stream, coord=coord, atype=atype, nlist=nlist, status=status)
    _check(_lib.dpc_nlist_build_noalloc(_stream(stream), int(nloc), int(ntypes), _sel(sel), float(box),
                                        float(rc), _ptr(coord, name="coord"), _ptr(atype, name="atype"),
                                        _ptr(nlist, name="nlist"), _ptr(status, name="status")),
           "dpc_nlist_build_noalloc")


def dpc_fitting_workspace_bytes(nloc, width):
    return int(_lib.dpc_fitting_workspace_bytes(int(nloc), int(width)))


def dpc_fitting_fwd_bwd(stream, blas, nloc, net, D, workspace, workspace_bytes, E, dE_dD=None):
    """``net``: a dpc_fitting_net whose pointers are device addresses;
    ``blas``: a rocblas_handle (int), see RocblasHandle."""
    _need(D, nloc * net.n_in, 8, "D"); _need(E, nloc, 8, "E"); _need(dE_dD, nloc * net.n_in, 8, "dE_dD")
    _need(workspace, workspace_bytes, 1, "workspace")
    _one_device(stream, D=D, workspace=workspace, E=E, dE_dD=dE_dD)
    _check(_lib.dpc_fitting_fwd_bwd(_stream(stream), blas, int(nloc), C.byref(net), _ptr(D, name="D"),
                                    _ptr(workspace, name="workspace"), int(workspace_bytes),
                                    _ptr(E, name="E"), _ptr(dE_dD, name="dE_dD")),
           "dpc_fitting_fwd_bwd")


# ---- routing and 8-bit layers: rows of any element type, with a row stride ----
_TORCH_ELEM = {} if torch is None else {torch.float64: DPC_ELEM_F64, torch.float32: DPC_ELEM_F32,
                                        torch.float16: DPC_ELEM_F16, torch.bfloat16: DPC_ELEM_BF16}


def elem_of(dtype):
    """The dpc_elem of a torch dtype."""
    e = _TORCH_ELEM.get(dtype)
    if e is None:
        raise TypeError(f"rows of {dtype} are not supported (float64, float32, float16, bfloat16)")
    return e


def i8_ld(cols):
    """Bytes of a row of codes (DPC_I8_LD in dpc.h)."""
    return (int(cols) + 127) // 128 * 128


_ELEM_TORCH = {e: t for t, e in _TORCH_ELEM.items()}


def _elem_dtype(elem, name="elem"):
    if int(elem) not in _ELEM_TORCH:
        raise DpcError(DPC_EINVAL, name)
    return _ELEM_TORCH[int(elem)]


def _rows_ptr(x, nrows, width, ld, dtype, name):
    """Address of the rows of a tensor: `nrows` rows of `width` elements, `ld`
    elements apart, which the tensor's storage has to hold (its own shape is not
    looked at).  An int is an address and taken as is."""
    if x is None or isinstance(x, int):
        return x
    if x.dtype != dtype:
        raise TypeError(f"{name} has dtype {x.dtype}, expected {dtype}")
    have = x.untyped_storage().nbytes() // x.element_size() - x.storage_offset()
    need = (int(nrows) - 1) * int(ld) + int(width) if nrows > 0 else 0
    if have < need:
        raise ValueError(f"{name} holds {have} elements, needs {need}")
    if not x.is_cuda:
        raise ValueError(f"{name} must be a tensor on a GPU device, not {x.device}")
    return x.data_ptr()


def _flat_ptr(x, count, dtype, name):
    """Address of a contiguous tensor of at least `count` elements."""
    if x is None or isinstance(x, int):
        return x
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return _rows_ptr(x, 1 if count > 0 else 0, count, count, dtype, name)


def _same_device(stream, **tensors):
    """Every tensor (and a torch stream) must be on one GPU."""
    devs = {k: v.device.index for k, v in tensors.items() if v is not None and not isinstance(v, int)}
    if stream is not None and not isinstance(stream, int) and hasattr(stream, "device"):
        devs["stream"] = stream.device.index
    if len(set(devs.values())) > 1:
        raise ValueError("arguments on different devices: " + ", ".join(f"{k}=cuda:{d}" for k, d in devs.items()))


def _wdtype(elem):
    return torch.float64 if int(elem) == DPC_ELEM_F64 else torch.float32


INT_MAX = 2 ** 31 - 1


def _sizes(where, *sizes):
    """Refuses sizes that are no C int: ctypes would drop their high bits, and the
    library would see a small size that passes its checks."""
    for v in sizes:
        if not -INT_MAX <= int(v) <= INT_MAX:
            raise DpcError(DPC_ENOTSUP if v > 0 else DPC_EINVAL, where)


def dpc_route_workspace_bytes(ntok, topk, nexpert):
    if max(ntok, topk, nexpert) > INT_MAX or min(ntok, topk, nexpert) < 0:
        return 0
    return int(_lib.dpc_route_workspace_bytes(int(ntok), int(topk), int(nexpert)))


def dpc_route_plan(stream, ntok, topk, nexpert, expert, workspace, workspace_bytes, offsets, rows, pos):
    _sizes("dpc_route_plan", ntok, topk, nexpert)
    m, i32 = int(ntok) * int(topk), torch.int32
    args = (_flat_ptr(expert, m, i32, "expert"), _flat_ptr(workspace, int(workspace_bytes), torch.uint8, "workspace"),
            int(workspace_bytes), _flat_ptr(offsets, int(nexpert) + 1, i32, "offsets"), _flat_ptr(rows, m, i32, "rows"),
            _flat_ptr(pos, m, i32, "pos"))
    _same_device(stream, expert=expert, workspace=workspace, offsets=offsets, rows=rows, pos=pos)
    _check(_lib.dpc_route_plan(_stream(stream), int(ntok), int(topk), int(nexpert), *args), "dpc_route_plan")


def dpc_route_gather(stream, elem, ntok, topk, width, x, ldx, weight, rows, pos, y, ldy):
    _sizes("dpc_route_gather", ntok, topk, width)
    m, dt = int(ntok) * int(topk), _elem_dtype(elem, "dpc_route_gather")
    args = (_rows_ptr(x, ntok, width, ldx, dt, "x"), int(ldx), _flat_ptr(weight, m, _wdtype(elem), "weight"),
            _flat_ptr(rows, m, torch.int32, "rows"), _flat_ptr(pos, m, torch.int32, "pos"),
            _rows_ptr(y, m, width, ldy, dt, "y"), int(ldy))
    _same_device(stream, x=x, weight=weight, rows=rows, pos=pos, y=y)
    _check(_lib.dpc_route_gather(_stream(stream), int(elem), int(ntok), int(topk), int(width), *args),
           "dpc_route_gather")


def dpc_route_combine(stream, elem, ntok, topk, width, x, ldx, weight, pos, y, ldy):
    _sizes("dpc_route_combine", ntok, topk, width)
    m, dt = int(ntok) * int(topk), _elem_dtype(elem, "dpc_route_combine")
    args = (_rows_ptr(x, m, width, ldx, dt, "x"), int(ldx), _flat_ptr(weight, m, _wdtype(elem), "weight"),
            _flat_ptr(pos, m, torch.int32, "pos"), _rows_ptr(y, ntok, width, ldy, dt, "y"), int(ldy))
    _same_device(stream, x=x, weight=weight, pos=pos, y=y)
    _check(_lib.dpc_route_combine(_stream(stream), int(elem), int(ntok), int(topk), int(width), *args),
           "dpc_route_combine")


def dpc_route_combine_bwd(stream, elem, ntok, topk, width, x, ldx, weight, rows, pos, dy, lddy, dx, lddx, dweight):
    _sizes("dpc_route_combine_bwd", ntok, topk, width)
    m, dt = int(ntok) * int(topk), _elem_dtype(elem, "dpc_route_combine_bwd")
    wt, i32 = _wdtype(elem), torch.int32
    args = (_rows_ptr(x, m, width, ldx, dt, "x"), int(ldx), _flat_ptr(weight, m, wt, "weight"),
            _flat_ptr(rows, m, i32, "rows"), _flat_ptr(pos, m, i32, "pos"), _rows_ptr(dy, ntok, width, lddy, dt, "dy"),
            int(lddy), _rows_ptr(dx, m, width, lddx, dt, "dx"), int(lddx), _flat_ptr(dweight, m, wt, "dweight"))
    _same_device(stream, x=x, weight=weight, rows=rows, pos=pos, dy=dy, dx=dx, dweight=dweight)
    _check(_lib.dpc_route_combine_bwd(_stream(stream), int(elem), int(ntok), int(topk), int(width), *args),
           "dpc_route_combine_bwd")


def dpc_quant_rows(stream, elem, nrows, ncols, x, ldx, q, scale):
    _sizes("dpc_quant_rows", nrows, ncols)
    dt = _elem_dtype(elem, "dpc_quant_rows")
    args = (_rows_ptr(x, nrows, ncols, ldx, dt, "x"), int(ldx),
            _flat_ptr(q, int(nrows) * i8_ld(ncols), torch.int8, "q"),
            _flat_ptr(scale, int(nrows), torch.float32, "scale"))
    _same_device(stream, x=x, q=q, scale=scale)
    _check(_lib.dpc_quant_rows(_stream(stream), int(elem), int(nrows), int(ncols), *args), "dpc_quant_rows")


def _layer_args(elem_y, ntok, topk, n, k, ngroup, rows, offsets, qw, sw, bias, y, ldy, where):
    _sizes(where, ntok, topk, n, k, ngroup)
    m, f32 = int(ntok) * int(topk), torch.float32
    head = (_flat_ptr(rows, m, torch.int32, "rows"), _flat_ptr(offsets, int(ngroup) + 1, torch.int32, "offsets"),
            _flat_ptr(qw, int(ngroup) * int(n) * i8_ld(k), torch.int8, "qw"),
            _flat_ptr(sw, int(ngroup) * int(n), f32, "sw"), _flat_ptr(bias, int(ngroup) * int(n), f32, "bias"))
    return head, (_rows_ptr(y, m, n, ldy, _elem_dtype(elem_y, where), "y"), int(ldy))


def dpc_matmul_i8(stream, elem_y, ntok, topk, n, k, ngroup, qx, sx, rows, offsets, qw, sw, bias, y, ldy):
    head, tail = _layer_args(elem_y, ntok, topk, n, k, ngroup, rows, offsets, qw, sw, bias, y, ldy, "dpc_matmul_i8")
    px = (_flat_ptr(qx, int(ntok) * i8_ld(k), torch.int8, "qx"), _flat_ptr(sx, int(ntok), torch.float32, "sx"))
    _same_device(stream, qx=qx, sx=sx, rows=rows, offsets=offsets, qw=qw, sw=sw, bias=bias, y=y)
    _check(_lib.dpc_matmul_i8(_stream(stream), int(elem_y), int(ntok), int(topk), int(n), int(k), int(ngroup), *px,
                              *head, *tail), "dpc_matmul_i8")


def dpc_linear_i8_workspace_bytes(ntok, k):
    if max(ntok, k) > INT_MAX or min(ntok, k) < 0:
        return 0
    return int(_lib.dpc_linear_i8_workspace_bytes(int(ntok), int(k)))


def dpc_linear_i8(stream, elem_x, elem_y, ntok, topk, n, k, ngroup, x, ldx, rows, offsets, qw, sw, bias, workspace,
                  workspace_bytes, y, ldy):
    head, tail = _layer_args(elem_y, ntok, topk, n, k, ngroup, rows, offsets, qw, sw, bias, y, ldy, "dpc_linear_i8")
    px = _rows_ptr(x, ntok, k, ldx, _elem_dtype(elem_x, "dpc_linear_i8"), "x")
    pw = _flat_ptr(workspace, int(workspace_bytes), torch.uint8, "workspace")
    _same_device(stream, x=x, rows=rows, offsets=offsets, qw=qw, sw=sw, bias=bias, workspace=workspace, y=y)
    _check(_lib.dpc_linear_i8(_stream(stream), int(elem_x), int(elem_y), int(ntok), int(topk), int(n), int(k),
                              int(ngroup), px, int(ldx), *head, pw, int(workspace_bytes), *tail), "dpc_linear_i8")


class RocblasHandle:
    """A rocBLAS handle for dpc_fitting_fwd_bwd, created and destroyed through
    librocblas (the caller owns it; the library leaves its stream set to the
    call's and restores its pointer mode)."""

    def __init__(self):
        self._rb = C.CDLL("librocblas.so.5")
        self._rb.rocblas_create_handle.argtypes = [C.POINTER(C.c_void_p)]
        self._rb.rocblas_destroy_handle.argtypes = [C.c_void_p]
        h = C.c_void_p()
        if self._rb.rocblas_create_handle(C.byref(h)) != 0:
            raise RuntimeError("rocblas_create_handle failed")
        self.value = h.value

    def pointer_mode(self):
        """0 = host, 1 = device (rocblas_pointer_mode)."""
        m = C.c_int()
        self._rb.rocblas_get_pointer_mode.argtypes = [C.c_void_p, C.POINTER(C.c_int)]
        if self._rb.rocblas_get_pointer_mode(C.c_void_p(self.value), C.byref(m)) != 0:
            raise RuntimeError("rocblas_get_pointer_mode failed")
        return m.value

    def set_pointer_mode(self, mode):
        self._rb.rocblas_set_pointer_mode.argtypes = [C.c_void_p, C.c_int]
        if self._rb.rocblas_set_pointer_mode(C.c_void_p(self.value), int(mode)) != 0:
            raise RuntimeError("rocblas_set_pointer_mode failed")

    def close(self):
        if self.value:
            self._rb.rocblas_destroy_handle(C.c_void_p(self.value))
            self.value = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
