"""ctypes binding of the C ABI declared in include/spt.h (same names).

PyTorch is used for device memory and streams only. `DeviceTensor` uploads the
level arrays of a format description (any object with .dims, .levels[] having
kind/mode/N/M/pos/crd/offset/ordered/unique, and .vals) and packs the pointers
into an spt_tensor struct.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_SO = os.path.join(_HERE, "libspt.so")
_lib = None

SPT_OK, SPT_ERR_INVALID_ARG, SPT_ERR_UNSUPPORTED, SPT_ERR_WORKSPACE, SPT_ERR_DEVICE = range(5)
SPT_OP_SPMV, SPT_OP_COO_TO_CSR, SPT_OP_TTV, SPT_OP_MTTKRP, SPT_OP_INNERPROD, SPT_OP_TTM = range(6)
SPT_OP_TO_CSF, SPT_OP_TO_ELL, SPT_OP_DIA_OFFSETS, SPT_OP_TO_COO = 6, 7, 8, 9
SPT_OP_SPMV_SPARSE_X, SPT_OP_SPDM = 10, 11
SPT_ORDER_ROW_COL, SPT_ORDER_ROW_STABLE = 0, 1
SPT_ORDERED, SPT_UNIQUE = 1, 2
SPT_F32, SPT_F64, SPT_F16, SPT_BF16 = range(4)
SPT_CACHE_EXTEND, SPT_CACHE_ATTENTION = 0, 1
SPT_STATIC_SCRATCH_BYTES = 4 << 20

SYMBOLS = ["spt_spmv", "spt_coo_to_csr", "spt_ttv", "spt_mttkrp", "spt_workspace_bytes",
           "spt_last_error", "spt_version", "spt_probe_read", "spt_probe_gather",
           "spt_spmv_sparse_x", "spt_spdm", "spt_innerprod", "spt_ttm",
           "spt_add", "spt_mul", "spt_add_workspace_bytes", "spt_mul_dense", "spt_add_to_dense", "spt_coo3_to_csf", "spt_to_ell",
           "spt_coo_dia_offsets", "spt_coo_to_dia", "spt_to_coo", "spt_to_hashed_rows", "spt_spmv_static", "spt_validate",
           "spt_cache_extend", "spt_cache_write", "spt_cache_compact", "spt_cache_free", "spt_cache_fork",
           "spt_cache_attention", "spt_cache_workspace_bytes", "spt_adjust_logits"]


class SptLevel(C.Structure):
    _fields_ = [("kind", C.c_int32), ("mode", C.c_int32), ("flags", C.c_int32),
                ("max_children", C.c_int32), ("N", C.c_int64), ("M", C.c_int64),
                ("pos", C.c_void_p), ("crd", C.c_void_p), ("offset", C.c_void_p),
                ("crd_stride", C.c_int64)]


class SptTensor(C.Structure):
    _fields_ = [("order", C.c_int32), ("nlevels", C.c_int32), ("dtype", C.c_int32),
                ("reserved", C.c_int32), ("level", SptLevel * 4), ("vals", C.c_void_p),
                ("nvals", C.c_int64)]


class SptCache(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "layers", "heads", "width", "page", "rows", "row_pages", "reserved")]
                + [(n, C.c_int64) for n in ("pages", "layer_stride", "page_stride", "slot_stride", "head_stride")]
                + [(n, C.c_void_p) for n in ("K", "V", "table", "len", "refs")])


class SptLogitRules(C.Structure):
    _fields_ = [("first", C.c_void_p), ("sequences", C.c_int64), ("seen", C.c_void_p), ("tree", C.c_void_p),
                ("drafts", C.c_void_p), ("repetition", C.c_void_p), ("presence", C.c_void_p), ("frequency", C.c_void_p),
                ("bias", C.c_void_p), ("allowed", C.c_void_p), ("allowed_stride", C.c_int64)]


class SptError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"spt status {status}: {message}")
        self.status = status


def library_path() -> str:
    return _SO


def lib():
    """Loads libspt.so; builds it first only if it has never been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_SO):
            from . import build as _build
            _build.build()
        L = C.CDLL(_SO)
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        L.spt_spmv.restype = i32
        L.spt_spmv.argtypes = [vp, vp, vp, vp, sz, vp]
        L.spt_validate.restype = i32
        L.spt_validate.argtypes = [vp, vp, vp]
        L.spt_spmv_static.restype = i32
        L.spt_spmv_static.argtypes = [vp, vp, vp, vp]
        L.spt_spmv_sparse_x.restype = i32
        L.spt_spmv_sparse_x.argtypes = [vp, vp, vp, vp, sz, vp]
        L.spt_coo_to_csr.restype = i32
        L.spt_coo_to_csr.argtypes = [vp, i32, vp, vp, vp, vp, sz, vp]
        L.spt_ttv.restype = i32
        L.spt_ttv.argtypes = [vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.spt_mttkrp.restype = i32
        L.spt_mttkrp.argtypes = [vp, vp, vp, i32, vp, vp, sz, vp]
        L.spt_coo3_to_csf.restype = i32
        L.spt_coo3_to_csf.argtypes = [vp] * 10 + [sz, vp]
        L.spt_to_ell.restype = i32
        L.spt_to_ell.argtypes = [vp, i32, vp, vp, vp, vp, sz, vp]
        L.spt_coo_dia_offsets.restype = i32
        L.spt_coo_dia_offsets.argtypes = [vp, vp, C.c_int64, vp, vp, sz, vp]
        L.spt_coo_to_dia.restype = i32
        L.spt_coo_to_dia.argtypes = [vp, i32, vp, vp, vp]
        L.spt_to_hashed_rows.restype = i32
        L.spt_to_hashed_rows.argtypes = [vp, i32, vp, vp, vp, vp]
        L.spt_to_coo.restype = i32
        L.spt_to_coo.argtypes = [vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.spt_add.restype = i32
        L.spt_add.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.spt_mul.restype = i32
        L.spt_mul.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.spt_mul_dense.restype = i32
        L.spt_mul_dense.argtypes = [vp, vp, C.c_int64, vp, vp]
        L.spt_add_to_dense.restype = i32
        L.spt_add_to_dense.argtypes = [vp, vp, vp, C.c_int64, vp]
        L.spt_add_workspace_bytes.restype = sz
        L.spt_add_workspace_bytes.argtypes = [vp, vp]
        L.spt_ttm.restype = i32
        L.spt_ttm.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.spt_innerprod.restype = i32
        L.spt_innerprod.argtypes = [vp, vp, vp, vp, sz, vp]
        L.spt_spdm.restype = i32
        L.spt_spdm.argtypes = [vp, vp, i32, vp, vp, sz, vp]
        L.spt_workspace_bytes.restype = sz
        L.spt_workspace_bytes.argtypes = [i32, vp, i32]
        L.spt_last_error.restype = C.c_char_p
        L.spt_last_error.argtypes = []
        L.spt_version.restype = C.c_char_p
        L.spt_version.argtypes = []
        L.spt_probe_read.restype = i32
        L.spt_probe_read.argtypes = [vp, sz, i32, vp, vp]
        L.spt_probe_gather.restype = i32
        L.spt_probe_gather.argtypes = [vp, C.c_int64, vp, i32, vp, vp]
        i64 = C.c_int64
        L.spt_cache_extend.argtypes = [vp, vp, vp, vp, sz, vp]
        L.spt_cache_write.argtypes = [vp, i32, vp, i64, vp, vp, i64, i64, vp]
        L.spt_cache_compact.argtypes = [vp, vp, vp, vp]
        L.spt_cache_free.argtypes = [vp, vp, vp]
        L.spt_cache_fork.argtypes = [vp, i64, vp, vp, vp]
        L.spt_cache_attention.argtypes = [vp, i32, vp, i64, vp, vp, i32, i64, i64, C.c_float, vp, i64, i64, vp, vp, sz, vp]
        L.spt_adjust_logits.argtypes = [i32, i64, i64, vp, i64, vp, vp, i64, vp]
        for name in ("extend", "write", "compact", "free", "fork", "attention"):
            getattr(L, "spt_cache_" + name).restype = i32
        L.spt_adjust_logits.restype = i32
        L.spt_cache_workspace_bytes.restype = sz
        L.spt_cache_workspace_bytes.argtypes = [i32, vp, i32]
        _lib = L
    return _lib


def spt_last_error() -> str:
    return lib().spt_last_error().decode()


def spt_version() -> str:
    return lib().spt_version().decode()


def _check(status):
    if status != SPT_OK:
        raise SptError(status, spt_last_error())


def _p(t):
    """Device pointer of a torch tensor (None -> NULL)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _desc(T):
    return C.addressof(T.c) if isinstance(T, (DeviceTensor, DeviceCSR)) else C.addressof(T)


_raw_stream = _device = None


def _current_stream():
    """torch's current stream as an integer (None without a GPU). Asking through the torch.cuda
    module costs 3.3 us, a kernel launch's worth, so once it is initialised the two C functions
    behind it are called directly (0.15 us)."""
    global _raw_stream, _device
    if _raw_stream is not None:
        return _raw_stream(_device())
    import torch
    if not torch.cuda.is_available():
        return None
    stream = torch.cuda.current_stream().cuda_stream
    _device, _raw_stream = (getattr(torch._C, n, None) for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))
    if _device is None:
        _raw_stream = None
    return stream


def _stream(stream):
    """hipStream_t as an integer; None = torch's current stream (null stream without a GPU)."""
    if stream is None:
        return _current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def _ws(ws):
    if ws is None or isinstance(ws, int):
        return None, 0
    return ws.data_ptr(), ws.nbytes


def spt_workspace_bytes(op, T, J=0) -> int:
    n = lib().spt_workspace_bytes(op, _desc(T), J)
    if n == 0:
        raise SptError(SPT_ERR_INVALID_ARG, spt_last_error())
    return n


def spt_spmv(A, x, y, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_spmv(_desc(A), _p(x), _p(y), p, n, _stream(stream)))


SPT_BAD_POS, SPT_BAD_POS_END, SPT_BAD_CRD, SPT_BAD_ORDER, SPT_BAD_OFFSET = 1, 2, 4, 8, 16


def spt_validate(T, err_dev, stream=None):
    _check(lib().spt_validate(_desc(T), _p(err_dev), _stream(stream)))


def spt_spmv_static(A, x, y, stream=None):
    _check(lib().spt_spmv_static(_desc(A), _p(x), _p(y), _stream(stream)))


def spt_spmv_sparse_x(A, x, y, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_spmv_sparse_x(_desc(A), _desc(x), _p(y), p, n, _stream(stream)))


def spt_coo_to_csr(A, order, pos_out, crd_out, vals_out, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_coo_to_csr(_desc(A), order, _p(pos_out), _p(crd_out), _p(vals_out), p, n,
                                _stream(stream)))


def spt_ttv(B, c, out_crd0, out_crd1, out_vals, out_nnz_dev, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_ttv(_desc(B), _p(c), _p(out_crd0), _p(out_crd1), _p(out_vals),
                         _p(out_nnz_dev), p, n, _stream(stream)))


def spt_mttkrp(B, Cm, Dm, J, A_out, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_mttkrp(_desc(B), _p(Cm), _p(Dm), J, _p(A_out), p, n, _stream(stream)))


def spt_probe_read(src, nbytes, lane_bytes, sink, stream=None):
    _check(lib().spt_probe_read(_p(src), nbytes, lane_bytes, _p(sink), _stream(stream)))


def spt_probe_gather(idx, n, table, dtype, out, stream=None):
    _check(lib().spt_probe_gather(_p(idx), n, _p(table), dtype, _p(out), _stream(stream)))


def spt_spdm(B, Cm, J, A_out, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_spdm(_desc(B), _p(Cm), J, _p(A_out), p, n, _stream(stream)))


def spt_ttm(B, Cm, K, out_crd0, out_crd1, out_vals, out_nfib_dev, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_ttm(_desc(B), _p(Cm), K, _p(out_crd0), _p(out_crd1), _p(out_vals),
                         _p(out_nfib_dev), p, n, _stream(stream)))


def spt_coo3_to_csf(B, pos0, crd0, pos1, crd1, pos2, crd2, vals_out, counts_dev, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_coo3_to_csf(_desc(B), _p(pos0), _p(crd0), _p(pos1), _p(crd1), _p(pos2), _p(crd2),
                                 _p(vals_out), _p(counts_dev), p, n, _stream(stream)))


def spt_to_ell(A, W, crd_out, vals_out, longest_dev, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_to_ell(_desc(A), W, _p(crd_out), _p(vals_out), _p(longest_dev), p, n,
                            _stream(stream)))


def spt_coo_dia_offsets(A, offsets_out, cap, K_dev, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_coo_dia_offsets(_desc(A), _p(offsets_out), cap, _p(K_dev), p, n, _stream(stream)))


def spt_coo_to_dia(A, K, offsets, vals_out, stream=None):
    _check(lib().spt_coo_to_dia(_desc(A), K, _p(offsets), _p(vals_out), _stream(stream)))


def spt_to_hashed_rows(A, W, crd_out, vals_out, dropped_dev, stream=None):
    _check(lib().spt_to_hashed_rows(_desc(A), W, _p(crd_out), _p(vals_out), _p(dropped_dev),
                                    _stream(stream)))


def spt_to_coo(T, out_crd0, out_crd1, out_crd2, out_vals, out_nnz_dev, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_to_coo(_desc(T), _p(out_crd0), _p(out_crd1), _p(out_crd2), _p(out_vals),
                            _p(out_nnz_dev), p, n, _stream(stream)))


def spt_add(B, Ct, out_pos, out_crd0, out_crd1, out_crd2, out_vals, out_nnz_dev, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_add(_desc(B), _desc(Ct), _p(out_pos), _p(out_crd0), _p(out_crd1), _p(out_crd2),
                         _p(out_vals), _p(out_nnz_dev), p, n, _stream(stream)))


def spt_mul(B, Ct, out_pos, out_crd0, out_crd1, out_crd2, out_vals, out_nnz_dev, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_mul(_desc(B), _desc(Ct), _p(out_pos), _p(out_crd0), _p(out_crd1), _p(out_crd2),
                         _p(out_vals), _p(out_nnz_dev), p, n, _stream(stream)))


def spt_mul_dense(B, D, ld, out_vals, stream=None):
    _check(lib().spt_mul_dense(_desc(B), _p(D), ld, _p(out_vals), _stream(stream)))


def spt_add_to_dense(B, Ct, A, ld, stream=None):
    _check(lib().spt_add_to_dense(_desc(B), _desc(Ct), _p(A), ld, _stream(stream)))


def spt_add_workspace_bytes(B, Ct):
    n = lib().spt_add_workspace_bytes(_desc(B), _desc(Ct))
    if n == 0:
        raise SptError(SPT_ERR_INVALID_ARG, spt_last_error())
    return n


def spt_innerprod(B, Ct, alpha_out, ws=None, stream=None):
    p, n = _ws(ws)
    _check(lib().spt_innerprod(_desc(B), _desc(Ct), _p(alpha_out), p, n, _stream(stream)))


class DeviceTensor:
    """spt_tensor descriptor whose level arrays live in device memory."""

    def __init__(self, spec, device="cuda:0", misalign=False):
        """misalign=True places every array one element past a 256-byte boundary
        (exercises the kernels' paths for buffers that are not 16-byte aligned)."""
        import torch
        self.spec = spec
        self.device = device
        self.keep = []
        t = SptTensor()
        t.order = len(spec.dims)
        t.nlevels = len(spec.levels)
        vals = np.ascontiguousarray(spec.vals)
        if vals.dtype == np.float64:
            t.dtype = SPT_F64
        elif vals.dtype == np.float32:
            t.dtype = SPT_F32
        else:
            raise TypeError(f"values must be float32 or float64, got {vals.dtype}")
        shared = {}
        for k, lv in enumerate(spec.levels):
            o = t.level[k]
            o.kind, o.mode, o.N, o.M = int(lv.kind), int(lv.mode), int(lv.N), int(lv.M)
            o.flags = (SPT_ORDERED if lv.ordered else 0) | (SPT_UNIQUE if lv.unique else 0)
            o.max_children = int(getattr(lv, "max_children", 0))
            o.crd_stride = int(getattr(lv, "crd_stride", 1))
            for name in ("pos", "crd", "offset"):
                a = getattr(lv, name)
                if a is None:
                    continue
                if name == "crd" and o.crd_stride > 1 and a.base is not None:
                    # interleaved coordinates: the levels are views into one array, which is
                    # uploaded once; each level points at its own first element of it
                    base = a.base
                    if id(base) not in shared:
                        d = self._upload(np.ascontiguousarray(base, dtype=np.int32).reshape(-1), device, misalign)
                        shared[id(base)] = d
                        self.keep.append(d)
                        setattr(self, "crd_interleaved", d)
                    off = a.__array_interface__["data"][0] - base.__array_interface__["data"][0]
                    o.crd = shared[id(base)].data_ptr() + off
                    continue
                if id(a) not in shared:   # DIA shares one offset array between two levels
                    d = self._upload(np.ascontiguousarray(a, dtype=np.int32), device, misalign)
                    shared[id(a)] = d
                    self.keep.append(d)
                    setattr(self, f"{name}{k}", d)
                setattr(o, name, shared[id(a)].data_ptr())
        self.vals = self._upload(vals, device, misalign)
        t.vals = self.vals.data_ptr()
        t.nvals = vals.size
        self.torch_dtype = self.vals.dtype
        self.c = t

    @staticmethod
    def _upload(a, device, misalign):
        import torch
        if not misalign:
            return torch.from_numpy(a).to(device)
        buf = torch.empty(a.size + 1, dtype=torch.from_numpy(a).dtype, device=device)
        buf[1:].copy_(torch.from_numpy(a))
        return buf[1:]

    def workspace(self, op, J=0):
        import torch
        n = spt_workspace_bytes(op, self, J)
        return torch.empty(n, dtype=torch.uint8, device=self.device)


def _invalid(message):
    raise SptError(SPT_ERR_INVALID_ARG, message)


_codes = {}


def _dtype_code(dtype):
    if not _codes:
        import torch
        _codes.update({torch.float32: SPT_F32, torch.float64: SPT_F64, torch.float16: SPT_F16, torch.bfloat16: SPT_BF16})
    if dtype not in _codes:
        raise TypeError(f"values must be float32, float16 or bfloat16, got {dtype}")
    return _codes[dtype]


_int32 = None   # torch.int32, once a descriptor has imported torch: an import statement in a call costs a tenth of it


def _use_torch():
    global _int32
    import torch
    _int32 = torch.int32
    return torch


def _on_device(t, device, name):
    if t.get_device() != device:
        _invalid(f"{name} is on another device than the rest")


def _stream_of(device, stream):
    """As _stream, for tensors that all lie on `device`: refused are tensors on the host, torch's current stream where another device
    is the current one, and a stream of torch's that belongs to another device (a plain handle does not say to which it belongs)."""
    if device < 0:
        _invalid("the tensors are not on a GPU")
    if stream is not None:
        if getattr(stream, "device_index", device) != device:
            _invalid(f"the tensors are on device {device}, the stream is of device {stream.device_index}")
        return _stream(stream)
    handle = _current_stream()  # finds out how to ask for the current device, in a process's first call
    if _device is not None and _device() != device:
        _invalid(f"the tensors are on device {device}, the current device is {_device()}")
    return handle


def _i32(t, count, name, device=None):
    """Pointer of a contiguous int32 tensor of at least `count` entries, on `device` if that is given (None -> NULL)."""
    if t is None:
        return None
    if t.dtype is not _int32 or t.numel() < count or not t.is_contiguous():
        _invalid(f"{name} must be a contiguous int32 tensor of at least {count} entries")
    if device is not None:
        _on_device(t, device, name)
    return t.data_ptr()


def _matrix_device(m):
    """The device of a sparse matrix, None of a plain descriptor, which does not say it."""
    return m.device if isinstance(m, DeviceCSR) else m.vals.get_device() if isinstance(m, DeviceTensor) else None


def _matrix(m, device, name):
    """Descriptor of a sparse matrix that lies on `device` (None -> NULL)."""
    if m is None:
        return None
    if _matrix_device(m) not in (device, None):
        _invalid(f"{name} is on another device than the rest")
    return _desc(m)


def _ws_on(ws, device):
    if ws is not None and not isinstance(ws, int):
        _on_device(ws, device, "the workspace")
    return _ws(ws)


def _stride(t, d):
    """A stride, 0 where it is never used (torch leaves those of a dimension of one or none as they come)."""
    return t.stride(d) if t.shape[d] > 1 else 0


class DeviceCSR:
    """spt_tensor descriptor of a CSR matrix whose arrays are device tensors already: pos (rows + 1 entries) and crd int32,
    vals float32 or float64; without vals a pattern."""

    def __init__(self, pos, crd, cols, vals=None, ordered=False, unique=False):
        _use_torch()
        rows = pos.numel() - 1
        t = SptTensor()
        t.order = t.nlevels = 2
        t.dtype = SPT_F32 if vals is None else _dtype_code(vals.dtype)
        t.level[0].kind, t.level[0].mode, t.level[0].N, t.level[0].flags = 0, 0, rows, SPT_ORDERED | SPT_UNIQUE
        o = t.level[1]
        o.kind, o.mode, o.N, o.M = 1, 1, int(cols), rows
        o.flags = (SPT_ORDERED if ordered else 0) | (SPT_UNIQUE if unique else 0)
        self.device = pos.get_device()
        o.pos, o.crd = _i32(pos, 1, "pos"), _i32(crd, 0, "crd", self.device)
        if vals is not None:
            if vals.numel() != crd.numel() or not vals.is_contiguous():
                _invalid("vals must be contiguous, one value for each entry of crd")
            _on_device(vals, self.device, "vals")
        t.vals, t.nvals = _p(vals), crd.numel()
        self.keep = (pos, crd, vals)
        self.c = t


class DeviceCache:
    """spt_cache descriptor of device tensors: K and V (layers, pages, slots of a page, heads, width) in any strides with
    contiguous values of a head, table (rows, pages of a row), len (rows) and refs (pages), int32 and contiguous."""

    def __init__(self, K, V, table, length, refs):
        _use_torch()
        if K.dim() != 5 or K.shape != V.shape or K.dtype != V.dtype:
            _invalid("K and V must be alike: (layers, pages, slots of a page, heads, width)")
        strides = [_stride(K, d) for d in range(4)]
        if strides != [_stride(V, d) for d in range(4)]:
            _invalid("K and V must have the same strides")
        if K.stride(4) != 1 or V.stride(4) != 1:
            _invalid("the values of a head must be contiguous")
        if table.dim() != 2:
            _invalid("table must be (rows, pages of a row)")
        c = SptCache()
        c.dtype = _dtype_code(K.dtype)
        c.layers, c.pages, c.page, c.heads, c.width = K.shape
        c.rows, c.row_pages = table.shape
        c.layer_stride, c.page_stride, c.slot_stride, c.head_stride = strides
        c.K, c.V = K.data_ptr(), V.data_ptr()
        c.table, c.len, c.refs = _i32(table, 0, "table"), _i32(length, c.rows, "len"), _i32(refs, c.pages, "refs")
        self.K, self.V, self.table, self.len, self.refs = K, V, table, length, refs
        self.c, self.address = c, C.addressof(c)
        self.rows, self.heads, self.width, self.dtype, self.device = c.rows, c.heads, c.width, K.dtype, K.get_device()
        for t, name in ((V, "V"), (table, "table"), (length, "len"), (refs, "refs")):
            _on_device(t, self.device, name)

    def workspace(self, op, q_heads=0):
        import torch
        return torch.empty(spt_cache_workspace_bytes(op, self, q_heads), dtype=torch.uint8, device=self.K.device)

    def _tokens(self, t, name, heads):
        """(tokens, heads, width) of the cache's dtype: token and head strides."""
        shape, stride = t.shape, t.stride()
        if t.dtype is not self.dtype or len(shape) != 3 or shape[2] != self.width or shape[1] != heads or stride[2] != 1:
            _invalid(f"{name} must be (tokens, {heads}, {self.width}), {self.dtype}, values of a head contiguous")
        _on_device(t, self.device, name)
        return (stride[0] if shape[0] > 1 else 0), (stride[1] if heads > 1 else 0)


def spt_cache_workspace_bytes(op, cache, q_heads=0) -> int:
    n = lib().spt_cache_workspace_bytes(op, cache.address, q_heads)
    if n == 0:
        raise SptError(SPT_ERR_INVALID_ARG, spt_last_error())
    return n


def spt_cache_extend(cache, add, refused_dev, ws=None, stream=None):
    device = cache.device
    p, n = _ws_on(ws, device)
    _check(lib().spt_cache_extend(cache.address, _i32(add, cache.rows, "add", device), _i32(refused_dev, 1, "refused_dev", device), p, n,
                                  _stream_of(device, stream)))


def spt_cache_write(cache, layer, first, k, v, stream=None):
    token, head = cache._tokens(k, "k", cache.heads)
    tokens = k.shape[0]
    if cache._tokens(v, "v", cache.heads) != (token, head) or v.shape[0] != tokens:
        _invalid("k and v must be alike")
    device = cache.device
    _check(lib().spt_cache_write(cache.address, layer, _i32(first, cache.rows + 1, "first", device), tokens, k.data_ptr(), v.data_ptr(),
                                 token, head, _stream_of(device, stream)))


def spt_cache_compact(cache, first, keep, stream=None):
    device = cache.device
    _check(lib().spt_cache_compact(cache.address, _i32(first, cache.rows + 1, "first", device), _matrix(keep, device, "keep"),
                                   _stream_of(device, stream)))


def spt_cache_free(cache, new_len, stream=None):
    device = cache.device
    _check(lib().spt_cache_free(cache.address, _i32(new_len, cache.rows, "new_len", device), _stream_of(device, stream)))


def spt_cache_fork(cache, parents, children, stream=None):
    n, device = children.numel(), cache.device
    _check(lib().spt_cache_fork(cache.address, n, _i32(parents, n, "parents", device), _i32(children, n, "children", device),
                                _stream_of(device, stream)))


def spt_cache_attention(cache, layer, first, tree, q, scale, out, lse=None, ws=None, stream=None):
    """q, out: (tokens, q_heads, width); tree: DeviceCSR or None; lse: float32 (tokens, q_heads), contiguous, or None."""
    shape = q.shape
    heads = shape[1] if len(shape) == 3 else 0
    q_token, q_head = cache._tokens(q, "q", heads)
    out_token, out_head = cache._tokens(out, "out", heads)
    if out.shape != shape:
        _invalid("q and out have different numbers of tokens")
    device = cache.device
    if lse is not None:
        if lse.shape != shape[:2] or lse.element_size() != 4 or not lse.is_floating_point() or not lse.is_contiguous():
            _invalid("lse must be float32, (tokens, q_heads), contiguous")
        _on_device(lse, device, "lse")
    p, n = _ws_on(ws, device)
    _check(lib().spt_cache_attention(cache.address, layer, _i32(first, cache.rows + 1, "first", device), shape[0],
                                     _matrix(tree, device, "tree"), q.data_ptr(), heads, q_token, q_head, scale, out.data_ptr(), out_token,
                                     out_head, _p(lse), p, n, _stream_of(device, stream)))


class LogitRules:
    """spt_logit_rules of device tensors and DeviceCSR matrices; the number of sequences follows from first, else from what is
    given for each sequence."""

    def __init__(self, first=None, seen=None, tree=None, drafts=None, repetition=None, presence=None, frequency=None, bias=None,
                 allowed=None, sequences=None):
        torch = _use_torch()
        per_sequence = [t for t in (repetition, presence, frequency) if t is not None]
        if sequences is None:
            counts = ([first.numel() - 1] if first is not None else []) + [m.c.level[0].N for m in (seen, bias) if m is not None]
            counts += [t.numel() for t in per_sequence]
            if not counts:
                _invalid("the number of sequences is not given")
            sequences = counts[0]
        for t in per_sequence:
            if t.dtype != torch.float32 or not t.is_contiguous() or t.numel() < sequences:
                _invalid(f"repetition, presence and frequency must be contiguous float32 tensors of {sequences} entries")
        if allowed is not None:
            if allowed.dtype not in (torch.int32, torch.uint32) or allowed.dim() != 2:
                _invalid("allowed must be (rows, words) of 32 bits")
            rows, words = allowed.shape
            # one mask for all rows (expand) has stride 0, which no rule has: it would be read as rows side by side
            if (words > 1 and allowed.stride(1) != 1) or (rows > 1 and allowed.stride(0) < words):
                _invalid("the words of a row of allowed must be contiguous, its rows apart")
        devices = {t.get_device() for t in (first, drafts, *per_sequence, allowed) if t is not None}
        devices |= {_matrix_device(m) for m in (seen, tree, bias) if m is not None} - {None}
        if len(devices) > 1:
            _invalid("the rules are on several devices")
        self.device = devices.pop() if devices else None
        r = SptLogitRules()
        r.first, r.sequences = _i32(first, sequences + 1, "first"), sequences
        r.seen, r.tree, r.bias = (m and _desc(m) for m in (seen, tree, bias))
        r.drafts = _i32(drafts, 0, "drafts")
        r.repetition, r.presence, r.frequency = _p(repetition), _p(presence), _p(frequency)
        if allowed is not None:
            r.allowed, r.allowed_stride = allowed.data_ptr(), allowed.stride(0) if rows > 1 else words
        self.keep = (first, seen, tree, drafts, repetition, presence, frequency, bias, allowed)
        self.rows = min([t.shape[0] for t in (drafts, allowed) if t is not None], default=None)
        self.columns = None if allowed is None else 32 * words
        self.c, self.address = r, C.addressof(r)


def spt_adjust_logits(logits, rules, out, stream=None):
    """logits, out: (rows, vocabulary) of one dtype, values of a row contiguous; they may be the same tensor."""
    shape, dtype = logits.shape, logits.dtype
    if len(shape) != 2 or out.shape != shape or out.dtype is not dtype:
        _invalid("logits and out must be alike: (rows, vocabulary)")
    R, V = shape
    (stride, inner), (out_stride, out_inner) = logits.stride(), out.stride()
    if V > 1 and (inner != 1 or out_inner != 1):
        _invalid("the values of a row of logits and out must be contiguous")
    if R <= 1:
        stride = out_stride = V
    device = logits.get_device()
    _on_device(out, device, "out")
    if rules.device is not None and rules.device != device:
        _invalid("the rules are on another device than the logits")
    if rules.rows is not None and rules.rows < R:
        _invalid("drafts or allowed have fewer rows than logits")
    if rules.columns is not None and rules.columns < V:
        _invalid(f"allowed has {rules.columns // 32} words a row, {V} logits need {(V + 31) // 32}")
    _check(lib().spt_adjust_logits(_dtype_code(dtype), R, V, logits.data_ptr(), stride, rules.address, out.data_ptr(), out_stride,
                                   _stream_of(device, stream)))
