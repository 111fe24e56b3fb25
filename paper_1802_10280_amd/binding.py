"""ctypes binding of libescoin.so: the same names as the C ABI, argument marshalling only.

Host arguments are numpy arrays, device arguments are torch CUDA tensors (PyTorch supplies
device memory and streams, nothing else); every step of the path runs inside the library.
There is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libescoin.so")

OK, EINVAL, ERANGE, EHIP, ESIZE = 0, -1, -2, -3, -4
F_BIAS, F_RELU = 1, 2
F_RESIDUAL, F_SILU, F_GELU, F_GELU_TANH = 4, 8, 16, 32
T_F32, T_F16, T_BF16 = 0, 1, 2
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2


class escoin_conv_desc(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("N", "C", "H", "W", "M", "R", "S", "stride", "pad")]


class escoin_sconv_tuning(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("K", "Q", "B", "WM", "CC", "NB", "TH", "CS", "WS", "CC0")]


class escoin_linear_desc(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int32) for k in ("T", "K", "M", "type", "gated")]
                + [(k, ctypes.c_int64) for k in ("ld_in", "ld_out", "ld_residual")])


class escoin_linear_kernel_info(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("kept", "rows", "tokens", "waves", "inputs", "pieces", "lane_words", "steps", "step_bytes", "lds_bytes")]


class escoin_norm_desc(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int32) for k in ("T", "D", "type", "post", "pre", "gate_rows")]
                + [(k, ctypes.c_float) for k in ("eps", "alpha", "beta", "weight_offset")]
                + [(k, ctypes.c_int64) for k in ("ld_x", "ld_y", "ld_gate", "ld_h", "ld_n")])


class EscoinError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


_lib = None


def lib() -> ctypes.CDLL:
    """Loads the HIP library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_1802_10280_amd.build` "
                "(or __graft_entry__.build()); there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        D = ctypes.POINTER(escoin_conv_desc)
        vp, i32p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32)
        L.escoin_strerror.restype = ctypes.c_char_p
        L.escoin_strerror.argtypes = [ctypes.c_int]
        L.escoin_check_desc.argtypes = [D]
        L.escoin_output_dims.argtypes = [D, i32p, i32p]
        L.escoin_padded_elems.restype = ctypes.c_size_t
        L.escoin_padded_elems.argtypes = [D]
        L.escoin_output_elems.restype = ctypes.c_size_t
        L.escoin_output_elems.argtypes = [D]
        L.escoin_sconv_pack.argtypes = [D, vp, vp, vp]
        L.escoin_pad_in.argtypes = [D, vp, vp, vp]
        L.escoin_sconv_forward.argtypes = [D, vp, vp, vp, vp, vp, vp, ctypes.c_uint32, vp]
        T = ctypes.POINTER(escoin_sconv_tuning)
        L.escoin_sconv_plan_size.argtypes = [D, vp, vp, T, ctypes.POINTER(ctypes.c_size_t)]
        L.escoin_sconv_plan_build.argtypes = [D, vp, vp, vp, T, vp, ctypes.c_size_t]
        L.escoin_sconv_forward_tiled.argtypes = [D, vp, vp, vp, vp, vp, ctypes.c_uint32, vp]
        L.escoin_sconv_tiled_on_matrix_cores.argtypes = [D, vp]
        L.escoin_sconv_tiled_kernel.argtypes = [D, vp]
        LD, ND = ctypes.POINTER(escoin_linear_desc), ctypes.POINTER(escoin_norm_desc)
        L.escoin_linear_check_desc.argtypes = [LD]
        L.escoin_linear_plan_size.argtypes = [LD, vp, vp, ctypes.POINTER(ctypes.c_size_t)]
        L.escoin_linear_plan_build.argtypes = [LD, vp, vp, vp, vp, ctypes.c_size_t]
        L.escoin_linear_forward.argtypes = [LD, vp, vp, vp, vp, vp, vp, ctypes.c_uint32, vp]
        L.escoin_linear_few_tokens.argtypes = [LD, vp]
        L.escoin_linear_kernel.argtypes = [LD, vp, vp, ctypes.POINTER(escoin_linear_kernel_info)]
        L.escoin_norm_check_desc.argtypes = [ND]
        L.escoin_norm_forward.argtypes = [ND, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        _lib = L
    return _lib


def make_desc(N, C, H, W, M, R, S, stride, pad) -> escoin_conv_desc:
    return escoin_conv_desc(N, C, H, W, M, R, S, stride, pad)


def desc_of(spec) -> escoin_conv_desc:
    """Descriptor from any object with the Table-1 attribute names."""
    return make_desc(spec.N, spec.C, spec.H, spec.W, spec.M, spec.R, spec.S, spec.stride, spec.pad)


def _check(rc: int, where: str):
    if rc != OK:
        raise EscoinError(rc, where)


def _hptr(a, dtype=None):
    """Pointer to a host numpy array (C-contiguous, expected dtype) or None."""
    if a is None:
        return None
    if not isinstance(a, np.ndarray) or not a.flags["C_CONTIGUOUS"]:
        raise TypeError("host arguments must be C-contiguous numpy arrays")
    if dtype is not None and a.dtype != dtype:
        raise TypeError(f"host array has dtype {a.dtype}, expected {dtype}")
    return a.ctypes.data


def _dptr(t, dtype=None):
    """Pointer to a contiguous torch CUDA tensor or None."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise TypeError("device arguments must be contiguous CUDA tensors")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"device tensor has dtype {t.dtype}, expected {dtype}")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


def strerror(code: int) -> str:
    return lib().escoin_strerror(code).decode()


def escoin_check_desc(desc) -> int:
    return lib().escoin_check_desc(ctypes.byref(desc))


def escoin_output_dims(desc):
    E, F = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().escoin_output_dims(ctypes.byref(desc), ctypes.byref(E), ctypes.byref(F)),
           "escoin_output_dims")
    return E.value, F.value


def escoin_padded_elems(desc) -> int:
    return lib().escoin_padded_elems(ctypes.byref(desc))


def escoin_output_elems(desc) -> int:
    return lib().escoin_output_elems(ctypes.byref(desc))


def escoin_sconv_pack(desc, rowptr: np.ndarray, colidx: np.ndarray,
                      colidx_stretched: np.ndarray | None = None) -> np.ndarray:
    if colidx_stretched is None:
        colidx_stretched = np.empty_like(colidx)
    _check(lib().escoin_sconv_pack(ctypes.byref(desc), _hptr(rowptr, np.int32),
                                   _hptr(colidx, np.int32), _hptr(colidx_stretched, np.int32)),
           "escoin_sconv_pack")
    return colidx_stretched


def escoin_pad_in(desc, d_in, d_padded, stream=None):
    import torch
    _check(lib().escoin_pad_in(ctypes.byref(desc), _dptr(d_in, torch.float32),
                               _dptr(d_padded, torch.float32), _stream(stream)), "escoin_pad_in")


def escoin_sconv_forward(desc, d_rowptr, d_colidx_stretched, d_value, d_padded, d_out,
                         d_bias=None, flags=0, stream=None):
    import torch
    _check(lib().escoin_sconv_forward(ctypes.byref(desc), _dptr(d_rowptr, torch.int32),
                                      _dptr(d_colidx_stretched, torch.int32),
                                      _dptr(d_value, torch.float32),
                                      _dptr(d_padded, torch.float32),
                                      _dptr(d_out, torch.float32), _dptr(d_bias, torch.float32),
                                      flags, _stream(stream)), "escoin_sconv_forward")


def make_tuning(**kw):
    """Tiling knobs for the plan (K, Q, B, WM, CC, NB, TH, CS, WS, CC0); omitted fields are chosen by the
    library.  Returns None when nothing is given."""
    if not kw:
        return None
    return escoin_sconv_tuning(**{k: int(v) for k, v in kw.items()})


def _tref(tuning):
    return ctypes.byref(tuning) if tuning is not None else None


def escoin_sconv_plan_size(desc, rowptr: np.ndarray, colidx_stretched: np.ndarray, tuning=None) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().escoin_sconv_plan_size(ctypes.byref(desc), _hptr(rowptr, np.int32),
                                        _hptr(colidx_stretched, np.int32), _tref(tuning),
                                        ctypes.byref(n)), "escoin_sconv_plan_size")
    return n.value


def escoin_sconv_plan_build(desc, rowptr: np.ndarray, colidx_stretched: np.ndarray,
                            value: np.ndarray, tuning=None, plan: np.ndarray | None = None) -> np.ndarray:
    """Returns the plan blob as a uint8 numpy array (host)."""
    if plan is None:
        plan = np.empty(escoin_sconv_plan_size(desc, rowptr, colidx_stretched, tuning), dtype=np.uint8)
    _check(lib().escoin_sconv_plan_build(ctypes.byref(desc), _hptr(rowptr, np.int32),
                                         _hptr(colidx_stretched, np.int32), _hptr(value, np.float32),
                                         _tref(tuning), _hptr(plan, np.uint8), plan.nbytes),
           "escoin_sconv_plan_build")
    return plan


def escoin_sconv_forward_tiled(desc, plan_host: np.ndarray, d_plan, d_in, d_out, d_bias=None,
                               flags=0, stream=None):
    import torch
    _check(lib().escoin_sconv_forward_tiled(ctypes.byref(desc), _hptr(plan_host, np.uint8),
                                            _dptr(d_plan, torch.uint8), _dptr(d_in, torch.float32),
                                            _dptr(d_out, torch.float32), _dptr(d_bias, torch.float32),
                                            flags, _stream(stream)), "escoin_sconv_forward_tiled")


def escoin_sconv_tiled_on_matrix_cores(desc, plan_host: np.ndarray) -> bool:
    rc = lib().escoin_sconv_tiled_on_matrix_cores(ctypes.byref(desc), _hptr(plan_host, np.uint8))
    if rc < 0:
        _check(rc, "escoin_sconv_tiled_on_matrix_cores")
    return rc == 1


def escoin_sconv_tiled_kernel(desc, plan_host: np.ndarray) -> int:
    rc = lib().escoin_sconv_tiled_kernel(ctypes.byref(desc), _hptr(plan_host, np.uint8))
    if rc < 0:
        _check(rc, "escoin_sconv_tiled_kernel")
    return rc


def make_linear_desc(T, K, M, type, gated=False, ld_in=0, ld_out=0, ld_residual=0) -> escoin_linear_desc:
    """T tokens (for a plan: the most a call may have), K input and M output features, type T_F32, T_F16 or T_BF16."""
    return escoin_linear_desc(T, K, M, type, int(gated), ld_in, ld_out, ld_residual)


def make_norm_desc(T, D, type, post=NORM_NONE, pre=NORM_RMS, gate_rows=0, eps=1e-5, alpha=1.0, beta=1.0, weight_offset=0.0,
                   ld_x=0, ld_y=0, ld_gate=0, ld_h=0, ld_n=0) -> escoin_norm_desc:
    return escoin_norm_desc(T, D, type, post, pre, gate_rows, eps, alpha, beta, weight_offset, ld_x, ld_y, ld_gate, ld_h, ld_n)


_torch_types = []


class _Rows:
    """Checks the device tensors of one call: all on one device, of one type; rows of contiguous elements, or vectors.  A call
    of one token takes some microseconds: the checks are few and cheap."""
    __slots__ = ("type", "device")

    def __init__(self, type):
        if not _torch_types:
            import torch
            _torch_types.extend((torch.float32, torch.float16, torch.bfloat16))
        if not T_F32 <= type <= T_BF16:
            raise EscoinError(EINVAL, f"unknown type {type}")
        self.type, self.device = _torch_types[type], -2    # (a CPU tensor's is -1)

    def _seen(self, t):
        if t.dtype is not self.type:
            raise TypeError(f"device tensor has dtype {t.dtype}, expected {self.type}")
        device = t.get_device()
        if device < 0:
            raise TypeError("device arguments must be CUDA tensors")
        if device != self.device:
            if self.device >= 0:
                raise TypeError(f"tensors of one call lie on devices {self.device} and {device}")
            self.device = device

    def rows(self, t, T, width, ld):
        """Pointer to T rows of `width` elements, `ld` (0: width) apart, or None."""
        if t is None:
            return None
        if t.dtype is not self.type or t.get_device() != self.device:
            self._seen(t)
        shape, stride = t.shape, t.stride()
        if len(shape) != 2 or shape[0] < T or shape[1] != width or (width > 1 and stride[1] != 1) or (T > 1 and stride[0] != (ld or width)):
            raise TypeError(f"expected {T} rows of {width}, {ld or width} elements apart: got shape {tuple(shape)}, strides {stride}")
        return t.data_ptr()

    def vector(self, t, width):
        if t is None:
            return None
        if t.dtype is not self.type or t.get_device() != self.device:
            self._seen(t)
        if t.numel() != width or not t.is_contiguous():
            raise TypeError(f"expected {width} contiguous elements: got shape {tuple(t.shape)}, strides {t.stride()}")
        return t.data_ptr()

    def call(self, where, fn, *args, stream):
        """The library launches on the current device: the tensors' own for the time of the call."""
        import torch
        if self.device < 0:
            raise TypeError("a call without tensors")
        if self.device != torch._C._cuda_getDevice():  # (the runtime runs: there are tensors)
            with torch.cuda.device(self.device):
                return _check(fn(*args, _stream(stream)), where)
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(self.device) if stream is None else _stream(stream))
        if rc != OK:
            _check(rc, where)


def escoin_linear_check_desc(desc) -> int:
    return lib().escoin_linear_check_desc(ctypes.byref(desc))


def _csr(desc, rowptr, colidx, value=None):
    """The arrays' pointers, once they are as long as they say (the library cannot tell)."""
    p = _hptr(rowptr, np.int32), _hptr(colidx, np.int32), _hptr(value, np.float32)
    rows = desc.M * (2 if desc.gated else 1)
    if rowptr is not None:
        if rowptr.size != rows + 1:
            raise TypeError(f"rowptr has {rowptr.size} entries, expected {rows + 1}")
        for a in (colidx, value):
            if a is not None and a.size < rowptr[-1]:
                raise TypeError(f"an array of {a.size} elements for {rowptr[-1]} nonzeros")
    return p


def escoin_linear_plan_size(desc, rowptr: np.ndarray, colidx: np.ndarray) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().escoin_linear_plan_size(ctypes.byref(desc), *_csr(desc, rowptr, colidx)[:2], ctypes.byref(n)), "escoin_linear_plan_size")
    return n.value


def escoin_linear_plan_build(desc, rowptr: np.ndarray, colidx: np.ndarray, value: np.ndarray, plan: np.ndarray | None = None) -> np.ndarray:
    """Returns the plan blob as a uint8 numpy array (host)."""
    if plan is None:
        plan = np.empty(escoin_linear_plan_size(desc, rowptr, colidx), dtype=np.uint8)
    _check(lib().escoin_linear_plan_build(ctypes.byref(desc), *_csr(desc, rowptr, colidx, value), _hptr(plan, np.uint8), plan.nbytes),
           "escoin_linear_plan_build")
    return plan


def escoin_linear_few_tokens(desc, plan_host: np.ndarray) -> int:
    rc = lib().escoin_linear_few_tokens(ctypes.byref(desc), _plan_header(plan_host))
    if rc < 0:
        _check(rc, "escoin_linear_few_tokens")
    return rc


def escoin_linear_kernel(desc, plan_host: np.ndarray, address: int = 0) -> dict:
    """Which kernel a call takes whose input lies at `address` (0: wherever rows start on 16 bytes)."""
    info = escoin_linear_kernel_info()
    _check(lib().escoin_linear_kernel(ctypes.byref(desc), _plan_header(plan_host), address, ctypes.byref(info)), "escoin_linear_kernel")
    return {k: int(getattr(info, k)) for k, _ in info._fields_}


class _LinearHeader(ctypes.Structure):
    """Mirror of the linear plan's header (csrc/linear.h), for diagnostics and tests."""
    _fields_ = ([(k, ctypes.c_uint32) for k in ("magic", "version")]
                + [(k, ctypes.c_int32) for k in ("K", "M", "type", "gated", "most_tokens", "few_tokens", "most_lane_words", "reserved")]
                + [(k, ctypes.c_uint64) for k in ("off_zero", "off_mask", "off_start", "off_kept", "off_whole", "total_bytes")])


_BYTES, _HEADER_BYTES = np.dtype(np.uint8), ctypes.sizeof(_LinearHeader)
_TOTAL = slice(_LinearHeader.total_bytes.offset, _HEADER_BYTES)  # where it says how long a plan is


def _plan_header(plan: np.ndarray) -> bytes:
    """The bytes of the plan that a call reads on the host (a copy of them is had sooner than the array's address)."""
    if not isinstance(plan, np.ndarray) or plan.dtype != _BYTES or plan.ndim != 1 or plan.strides[0] != 1 or plan.size < _HEADER_BYTES:
        raise TypeError("this is no plan of a linear layer")
    return plan[:_HEADER_BYTES].tobytes()


def linear_plan_header(plan: np.ndarray) -> dict:
    """Decodes the (opaque) header of a linear layer's plan."""
    h = _LinearHeader.from_buffer_copy(plan[:ctypes.sizeof(_LinearHeader)].tobytes())
    return {k: int(getattr(h, k)) for k, _ in _LinearHeader._fields_}


def escoin_linear_forward(desc, plan_host: np.ndarray, d_plan, d_in, d_out, d_bias=None, d_residual=None, flags=0, stream=None):
    t = _Rows(desc.type)
    T, rows = max(desc.T, 0), desc.M * (2 if desc.gated else 1)
    args = (t.rows(d_in, T, desc.K, desc.ld_in), t.rows(d_out, T, desc.M, desc.ld_out), t.vector(d_bias, rows),
            t.rows(d_residual, T, desc.M, desc.ld_residual))
    plan = _plan_header(plan_host)
    if d_plan is None or d_plan.get_device() != t.device or d_plan.nbytes < int.from_bytes(plan[_TOTAL], "little") or not d_plan.is_contiguous():
        raise TypeError("the plan's copy has to be whole and on the tensors' device")
    t.call("escoin_linear_forward", lib().escoin_linear_forward, ctypes.byref(desc), plan, d_plan.data_ptr(), *args, flags, stream=stream)


def escoin_norm_check_desc(desc) -> int:
    return lib().escoin_norm_check_desc(ctypes.byref(desc))


def escoin_norm_forward(desc, d_x, d_h, d_n, d_y=None, d_gate=None, d_post_weight=None, d_post_bias=None, d_pre_weight=None,
                        d_pre_bias=None, stream=None):
    """`d_h` or `d_n` may be None: that output is not wanted."""
    t = _Rows(desc.type)
    T, D = max(desc.T, 0), desc.D
    gate = t.rows(d_gate, T, D, desc.ld_gate) if desc.gate_rows else t.vector(d_gate, D)
    x, y, h, n = (t.rows(v, T, D, ld) for v, ld in ((d_x, desc.ld_x), (d_y, desc.ld_y), (d_h, desc.ld_h), (d_n, desc.ld_n)))
    params = [t.vector(v, D) for v in (d_post_weight, d_post_bias, d_pre_weight, d_pre_bias)]
    t.call("escoin_norm_forward", lib().escoin_norm_forward, ctypes.byref(desc), x, y, gate, *params, h, n, stream=stream)


class _PlanHeader(ctypes.Structure):
    """Mirror of the plan blob's header (csrc/plan.h), for diagnostics, tests and the bench."""
    _fields_ = ([("magic", ctypes.c_uint32), ("version", ctypes.c_uint32)]
                + [(k, ctypes.c_int32) for k in (
                    "C", "H", "W", "M", "R", "S", "stride", "pad", "E", "F", "K", "Q", "B", "WM", "WQ",
                    "CC", "NB", "TH", "n_tiles", "n_mgroups", "n_chunks", "n_phases", "pitch", "front",
                    "rows_in", "plane_stride", "P4", "n_items", "buf_floats", "tail_floats",
                    "rec_buf_bytes", "lds_bytes", "nnz", "n_records")]
                + [(k, ctypes.c_uint64) for k in (
                    "off_items", "off_lanes", "off_dst_lut", "off_perm", "off_blk", "off_seg", "off_rec",
                    "total_bytes")]
                + [(k, ctypes.c_int32) for k in (
                    "CS", "pitch1", "VW", "WW", "WS", "CC0", "zero_floats", "max_regions", "MB", "n_dma")]
                + [("off_dma", ctypes.c_uint64), ("off_zero", ctypes.c_uint64),
                   ("mfma", ctypes.c_int32), ("mfma_nnz", ctypes.c_int32), ("off_mfma", ctypes.c_uint64),
                   ("pair", ctypes.c_int32), ("pair_nnz", ctypes.c_int32), ("off_pair", ctypes.c_uint64), ("off_nz", ctypes.c_uint64),
                   ("pair_least", ctypes.c_int32), ("pair_few2", ctypes.c_int32), ("pair_few4", ctypes.c_int32),
                   ("pair_few8", ctypes.c_int32)])


def plan_header(plan: np.ndarray) -> dict:
    """Decodes the (opaque) plan header for diagnostics, tests and the bench's reporting."""
    h = _PlanHeader.from_buffer_copy(plan[:ctypes.sizeof(_PlanHeader)].tobytes())
    return {k: int(getattr(h, k)) for k, _ in _PlanHeader._fields_}
