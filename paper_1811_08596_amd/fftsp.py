"""Thin ctypes binding over libfftsp.so (include/fftsp.h): argument marshalling only.

Every step of the codec runs in the HIP kernels behind the C ABI; torch is used
for device memory and streams.  There is no CPU fallback: if the shared library
is missing or fails to load, importing callers get an ImportError.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfftsp.so")

OK, EINVAL, ENOSPC, EWORKSPACE, EUNSUPPORTED, EHIP, EFORMAT = range(7)

# name -> (restype, argtypes); every symbol include/fftsp.h declares
_szp = C.POINTER(C.c_size_t)
class Quantizer(C.Structure):
    """fftsp_quantizer: mantissa_bits (0 = default for the width), range_max (0 = fitted per chunk)."""
    _fields_ = [("mantissa_bits", C.c_int), ("range_max", C.c_float)]


_qp = C.POINTER(Quantizer)


class Matrix(C.Structure):
    """fftsp_matrix: `rows` rows of `cols` values, the first at element `offset` of flat arrays, rows `stride` apart
    (None: cols); gain: factor on the orthogonalised form."""
    _fields_ = [("offset", C.c_uint64), ("stride", C.c_uint64), ("rows", C.c_uint32), ("cols", C.c_uint32),
                ("gain", C.c_float), ("reserved", C.c_uint32)]

    def __init__(self, offset: int, rows: int, cols: int, stride: Optional[int] = None, gain: float = 1.0):
        stride = cols if stride is None else stride
        # a field takes any number modulo its range
        if not (0 <= offset < 1 << 64 and 0 <= stride < 1 << 64 and 0 <= rows < 1 << 32 and 0 <= cols < 1 << 32):
            raise ValueError(f"no such matrix: {rows} x {cols} at {offset}, stride {stride}")
        super().__init__(offset, stride, rows, cols, gain, 0)


_mp = C.POINTER(Matrix)


class Step(C.Structure):
    """fftsp_step"""
    _fields_ = [("lr", C.c_float), ("beta", C.c_float), ("weight_decay", C.c_float), ("eps", C.c_float),
                ("nesterov", C.c_int), ("nsteps", C.c_int), ("coefficients", C.POINTER(C.c_float))]


_sp = C.POINTER(Step)

SIGNATURES = {
    "fftsp_kept_per_chunk": (C.c_int, [C.c_uint32, C.c_float, C.POINTER(C.c_uint32)]),
    "fftsp_mantissa_bits": (C.c_int, [C.c_int]),
    "fftsp_packed_bytes": (C.c_size_t, [C.c_size_t, C.c_uint32, C.c_float, C.c_int]),
    "fftsp_workspace_bytes": (C.c_size_t, [C.c_size_t, C.c_uint32, C.c_int]),
    "fftsp_compress": (C.c_int, [C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int, C.c_void_p, C.c_size_t,
                                 C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_decompress": (C.c_int, [C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int,
                                   C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_compress_static": (C.c_int, [C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int, C.c_void_p,
                                        C.c_size_t, C.c_void_p]),
    "fftsp_compress_h": (C.c_int, [C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int, C.c_int, C.c_void_p,
                                   C.c_size_t, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_decompress_h": (C.c_int, [C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int,
                                     C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_topk_kept_per_chunk": (C.c_int, [C.c_uint32, C.c_float, C.POINTER(C.c_uint32)]),
    "fftsp_topk_packed_bytes": (C.c_size_t, [C.c_size_t, C.c_uint32, C.c_float, C.c_int]),
    "fftsp_topk_workspace_bytes": (C.c_size_t, [C.c_size_t, C.c_uint32, C.c_int]),
    "fftsp_topk_compress": (C.c_int, [C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int, C.c_void_p, C.c_size_t,
                                      C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_topk_decompress": (C.c_int, [C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_uint32, C.c_float,
                                        C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_compress_q": (C.c_int, [C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int, C.c_void_p, C.c_size_t,
                                   C.c_void_p, C.c_size_t, _qp, C.c_void_p]),
    "fftsp_decompress_q": (C.c_int, [C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int,
                                     C.c_void_p, C.c_size_t, _qp, C.c_void_p]),
    "fftsp_encode_spectrum_q": (C.c_int, [C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int, C.c_void_p,
                                          C.c_size_t, C.c_void_p, C.c_size_t, _qp, C.c_void_p]),
    "fftsp_decode_spectrum_q": (C.c_int, [C.c_void_p, C.c_size_t, C.c_size_t, C.c_uint32, C.c_float, C.c_int,
                                          C.c_void_p, C.c_void_p, C.c_size_t, _qp, C.c_void_p]),
    "fftsp_workspace_bytes_accumulate": (C.c_size_t, [C.c_size_t, C.c_uint32, C.c_int, C.c_int]),
    "fftsp_decompress_accumulate": (C.c_int, [C.POINTER(C.c_void_p), C.c_int, C.c_size_t, C.c_float, C.c_void_p,
                                              C.c_size_t, C.c_uint32, C.c_float, C.c_int, C.c_void_p, C.c_size_t,
                                              C.c_void_p]),
    "fftsp_decode_accumulate_spectrum": (C.c_int, [C.POINTER(C.c_void_p), C.c_int, C.c_size_t, C.c_size_t, C.c_uint32,
                                                   C.c_float, C.c_int, C.c_void_p, C.c_void_p, C.c_size_t,
                                                   C.c_void_p]),
    "fftsp_rfft": (C.c_int, [C.c_void_p, C.c_size_t, C.c_uint32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_irfft": (C.c_int, [C.c_void_p, C.c_size_t, C.c_uint32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_encode_spectrum": (C.c_int, [C.c_void_p, C.c_size_t, C.c_uint32, C.c_float, C.c_int, C.c_void_p,
                                        C.c_size_t, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_decode_spectrum": (C.c_int, [C.c_void_p, C.c_size_t, C.c_size_t, C.c_uint32, C.c_float, C.c_int,
                                        C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_packed_bytes_segments": (C.c_size_t, [_szp, C.c_int, C.c_float, C.c_int]),
    "fftsp_workspace_bytes_segments": (C.c_size_t, [_szp, C.c_int, C.c_int]),
    "fftsp_compress_segments": (C.c_int, [C.c_void_p, _szp, C.c_int, C.c_float, C.c_int, C.c_void_p, C.c_size_t,
                                          C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_decompress_segments": (C.c_int, [C.c_void_p, C.c_size_t, C.c_void_p, _szp, C.c_int, C.c_float, C.c_int,
                                            C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_embedding": (C.c_int, [C.c_void_p, C.c_int, C.c_size_t, C.c_uint32, C.c_size_t, C.c_void_p, C.c_int,
                                  C.c_size_t, C.c_float, C.c_void_p, C.c_int, C.c_size_t, C.c_void_p]),
    "fftsp_workspace_bytes_embedding": (C.c_size_t, [C.c_size_t, C.c_uint32, C.c_size_t]),
    "fftsp_embedding_gradient": (C.c_int, [C.c_void_p, C.c_int, C.c_size_t, C.c_void_p, C.c_int, C.c_size_t, C.c_float,
                                           C.c_void_p, C.c_void_p, C.c_int, C.c_size_t, C.c_uint32, C.c_size_t,
                                           C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_workspace_bytes_orthogonal": (C.c_size_t, [_mp, C.c_int]),
    "fftsp_orthogonal": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_int, _mp, C.c_int, C.POINTER(C.c_float),
                                   C.c_int, C.c_float, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_orthogonal_step": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int,
                                        _mp, C.c_int, _sp, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fftsp_device_status": (C.c_int, [C.c_void_p, C.POINTER(C.c_int)]),
    "fftsp_profile_enable": (C.c_int, [C.c_int]),
    "fftsp_profile_report": (C.c_size_t, [C.c_char_p, C.c_size_t]),
    "fftsp_strerror": (C.c_char_p, [C.c_int]),
    "fftsp_version": (C.c_char_p, []),
}

_lib = None


def load(path: Optional[str] = None):
    """dlopen the C-ABI library and attach prototypes; raises ImportError if it is not built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise ImportError(f"{p} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "(there is no CPU fallback)")
    try:
        lib = C.CDLL(p)
    except OSError as e:
        raise ImportError(f"cannot load {p}: {e}") from e
    for name, (res, args) in SIGNATURES.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    if path is None:
        _lib = lib
    return lib


class FftspError(RuntimeError):
    def __init__(self, code: int, where: str):
        msg = load().fftsp_strerror(code).decode()
        super().__init__(f"{where}: {msg} (status {code})")
        self.code = code


def _check(code: int, where: str):
    if code != OK:
        raise FftspError(code, where)


def _stream(stream=None) -> int:
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


def _offsets(seg_offsets: Sequence[int]):
    arr = (C.c_size_t * len(seg_offsets))(*[int(v) for v in seg_offsets])
    return arr, len(seg_offsets) - 1


# ---- host arithmetic ----
def kept_per_chunk(chunk_len: int, theta: float) -> int:
    k = C.c_uint32()
    _check(load().fftsp_kept_per_chunk(chunk_len, theta, C.byref(k)), "fftsp_kept_per_chunk")
    return k.value


def mantissa_bits(bits: int) -> int:
    return load().fftsp_mantissa_bits(bits)


def packed_bytes(n: int, chunk_len: int, theta: float, bits: int) -> int:
    return load().fftsp_packed_bytes(n, chunk_len, theta, bits)


def workspace_bytes(n: int, chunk_len: int, bits: int) -> int:
    return load().fftsp_workspace_bytes(n, chunk_len, bits)


def packed_bytes_segments(seg_offsets, theta: float, bits: int) -> int:
    arr, nseg = _offsets(seg_offsets)
    return load().fftsp_packed_bytes_segments(arr, nseg, theta, bits)


def workspace_bytes_segments(seg_offsets, bits: int) -> int:
    arr, nseg = _offsets(seg_offsets)
    return load().fftsp_workspace_bytes_segments(arr, nseg, bits)


# ---- device entry points: tensors are torch CUDA tensors, contiguous ----
def _ptr(t) -> int:
    assert t.is_cuda and t.is_contiguous(), "device entry points take contiguous CUDA tensors"
    return t.data_ptr()


def _nbytes(t) -> int:
    return t.numel() * t.element_size()


def compress(grad, chunk_len: int, theta: float, bits: int, packed, workspace, stream=None):
    _check(load().fftsp_compress(_ptr(grad), grad.numel(), chunk_len, theta, bits, _ptr(packed), _nbytes(packed),
                                 _ptr(workspace), _nbytes(workspace), _stream(stream)), "fftsp_compress")


STATIC_SCRATCH_BYTES = 16 << 20  # FFTSP_STATIC_SCRATCH_BYTES


def compress_static(grad, chunk_len: int, theta: float, bits: int, packed, stream=None):
    """fftsp_compress on the library's own fixed scratch array: no workspace argument, no allocation."""
    _check(load().fftsp_compress_static(_ptr(grad), grad.numel(), chunk_len, theta, bits, _ptr(packed),
                                        _nbytes(packed), _stream(stream)), "fftsp_compress_static")


def decompress(packed, packed_nbytes: int, grad_out, chunk_len: int, theta: float, bits: int, workspace, stream=None):
    _check(load().fftsp_decompress(_ptr(packed), packed_nbytes, _ptr(grad_out), grad_out.numel(), chunk_len, theta,
                                   bits, _ptr(workspace), _nbytes(workspace), _stream(stream)), "fftsp_decompress")


def compress_h(grad, chunk_len: int, theta: float, bits: int, scale_log2: int, packed, workspace, stream=None):
    _check(load().fftsp_compress_h(_ptr(grad), grad.numel(), chunk_len, theta, bits, scale_log2, _ptr(packed),
                                   _nbytes(packed), _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "fftsp_compress_h")


def decompress_h(packed, packed_nbytes: int, grad_out, chunk_len: int, theta: float, bits: int, scale_log2: int,
                 workspace, stream=None):
    _check(load().fftsp_decompress_h(_ptr(packed), packed_nbytes, _ptr(grad_out), grad_out.numel(), chunk_len, theta,
                                     bits, scale_log2, _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "fftsp_decompress_h")


def topk_kept_per_chunk(chunk_len: int, theta: float) -> int:
    k = C.c_uint32()
    _check(load().fftsp_topk_kept_per_chunk(chunk_len, theta, C.byref(k)), "fftsp_topk_kept_per_chunk")
    return k.value


def topk_packed_bytes(n: int, chunk_len: int, theta: float, bits: int) -> int:
    return load().fftsp_topk_packed_bytes(n, chunk_len, theta, bits)


def topk_workspace_bytes(n: int, chunk_len: int, bits: int) -> int:
    return load().fftsp_topk_workspace_bytes(n, chunk_len, bits)


def topk_compress(grad, chunk_len: int, theta: float, bits: int, packed, workspace, stream=None):
    _check(load().fftsp_topk_compress(_ptr(grad), grad.numel(), chunk_len, theta, bits, _ptr(packed), _nbytes(packed),
                                      _ptr(workspace), _nbytes(workspace), _stream(stream)), "fftsp_topk_compress")


def topk_decompress(packed, packed_nbytes: int, grad_out, chunk_len: int, theta: float, bits: int, workspace,
                    stream=None):
    _check(load().fftsp_topk_decompress(_ptr(packed), packed_nbytes, _ptr(grad_out), grad_out.numel(), chunk_len,
                                        theta, bits, _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "fftsp_topk_decompress")


def compress_q(grad, chunk_len: int, theta: float, bits: int, packed, workspace, mantissa_bits=0, range_max=0.0,
               stream=None):
    q = Quantizer(mantissa_bits, range_max)  # kept alive until the call returns
    _check(load().fftsp_compress_q(_ptr(grad), grad.numel(), chunk_len, theta, bits, _ptr(packed), _nbytes(packed),
                                   _ptr(workspace), _nbytes(workspace), C.byref(q),
                                   _stream(stream)), "fftsp_compress_q")


def decompress_q(packed, packed_nbytes: int, grad_out, chunk_len: int, theta: float, bits: int, workspace,
                 mantissa_bits=0, stream=None):
    q = Quantizer(mantissa_bits, 0.0)  # kept alive until the call returns
    _check(load().fftsp_decompress_q(_ptr(packed), packed_nbytes, _ptr(grad_out), grad_out.numel(), chunk_len, theta,
                                     bits, _ptr(workspace), _nbytes(workspace),
                                     C.byref(q), _stream(stream)), "fftsp_decompress_q")


def encode_spectrum_q(spec, n: int, chunk_len: int, theta: float, bits: int, packed, workspace, mantissa_bits=0,
                      range_max=0.0, stream=None):
    q = Quantizer(mantissa_bits, range_max)  # kept alive until the call returns
    _check(load().fftsp_encode_spectrum_q(_ptr(spec), n, chunk_len, theta, bits, _ptr(packed), _nbytes(packed),
                                          _ptr(workspace), _nbytes(workspace),
                                          C.byref(q), _stream(stream)),
           "fftsp_encode_spectrum_q")


def decode_spectrum_q(packed, packed_nbytes: int, n: int, chunk_len: int, theta: float, bits: int, spec, workspace,
                      mantissa_bits=0, stream=None):
    q = Quantizer(mantissa_bits, 0.0)  # kept alive until the call returns
    _check(load().fftsp_decode_spectrum_q(_ptr(packed), packed_nbytes, n, chunk_len, theta, bits, _ptr(spec),
                                          _ptr(workspace), _nbytes(workspace),
                                          C.byref(q), _stream(stream)),
           "fftsp_decode_spectrum_q")


def workspace_bytes_accumulate(n: int, chunk_len: int, bits: int, npeers: int) -> int:
    return load().fftsp_workspace_bytes_accumulate(n, chunk_len, bits, npeers)


def _peer_array(packed_list):
    return (C.c_void_p * len(packed_list))(*[_ptr(p) for p in packed_list])


def decompress_accumulate(packed_list, packed_nbytes: int, scale: float, grad_out, chunk_len: int, theta: float,
                          bits: int, workspace, stream=None):
    """grad_out = scale * iFFT(sum of the peers' decoded spectra); packed_list: equally long device buffers."""
    _check(load().fftsp_decompress_accumulate(_peer_array(packed_list), len(packed_list), packed_nbytes, scale,
                                              _ptr(grad_out), grad_out.numel(), chunk_len, theta, bits,
                                              _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "fftsp_decompress_accumulate")


def decode_accumulate_spectrum(packed_list, packed_nbytes: int, n: int, chunk_len: int, theta: float, bits: int, spec,
                               workspace, stream=None):
    _check(load().fftsp_decode_accumulate_spectrum(_peer_array(packed_list), len(packed_list), packed_nbytes, n,
                                                   chunk_len, theta, bits, _ptr(spec), _ptr(workspace),
                                                   _nbytes(workspace), _stream(stream)),
           "fftsp_decode_accumulate_spectrum")


def rfft(grad, chunk_len: int, spec, workspace, stream=None):
    _check(load().fftsp_rfft(_ptr(grad), grad.numel(), chunk_len, _ptr(spec), _ptr(workspace), _nbytes(workspace),
                             _stream(stream)), "fftsp_rfft")


def irfft(spec, n: int, chunk_len: int, grad_out, workspace, stream=None):
    _check(load().fftsp_irfft(_ptr(spec), n, chunk_len, _ptr(grad_out), _ptr(workspace), _nbytes(workspace),
                              _stream(stream)), "fftsp_irfft")


def encode_spectrum(spec, n: int, chunk_len: int, theta: float, bits: int, packed, workspace, stream=None):
    _check(load().fftsp_encode_spectrum(_ptr(spec), n, chunk_len, theta, bits, _ptr(packed), _nbytes(packed),
                                        _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "fftsp_encode_spectrum")


def decode_spectrum(packed, packed_nbytes: int, n: int, chunk_len: int, theta: float, bits: int, spec, workspace,
                    stream=None):
    _check(load().fftsp_decode_spectrum(_ptr(packed), packed_nbytes, n, chunk_len, theta, bits, _ptr(spec),
                                        _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "fftsp_decode_spectrum")


def compress_segments(grad, seg_offsets, theta: float, bits: int, packed, workspace, stream=None):
    arr, nseg = _offsets(seg_offsets)
    _check(load().fftsp_compress_segments(_ptr(grad), arr, nseg, theta, bits, _ptr(packed), _nbytes(packed),
                                          _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "fftsp_compress_segments")


def decompress_segments(packed, packed_nbytes: int, grad_out, seg_offsets, theta: float, bits: int, workspace,
                        stream=None):
    arr, nseg = _offsets(seg_offsets)
    _check(load().fftsp_decompress_segments(_ptr(packed), packed_nbytes, _ptr(grad_out), arr, nseg, theta, bits,
                                            _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "fftsp_decompress_segments")


# ---- the embedding and the orthogonalised update: any element's alignment, rows with strides ----
F32, BF16, F16 = range(3)


_TYPES: dict = {}   # torch's types as fftsp_type, filled at the first call (torch is not loaded at import)
_INDEX: dict = {}
_torch = None


def _load_torch():
    global _torch
    if _torch is None:
        import torch
        _TYPES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
        _INDEX.update({torch.int32: 32, torch.int64: 64})
        _torch = torch
    return _torch


def _type(t) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        _load_torch()
        code = _TYPES.get(t.dtype)
        if code is None:
            raise TypeError(f"{t.dtype}: float32, bfloat16 or float16 is wanted")
    return code


def _same_device(*tensors) -> int:
    """The tensors' one GPU; calls are made with it as the current device and, by default, on its current stream."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t.get_device() != dev or dev < 0:
            raise ValueError("device entry points take CUDA tensors of one device")
    return dev


def _call(function, where: str, dev: int, stream, *args):
    """function(*args, stream) on device `dev`; `stream`: a torch stream, or None for the device's current one"""
    torch = _load_torch()
    s = (stream if stream is not None else torch.cuda.current_stream(dev)).cuda_stream
    if torch.cuda.current_device() == dev:
        code = function(*args, s)
    else:
        with torch.cuda.device(dev):
            code = function(*args, s)
    if code != OK:
        raise FftspError(code, where)


def _rows(t, width: int):
    """(data pointer, rows, distance of rows) of a tensor whose last axis holds `width` consecutive values; more than two
    axes have to be contiguous"""
    shape = t.shape
    if len(shape) != 2:
        if len(shape) < 2 or not t.is_contiguous():
            raise ValueError("rows are a 2-D tensor, or a contiguous one of more axes")
        t = t.view(-1, shape[-1])
        shape = t.shape
    rows, values = shape
    stride, one = t.stride()
    if width >> 32:
        raise ValueError(f"rows of {width} values are too long")
    if values != width or (width > 1 and one != 1):
        raise ValueError(f"rows of {width} consecutive values are wanted, got {tuple(shape)} with strides {t.stride()}")
    return t.data_ptr(), rows, stride if rows > 1 else max(width, stride)


def _tokens(t, count: int) -> int:
    _load_torch()
    bits = _INDEX.get(t.dtype)
    if bits is None:
        raise TypeError(f"tokens are int32 or int64, got {t.dtype}")
    if not t.is_contiguous() or t.numel() != count:
        raise ValueError(f"{count} contiguous tokens are wanted, got {tuple(t.shape)}")
    return bits


def embedding(table, tokens, out, scale: float = 1.0, stream=None):
    """out[t] = scale * table[tokens[t]]; a token outside the table gives a row of zeros.  table: [rows, width], out:
    [number of tokens, width] (or the tokens' shape with an axis of `width` behind it); each float32, bfloat16 or float16."""
    dev = _same_device(table, tokens, out)
    tp, rows, ts = _rows(table, table.shape[-1])
    op, count, os_ = _rows(out, table.shape[-1])
    bits = _tokens(tokens, count)
    _call(load().fftsp_embedding, "fftsp_embedding", dev, stream, tp, _type(table), rows, table.shape[-1], ts,
          tokens.data_ptr(), bits, count, scale, op, _type(out), os_)


def workspace_bytes_embedding(rows: int, width: int, ntokens: int) -> int:
    return 0 if width >> 32 else load().fftsp_workspace_bytes_embedding(rows, width, ntokens)


def embedding_gradient(out_grad, tokens, table_grad, workspace, scale: float = 1.0, base=None, stream=None):
    """table_grad[v] = base[v] + scale * (sum of out_grad[t] over the t with tokens[t] == v), every row written.
    base: None (zeros), table_grad itself (added in place) or a tensor of its type and strides."""
    width = table_grad.shape[-1]
    dev = _same_device(table_grad, out_grad, tokens, workspace, *([] if base is None else [base]))
    gp, count, gs = _rows(out_grad, width)
    tp, rows, ts = _rows(table_grad, width)
    bits = _tokens(tokens, count)
    bp = None
    if base is not None:
        bp, brows, bs = _rows(base, width)
        if brows != rows or bs != ts or base.dtype != table_grad.dtype:
            raise ValueError("base has the shape, strides and type of table_grad")
    _call(load().fftsp_embedding_gradient, "fftsp_embedding_gradient", dev, stream, gp, _type(out_grad), gs,
          tokens.data_ptr(), bits, count, scale, bp, tp, _type(table_grad), rows, width, ts, _ptr(workspace),
          _nbytes(workspace))


class Matrices:
    """A list of fftsp_matrix for the calls below, and the elements that a flat array needs to hold it."""

    def __init__(self, matrices: Sequence[Matrix]):
        self.count = len(matrices)
        self.array = (Matrix * max(1, self.count))(*matrices) if self.count else None
        self.end = max((m.offset + (m.rows - 1) * m.stride + m.cols for m in matrices), default=0)


def matrices(listing: Sequence[Matrix]) -> Matrices:
    return Matrices(listing)


def _flat(t, listing: Matrices, name: str) -> int:
    if not t.is_contiguous() or t.numel() < listing.end:
        raise ValueError(f"{name}: a contiguous tensor of {listing.end} or more elements is wanted")
    return t.data_ptr()


def _coefficients(coefficients):
    """[(a, b, c), ...] or None"""
    if coefficients is None:
        return None, 0
    flat = [float(v) for abc in coefficients for v in abc]
    if len(flat) != 3 * len(coefficients):
        raise ValueError("coefficients are triples")
    return (C.c_float * max(1, len(flat)))(*flat), len(coefficients)


def workspace_bytes_orthogonal(listing: Matrices) -> int:
    return load().fftsp_workspace_bytes_orthogonal(listing.array, listing.count)


def orthogonal(x, out, listing: Matrices, workspace, coefficients=None, eps: float = 1e-7, stream=None):
    """Newton-Schulz orthogonalisation of every matrix of `listing`, from the flat array x into the flat array out (which
    may be x).  coefficients: (a, b, c) of every step; None: five steps of (3.4445, -4.7750, 2.0315)."""
    dev = _same_device(x, out, workspace)
    co, steps = _coefficients(coefficients)  # kept alive until the call returns
    _call(load().fftsp_orthogonal, "fftsp_orthogonal", dev, stream, _flat(x, listing, "x"), _type(x),
          _flat(out, listing, "out"), _type(out), listing.array, listing.count, co, steps, eps, _ptr(workspace),
          _nbytes(workspace))


def orthogonal_step(grad, momentum, weights, listing: Matrices, workspace, lr: float, beta: float = 0.95,
                    weight_decay: float = 0.0, nesterov: bool = True, coefficients=None, eps: float = 1e-7,
                    momentum_out=None, weights_out=None, stream=None):
    """M <- beta M + G; W <- (1 - lr weight_decay) W - lr gain O(G + beta M) for every matrix of `listing` in the flat
    arrays grad, momentum (float32) and weights; in place unless momentum_out, weights_out are given."""
    torch = _load_torch()
    momentum_out = momentum if momentum_out is None else momentum_out
    weights_out = weights if weights_out is None else weights_out
    dev = _same_device(grad, momentum, weights, workspace, momentum_out, weights_out)
    if momentum.dtype != torch.float32 or momentum_out.dtype != torch.float32:
        raise TypeError("momentum is float32")
    if weights_out.dtype != weights.dtype:
        raise TypeError("weights_out has the type of weights")
    co, steps = _coefficients(coefficients)
    step = Step(lr, beta, weight_decay, eps, 1 if nesterov else 0, steps, co)
    _call(load().fftsp_orthogonal_step, "fftsp_orthogonal_step", dev, stream, _flat(grad, listing, "grad"), _type(grad),
          _flat(momentum, listing, "momentum"), _flat(momentum_out, listing, "momentum_out"),
          _flat(weights, listing, "weights"), _flat(weights_out, listing, "weights_out"), _type(weights), listing.array,
          listing.count, C.byref(step), _ptr(workspace), _nbytes(workspace))


def device_status(workspace) -> int:
    st = C.c_int()
    _check(load().fftsp_device_status(_ptr(workspace), C.byref(st)), "fftsp_device_status")
    return st.value


def profile_enable(on: bool) -> None:
    _check(load().fftsp_profile_enable(1 if on else 0), "fftsp_profile_enable")


def profile_report() -> dict:
    """{kernel name: (calls, total milliseconds)} of the launches since profile_enable(True)"""
    need = load().fftsp_profile_report(None, 0)
    buf = C.create_string_buffer(need + 64)
    load().fftsp_profile_report(buf, len(buf))
    out = {}
    for line in buf.value.decode().splitlines():
        name, calls, ms = line.split()
        out[name] = (int(calls), float(ms))
    return out


def version() -> str:
    return load().fftsp_version().decode()
