"""Binding of libzc.so by ctypes, and by native code for the calls that a program makes often: argument marshalling only.

Buffers are torch tensors on the GPU (PyTorch is used for device memory and streams only);
the functions have the names and argument order of include/zc.h.  There is no CPU fallback:
if the HIP library has not been built, loading it raises.
"""
import ctypes as C
import importlib.util
import os
import sysconfig
from array import array

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libzc.so")

ZC_OK, ZC_ERR_ARG, ZC_ERR_CAPACITY, ZC_ERR_FORMAT, ZC_ERR_NONFINITE, ZC_ERR_RANGE, ZC_ERR_BOUND, \
    ZC_ERR_MISMATCH, ZC_ERR_HIP = range(9)
ZC_MAX_K = 64

ZC_STREAM_PLAIN, ZC_TILES_BY_TICKET, ZC_CHAINS_COHERENT = 1, 2, 4

EXPORTS = [
    "zc_compress_bound", "zc_compress_bound_ex", "zc_workspace_bytes", "zc_compress", "zc_compress_ex", "zc_compress_noalloc",
    "zc_compress_part", "zc_decompress", "zc_decompress_ex", "zc_decompress_many", "zc_reduce_compressed",
    "zc_reduce_compressed_ex", "zc_reduce_compressed_op", "zc_reduce_compressed_part", "zc_reduce_step_part", "zc_reduce_step", "zc_reduce_step_op", "zc_decompress_average", "zc_decompress_range",
    "zc_quality", "zc_finish", "zc_peek_header", "zc_strerror", "zc_debug_quantize", "zc_debug_block_offsets", "zc_debug_stream",
    "zc_profile_enable", "zc_profile_collect",
    "zc_adamw", "zc_adamw_state_bytes", "zc_mx_codes_stride", "zc_mx_scales_stride", "zc_mx_quantize", "zc_mx_dequantize", "zc_mx_workspace_bytes",
    "zc_mx_product", "zc_mx_linear",
    "zc_layer_norm", "zc_layer_norm_workspace_bytes", "zc_layer_norm_backward", "zc_embedding", "zc_embedding_workspace_bytes", "zc_embedding_backward",
    "zc_muon", "zc_muon_state_bytes", "zc_muon_workspace_bytes",
]

_lib = None
_native = None       # csrc/zc_calls.cpp: the same calls for arguments of the plainest form (NotImplemented for others), once libzc.so is loaded
_native_layers = None    # csrc/zc_layer_calls.cpp, likewise for the layer calls


class ZcError(RuntimeError):
    def __init__(self, status, what):
        super().__init__(f"{what}: {zc_strerror(status)} (status {status})")
        self.status = status


def lib():
    """Loads libzc.so (built by paper_2502_18554_amd/build.py); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} not found: build it with `python -m paper_2502_18554_amd.build` "
                               "(there is no CPU fallback)")
        L = C.CDLL(_LIB_PATH)
        vp, sz, szp = C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)
        u = C.c_uint
        L.zc_compress_bound.restype = sz
        L.zc_compress_bound.argtypes = [sz]
        L.zc_compress_bound_ex.restype = sz
        L.zc_compress_bound_ex.argtypes = [sz, u]
        L.zc_workspace_bytes.restype = sz
        L.zc_workspace_bytes.argtypes = [sz, C.c_int]
        L.zc_compress.argtypes = [vp, sz, C.c_float, vp, sz, szp, vp, sz, vp]
        L.zc_compress_ex.argtypes = [vp, sz, C.c_float, vp, sz, szp, vp, sz, vp, u]
        L.zc_compress_noalloc.argtypes = [vp, sz, C.c_float, vp, sz, szp, vp]
        L.zc_compress_part.argtypes = [vp, sz, C.c_float, sz, sz, vp, sz, szp, vp, sz, vp, u]
        L.zc_decompress.argtypes = [vp, sz, vp, sz, szp, vp, sz, vp]
        L.zc_decompress_ex.argtypes = [vp, sz, vp, sz, szp, vp, sz, vp, u]
        L.zc_reduce_compressed.argtypes = [vp, vp, C.c_int, vp, sz, szp, vp, sz, vp]
        L.zc_reduce_compressed_ex.argtypes = [vp, vp, C.c_int, vp, sz, szp, vp, sz, vp, u]
        L.zc_reduce_compressed_op.argtypes = [vp, vp, C.c_int, C.c_int, vp, sz, szp, vp, sz, vp, u]
        L.zc_reduce_compressed_part.argtypes = [vp, vp, C.c_int, sz, sz, sz, vp, sz, szp, vp, sz, vp, u]
        L.zc_reduce_step_part.argtypes = [vp, sz, vp, sz, C.c_int, sz, sz, vp, sz, szp, vp, sz, vp, u]
        L.zc_reduce_step.argtypes = [vp, sz, vp, sz, vp, sz, szp, vp, sz, vp]
        L.zc_reduce_step_op.argtypes = [vp, sz, vp, sz, C.c_int, vp, sz, szp, vp, sz, vp, u]
        L.zc_decompress_average.argtypes = [vp, sz, vp, sz, szp, vp, sz, vp, u]
        L.zc_decompress_range.argtypes = [vp, sz, sz, sz, vp, sz, szp, vp, sz, vp, u]
        L.zc_quality.argtypes = [vp, vp, sz, C.POINTER(C.c_double), vp, sz, vp]
        L.zc_decompress_many.argtypes = [vp, vp, C.c_int, vp, vp, szp, vp, sz, vp, u]
        L.zc_finish.argtypes = [vp, szp, vp]
        L.zc_peek_header.argtypes = [vp, sz, szp, C.POINTER(C.c_float), C.POINTER(C.c_uint), szp, C.POINTER(C.c_uint), vp]
        L.zc_strerror.restype = C.c_char_p
        L.zc_strerror.argtypes = [C.c_int]
        L.zc_debug_quantize.argtypes = [vp, sz, C.c_float, vp, vp, sz, vp]
        L.zc_debug_block_offsets.argtypes = [vp, sz, vp, sz, vp, sz, vp, u]
        L.zc_debug_stream.argtypes = [vp, vp, sz, C.c_int, C.c_int, vp]
        i, d, u64 = C.c_int, C.c_double, C.c_uint64
        for name in ("zc_adamw_state_bytes", "zc_mx_codes_stride", "zc_mx_scales_stride", "zc_mx_workspace_bytes"):
            getattr(L, name).restype = sz
        L.zc_adamw_state_bytes.argtypes = [vp, i, i]
        L.zc_adamw.argtypes = [i, vp, vp, i, vp, i, vp, i, vp, sz, i, u64, d, d, d, d, d, vp, u64, vp]
        L.zc_mx_codes_stride.argtypes = L.zc_mx_scales_stride.argtypes = [sz]
        L.zc_mx_workspace_bytes.argtypes = [sz, sz, sz]
        L.zc_mx_quantize.argtypes = [vp, i, sz, sz, sz, vp, sz, vp, sz, vp, sz, vp, sz, vp]
        L.zc_mx_dequantize.argtypes = [vp, sz, vp, sz, sz, sz, vp, i, sz, vp]
        L.zc_mx_product.argtypes = [vp, sz, vp, sz, vp, sz, vp, sz, sz, sz, sz, vp, vp, i, sz, u, vp, sz, vp]
        L.zc_mx_linear.argtypes = [vp, i, sz, vp, sz, vp, sz, sz, sz, sz, vp, vp, i, sz, u, vp, sz, vp]
        for name in ("zc_layer_norm_workspace_bytes", "zc_embedding_workspace_bytes", "zc_muon_state_bytes", "zc_muon_workspace_bytes"):
            getattr(L, name).restype = sz
        L.zc_layer_norm_workspace_bytes.argtypes = [sz, sz]
        L.zc_layer_norm.argtypes = [vp, i, sz, sz, sz, vp, vp, i, d, vp, i, sz, vp, vp]
        L.zc_layer_norm_backward.argtypes = [vp, i, sz, vp, i, sz, vp, vp, i, sz, sz, vp, i, sz, vp, vp, i, u, vp, sz, vp]
        L.zc_embedding_workspace_bytes.argtypes = [sz, sz, sz]
        L.zc_embedding.argtypes = [vp, i, sz, sz, sz, vp, i, sz, d, vp, i, sz, vp]
        L.zc_embedding_backward.argtypes = [vp, i, sz, vp, i, sz, d, vp, i, sz, sz, sz, u, vp, sz, vp]
        L.zc_muon_state_bytes.argtypes = [i, vp, vp]
        L.zc_muon_workspace_bytes.argtypes = [i, vp, vp, u]
        L.zc_muon.argtypes = [i, vp, vp, vp, i, vp, i, vp, i, vp, sz, d, d, d, i, u, vp, vp, sz, vp]
        L.zc_profile_enable.argtypes = [C.c_int]
        L.zc_profile_collect.argtypes = [C.POINTER(C.c_float), C.POINTER(C.c_int), C.c_int]
        _lib = L
        _load_native(L)
    return _lib


def _module(name):
    """A module of native calls that was built for this Python, or None: ctypes takes its calls then."""
    path = os.path.join(_HERE, name + sysconfig.get_config_var("EXT_SUFFIX"))
    if not os.path.exists(path):
        return None
    try:
        spec = importlib.util.spec_from_file_location(name, path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError:              # one that does not load
        return None
    return module


def _load_native(L):
    global _native, _native_layers
    stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    native = _module("_zc_calls") if stream_of is not None else None
    if native is None:
        return
    calls = (L.zc_compress_ex, L.zc_decompress_ex, L.zc_reduce_compressed_op, L.zc_reduce_step_op, L.zc_decompress_many)
    native.setup(*(C.cast(f, C.c_void_p).value for f in calls), torch._C._cuda_getDevice, stream_of)
    _native = native
    layers = _module("_zc_layer_calls")
    if layers is None:
        return
    for name in ("setup_layers", "adamw", "quantize", "dequantize", "product", "linear"):      # (the native calls in one place)
        setattr(native, name, getattr(layers, name))
    layers.setup_streams(torch._C._cuda_getDevice, stream_of)
    calls = (L.zc_adamw, L.zc_mx_quantize, L.zc_mx_dequantize, L.zc_mx_product, L.zc_mx_linear)
    if layers.setup_layers(*(C.cast(f, C.c_void_p).value for f in calls), str(torch.__version__).split("+")[0]):
        _native_layers = layers
        layers.setup_training(*(C.cast(f, C.c_void_p).value for f in (L.zc_layer_norm, L.zc_layer_norm_backward, L.zc_embedding, L.zc_embedding_backward, L.zc_muon)))


# Small calls are bound by what happens here (a chunk of a few thousand values runs for 4 us).  Where ctypes takes a call, addresses go to
# it as plain integers, the current stream's handle is read without building a Stream object around it, and
# the result words exist only where a call waits for them.
def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _p(t):
    return t.data_ptr() if t is not None else None


# The lists of a call with k streams (any sequences of whole numbers, arrays and tensors among them), one behind the other in memory: the
# words and their address, k of them (8 * k bytes) a list.  (16 buffers of a few thousand values decompressed 11.5 us with a ctypes array for
# each list, now 9.0.)
def _lists(k, *lists):
    room = k if k > 1 else 1                     # (no streams are for the call to refuse)
    flat = []
    for values in lists:
        if not hasattr(values, "__len__"):
            values = [*values]
        missing = room - len(values)
        if missing < 0:
            raise IndexError("more entries than streams")
        flat.extend(values)                      # (not +=, by which an array is added to the entries)
        if missing:
            flat.extend([0] * missing)           # which the calls refuse
    try:
        words = array("Q", flat)
    except (TypeError, OverflowError):
        words = array("Q", [int(v) & 0xFFFFFFFFFFFFFFFF for v in flat])
    return words, words.buffer_info()[0]


def zc_strerror(status):
    return lib().zc_strerror(int(status)).decode()


def zc_compress_bound(n, flags=0):
    return int(lib().zc_compress_bound_ex(int(n), int(flags))) if flags else int(lib().zc_compress_bound(int(n)))


def zc_workspace_bytes(n_max, k_max=1):
    return int(lib().zc_workspace_bytes(int(n_max), int(k_max)))


def _size(t):
    return t.nbytes


def zc_compress(d_in, n, abs_eb, d_out, d_ws, sync=True, stream=None, out_cap=None, flags=0):
    """zc_compress, or zc_compress_ex with flags, which is the same with flags 0.
    Returns (status, total_bytes); total_bytes is None in the asynchronous form."""
    if _native:
        r = _native.compress(d_in, n, abs_eb, d_out, d_ws, sync, stream, out_cap, flags)
        if r is not NotImplemented:
            return r
    nbytes = C.c_size_t(0) if sync else None
    cap = _size(d_out) if out_cap is None else out_cap
    args = [_p(d_in), n, abs_eb, _p(d_out), cap, C.byref(nbytes) if sync else None, _p(d_ws), _size(d_ws), _stream(stream)]
    st = lib().zc_compress_ex(*args, int(flags)) if flags else lib().zc_compress(*args)
    return st, (nbytes.value if sync else None)


ZC_NOALLOC_MAX_N = 1 << 27


def zc_compress_noalloc(d_in, n, abs_eb, d_out, sync=True, stream=None, out_cap=None):
    """zc_compress on the library's own static workspace.  Returns (status, total_bytes)."""
    nbytes = C.c_size_t(0) if sync else None
    cap = _size(d_out) if out_cap is None else out_cap
    st = lib().zc_compress_noalloc(_p(d_in), n, abs_eb, _p(d_out), cap, C.byref(nbytes) if sync else None,
                                   _stream(stream))
    return st, (nbytes.value if sync else None)


def zc_compress_part(d_in, n, abs_eb, first_value, count, d_out, d_ws, sync=True, stream=None, out_cap=None, flags=0):
    """One part of a stream compressed in parts.  Returns (status, bytes of the stream final so far)."""
    nbytes = C.c_size_t(0) if sync else None
    cap = _size(d_out) if out_cap is None else out_cap
    st = lib().zc_compress_part(_p(d_in), int(n), float(abs_eb), int(first_value), int(count), _p(d_out), cap,
                                C.byref(nbytes) if sync else None, _p(d_ws), _size(d_ws), _stream(stream), int(flags))
    return st, (nbytes.value if sync else None)


def zc_decompress(d_in, in_bytes, d_out, d_ws, sync=True, stream=None, out_cap_elems=None, flags=0):
    """zc_decompress, or zc_decompress_ex with flags, which is the same with flags 0.
    Returns (status, n); n is None in the asynchronous form."""
    if _native:
        r = _native.decompress(d_in, in_bytes, d_out, d_ws, sync, stream, out_cap_elems, flags)
        if r is not NotImplemented:
            return r
    n = C.c_size_t(0)
    cap = (d_out.numel() if d_out is not None else 0) if out_cap_elems is None else out_cap_elems
    args = [_p(d_in), in_bytes, _p(d_out), cap, C.byref(n) if sync else None, _p(d_ws), _size(d_ws), _stream(stream)]
    st = lib().zc_decompress_ex(*args, int(flags)) if flags else lib().zc_decompress(*args)
    return st, (n.value if sync else None)


def zc_decompress_average(d_in, in_bytes, d_out, d_ws, sync=True, stream=None, out_cap_elems=None, flags=0):
    """zc_decompress with every value divided by the stream's nsum.  Returns (status, n)."""
    n = C.c_size_t(0)
    cap = (d_out.numel() if d_out is not None else 0) if out_cap_elems is None else out_cap_elems
    st = lib().zc_decompress_average(_p(d_in), in_bytes, _p(d_out), cap, C.byref(n) if sync else None,
                                     _p(d_ws), _size(d_ws), _stream(stream), int(flags))
    return st, (n.value if sync else None)


def zc_decompress_range(d_in, in_bytes, first_value, count, d_out, d_ws, sync=True, stream=None, out_cap_elems=None,
                        flags=0):
    """Values [first_value, first_value + count) of the stream into d_out.  Returns (status, n)."""
    n = C.c_size_t(0)
    cap = (d_out.numel() if d_out is not None else 0) if out_cap_elems is None else out_cap_elems
    st = lib().zc_decompress_range(_p(d_in), in_bytes, int(first_value), int(count), _p(d_out), cap,
                                   C.byref(n) if sync else None, _p(d_ws), _size(d_ws), _stream(stream), int(flags))
    return st, (n.value if sync else None)


def zc_reduce_compressed(d_chunks, chunk_bytes, d_out, d_ws, sync=True, stream=None, out_cap=None, flags=0):
    """zc_reduce_compressed, or zc_reduce_compressed_ex with flags: zc_reduce_compressed_op of a Sum is the same.
    d_chunks: list of device tensors holding the k operand streams.  Returns (status, total_bytes)."""
    if _native:
        r = _native.reduce(d_chunks, chunk_bytes, ZC_OP_SUM, d_out, d_ws, sync, stream, out_cap, flags)
        if r is not NotImplemented:
            return r
    k = len(d_chunks)
    lists, at = _lists(k, [t.data_ptr() for t in d_chunks], chunk_bytes)
    nbytes = C.c_size_t(0) if sync else None
    cap = _size(d_out) if out_cap is None else out_cap
    args = [at, at + 8 * k, k, _p(d_out), cap, C.byref(nbytes) if sync else None, _p(d_ws), _size(d_ws), _stream(stream)]
    st = lib().zc_reduce_compressed_ex(*args, int(flags)) if flags else lib().zc_reduce_compressed(*args)
    return st, (nbytes.value if sync else None)


def zc_reduce_compressed_op(d_chunks, chunk_bytes, op, d_out, d_ws, sync=True, stream=None, out_cap=None, flags=0):
    """zc_reduce_compressed for Sum, Max or Min (ZC_OP_*).  Returns (status, total_bytes)."""
    if _native:
        r = _native.reduce(d_chunks, chunk_bytes, op, d_out, d_ws, sync, stream, out_cap, flags)
        if r is not NotImplemented:
            return r
    k = len(d_chunks)
    lists, at = _lists(k, [t.data_ptr() for t in d_chunks], chunk_bytes)
    nbytes = C.c_size_t(0) if sync else None
    cap = _size(d_out) if out_cap is None else out_cap
    st = lib().zc_reduce_compressed_op(at, at + 8 * k, k, int(op), _p(d_out), cap, C.byref(nbytes) if sync else None, _p(d_ws),
                                       _size(d_ws), _stream(stream), int(flags))
    return st, (nbytes.value if sync else None)


def zc_reduce_compressed_part(d_chunks, chunk_bytes, n, first_value, count, d_out, d_ws, sync=True, stream=None, out_cap=None,
                              flags=0):
    """One part of a k-way Sum done in parts.  Returns (status, bytes of the stream final so far)."""
    k = len(d_chunks)
    lists, at = _lists(k, [t.data_ptr() for t in d_chunks], chunk_bytes)
    nbytes = C.c_size_t(0) if sync else None
    cap = _size(d_out) if out_cap is None else out_cap
    st = lib().zc_reduce_compressed_part(at, at + 8 * k, k, int(n), int(first_value), int(count), _p(d_out), cap,
                                         C.byref(nbytes) if sync else None, _p(d_ws), _size(d_ws), _stream(stream), int(flags))
    return st, (nbytes.value if sync else None)


def zc_reduce_step_part(d_chunk, chunk_bytes, d_local, n_local, op, first_value, count, d_out, d_ws, sync=True, stream=None,
                        out_cap=None, flags=0):
    """One part of a ring round done in parts.  Returns (status, bytes of the stream final so far)."""
    nbytes = C.c_size_t(0) if sync else None
    cap = _size(d_out) if out_cap is None else out_cap
    st = lib().zc_reduce_step_part(_p(d_chunk), int(chunk_bytes), _p(d_local), int(n_local), int(op), int(first_value),
                                   int(count), _p(d_out), cap, C.byref(nbytes) if sync else None, _p(d_ws), _size(d_ws),
                                   _stream(stream), int(flags))
    return st, (nbytes.value if sync else None)


def zc_decompress_many(d_chunks, chunk_bytes, d_outs, d_ws, sync=True, stream=None, out_cap_elems=None, flags=0):
    """d_chunks / d_outs: lists of k device tensors.  Returns (status, [n of every stream]) (None when not sync)."""
    if _native:
        r = _native.many(d_chunks, chunk_bytes, d_outs, d_ws, sync, stream, out_cap_elems, flags)
        if r is not NotImplemented:
            return r
    k = len(d_chunks)
    lists, at = _lists(k, [t.data_ptr() for t in d_chunks], chunk_bytes, [t.data_ptr() for t in d_outs],
                       [t.numel() for t in d_outs] if out_cap_elems is None else out_cap_elems)
    ns = (C.c_size_t * max(k, 1))() if sync else None
    st = lib().zc_decompress_many(at, at + 8 * k, k, at + 16 * k, at + 24 * k, ns, _p(d_ws), _size(d_ws),
                                  _stream(stream), int(flags))
    return st, ([int(ns[i]) for i in range(k)] if sync else None)


ZC_OP_SUM, ZC_OP_MAX, ZC_OP_MIN = 0, 1, 2


def zc_reduce_step(d_chunk, chunk_bytes, d_local, n_local, d_out, d_ws, sync=True, stream=None, out_cap=None, flags=0):
    """One ring round: received stream + local fp32 values -> stream of the sums: zc_reduce_step, or with flags zc_reduce_step_op of a Sum, which is
    the same with flags 0.  Returns (status, total_bytes)."""
    if flags or _native:
        return zc_reduce_step_op(d_chunk, chunk_bytes, d_local, n_local, ZC_OP_SUM, d_out, d_ws, sync, stream, out_cap, flags)
    nbytes = C.c_size_t(0) if sync else None
    cap = _size(d_out) if out_cap is None else out_cap
    st = lib().zc_reduce_step(_p(d_chunk), int(chunk_bytes), _p(d_local), int(n_local), _p(d_out), cap,
                              C.byref(nbytes) if sync else None, _p(d_ws), _size(d_ws), _stream(stream))
    return st, (nbytes.value if sync else None)


def zc_reduce_step_op(d_chunk, chunk_bytes, d_local, n_local, op, d_out, d_ws, sync=True, stream=None, out_cap=None,
                      flags=0):
    """zc_reduce_step for Sum, Max or Min.  Returns (status, total_bytes)."""
    if _native:
        r = _native.step(d_chunk, chunk_bytes, d_local, n_local, op, d_out, d_ws, sync, stream, out_cap, flags)
        if r is not NotImplemented:
            return r
    nbytes = C.c_size_t(0) if sync else None
    cap = _size(d_out) if out_cap is None else out_cap
    st = lib().zc_reduce_step_op(_p(d_chunk), int(chunk_bytes), _p(d_local), int(n_local), int(op), _p(d_out), cap,
                                 C.byref(nbytes) if sync else None, _p(d_ws), _size(d_ws), _stream(stream), int(flags))
    return st, (nbytes.value if sync else None)


def zc_quality(d_ref, d_test, n, d_ws, stream=None):
    """Returns (status, [max |ref - test|, sum of squared differences, min(ref), max(ref)])."""
    out = (C.c_double * 4)()
    st = lib().zc_quality(_p(d_ref), _p(d_test), int(n), out, _p(d_ws), d_ws.numel() * d_ws.element_size(),
                          _stream(stream))
    return st, [float(v) for v in out]


def zc_finish(d_ws, stream=None):
    """Returns (status, size result) of the last asynchronous call that used d_ws."""
    r = C.c_size_t(0)      # d_ws None: the call was zc_compress_noalloc
    st = lib().zc_finish(_p(d_ws), C.byref(r), _stream(stream))
    return st, r.value


def zc_peek_header(d_in, in_bytes, stream=None):
    """Returns (status, n, abs_eb, nsum, total_bytes, flags of the stream's variant)."""
    n, eb, nsum, total, flags = C.c_size_t(0), C.c_float(0), C.c_uint(0), C.c_size_t(0), C.c_uint(0)
    st = lib().zc_peek_header(_p(d_in), in_bytes, C.byref(n), C.byref(eb), C.byref(nsum), C.byref(total),
                              C.byref(flags), _stream(stream))
    return st, n.value, eb.value, nsum.value, total.value, flags.value


def zc_debug_quantize(d_in, n, abs_eb, d_q, d_ws, stream=None):
    return lib().zc_debug_quantize(_p(d_in), n, abs_eb, _p(d_q), _p(d_ws), _size(d_ws), _stream(stream))


def zc_debug_block_offsets(d_in, in_bytes, d_off_words, d_ws, stream=None, flags=0):
    return lib().zc_debug_block_offsets(_p(d_in), in_bytes, _p(d_off_words), d_off_words.numel(), _p(d_ws),
                                        _size(d_ws), _stream(stream), int(flags))


def zc_debug_stream(d_in, d_out, tiles, loads, stores, stream=None):
    """A kernel that only streams: workgroup t reads loads x 8 KiB of d_in and writes stores x 8 KiB of d_out."""
    return lib().zc_debug_stream(_p(d_in) if d_in is not None else None, _p(d_out) if d_out is not None else None,
                                 int(tiles), int(loads), int(stores), _stream(stream))


KERNEL_NAMES = {1: "compress", 2: "decompress", 3: "reduce", 4: "reduce_step", 5: "stream"}


def zc_profile_enable(on, only=None):
    """Times the main kernels from now on (on=True), or stops (False).  only: names from KERNEL_NAMES to time just those."""
    if on and only:
        code = sum(1 << k for k, name in KERNEL_NAMES.items() if name in only)
        return lib().zc_profile_enable(code)
    return lib().zc_profile_enable(1 if on else 0)


def zc_profile_collect(cap=65536):
    """Returns [(kernel name, milliseconds)] for the main kernels launched since zc_profile_enable(True)."""
    ms = (C.c_float * cap)()
    kind = (C.c_int * cap)()
    count = lib().zc_profile_collect(ms, kind, cap)
    if count < 0:
        raise ZcError(-count, "zc_profile_collect")
    return [(KERNEL_NAMES.get(kind[i], str(kind[i])), float(ms[i])) for i in range(count)]


# ---- The calls around the collective.  Sizes, types and strides are the tensors' own; what does not fit together, or is not on the GPU, is ZC_ERR_ARG.

ZC_F32, ZC_BF16, ZC_F16 = 0, 1, 2
ZC_MX_ADD = 1
_TYPES = {torch.float32: ZC_F32, torch.bfloat16: ZC_BF16, torch.float16: ZC_F16}


def _words(values):
    words = array("Q", values)
    return words, words.buffer_info()[0] if words else None


def zc_adamw_state_bytes(counts, state_bits=32):
    """Bytes of the state of tensors with these numbers of values; 0 for what there is no state of."""
    words, at = _words([int(n) for n in counts])
    return int(lib().zc_adamw_state_bytes(at, len(words), int(state_bits)))


def _one_type(tensors):
    kinds = {t.dtype for t in tensors}
    return _TYPES.get(kinds.pop(), -1) if len(kinds) == 1 else ZC_F32 if not kinds else -1


def _own_bytes(t):
    """Whether a state or a workspace is None or on the GPU in one piece: of a tensor with strides the bytes lie elsewhere, or are not all there."""
    return t is None or (t.is_cuda and t.is_contiguous())


def zc_adamw(d_params, d_grads, d_state, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, state_bits=32, seed=0, d_copies=None,
             d_grad_scale=None, stream=None):
    """One AdamW step over the tensors of the list d_params (contiguous, of one type; d_grads: as many of the same sizes, of one type), in place.
    d_copies: None, or a list with a tensor or None for each.  Returns the status."""
    lib()
    if _native_layers:
        r = _native_layers.adamw(d_params, d_grads, d_state, step, lr, beta1, beta2, eps, weight_decay, state_bits, seed, d_copies, d_grad_scale, stream)
        if r is not NotImplemented:
            return r
    k = len(d_params)
    if len(d_grads) != k or (d_copies is not None and len(d_copies) != k):
        return ZC_ERR_ARG
    copies = [] if d_copies is None else [t for t in d_copies if t is not None]
    sizes = [t.numel() for t in d_params]
    if [t.numel() for t in d_grads] != sizes or not all(t.is_contiguous() and t.is_cuda for t in (*d_params, *d_grads, *copies)) or \
            any(t is not None and t.numel() != n for t, n in zip(d_copies or (), sizes)) or \
            not _own_bytes(d_state) or not (d_grad_scale is None or d_grad_scale.is_cuda) or (d_grad_scale is not None and (d_grad_scale.dtype != torch.float32 or d_grad_scale.numel() != 1)):
        return ZC_ERR_ARG
    lists = [_words(sizes), _words([t.data_ptr() for t in d_params]), _words([t.data_ptr() for t in d_grads]),
             _words([t.data_ptr() if t is not None else 0 for t in d_copies]) if d_copies is not None else (None, None)]
    if not 0 <= int(step) < 1 << 64 or not 0 <= int(seed) < 1 << 64:
        return ZC_ERR_ARG
    return lib().zc_adamw(k, lists[0][1], lists[1][1], _one_type(d_params), lists[2][1], _one_type(d_grads), lists[3][1], _one_type(copies),
                          _p(d_state), _size(d_state) if d_state is not None else 0, int(state_bits), int(step), float(lr), float(beta1),
                          float(beta2), float(eps), float(weight_decay), _p(d_grad_scale), int(seed), _stream(stream))


def zc_mx_codes_stride(cols):
    return int(lib().zc_mx_codes_stride(int(cols)))


def zc_mx_scales_stride(cols):
    return int(lib().zc_mx_scales_stride(int(cols)))


def zc_mx_workspace_bytes(m, n, k):
    return int(lib().zc_mx_workspace_bytes(int(m), int(n), int(k)))


def _matrix(t):
    """(address, type, rows, columns, values from row to row), or None for what is no matrix with its rows' values side by side."""
    if t.dim() != 2 or t.dtype not in _TYPES or not t.is_cuda:
        return None
    (rows, cols), (stride, one) = t.shape, t.stride()
    if (cols > 1 and one != 1) or stride < 0:
        return None
    return t.data_ptr(), _TYPES[t.dtype], rows, cols, stride if rows > 1 else max(cols, stride)


def _held(codes, scales, rows):
    """(address, bytes from row to row) of the codes and of the scale bytes of a matrix of so many rows, or None."""
    found = []
    for t in (codes, scales):
        if t.dim() != 2 or t.dtype != torch.uint8 or not t.is_cuda or t.shape[0] != rows or (t.shape[1] > 1 and t.stride(1) != 1):
            return None
        if rows > 1 and t.stride(0) < t.shape[1]:
            return None
        found += [t.data_ptr(), t.stride(0) if rows > 1 else t.shape[1]]
    return found


def _covers(codes, scales, cols):
    """Whether rows of codes and scale bytes have room for so many values."""
    blocks = -(-cols // 32)
    return codes.dim() == scales.dim() == 2 and codes.shape[1] >= 16 * blocks and scales.shape[1] >= blocks


def zc_mx_quantize(d_in, d_codes, d_scales, d_codes_t=None, d_scales_t=None, stream=None):
    """A matrix (its rows may lie apart) into 4-bit blocks along its rows (d_codes, d_scales: uint8 matrices with a row for each), along its columns
    (d_codes_t, d_scales_t: a row for each column), or both.  Returns the status."""
    lib()
    if _native_layers:
        r = _native_layers.quantize(d_in, d_codes, d_scales, d_codes_t, d_scales_t, stream)
        if r is not NotImplemented:
            return r
    x = _matrix(d_in)
    if x is None:
        return ZC_ERR_ARG
    held = []
    for codes, scales, rows, cols in ((d_codes, d_scales, x[2], x[3]), (d_codes_t, d_scales_t, x[3], x[2])):
        if codes is None and scales is None:
            held += [None, 0, None, 0]
            continue
        if codes is None or scales is None or not _covers(codes, scales, cols):
            return ZC_ERR_ARG
        one = _held(codes, scales, rows)
        if one is None:
            return ZC_ERR_ARG
        held += one
    return lib().zc_mx_quantize(*x, *held, _stream(stream))


def zc_mx_dequantize(d_codes, d_scales, d_out, stream=None):
    """What the blocks stand for, into the matrix d_out.  Returns the status."""
    lib()
    if _native_layers:
        r = _native_layers.dequantize(d_codes, d_scales, d_out, stream)
        if r is not NotImplemented:
            return r
    out = _matrix(d_out)
    held = out and _held(d_codes, d_scales, out[2])
    if not held or not _covers(d_codes, d_scales, out[3]):
        return ZC_ERR_ARG
    return lib().zc_mx_dequantize(*held, out[2], out[3], out[0], out[1], out[4], _stream(stream))


def _product_end(d_w_codes, d_w_scales, k, d_out, d_bias):
    """The operand b, the output and the bias of a product, checked against each other; None where they do not fit."""
    out = _matrix(d_out)
    if out is None or not _covers(d_w_codes, d_w_scales, k):
        return None
    held = _held(d_w_codes, d_w_scales, out[3])
    if held is None or (d_bias is not None and (d_bias.dtype != torch.float32 or not d_bias.is_cuda or d_bias.numel() != out[3] or not d_bias.is_contiguous())):
        return None
    return out, held


def zc_mx_product(d_a_codes, d_a_scales, d_b_codes, d_b_scales, k, d_out, d_ws, d_bias=None, add=False, stream=None):
    """d_out (m x n) = a (m rows of k values, in blocks) times b (n rows) transposed, + d_bias, + d_out itself with add; d_ws may be None.  Returns the status."""
    lib()
    if _native_layers:
        r = _native_layers.product(d_a_codes, d_a_scales, d_b_codes, d_b_scales, k, d_out, d_ws, d_bias, add, stream)
        if r is not NotImplemented:
            return r
    k = int(k)
    end = _product_end(d_b_codes, d_b_scales, k, d_out, d_bias)
    a = end and _held(d_a_codes, d_a_scales, end[0][2])
    if not a or not _covers(d_a_codes, d_a_scales, k) or not _own_bytes(d_ws):
        return ZC_ERR_ARG
    out, b = end
    return lib().zc_mx_product(*a, *b, out[2], out[3], k, _p(d_bias), out[0], out[1], out[4], ZC_MX_ADD if add else 0, _p(d_ws),
                               _size(d_ws) if d_ws is not None else 0, _stream(stream))


def zc_mx_linear(d_x, d_w_codes, d_w_scales, d_out, d_ws, d_bias=None, add=False, stream=None):
    """d_out (m x n) = d_x (m x k values, quantised by the call) times the weights (n rows of k values, in blocks) transposed, + d_bias, + d_out itself
    with add.  Returns the status."""
    lib()
    if _native_layers:
        r = _native_layers.linear(d_x, d_w_codes, d_w_scales, d_out, d_ws, d_bias, add, stream)
        if r is not NotImplemented:
            return r
    x = _matrix(d_x)
    end = x and _product_end(d_w_codes, d_w_scales, x[3], d_out, d_bias)
    if not end or end[0][2] != x[2] or not _own_bytes(d_ws):
        return ZC_ERR_ARG
    out, w = end
    return lib().zc_mx_linear(x[0], x[1], x[4], *w, out[2], out[3], x[3], _p(d_bias), out[0], out[1], out[4], ZC_MX_ADD if add else 0, _p(d_ws),
                              _size(d_ws) if d_ws is not None else 0, _stream(stream))


# ---- The other calls of a training step.  Tensors are on torch's current device, whose current stream a call without one goes to.

ZC_ADD, ZC_ADD_WEIGHTS = 1, 2
ZC_MUON_NESTEROV, ZC_MUON_MATCH_RMS, ZC_MUON_WIDE = 1, 2, 4
_TOKENS = {torch.int32: 32, torch.int64: 64}


def _here(*tensors):
    """Whether all of these that are there are on the current device."""
    there = [t for t in tensors if t is not None]
    return all(t.is_cuda for t in there) and (not there or {t.device.index for t in there} == {torch._C._cuda_getDevice()})


def _vectors(n, *tensors):
    """(type, addresses) of tensors, or None for each, of n values in one piece and of one type; None for others."""
    there = [t for t in tensors if t is not None]
    if not all(t.is_cuda and t.is_contiguous() and t.numel() == n for t in there) or (there and _one_type(there) < 0):
        return None
    return (_one_type(there), *(_p(t) for t in tensors))


def _alike(a, b):
    return a is not None and b is not None and a[2:4] == b[2:4]


def zc_layer_norm_workspace_bytes(rows, cols):
    return int(lib().zc_layer_norm_workspace_bytes(int(rows), int(cols)))


def zc_layer_norm(d_x, d_w, d_b, d_out, d_stats=None, eps=1e-5, stream=None):
    """d_out = the layer norm of the rows of d_x, with weights and bias (contiguous, of one type, either may be None); d_stats: 2 x rows binary32 values
    for the backward pass, or None.  d_out may be d_x.  Returns the status."""
    lib()
    if _native_layers:
        r = _native_layers.layer_norm(d_x, d_w, d_b, d_out, d_stats, eps, stream)
        if r is not NotImplemented:
            return r
    x, out = _matrix(d_x), _matrix(d_out)
    if not _alike(x, out) or not _here(d_x, d_w, d_b, d_out, d_stats):
        return ZC_ERR_ARG
    weights, stats = _vectors(x[3], d_w, d_b), _vectors(2 * x[2], d_stats)
    if weights is None or stats is None or stats[0] != ZC_F32:
        return ZC_ERR_ARG
    return lib().zc_layer_norm(*x, weights[1], weights[2], weights[0], float(eps), out[0], out[1], out[4], stats[1], _stream(stream))


def zc_layer_norm_backward(d_dy, d_x, d_stats, d_w, d_dx, d_dw, d_db, d_ws, add=False, add_weights=False, stream=None):
    """The gradients of zc_layer_norm's input, weights and bias (d_dx, d_dw, d_db: any may be None) from that of its output; add: d_dx is added to, add_weights: d_dw and
    d_db are.  Returns the status."""
    lib()
    if _native_layers:
        r = _native_layers.layer_norm_backward(d_dy, d_x, d_stats, d_w, d_dx, d_dw, d_db, d_ws, add, add_weights, stream)
        if r is not NotImplemented:
            return r
    dy, x, dx = _matrix(d_dy), _matrix(d_x), _matrix(d_dx) if d_dx is not None else None
    if not _alike(dy, x) or (d_dx is not None and not _alike(dx, x)) or d_stats is None or not _here(d_dy, d_x, d_stats, d_w, d_dx, d_dw, d_db, d_ws) or not _own_bytes(d_ws):
        return ZC_ERR_ARG
    weights, stats, sums = _vectors(x[3], d_w), _vectors(2 * x[2], d_stats), _vectors(x[3], d_dw, d_db)
    if weights is None or stats is None or sums is None or stats[0] != ZC_F32:
        return ZC_ERR_ARG
    return lib().zc_layer_norm_backward(dy[0], dy[1], dy[4], x[0], x[1], x[4], stats[1], weights[1], weights[0], x[2], x[3], *((dx[0], dx[1], dx[4]) if dx else (None, ZC_F32, 0)),
                                        sums[1], sums[2], sums[0], (ZC_ADD if add else 0) | (ZC_ADD_WEIGHTS if add_weights else 0), _p(d_ws),
                                        _size(d_ws) if d_ws is not None else 0, _stream(stream))


def _tokens(t, rows):
    """(address, bits) of as many tokens as there are rows, or None."""
    if t.dtype not in _TOKENS or not t.is_cuda or not t.is_contiguous() or t.numel() != rows:
        return None
    return t.data_ptr(), _TOKENS[t.dtype]


def zc_embedding(d_table, d_tokens, d_out, scale=1.0, stream=None):
    """d_out (a row for each token) = scale times the tokens' rows of d_table, zeros for tokens outside it.  d_tokens: int32 or int64, of any shape, contiguous.  Returns the status."""
    lib()
    if _native_layers:
        r = _native_layers.embedding(d_table, d_tokens, d_out, scale, stream)
        if r is not NotImplemented:
            return r
    table, out = _matrix(d_table), _matrix(d_out)
    tokens = out and _tokens(d_tokens, out[2])
    if not table or not tokens or table[3] != out[3] or not _here(d_table, d_tokens, d_out):
        return ZC_ERR_ARG
    return lib().zc_embedding(*table, *tokens, out[2], float(scale), out[0], out[1], out[4], _stream(stream))


def zc_embedding_workspace_bytes(n, table_rows, cols):
    return int(lib().zc_embedding_workspace_bytes(int(n), int(table_rows), int(cols)))


def zc_embedding_backward(d_dy, d_tokens, d_grad, d_ws, scale=1.0, add=False, stream=None):
    """d_grad (a row for each of the table's) = scale times the sums of the rows of d_dy by token, or that added to what it holds.  Returns the status."""
    lib()
    if _native_layers:
        r = _native_layers.embedding_backward(d_dy, d_tokens, d_grad, d_ws, scale, add, stream)
        if r is not NotImplemented:
            return r
    dy, grad = _matrix(d_dy), _matrix(d_grad)
    tokens = dy and _tokens(d_tokens, dy[2])
    if not grad or not tokens or dy[3] != grad[3] or not _here(d_dy, d_tokens, d_grad, d_ws) or not _own_bytes(d_ws):
        return ZC_ERR_ARG
    return lib().zc_embedding_backward(dy[0], dy[1], dy[4], *tokens, dy[2], float(scale), grad[0], grad[1], grad[2], grad[3], grad[4], ZC_ADD if add else 0, _p(d_ws),
                                       _size(d_ws) if d_ws is not None else 0, _stream(stream))


def _shapes(shapes):
    rows, cols = _words([int(r) for r, _ in shapes]), _words([int(c) for _, c in shapes])
    return len(shapes), rows, cols


def zc_muon_state_bytes(shapes):
    """Bytes of the state of matrices with these (rows, columns); 0 for what there is no state of."""
    k, rows, cols = _shapes(shapes)
    return int(lib().zc_muon_state_bytes(k, rows[1], cols[1]))


def zc_muon_workspace_bytes(shapes, wide=False):
    k, rows, cols = _shapes(shapes)
    return int(lib().zc_muon_workspace_bytes(k, rows[1], cols[1], ZC_MUON_WIDE if wide else 0))


def zc_muon(d_params, d_grads, d_state, d_ws, lr, momentum=0.95, weight_decay=0.0, iterations=5, nesterov=True, match_rms=False, wide=False, d_copies=None, d_grad_scale=None,
            stream=None):
    """One step with orthogonalised momentum over the matrices of the list d_params (contiguous, of one type; d_grads: as many of the same shapes, of one type), in
    place.  d_copies: None, or a list with a matrix or None for each; one that is the matrix of d_params itself, as .to() of its own type gives, is left out.  Returns the status."""
    lib()
    flags = (ZC_MUON_NESTEROV if nesterov else 0) | (ZC_MUON_MATCH_RMS if match_rms else 0) | (ZC_MUON_WIDE if wide else 0)
    if _native_layers:
        r = _native_layers.muon(d_params, d_grads, d_state, d_ws, lr, momentum, weight_decay, iterations, flags, d_copies, d_grad_scale, stream)
        if r is not NotImplemented:
            return r
    k = len(d_params)
    if len(d_grads) != k or (d_copies is not None and len(d_copies) != k):
        return ZC_ERR_ARG
    copies = [] if d_copies is None else [t for t in d_copies if t is not None]
    shapes = [tuple(t.shape) for t in d_params]
    if any(len(s) != 2 for s in shapes) or [tuple(t.shape) for t in d_grads] != shapes or not all(t.is_contiguous() for t in (*d_params, *d_grads, *copies)) or \
            any(t is not None and tuple(t.shape) != s for t, s in zip(d_copies or (), shapes)) or not _here(*d_params, *d_grads, *copies, d_state, d_ws, d_grad_scale) or \
            not _own_bytes(d_state) or not _own_bytes(d_ws) or (d_grad_scale is not None and (d_grad_scale.dtype != torch.float32 or d_grad_scale.numel() != 1)):
        return ZC_ERR_ARG
    _, rows, cols = _shapes(shapes)
    lists = [_words([t.data_ptr() for t in d_params]), _words([t.data_ptr() for t in d_grads]),
             _words([0 if t is None or (t.dtype == p.dtype and t.data_ptr() == p.data_ptr()) else t.data_ptr() for t, p in zip(d_copies, d_params)]) if d_copies is not None else (None, None)]
    if not 0 <= int(iterations) < 1 << 31:
        return ZC_ERR_ARG
    return lib().zc_muon(k, rows[1], cols[1], lists[0][1], _one_type(d_params), lists[1][1], _one_type(d_grads), lists[2][1], _one_type(copies), _p(d_state),
                         _size(d_state) if d_state is not None else 0, float(lr), float(momentum), float(weight_decay), int(iterations), flags, _p(d_grad_scale), _p(d_ws),
                         _size(d_ws) if d_ws is not None else 0, _stream(stream))
