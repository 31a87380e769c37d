"""Thin ctypes binding of ``csrc/libbwta.so`` (the C ABI declared in ``include/bwta.h``).

Argument marshalling only: every step of the path runs in the HIP kernels.  Tensors are
torch CUDA tensors used as device buffers; the current torch stream is passed through.
The calls a program makes per layer are marshalled by ``csrc/binding_native.cpp`` where they come in
their ordinary form (device tensors, Python integers, the current stream); the functions below say
what every other form does.
Importing this module without the compiled library raises -- there is no fallback.  Without the native marshalling it
warns and makes every call in its Python form.
"""
import ctypes
import importlib.machinery
import importlib.util
import os
import struct
import sys
import warnings

# torch ships its own HIP runtime; load it first so that libbwta.so binds to the same runtime
# (same SONAME) instead of bringing a second one into the process.
import torch  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
# BWTA_LIB: load this build of the same sources instead (the sanitizer test's host-instrumented one)
LIB_PATH = os.environ.get("BWTA_LIB") or os.path.join(_HERE, "csrc", "libbwta.so")
NATIVE_PATH = os.path.join(_HERE, "csrc", "_bwta_native.so")

OK = 0
ERR_NULL, ERR_SHAPE, ERR_ALIGN, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP, ERR_TOO_LARGE = -1, -2, -3, -4, -5, -6, -7
DTYPE_FP16, DTYPE_INT8, DTYPE_BF16 = 0, 1, 2
SCALE_NONE, SCALE_SCALAR, SCALE_VECTOR = 0, 1, 2
PATH_AUTO, PATH_POPC, PATH_MFMA, PATH_FP4 = 0, 1, 2, 3
PREPARED_PLANES, PREPARED_FP4 = 1, 2
KERNEL_GEMV_POPC, KERNEL_GEMV_FP4, KERNEL_GEMM_FP4, KERNEL_GEMM_MFMA_I8, KERNEL_GEMM_POPC = 1, 2, 3, 4, 5
KERNEL_LINEAR_FUSED, KERNEL_LINEAR_STRIP, KERNEL_LINEAR_ONE, KERNEL_LINEAR_ROWS = 6, 7, 8, 9
OPERAND_FP16 = 3

EXPORTS = ["bwta_plane_row_words", "bwta_workspace_bytes", "bwta_quantize_pack_act",
           "bwta_pack_weights", "bwta_gemm", "bwta_linear", "bwta_linear_static", "bwta_static_scratch_bytes",
           "bwta_static_scratch_init", "bwta_strerror", "bwta_last_hip_error",
           "bwta_build_id", "bwta_set_path", "bwta_get_path", "bwta_auto_path", "bwta_linear_launches", "bwta_linear_call", "bwta_version",
           "bwta_set_tile", "bwta_planned_tile", "bwta_planned_wide", "bwta_planned_wide_prepared", "bwta_planned_rows", "bwta_planned_decode_blocks",
           "bwta_prepared_bytes", "bwta_prepared_format", "bwta_planned_kernel", "bwta_prepare_act", "bwta_gemm_prepared", "bwta_gemm_grouped",
           "bwta_quantize_pack_bool", "bwta_matmul_tt", "bwta_prepare_weights", "bwta_act_scale",
           "bwta_prepare_act_autoscale", "bwta_matmul_bool_prepared", "bwta_head_norm_rope", "bwta_cache_write", "bwta_cache_read",
           "bwta_cache_attention", "bwta_cache_attention_workspace_bytes"]

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "%s is missing: build it first (python -c 'import __graft_entry__ as g; g.build()' "
        "or python paper_2604_03957_amd/build.py); there is no CPU fallback" % LIB_PATH)

_lib = ctypes.CDLL(LIB_PATH)
_c = ctypes
_P = _c.c_void_p
_lib.bwta_plane_row_words.restype = _c.c_int64
_lib.bwta_plane_row_words.argtypes = [_c.c_int]
_lib.bwta_workspace_bytes.restype = _c.c_size_t
_lib.bwta_workspace_bytes.argtypes = [_c.c_int, _c.c_int, _c.c_int]
_lib.bwta_quantize_pack_act.restype = _c.c_int
_lib.bwta_quantize_pack_act.argtypes = [_P, _c.c_int, _c.c_int64, _P, _c.c_int, _c.c_int, _c.c_int,
                                        _P, _P, _P, _P]
_lib.bwta_pack_weights.restype = _c.c_int
_lib.bwta_pack_weights.argtypes = [_P, _c.c_int, _c.c_int64, _c.c_int, _c.c_int, _P, _P]
_lib.bwta_gemm.restype = _c.c_int
_lib.bwta_gemm.argtypes = [_P, _P, _P, _c.c_int, _c.c_int, _c.c_int, _P, _c.c_int, _P, _c.c_int,
                           _P, _P, _c.c_int64, _P, _c.c_size_t, _P]
_lib.bwta_linear.restype = _c.c_int
_lib.bwta_linear.argtypes = [_P, _c.c_int64, _P, _c.c_int, _P, _P, _c.c_int, _c.c_int, _c.c_int,
                             _c.c_int, _P, _c.c_int64, _P, _c.c_size_t, _P]
# the same call with its arguments packed into one block (15 ctypes conversions cost more): addresses given as integers,
# which the native marshalling leaves to this form
_linear_call = _lib.bwta_linear_call
_linear_call.restype = _c.c_int
_linear_call.argtypes = [_c.c_char_p]
_linear_args = struct.Struct("=QqQQQQqQQQiiiiii")  # bwta_linear_args of bwta_tuning.h
_linear_pack, _LINEAR_ARGS_SIZE = _linear_args.pack, _linear_args.size
_lib.bwta_linear_static.restype = _c.c_int
_lib.bwta_linear_static.argtypes = [_P, _c.c_int64, _P, _c.c_int, _P, _P, _c.c_int, _c.c_int, _c.c_int,
                                    _c.c_int, _P, _c.c_int64, _P]
_lib.bwta_static_scratch_bytes.restype = _c.c_size_t
_lib.bwta_static_scratch_init.restype = _c.c_int
_lib.bwta_prepared_bytes.restype = _c.c_size_t
_lib.bwta_prepared_bytes.argtypes = [_c.c_int, _c.c_int]
_lib.bwta_prepare_act.restype = _c.c_int
_lib.bwta_planned_kernel.restype = _c.c_int
_lib.bwta_planned_kernel.argtypes = [_c.c_int, _c.c_int, _c.c_int, _c.c_int]
_lib.bwta_prepared_format.restype = _c.c_int
_lib.bwta_prepared_format.argtypes = [_c.c_int, _c.c_int]
_lib.bwta_prepare_act.argtypes = [_P, _c.c_int64, _P, _c.c_int, _c.c_int, _c.c_int, _P, _c.c_size_t,
                                  _c.POINTER(_c.c_int), _P]
_lib.bwta_gemm_prepared.restype = _c.c_int
_lib.bwta_gemm_prepared.argtypes = [_P, _c.c_size_t, _c.c_int, _P, _c.c_int, _c.c_int, _c.c_int, _P, _c.c_int, _P,
                                    _c.c_int, _P, _P, _c.c_int64, _P]


class GemmProblem(_c.Structure):
    _fields_ = [("mask", _P), ("sign", _P), ("wsign", _P), ("s_a", _P), ("s_w", _P), ("acc", _P), ("out", _P)]


_lib.bwta_gemm_grouped.restype = _c.c_int
_lib.bwta_gemm_grouped.argtypes = [_c.POINTER(GemmProblem), _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                   _c.c_int64, _P, _c.c_size_t, _P]
_lib.bwta_quantize_pack_bool.restype = _c.c_int
_lib.bwta_quantize_pack_bool.argtypes = [_P, _c.c_int64, _P, _c.c_int, _c.c_int, _c.c_int, _P, _P]
_lib.bwta_matmul_tt.restype = _c.c_int
_lib.bwta_matmul_tt.argtypes = [_P, _P, _c.c_int64, _P, _P, _c.c_int64, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                _P, _c.c_int, _P, _c.c_int, _c.c_float, _P, _P, _c.c_int64, _c.c_int64, _P]
_lib.bwta_prepare_weights.restype = _c.c_int
_lib.bwta_prepare_weights.argtypes = [_P, _c.c_int64, _c.c_int, _c.c_int, _P, _P, _P]
_lib.bwta_act_scale.restype = _c.c_int
_lib.bwta_act_scale.argtypes = [_P, _c.c_int64, _c.c_int, _c.c_int, _P, _P]
_lib.bwta_prepare_act_autoscale.restype = _c.c_int
_lib.bwta_matmul_bool_prepared.restype = _c.c_int
_lib.bwta_matmul_bool_prepared.argtypes = [_P, _c.c_int64, _P, _c.c_size_t, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _P, _c.c_int,
                                           _P, _c.c_int, _c.c_float, _P, _c.c_int64, _c.c_int64, _P]
_lib.bwta_prepare_act_autoscale.argtypes = [_P, _c.c_int64, _c.c_int, _c.c_int, _P, _P, _c.c_size_t,
                                            _c.POINTER(_c.c_int), _P]


class Cache(_c.Structure):
    """bwta_cache of bwta.h, and behind it one more than the number of its tensors' device (0: not known).  `tensors` keeps what the
    addresses point to alive (see make_cache)."""
    _fields_ = [("k", _P), ("v", _P), ("k_scale", _P), ("v_scale", _P), ("blocks", _c.c_int32), ("kv_heads", _c.c_int32),
                ("block", _c.c_int32), ("dim", _c.c_int32), ("place", _c.c_int32)]


_CP = _c.POINTER(Cache)
_lib.bwta_head_norm_rope.restype = _c.c_int
_lib.bwta_head_norm_rope.argtypes = [_P, _c.c_int64, _c.c_int, _P, _P, _c.c_int64, _c.c_int, _P, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                     _c.c_float, _P, _P, _c.c_int, _c.c_int, _P, _c.c_int64, _P, _c.c_int64, _P]
for _f in (_lib.bwta_cache_write, _lib.bwta_cache_read):
    _f.restype = _c.c_int
    _f.argtypes = [_CP, _P, _c.c_int64, _P, _c.c_int64, _c.c_int, _P, _c.c_int64, _P, _P, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _P]
_lib.bwta_cache_attention.restype = _c.c_int
_lib.bwta_cache_attention.argtypes = [_CP, _P, _c.c_int64, _P, _c.c_int64, _c.c_int, _P, _P, _c.c_int64, _P, _P, _c.c_int, _c.c_int,
                                      _c.c_int, _c.c_int, _c.c_int, _c.c_float, _c.c_int, _c.c_int, _P, _c.c_size_t, _P]
_lib.bwta_cache_attention_workspace_bytes.restype = _c.c_size_t
_lib.bwta_cache_attention_workspace_bytes.argtypes = [_c.c_int] * 7
_lib.bwta_strerror.restype = _c.c_char_p
_lib.bwta_strerror.argtypes = [_c.c_int]
_lib.bwta_last_hip_error.restype = _c.c_int
_lib.bwta_set_path.restype = _c.c_int
_lib.bwta_set_path.argtypes = [_c.c_int]
_lib.bwta_get_path.restype = _c.c_int
_lib.bwta_auto_path.restype = _c.c_int
_lib.bwta_auto_path.argtypes = [_c.c_int, _c.c_int, _c.c_int]
_lib.bwta_linear_launches.restype = _c.c_int
_lib.bwta_linear_launches.argtypes = [_c.c_int, _c.c_int, _c.c_int]
_lib.bwta_version.restype = _c.c_int
_lib.bwta_build_id.restype = _c.c_char_p
_lib.bwta_planned_tile.restype = _c.c_int
_lib.bwta_planned_tile.argtypes = [_c.c_int, _c.c_int, _c.c_int]
_lib.bwta_planned_rows.restype = _c.c_int
_lib.bwta_planned_rows.argtypes = [_c.c_int, _c.c_int, _c.c_int]
_lib.bwta_planned_wide.restype = _c.c_int
_lib.bwta_planned_wide.argtypes = [_c.c_int, _c.c_int, _c.c_int]
_lib.bwta_planned_wide_prepared.restype = _c.c_int
_lib.bwta_planned_wide_prepared.argtypes = [_c.c_int, _c.c_int, _c.c_int]
_lib.bwta_planned_decode_blocks.restype = _c.c_int
_lib.bwta_planned_decode_blocks.argtypes = [_c.c_int, _c.c_int, _c.c_int, _c.c_int]
_lib.bwta_set_tile.restype = _c.c_int
_lib.bwta_set_tile.argtypes = [_c.c_int]


class BwtaError(RuntimeError):
    def __init__(self, code):
        self.code = code
        msg = _lib.bwta_strerror(code).decode()
        if code == ERR_HIP:
            msg += " [hipError %d]" % _lib.bwta_last_hip_error()
        super().__init__("bwta error %d: %s" % (code, msg))


def raw():
    """The ctypes library handle, for tests that probe error codes directly."""
    return _lib


def _check(code):
    if code != OK:
        raise BwtaError(code)


def _ptr(x):
    """Device pointer of a torch tensor, a raw integer address, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


# The raw handle of torch's current stream: the two C entry points below cost ~0.3 us together,
# torch.cuda.current_stream().cuda_stream ~3 us (it builds a Python Stream object per call), which
# is as much as the kernel launch itself.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_cur_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    if _raw_stream is not None and _cur_device is not None:
        return _raw_stream(_cur_device())
    return torch.cuda.current_stream().cuda_stream


def _mode(s, mode):
    if mode is not None:
        return mode
    if s is None:
        return SCALE_NONE
    return SCALE_SCALAR if s.numel() == 1 else SCALE_VECTOR


def plane_row_words(K):
    return int(_lib.bwta_plane_row_words(K))


def workspace_bytes(M, N, K):
    return int(_lib.bwta_workspace_bytes(M, N, K))


def strerror(code):
    return _lib.bwta_strerror(code).decode()


def set_path(path):
    _check(_lib.bwta_set_path(path))


def get_path():
    return int(_lib.bwta_get_path())


def auto_path(M, N, K):
    return int(_lib.bwta_auto_path(M, N, K))


def linear_launches(M, N, K):
    return int(_lib.bwta_linear_launches(M, N, K))


def set_tile(tile):
    _check(_lib.bwta_set_tile(int(tile)))


def version():
    return int(_lib.bwta_version())


def build_id():
    return _lib.bwta_build_id().decode()


def bwta_quantize_pack_act(A, s_a, mask, sign, nnz=None, *, M, K, lda=None, a_dtype=DTYPE_FP16,
                           scale_mode=None, stream=None):
    lda = K if lda is None else lda
    _check(_lib.bwta_quantize_pack_act(_ptr(A), a_dtype, lda, _ptr(s_a), _mode(s_a, scale_mode), M, K,
                                       _ptr(mask), _ptr(sign), _ptr(nnz), _stream(stream)))


def bwta_pack_weights(W, wsign, *, N, K, ldw=None, w_dtype=DTYPE_INT8, stream=None):
    ldw = K if ldw is None else ldw
    _check(_lib.bwta_pack_weights(_ptr(W), w_dtype, ldw, N, K, _ptr(wsign), _stream(stream)))


def bwta_gemm(mask, sign, wsign, s_a, s_w, acc, out, workspace, *, M, N, K, ldo=None,
              a_scale_mode=None, w_scale_mode=None, workspace_bytes=None, stream=None):
    ldo = N if ldo is None else ldo
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None or isinstance(workspace, int) else workspace.nbytes
    _check(_lib.bwta_gemm(_ptr(mask), _ptr(sign), _ptr(wsign), M, N, K, _ptr(s_a), _mode(s_a, a_scale_mode),
                          _ptr(s_w), _mode(s_w, w_scale_mode), _ptr(acc), _ptr(out), ldo,
                          _ptr(workspace), workspace_bytes, _stream(stream)))


def bwta_linear(A, s_a, wsign, s_w, out, workspace, *, M, N, K, lda=None, ldo=None, a_scale_mode=None,
                w_scale_mode=None, workspace_bytes=None, stream=None):
    lda = K if lda is None else lda
    ldo = N if ldo is None else ldo
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None or isinstance(workspace, int) else workspace.nbytes
    try:
        code = _linear_call(_linear_pack(_ptr(A) or 0, lda, _ptr(s_a) or 0, _ptr(wsign) or 0, _ptr(s_w) or 0,
                                         _ptr(out) or 0, ldo, _ptr(workspace) or 0, workspace_bytes, _stream(stream),
                                         _mode(s_a, a_scale_mode), _mode(s_w, w_scale_mode), M, N, K, _LINEAR_ARGS_SIZE))
    except struct.error:  # no integer, or one outside its field: what the other calls' conversions make of it
        code = _lib.bwta_linear(_ptr(A), lda, _ptr(s_a), _mode(s_a, a_scale_mode), _ptr(wsign), _ptr(s_w),
                                _mode(s_w, w_scale_mode), M, N, K, _ptr(out), ldo, _ptr(workspace), workspace_bytes,
                                _stream(stream))
    if code != OK:
        _check(code)


def static_scratch_bytes():
    return int(_lib.bwta_static_scratch_bytes())


def static_scratch_init():
    _check(_lib.bwta_static_scratch_init())


def bwta_linear_static(A, s_a, wsign, s_w, out, *, M, N, K, lda=None, ldo=None, a_scale_mode=None,
                       w_scale_mode=None, stream=None):
    lda = K if lda is None else lda
    ldo = N if ldo is None else ldo
    _check(_lib.bwta_linear_static(_ptr(A), lda, _ptr(s_a), _mode(s_a, a_scale_mode), _ptr(wsign), _ptr(s_w),
                                   _mode(s_w, w_scale_mode), M, N, K, _ptr(out), ldo, _stream(stream)))


def bwta_quantize_pack_bool(A, s_a, mask, *, M, K, lda=None, scale_mode=None, stream=None):
    lda = K if lda is None else lda
    _check(_lib.bwta_quantize_pack_bool(_ptr(A), lda, _ptr(s_a), _mode(s_a, scale_mode), M, K, _ptr(mask),
                                        _stream(stream)))


def bwta_matmul_tt(maskA, signA, maskB, signB, s_a, s_b, acc, out, *, batch, M, N, K, alpha=1.0, strideA=None,
                   strideB=None, ldo=None, stride_out=None, a_scale_mode=None, b_scale_mode=None, stream=None):
    rw = plane_row_words(K)
    strideA = M * rw if strideA is None else strideA
    strideB = N * rw if strideB is None else strideB
    ldo = N if ldo is None else ldo
    stride_out = M * ldo if stride_out is None else stride_out
    _check(_lib.bwta_matmul_tt(_ptr(maskA), _ptr(signA), strideA, _ptr(maskB), _ptr(signB), strideB, batch, M, N, K,
                               _ptr(s_a), _mode(s_a, a_scale_mode), _ptr(s_b), _mode(s_b, b_scale_mode), float(alpha),
                               _ptr(acc), _ptr(out), ldo, stride_out, _stream(stream)))


def bwta_prepare_weights(W, wsign, s_w, *, N, K, ldw=None, stream=None):
    ldw = K if ldw is None else ldw
    _check(_lib.bwta_prepare_weights(_ptr(W), ldw, N, K, _ptr(wsign), _ptr(s_w), _stream(stream)))


def bwta_act_scale(A, s, *, M, K, lda=None, stream=None):
    lda = K if lda is None else lda
    _check(_lib.bwta_act_scale(_ptr(A), lda, M, K, _ptr(s), _stream(stream)))


def _nbytes(buf, given):
    if given is not None:
        return given
    return 0 if buf is None or isinstance(buf, int) else buf.nbytes


def prepared_bytes(M, K):
    return int(_lib.bwta_prepared_bytes(M, K))


def planned_kernel(operand, M, N, K):
    return int(_lib.bwta_planned_kernel(operand, M, N, K))


def planned_tile(M, N, K):
    return int(_lib.bwta_planned_tile(M, N, K))


def planned_rows(M, N, K):
    return int(_lib.bwta_planned_rows(M, N, K))


def planned_wide(M, N, K, prepared=False):
    return int((_lib.bwta_planned_wide_prepared if prepared else _lib.bwta_planned_wide)(M, N, K))


def planned_decode_blocks(M, N, K, count):
    return int(_lib.bwta_planned_decode_blocks(M, N, K, count))


def prepared_format(M, K):
    return int(_lib.bwta_prepared_format(M, K))


def bwta_prepare_act(A, s_a, prepared, *, M, K, lda=None, a_scale_mode=None, prepared_bytes=None, stream=None):
    """Returns the format id of what was written; hand it to the call that consumes `prepared`."""
    lda = K if lda is None else lda
    fmt = _c.c_int(0)
    _check(_lib.bwta_prepare_act(_ptr(A), lda, _ptr(s_a), _mode(s_a, a_scale_mode), M, K, _ptr(prepared),
                                 _nbytes(prepared, prepared_bytes), _c.byref(fmt), _stream(stream)))
    return fmt.value


def bwta_prepare_act_autoscale(A, s_a, prepared, *, M, K, lda=None, prepared_bytes=None, stream=None):
    """Returns the format id of what was written, as bwta_prepare_act."""
    lda = K if lda is None else lda
    fmt = _c.c_int(0)
    _check(_lib.bwta_prepare_act_autoscale(_ptr(A), lda, M, K, _ptr(s_a), _ptr(prepared),
                                           _nbytes(prepared, prepared_bytes), _c.byref(fmt), _stream(stream)))
    return fmt.value


def bwta_matmul_bool_prepared(maskA, preparedB, s_a, s_b, out, *, fmt, batch, M, N, K, alpha=1.0, strideA=None, ldo=None,
                              stride_out=None, a_scale_mode=None, b_scale_mode=None, prepared_bytes=None, stream=None):
    rw = plane_row_words(K)
    strideA = M * rw if strideA is None else strideA
    ldo = N if ldo is None else ldo
    stride_out = M * ldo if stride_out is None else stride_out
    _check(_lib.bwta_matmul_bool_prepared(_ptr(maskA), strideA, _ptr(preparedB), _nbytes(preparedB, prepared_bytes),
                                          fmt, batch, M, N, K, _ptr(s_a), _mode(s_a, a_scale_mode), _ptr(s_b),
                                          _mode(s_b, b_scale_mode), float(alpha), _ptr(out), ldo, stride_out,
                                          _stream(stream)))


def bwta_gemm_prepared(prepared, wsign, s_a, s_w, acc, out, *, fmt, M, N, K, ldo=None, a_scale_mode=None,
                       w_scale_mode=None, prepared_bytes=None, stream=None):
    ldo = N if ldo is None else ldo
    _check(_lib.bwta_gemm_prepared(_ptr(prepared), _nbytes(prepared, prepared_bytes), fmt, _ptr(wsign), M, N, K,
                                   _ptr(s_a), _mode(s_a, a_scale_mode), _ptr(s_w), _mode(s_w, w_scale_mode),
                                   _ptr(acc), _ptr(out), ldo, _stream(stream)))


def make_problems(problems):
    """problems: list of (mask, sign, wsign, s_a, s_w, acc, out) tensors/addresses -> ctypes array
    (build once, reuse across calls)."""
    arr = (GemmProblem * len(problems))()
    for i, p in enumerate(problems):
        for name, v in zip(("mask", "sign", "wsign", "s_a", "s_w", "acc", "out"), p):
            setattr(arr[i], name, _ptr(v))
    return arr


def bwta_gemm_grouped(problem_array, workspace, *, M, N, K, a_scale_mode=SCALE_VECTOR, w_scale_mode=SCALE_VECTOR,
                      ldo=None, workspace_bytes=None, stream=None):
    ldo = N if ldo is None else ldo
    _check(_lib.bwta_gemm_grouped(problem_array, len(problem_array), M, N, K, a_scale_mode, w_scale_mode, ldo,
                                  _ptr(workspace), _nbytes(workspace, workspace_bytes), _stream(stream)))


# ---- operators on heads ------------------------------------------------------------------------------
#
# Unless given, ld and ldt are as the tensors have their rows.  Tensors have to be on the current device, of the type that the
# header or dtype= says, and hold what the call's sizes say; of addresses nothing of this is known.


def _dtype(dtype, x, *others):
    """The dtype argument of an operator on heads: as given, or the tensors', whose rows have no gaps between elements."""
    for y in (x, *others):
        if isinstance(y, torch.Tensor) and y.dim() and y.stride(-1) != 1 and y.shape[-1] > 1:
            raise ValueError("elements of a row lie next to each other, got strides %s" % (tuple(y.stride()),))
    if dtype is not None:
        if dtype in (DTYPE_FP16, DTYPE_BF16):
            named = torch.float16 if dtype == DTYPE_FP16 else torch.bfloat16
            for y in (x, *others):  # of that type, or the bits of it as whole numbers
                if isinstance(y, torch.Tensor) and y.dtype not in (named, torch.int16, torch.uint16):
                    raise TypeError("dtype= says %s, a tensor is %s" % (named, y.dtype))
        return dtype
    try:
        given = {torch.float16: DTYPE_FP16, torch.bfloat16: DTYPE_BF16}[x.dtype]
    except (AttributeError, KeyError):
        raise TypeError("pass dtype= with addresses; tensors are float16 or bfloat16, got %s" % getattr(x, "dtype", type(x).__name__)) from None
    for y in others:
        if isinstance(y, torch.Tensor) and y.dtype != x.dtype:
            raise TypeError("tensors of one type, got %s beside %s" % (y.dtype, x.dtype))
    return given


def _dense(dtype, *xs):
    """Positions, lengths, offsets, frequencies and the like are what the header says, one after the other."""
    for x in xs:
        if isinstance(x, torch.Tensor):
            if x.dtype != dtype:
                raise TypeError("a tensor of %s has to be %s" % (x.dtype, dtype))
            if not x.is_contiguous():
                raise ValueError("a tensor of strides %s has to be contiguous" % (tuple(x.stride()),))


def _apart(x, given, width):
    """How far apart the rows of an operator on heads are: as given, or as they are in the tensor, whose last dimensions, `width` elements
    or more together, are a row ([M, width or more], [M, heads, dim], [batch, tokens, heads, dim]) and lie side by side."""
    if isinstance(x, torch.Tensor) and x.numel() and width > 0:
        size, i = 1, x.dim()
        while i > 0 and size < width:
            i -= 1
            if x.shape[i] > 1 and x.stride(i) != size:
                raise ValueError("a row's heads lie side by side, got shape %s and strides %s for rows of %d" % (tuple(x.shape), tuple(x.stride()), width))
            size *= x.shape[i]
        if given is None:
            apart = None  # of the rows in the dimensions so far, and how far the next dimension's have to be
            for n, stride in reversed([d for d in zip(x.shape[:i], x.stride()) if d[0] > 1]):
                if apart is not None and stride != step:
                    raise ValueError("rows are not equally far apart, got shape %s and strides %s: pass ld" % (tuple(x.shape), tuple(x.stride())))
                apart, step = stride if apart is None else apart, stride * n
            return width if apart is None else apart
    return width if given is None else given


def _span(x):
    """Bytes from a tensor's first element to behind its last."""
    return (1 + sum((n - 1) * stride for n, stride in zip(x.shape, x.stride()))) * x.element_size() if x.numel() else 0


def _holds(x, apart, rows, width, size):
    """A tensor has the `rows` rows of `width` elements of `size` bytes that a call reads or writes of it."""
    if isinstance(x, torch.Tensor) and rows > 0 and width > 0 and _span(x) < ((rows - 1) * apart + width) * size:
        raise ValueError("%d rows of %d, %d apart, are not in a tensor of shape %s and strides %s" % (rows, width, apart, tuple(x.shape), tuple(x.stride())))


def _rows(x, given, M, width):
    """_apart, and _holds for M such rows of 16-bit elements: the forms that most calls have at once, others by those two."""
    if not isinstance(x, torch.Tensor):
        return width if given is None else given
    shape, strides = x.shape, x.stride()
    if M > 0 and width > 0 and len(shape) in (2, 3) and strides[-1] == 1 and shape[0] >= M and x.element_size() == 2:
        size = shape[1] if len(shape) == 2 else shape[1] * shape[2] if strides[1] == shape[2] < width else 0
        if size >= width and (given is None or M == 1 or given == strides[0]):
            return given if given is not None else strides[0] if shape[0] > 1 else width
    apart = _apart(x, given, width)
    _holds(x, apart, M, width, 2)
    return apart


def _here(*xs):
    """These calls launch on the current device: tensors have to be there."""
    for x in xs:
        if isinstance(x, torch.Tensor) and not (x.is_cuda and x.get_device() == torch.cuda.current_device()):
            raise ValueError("a tensor on %s, the current device is %s" % (x.device, torch.cuda.current_device() if torch.cuda.is_available() else "none"))
        if isinstance(x, Cache) and x.place > 0 and x.place - 1 != torch.cuda.current_device():
            raise ValueError("a cache on device %d, the current one is %d" % (x.place - 1, torch.cuda.current_device()))


def make_cache(k, v, k_scale, v_scale, *, blocks=None, kv_heads=None, block=None, dim=None):
    """The cache of 8-bit keys and values as the calls below take it (build once, reuse).  k [blocks, kv_heads, block, dim]
    and v [blocks, kv_heads, dim, block] are contiguous tensors of one byte an element (uint8 or float8_e4m3fn), k_scale and
    v_scale contiguous float32 [blocks, kv_heads]; or all four are addresses and the sizes are given.  The tensors are kept
    alive."""
    if not isinstance(k, int):
        if k.dim() != 4:
            raise ValueError("keys are [blocks, kv_heads, block, dim]")
        sizes = tuple(k.shape)
        for name, t, shape in (("k", k, sizes), ("v", v, (sizes[0], sizes[1], sizes[3], sizes[2])), ("k_scale", k_scale, sizes[:2]), ("v_scale", v_scale, sizes[:2])):
            if tuple(t.shape) != shape or not t.is_contiguous() or t.device != k.device:
                raise ValueError("%s has to be contiguous, of shape %s and on %s" % (name, shape, k.device))
            if t.dtype not in ((torch.float32,) if "scale" in name else (torch.uint8, torch.float8_e4m3fn)):
                raise TypeError("%s is %s" % (name, t.dtype))
        given = (blocks, kv_heads, block, dim)
        if any(g is not None and g != s for g, s in zip(given, sizes)):
            raise ValueError("sizes %s given, the tensors have %s" % (given, sizes))
        blocks, kv_heads, block, dim = sizes
    place = k.get_device() + 1 if isinstance(k, torch.Tensor) else 0
    c = Cache(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), blocks, kv_heads, block, dim, place)
    c.tensors = (k, v, k_scale, v_scale)
    return c


def bwta_head_norm_rope(Q, K, wq, wk, positions, inv_freq, Qout, Kout, *, M, heads, kv_heads, dim, rot_dim=None, eps=1e-6,
                        norm=True, interleaved=False, ldq=None, ldk=None, ldqo=None, ldko=None, dtype=None, stream=None):
    """rot_dim: all of dim unless given.  norm: whether heads are normalised (weights None: by 1)."""
    _here(Q, K, wq, wk, positions, inv_freq, Qout, Kout)
    _dense(torch.int32, positions)
    _dense(torch.float32, inv_freq)
    dtype = _dtype(dtype, *((K, wk, Kout) if Q is None else (Q, K, wq, wk, Qout, Kout)))
    wide, kv_wide, rot_dim = heads * dim, kv_heads * dim, dim if rot_dim is None else rot_dim
    ldq, ldk, ldqo, ldko = _rows(Q, ldq, M, wide), _rows(K, ldk, M, kv_wide), _rows(Qout, ldqo, M, wide), _rows(Kout, ldko, M, kv_wide)
    if M > 0:
        _counts((wq, dim if norm and heads > 0 else 0), (wk, dim if norm and kv_heads > 0 else 0), (positions, M if rot_dim > 0 else 0), (inv_freq, rot_dim // 2))
    _check(_lib.bwta_head_norm_rope(_ptr(Q), ldq, heads, _ptr(wq), _ptr(K), ldk, kv_heads, _ptr(wk), dtype, M, dim, int(norm), eps, _ptr(positions),
                                    _ptr(inv_freq), rot_dim, int(interleaved), _ptr(Qout), ldqo, _ptr(Kout), ldko, _stream(stream)))


def _ldt(table, given, batch):
    if isinstance(table, torch.Tensor) and (table.dtype != torch.int32 or (table.dim() and table.stride(-1) != 1 and table.shape[-1] > 1)):
        raise TypeError("a block table is int32, its rows without gaps, got %s of strides %s" % (table.dtype, tuple(table.stride())))
    if given is not None:
        return given
    if table is None or isinstance(table, int) or table.dim() == 0:
        return 0
    if batch == 1 and (table.dim() == 1 or table.shape[0] == 1):
        return table.numel()  # one row, whatever its stride
    return table.stride(0)


def _room(workspace, given):
    """Bytes of a workspace: a contiguous tensor's own, or as many of them as are given."""
    n = _nbytes(workspace, given)
    if isinstance(workspace, torch.Tensor) and (not workspace.is_contiguous() or n > workspace.nbytes):
        raise ValueError("a workspace of %d bytes is not in a tensor of shape %s and strides %s" % (n, tuple(workspace.shape), tuple(workspace.stride())))
    return n


def _counts(*xs):
    """Tensors without gaps have as many elements as a call reads of them."""
    for x, n in xs:
        if isinstance(x, torch.Tensor) and x.numel() < n:
            raise ValueError("a tensor of %d elements, the call's sizes say %d" % (x.numel(), n))


def _sequences_hold(cache, table, ldt, lens, cu, M, batch, max_new, max_len):
    if M > 0 and batch > 0 and max_new > 0:
        _counts((lens, batch), (cu, batch + 1))
        blocks = -(-max_len // cache.block) if cache.block > 0 else 0
        if not (isinstance(table, torch.Tensor) and table.dim() == 2 and table.shape[0] >= batch and table.shape[1] >= blocks and table.stride(0) == ldt):
            _holds(table, ldt, batch, blocks, 4)


def _cache_rows(call, cache, K, V, table, lens, cu, M, batch, max_new, max_len, ldk, ldv, ldt, dtype, stream):
    _here(cache, K, V, table, lens, cu)
    _dense(torch.int32, lens, cu)
    width, dtype = cache.kv_heads * cache.dim, _dtype(dtype, K, V)
    ldk, ldv, ldt = _rows(K, ldk, M, width), _rows(V, ldv, M, width), _ldt(table, ldt, batch)
    _sequences_hold(cache, table, ldt, lens, cu, M, batch, max_new, max_len)
    _check(call(cache, _ptr(K), ldk, _ptr(V), ldv, dtype, _ptr(table), ldt, _ptr(lens), _ptr(cu), batch, M, max_new, max_len, _stream(stream)))


def bwta_cache_write(cache, K, V, table, lens, cu=None, *, M, batch, max_new, max_len, ldk=None, ldv=None, ldt=None, dtype=None, stream=None):
    _cache_rows(_lib.bwta_cache_write, cache, K, V, table, lens, cu, M, batch, max_new, max_len, ldk, ldv, ldt, dtype, stream)


def bwta_cache_read(cache, K, V, table, lens, cu=None, *, M, batch, max_new, max_len, ldk=None, ldv=None, ldt=None, dtype=None, stream=None):
    _cache_rows(_lib.bwta_cache_read, cache, K, V, table, lens, cu, M, batch, max_new, max_len, ldk, ldv, ldt, dtype, stream)


def cache_attention_workspace_bytes(*, M, heads, kv_heads, dim, batch, max_new, max_len):
    return int(_lib.bwta_cache_attention_workspace_bytes(M, heads, kv_heads, dim, batch, max_new, max_len))


def bwta_cache_attention(cache, Q, out, lse, table, lens, cu=None, workspace=None, *, M, batch, max_new, max_len, heads, alpha, causal=True, window=0,
                         ldq=None, ldo=None, ldt=None, dtype=None, workspace_bytes=None, stream=None):
    _here(cache, Q, out, lse, table, lens, cu, workspace)
    _dense(torch.int32, lens, cu)
    _dense(torch.float32, lse)
    width, dtype = heads * cache.dim, _dtype(dtype, Q, out)
    ldq, ldo, ldt = _rows(Q, ldq, M, width), _rows(out, ldo, M, width), _ldt(table, ldt, batch)
    _counts((lse, M * heads if M > 0 and heads > 0 else 0))
    _sequences_hold(cache, table, ldt, lens, cu, M, batch, max_new, max_len)
    _check(_lib.bwta_cache_attention(cache, _ptr(Q), ldq, _ptr(out), ldo, dtype, _ptr(lse), _ptr(table), ldt, _ptr(lens), _ptr(cu), batch, M, max_new, max_len, heads,
                                     alpha, int(causal), window, _ptr(workspace), _room(workspace, workspace_bytes), _stream(stream)))


def _native_identity():
    return "%s %s %d.%d" % ((build_id(), torch.__version__) + sys.version_info[:2])


def _load_native():
    """(the extension or None, what it was built from and for)"""
    try:
        loader = importlib.machinery.ExtensionFileLoader("_bwta_native", NATIVE_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_bwta_native", NATIVE_PATH, loader=loader))
        loader.exec_module(module)
    except ImportError as e:  # no such file, or one for another Python or torch
        return None, str(e)
    module.setup(_check, _raw_stream, _cur_device, Cache)
    return module, module.identity() if hasattr(module, "identity") else "unknown"


# From here on each of these names is the native function, with the Python form above as what it falls back to.  An
# extension of other sources than the library's (its arguments may be others), or for another torch, is not called.
_native, _built = _load_native()
if _built == _native_identity():
    for _name in (*_native.parameters(), *_native.head_parameters()):
        globals()[_name] = _native.bind(_name, _c.cast(getattr(_lib, _name), _P).value, globals()[_name])
else:
    warnings.warn("%s is of build %r, the library and this interpreter are %r: the calls are marshalled in Python; build again"
                  % (NATIVE_PATH, _built, _native_identity()), RuntimeWarning)
