"""ctypes binding of ``libsdp4.so`` -- argument marshalling only.

Each function has the name and argument order of the C entry point it
wraps, takes torch tensors (device memory) or raw integer device pointers
for the arrays, derives element counts and dtypes from tensors where the C
call needs them, passes torch's current HIP stream unless one is given, and
raises :class:`Sdp4Error` on a non-zero status.  No computation happens
here, and there is no fallback: without the built library every call raises.

A call's way to its launch costs more than most small kernels run, so the
marshalling of ordinary arguments (torch tensors or addresses, plain ints,
the current stream or a stream's address) is native, in ``_binding.so``;
whatever that hands back as out of the ordinary takes the general path here,
which also reports what is wrong with it.
"""
from __future__ import annotations

import ctypes as C
import os
import threading
import warnings

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsdp4.so")
_lock = threading.Lock()
_lib = None
_fast = None  # the native marshalling, bound to the loaded library

OK, EINVAL, EALIGN, ERANGE, EHIP = 0, 1, 2, 3, 4
F32, BF16 = 0, 1
MIN_GROUP, MAX_GROUP, MAX_HADAMARD, MAX_PEERS = 32, 4096, 1024, 16
MAX_TOP, MAX_VOCAB, MAX_HEAD_DIM = 32, 1 << 20, 512
MIN_ATTENTION_DIM, MAX_ATTENTION_DIM, MAX_TOKENS, MAX_HIDDEN, MAX_GRAD_TOKENS = 8, 256, 1 << 30, 16384, 1 << 21


class Sdp4Error(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        msg = lib().sdp4_status_string(status).decode()
        if status == EHIP:
            msg += f" (hip error {lib().sdp4_last_hip_error()})"
        super().__init__(f"{fn}: status {status}: {msg}")


class Heads(C.Structure):
    """``sdp4_heads``: query or key heads of all tokens."""
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("heads", C.c_int)]


class QkParams(C.Structure):
    """``sdp4_qk_params``: how heads are normed and rotated."""
    _fields_ = [("dtype", C.c_int), ("head_dim", C.c_int), ("norm", C.c_int), ("eps", C.c_float),
                ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("table", C.c_void_p), ("table_rows", C.c_int64),
                ("rot_dim", C.c_int), ("interleaved", C.c_int), ("positions", C.c_void_p)]


class AttentionParams(C.Structure):
    """``sdp4_attention_params``: packed sequences and their scores' scale."""
    _fields_ = [("dtype", C.c_int), ("head_dim", C.c_int), ("scale", C.c_float), ("offsets", C.c_void_p),
                ("sequences", C.c_int64)]


class BlockParams(C.Structure):
    """``sdp4_block_params``: the joint of two blocks."""
    _fields_ = [("x_dtype", C.c_int), ("y_dtype", C.c_int), ("post_norm", C.c_int), ("post_eps", C.c_float),
                ("pre_eps", C.c_float), ("post_weight", C.c_void_p), ("pre_weight", C.c_void_p), ("gate", C.c_void_p),
                ("branch_scale", C.c_float), ("residual_scale", C.c_float)]


def lib() -> C.CDLL:
    """The loaded HIP library (raises if it has not been built)."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(_LIB_PATH):
                raise ImportError(f"{_LIB_PATH} is missing: build it with "
                                  "`python -c 'import __graft_entry__ as g; g.build()'`")
            L = C.CDLL(_LIB_PATH)
            vp, i64, i32, f32 = C.c_void_p, C.c_int64, C.c_int, C.c_float
            sig = {
                "sdp4_qwd_encode": (i32, [vp, vp, i32, i64, i32, vp, vp, vp, vp]),
                "sdp4_qwd_decode": (i32, [vp, vp, vp, i64, i32, vp, i32, vp]),
                "sdp4_qwd_encode_sym": (i32, [vp, vp, i32, i64, i32, vp, vp, vp]),
                "sdp4_qwd_decode_sym": (i32, [vp, vp, i64, i32, vp, i32, vp]),
                "sdp4_grad_quant": (i32, [vp, i64, i32, i32, i32, vp, vp, vp]),
                "sdp4_dequant_reduce": (i32, [i32, vp, vp, i64, i32, i32, i32, i32, f32, vp, vp, vp, vp]),
                "sdp4_grad_quant_sr": (i32, [vp, i64, i32, i32, i32, C.c_uint64, C.c_uint64, vp, vp, vp]),
                "sdp4_dequant_reduce_sr": (i32, [i32, vp, vp, i64, i32, i32, i32, C.c_uint64, C.c_uint64, vp, vp,
                                                 vp, vp]),
                "sdp4_hadamard": (i32, [vp, vp, i64, i32, vp]),
                "sdp4_reduce_f32": (i32, [i32, vp, vp, i64, vp]),
                "sdp4_copy_f32": (i32, [vp, vp, i64, vp]),
                "sdp4_read_f32": (i32, [vp, i64, vp, vp]),
                "sdp4_fill_f32": (i32, [vp, i64, f32, vp]),
                "sdp4_dropout_add": (i32, [vp, i32, i64, vp, vp, i64, i64, i64, f32, C.c_uint64, C.c_uint64, vp, i32,
                                           i64, vp]),
                "sdp4_dropout_add_grad": (i32, [vp, i32, i64, i64, i64, f32, C.c_uint64, C.c_uint64, vp, i32, i64, vp,
                                                vp, i64, vp]),
                "sdp4_dropout_grad_workspace": (i64, [i64, i64]),
                "sdp4_token_logprob": (i32, [vp, i32, i64, i64, i64, vp, i32, vp, vp, vp, vp, vp, vp, i64, vp]),
                "sdp4_token_logprob_workspace": (i64, [i64, i64, i32]),
                "sdp4_token_logprob_grad": (i32, [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, i64, i64, vp]),
                "sdp4_token_loss": (i32, [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, vp, i64,
                                          vp]),
                "sdp4_qk_norm_rope": (i32, [vp, vp, vp, i64, vp, vp, vp]),
                "sdp4_qk_norm_rope_grad": (i32, [vp, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, i64, vp]),
                "sdp4_qk_grad_workspace": (i64, [i64, i32, i32, i32]),
                "sdp4_rope_table": (i32, [vp, i32, i64, i64, C.c_double, vp, vp]),
                "sdp4_attention": (i32, [vp, vp, vp, vp, i64, vp, vp, vp]),
                "sdp4_attention_grad": (i32, [vp, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp, i64, vp]),
                "sdp4_attention_grad_workspace": (i64, [i64, i32, i32, i32]),
                "sdp4_block_norm": (i32, [vp, i64, vp, i64, i64, i64, vp, vp, i64, vp, i64, vp]),
                "sdp4_block_norm_grad": (i32, [vp, i64, vp, i64, vp, i64, vp, i64, i64, i64, vp, vp, i64, vp, i64, vp, vp, vp,
                                               vp, i64, vp]),
                "sdp4_block_norm_grad_workspace": (i64, [i64, i64]),
                "sdp4_embedding": (i32, [vp, i64, vp, i32, i64, i64, i64, f32, vp, i32, i64, vp]),
                "sdp4_embedding_grad": (i32, [vp, i64, vp, i32, i64, i64, i64, f32, i32, vp, i32, i64, vp, i64, vp]),
                "sdp4_embedding_grad_workspace": (i64, [i64, i64, i64]),
                "sdp4_codes_bytes": (i64, [i64, i32]),
                "sdp4_num_groups": (i64, [i64, i32]),
                "sdp4_status_string": (C.c_char_p, [i32]),
                "sdp4_version": (C.c_char_p, []),
                "sdp4_last_hip_error": (i32, []),
            }
            for name, (res, args) in sig.items():
                fn = getattr(L, name)
                fn.restype, fn.argtypes = res, args
            _bind(L)
            _lib = L
    return _lib


def _bind(L) -> None:
    """Point the native marshalling at the library's entry points.  Without
    it -- not built, or built for another torch, whose tensors it would
    misread -- every call takes the general path, which a warning says."""
    global _fast
    try:
        import torch  # the extension's libraries come with torch
    except ImportError:
        return  # addresses only, on the general path
    try:
        from . import _binding
    except ImportError as e:
        warnings.warn(f"sdp4: no native argument marshalling, calls take longer on the host: {e}", RuntimeWarning)
        return
    built_for = getattr(_binding, "torch_version", None)  # None: built before it was recorded
    if built_for != torch.__version__:
        warnings.warn(f"sdp4: native argument marshalling was built for torch {built_for}, not "
                      f"{torch.__version__}, and is not used: calls take longer on the host", RuntimeWarning)
        return
    addresses = [C.cast(getattr(L, "sdp4_" + n), C.c_void_p).value for n in
                 ("qwd_encode", "qwd_decode", "qwd_encode_sym", "qwd_decode_sym", "grad_quant", "grad_quant_sr",
                  "dequant_reduce", "dequant_reduce_sr", "dropout_add", "dropout_add_grad", "token_logprob",
                  "token_logprob_grad", "token_loss", "qk_norm_rope", "qk_norm_rope_grad", "attention", "attention_grad",
                  "block_norm", "block_norm_grad", "embedding", "embedding_grad")]
    try:
        _binding.bind(*addresses)
    except TypeError:
        warnings.warn("sdp4: native argument marshalling was built for other entry points and is not used: calls take "
                      "longer on the host", RuntimeWarning)
        return
    _fast = _binding


def _done(name: str, rc) -> bool:
    """Whether the native path made the call (rc None: it did not)."""
    if rc is None:
        return False
    if rc != OK:
        raise Sdp4Error(name, rc)
    return True


def _ptr(x):
    """Device address of a tensor (must live on a GPU), an int address, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not x.is_cuda:
        raise ValueError("sdp4: arrays must be device tensors")
    if not x.is_contiguous():
        raise ValueError("sdp4: arrays must be contiguous")
    return x.data_ptr()


def _need(x, nbytes: int, what: str) -> None:
    """A tensor argument must hold every byte the call reads or writes
    through it: the library sees only its address, so a short tensor would
    be overrun on the device.  Integer addresses are the caller's to size."""
    if x is None or isinstance(x, int):
        return
    have = x.numel() * x.element_size()
    if have < nbytes:
        raise ValueError(f"sdp4: {what} holds {have} bytes; the call touches {nbytes}")


def _ng(n: int, group: int) -> int:
    """Groups in n elements; 0 for a group the library will reject itself."""
    ok = isinstance(group, int) and group > 0 and group & (group - 1) == 0
    return n // group if ok else 0


def _prev_bytes(w_prev, n: int) -> int:
    import torch
    return (4 if w_prev.dtype == torch.float32 else 2) * n


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _prev_dtype(w_prev) -> int:
    import torch
    if w_prev.dtype == torch.float32:
        return F32
    if w_prev.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        return BF16
    raise ValueError(f"sdp4: model weights must be float32 or bfloat16, not {w_prev.dtype}")


def _ck(name: str, rc: int) -> None:
    if rc != OK:
        raise Sdp4Error(name, rc)


def sdp4_qwd_encode(w_new, w_prev, group, codes, scale, minv, n=None, stream=None):
    """codes/scale/minv <- 4-bit quantized (w_new - w_prev); see include/sdp4.h."""
    if _fast is not None and _done("sdp4_qwd_encode", _fast.qwd_encode(
            w_new, w_prev, group, codes, scale, minv, n, stream)):
        return
    n = w_new.numel() if n is None else n
    _need(w_new, 4 * n, "w_new"); _need(w_prev, _prev_bytes(w_prev, n), "w_prev"); _need(codes, n // 2, "codes")
    _need(scale, 4 * _ng(n, group), "scale"); _need(minv, 4 * _ng(n, group), "minv")
    _ck("sdp4_qwd_encode", lib().sdp4_qwd_encode(_ptr(w_new), _ptr(w_prev), _prev_dtype(w_prev), n, group,
                                                 _ptr(codes), _ptr(scale), _ptr(minv), _stream(stream)))


def sdp4_qwd_decode(codes, scale, minv, group, w_prev, n=None, stream=None):
    """w_prev <- w_prev + dequantized message, in place."""
    if _fast is not None and _done("sdp4_qwd_decode", _fast.qwd_decode(codes, scale, minv, group, w_prev, n, stream)):
        return
    n = w_prev.numel() if n is None else n
    _need(codes, n // 2, "codes"); _need(scale, 4 * _ng(n, group), "scale"); _need(minv, 4 * _ng(n, group), "minv")
    _need(w_prev, _prev_bytes(w_prev, n), "w_prev")
    _ck("sdp4_qwd_decode", lib().sdp4_qwd_decode(_ptr(codes), _ptr(scale), _ptr(minv), n, group,
                                                 _ptr(w_prev), _prev_dtype(w_prev), _stream(stream)))


def sdp4_qwd_encode_sym(w_new, w_prev, group, codes, scale, n=None, stream=None):
    """codes/scale <- symmetric 4-bit quantized (w_new - w_prev); see include/sdp4.h."""
    if _fast is not None and _done("sdp4_qwd_encode_sym", _fast.qwd_encode_sym(
            w_new, w_prev, group, codes, scale, n, stream)):
        return
    n = w_new.numel() if n is None else n
    _need(w_new, 4 * n, "w_new"); _need(w_prev, _prev_bytes(w_prev, n), "w_prev"); _need(codes, n // 2, "codes")
    _need(scale, 4 * _ng(n, group), "scale")
    _ck("sdp4_qwd_encode_sym", lib().sdp4_qwd_encode_sym(_ptr(w_new), _ptr(w_prev), _prev_dtype(w_prev), n, group,
                                                         _ptr(codes), _ptr(scale), _stream(stream)))


def sdp4_qwd_decode_sym(codes, scale, group, w_prev, n=None, stream=None):
    """w_prev <- w_prev + dequantized symmetric message, in place."""
    if _fast is not None and _done("sdp4_qwd_decode_sym", _fast.qwd_decode_sym(codes, scale, group, w_prev, n, stream)):
        return
    n = w_prev.numel() if n is None else n
    _need(codes, n // 2, "codes"); _need(scale, 4 * _ng(n, group), "scale"); _need(w_prev, _prev_bytes(w_prev, n), "w_prev")
    _ck("sdp4_qwd_decode_sym", lib().sdp4_qwd_decode_sym(_ptr(codes), _ptr(scale), n, group, _ptr(w_prev),
                                                         _prev_dtype(w_prev), _stream(stream)))


def sdp4_grad_quant(x, bits, hadamard_block, group, codes, scale, n=None, stream=None):
    if _fast is not None and _done("sdp4_grad_quant", _fast.grad_quant(
            x, bits, hadamard_block, group, codes, scale, n, stream)):
        return
    n = x.numel() if n is None else n
    _need(x, 4 * n, "x"); _need(codes, n * bits // 8, "codes"); _need(scale, 4 * _ng(n, group), "scale")
    _ck("sdp4_grad_quant", lib().sdp4_grad_quant(_ptr(x), n, bits, hadamard_block, group, _ptr(codes),
                                                 _ptr(scale), _stream(stream)))


def _need_reduce(codes, scales, n_chunk, bits_in, group, bits_out, out_codes, out_scales, out_f32):
    for p, (c, sc) in enumerate(zip(codes, scales)):
        _need(c, n_chunk * bits_in // 8, f"codes[{p}]")
        _need(sc, 4 * _ng(n_chunk, group), f"scales[{p}]")
    if bits_out:
        _need(out_codes, n_chunk * bits_out // 8, "out_codes")
        _need(out_scales, 4 * _ng(n_chunk, group), "out_scales")
    _need(out_f32, 4 * n_chunk, "out_f32")


def sdp4_dequant_reduce(codes, scales, n_chunk, bits_in, group, bits_out, hadamard_block=0,
                        out_scale=1.0, out_codes=None, out_scales=None, out_f32=None, stream=None):
    """``codes``/``scales``: sequences of P chunk tensors (or addresses)."""
    if _fast is not None and _done("sdp4_dequant_reduce", _fast.dequant_reduce(
            codes, scales, n_chunk, bits_in, group, bits_out, hadamard_block, out_scale, out_codes, out_scales, out_f32, stream)):
        return
    P = len(codes)
    if len(scales) != P:
        raise ValueError("sdp4_dequant_reduce: codes and scales differ in length")
    _need_reduce(codes, scales, n_chunk, bits_in, group, bits_out, out_codes, out_scales, out_f32)
    cp = (C.c_void_p * max(P, 1))(*[_ptr(c) for c in codes])
    sp = (C.c_void_p * max(P, 1))(*[_ptr(s) for s in scales])
    _ck("sdp4_dequant_reduce", lib().sdp4_dequant_reduce(
        P, C.cast(cp, C.c_void_p), C.cast(sp, C.c_void_p), n_chunk, bits_in, group, bits_out,
        hadamard_block, float(out_scale), _ptr(out_codes), _ptr(out_scales), _ptr(out_f32),
        _stream(stream)))


def chunk_addresses(codes, scales, count, code_bytes, headers):
    """Device addresses of ``count`` consecutive chunks of a message (each
    ``code_bytes`` of codes and ``headers`` group headers) as two lists for
    sdp4_dequant_reduce, or None where the tensors are not plain device
    buffers that hold them all."""
    return None if _fast is None else _fast.chunk_addresses(codes, scales, count, code_bytes, headers)


def sdp4_grad_quant_sr(x, bits, hadamard_block, group, seed, offset, codes, scale, n=None, stream=None):
    """Stochastically rounded sdp4_grad_quant (unbiased; see include/sdp4.h)."""
    if _fast is not None and _done("sdp4_grad_quant_sr", _fast.grad_quant_sr(
            x, bits, hadamard_block, group, seed, offset, codes, scale, n, stream)):
        return
    n = x.numel() if n is None else n
    _need(x, 4 * n, "x"); _need(codes, n * bits // 8, "codes"); _need(scale, 4 * _ng(n, group), "scale")
    _ck("sdp4_grad_quant_sr", lib().sdp4_grad_quant_sr(_ptr(x), n, bits, hadamard_block, group, seed, offset,
                                                       _ptr(codes), _ptr(scale), _stream(stream)))


def sdp4_dequant_reduce_sr(codes, scales, n_chunk, bits_in, group, bits_out, seed, offset, out_codes, out_scales,
                           out_f32=None, stream=None):
    if _fast is not None and _done("sdp4_dequant_reduce_sr", _fast.dequant_reduce_sr(
            codes, scales, n_chunk, bits_in, group, bits_out, seed, offset, out_codes, out_scales, out_f32, stream)):
        return
    P = len(codes)
    if len(scales) != P:
        raise ValueError("sdp4_dequant_reduce_sr: codes and scales differ in length")
    _need_reduce(codes, scales, n_chunk, bits_in, group, bits_out, out_codes, out_scales, out_f32)
    cp = (C.c_void_p * max(P, 1))(*[_ptr(c) for c in codes])
    sp = (C.c_void_p * max(P, 1))(*[_ptr(s) for s in scales])
    _ck("sdp4_dequant_reduce_sr", lib().sdp4_dequant_reduce_sr(
        P, C.cast(cp, C.c_void_p), C.cast(sp, C.c_void_p), n_chunk, bits_in, group, bits_out, seed, offset,
        _ptr(out_codes), _ptr(out_scales), _ptr(out_f32), _stream(stream)))


def sdp4_hadamard(x, y, block, n=None, stream=None):
    n = x.numel() if n is None else n
    _need(x, 4 * n, "x"); _need(y, 4 * n, "y")
    _ck("sdp4_hadamard", lib().sdp4_hadamard(_ptr(x), _ptr(y), n, block, _stream(stream)))


def sdp4_reduce_f32(xs, y, n=None, stream=None):
    n = y.numel() if n is None else n
    for i, x in enumerate(xs):
        _need(x, 4 * n, f"xs[{i}]")
    _need(y, 4 * n, "y")
    xp = (C.c_void_p * max(len(xs), 1))(*[_ptr(x) for x in xs])
    _ck("sdp4_reduce_f32", lib().sdp4_reduce_f32(len(xs), C.cast(xp, C.c_void_p), _ptr(y), n,
                                                 _stream(stream)))


def sdp4_copy_f32(x, y, n=None, stream=None):
    n = x.numel() if n is None else n
    _need(x, 4 * n, "x"); _need(y, 4 * n, "y")
    _ck("sdp4_copy_f32", lib().sdp4_copy_f32(_ptr(x), _ptr(y), n, _stream(stream)))


def sdp4_read_f32(x, sink, n=None, stream=None):
    """Read-only stream over x; XORs the bit patterns of x[i] into sink[i % 4]
    (sink: 4 int32 or uint32 words on the device, cleared by the caller)."""
    n = x.numel() if n is None else n
    _need(x, 4 * n, "x"); _need(sink, 16, "sink")
    _ck("sdp4_read_f32", lib().sdp4_read_f32(_ptr(x), n, _ptr(sink), _stream(stream)))


def sdp4_fill_f32(y, value, n=None, stream=None):
    n = y.numel() if n is None else n
    _need(y, 4 * n, "y")
    _ck("sdp4_fill_f32", lib().sdp4_fill_f32(_ptr(y), n, float(value), _stream(stream)))


# -- training-step operators ---------------------------------------------------
# Matrices are two-dimensional device tensors with unit stride in a row (any stride from row to row), heads
# three-dimensional ones [tokens, heads, head_dim] with unit stride in a head; float32 or bfloat16.
def _matrix(x, what, shape=None):
    """(address, element type, row stride, shape) of a matrix."""
    dt = _float_dtype(x, what)
    if x.dim() != 2 or (shape is not None and tuple(x.shape) != tuple(shape)):
        raise ValueError(f"sdp4: {what} must be a matrix{'' if shape is None else ' ' + str(tuple(shape))}, "
                         f"not {tuple(x.shape)}")
    if x.shape[1] > 1 and x.stride(1) != 1:
        raise ValueError(f"sdp4: {what} must have unit stride in its rows")
    return x.data_ptr(), dt, x.stride(0), tuple(x.shape)


def _float_dtype(x, what) -> int:
    import torch
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"sdp4: {what} must be a device tensor")
    if x.dtype == torch.float32:
        return F32
    if x.dtype == torch.bfloat16:
        return BF16
    raise ValueError(f"sdp4: {what} must be float32 or bfloat16, not {x.dtype}")


def _vector(x, shape, dtype, what, optional=True):
    """Address of a contiguous tensor of one shape and type, or None."""
    import torch
    if x is None and optional:
        return None
    if not isinstance(x, torch.Tensor) or not x.is_cuda or tuple(x.shape) != tuple(shape) or not x.is_contiguous() \
            or x.dtype != dtype:
        raise ValueError(f"sdp4: {what} must be a contiguous device tensor {tuple(shape)} of {dtype}")
    return x.data_ptr()


def _scratch(x):
    """Address and size of a workspace."""
    if x is None:
        return None, 0
    return _ptr(x), x.numel() * x.element_size()


def _u64(v) -> int:
    return int(v) & 0xFFFFFFFFFFFFFFFF


def sdp4_dropout_add(x, bias, residual, p, seed, offset, y, stream=None):
    """y <- residual + dropout(x + bias); bias and residual may be None.  The
    mask follows from (seed, offset): see include/sdp4.h."""
    if _fast is not None and _done("sdp4_dropout_add", _fast.dropout_add(x, bias, residual, p, seed, offset, y, stream)):
        return
    xp, xt, xs, shape = _matrix(x, "x")
    yp, yt, ys, _ = _matrix(y, "y", shape)
    rp, rt, rs = None, yt, 0
    if residual is not None:
        rp, rt, rs, _ = _matrix(residual, "residual", shape)
    if rt != yt:
        raise ValueError("sdp4: residual and y must have one type")
    bp = _vector(bias, shape[1:], x.dtype, "bias")
    _ck("sdp4_dropout_add", lib().sdp4_dropout_add(xp, xt, xs, bp, rp, rs, *shape, float(p), _u64(seed), _u64(offset), yp,
                                                   yt, ys, _stream(stream)))


def sdp4_dropout_add_grad(dy, p, seed, offset, dx, dbias=None, workspace=None, stream=None):
    """dx <- the gradient of sdp4_dropout_add's x; dbias <- that of its bias
    (float32; needs a workspace of sdp4_dropout_grad_workspace bytes)."""
    if _fast is not None and _done("sdp4_dropout_add_grad", _fast.dropout_add_grad(
            dy, p, seed, offset, dx, dbias, workspace, stream)):
        return
    import torch
    yp, yt, ys, shape = _matrix(dy, "dy")
    xp, xt, xs, _ = _matrix(dx, "dx", shape)
    bp = _vector(dbias, shape[1:], torch.float32, "dbias")
    _ck("sdp4_dropout_add_grad", lib().sdp4_dropout_add_grad(
        yp, yt, ys, *shape, float(p), _u64(seed), _u64(offset), xp, xt, xs, bp, *_scratch(workspace), _stream(stream)))


def sdp4_dropout_grad_workspace(rows, cols) -> int:
    return lib().sdp4_dropout_grad_workspace(rows, cols)


def _logits(logits, vocab):
    p, dt, stride, shape = _matrix(logits, "logits")
    if vocab is None:
        vocab = shape[1]
    if not 0 < vocab <= shape[1]:
        raise ValueError(f"sdp4: vocab must be in 1..{shape[1]}, the logits' width, not {vocab}")
    return p, dt, stride, shape[0], vocab


def sdp4_token_logprob(logits, targets, top_k, logp, lse, entropy, top_logp=None, top_ids=None, workspace=None,
                       vocab=None, stream=None):
    """Per row of logits: log probability of its target, logsumexp, entropy and
    the top_k alternatives.  Outputs that are None are left out; ``vocab`` is
    the number of columns that count (all by default)."""
    if _fast is not None and _done("sdp4_token_logprob", _fast.token_logprob(
            logits, targets, top_k, logp, lse, entropy, top_logp, top_ids, workspace, vocab, stream)):
        return
    import torch
    f32, i64 = torch.float32, torch.int64
    p, dt, stride, rows, vocab = _logits(logits, vocab)
    top = top_k > 0
    _ck("sdp4_token_logprob", lib().sdp4_token_logprob(
        p, dt, stride, rows, vocab, _vector(targets, (rows,), i64, "targets"), top_k,
        _vector(logp, (rows,), f32, "logp"), _vector(lse, (rows,), f32, "lse"),
        _vector(entropy, (rows,), f32, "entropy"),
        _vector(top_logp, (rows, top_k), f32, "top_logp", False) if top else None,
        _vector(top_ids, (rows, top_k), i64, "top_ids", False) if top else None, *_scratch(workspace), _stream(stream)))


def sdp4_token_logprob_workspace(rows, vocab, top_k=0) -> int:
    return lib().sdp4_token_logprob_workspace(rows, vocab, top_k)


def _gradients(logits, targets, g_logp, g_entropy, g_lse, dlogits, vocab):
    import torch
    f32 = torch.float32
    p, dt, stride, rows, vocab = _logits(logits, vocab)
    dp, ddt, dstride, dshape = _matrix(dlogits, "dlogits")
    if ddt != dt or dshape[0] != rows or dshape[1] < vocab:
        raise ValueError("sdp4: dlogits must have the logits' type and rows, and vocab columns or more")
    return (p, dt, stride, rows, vocab, _vector(targets, (rows,), torch.int64, "targets")), \
        [_vector(g, (rows,), f32, n) for g, n in ((g_logp, "g_logp"), (g_entropy, "g_entropy"), (g_lse, "g_lse"))], \
        (dp, dstride, dshape[1])


def sdp4_token_logprob_grad(logits, targets, lse, entropy, g_logp, g_entropy, g_lse, dlogits, vocab=None, stream=None):
    """dlogits <- the gradient of a loss by the logits, from its gradients by
    logp, entropy and lse (None: zero); columns from vocab on are set to 0."""
    if _fast is not None and _done("sdp4_token_logprob_grad", _fast.token_logprob_grad(
            logits, targets, lse, entropy, g_logp, g_entropy, g_lse, dlogits, vocab, stream)):
        return
    import torch
    f32 = torch.float32
    head, g, tail = _gradients(logits, targets, g_logp, g_entropy, g_lse, dlogits, vocab)
    rows = (head[3],)
    _ck("sdp4_token_logprob_grad", lib().sdp4_token_logprob_grad(
        *head, _vector(lse, rows, f32, "lse", False), _vector(entropy, rows, f32, "entropy"), *g, *tail,
        _stream(stream)))


def sdp4_token_loss(logits, targets, g_logp, g_entropy, g_lse, logp, lse, entropy, dlogits, workspace=None, vocab=None,
                    stream=None):
    """sdp4_token_logprob (without alternatives) and sdp4_token_logprob_grad in
    one pass over the logits, for weights that are known before."""
    if _fast is not None and _done("sdp4_token_loss", _fast.token_loss(
            logits, targets, g_logp, g_entropy, g_lse, logp, lse, entropy, dlogits, workspace, vocab, stream)):
        return
    import torch
    f32 = torch.float32
    head, g, tail = _gradients(logits, targets, g_logp, g_entropy, g_lse, dlogits, vocab)
    rows = (head[3],)
    _ck("sdp4_token_loss", lib().sdp4_token_loss(
        *head, *g, _vector(logp, rows, f32, "logp"), _vector(lse, rows, f32, "lse", False),
        _vector(entropy, rows, f32, "entropy", False), *tail, *_scratch(workspace), _stream(stream)))


def _heads(x, what, like=None, dtype=None):
    """``sdp4_heads`` of a tensor [tokens, heads, head_dim]."""
    _float_dtype(x, what)
    if x.dim() != 3 or (like is not None and x.shape != like.shape) or (dtype is not None and x.dtype != dtype):
        raise ValueError(f"sdp4: {what} must be [tokens, heads, head_dim]"
                         + ("" if like is None else f" = {tuple(like.shape)}")
                         + ("" if dtype is None else f" of {dtype}") + f", not {tuple(x.shape)} of {x.dtype}")
    if x.shape[2] > 1 and x.stride(2) != 1:
        raise ValueError(f"sdp4: {what} must have unit stride in its heads")
    return Heads(x.data_ptr(), x.stride(0), x.stride(1), x.shape[1])


def _by_ref(h):
    return None if h is None else C.addressof(h)


def _qk_params(x, q_weight, k_weight, eps, table, positions, interleaved):
    import torch
    tokens, _, dim = x.shape
    rows = rot = 0
    if table is not None:
        if table.dim() != 2:
            raise ValueError("sdp4: table must be [positions, rot_dim]")
        rows, rot = table.shape
    return QkParams(_float_dtype(x, "heads"), dim, eps is not None, 0.0 if eps is None else eps,
                    _vector(q_weight, (dim,), x.dtype, "q_weight"), _vector(k_weight, (dim,), x.dtype, "k_weight"),
                    _vector(table, (rows, rot), torch.float32, "table"), rows, rot, bool(interleaved),
                    _vector(positions, (tokens,), torch.int64, "positions"))


def sdp4_qk_norm_rope(q, k, q_weight, k_weight, eps, table, positions, q_out, k_out, interleaved=False, stream=None):
    """q_out, k_out <- RMS norm (none if eps is None) and rotation of query and
    key heads [tokens, heads, head_dim]; k and k_out may be None.  The first
    table.shape[1] elements of a head turn by the angles of its token's row
    (cosines, then sines; table None: no rotation)."""
    if _fast is not None and _done("sdp4_qk_norm_rope", _fast.qk_norm_rope(
            q, k, q_weight, k_weight, eps, table, positions, q_out, k_out, interleaved, stream)):
        return
    qh, qo = _heads(q, "q"), _heads(q_out, "q_out", q, q.dtype)
    kh, ko = _keys(q, k, k_out, "k", "k_out")
    prm = _qk_params(q, q_weight, k_weight, eps, table, positions, interleaved)
    _ck("sdp4_qk_norm_rope", lib().sdp4_qk_norm_rope(_by_ref(qh), _by_ref(kh), C.addressof(prm), q.shape[0], _by_ref(qo),
                                                     _by_ref(ko), _stream(stream)))


def _keys(q, k, out, name, out_name):
    """Keys beside the queries ``q``, and the array of their shape: both or neither."""
    if (k is None) != (out is None):
        raise ValueError(f"sdp4: {name} and {out_name} must both be given or both be None")
    if k is None:
        return None, None
    kh, ko = _heads(k, name, None, q.dtype), _heads(out, out_name, k, q.dtype)
    if k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2]:
        raise ValueError(f"sdp4: {name} must have the queries' tokens and head_dim")
    return kh, ko


def sdp4_qk_norm_rope_grad(dq_out, dk_out, q, k, q_weight, k_weight, eps, table, positions, dq, dk, dq_weight=None,
                           dk_weight=None, workspace=None, interleaved=False, stream=None):
    """dq, dk and the float32 dq_weight, dk_weight (each may be None) <- the
    gradients of sdp4_qk_norm_rope from dq_out, dk_out; q and k may be None
    without a norm.  Weight gradients need a workspace of
    sdp4_qk_grad_workspace bytes."""
    if _fast is not None and _done("sdp4_qk_norm_rope_grad", _fast.qk_norm_rope_grad(
            dq_out, dk_out, q, k, q_weight, k_weight, eps, table, positions, dq, dk, dq_weight, dk_weight, workspace,
            interleaved, stream)):
        return
    import torch
    norm, dim = eps is not None, dq_out.shape[-1]
    gq, oq = _heads(dq_out, "dq_out"), _heads(dq, "dq", dq_out, dq_out.dtype)
    gk, ok = _keys(dq_out, dk_out, dk, "dk_out", "dk")
    hq = _heads(q, "q", dq_out, dq_out.dtype) if norm else None
    hk = _heads(k, "k", dk_out, dq_out.dtype) if norm and dk is not None else None
    prm = _qk_params(dq_out, q_weight, k_weight, eps, table, positions, interleaved)
    _ck("sdp4_qk_norm_rope_grad", lib().sdp4_qk_norm_rope_grad(
        _by_ref(gq), _by_ref(gk), _by_ref(hq), _by_ref(hk), C.addressof(prm), dq_out.shape[0], _by_ref(oq), _by_ref(ok),
        _vector(dq_weight, (dim,), torch.float32, "dq_weight"), _vector(dk_weight, (dim,), torch.float32, "dk_weight"),
        *_scratch(workspace), _stream(stream)))


def sdp4_qk_grad_workspace(tokens, q_heads, k_heads, head_dim) -> int:
    return lib().sdp4_qk_grad_workspace(tokens, q_heads, k_heads, head_dim)


def sdp4_rope_table(inv_freq, table, start=0, scale=1.0, stream=None):
    """table[r] <- scale * (cosines, then sines) of (start + r) * inv_freq, for
    float64 frequencies and a float32 table [rows, 2 * len(inv_freq)]."""
    import torch
    half = inv_freq.numel()
    _ck("sdp4_rope_table", lib().sdp4_rope_table(
        _vector(inv_freq, (half,), torch.float64, "inv_freq", False), half, start, table.shape[0], float(scale),
        _vector(table, (table.shape[0], 2 * half), torch.float32, "table", False), _stream(stream)))


# Attention, block norms and the embedding run on the device of their arrays, which have to lie on one.
class _device:
    """Makes the tensors' device the current one; raises where they lie on several."""

    def __init__(self, *tensors):
        import torch
        devices = {t.device for t in tensors if isinstance(t, torch.Tensor)}
        if len(devices) > 1:
            raise ValueError(f"sdp4: arrays must lie on one device, not on {sorted(map(str, devices))}")
        device = devices.pop() if devices else None
        self.guard = torch.cuda.device(device if device is not None and device.type == "cuda" else None)

    def __enter__(self):
        self.guard.__enter__()

    def __exit__(self, *error):
        self.guard.__exit__(*error)


def _attention_params(q, scale, offsets):
    import torch
    if offsets is None:
        return AttentionParams(_float_dtype(q, "q"), q.shape[2], scale, None, 0)
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("sdp4: offsets must be [sequences + 1]")
    count = offsets.shape[0] - 1
    return AttentionParams(_float_dtype(q, "q"), q.shape[2], scale, _vector(offsets, (count + 1,), torch.int64, "offsets"),
                           count)


def _key_heads(x, what, q, like=None):
    h = _heads(x, what, like, q.dtype)
    if x.shape[0] != q.shape[0] or x.shape[2] != q.shape[2]:
        raise ValueError(f"sdp4: {what} must have the queries' tokens and head_dim")
    return h


def sdp4_attention(q, k, v, scale, offsets, out, lse=None, stream=None):
    """out <- causal attention of heads [tokens, heads, head_dim] over packed
    sequences: rows offsets[n] .. offsets[n + 1] - 1 (int64, on the device;
    None: one sequence), k and v with a divisor of q's heads.  lse
    [q heads, tokens] float32 may be None."""
    if _fast is not None and _done("sdp4_attention", _fast.attention(q, k, v, scale, offsets, out, lse, stream)):
        return
    import torch
    hs = [_heads(q, "q"), _key_heads(k, "k", q), _key_heads(v, "v", q, k), _heads(out, "out", q, q.dtype)]
    prm = _attention_params(q, scale, offsets)
    lp = _vector(lse, (q.shape[1], q.shape[0]), torch.float32, "lse")
    with _device(q, k, v, offsets, out, lse):
        _ck("sdp4_attention", lib().sdp4_attention(*(C.addressof(h) for h in hs[:3]), C.addressof(prm), q.shape[0],
                                                   C.addressof(hs[3]), lp, _stream(stream)))


def sdp4_attention_grad(dout, q, k, v, out, lse, scale, offsets, dq, dk, dv, workspace, stream=None):
    """dq, dk, dv <- the gradients of sdp4_attention from that of its out;
    needs out and lse as it left them and a workspace of
    sdp4_attention_grad_workspace bytes."""
    if _fast is not None and _done("sdp4_attention_grad", _fast.attention_grad(
            dout, q, k, v, out, lse, scale, offsets, dq, dk, dv, workspace, stream)):
        return
    import torch
    hs = [_heads(dout, "dout", q, q.dtype), _heads(q, "q"), _key_heads(k, "k", q), _key_heads(v, "v", q, k),
          _heads(out, "out", q, q.dtype)]
    outs = [_heads(dq, "dq", q, q.dtype), _heads(dk, "dk", k, q.dtype), _heads(dv, "dv", k, q.dtype)]
    prm = _attention_params(q, scale, offsets)
    lp = _vector(lse, (q.shape[1], q.shape[0]), torch.float32, "lse", False)
    with _device(dout, q, k, v, out, lse, offsets, dq, dk, dv, workspace):
        _ck("sdp4_attention_grad", lib().sdp4_attention_grad(
            *(C.addressof(h) for h in hs), lp, C.addressof(prm), q.shape[0], *(C.addressof(h) for h in outs),
            *_scratch(workspace), _stream(stream)))


def sdp4_attention_grad_workspace(tokens, q_heads, k_heads, head_dim) -> int:
    return lib().sdp4_attention_grad_workspace(tokens, q_heads, k_heads, head_dim)


def _block(arrays, post_eps, post_weight, gate, branch_scale, residual_scale, pre_eps, pre_weight):
    """``sdp4_block_params``, the matrices' addresses and strides, and their shape; ``arrays``: (matrix or None, name, whether
    it is of the residual stream)."""
    import torch
    shape, types, out = None, [None, None], []
    for x, what, stream in arrays:
        if x is None:
            out.append((None, 0))
            continue
        p, dt, stride, shape = _matrix(x, what, shape)
        if types[stream] not in (None, dt):
            raise ValueError(f"sdp4: {what} must have the type of the {'residual stream' if stream else 'branch'}")
        types[stream] = dt
        out.append((p, stride))
    if shape is None:
        raise ValueError("sdp4: no matrix given")
    for w, what in ((post_weight, "post_weight"), (pre_weight, "pre_weight")):
        if types[0] is None and w is not None:      # no matrix of the branch's type: its weights have it
            types[0] = _float_dtype(w, what)
    x_type = types[0] if types[0] is not None else types[1]
    y_type = types[1] if types[1] is not None else types[0]
    weight = torch.float32 if x_type == F32 else torch.bfloat16
    prm = BlockParams(x_type, y_type, post_eps is not None, 0.0 if post_eps is None else post_eps,
                      0.0 if pre_eps is None else pre_eps, _vector(post_weight, shape[1:], weight, "post_weight"),
                      _vector(pre_weight, shape[1:], weight, "pre_weight"),
                      _vector(gate, shape[:1], torch.float32, "gate"), branch_scale, residual_scale)
    return prm, out, shape


def sdp4_block_norm(branch, residual, post_eps, post_weight, gate, branch_scale, residual_scale, y, pre_eps, pre_weight, h,
                    stream=None):
    """u <- the RMS norm of branch times post_weight (post_eps None: no norm),
    y <- residual_scale * residual + branch_scale * gate * u, h <- the RMS norm
    of y times pre_weight.  gate [rows] is float32; branch or residual, y or
    h, weights and gate may be None."""
    if _fast is not None and _done("sdp4_block_norm", _fast.block_norm(
            branch, residual, post_eps, post_weight, gate, branch_scale, residual_scale, y, pre_eps, pre_weight, h, stream)):
        return
    prm, (b, r, yo, ho), shape = _block([(branch, "branch", 0), (residual, "residual", 1), (y, "y", 1), (h, "h", 0)], post_eps,
                                        post_weight, gate, branch_scale, residual_scale, pre_eps, pre_weight)
    with _device(branch, residual, post_weight, gate, y, pre_weight, h):
        _ck("sdp4_block_norm", lib().sdp4_block_norm(*b, *r, *shape, C.addressof(prm), *yo, *ho, _stream(stream)))


def sdp4_block_norm_grad(dh, dy, branch, y, post_eps, post_weight, gate, branch_scale, residual_scale, pre_eps, pre_weight,
                         dbranch, dresidual, dpost_weight=None, dpre_weight=None, dgate=None, workspace=None, stream=None):
    """dbranch, dresidual and the float32 dpost_weight, dpre_weight, dgate <-
    the gradients of sdp4_block_norm from those of h and y (None: zero); what
    is None is left out.  Weight gradients need a workspace of
    sdp4_block_norm_grad_workspace bytes."""
    if _fast is not None and _done("sdp4_block_norm_grad", _fast.block_norm_grad(
            dh, dy, branch, y, post_eps, post_weight, gate, branch_scale, residual_scale, pre_eps, pre_weight, dbranch, dresidual,
            dpost_weight, dpre_weight, dgate, workspace, stream)):
        return
    import torch
    prm, (g, gy, b, yi, db, dr), shape = _block(
        [(dh, "dh", 0), (dy, "dy", 1), (branch, "branch", 0), (y, "y", 1), (dbranch, "dbranch", 0), (dresidual, "dresidual", 1)],
        post_eps, post_weight, gate, branch_scale, residual_scale, pre_eps, pre_weight)
    with _device(dh, dy, branch, y, post_weight, gate, pre_weight, dbranch, dresidual, dpost_weight, dpre_weight, dgate,
                 workspace):
        _ck("sdp4_block_norm_grad", lib().sdp4_block_norm_grad(
            *g, *gy, *b, *yi, *shape, C.addressof(prm), *db, *dr, _vector(dpost_weight, shape[1:], torch.float32, "dpost_weight"),
            _vector(dpre_weight, shape[1:], torch.float32, "dpre_weight"), _vector(dgate, shape[:1], torch.float32, "dgate"),
            *_scratch(workspace), _stream(stream)))


def sdp4_block_norm_grad_workspace(rows, cols) -> int:
    return lib().sdp4_block_norm_grad_workspace(rows, cols)


def sdp4_embedding(tokens, table, scale, out, stream=None):
    """out[r] <- scale * table[tokens[r]] for int64 tokens (negative: zeros)."""
    if _fast is not None and _done("sdp4_embedding", _fast.embedding(tokens, table, scale, out, stream)):
        return
    import torch
    tp, tt, ts, (vocab, cols) = _matrix(table, "table")
    op, ot, os_, (rows, _) = _matrix(out, "out", (out.shape[0], cols))
    ids = _vector(tokens, (rows,), torch.int64, "tokens", False)
    with _device(tokens, table, out):
        _ck("sdp4_embedding", lib().sdp4_embedding(ids, rows, tp, tt, ts, vocab, cols, scale, op, ot, os_, _stream(stream)))


def sdp4_embedding_grad(tokens, dout, scale, dtable, workspace, accumulate=False, stream=None):
    """dtable <- (accumulate: +=) the gradient of sdp4_embedding's table;
    needs a workspace of sdp4_embedding_grad_workspace bytes."""
    if _fast is not None and _done("sdp4_embedding_grad", _fast.embedding_grad(
            tokens, dout, scale, dtable, workspace, accumulate, stream)):
        return
    import torch
    tp, tt, ts, (vocab, cols) = _matrix(dtable, "dtable")
    dp, dt, ds, (rows, _) = _matrix(dout, "dout", (dout.shape[0], cols))
    ids = _vector(tokens, (rows,), torch.int64, "tokens", False)
    with _device(tokens, dout, dtable, workspace):
        _ck("sdp4_embedding_grad", lib().sdp4_embedding_grad(ids, rows, dp, dt, ds, vocab, cols, scale, bool(accumulate), tp, tt,
                                                             ts, *_scratch(workspace), _stream(stream)))


def sdp4_embedding_grad_workspace(rows, vocab, cols) -> int:
    return lib().sdp4_embedding_grad_workspace(rows, vocab, cols)


def sdp4_codes_bytes(n, bits):
    return lib().sdp4_codes_bytes(n, bits)


def sdp4_num_groups(n, group):
    return lib().sdp4_num_groups(n, group)


def sdp4_version() -> str:
    return lib().sdp4_version().decode()
