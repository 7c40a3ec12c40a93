"""Thin ctypes binding of libmnmt (include/mnmt.h): the same calls, argument
marshalling only.  Every step of the translation path runs in the library's
sm_103a kernels; if the library is missing or fails to load, importing this
module's functions raises — there is no fallback.

Host arrays are numpy arrays; device arrays are torch CUDA tensors (or raw
integer device addresses) — torch is used only for device memory and streams.
"""
from __future__ import annotations

import ctypes as C
import os
import threading

import numpy as np

from . import build as _build

OK, EINVAL, ENOMEM, ECUDA, ETIMEOUT, EFORMAT, EOVERFLOW = 0, -1, -2, -3, -4, -5, -6
DEVICE_PTRS = 1
F32, BF16, F16 = 0, 1, 2
FP4_MX, FP4_NV = 0, 1
DROPOUT_WORKSPACE = 16384
EPI_Q8, EPI_RELU_Q8, EPI_RESID, EPI_F32, EPI_ARGMAX = 0, 1, 2, 3, 4
(TAP_ENC_OUT, TAP_CROSS_K, TAP_CROSS_V, TAP_SELF_K, TAP_SELF_V, TAP_DEC_OUT, TAP_LOGITS, TAP_RESID,
 TAP_HISTORY, TAP_PARENTS, TAP_ANCESTRY, TAP_STEP) = range(1, 13)

_lock = threading.Lock()
_lib = None


class MnmtError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"mnmt error {code}: {msg}")
        self.code = code


class _Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ["n_enc", "n_dec", "d_model", "n_heads", "d_ffn", "vocab", "d_embed",
                                         "pre_ln", "tied_output", "max_pos", "pad_id", "bos_id", "eos_id"]]


class Fp4(C.Structure):
    """A matrix in microscaled 4-bit floating point (mnmt_fp4): where its codes
    and scales are (device buffers, kept alive by this object; None: none)."""
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("rows", C.c_int32), ("cols", C.c_int32),
                ("format", C.c_int32), ("tensor_scale", C.c_float)]

    def __init__(self, rows, cols, format, tensor_scale=1.0, codes=None, scales=None):
        super().__init__(_ptr(codes), _ptr(scales), rows, cols, format, tensor_scale)
        self.buffers = codes, scales


class AttentionShape(C.Structure):
    """A batch of sequences and its heads (mnmt_attention_shape): starts and lengths are device buffers, kept alive by
    this object."""
    _fields_ = [(n, C.c_int32) for n in ["n_seqs", "q_rows", "k_rows", "q_heads", "kv_heads", "d_head", "dtype", "causal"]] + \
        [("scale", C.c_float)] + [(n, C.c_void_p) for n in ["q_start", "q_len", "k_start", "k_len"]]

    def __init__(self, n_seqs, q_rows, k_rows, q_heads, kv_heads, d_head, dtype, causal, scale, q_start, k_start, q_len=None,
                 k_len=None):
        super().__init__(n_seqs, q_rows, k_rows, q_heads, kv_heads, d_head, dtype, int(causal), scale, _ptr(q_start), _ptr(q_len),
                         _ptr(k_start), _ptr(k_len))
        self.buffers = q_start, q_len, k_start, k_len


class Heads(C.Structure):
    """Rows of heads (mnmt_heads): the buffer and its row and head strides in elements."""
    _fields_ = [("data", C.c_void_p), ("row", C.c_int64), ("head", C.c_int64)]

    def __init__(self, data, row, head):
        super().__init__(_ptr(data), row, head)
        self.buffer = data


def heads(x) -> Heads:
    """The Heads of a tensor [rows][heads][d] whose elements of a head lie one after another."""
    row, head, one = x.stride()
    if one != 1 and x.shape[2] > 1:
        raise ValueError("heads: elements of a head must lie one after another")
    return Heads(x, row, head)


def lib_path() -> str:
    return _build.LIB


def lib():
    """Load libmnmt.so (building it first if its sources are newer)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            path = _build.build()
            if not os.path.exists(path):
                raise RuntimeError(f"libmnmt.so missing at {path}")
            L = C.CDLL(path)
            _declare(L)
            _lib = L
    return _lib


def _declare(L):
    p, i32, sz, f = C.c_void_p, C.c_int32, C.c_size_t, C.c_float
    L.mnmt_blob_check.argtypes = [p, sz, C.POINTER(_Config)]
    L.mnmt_load_weights.argtypes = [p, sz, p, C.POINTER(p)]
    L.mnmt_load_weights_ex.argtypes = [p, sz, p, i32, C.POINTER(p)]
    L.mnmt_session_create_ex.argtypes = [p, i32, i32, i32, i32, i32, C.POINTER(p)]
    L.mnmt_model_device_bytes.argtypes = [p]; L.mnmt_model_device_bytes.restype = C.c_int64
    L.mnmt_session_device_bytes.argtypes = [p]; L.mnmt_session_device_bytes.restype = C.c_int64
    L.mnmt_model_free.argtypes = [p]; L.mnmt_model_free.restype = None
    L.mnmt_model_config.argtypes = [p, C.POINTER(_Config)]
    L.mnmt_session_create.argtypes = [p, i32, i32, i32, i32, C.POINTER(p)]
    L.mnmt_session_free.argtypes = [p]; L.mnmt_session_free.restype = None
    L.mnmt_encode.argtypes = [p, p, p, i32, i32, i32]
    L.mnmt_decode_step.argtypes = [p, p, p, p, p]
    L.mnmt_decode_steps.argtypes = [p, i32]; L.mnmt_decode_steps.restype = C.c_int
    L.mnmt_translate.argtypes = [p, p, p, i32, i32, i32, i32, p, p, p]
    L.mnmt_debug_tap.argtypes = [p, i32, i32, p, sz]; L.mnmt_debug_tap.restype = C.c_int64
    L.mnmt_session_decode_path.argtypes = [p]; L.mnmt_session_decode_path.restype = C.c_int
    L.mnmt_last_error.argtypes = []; L.mnmt_last_error.restype = C.c_char_p
    L.mnmt_linear.argtypes = [p, p, p, p, f, p, f, i32, i32, i32, i32, p, p, p]
    L.mnmt_linear_argmax.argtypes = [p, p, p, p, f, i32, i32, i32, p, p]
    L.mnmt_linear_argmax_ids_noalloc.argtypes = [p, p, p, p, f, i32, i32, i32, p, p]
    L.mnmt_linear_argmax_ids_noalloc.restype = C.c_int
    L.mnmt_attention_decode.argtypes = [p, p, p, p, i32, i32, i32, i32, f, f, p, p]
    L.mnmt_layernorm.argtypes = [p, p, p, i32, i32, f, p, p, p, p]
    L.mnmt_linear_tc.argtypes = [p, p, p, p, f, p, f, i32, i32, i32, i32, p, p, p, p, p]
    L.mnmt_codes_to_f16.argtypes = [p, p, sz, p]
    L.mnmt_linear_w4.argtypes = [p, p, p, p, p, f, p, f, i32, i32, i32, i32, p, p, p, p]
    L.mnmt_linear_w4.restype = C.c_int
    L.mnmt_fake_quant.argtypes = [p, sz, f, f, i32, i32, p, p, p]
    L.mnmt_fake_quant_backward.argtypes = [p, p, sz, f, f, i32, i32, p, p, p, p]
    L.mnmt_fake_quant_linear.argtypes = [p, p, f, p, p, i32, i32, i32, i32, p, p, p]
    fp4, i64, u64 = C.POINTER(Fp4), C.c_int64, C.c_uint64
    L.mnmt_fp4_pitch.argtypes = [i32]; L.mnmt_fp4_pitch.restype = sz
    L.mnmt_fp4_scale_bytes.argtypes = [i32, i32, i32]; L.mnmt_fp4_scale_bytes.restype = sz
    L.mnmt_fp4_quantize.argtypes = [fp4, p, i32, i64, p, i64, p]
    L.mnmt_fp4_dequantize.argtypes = [fp4, p, i32, i64, p]
    L.mnmt_fp4_quantize_backward.argtypes = [fp4, p, i32, i64, p, i64, p, i64, p]
    L.mnmt_fp4_linear.argtypes = [fp4, fp4, p, i32, i64, p, i32, p, i32, i64, p, p]
    L.mnmt_fp4_linear_backward_workspace.argtypes = [i32, i32, i32]
    L.mnmt_fp4_linear_backward_workspace.restype = sz
    L.mnmt_fp4_linear_backward.argtypes = [fp4, fp4, p, i64, p, i32, i64, p, i32, i64, p, p, i64, p, i64, p, p, p]
    L.mnmt_dropout.argtypes = [p, i32, i64, p, i64, f, f, u64, u64, i32, i32, i32, p, i32, i64, p]
    L.mnmt_dropout_backward.argtypes = [p, i32, i64, p, i32, i64, p, i64, f, f, u64, u64, i32, i32, i32, p, i64, p, i64,
                                        p, p, p]
    shape, hd = C.POINTER(AttentionShape), C.POINTER(Heads)
    for n in ["forward", "backward", "token"]:
        size = getattr(L, f"mnmt_attention_{n}_workspace")
        size.argtypes, size.restype = [shape], sz
    L.mnmt_attention_forward.argtypes = L.mnmt_attention_token.argtypes = [shape, hd, hd, hd, hd, p, p, p, p]
    L.mnmt_attention_backward.argtypes = [shape, hd, hd, hd, hd, p, hd, hd, hd, hd, p, p, p]
    L.mnmt_embed.argtypes = [p, i32, p, i32, i64, i32, i32, f, p, p, i64, i32, p, i32, i64, p, p]
    L.mnmt_embed_backward_workspace.argtypes = [i32, i32, i32]; L.mnmt_embed_backward_workspace.restype = sz
    L.mnmt_embed_backward.argtypes = [p, i32, p, i32, i64, f, i32, i32, i32, p, i32, i64, i32, p, p, p]
    for n in ["mnmt_attention_forward", "mnmt_attention_backward", "mnmt_attention_token", "mnmt_embed", "mnmt_embed_backward"]:
        getattr(L, n).restype = C.c_int
    for n in ["mnmt_fp4_quantize", "mnmt_fp4_dequantize", "mnmt_fp4_quantize_backward", "mnmt_fp4_linear",
              "mnmt_fp4_linear_backward", "mnmt_dropout", "mnmt_dropout_backward"]:
        getattr(L, n).restype = C.c_int
    for n in ["mnmt_fake_quant", "mnmt_fake_quant_backward", "mnmt_fake_quant_linear"]:
        getattr(L, n).restype = C.c_int
    L.mnmt_wait_timeout_selftest.argtypes = [p, p]
    for n in ["mnmt_blob_check", "mnmt_load_weights", "mnmt_load_weights_ex", "mnmt_session_create_ex",
              "mnmt_model_config", "mnmt_session_create", "mnmt_encode",
              "mnmt_decode_step", "mnmt_translate", "mnmt_linear", "mnmt_linear_argmax", "mnmt_attention_decode", "mnmt_layernorm",
              "mnmt_linear_tc", "mnmt_codes_to_f16", "mnmt_wait_timeout_selftest"]:
        getattr(L, n).restype = C.c_int


def last_error() -> str:
    return lib().mnmt_last_error().decode()


def _chk(code):
    if code != OK:
        raise MnmtError(code, last_error())
    return code


def _ptr(x):
    """Address of a numpy array, a torch tensor, or an integer address."""
    if x is None:
        return None
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    return x


def _stream_handle(stream):
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# --------------------------------------------------------------------------- C calls
def mnmt_blob_check(blob: bytes) -> dict:
    cfg = _Config()
    _chk(lib().mnmt_blob_check(blob, len(blob), C.byref(cfg)))
    return {n: getattr(cfg, n) for n, _ in _Config._fields_}


LOAD_LEAN = 1
SESSION_LEAN = 1


def mnmt_load_weights(blob: bytes, stream=None, flags: int = 0) -> int:
    h = C.c_void_p()
    if flags:
        _chk(lib().mnmt_load_weights_ex(blob, len(blob), _stream_handle(stream), flags, C.byref(h)))
    else:
        _chk(lib().mnmt_load_weights(blob, len(blob), _stream_handle(stream), C.byref(h)))
    return h.value


def mnmt_model_device_bytes(model: int) -> int:
    r = lib().mnmt_model_device_bytes(model)
    if r < 0:
        raise MnmtError(int(r), last_error())
    return int(r)


def mnmt_session_device_bytes(session: int) -> int:
    r = lib().mnmt_session_device_bytes(session)
    if r < 0:
        raise MnmtError(int(r), last_error())
    return int(r)


def mnmt_model_free(model: int):
    lib().mnmt_model_free(model)


def mnmt_model_config(model: int) -> dict:
    cfg = _Config()
    _chk(lib().mnmt_model_config(model, C.byref(cfg)))
    return {n: getattr(cfg, n) for n, _ in _Config._fields_}


def mnmt_session_create(model: int, max_batch: int, max_src_len: int, beam: int, max_len: int,
                        flags: int = 0) -> int:
    h = C.c_void_p()
    if flags:
        _chk(lib().mnmt_session_create_ex(model, max_batch, max_src_len, beam, max_len, flags, C.byref(h)))
    else:
        _chk(lib().mnmt_session_create(model, max_batch, max_src_len, beam, max_len, C.byref(h)))
    return h.value


def mnmt_session_free(session: int):
    lib().mnmt_session_free(session)


def mnmt_encode(session: int, src_ids, src_lens, B: int, S_pad: int, flags: int = 0):
    _chk(lib().mnmt_encode(session, _ptr(src_ids), _ptr(src_lens), B, S_pad, flags))


def mnmt_decode_steps(session: int, n: int) -> int:
    """Queue n decode steps without waiting; returns the number queued."""
    r = lib().mnmt_decode_steps(session, n)
    if r < 0:
        raise MnmtError(r, last_error())
    return r


def mnmt_decode_step(session: int, R: int):
    """One decode step; returns (tokens [R], parents [R], scores [R], all_done)."""
    tok = np.zeros(R, np.int32); par = np.zeros(R, np.int32); sc = np.zeros(R, np.float32)
    done = C.c_int32(0)
    _chk(lib().mnmt_decode_step(session, _ptr(tok), _ptr(par), _ptr(sc), C.byref(done)))
    return tok, par, sc, bool(done.value)


def mnmt_translate(session: int, src_ids, src_lens, B: int, S_pad: int, max_len: int, flags: int,
                   out_ids, out_lens, out_scores):
    _chk(lib().mnmt_translate(session, _ptr(src_ids), _ptr(src_lens), B, S_pad, max_len, flags,
                              _ptr(out_ids), _ptr(out_lens), _ptr(out_scores)))


def mnmt_debug_tap(session: int, tap: int, layer: int = 0, dtype=np.int8, shape=None) -> np.ndarray:
    n = lib().mnmt_debug_tap(session, tap, layer, None, 0)
    if n < 0:
        raise MnmtError(int(n), last_error())
    out = np.zeros(n // np.dtype(dtype).itemsize, dtype)
    _chk(int(lib().mnmt_debug_tap(session, tap, layer, _ptr(out), n)))
    return out.reshape(shape) if shape is not None else out


def mnmt_session_decode_path(session: int) -> int:
    """1 if the session's decode step runs on one thread-block cluster, 0 for the multi-kernel step."""
    r = lib().mnmt_session_decode_path(session)
    if r < 0:
        raise MnmtError(r, last_error())
    return r


def mnmt_linear(A, W, s_w, bias, s_x, inv_out, gamma, M, N, K, mode, out_q, out_f, stream=None):
    _chk(lib().mnmt_linear(_ptr(A), _ptr(W), _ptr(s_w), _ptr(bias), float(s_x), _ptr(inv_out), float(gamma),
                           M, N, K, mode, _ptr(out_q), _ptr(out_f), _stream_handle(stream)))


def mnmt_linear_argmax(A, W, s_w, bias, s_x, M, N, K, keys, stream=None):
    _chk(lib().mnmt_linear_argmax(_ptr(A), _ptr(W), _ptr(s_w), _ptr(bias), float(s_x), M, N, K, _ptr(keys),
                                  _stream_handle(stream)))


def mnmt_linear_argmax_ids_noalloc(A, W, s_w, bias, s_x, M, N, K, ids, stream=None):
    """Greedy vocabulary argmax into int32 ids with library-owned scratch (no allocation)."""
    _chk(lib().mnmt_linear_argmax_ids_noalloc(_ptr(A), _ptr(W), _ptr(s_w), _ptr(bias), float(s_x), M, N, K,
                                              _ptr(ids), _stream_handle(stream)))


def mnmt_linear_tc(A16, W16, s_w, bias, s_x, inv_out, gamma, M, N, K, mode, out_q=None, out_f=None, keys=None,
                   status=None, stream=None):
    """Tensor-core quantised linear over fp16 copies of the int8 codes (see mnmt_codes_to_f16)."""
    _chk(lib().mnmt_linear_tc(_ptr(A16), _ptr(W16), _ptr(s_w), _ptr(bias), float(s_x), _ptr(inv_out), float(gamma),
                              M, N, K, mode, _ptr(out_q), _ptr(out_f), _ptr(keys), _ptr(status),
                              _stream_handle(stream)))


def mnmt_linear_w4(A, Wp, s_w, m_w, bias, s_x, inv_out, gamma, M, N, K, mode, out_q=None, out_f=None, keys=None,
                   stream=None):
    """Quantised linear with row-wise 4-bit weights (m_w None: symmetric rows)."""
    _chk(lib().mnmt_linear_w4(_ptr(A), _ptr(Wp), _ptr(s_w), _ptr(m_w), _ptr(bias), float(s_x), _ptr(inv_out),
                              float(gamma), M, N, K, mode, _ptr(out_q), _ptr(out_f), _ptr(keys),
                              _stream_handle(stream)))


def mnmt_fake_quant(x, n, s, r_m=0.0, bits=8, minmax=False, y=None, codes=None, stream=None):
    """QAT fake quantisation (device buffers): y = Q(x), codes = q (int32)."""
    _chk(lib().mnmt_fake_quant(_ptr(x), n, float(s), float(r_m), bits, int(minmax), _ptr(y), _ptr(codes),
                               _stream_handle(stream)))


def mnmt_fake_quant_backward(x, g, n, s, gx, gs, gr=None, r_m=0.0, bits=8, minmax=False, stream=None):
    """STE gradient gx and the scale / offset gradients gs, gr (device fp64 scalars)."""
    _chk(lib().mnmt_fake_quant_backward(_ptr(x), _ptr(g), n, float(s), float(r_m), bits, int(minmax), _ptr(gx),
                                        _ptr(gs), _ptr(gr), _stream_handle(stream)))


def mnmt_fake_quant_linear(X, W, s_x, s_w, bias, M, N, K, wbits, workspace, y, stream=None):
    """QAT forward of a linear from fp32 input and weights (learnable scales)."""
    _chk(lib().mnmt_fake_quant_linear(_ptr(X), _ptr(W), float(s_x), _ptr(s_w), _ptr(bias), M, N, K, wbits,
                                      _ptr(workspace), _ptr(y), _stream_handle(stream)))


def mnmt_fp4_pitch(cols: int) -> int:
    return lib().mnmt_fp4_pitch(cols)


def mnmt_fp4_scale_bytes(rows: int, cols: int, format: int) -> int:
    return lib().mnmt_fp4_scale_bytes(rows, cols, format)


def mnmt_fp4_quantize(q: Fp4, x, dtype, ldx, values=None, ldv=0, stream=None):
    """x into q's codes and scales (where it has them) and into values (device buffers)."""
    _chk(lib().mnmt_fp4_quantize(q, _ptr(x), dtype, ldx, _ptr(values), ldv, _stream_handle(stream)))


def mnmt_fp4_dequantize(q: Fp4, values, dtype, ldv, stream=None):
    _chk(lib().mnmt_fp4_dequantize(q, _ptr(values), dtype, ldv, _stream_handle(stream)))


def mnmt_fp4_quantize_backward(q: Fp4, x, dtype, ldx, g, ldg, gx, ldgx, stream=None):
    """Straight-through gradient of mnmt_fp4_quantize's values."""
    _chk(lib().mnmt_fp4_quantize_backward(q, _ptr(x), dtype, ldx, _ptr(g), ldg, _ptr(gx), ldgx, _stream_handle(stream)))


def mnmt_fp4_linear(xq: Fp4, w: Fp4, x, xdtype, ldx, bias, relu, y, ydtype, ldy, status=None, stream=None):
    """Linear on 4-bit floating-point operands; x (None: xq holds it already) is quantised into xq first."""
    _chk(lib().mnmt_fp4_linear(xq, w, _ptr(x), xdtype, ldx, _ptr(bias), int(relu), _ptr(y), ydtype, ldy, _ptr(status),
                               _stream_handle(stream)))


def mnmt_fp4_linear_backward_workspace(M: int, N: int, K: int) -> int:
    return lib().mnmt_fp4_linear_backward_workspace(M, N, K)


def mnmt_fp4_linear_backward(xq: Fp4, wq: Fp4, g, ldg, x, xdtype, ldx, w, wdtype, ldw, workspace, gx=None, ldgx=0, gw=None,
                             ldgw=0, gb=None, status=None, stream=None):
    """Gradients of mnmt_fp4_linear for bf16 output gradients g (x, w: the originals, None: no straight-through mask)."""
    _chk(lib().mnmt_fp4_linear_backward(xq, wq, _ptr(g), ldg, _ptr(x), xdtype, ldx, _ptr(w), wdtype, ldw, _ptr(workspace),
                                        _ptr(gx), ldgx, _ptr(gw), ldgw, _ptr(gb), _ptr(status), _stream_handle(stream)))


def mnmt_dropout(x, dtype, ldx, r, ldr, gamma, p, seed, offset, relu, M, d, out, otype, ldo, stream=None):
    """out = gamma r + dropout(relu?(x)) (r None: no residual)."""
    _chk(lib().mnmt_dropout(_ptr(x), dtype, ldx, _ptr(r), ldr, gamma, p, seed, offset, int(relu), M, d, _ptr(out), otype,
                            ldo, _stream_handle(stream)))


def mnmt_dropout_backward(g, otype, ldg, x, dtype, ldx, r, ldr, gamma, p, seed, offset, relu, M, d, gx=None, ldgx=0, gr=None,
                          ldgr=0, ggamma=None, workspace=None, stream=None):
    """Gradients of mnmt_dropout: gx, gr and the scalar ggamma, each where given."""
    _chk(lib().mnmt_dropout_backward(_ptr(g), otype, ldg, _ptr(x), dtype, ldx, _ptr(r), ldr, gamma, p, seed, offset,
                                     int(relu), M, d, _ptr(gx), ldgx, _ptr(gr), ldgr, _ptr(ggamma), _ptr(workspace),
                                     _stream_handle(stream)))


def mnmt_attention_forward_workspace(shape: AttentionShape) -> int:
    return lib().mnmt_attention_forward_workspace(shape)


def mnmt_attention_backward_workspace(shape: AttentionShape) -> int:
    return lib().mnmt_attention_backward_workspace(shape)


def mnmt_attention_token_workspace(shape: AttentionShape) -> int:
    return lib().mnmt_attention_token_workspace(shape)


def mnmt_attention_forward(shape: AttentionShape, q: Heads, k: Heads, v: Heads, o: Heads, lse, workspace, status=None, stream=None):
    """Softmax attention of a batch of sequences into o and (where given) lse [q_heads][q_rows]."""
    _chk(lib().mnmt_attention_forward(shape, q, k, v, o, _ptr(lse), _ptr(workspace), _ptr(status), _stream_handle(stream)))


def mnmt_attention_backward(shape: AttentionShape, q: Heads, k: Heads, v: Heads, o: Heads, lse, g: Heads, dq: Heads, dk: Heads, dv: Heads,
                            workspace, status=None, stream=None):
    """Gradients dq, dk and dv of mnmt_attention_forward for the gradient g of o."""
    _chk(lib().mnmt_attention_backward(shape, q, k, v, o, _ptr(lse), g, dq, dk, dv, _ptr(workspace), _ptr(status), _stream_handle(stream)))


def mnmt_attention_token(shape: AttentionShape, q: Heads, k: Heads, v: Heads, o: Heads, lse, workspace, status=None, stream=None):
    """Attention of one query per sequence against a cache of keys and values."""
    _chk(lib().mnmt_attention_token(shape, q, k, v, o, _ptr(lse), _ptr(workspace), _ptr(status), _stream_handle(stream)))


def mnmt_embed(ids, T, table, dtype, ldt, V, d, scale, out, otype, ldo, pos=None, pe=None, ldpe=0, P=0, status=None, stream=None):
    """out[t] = scale table[ids[t]] + pe[pos[t]] (pe None: nothing added, pos None: position t)."""
    _chk(lib().mnmt_embed(_ptr(ids), T, _ptr(table), dtype, ldt, V, d, scale, _ptr(pos), _ptr(pe), ldpe, P, _ptr(out), otype, ldo,
                          _ptr(status), _stream_handle(stream)))


def mnmt_embed_backward_workspace(T: int, V: int, d: int) -> int:
    return lib().mnmt_embed_backward_workspace(T, V, d)


def mnmt_embed_backward(ids, T, g, gtype, ldg, scale, pad_id, V, d, gtable, otype, ldt, accumulate, workspace, status=None, stream=None):
    """Gradient of mnmt_embed's table for the gradient g of its output."""
    _chk(lib().mnmt_embed_backward(_ptr(ids), T, _ptr(g), gtype, ldg, scale, pad_id, V, d, _ptr(gtable), otype, ldt, int(accumulate),
                                   _ptr(workspace), _ptr(status), _stream_handle(stream)))


def mnmt_codes_to_f16(src, dst, n, stream=None):
    """dst[i] = fp16(src[i]) for n int8 codes (device buffers)."""
    _chk(lib().mnmt_codes_to_f16(_ptr(src), _ptr(dst), n, _stream_handle(stream)))


def mnmt_wait_timeout_selftest(status, stream=None):
    """Queue one block whose barrier wait runs out (one second): *status -> ETIMEOUT."""
    _chk(lib().mnmt_wait_timeout_selftest(_ptr(status), _stream_handle(stream)))


def argmax_from_keys(keys: np.ndarray) -> np.ndarray:
    """Token ids encoded in mnmt_linear_argmax keys (uint64 viewed as int64 is fine)."""
    k = keys.view(np.uint64)
    return (np.uint64(0xFFFFFFFF) - (k & np.uint64(0xFFFFFFFF))).astype(np.int64)


def mnmt_attention_decode(q, Kc, Vc, n_keys, R, H, dh, T, sigma, rho, ctx, stream=None):
    _chk(lib().mnmt_attention_decode(_ptr(q), _ptr(Kc), _ptr(Vc), _ptr(n_keys), R, H, dh, T, float(sigma),
                                     float(rho), _ptr(ctx), _stream_handle(stream)))


def mnmt_layernorm(r, g, b, M, d, inv, out_f, out_q, status=None, stream=None):
    _chk(lib().mnmt_layernorm(_ptr(r), _ptr(g), _ptr(b), M, d, float(inv), _ptr(out_f), _ptr(out_q),
                              _ptr(status), _stream_handle(stream)))


# --------------------------------------------------------------------------- convenience
class Translator:
    """A loaded model plus one session (owner of both handles)."""

    def __init__(self, blob: bytes, max_batch: int, max_src_len: int, beam: int, max_len: int, stream=None,
                 lean: bool = False):
        """lean=True: memory-minimal model and session (MNMT_LOAD_LEAN, MNMT_SESSION_LEAN)."""
        self.model = mnmt_load_weights(blob, stream, LOAD_LEAN if lean else 0)
        try:
            self.session = mnmt_session_create(self.model, max_batch, max_src_len, beam, max_len,
                                               SESSION_LEAN if lean else 0)
        except Exception:
            mnmt_model_free(self.model)
            raise
        self.cfg = mnmt_model_config(self.model)
        self.beam = beam

    def translate(self, src_ids: np.ndarray, src_lens: np.ndarray, max_len: int):
        """Host arrays in, host arrays out (ids [B][max_len], lens [B], scores [B])."""
        src_ids = np.ascontiguousarray(src_ids, np.int32)
        src_lens = np.ascontiguousarray(src_lens, np.int32)
        B, S = src_ids.shape
        ids = np.zeros((B, max_len), np.int32); lens = np.zeros(B, np.int32); sc = np.zeros(B, np.float32)
        mnmt_translate(self.session, src_ids, src_lens, B, S, max_len, 0, ids, lens, sc)
        return ids, lens, sc

    def close(self):
        if getattr(self, "session", None):
            mnmt_session_free(self.session)
            self.session = None
        if getattr(self, "model", None):
            mnmt_model_free(self.model)
            self.model = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
