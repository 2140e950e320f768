"""ctypes binding of libco3.so: argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libco3.so")

OK, ERR_INVALID_ARG, ERR_CAPACITY, ERR_NO_CODEWORD, ERR_NONFINITE, ERR_CORRUPT, ERR_CUDA = range(7)
MAX_CODE_LEN, CHUNK_SYMS, SUB_SYMS = 16, 2048, 128

FMT_DTYPE = np.dtype([("exp_bits", np.uint8), ("mant_bits", np.uint8), ("flags", np.uint16),
                      ("scale", np.float32), ("inv_scale", np.float32)])
FMT_FLUSH_SUBNORMALS = 1
CODE_DTYPE = np.dtype([("len", np.uint8, (256,)), ("bits", np.uint16, (256,))])
SEG_DTYPE = np.dtype([("elem_off", np.uint64), ("n_elem", np.uint64)])
RESULT_DTYPE = np.dtype([("status", np.int32), ("first_bad_chunk", np.uint32), ("payload_bits", np.uint64),
                         ("container_bytes", np.uint64), ("n_saturated", np.uint64), ("n_nonfinite", np.uint64)])
assert FMT_DTYPE.itemsize == 12 and CODE_DTYPE.itemsize == 768 and SEG_DTYPE.itemsize == 16
assert RESULT_DTYPE.itemsize == 40
MAT_DTYPE = np.dtype([("offset", np.uint64), ("row_stride", np.uint64), ("rows", np.uint32), ("cols", np.uint32),
                      ("scale", np.float32), ("flags", np.uint32)])
MAT_PLAIN = 1
NS_MAX_STEPS = 16
NS_DTYPE = np.dtype([("steps", np.uint32), ("eps", np.float32), ("coef", np.float32, (NS_MAX_STEPS, 3))])
assert MAT_DTYPE.itemsize == 32 and NS_DTYPE.itemsize == 8 + 12 * NS_MAX_STEPS
_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}

_lib = None
_F32 = torch.float32
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


def library_path() -> str:
    return _LIB_PATH


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError("libco3.so is not built (%s): run `python -m paper_2204_08211_b200.build`; "
                           "there is no fallback path" % _LIB_PATH)
    L = C.CDLL(_LIB_PATH)
    vp, u32, u64, sz, f32 = C.c_void_p, C.c_uint32, C.c_uint64, C.c_size_t, C.c_float
    L.co3_status_string.restype = C.c_char_p
    L.co3_status_string.argtypes = [C.c_int]
    L.co3_workspace_bytes.argtypes = [u64, u32, u32, u32, C.POINTER(sz)]
    L.co3_stream_capacity_bytes.argtypes = [u64, u32, u32, C.POINTER(sz)]
    L.co3_convert.argtypes = [vp, vp, f32, vp, vp, u32, u64, u32, u64, vp, vp, vp, vp, sz, vp]
    L.co3_histogram.argtypes = [vp, vp, f32, vp, vp, u32, u64, u32, u64, vp, vp, vp, sz, vp]
    L.co3_convert_dither.argtypes = [vp, vp, f32, vp, vp, u32, u64, u32, u64, u32, vp, vp, vp, vp, sz, vp]
    L.co3_histogram_dither.argtypes = [vp, vp, f32, vp, vp, u32, u64, u32, u64, u32, vp, vp, vp, sz, vp]
    L.co3_encode_dither.argtypes = [vp, vp, f32, vp, vp, vp, u32, u64, u32, u64, u32, vp, sz, u32, vp, sz, vp, vp]
    L.co3_convert_static.argtypes = [vp, vp, f32, vp, vp, u32, u64, u32, u64, vp, vp, vp, vp]
    L.co3_code_build.argtypes = [vp, vp, vp]
    L.co3_code_build_device.argtypes = [vp, vp, u32, vp, vp, vp]
    L.co3_fit_scale.argtypes = [vp, vp, f32, vp, vp, u32, u64, u32, u64, vp, vp, u32, u32, f32, f32, vp, vp, vp, sz, vp]
    L.co3_error_magnitude.argtypes = [vp, vp, vp, u32, u64, u32, u64, vp, vp, vp, sz, vp]
    L.co3_model_weights.argtypes = [vp, vp, u32, vp, vp, vp]
    L.co3_encode.argtypes = [vp, vp, f32, vp, vp, vp, u32, u64, u32, u64, vp, sz, u32, vp, sz, vp, vp]
    L.co3_encode_symbols.argtypes = [vp, vp, vp, u32, u64, u32, u64, vp, sz, u32, vp, sz, vp, vp]
    L.co3_decode_aggregate.argtypes = [vp, sz, u32, vp, vp, vp, u32, u64, u32, vp, vp, sz, vp, vp]
    L.co3_decode_aggregate_update.argtypes = [vp, sz, u32, vp, vp, vp, u32, u64, u32, f32, vp, vp, vp, sz, vp, vp]
    L.co3_decode.argtypes = [vp, sz, vp, vp, vp, u32, u64, u32, vp, vp, vp, sz, vp, vp]
    L.co3_layer_norm.argtypes = [vp, C.c_int, vp, vp, vp, u64, u32, u64, u64, f32, vp, vp, vp]
    L.co3_layer_norm_workspace_bytes.argtypes = [u64, u32, u32, C.POINTER(sz)]
    L.co3_layer_norm_backward.argtypes = [vp, vp, C.c_int, vp, vp, vp, vp, vp, vp, u64, u32, u64, u64, u64, u32, u64,
                                          C.c_int, vp, sz, vp]
    L.co3_ns_default.argtypes = [vp]
    L.co3_orthogonalize_workspace_bytes.argtypes = [vp, u32, C.POINTER(sz)]
    L.co3_orthogonalize.argtypes = [vp, C.c_int, vp, vp, C.c_int, vp, u32, vp, vp, vp, sz, vp]
    L.co3_muon_update.argtypes = [vp, vp, vp, vp, u32, f32, C.c_int, f32, f32, vp, vp, vp, sz, vp]
    L.co3_profile_enable.argtypes = [C.c_int]
    L.co3_profile_read.argtypes = [vp, vp]
    for name in ("co3_layer_norm", "co3_layer_norm_workspace_bytes", "co3_layer_norm_backward", "co3_ns_default", "co3_orthogonalize_workspace_bytes", "co3_orthogonalize", "co3_muon_update", "co3_histogram", "co3_convert_dither", "co3_histogram_dither", "co3_encode_dither", "co3_error_magnitude", "co3_model_weights", "co3_fit_scale", "co3_profile_enable", "co3_profile_read", "co3_convert_static", "co3_workspace_bytes", "co3_stream_capacity_bytes", "co3_convert", "co3_code_build", "co3_code_build_device", "co3_encode",
                 "co3_encode_symbols", "co3_decode_aggregate", "co3_decode_aggregate_update", "co3_decode"):
        getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _dev(t, allow_none: bool = False):
    """Device pointer of a CUDA tensor (or 0 for None)."""
    if t is None:
        if allow_none:
            return None
        raise ValueError("tensor required")
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
        raise ValueError("expected a contiguous CUDA tensor")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


# ------------------------------------------------------------------------------------------------ helpers
def make_fmts(fmts) -> np.ndarray:
    """co3_fmt[n] from (exp_bits, mant_bits, flags, scale, inv_scale) tuples."""
    a = np.zeros(len(fmts), dtype=FMT_DTYPE)
    for k, f in enumerate(fmts):
        a[k] = tuple(f)
    return a


def make_segs(sizes) -> np.ndarray:
    """co3_seg[n] for contiguous segments of the given sizes."""
    a = np.zeros(len(sizes), dtype=SEG_DTYPE)
    off = 0
    for k, n in enumerate(sizes):
        a[k] = (off, int(n))
        off += int(n)
    return a


def make_mats(mats) -> np.ndarray:
    """co3_mat[n] from (offset, rows, cols[, row_stride[, scale[, flags]]]) tuples; row_stride defaults to cols,
    scale to 1, flags to 0."""
    a = np.zeros(len(mats), dtype=MAT_DTYPE)
    for k, m in enumerate(mats):
        offset, rows, cols, row_stride, scale, flags = (*m, *((m[2], 1.0, 0)[len(m) - 3:]))
        a[k] = (offset, row_stride, rows, cols, scale, flags)
    return a


def make_ns(coef=None, steps: int = 5, eps: float = 1e-7) -> np.ndarray:
    """co3_ns: coef is one (a, b, c) for every step or a list with one per step; None: the default coefficients."""
    a = np.zeros(1, dtype=NS_DTYPE)
    c = np.asarray((3.4445, -4.7750, 2.0315) if coef is None else coef, dtype=np.float32)
    n = steps if c.ndim == 1 else len(c)
    a["steps"], a["eps"] = n, eps
    a["coef"][0, :min(n, NS_MAX_STEPS)] = c[:NS_MAX_STEPS] if c.ndim == 2 else c
    return a


def to_device(arr: np.ndarray, device="cuda") -> torch.Tensor:
    """Raw bytes of a (structured) numpy array as a uint8 CUDA tensor (at least 16 bytes)."""
    raw = np.frombuffer(arr.tobytes(), dtype=np.uint8)
    if raw.size < 16:
        raw = np.concatenate([raw, np.zeros(16 - raw.size, dtype=np.uint8)])
    return torch.from_numpy(raw.copy()).to(device)


def read_results(res: torch.Tensor, n: int) -> np.ndarray:
    """co3_result[n] from the device buffer (synchronises)."""
    return np.frombuffer(res.cpu().numpy().tobytes()[:n * RESULT_DTYPE.itemsize], dtype=RESULT_DTYPE).copy()


# ------------------------------------------------------------------------------------------------ entry points
def co3_status_string(status: int) -> str:
    return _load().co3_status_string(int(status)).decode()


def co3_workspace_bytes(n_elem: int, n_seg: int, n_clients: int, chunk_syms: int = CHUNK_SYMS) -> int:
    out = C.c_size_t(0)
    st = _load().co3_workspace_bytes(n_elem, n_seg, n_clients, chunk_syms, C.byref(out))
    if st != OK:
        raise ValueError("co3_workspace_bytes: " + co3_status_string(st))
    return out.value


def co3_stream_capacity_bytes(n_elem: int, n_seg: int, chunk_syms: int = CHUNK_SYMS) -> int:
    out = C.c_size_t(0)
    st = _load().co3_stream_capacity_bytes(n_elem, n_seg, chunk_syms, C.byref(out))
    if st != OK:
        raise ValueError("co3_stream_capacity_bytes: " + co3_status_string(st))
    return out.value


def co3_code_build(weights: np.ndarray, fmt: np.ndarray) -> tuple[int, np.ndarray]:
    """Host call: (status, co3_code as a CODE_DTYPE scalar array of shape (1,))."""
    w = np.ascontiguousarray(weights, dtype=np.uint64)
    f = np.ascontiguousarray(fmt, dtype=FMT_DTYPE).reshape(-1)[:1].copy()
    if w.size != 256:
        raise ValueError("256 weights required")
    out = np.zeros(1, dtype=CODE_DTYPE)
    st = _load().co3_code_build(w.ctypes.data, f.ctypes.data, out.ctypes.data)
    return st, out


def co3_code_build_device(weights, fmts, n_seg, codes_out, res, stream=None) -> int:
    """Device call: weights uint64/int64[n_seg * 256], fmts and codes_out as uploaded descriptor arrays."""
    return _load().co3_code_build_device(_dev(weights), _dev(fmts), n_seg, _dev(codes_out), _dev(res), _stream(stream))


def co3_convert(grad, mem, decay, fmts, segs, n_seg, n_elem, n_clients, client_stride_elems, sym_out, hist_out,
                res, workspace, stream=None) -> int:
    return _load().co3_convert(_dev(grad), _dev(mem), float(decay), _dev(fmts), _dev(segs), n_seg, n_elem,
                               n_clients, client_stride_elems, _dev(sym_out, True), _dev(hist_out, True),
                               _dev(res), _dev(workspace), workspace.numel() * workspace.element_size(),
                               _stream(stream))


def co3_histogram(grad, mem, decay, fmts, segs, n_seg, n_elem, n_clients, client_stride_elems, hist_out, res,
                  workspace, stream=None) -> int:
    """Symbol counts of this round (uint64/int64[n_seg * 256]) without touching the memory or writing symbols."""
    return _load().co3_histogram(_dev(grad), _dev(mem), float(decay), _dev(fmts), _dev(segs), n_seg, n_elem,
                                 n_clients, client_stride_elems, _dev(hist_out), _dev(res), _dev(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream))


def co3_convert_dither(grad, mem, decay, fmts, segs, n_seg, n_elem, n_clients, client_stride_elems, seed, sym_out,
                       hist_out, res, workspace, stream=None) -> int:
    """co3_convert with dithered (stochastic) rounding; `seed` keys the draw stream: another one every round."""
    return _load().co3_convert_dither(_dev(grad), _dev(mem), float(decay), _dev(fmts), _dev(segs), n_seg, n_elem,
                                      n_clients, client_stride_elems, int(seed), _dev(sym_out, True),
                                      _dev(hist_out, True), _dev(res), _dev(workspace),
                                      workspace.numel() * workspace.element_size(), _stream(stream))


def co3_histogram_dither(grad, mem, decay, fmts, segs, n_seg, n_elem, n_clients, client_stride_elems, seed, hist_out,
                         res, workspace, stream=None) -> int:
    """co3_histogram for a round that will be converted with dithered rounding under the same seed."""
    return _load().co3_histogram_dither(_dev(grad), _dev(mem), float(decay), _dev(fmts), _dev(segs), n_seg, n_elem,
                                        n_clients, client_stride_elems, int(seed), _dev(hist_out), _dev(res),
                                        _dev(workspace), workspace.numel() * workspace.element_size(),
                                        _stream(stream))


def co3_encode_dither(grad, mem, decay, fmts, codes, segs, n_seg, n_elem, n_clients, client_stride_elems, seed,
                      streams_out, stream_capacity, workspace, res, chunk_syms: int = CHUNK_SYMS, stream=None) -> int:
    """co3_encode with dithered (stochastic) rounding."""
    return _load().co3_encode_dither(_dev(grad), _dev(mem), float(decay), _dev(fmts), _dev(codes), _dev(segs), n_seg,
                                     n_elem, n_clients, client_stride_elems, int(seed), _dev(streams_out),
                                     stream_capacity, chunk_syms, _dev(workspace),
                                     workspace.numel() * workspace.element_size(), _dev(res), _stream(stream))


STATIC_SCRATCH_BYTES = 2 << 20


def co3_convert_static(grad, mem, decay, fmts, segs, n_seg, n_elem, n_clients, client_stride_elems, sym_out, hist_out,
                       res, stream=None) -> int:
    """co3_convert on the library's built-in scratch array: no workspace tensor, nothing is allocated.
    For hosts that may not allocate device memory where they call this; layouts needing more than
    STATIC_SCRATCH_BYTES of workspace return ERR_CAPACITY.  Calls on one device share the array: order them."""
    return _load().co3_convert_static(_dev(grad), _dev(mem), float(decay), _dev(fmts), _dev(segs), n_seg, n_elem,
                                      n_clients, client_stride_elems, _dev(sym_out, True), _dev(hist_out, True),
                                      _dev(res), _stream(stream))


def co3_fit_scale(grad, mem, decay, fmts, segs, n_seg, n_elem, n_clients, client_stride_elems, log_tab, seg_tab,
                  n_tab, n_beta, beta0, dbeta, stats_out, res, workspace, stream=None) -> int:
    """Writes scale / inv_scale of every layer's co3_fmt on the device; mem, seg_tab, stats_out may be None."""
    return _load().co3_fit_scale(_dev(grad), _dev(mem, True), float(decay), _dev(fmts), _dev(segs), n_seg, n_elem,
                                 n_clients, client_stride_elems, _dev(log_tab), _dev(seg_tab, True), n_tab, n_beta,
                                 float(beta0), float(dbeta), _dev(stats_out, True), _dev(res), _dev(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream))


def co3_error_magnitude(grad, mem, segs, n_seg, n_elem, n_clients, client_stride_elems, norms_out, res, workspace,
                        stream=None) -> int:
    """norms_out float64[n_clients * n_seg * 2]: l1 norms of gradient and memory per client and layer."""
    return _load().co3_error_magnitude(_dev(grad), _dev(mem), _dev(segs), n_seg, n_elem, n_clients, client_stride_elems,
                                       _dev(norms_out), _dev(res), _dev(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream))


def co3_model_weights(fmts, stats, n_seg, weights_out, res, stream=None) -> int:
    """weights_out int64/uint64[n_seg * 256] from the formats and the (beta, alpha) columns of co3_fit_scale's stats."""
    return _load().co3_model_weights(_dev(fmts), _dev(stats), n_seg, _dev(weights_out), _dev(res), _stream(stream))


def co3_encode(grad, mem, decay, fmts, codes, segs, n_seg, n_elem, n_clients, client_stride_elems, streams_out,
               stream_capacity, workspace, res, chunk_syms: int = CHUNK_SYMS, stream=None) -> int:
    return _load().co3_encode(_dev(grad), _dev(mem), float(decay), _dev(fmts), _dev(codes), _dev(segs), n_seg,
                              n_elem, n_clients, client_stride_elems, _dev(streams_out), stream_capacity, chunk_syms,
                              _dev(workspace), workspace.numel() * workspace.element_size(), _dev(res),
                              _stream(stream))


def co3_encode_symbols(sym, codes, segs, n_seg, n_elem, n_clients, client_stride_elems, streams_out,
                       stream_capacity, workspace, res, chunk_syms: int = CHUNK_SYMS, stream=None) -> int:
    return _load().co3_encode_symbols(_dev(sym), _dev(codes), _dev(segs), n_seg, n_elem, n_clients,
                                      client_stride_elems, _dev(streams_out), stream_capacity, chunk_syms,
                                      _dev(workspace), workspace.numel() * workspace.element_size(), _dev(res),
                                      _stream(stream))


def co3_decode_aggregate(stream_ptrs, stream_bytes, n_clients, fmts, codes, segs, n_seg, n_elem, avg_out, workspace,
                         res, chunk_syms: int = CHUNK_SYMS, stream=None) -> int:
    """stream_ptrs: int64 CUDA tensor holding the n_clients device addresses of the streams."""
    return _load().co3_decode_aggregate(_dev(stream_ptrs), stream_bytes, n_clients, _dev(fmts), _dev(codes),
                                        _dev(segs), n_seg, n_elem, chunk_syms, _dev(avg_out), _dev(workspace),
                                        workspace.numel() * workspace.element_size(), _dev(res), _stream(stream))


def co3_decode_aggregate_update(stream_ptrs, stream_bytes, n_clients, fmts, codes, segs, n_seg, n_elem, lr, params,
                                avg_out, workspace, res, chunk_syms: int = CHUNK_SYMS, stream=None) -> int:
    """co3_decode_aggregate with params <- params - lr * avg folded in; avg_out may be None."""
    return _load().co3_decode_aggregate_update(_dev(stream_ptrs), stream_bytes, n_clients, _dev(fmts), _dev(codes),
                                               _dev(segs), n_seg, n_elem, chunk_syms, float(lr), _dev(params),
                                               _dev(avg_out, True), _dev(workspace),
                                               workspace.numel() * workspace.element_size(), _dev(res), _stream(stream))


def co3_decode(stream_in, stream_bytes, fmts, codes, segs, n_seg, n_elem, ghat_out, sym_out, workspace, res,
               chunk_syms: int = CHUNK_SYMS, stream=None) -> int:
    return _load().co3_decode(_dev(stream_in), stream_bytes, _dev(fmts), _dev(codes), _dev(segs), n_seg, n_elem,
                              chunk_syms, _dev(ghat_out, True), _dev(sym_out, True), _dev(workspace),
                              workspace.numel() * workspace.element_size(), _dev(res), _stream(stream))


def _rows(t, like=None):
    """(pointer, rows, cols, row stride) of a 2-D CUDA tensor whose rows are contiguous, of the shape and type of `like`."""
    shape = t.shape
    if like is None:
        if not t.is_cuda or len(shape) != 2 or t.dtype not in _TYPES:
            raise ValueError("expected a 2-D CUDA tensor of fp32, fp16 or bf16")
    elif shape != like.shape or t.dtype is not like.dtype or not t.is_cuda:
        raise ValueError("expected tensors of one shape and type")
    rows, cols = shape
    rs, cs = t.stride()
    if (cs != 1 and cols > 1) or (rs < cols and rows > 1):
        raise ValueError("expected contiguous rows that do not overlap")
    return t.data_ptr(), rows, cols, rs if rows > 1 or rs > cols else cols


def _stream_of(t, stream):
    """The current stream of t's device unless one is given (the short way: these calls can be microseconds long)."""
    return _current_stream(t.get_device()) if stream is None else _stream(stream)


def _vec(t, n):
    """Device pointer of n fp32 values (or None)."""
    if t is None:
        return None
    if t.dtype is not _F32 or not t.is_cuda or t.numel() < n or not t.is_contiguous():
        raise ValueError("expected a contiguous fp32 CUDA tensor of at least %d elements" % n)
    return t.data_ptr()


def co3_layer_norm(x, weight, bias, y, mean=None, rstd=None, eps=1e-5, stream=None) -> int:
    """y <- layer norm of the rows of x; weight, bias (fp32) and the statistics mean, rstd (fp32, out) may be None."""
    px, rows, cols, xs = _rows(x)
    py, _, _, ys = _rows(y, x)
    return (_lib or _load()).co3_layer_norm(px, _TYPES[x.dtype], _vec(weight, cols), _vec(bias, cols), py, rows, cols, xs,
                                            ys, eps, _vec(mean, rows), _vec(rstd, rows), _stream_of(x, stream))


def co3_layer_norm_workspace_bytes(rows: int, cols: int, n_clients: int = 1) -> int:
    """Device workspace of co3_layer_norm_backward for n_clients batches of `rows` rows each."""
    out = C.c_size_t(0)
    st = _load().co3_layer_norm_workspace_bytes(rows, cols, n_clients, C.byref(out))
    if st != OK:
        raise ValueError("co3_layer_norm_workspace_bytes: " + co3_status_string(st))
    return out.value


def co3_layer_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, n_clients, client_stride_elems, workspace,
                            accumulate: bool = False, stream=None) -> int:
    """Gradients of co3_layer_norm; the rows are n_clients equal batches.  dweight and dbias are fp32 tensors that start
    at client 0's gradient of that layer (a slice of the clients' gradient buffer); dx, dweight, dbias may be None."""
    pd, rows, cols, ds = _rows(dy)
    px, _, _, xs = _rows(x, dy)
    po, _, _, os_ = (None, 0, 0, 0) if dx is None else _rows(dx, dy)
    if n_clients < 1 or rows % n_clients:
        raise ValueError("co3_layer_norm_backward: the rows do not divide into n_clients batches")
    if client_stride_elems < 0:  # the library takes it as unsigned
        raise ValueError("co3_layer_norm_backward: clients' vectors that lie backwards")
    reach = (n_clients - 1) * client_stride_elems + cols
    return (_lib or _load()).co3_layer_norm_backward(
        pd, px, _TYPES[dy.dtype], _vec(weight, cols), _vec(mean, rows), _vec(rstd, rows), po, _vec(dweight, reach),
        _vec(dbias, reach), rows // n_clients, cols, ds, xs, os_, n_clients, client_stride_elems, 1 if accumulate else 0,
        _dev(workspace), workspace.numel() * workspace.element_size(), _stream_of(dy, stream))


def _mats(mats):
    if not (isinstance(mats, np.ndarray) and mats.dtype == MAT_DTYPE and mats.flags.c_contiguous):
        raise ValueError("expected the array make_mats returns")
    return mats.ctypes.data, mats.size


def _ns(ns):
    if ns is None:
        return None
    if not (isinstance(ns, np.ndarray) and ns.dtype == NS_DTYPE and ns.size == 1):
        raise ValueError("expected the array make_ns returns")
    return ns.ctypes.data


def _fits(mats, tensors, what) -> None:
    """The library cannot see a buffer's length: every listed matrix has to end inside the tensors."""
    room = min(t.numel() for t in tensors)
    rows, cols, offset, stride = (mats[f].astype(np.float64) for f in ("rows", "cols", "offset", "row_stride"))
    ends = np.where((rows > 0) & (cols > 0), offset + (rows - 1) * stride + cols, 0.0)
    worst = ends.max(initial=0.0)
    if worst > room:  # (a double counts exactly up to far beyond any memory)
        raise ValueError("%s: a matrix ends beyond the tensor" % what)


def co3_orthogonalize_workspace_bytes(mats: np.ndarray) -> int:
    """Device workspace of co3_orthogonalize / co3_muon_update for these matrices (as make_mats returns them)."""
    out = C.c_size_t(0)
    p, n = _mats(mats)
    st = _load().co3_orthogonalize_workspace_bytes(p, n, C.byref(out))
    if st != OK:
        raise ValueError("co3_orthogonalize_workspace_bytes: " + co3_status_string(st))
    return out.value


def co3_orthogonalize(inp, in_mats, out, out_mats, workspace, res, ns=None, stream=None) -> int:
    """out <- scale * orthogonalised inp for every listed matrix; contiguous fp32, fp16 or bf16 tensors of any shape
    whose elements the layouts index (out_mats None: as in_mats)."""
    p, n = _mats(in_mats)
    q, nq = (None, n) if out_mats is None or out_mats is in_mats else _mats(out_mats)
    if nq != n or inp.dtype not in _TYPES or out.dtype not in _TYPES:
        raise ValueError("co3_orthogonalize: fp32, fp16 or bf16 tensors and as many layouts for out as for in")
    if q is None:
        _fits(in_mats, (inp, out), "co3_orthogonalize")
    else:
        _fits(in_mats, (inp,), "co3_orthogonalize")
        _fits(out_mats, (out,), "co3_orthogonalize")
    return _load().co3_orthogonalize(_dev(inp), _TYPES[inp.dtype], p, _dev(out), _TYPES[out.dtype], q, n, _ns(ns),
                                     _dev(res), _dev(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(stream))


def co3_muon_update(grad, momentum, params, mats, mu, nesterov, lr, weight_decay, workspace, res, ns=None,
                    stream=None) -> int:
    """One server step on fp32 vectors: momentum, orthogonalisation of the matrices, weight decay and parameters."""
    p, n = _mats(mats)
    for t in (grad, momentum, params):
        if t.dtype != torch.float32:
            raise ValueError("co3_muon_update: fp32 tensors")
    _fits(mats, (grad, momentum, params), "co3_muon_update")
    return _load().co3_muon_update(_dev(grad), _dev(momentum), _dev(params), p, n, float(mu), 1 if nesterov else 0,
                                   float(lr), float(weight_decay), _ns(ns), _dev(res), _dev(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream))


KERNEL_NAMES = ("prepare", "convert", "pack", "scan", "compact", "code_build", "decode", "fit", "clear")


def co3_profile_enable(on: bool) -> int:
    return _load().co3_profile_enable(1 if on else 0)


def co3_profile_read() -> dict:
    """{kernel name: (launches, total ms)} since profiling was enabled or last read (synchronises)."""
    ms = np.zeros(len(KERNEL_NAMES), dtype=np.float64)
    n = np.zeros(len(KERNEL_NAMES), dtype=np.uint32)
    st = _load().co3_profile_read(ms.ctypes.data, n.ctypes.data)
    if st != OK:
        raise RuntimeError("co3_profile_read: " + co3_status_string(st))
    return {k: (int(n[i]), float(ms[i])) for i, k in enumerate(KERNEL_NAMES)}
