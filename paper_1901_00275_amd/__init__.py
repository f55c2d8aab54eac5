"""Python binding of libvlq (VLQ-ADC index for MI355X, HIP/gfx950).

Argument marshalling only: every function has the name and the argument order
of its C entry point in ``include/vlq.h`` and hands device pointers of torch
tensors to it; all computation happens in the HIP kernels of the library.
torch is used for device memory and streams.  There is no CPU fallback: a
missing library raises at the first call.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvlq.so")

VLQ_OK, VLQ_EINVAL, VLQ_ENOMEM, VLQ_EHIP = 0, -1, -2, -3
STAGES = ("coarse", "select_cells", "subregions", "scan", "merge")
(VLQ_OPT_COARSE_FP32, VLQ_OPT_NEIGHBOURS_PER_QUERY, VLQ_OPT_SCAN_PACKED, VLQ_OPT_SCAN_GENERIC,
 VLQ_OPT_ENCODE_WAVE, VLQ_OPT_PIPELINE_PARTS, VLQ_OPT_SMALL_BATCH, VLQ_OPT_COARSE_SPLIT) = range(8)
VLQ_F32, VLQ_F16, VLQ_BF16 = range(3)
_TYPES = {torch.float32: VLQ_F32, torch.float16: VLQ_F16, torch.bfloat16: VLQ_BF16}


class VlqError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libvlq error {code}: {msg}")
        self.code = code


class vlq_params_t(C.Structure):
    _fields_ = [("d", C.c_int32), ("nlist", C.c_int32), ("n_edges", C.c_int32), ("m", C.c_int32),
                ("lambda_lo", C.c_float), ("lambda_hi", C.c_float)]


_lib = None
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def lib():
    """The loaded shared library (built in-tree by ``build.py``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -m paper_1901_00275_amd.build` "
                                    "(or __graft_entry__.build()) first; there is no fallback path")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        sig = {
            "vlq_build_index": [C.POINTER(vlq_params_t), vp, vp, vp, i64, vp, vp, C.POINTER(vp)],
            "vlq_encode": [vp, vp, i64, vp, vp, vp, vp, vp],
            "vlq_line_residuals": [vp, vp, i64, vp, vp],
            "vlq_kmeans": [vp, i64, i32, i32, i32, vp, vp, vp, vp],
            "vlq_index_add": [vp, vp, i64, vp, vp],
            "vlq_index_add_encoded": [vp, vp, vp, vp, vp, vp, i64, vp],
            "vlq_index_reserve": [vp, i64],
            "vlq_index_finalize": [vp, vp],
            "vlq_index_is_finalized": [vp],
            "vlq_index_params": [vp, C.POINTER(vlq_params_t)],
            "vlq_index_set_option": [vp, C.c_int, C.c_int],
            "vlq_index_set_query_lambda_range": [vp, C.c_float, C.c_float],
            "vlq_search": [vp, vp, i32, i32, i32, i32, vp, vp, vp],
            "vlq_search_noalloc": [vp, vp, i32, i32, i32, i32, vp, vp, vp],
            "vlq_search_debug": [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp],
            "vlq_index_get_graph": [vp, vp, vp, vp],
            "vlq_index_get_lists": [vp, vp, vp, vp, vp, vp],
            "vlq_profile_enable": [vp, C.c_int],
            "vlq_profile_read": [vp, C.POINTER(C.c_float), C.POINTER(i32)],
            "vlq_softmax_loss": [C.c_int, vp, i64, i32, vp, i32, vp, C.c_float, vp, vp, vp, vp, i64, vp],
            "vlq_softmax_loss_backward": [C.c_int, vp, i64, i32, vp, i32, vp, C.c_float, vp, vp, vp, vp, vp, vp, vp, i64, vp],
            "vlq_group_rows": [vp, i64, i32, i32, vp, vp, vp, vp, i64, vp],
            "vlq_gather_rows": [C.c_int, vp, i64, i32, i32, vp, vp, vp],
            "vlq_combine_rows": [C.c_int, vp, i64, i32, i32, vp, vp, vp, vp],
            "vlq_combine_rows_backward": [C.c_int, vp, vp, i64, i32, i32, vp, vp, vp, vp, vp],
            "vlq_clip_grads": [i32, vp, vp, vp, C.c_float, vp, vp, vp, i64, vp],
            "vlq_version": [],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = C.c_int
        L.vlq_index_free.argtypes = [vp]
        L.vlq_index_free.restype = None
        L.vlq_index_ntotal.argtypes = [vp]
        L.vlq_index_ntotal.restype = i64
        L.vlq_softmax_loss_workspace.argtypes = [C.c_int, i64, i32, i32, C.c_int]
        L.vlq_softmax_loss_workspace.restype = i64
        L.vlq_group_rows_workspace.argtypes = [i64, i32, i32]
        L.vlq_group_rows_workspace.restype = i64
        L.vlq_clip_grads_workspace.argtypes = [i32, vp]
        L.vlq_clip_grads_workspace.restype = i64
        L.vlq_last_error.argtypes = []
        L.vlq_last_error.restype = C.c_char_p
        _lib = L
    return _lib


def _chk(rc):
    if rc != 0:
        raise VlqError(rc, lib().vlq_last_error().decode())


def _ptr(t, dtype=None):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors passed to libvlq must be contiguous device tensors")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None and _raw_stream is not None:  # (the stream's handle without an object for it: 0.2 instead of 2.8 us)
        return C.c_void_p(_raw_stream(torch.cuda.current_device()))
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def vlq_version() -> int:
    return lib().vlq_version()


def vlq_last_error() -> str:
    return lib().vlq_last_error().decode()


def vlq_build_index(params: vlq_params_t, d_centroids, d_pq, d_base=None, N=0, d_ids=None, stream=None):
    """Returns the opaque index handle (free it with vlq_index_free)."""
    out = C.c_void_p()
    _chk(lib().vlq_build_index(C.byref(params), _ptr(d_centroids, torch.float32), _ptr(d_pq, torch.float32),
                               _ptr(d_base, torch.float32), int(N), _ptr(d_ids, torch.int32), _stream(stream),
                               C.byref(out)))
    return out


def vlq_index_free(idx):
    lib().vlq_index_free(idx)


def vlq_encode(idx, d_x, nb, d_cell, d_edge, d_lambda, d_codes, stream=None):
    _chk(lib().vlq_encode(idx, _ptr(d_x, torch.float32), int(nb), _ptr(d_cell, torch.int32), _ptr(d_edge, torch.int32),
                          _ptr(d_lambda, torch.uint8), _ptr(d_codes, torch.uint8), _stream(stream)))


def vlq_line_residuals(idx, d_x, nb, d_res, stream=None):
    _chk(lib().vlq_line_residuals(idx, _ptr(d_x, torch.float32), int(nb), _ptr(d_res, torch.float32), _stream(stream)))


def vlq_kmeans(d_x, nt, d, k, iters, d_centroids, d_assign=None, d_counts=None, stream=None):
    _chk(lib().vlq_kmeans(_ptr(d_x, torch.float32), int(nt), int(d), int(k), int(iters), _ptr(d_centroids, torch.float32),
                          _ptr(d_assign, torch.int32), _ptr(d_counts, torch.int32), _stream(stream)))


def vlq_index_add(idx, d_x, nb, d_ids=None, stream=None):
    _chk(lib().vlq_index_add(idx, _ptr(d_x, torch.float32), int(nb), _ptr(d_ids, torch.int32), _stream(stream)))


def vlq_index_add_encoded(idx, d_cell, d_edge, d_lambda, d_codes, d_ids, nb, stream=None):
    _chk(lib().vlq_index_add_encoded(idx, _ptr(d_cell, torch.int32), _ptr(d_edge, torch.int32),
                                     _ptr(d_lambda, torch.uint8), _ptr(d_codes, torch.uint8),
                                     _ptr(d_ids, torch.int32), int(nb), _stream(stream)))


def vlq_index_reserve(idx, total):
    _chk(lib().vlq_index_reserve(idx, int(total)))


def vlq_index_finalize(idx, stream=None):
    _chk(lib().vlq_index_finalize(idx, _stream(stream)))


def vlq_index_ntotal(idx) -> int:
    return int(lib().vlq_index_ntotal(idx))


def vlq_index_is_finalized(idx) -> bool:
    return bool(lib().vlq_index_is_finalized(idx))


def vlq_index_params(idx) -> vlq_params_t:
    p = vlq_params_t()
    _chk(lib().vlq_index_params(idx, C.byref(p)))
    return p


def vlq_index_set_option(idx, option, value):
    _chk(lib().vlq_index_set_option(idx, int(option), int(value)))


def vlq_index_set_query_lambda_range(idx, lo, hi):
    _chk(lib().vlq_index_set_query_lambda_range(idx, float(lo), float(hi)))


def vlq_search(idx, d_q, nq, w1, w2, K, d_out_dist, d_out_ids, stream=None):
    _chk(lib().vlq_search(idx, _ptr(d_q, torch.float32), int(nq), int(w1), int(w2), int(K),
                          _ptr(d_out_dist, torch.float32), _ptr(d_out_ids, torch.int32), _stream(stream)))


def vlq_search_noalloc(idx, d_q, nq, w1, w2, K, d_out_dist, d_out_ids, stream=None):
    _chk(lib().vlq_search_noalloc(idx, _ptr(d_q, torch.float32), int(nq), int(w1), int(w2), int(K),
                                  _ptr(d_out_dist, torch.float32), _ptr(d_out_ids, torch.int32), _stream(stream)))


def vlq_search_debug(idx, d_q, nq, w1, w2, K, d_out_dist, d_out_ids, d_cells=None, d_cell_dist=None, d_sub=None,
                     d_sub_score=None, stream=None):
    _chk(lib().vlq_search_debug(idx, _ptr(d_q, torch.float32), int(nq), int(w1), int(w2), int(K),
                                _ptr(d_out_dist, torch.float32), _ptr(d_out_ids, torch.int32),
                                _ptr(d_cells, torch.int32), _ptr(d_cell_dist, torch.float32),
                                _ptr(d_sub, torch.int32), _ptr(d_sub_score, torch.float32), _stream(stream)))


def vlq_index_get_graph(idx, d_S, d_E, stream=None):
    _chk(lib().vlq_index_get_graph(idx, _ptr(d_S, torch.int32), _ptr(d_E, torch.float32), _stream(stream)))


def vlq_index_get_lists(idx, d_off, d_ids, d_codes, d_lambda, stream=None):
    _chk(lib().vlq_index_get_lists(idx, _ptr(d_off, torch.int64), _ptr(d_ids, torch.int32), _ptr(d_codes, torch.uint8),
                                   _ptr(d_lambda, torch.uint8), _stream(stream)))


def vlq_profile_enable(idx, enable: bool):
    _chk(lib().vlq_profile_enable(idx, int(bool(enable))))


def vlq_profile_read(idx):
    """{stage: (milliseconds, launches)} since the last read."""
    ms = (C.c_float * len(STAGES))()
    ln = (C.c_int32 * len(STAGES))()
    _chk(lib().vlq_profile_read(idx, ms, ln))
    return {s: (float(ms[i]), int(ln[i])) for i, s in enumerate(STAGES)}


# ---------------------------------------------------------------------------
# learning cells by gradient: the value type follows from the tensors, the workspace is a uint8 tensor
# ---------------------------------------------------------------------------
def _type(t):
    dtype = t.dtype if isinstance(t, torch.Tensor) else t
    if dtype not in _TYPES:
        raise ValueError(f"expected float32, float16 or bfloat16, got {dtype}")
    return _TYPES[dtype]


def _ptrs(*pairs):
    """Addresses of (tensor or None, dtype, least number of values), all of them on the current device."""
    out, dev = [], None
    for t, dtype, count in pairs:
        if t is None:
            out.append(None)
            continue
        if dev is None and t.is_cuda:
            dev = torch.cuda.current_device()
        if t.get_device() != dev or not t.is_contiguous() or t.numel() < count or not (dtype is None or t.dtype is dtype):
            if not t.is_cuda or not t.is_contiguous():
                raise ValueError("tensors passed to libvlq must be contiguous device tensors")
            if t.get_device() != dev:
                raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{dev}")
            if t.numel() < count:
                raise ValueError(f"a tensor has {t.numel()} values, {count} are needed")
            raise ValueError(f"expected {dtype}, got {t.dtype}")
        out.append(t.data_ptr())
    return out


def _bytes(n):
    if n < 0:
        _chk(int(n))
    return int(n)


def vlq_softmax_loss_workspace(dtype, n, d, k, backward) -> int:
    return _bytes(lib().vlq_softmax_loss_workspace(_type(dtype), int(n), int(d), int(k), int(bool(backward))))


def vlq_softmax_loss(d_x, n, d, d_c, k, d_bias, scale, d_label, d_loss, d_stats, d_ws, stream=None):
    n, d, k = int(n), int(d), int(k)
    x, c, bias, label, loss, stats, ws = _ptrs(
        (d_x, d_c.dtype, n * d), (d_c, None, k * d), (d_bias, torch.float32, k), (d_label, torch.int32, n), (d_loss, torch.float32, n),
        (d_stats, torch.float32, 2 * n), (d_ws, torch.uint8, 0))
    _chk(lib().vlq_softmax_loss(_type(d_c), x, n, d, c, k, bias, float(scale), label, loss, stats, ws, d_ws.numel(), _stream(stream)))


def vlq_softmax_loss_backward(d_x, n, d, d_c, k, d_bias, scale, d_label, d_stats, d_grad, d_dx, d_dc, d_dbias, d_ws, stream=None):
    n, d, k = int(n), int(d), int(k)
    x, c, bias, label, stats, grad, dx, dc, dbias, ws = _ptrs(
        (d_x, d_c.dtype, n * d), (d_c, None, k * d), (d_bias, torch.float32, k), (d_label, torch.int32, n),
        (d_stats, torch.float32, 2 * n), (d_grad, torch.float32, n), (d_dx, d_c.dtype, n * d), (d_dc, d_c.dtype, k * d),
        (d_dbias, torch.float32, k), (d_ws, torch.uint8, 0))
    _chk(lib().vlq_softmax_loss_backward(_type(d_c), x, n, d, c, k, bias, float(scale), label, stats, grad, dx, dc, dbias, ws,
                                         d_ws.numel(), _stream(stream)))


def vlq_group_rows_workspace(n, w, cells) -> int:
    return _bytes(lib().vlq_group_rows_workspace(int(n), int(w), int(cells)))


def vlq_group_rows(d_cell, n, w, cells, d_off, d_place, d_source, d_ws, stream=None):
    n, w, cells = int(n), int(w), int(cells)
    cell, off, place, source, ws = _ptrs((d_cell, torch.int32, n * w), (d_off, torch.int64, cells + 1), (d_place, torch.int32, n * w),
                                         (d_source, torch.int32, n * w), (d_ws, torch.uint8, 0))
    _chk(lib().vlq_group_rows(cell, n, w, cells, off, place, source, ws, d_ws.numel(), _stream(stream)))


def vlq_gather_rows(d_x, n, w, d, d_source, d_y, stream=None):
    n, w, d = int(n), int(w), int(d)
    x, source, y = _ptrs((d_x, None, n * d), (d_source, torch.int32, n * w), (d_y, d_x.dtype, n * w * d))
    _chk(lib().vlq_gather_rows(_type(d_x), x, n, w, d, source, y, _stream(stream)))


def vlq_combine_rows(d_y, n, w, d, d_place, d_weight, d_out, stream=None):
    n, w, d = int(n), int(w), int(d)
    y, place, weight, out = _ptrs((d_y, None, n * w * d), (d_place, torch.int32, n * w), (d_weight, torch.float32, n * w),
                                  (d_out, d_y.dtype, n * d))
    _chk(lib().vlq_combine_rows(_type(d_y), y, n, w, d, place, weight, out, _stream(stream)))


def vlq_combine_rows_backward(d_dout, d_y, n, w, d, d_place, d_weight, d_dy, d_dweight, stream=None):
    n, w, d = int(n), int(w), int(d)
    dout, y, place, weight, dy, dweight = _ptrs(
        (d_dout, None, n * d), (d_y, d_dout.dtype, n * w * d), (d_place, torch.int32, n * w), (d_weight, torch.float32, n * w),
        (d_dy, d_dout.dtype, n * w * d), (d_dweight, torch.float32, n * w))
    _chk(lib().vlq_combine_rows_backward(_type(d_dout), dout, y, n, w, d, place, weight, dy, dweight, _stream(stream)))


def vlq_clip_grads_workspace(grads) -> int:
    counts = array("q", [g.numel() for g in grads])
    return _bytes(lib().vlq_clip_grads_workspace(len(grads), counts.buffer_info()[0]))


def vlq_clip_grads(d_grads, max_norm, d_out, d_norm, d_ws, stream=None):
    """d_grads: a list of tensors; d_out: a list as long (its tensors may be those of d_grads), or None for the norm alone."""
    norm, ws = _ptrs((d_norm, torch.float32, 1), (d_ws, torch.uint8, 0))
    dev = d_ws.get_device()
    counts = array("q", [g.numel() for g in d_grads])
    types = array("i", [_TYPES.get(g.dtype, -1) for g in d_grads])
    if -1 in types or any(g.get_device() != dev or not g.is_contiguous() for g in d_grads):
        raise ValueError("gradients must be contiguous float32, float16 or bfloat16 tensors on the current device")
    ptrs, outs = array("Q", [g.data_ptr() for g in d_grads]), None
    if d_out is not None:
        if len(d_out) != len(d_grads):
            raise ValueError("d_out must have a tensor for every tensor of d_grads")
        if d_out is not d_grads:
            for g, o, count in zip(d_grads, d_out, counts):
                if o is not g and (o.dtype is not g.dtype or o.get_device() != dev or not o.is_contiguous() or o.numel() != count):
                    raise ValueError("d_out must have a contiguous tensor of the same type, size and device for every tensor of d_grads")
        outs = array("Q", [o.data_ptr() for o in d_out])
    _chk(lib().vlq_clip_grads(len(d_grads), types.buffer_info()[0], counts.buffer_info()[0], ptrs.buffer_info()[0], float(max_norm),
                              None if outs is None else outs.buffer_info()[0], norm, ws, d_ws.numel(), _stream(stream)))
