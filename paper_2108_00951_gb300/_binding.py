"""ctypes binding of libefsparse.so — argument marshalling only.

Every function here has the name of the C entry point it calls (declared in
``include/efsparse.h``), takes torch CUDA tensors, checks their dtype, device,
shape and contiguity, and passes raw device pointers and the current CUDA
stream across the C ABI. All computation happens in the library's kernels;
there is no fallback: if the library cannot be loaded, every call raises.
"""
from __future__ import annotations

import array
import ctypes
import os
import threading

import numpy as np
import torch

from . import build as _build

EF_OK = 0
EF_ERR_INVALID_ARG = 1
EF_ERR_CUDA = 2
EF_ERR_TIMEOUT = 3
EF_ERR_BAD_INPUT = 4
EF_ERR_NO_MEMORY = 5


class EfError(RuntimeError):
    """A non-OK ef_status returned by the library."""

    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s" % (where, status_string(status)))


_lock = threading.Lock()
_lib = None


def library_path() -> str:
    return _build.LIBPATH


def load_library(build_if_missing: bool = True):
    """Load libefsparse.so (building it in-tree first if it is missing)."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        path = _build.LIBPATH
        if not os.path.exists(path) or not _build.up_to_date():
            if not build_if_missing:
                raise RuntimeError("libefsparse.so is not built: run __graft_entry__.build()")
            _build.build()
        lib = ctypes.CDLL(path)
        vp, u64, f32, u32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_float, ctypes.c_uint32
        f64 = ctypes.c_double
        sig = {
            "ef_hard_threshold": [vp, vp, f32, f32, u64, vp, vp, vp, vp],
            "ef_hard_threshold_bf16": [vp, vp, f32, f32, u64, vp, vp, vp, vp],
            "ef_topk": [vp, vp, f32, u64, u64, vp, vp, vp, vp],
            "ef_topk_bf16": [vp, vp, f32, u64, u64, vp, vp, vp, vp],
            "ef_topk_layerwise": [vp, vp, f32, u32, vp, vp, u64, vp, vp, vp, vp],
            "ef_topk_layerwise_bf16": [vp, vp, f32, u32, vp, vp, u64, vp, vp, vp, vp],
            "ef_hard_threshold_ex": [vp, ctypes.c_int, vp, f32, f32, u64, vp, vp, vp, vp, vp],
            "ef_topk_ex": [vp, ctypes.c_int, vp, f32, u64, u64, vp, vp, vp, vp, vp],
            "ef_topk_layerwise_ex": [vp, ctypes.c_int, vp, f32, u32, vp, vp, u64, vp, vp, vp, vp,
                                     vp],
            "ef_scaled_round_ex": [vp, ctypes.c_int, vp, f32, ctypes.c_int32, u64, vp, vp, vp,
                                   vp],
            "int_aggregate": [u32, ctypes.POINTER(vp), u64, ctypes.c_int32, vp, vp],
            "sparse_aggregate": [u32, ctypes.POINTER(vp), ctypes.POINTER(vp), vp, u64, vp, vp],
            "sparse_aggregate_apply": [u32, ctypes.POINTER(vp), ctypes.POINTER(vp), vp, u64, f32,
                                       vp, vp, f32, f32, vp],
            "ef_hard_threshold_tiled": [vp, ctypes.c_int, vp, f32, f32, u64, vp, vp, vp, vp, vp,
                                        vp],
            "sparse_aggregate_tiled": [u32, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                       ctypes.POINTER(vp), vp, u64, vp, vp],
            "sparse_aggregate_apply_tiled": [u32, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                             ctypes.POINTER(vp), vp, u64, f32, vp, vp, f32, f32,
                                             vp],
            "ef_vocab_loss": [vp, u64, vp, u64, vp, vp, u64, u64, u64, vp, vp, vp],
            "ef_vocab_loss_grad": [vp, u64, vp, u64, vp, vp, vp, vp, u64, u64, u64, vp, u64, vp,
                                   u64, vp, vp],
            "ef_orthogonalize": [u32, vp, vp, vp, vp, ctypes.c_int, vp, vp, f32, vp, vp, vp],
            "ef_embed": [vp, u64, ctypes.c_int, vp, u64, u64, u64, f32, vp, u64, ctypes.c_int, vp],
            "ef_embed_grad": [vp, u64, ctypes.c_int, vp, u64, u64, u64, f32, ctypes.c_int, vp, u64,
                              ctypes.c_int, vp],
            "ef_layer_norm": [vp, u64, ctypes.c_int, vp, vp, ctypes.c_int, f32, u64, u64, vp, u64,
                              ctypes.c_int, vp, vp, vp],
            "ef_layer_norm_grad": [vp, u64, ctypes.c_int, vp, ctypes.c_int, vp, vp, vp, u64,
                                   ctypes.c_int, u64, u64, vp, u64, vp, vp, vp],
            "ef_adamw": [u32, vp, vp, vp, ctypes.c_int, vp, vp, vp, vp, vp, f64, f64, f64, f64, f64,
                         u64, u64, vp, vp, vp, vp],
            "ef_adamw_states": [u32, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, vp],
            "ef_check_status": [vp],
            "ef_workspace_release": [],
        }
        for name, args in sig.items():
            fn = getattr(lib, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        lib.ef_status_string.argtypes = [ctypes.c_int]
        lib.ef_status_string.restype = ctypes.c_char_p
        lib.ef_kernel_launches.argtypes = []
        lib.ef_kernel_launches.restype = ctypes.c_uint64
        lib.ef_test_set_lookback_fault.argtypes = [ctypes.c_int64, ctypes.c_uint32]
        lib.ef_test_set_lookback_fault.restype = None
        lib.ef_test_set_stream_kernel.argtypes = [ctypes.c_int]
        lib.ef_test_set_stream_kernel.restype = None
        _lib = lib
        return lib


def status_string(status: int) -> str:
    return load_library().ef_status_string(int(status)).decode()


# A call's marshalling is on the path of every step of a training loop: at
# d = 100,000 the hard-threshold kernel takes less time than the checks of its
# seven arguments once did. So pointers go to ctypes as plain integers (the
# declared argument types convert them), the stream is read without building
# a torch.cuda.Stream, and an argument that passes its checks costs one call.
# Measured on the Grace host of a GB300, us a call, before -> after:
# ef_hard_threshold 11.2 -> 5.6 (2.6 of it the library), sparse_aggregate of 4
# lists 18.6 -> 11.
# (A torch without CUDA has neither of the two functions; its tensors are
# refused before a stream is asked for.)
_Tensor = torch.Tensor
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is None or _current_device is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(_current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(status: int, where: str):
    if status != EF_OK:
        raise EfError(status, where)


def _dev(t: torch.Tensor, name: str, dtype, numel=0):
    """The device pointer of a contiguous CUDA tensor of this dtype with at
    least `numel` elements (0 for an empty one)."""
    if isinstance(t, _Tensor) and t.dtype is dtype and t.is_cuda and t.is_contiguous():
        n = t.numel()
        if n >= numel:
            return t.data_ptr() if n else 0
    _refuse(t, name, dtype, numel)


def _refuse(t, name, dtype, numel):
    if not isinstance(t, _Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    raise ValueError("%s holds %d elements, needs %d" % (name, t.numel(), numel))


def _pointers(tensors, name, dtype, numel=0):
    """HOST array of the tensors' device pointers, checked as by _dev."""
    try:
        if numel:
            p = [t.data_ptr() if t.dtype is dtype and t.is_cuda and t.is_contiguous()
                 and t.numel() >= numel else _dev(t, name, dtype, numel) for t in tensors]
        else:  # an empty tensor's data_ptr() is 0
            p = [t.data_ptr() if t.dtype is dtype and t.is_cuda and t.is_contiguous()
                 else _dev(t, name, dtype) for t in tensors]
    except AttributeError:  # something that is no tensor: refused by name
        p = [_dev(t, name, dtype, numel) for t in tensors]
    return (ctypes.c_void_p * max(len(p), 1))(*p)


def _real(x):
    """x for a c_float parameter; what is no number is a TypeError here (in a
    call's arguments ctypes makes it an ArgumentError)."""
    return x if type(x) is float else ctypes.c_float(x)


def _gradient(g: torch.Tensor):
    if g.dtype is torch.float32:
        return False
    if g.dtype is torch.bfloat16:
        return True
    raise TypeError("g must be float32 or bfloat16")


def _err(err_sq_out):
    return None if err_sq_out is None else _dev(err_sq_out, "err_sq_out", torch.float64, 1)


TILE = 4096  # coordinates per tile of a message's tile index


def tiles_for(d: int) -> int:
    """Length of a message's tile index for dimension d: ceil(d / TILE) + 1."""
    return (int(d) + TILE - 1) // TILE + 1


def ef_hard_threshold(g, e, gamma, lam, idx_out, val_out, count_out, stream=None,
                      err_sq_out=None, tiles_out=None):
    """EF accumulate + hard-threshold + compaction (``ef_hard_threshold[_bf16]``;
    ``ef_hard_threshold_ex`` when ``err_sq_out`` is given,
    ``ef_hard_threshold_tiled`` when ``tiles_out`` is given).

    ``g`` float32 or bfloat16 [d]; ``e`` float32 [d], updated in place;
    ``idx_out`` int32 [>= d] (uint32 bit patterns), ``val_out`` float32 [>= d],
    ``count_out`` int32 [>= 1]; ``err_sq_out`` optional float64 [>= 1]:
    ||e'||^2 of the step; ``tiles_out`` optional int32 [>= tiles_for(d)]: the
    message's tile index (pairs below each multiple of TILE, then the count).
    """
    lib = load_library()
    bf16 = _gradient(g)
    d = e.numel()
    if g.numel() != d:
        raise ValueError("g and e differ in length")
    head = (_dev(g, "g", g.dtype), _dev(e, "e", torch.float32), _real(gamma), _real(lam), d,
            _dev(idx_out, "idx_out", torch.int32, d),
            _dev(val_out, "val_out", torch.float32, d),
            _dev(count_out, "count_out", torch.int32, 1))
    if tiles_out is not None:
        _check(lib.ef_hard_threshold_tiled(
            head[0], int(bf16), *head[1:], _dev(tiles_out, "tiles_out", torch.int32, tiles_for(d)),
            _err(err_sq_out), _stream(stream)), "ef_hard_threshold_tiled")
        return
    if err_sq_out is not None:
        _check(lib.ef_hard_threshold_ex(head[0], int(bf16), *head[1:], _err(err_sq_out),
                                        _stream(stream)), "ef_hard_threshold_ex")
        return
    fn = lib.ef_hard_threshold_bf16 if bf16 else lib.ef_hard_threshold
    _check(fn(*head, _stream(stream)), "ef_hard_threshold")


def ef_topk(g, e, gamma, k, idx_out, val_out, count_out, stream=None, err_sq_out=None):
    """EF accumulate + Top-k + compaction (``ef_topk[_bf16]``, ``ef_topk_ex`` with
    ``err_sq_out``); exactly k pairs."""
    lib = load_library()
    bf16 = _gradient(g)
    d = e.numel()
    if g.numel() != d:
        raise ValueError("g and e differ in length")
    head = (_dev(g, "g", g.dtype), _dev(e, "e", torch.float32), _real(gamma), int(k), d,
            _dev(idx_out, "idx_out", torch.int32, k),
            _dev(val_out, "val_out", torch.float32, k),
            _dev(count_out, "count_out", torch.int32, 1))
    if err_sq_out is not None:
        _check(lib.ef_topk_ex(head[0], int(bf16), *head[1:], _err(err_sq_out), _stream(stream)),
               "ef_topk_ex")
        return
    fn = lib.ef_topk_bf16 if bf16 else lib.ef_topk
    _check(fn(*head, _stream(stream)), "ef_topk")


def ef_topk_layerwise(g, e, gamma, seg_end, seg_k, idx_out, val_out, count_out, stream=None,
                      err_sq_out=None):
    """EF accumulate + layer-wise Top-k + compaction (``ef_topk_layerwise[_bf16]``).

    ``seg_end``/``seg_k``: sequences of n_seg integers (host side): segment s
    is ``[seg_end[s-1], seg_end[s])`` and sends its ``seg_k[s]`` largest
    coordinates; exactly ``sum(seg_k)`` pairs are written.
    """
    lib = load_library()
    bf16 = _gradient(g)
    d = e.numel()
    if g.numel() != d:
        raise ValueError("g and e differ in length")
    ends = np.ascontiguousarray(seg_end, dtype=np.uint64)
    ks = np.ascontiguousarray(seg_k, dtype=np.uint64)
    if ends.ndim != 1 or ks.shape != ends.shape:
        raise ValueError("seg_end and seg_k must be 1-D of one length")
    total = int(ks.sum()) if ks.size else 0
    head = (_dev(g, "g", g.dtype), _dev(e, "e", torch.float32), _real(gamma), ends.size,
            ends.ctypes.data, ks.ctypes.data, d, _dev(idx_out, "idx_out", torch.int32, total),
            _dev(val_out, "val_out", torch.float32, total),
            _dev(count_out, "count_out", torch.int32, 1))
    if err_sq_out is not None:
        _check(lib.ef_topk_layerwise_ex(head[0], int(bf16), *head[1:], _err(err_sq_out),
                                        _stream(stream)), "ef_topk_layerwise_ex")
        return
    fn = lib.ef_topk_layerwise_bf16 if bf16 else lib.ef_topk_layerwise
    _check(fn(*head, _stream(stream)), "ef_topk_layerwise")


def _tile_array(tiles, n, d):
    if len(tiles) != n:
        raise ValueError("one tile index per list")
    return _pointers(tiles, "tiles", torch.int32, tiles_for(d))


def sparse_aggregate(idx_list, val_list, counts, d, dense_out, stream=None, tiles=None):
    """Worker-ordered sum of n sparse vectors into ``dense_out`` (float32 [d]).

    ``idx_list``/``val_list``: n int32 / float32 CUDA tensors; ``counts``: int32
    CUDA tensor of n pair counts; ``tiles`` optional: the n lists' tile indexes
    (``sparse_aggregate_tiled``).
    """
    lib = load_library()
    n = len(idx_list)
    if n != len(val_list):
        raise ValueError("idx_list and val_list differ in length")
    idx_arr = _pointers(idx_list, "idx", torch.int32)
    val_arr = _pointers(val_list, "val", torch.float32)
    cnt = _dev(counts, "counts", torch.int32, n)
    out = _dev(dense_out, "dense_out", torch.float32, d)
    if tiles is not None:
        _check(lib.sparse_aggregate_tiled(n, idx_arr, val_arr, _tile_array(tiles, n, d), cnt,
                                          int(d), out, _stream(stream)), "sparse_aggregate_tiled")
        return
    _check(lib.sparse_aggregate(n, idx_arr, val_arr, cnt, int(d), out, _stream(stream)),
           "sparse_aggregate")


def sparse_aggregate_apply(idx_list, val_list, counts, d, alpha, x, m=None, momentum=0.0, lr=0.0,
                           stream=None, tiles=None):
    """Worker-ordered sum of n sparse vectors, scaled by ``alpha``, applied to
    the model ``x`` (float32 [d], in place): ``x -= Delta'`` without ``m``;
    with ``m`` (float32 [d], in place) ``m = fmaf(momentum, m, Delta')`` and
    ``x = fmaf(-lr, Delta' + m, x)``. ``tiles`` optional: the lists' tile
    indexes (``sparse_aggregate_apply_tiled``)."""
    lib = load_library()
    n = len(idx_list)
    if n != len(val_list):
        raise ValueError("idx_list and val_list differ in length")
    idx_arr = _pointers(idx_list, "idx", torch.int32)
    val_arr = _pointers(val_list, "val", torch.float32)
    m_ptr = None if m is None else _dev(m, "m", torch.float32, d)
    tail = (_dev(counts, "counts", torch.int32, n), int(d), _real(alpha),
            _dev(x, "x", torch.float32, d), m_ptr, _real(momentum), _real(lr), _stream(stream))
    if tiles is not None:
        _check(lib.sparse_aggregate_apply_tiled(n, idx_arr, val_arr, _tile_array(tiles, n, d),
                                                *tail), "sparse_aggregate_apply_tiled")
        return
    _check(lib.sparse_aggregate_apply(n, idx_arr, val_arr, *tail), "sparse_aggregate_apply")


def ef_scaled_round(g, e, gamma, scale_log2, q_out, unsent_out, stream=None, err_sq_out=None):
    """EF accumulate + scaled integer rounding (``ef_scaled_round_ex``):
    ``q_out`` int32 [d] = RNE(a 2^scale_log2), ``e`` becomes a - q 2^-scale_log2;
    ``unsent_out`` int32 [>= 1] counts the coordinates that did not fit."""
    lib = load_library()
    bf16 = _gradient(g)
    d = e.numel()
    if g.numel() != d:
        raise ValueError("g and e differ in length")
    _check(lib.ef_scaled_round_ex(_dev(g, "g", g.dtype), int(bf16), _dev(e, "e", torch.float32),
                                  _real(gamma), int(scale_log2), d,
                                  _dev(q_out, "q_out", torch.int32, d),
                                  _dev(unsent_out, "unsent_out", torch.int32, 1),
                                  _err(err_sq_out), _stream(stream)), "ef_scaled_round_ex")


def int_aggregate(q_list, d, scale_log2, dense_out, stream=None):
    """Exact integer sum of n dense int32 messages, as RN(S) 2^-scale_log2."""
    lib = load_library()
    n = len(q_list)
    arr = _pointers(q_list, "q", torch.int32, d)
    _check(lib.int_aggregate(n, arr, int(d), int(scale_log2),
                             _dev(dense_out, "dense_out", torch.float32, d), _stream(stream)),
           "int_aggregate")


def _rows(t, name, dtype, rows, cols):
    """(device pointer, row stride in elements) of a CUDA matrix of this dtype
    and shape whose rows are contiguous; 0 for an empty one."""
    if not isinstance(t, _Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError("%s must be [%d, %d], got %s" % (name, rows, cols, list(t.shape)))
    if t.numel() == 0:
        return 0, max(cols, 1)
    if cols > 1 and t.stride(1) != 1:
        raise ValueError("the rows of %s must be contiguous" % name)
    ld = t.stride(0) if rows > 1 else cols
    if ld < cols:
        raise ValueError("the rows of %s overlap" % name)
    return t.data_ptr(), ld


def _vocab_inputs(h, w, target, bias):
    if not isinstance(h, _Tensor) or not isinstance(w, _Tensor) or h.dim() != 2 or w.dim() != 2:
        raise TypeError("h and w must be matrices")
    n, d = h.shape
    v = w.shape[0]
    return (n, v, d, (*_rows(h, "h", torch.bfloat16, n, d), *_rows(w, "w", torch.bfloat16, v, d),
                      None if bias is None else _dev(bias, "bias", torch.bfloat16, v),
                      _dev(target, "target", torch.int64, n)))


def ef_vocab_loss(h, w, target, loss_out, lse_out, bias=None, stream=None):
    """Softmax cross entropy of hidden states against a vocabulary, without the
    logits in memory (``ef_vocab_loss``).

    ``h`` bfloat16 [n, d] and ``w`` bfloat16 [v, d], rows contiguous at any row
    stride; ``target`` int64 [n], a negative one skips its row; ``bias``
    optional bfloat16 [v]; ``loss_out``, ``lse_out`` float32 [>= n].
    """
    lib = load_library()
    n, v, d, head = _vocab_inputs(h, w, target, bias)
    _check(lib.ef_vocab_loss(*head, n, v, d, _dev(loss_out, "loss_out", torch.float32, n),
                             _dev(lse_out, "lse_out", torch.float32, n), _stream(stream)),
           "ef_vocab_loss")


def ef_vocab_loss_grad(h, w, target, lse, row_scale, dh_out, dw_out, bias=None, dbias_out=None,
                       stream=None):
    """Gradient of ``sum(row_scale * loss)`` (``ef_vocab_loss_grad``): ``lse`` as
    written by ``ef_vocab_loss``, ``row_scale`` float32 [n]; ``dh_out`` bfloat16
    [n, d], ``dw_out`` bfloat16 [v, d], rows contiguous at any row stride;
    ``dbias_out`` optional bfloat16 [>= v] (needs ``bias``)."""
    lib = load_library()
    n, v, d, head = _vocab_inputs(h, w, target, bias)
    _check(lib.ef_vocab_loss_grad(
        *head, _dev(lse, "lse", torch.float32, n), _dev(row_scale, "row_scale", torch.float32, n),
        n, v, d, *_rows(dh_out, "dh_out", torch.bfloat16, n, d),
        *_rows(dw_out, "dw_out", torch.bfloat16, v, d),
        None if dbias_out is None else _dev(dbias_out, "dbias_out", torch.bfloat16, v),
        _stream(stream)), "ef_vocab_loss_grad")


def _matrices(tensors, name, dtype, shapes):
    """Device pointers and row strides of matrices, checked as by _rows."""
    pointers, strides = array.array("Q"), array.array("Q")
    for t, shape in zip(tensors, shapes):
        if isinstance(t, _Tensor) and t.dtype is dtype and t.is_cuda and t.shape == shape:
            ld, step = t.stride()
            if step == 1 and ld >= shape[1] > 0:
                pointers.append(t.data_ptr())
                strides.append(ld)
                continue
        p, ld = _rows(t, name, dtype, *shape)  # unusual, or refused
        pointers.append(p)
        strides.append(ld)
    return pointers, strides


def ef_orthogonalize(updates, outs, momenta=None, momentum=0.0, stream=None):
    """Orthogonalised updates of a list of weight matrices (``ef_orthogonalize``):
    momentum (``momenta`` optional: float32 matrices, updated in place), then
    five Newton-Schulz steps. ``updates`` float32 or bfloat16 matrices of one
    dtype, ``outs`` bfloat16 matrices of the same shapes; rows contiguous at
    any row stride."""
    lib = load_library()
    n = len(updates)
    if len(outs) != n or (momenta is not None and len(momenta) != n):
        raise ValueError("updates, outs and momenta differ in length")
    momentum = _real(momentum)
    if n == 0:
        return
    if not all(isinstance(t, _Tensor) and t.dim() == 2 for t in updates):
        raise TypeError("updates must be matrices")
    dtype = updates[0].dtype
    if dtype is not torch.float32 and dtype is not torch.bfloat16:
        raise TypeError("updates must be float32 or bfloat16")
    shapes = [t.shape for t in updates]
    rows = array.array("Q", [s[0] for s in shapes])
    cols = array.array("Q", [s[1] for s in shapes])
    u, ld_u = _matrices(updates, "updates", dtype, shapes)
    out, ld_out = _matrices(outs, "outs", torch.bfloat16, shapes)
    m = ld_m = None
    if momenta is not None:
        m, ld_m = _matrices(momenta, "momenta", torch.float32, shapes)

    def at(words):
        return None if words is None else words.buffer_info()[0]
    _check(lib.ef_orthogonalize(n, at(rows), at(cols), at(u), at(ld_u),
                                int(dtype is torch.bfloat16), at(m), at(ld_m), momentum, at(out),
                                at(ld_out), _stream(stream)), "ef_orthogonalize")


_KINDS = {torch.float32: 0, torch.bfloat16: 1}  # ef_grad_type


# These entries' calls are on the path of single tokens and small layers, where a
# kernel takes 2 us: a tensor's checks are a handful of attribute reads in one
# expression, and what does not pass them goes to a function that says why.
# (_here: the current device, which these entries' tensors must be on.)
_here = torch.cuda.current_device if _current_device is None else _current_device


def _on_device(t, name, dev):
    if not isinstance(t, _Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if t.get_device() != dev:
        raise ValueError("%s is on another device than the current one" % name)


def _other_matrix(t, name, shape, dev):
    """(device pointer, row stride, ef_grad_type) of a matrix that is not contiguous,
    or is empty; others are refused."""
    _on_device(t, name, dev)
    if t.dtype not in _KINDS:
        raise TypeError("%s must be float32 or bfloat16, got %s" % (name, t.dtype))
    return (*_rows(t, name, t.dtype, *shape), _KINDS[t.dtype])


def _matrix(t, name, shape, dev):
    """(device pointer, row stride, ef_grad_type) of a float32 or bfloat16 matrix of
    this shape on the device whose rows are contiguous; 0 for an empty one."""
    try:
        if t.get_device() == dev and t.shape == shape and t.is_contiguous():
            return t.data_ptr(), shape[1], _KINDS[t.dtype]
    except (AttributeError, KeyError):
        pass
    return _other_matrix(t, name, shape, dev)


def _vector(t, name, dtype, numel, dev):
    """The device pointer of a contiguous tensor of this dtype on the device, with at
    least `numel` entries; None for None."""
    if t is None:
        return None
    try:
        if t.dtype is dtype and t.get_device() == dev and t.numel() >= numel and t.is_contiguous():
            return t.data_ptr() or None
    except AttributeError:
        pass
    _on_device(t, name, dev)
    return _dev(t, name, dtype, numel)


def _no_matrix(name):
    return TypeError("%s must be a matrix" % name)


def _tokens(t, n, dev):
    try:
        if t.dtype is torch.int64 and t.get_device() == dev and t.shape == (n,) and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _on_device(t, "token", dev)
    if t.dim() != 1 or t.shape[0] != n:
        raise ValueError("token must be a vector with an entry per row")
    return _dev(t, "token", torch.int64, n)


def ef_embed(table, token, out, scale=1.0, stream=None):
    """Rows of an embedding table by token (``ef_embed``): ``out[i] = scale *
    table[token[i]]``, a row of zeros where the token is negative.

    ``table`` [v, d] and ``out`` [n, d] float32 or bfloat16, rows contiguous at any
    row stride; ``token`` int64 [n].
    """
    lib = _lib or load_library()
    dev = _here()
    try:
        v, d = of_table = table.shape
        n, width = of_out = out.shape
    except (AttributeError, ValueError):
        raise _no_matrix("table and out") from None
    if width != d:
        raise ValueError("table and out differ in width")
    at, ld, kind = _matrix(table, "table", of_table, dev)
    to, ld_out, out_kind = _matrix(out, "out", of_out, dev)
    status = lib.ef_embed(at, ld, kind, _tokens(token, n, dev), n, v, d, _real(scale), to, ld_out,
                          out_kind, _raw_stream(dev) if stream is None else _stream(stream))
    if status:
        _check(status, "ef_embed")


def ef_embed_grad(dout, token, dtable_out, scale=1.0, accumulate=False, stream=None):
    """Gradient of an embedding table (``ef_embed_grad``): ``scale`` times the sums
    of the rows of ``dout`` [n, d] of one token, written to ``dtable_out`` [v, d]
    (zeros elsewhere) or, with ``accumulate``, added to it. float32 or bfloat16,
    rows contiguous at any row stride; ``token`` int64 [n]."""
    lib = _lib or load_library()
    dev = _here()
    try:
        n, d = of_dout = dout.shape
        v, width = of_table = dtable_out.shape
    except (AttributeError, ValueError):
        raise _no_matrix("dout and dtable_out") from None
    if width != d:
        raise ValueError("dout and dtable_out differ in width")
    at, ld, kind = _matrix(dout, "dout", of_dout, dev)
    to, ld_out, out_kind = _matrix(dtable_out, "dtable_out", of_table, dev)
    status = lib.ef_embed_grad(at, ld, kind, _tokens(token, n, dev), n, v, d, _real(scale),
                               1 if accumulate else 0, to, ld_out, out_kind,
                               _raw_stream(dev) if stream is None else _stream(stream))
    if status:
        _check(status, "ef_embed_grad")


def _weight(t, name, dtype, d, dev):
    """The device pointer of a weight vector of d entries; None for None."""
    if t is None:
        return None
    try:
        if t.dtype is dtype and t.get_device() == dev and t.shape == (d,) and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _on_device(t, name, dev)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != 1 or t.shape[0] != d:
        raise ValueError("%s must have an entry per column" % name)
    return _dev(t, name, dtype, d)


def _kind_of(t, name):
    """The ef_grad_type of a weight vector."""
    try:
        return _KINDS[t.dtype]
    except (AttributeError, KeyError):
        raise TypeError("%s must be a float32 or bfloat16 tensor" % name) from None


def ef_layer_norm(x, y_out, weight=None, bias=None, eps=1e-5, mean_out=None, rstd_out=None,
                  stream=None):
    """Layer norm over the rows of ``x`` (``ef_layer_norm``). ``x``, ``y_out`` [n, d]
    float32 or bfloat16, rows contiguous at any row stride; ``weight``, ``bias``
    [d] of one dtype, or None; ``mean_out``, ``rstd_out`` float32 [>= n] for the
    gradient, or None."""
    lib = _lib or load_library()
    dev = _here()
    try:
        n, d = shape = x.shape
    except (AttributeError, ValueError):
        raise _no_matrix("x") from None
    w = b = None
    kind = 0
    if weight is not None:
        kind = _kind_of(weight, "weight")
        w = _weight(weight, "weight", weight.dtype, d, dev)
    if bias is not None:
        if weight is None:
            kind = _kind_of(bias, "bias")
        b = _weight(bias, "bias", (bias if weight is None else weight).dtype, d, dev)
    at, ld, x_kind = _matrix(x, "x", shape, dev)
    to, ld_y, y_kind = _matrix(y_out, "y_out", shape, dev)
    status = lib.ef_layer_norm(
        at, ld, x_kind, w, b, kind, eps if type(eps) is float else _real(eps), n, d, to, ld_y, y_kind,
        None if mean_out is None else _vector(mean_out, "mean_out", torch.float32, n, dev),
        None if rstd_out is None else _vector(rstd_out, "rstd_out", torch.float32, n, dev),
        _raw_stream(dev) if stream is None else _stream(stream))
    if status:
        _check(status, "ef_layer_norm")


def ef_layer_norm_grad(x, mean, rstd, dy, dx_out=None, weight=None, dweight_out=None,
                       dbias_out=None, stream=None):
    """Gradient of layer norm (``ef_layer_norm_grad``): ``mean`` and ``rstd`` as
    written by ``ef_layer_norm`` for ``x`` and ``weight``; ``dx_out`` [n, d] of x's
    dtype, ``dweight_out`` and ``dbias_out`` [d] of the weight's, each optional."""
    lib = _lib or load_library()
    dev = _here()
    try:
        n, d = shape = x.shape
    except (AttributeError, ValueError):
        raise _no_matrix("x") from None
    at, ld, x_kind = _matrix(x, "x", shape, dev)
    dy_at, ld_dy, dy_kind = _matrix(dy, "dy", shape, dev)
    dx, ld_dx = None, d
    if dx_out is not None:
        dx, ld_dx, dx_kind = _matrix(dx_out, "dx_out", shape, dev)
        if dx_kind != x_kind:
            raise TypeError("dx_out must be %s, got %s" % (x.dtype, dx_out.dtype))
    w = dw = db = dtype = None
    kind = 0
    if weight is not None:
        kind, dtype = _kind_of(weight, "weight"), weight.dtype
        w = _weight(weight, "weight", dtype, d, dev)
    if dweight_out is not None:
        if dtype is None:
            kind, dtype = _kind_of(dweight_out, "dweight_out"), dweight_out.dtype
        dw = _weight(dweight_out, "dweight_out", dtype, d, dev)
    if dbias_out is not None:
        if dtype is None:
            kind, dtype = _kind_of(dbias_out, "dbias_out"), dbias_out.dtype
        db = _weight(dbias_out, "dbias_out", dtype, d, dev)
    if n and (mean is None or rstd is None):
        raise TypeError("mean and rstd must be CUDA tensors")
    status = lib.ef_layer_norm_grad(
        at, ld, x_kind, w, kind, _vector(mean, "mean", torch.float32, n, dev),
        _vector(rstd, "rstd", torch.float32, n, dev), dy_at, ld_dy, dy_kind, n, d, dx, ld_dx, dw, db,
        _raw_stream(dev) if stream is None else _stream(stream))
    if status:
        _check(status, "ef_layer_norm_grad")


class TensorList:
    """Tensors of a model as ``ef_adamw`` takes them: contiguous CUDA tensors of one
    dtype on one device, checked once. It holds the tensors, and their addresses
    as they are now (a tensor whose storage is replaced needs a new list)."""

    __slots__ = ("tensors", "dtype", "device", "numel", "pointers", "_sizes", "_at", "_blocks")

    def __init__(self, tensors, name="tensors"):
        self.tensors = tensors = tuple(tensors)
        self.dtype = self.device = None
        if tensors and isinstance(tensors[0], _Tensor):
            self.dtype, self.device = tensors[0].dtype, tensors[0].get_device()
        if not all(isinstance(t, _Tensor) and t.dtype is self.dtype and t.is_contiguous()
                   and t.get_device() == self.device >= 0 for t in tensors):
            self._refuse(name)
        self.numel = array.array("Q", [t.numel() for t in tensors])
        self.pointers = array.array("Q", [t.data_ptr() for t in tensors])
        self._sizes = self.numel.tobytes()
        self._blocks = None  # (sizes of the exponents of 8-bit states, once asked for)
        self._at = self.pointers.buffer_info()[0]

    def _refuse(self, name):
        for t in self.tensors:
            if not isinstance(t, _Tensor) or not t.is_cuda:
                raise TypeError("%s must be CUDA tensors" % name)
            if t.dtype is not self.dtype:
                raise TypeError("%s must be of one dtype, got %s and %s" % (name, self.dtype, t.dtype))
            if t.get_device() != self.device:
                raise ValueError("%s must be on one device" % name)
        raise ValueError("%s must be contiguous" % name)

    def __len__(self):
        return len(self.tensors)

    def __iter__(self):
        return iter(self.tensors)

    def __getitem__(self, i):
        return self.tensors[i]


def _list(tensors, name, dtypes, like, dev, sizes=None):
    """A TensorList of one of the dtypes on the device; as long as `like` and of its
    sizes (or of the bytes `sizes` of an array of them)."""
    x = tensors if type(tensors) is TensorList else TensorList(tensors, name)
    if x.dtype in dtypes and x.device == dev and (
            like is None or x._sizes == (like._sizes if sizes is None else sizes)):
        return x
    if not x.tensors:
        if like is None or not like.tensors:
            return x
    elif x.dtype not in dtypes:
        raise TypeError("%s must be %s, got %s" % (name, " or ".join(map(str, dtypes)), x.dtype))
    elif x.device != dev:
        raise ValueError("%s are on another device than the current one" % name)
    if like is not None and x._sizes != (like._sizes if sizes is None else sizes):
        raise ValueError("%s differ from the other lists in number or sizes" % name)
    return x


BLOCK = 128  # entries of an 8-bit state that share an exponent


def exponents_for(numel: int) -> int:
    """Length of the exponents of an 8-bit state of this size: ceil(numel / BLOCK)."""
    return (int(numel) + BLOCK - 1) // BLOCK


def _blocks(x):
    if x._blocks is None:
        x._blocks = array.array("Q", [exponents_for(n) for n in x.numel]).tobytes()
    return x._blocks


_F32, _U8, _GRADS = (torch.float32,), (torch.uint8,), (torch.float32, torch.bfloat16)


def ef_adamw(params, grads, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01,
             m_exponents=None, v_exponents=None, copies=None, grad_scale=None, seed=0, stream=None):
    """One AdamW step over lists of tensors (``ef_adamw``); a list may be a
    ``TensorList``, which is checked once.

    ``params`` float32, updated in place; ``grads`` float32 or bfloat16; ``m``, ``v``
    float32, or uint8 codes with uint8 ``m_exponents``, ``v_exponents`` (of
    ``exponents_for(numel)`` entries; all zero at the start), whose stochastic
    rounding ``seed`` and the step fix; ``copies`` optional bfloat16: the new
    parameters, rounded. ``step`` counts from 1; ``step`` and ``lr`` may be CUDA
    tensors of one int64 and one float32, and ``grad_scale`` one of a float32 that
    multiplies the gradients: they are read when the step runs (by a captured
    call at each replay).
    """
    lib = _lib or load_library()
    dev = _here()
    p = _list(params, "params", _F32, None, dev)
    g = _list(grads, "grads", _GRADS, p, dev)
    state = _F32 if m_exponents is None and v_exponents is None else _U8
    ms, vs = _list(m, "m", state, p, dev), _list(v, "v", state, p, dev)
    me = ve = c = None
    if state is _U8:
        if m_exponents is None or v_exponents is None:
            raise ValueError("m_exponents and v_exponents come together")
        sizes = _blocks(p)
        me = _list(m_exponents, "m_exponents", _U8, p, dev, sizes)
        ve = _list(v_exponents, "v_exponents", _U8, p, dev, sizes)
    if copies is not None:
        c = _list(copies, "copies", (torch.bfloat16,), p, dev)
    lr_dev = step_dev = None
    if isinstance(lr, _Tensor):
        lr_dev, lr = _vector(lr, "lr", torch.float32, 1, dev), 0.0
    if isinstance(step, _Tensor):
        step_dev, step = _vector(step, "step", torch.int64, 1, dev), 1
    elif step < 0:
        raise ValueError("step counts from 1")
    _check(lib.ef_adamw(len(p.tensors), p.numel.buffer_info()[0], p._at, g._at,
                        1 if g.dtype is torch.bfloat16 else 0, ms._at, vs._at,
                        None if me is None else me._at, None if ve is None else ve._at,
                        None if c is None else c._at, float(lr), float(beta1), float(beta2),
                        float(eps), float(weight_decay), int(step),
                        int(seed) & 0xFFFFFFFFFFFFFFFF, lr_dev, step_dev,
                        _vector(grad_scale, "grad_scale", torch.float32, 1, dev), _stream(stream)),
           "ef_adamw")


def ef_adamw_states(m, v, m_exponents, v_exponents, m_out, v_out, stream=None):
    """The values that 8-bit states stand for (``ef_adamw_states``): lists as
    ``ef_adamw`` takes them to ``m_out`` and ``v_out``, lists of float32 or
    bfloat16 tensors (exact in both)."""
    lib = _lib or load_library()
    dev = _here()
    ms = _list(m, "m", _U8, None, dev)
    vs = _list(v, "v", _U8, ms, dev)
    sizes = _blocks(ms)
    me = _list(m_exponents, "m_exponents", _U8, ms, dev, sizes)
    ve = _list(v_exponents, "v_exponents", _U8, ms, dev, sizes)
    mo, vo = _list(m_out, "m_out", _GRADS, ms, dev), _list(v_out, "v_out", _GRADS, ms, dev)
    if mo.dtype is not vo.dtype:
        raise TypeError("m_out and v_out differ in dtype")
    _check(lib.ef_adamw_states(len(ms.tensors), ms.numel.buffer_info()[0], ms._at, vs._at, me._at,
                               ve._at, mo._at, vo._at, 1 if mo.dtype is torch.bfloat16 else 0,
                               _stream(stream)), "ef_adamw_states")


def ef_check_status(stream=None) -> int:
    """Synchronise the stream; return (and clear) the latched device status."""
    return int(load_library().ef_check_status(_stream(stream)))


def ef_workspace_release():
    _check(load_library().ef_workspace_release(), "ef_workspace_release")


def ef_kernel_launches() -> int:
    return int(load_library().ef_kernel_launches())


def ef_test_set_lookback_fault(withheld_tile: int, spin_limit_us: int = 0):
    load_library().ef_test_set_lookback_fault(int(withheld_tile), int(spin_limit_us))


def ef_test_set_stream_kernel(mode: int):
    load_library().ef_test_set_stream_kernel(int(mode))
