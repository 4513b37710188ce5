"""ctypes binding of libflexmoe.so (include/flexmoe.h).

Argument marshalling only: every step of the layer runs in the HIP library.
Functions keep the C names; device buffers are passed as torch CUDA tensors
(their data pointers), the stream defaults to torch's current stream.  There
is no fallback: if the library is missing or a call fails, an exception is
raised.
"""
from __future__ import annotations

import ctypes
import math
import os
import threading
import warnings
from typing import Optional, Sequence

import numpy as np

from .build import LIB, TENSORS

FLEXMOE_F32 = 0
FLEXMOE_BF16 = 1

ERRORS = {
    -1: "FLEXMOE_EINVAL",
    -2: "FLEXMOE_ESHAPE",
    -3: "FLEXMOE_EKEEP",
    -4: "FLEXMOE_EWORKSPACE",
    -5: "FLEXMOE_EDTYPE",
    -6: "FLEXMOE_EHIP",
}

EXPORTED = ("flexmoe_workspace_bytes", "flexmoe_rank_reorder", "flexmoe_set_budget",
            "flexmoe_layer_forward", "flexmoe_keep_from_ratio", "flexmoe_last_error",
            "flexmoe_timing_enable", "flexmoe_timing_read", "flexmoe_clipped_channels",
            "flexmoe_export_clipped", "flexmoe_layer_forward_clipped",
            "flexmoe_layer_forward_bucketed", "flexmoe_saliency_workspace_bytes",
            "flexmoe_channel_saliency", "flexmoe_transpose_weights", "flexmoe_sample_actions",
            "flexmoe_train_workspace_bytes", "flexmoe_train_forward", "flexmoe_train_backward",
            "flexmoe_action_grad", "flexmoe_layer_forward_noalloc",
            "flexmoe_grouped_workspace_bytes", "flexmoe_grouped_forward", "flexmoe_grouped_input_grad",
            "flexmoe_grouped_weight_grad", "flexmoe_quantize_rows", "flexmoe_quantized_workspace_bytes",
            "flexmoe_quantized_forward", "flexmoe_adamw_step", "flexmoe_adamw_read_state")

# kernel indices of flexmoe_kernel_times
KERNELS = ("route", "dispatch_scan", "dispatch_scatter", "gate_up", "down", "combine",
           "gate_up_shared", "down_shared", "sal_transpose", "sal_prep", "sal_dgrad", "sal_wgrad",
           "sal_reduce", "act_dgrad", "act_dx", "act_other")
MAX_ACTIONS = 16
KEEP_AXES = {"none": 0, "N": 1, "K": 2}  # FLEXMOE_KEEP_*
STATE_BLOCK = 256                        # values that share a scale in 8-bit optimizer states


class FlexMoEError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("%s (%d): %s" % (ERRORS.get(code, "?"), code, msg))
        self.code = code


class flexmoe_layer_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("d", "E", "I", "top_k", "I_shared", "dtype", "norm_topk", "max_tokens")]


class flexmoe_kernel_times(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * len(KERNELS)), ("launches", ctypes.c_int64 * len(KERNELS))]


class flexmoe_grouped_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("groups", "N", "K", "dtype", "dw_dtype", "keep_axis", "max_rows", "ldx", "ldw", "ldy", "lddw")]


class flexmoe_adamw_tensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "master")] + \
               [("n", ctypes.c_int64)]


_TENSOR_BYTES = ctypes.sizeof(flexmoe_adamw_tensor)


class flexmoe_adamw_desc(ctypes.Structure):
    _fields_ = [("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("state_bits", ctypes.c_int32),
                ("seed", ctypes.c_uint32), ("step", ctypes.c_int64)] + \
               [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay", "grad_scale")] + \
               [("clock", ctypes.c_void_p)]


class flexmoe_action_set(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int32), ("ratio", ctypes.c_double * MAX_ACTIONS)]


def make_actions(ratios) -> flexmoe_action_set:
    a = flexmoe_action_set()
    a.K = len(ratios)
    for i, r in enumerate(ratios):
        a.ratio[i] = float(r)
    return a


class flexmoe_route_out(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("topk_idx", "topk_w", "counts", "offsets", "perm", "pos")]


_lib = None


def lib():
    """Load libflexmoe.so (built in-tree by build.py); raise if it is absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB):
            raise RuntimeError("libflexmoe.so is not built (%s); run "
                               "`python -m paper_2606_27866_amd.build`" % LIB)
        # torch ships its own HIP runtime (soname libamdhip64.so.7).  Loading
        # torch first makes the library's libamdhip64.so.7 dependency resolve
        # to that same runtime, so device pointers and streams are shared; a
        # second runtime in the process would not see the GPU.
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        D = ctypes.POINTER(flexmoe_layer_desc)
        L.flexmoe_workspace_bytes.argtypes = [D, i32]
        L.flexmoe_workspace_bytes.restype = sz
        L.flexmoe_rank_reorder.argtypes = [D] + [vp] * 9
        L.flexmoe_rank_reorder.restype = ctypes.c_int
        L.flexmoe_set_budget.argtypes = [D, vp, vp, vp]
        L.flexmoe_set_budget.restype = ctypes.c_int
        L.flexmoe_layer_forward.argtypes = [D, i32] + [vp] * 11 + [sz, ctypes.POINTER(flexmoe_route_out), vp]
        L.flexmoe_layer_forward.restype = ctypes.c_int
        L.flexmoe_layer_forward_noalloc.argtypes = [D, i32] + [vp] * 10 + [ctypes.POINTER(flexmoe_route_out), vp]
        L.flexmoe_layer_forward_noalloc.restype = ctypes.c_int
        L.flexmoe_clipped_channels.argtypes = [D, vp]
        L.flexmoe_clipped_channels.restype = ctypes.c_int64
        L.flexmoe_export_clipped.argtypes = [D] + [vp] * 8
        L.flexmoe_export_clipped.restype = ctypes.c_int
        L.flexmoe_layer_forward_clipped.argtypes = ([D, i32] + [vp] * 6 + [ctypes.c_int64] + [vp] * 5
                                                    + [sz, ctypes.POINTER(flexmoe_route_out), vp])
        L.flexmoe_layer_forward_clipped.restype = ctypes.c_int
        L.flexmoe_layer_forward_bucketed.argtypes = ([D, i32] + [vp] * 6 + [i32] + [vp] * 5
                                                     + [sz, ctypes.POINTER(flexmoe_route_out), vp])
        L.flexmoe_layer_forward_bucketed.restype = ctypes.c_int
        L.flexmoe_saliency_workspace_bytes.argtypes = [D, i32]
        L.flexmoe_saliency_workspace_bytes.restype = sz
        L.flexmoe_channel_saliency.argtypes = ([D, i32] + [vp] * 10 + [ctypes.c_float] + [vp] * 2
                                               + [sz, vp])
        L.flexmoe_channel_saliency.restype = ctypes.c_int
        AS = ctypes.POINTER(flexmoe_action_set)
        f32 = ctypes.c_float
        L.flexmoe_transpose_weights.argtypes = [D] + [vp] * 13
        L.flexmoe_transpose_weights.restype = ctypes.c_int
        L.flexmoe_sample_actions.argtypes = [D, AS] + [vp] * 5
        L.flexmoe_sample_actions.restype = ctypes.c_int
        L.flexmoe_train_workspace_bytes.argtypes = [D, i32]
        L.flexmoe_train_workspace_bytes.restype = sz
        L.flexmoe_train_forward.argtypes = [D, i32] + [vp] * 11 + [sz, vp]
        L.flexmoe_train_forward.restype = ctypes.c_int
        L.flexmoe_train_backward.argtypes = [D, i32] + [vp] * 12 + [sz, vp]
        L.flexmoe_train_backward.restype = ctypes.c_int
        L.flexmoe_action_grad.argtypes = [D, i32, AS, vp, vp, f32, f32, f32, vp, vp, vp, vp, sz, vp]
        L.flexmoe_action_grad.restype = ctypes.c_int
        G, i64 = ctypes.POINTER(flexmoe_grouped_desc), ctypes.c_int64
        for name in ("grouped", "quantized"):
            f = getattr(L, "flexmoe_%s_workspace_bytes" % name)
            f.argtypes, f.restype = [G, i32], sz
        L.flexmoe_grouped_forward.argtypes = [G, i32] + [vp] * 6 + [sz, vp]
        L.flexmoe_grouped_forward.restype = ctypes.c_int
        L.flexmoe_grouped_input_grad.argtypes = [G, i32] + [vp] * 6 + [sz, vp]
        L.flexmoe_grouped_input_grad.restype = ctypes.c_int
        L.flexmoe_grouped_weight_grad.argtypes = [G, i32] + [vp] * 5 + [i32, vp, sz, vp]
        L.flexmoe_grouped_weight_grad.restype = ctypes.c_int
        L.flexmoe_quantize_rows.argtypes = [i32, i32, i32, vp, vp, i64, vp, i64, vp, vp]
        L.flexmoe_quantize_rows.restype = ctypes.c_int
        L.flexmoe_quantized_forward.argtypes = [G, i32] + [vp] * 8 + [sz, vp]
        L.flexmoe_quantized_forward.restype = ctypes.c_int
        L.flexmoe_adamw_step.argtypes = [ctypes.POINTER(flexmoe_adamw_desc), vp, i32, vp]
        L.flexmoe_adamw_step.restype = ctypes.c_int
        L.flexmoe_adamw_read_state.argtypes = [i64] + [vp] * 4 + [i32] + [vp] * 3
        L.flexmoe_adamw_read_state.restype = ctypes.c_int
        L.flexmoe_keep_from_ratio.argtypes = [ctypes.c_double, i32]
        L.flexmoe_keep_from_ratio.restype = ctypes.c_int
        L.flexmoe_timing_enable.argtypes = [ctypes.c_int]
        L.flexmoe_timing_enable.restype = ctypes.c_int
        L.flexmoe_timing_read.argtypes = [ctypes.POINTER(flexmoe_kernel_times)]
        L.flexmoe_timing_read.restype = ctypes.c_int
        L.flexmoe_last_error.argtypes = []
        L.flexmoe_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


_tensors = None


def tensors():
    """The _tensors module (built in-tree by build.py); raise if it is absent."""
    global _tensors
    if _tensors is None:
        if not os.path.exists(TENSORS):
            raise RuntimeError("_tensors.so, which the optimizer needs, is not built (%s); run `python -m paper_2606_27866_amd.build`" % TENSORS)
        import torch  # noqa: F401  (its libraries are loaded first)
        from . import _tensors as module
        _tensors = module
    return _tensors


def _check(rc: int):
    if rc != 0:
        raise FlexMoEError(rc, lib().flexmoe_last_error().decode())


def _p(t) -> Optional[int]:
    """Device pointer of a tensor (or None)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    import torch
    # the raw handle of torch's current stream (torch.cuda.current_stream builds objects around it: 2.8 us against 0.1)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _capturing() -> bool:
    """Whether torch's current stream is being captured (tensors on the GPU exist, so CUDA is initialised)."""
    global _capturing
    import torch
    _capturing = torch._C._cuda_isCurrentStreamCapturing
    return _capturing()


def make_desc(d, E, I, top_k, I_shared=0, dtype=FLEXMOE_BF16, norm_topk=1, max_tokens=0):
    return flexmoe_layer_desc(d, E, I, top_k, I_shared, dtype, norm_topk, max_tokens)


def flexmoe_last_error() -> str:
    return lib().flexmoe_last_error().decode()


def flexmoe_timing_enable(on: bool):
    _check(lib().flexmoe_timing_enable(1 if on else 0))


def flexmoe_timing_read():
    """{kernel name: (total ms, launches)} since the last enable/read."""
    t = flexmoe_kernel_times()
    _check(lib().flexmoe_timing_read(ctypes.byref(t)))
    return {n: (t.ms[i], int(t.launches[i])) for i, n in enumerate(KERNELS)}


def flexmoe_keep_from_ratio(r: float, I: int) -> int:
    return int(lib().flexmoe_keep_from_ratio(float(r), int(I)))


def flexmoe_workspace_bytes(desc: flexmoe_layer_desc, T: int) -> int:
    n = lib().flexmoe_workspace_bytes(ctypes.byref(desc), int(T))
    if n == 0:
        raise FlexMoEError(-2, flexmoe_last_error())
    return int(n)


def flexmoe_set_budget(desc, keep_dev, keep_host: Sequence[int], stream=None):
    kh = np.ascontiguousarray(np.asarray(keep_host, dtype=np.int32))
    _check(lib().flexmoe_set_budget(ctypes.byref(desc), _p(keep_dev),
                                    kh.ctypes.data_as(ctypes.c_void_p), _stream(stream)))


def flexmoe_rank_reorder(desc, scores, w_gate, w_up, w_down, w_gate_r, w_up_r, w_down_r, perm,
                         stream=None):
    _check(lib().flexmoe_rank_reorder(ctypes.byref(desc), _p(scores), _p(w_gate), _p(w_up),
                                      _p(w_down), _p(w_gate_r), _p(w_up_r), _p(w_down_r), _p(perm),
                                      _stream(stream)))


def flexmoe_layer_forward(desc, T, x, logits, w_gate_r, w_up_r, w_down_r, keep_dev, ws_gate,
                          ws_up, ws_down, y, workspace, workspace_bytes=None, dbg=None,
                          stream=None):
    """dbg: optional dict with any of topk_idx, topk_w, counts, offsets, perm, pos tensors."""
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    ro = None
    if dbg:
        ro = flexmoe_route_out(*[_p(dbg.get(n)) for n, _ in flexmoe_route_out._fields_])
    _check(lib().flexmoe_layer_forward(
        ctypes.byref(desc), int(T), _p(x), _p(logits), _p(w_gate_r), _p(w_up_r), _p(w_down_r),
        _p(keep_dev), _p(ws_gate), _p(ws_up), _p(ws_down), _p(y), _p(workspace),
        int(workspace_bytes), ctypes.byref(ro) if ro is not None else None, _stream(stream)))


def flexmoe_layer_forward_noalloc(desc, T, x, logits, w_gate_r, w_up_r, w_down_r, keep_dev, ws_gate,
                                  ws_up, ws_down, y, dbg=None, stream=None):
    """flexmoe_layer_forward without a workspace (the library's static scratch)."""
    ro = None
    if dbg:
        ro = flexmoe_route_out(*[_p(dbg.get(n)) for n, _ in flexmoe_route_out._fields_])
    _check(lib().flexmoe_layer_forward_noalloc(
        ctypes.byref(desc), int(T), _p(x), _p(logits), _p(w_gate_r), _p(w_up_r), _p(w_down_r),
        _p(keep_dev), _p(ws_gate), _p(ws_up), _p(ws_down), _p(y),
        ctypes.byref(ro) if ro is not None else None, _stream(stream)))


def flexmoe_clipped_channels(desc, keep_host: Sequence[int]) -> int:
    kh = np.ascontiguousarray(np.asarray(keep_host, dtype=np.int32))
    n = int(lib().flexmoe_clipped_channels(ctypes.byref(desc), kh.ctypes.data_as(ctypes.c_void_p)))
    if n < 0:
        raise FlexMoEError(n, flexmoe_last_error())
    return n


def flexmoe_export_clipped(desc, keep_host, w_gate_r, w_up_r, w_down_r, w_gate_c, w_up_c, w_down_c,
                           stream=None):
    kh = np.ascontiguousarray(np.asarray(keep_host, dtype=np.int32))
    _check(lib().flexmoe_export_clipped(ctypes.byref(desc), kh.ctypes.data_as(ctypes.c_void_p),
                                        _p(w_gate_r), _p(w_up_r), _p(w_down_r), _p(w_gate_c),
                                        _p(w_up_c), _p(w_down_c), _stream(stream)))


def flexmoe_layer_forward_clipped(desc, T, x, logits, w_gate_c, w_up_c, w_down_c, keep_dev,
                                  packed_channels, ws_gate, ws_up, ws_down, y, workspace,
                                  workspace_bytes=None, dbg=None, stream=None):
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    ro = None
    if dbg:
        ro = flexmoe_route_out(*[_p(dbg.get(n)) for n, _ in flexmoe_route_out._fields_])
    _check(lib().flexmoe_layer_forward_clipped(
        ctypes.byref(desc), int(T), _p(x), _p(logits), _p(w_gate_c), _p(w_up_c), _p(w_down_c),
        _p(keep_dev), int(packed_channels), _p(ws_gate), _p(ws_up), _p(ws_down), _p(y),
        _p(workspace), int(workspace_bytes), ctypes.byref(ro) if ro is not None else None,
        _stream(stream)))


def flexmoe_layer_forward_bucketed(desc, T, x, logits, w_gate_r, w_up_r, w_down_r, keep_host, k_align,
                                   ws_gate, ws_up, ws_down, y, workspace, workspace_bytes=None,
                                   dbg=None, stream=None):
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size()
    kh = np.ascontiguousarray(np.asarray(keep_host, dtype=np.int32))
    ro = None
    if dbg:
        ro = flexmoe_route_out(*[_p(dbg.get(n)) for n, _ in flexmoe_route_out._fields_])
    _check(lib().flexmoe_layer_forward_bucketed(
        ctypes.byref(desc), int(T), _p(x), _p(logits), _p(w_gate_r), _p(w_up_r), _p(w_down_r),
        kh.ctypes.data_as(ctypes.c_void_p), int(k_align), _p(ws_gate), _p(ws_up), _p(ws_down), _p(y),
        _p(workspace), int(workspace_bytes), ctypes.byref(ro) if ro is not None else None,
        _stream(stream)))


def flexmoe_saliency_workspace_bytes(desc: flexmoe_layer_desc, T: int) -> int:
    n = lib().flexmoe_saliency_workspace_bytes(ctypes.byref(desc), int(T))
    if n == 0:
        raise FlexMoEError(-2, lib().flexmoe_last_error().decode())
    return n


def flexmoe_channel_saliency(desc, T, x, logits, w_gate, w_up, w_down, w_down_t, ws_gate, ws_up, ws_down,
                             y_target, scale, scores, workspace, workspace_bytes=None, stream=None):
    nbytes = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    _check(lib().flexmoe_channel_saliency(ctypes.byref(desc), int(T), _p(x), _p(logits), _p(w_gate),
                                          _p(w_up), _p(w_down), _p(w_down_t), _p(ws_gate), _p(ws_up),
                                          _p(ws_down), _p(y_target), float(scale), _p(scores), _p(workspace),
                                          nbytes, _stream(stream)))


def _nbytes(t, given):
    return t.numel() * t.element_size() if given is None else given


def flexmoe_transpose_weights(desc, w_gate, w_up, w_down, ws_gate, ws_up, ws_down, w_gate_t, w_up_t, w_down_t,
                              ws_gate_t, ws_up_t, ws_down_t, stream=None):
    _check(lib().flexmoe_transpose_weights(ctypes.byref(desc), *[_p(t) for t in (
        w_gate, w_up, w_down, ws_gate, ws_up, ws_down, w_gate_t, w_up_t, w_down_t, ws_gate_t, ws_up_t,
        ws_down_t)], _stream(stream)))


def flexmoe_sample_actions(desc, actions, alpha, gumbel, keep_dev, action_dev=None, stream=None):
    _check(lib().flexmoe_sample_actions(ctypes.byref(desc), ctypes.byref(actions), _p(alpha), _p(gumbel),
                                        _p(keep_dev), _p(action_dev), _stream(stream)))


def flexmoe_train_workspace_bytes(desc, T: int) -> int:
    n = lib().flexmoe_train_workspace_bytes(ctypes.byref(desc), int(T))
    if n == 0:
        raise FlexMoEError(-2, lib().flexmoe_last_error().decode())
    return n


def flexmoe_train_forward(desc, T, x, logits, w_gate, w_up, w_down, keep_dev, ws_gate, ws_up, ws_down, y,
                          workspace, workspace_bytes=None, stream=None):
    _check(lib().flexmoe_train_forward(ctypes.byref(desc), int(T), _p(x), _p(logits), _p(w_gate), _p(w_up),
                                       _p(w_down), _p(keep_dev), _p(ws_gate), _p(ws_up), _p(ws_down), _p(y),
                                       _p(workspace), _nbytes(workspace, workspace_bytes), _stream(stream)))


def flexmoe_train_backward(desc, T, logits, dy, w_gate_t, w_up_t, w_down_t, ws_gate_t, ws_up_t, ws_down_t, dx,
                           dlogits, dmask, workspace, workspace_bytes=None, stream=None):
    _check(lib().flexmoe_train_backward(ctypes.byref(desc), int(T), _p(logits), _p(dy), _p(w_gate_t),
                                        _p(w_up_t), _p(w_down_t), _p(ws_gate_t), _p(ws_up_t), _p(ws_down_t),
                                        _p(dx), _p(dlogits), _p(dmask), _p(workspace),
                                        _nbytes(workspace, workspace_bytes), _stream(stream)))


def flexmoe_action_grad(desc, T, actions, alpha, gumbel, tau, lambda_cost, beta, dmask, dalpha, stats,
                        workspace, workspace_bytes=None, stream=None):
    _check(lib().flexmoe_action_grad(ctypes.byref(desc), int(T), ctypes.byref(actions), _p(alpha), _p(gumbel),
                                     float(tau), float(lambda_cost), float(beta), _p(dmask), _p(dalpha),
                                     _p(stats), _p(workspace), _nbytes(workspace, workspace_bytes),
                                     _stream(stream)))


# ---- the experts' products, 8-bit products, AdamW ---------------------------
def make_grouped_desc(groups, N, K, dtype=FLEXMOE_BF16, dw_dtype=FLEXMOE_F32, keep_axis="none", max_rows=0, ldx=0, ldw=0,
                      ldy=0, lddw=0):
    return flexmoe_grouped_desc(groups, N, K, dtype, dw_dtype, KEEP_AXES[keep_axis], max_rows, ldx, ldw, ldy, lddw)


def flexmoe_grouped_workspace_bytes(desc, R: int) -> int:
    n = lib().flexmoe_grouped_workspace_bytes(ctypes.byref(desc), int(R))
    if n == 0:
        raise FlexMoEError(-2, flexmoe_last_error())
    return int(n)


def flexmoe_grouped_forward(desc, R, x, w, offsets, keep, y, workspace, workspace_bytes=None, stream=None):
    _check(lib().flexmoe_grouped_forward(ctypes.byref(desc), int(R), _p(x), _p(w), _p(offsets), _p(keep), _p(y),
                                         _p(workspace), _nbytes(workspace, workspace_bytes), _stream(stream)))


def flexmoe_grouped_input_grad(desc, R, dy, w, offsets, keep, dx, workspace, workspace_bytes=None, stream=None):
    _check(lib().flexmoe_grouped_input_grad(ctypes.byref(desc), int(R), _p(dy), _p(w), _p(offsets), _p(keep), _p(dx),
                                            _p(workspace), _nbytes(workspace, workspace_bytes), _stream(stream)))


def flexmoe_grouped_weight_grad(desc, R, dy, x, offsets, keep, dw, accumulate, workspace, workspace_bytes=None,
                                stream=None):
    _check(lib().flexmoe_grouped_weight_grad(ctypes.byref(desc), int(R), _p(dy), _p(x), _p(offsets), _p(keep), _p(dw),
                                             int(accumulate), _p(workspace), _nbytes(workspace, workspace_bytes),
                                             _stream(stream)))


def flexmoe_quantize_rows(rows, cols, dtype, x, x_gate, ldx, q, ldq, scale, stream=None):
    _check(lib().flexmoe_quantize_rows(int(rows), int(cols), int(dtype), _p(x), _p(x_gate), int(ldx), _p(q), int(ldq),
                                       _p(scale), _stream(stream)))


def flexmoe_quantized_workspace_bytes(desc, R: int) -> int:
    n = lib().flexmoe_quantized_workspace_bytes(ctypes.byref(desc), int(R))
    if n == 0:
        raise FlexMoEError(-2, flexmoe_last_error())
    return int(n)


def flexmoe_quantized_forward(desc, R, q, q_scale, w, w_scale, offsets, keep, y, workspace, workspace_bytes=None, stream=None):
    _check(lib().flexmoe_quantized_forward(ctypes.byref(desc), int(R), _p(q), _p(q_scale), _p(w), _p(w_scale), _p(offsets),
                                           _p(keep), _p(y), _p(workspace), _nbytes(workspace, workspace_bytes),
                                           _stream(stream)))


def flexmoe_adamw_step(desc, tensors, count=None, stream=None):
    """tensors: a ctypes array of flexmoe_adamw_tensor, or the address of one with `count` entries."""
    if count is None:
        count = len(tensors)
    _check(lib().flexmoe_adamw_step(ctypes.byref(desc), tensors if isinstance(tensors, int) else ctypes.addressof(tensors),
                                    int(count), _stream(stream)))


def flexmoe_adamw_read_state(n, m, v, m_scale, v_scale, dtype, m_out, v_out, stream=None):
    _check(lib().flexmoe_adamw_read_state(int(n), _p(m), _p(v), _p(m_scale), _p(v_scale), int(dtype), _p(m_out), _p(v_out),
                                          _stream(stream)))


_DTYPE_CODES = {}  # filled by the first call: the module does not import torch


def _dtype_code(dtype) -> int:
    code = _DTYPE_CODES.get(dtype)
    if code is None:
        import torch
        if dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("dtype must be torch.bfloat16 or torch.float32, got %s" % dtype)
        code = _DTYPE_CODES[dtype] = FLEXMOE_BF16 if dtype == torch.bfloat16 else FLEXMOE_F32
    return code


def _matrix(t, shape, dtype, name):
    """Row stride of a [..., rows, cols] tensor whose rows are contiguous and follow each other at one distance."""
    if t.dtype is dtype and t.shape == shape and t.is_cuda:
        st = t.stride()
        if st[-1] == 1:
            if shape[-2] > 1:
                if st[-2] >= shape[-1] and (len(st) == 2 or len(st) == 3 and st[0] == shape[1] * st[1]):
                    return st[-2]
            elif len(st) == 2:  # one row, or none
                return _pitch(shape[1], dtype.itemsize)
    return _matrix_checked(t, shape, dtype, name)


def _matrix_checked(t, shape, dtype, name):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be %s %s, got %s %s" % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU" % name)
    cols = t.shape[-1]
    if t.numel() and cols > 1 and t.stride(-1) != 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    ld, rows = None, 1  # of the dimensions so far, from the last but one on
    for n, step in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1:
            continue
        if ld is None:
            ld = step
        elif step != rows * ld and t.numel():
            raise ValueError("%s must hold its groups one after another (strides %s)" % (name, t.stride()))
        rows *= n
    if ld is None or not t.numel():
        return _pitch(cols, t.element_size())
    # an expanded tensor repeats one row with stride 0, which in a descriptor would stand for packed rows
    if ld < cols:
        raise ValueError("%s: rows overlap (strides %s); contiguous() makes a copy that can be used" % (name, t.stride()))
    return ld


def _pitch(cols, element_size) -> int:
    """Row length in elements rounded up to whole 16-byte units."""
    unit = 16 // element_size
    return -(-cols // unit) * unit


def _new(shape, dtype, device, stream=None):
    """A new tensor, made on the stream that will write it: memory of torch's current stream may still be in use there, and
    is used again there as soon as the tensor is dropped."""
    import torch
    if stream is None or torch.device(device).type == "cpu":
        return torch.empty(shape, dtype=dtype, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _padded(shape, dtype, device, stream=None):
    """A new tensor of `shape` whose rows start on 16-byte boundaries (a view of wider rows where they must)."""
    cols = _pitch(shape[-1], dtype.itemsize)
    if cols == shape[-1]:
        return _new(shape, dtype, device, stream)
    return _new((*shape[:-1], cols), dtype, device, stream)[..., :shape[-1]]


def _vector(t, n, dtype, name):
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("%s must be %d contiguous %s values on the GPU, got %s %s" % (name, n, dtype, t.dtype, tuple(t.shape)))
    return t.data_ptr()


class GroupedProduct:
    """The products of `groups` experts' matrices W_e [N][K] with their rows, and both gradients.

    A holder around the C calls (no arithmetic): it keeps the workspace for up to max_rows rows and allocates outputs.
    offsets [groups + 1] int32 on the device are the groups' row ranges (the forward's routing copies hold them); keep
    [groups] int32 limits W_e's rows (keep_axis "N") or columns ("K").  Calls on different streams need holders of their
    own: they share the workspace.  Threads may share a holder: its calls take their turn.
    """

    def __init__(self, groups, N, K, max_rows, dtype=None, keep_axis="none", device="cuda"):
        import torch
        self.groups, self.N, self.K, self.max_rows, self.keep_axis = groups, N, K, max_rows, keep_axis
        self.dtype = torch.bfloat16 if dtype is None else dtype
        self._i32, self._f32, self._w_shape = torch.int32, torch.float32, (groups, N, K)
        code = _dtype_code(self.dtype)
        es = self.dtype.itemsize
        self.desc = make_grouped_desc(groups, N, K, code, FLEXMOE_F32, keep_axis, max_rows, _pitch(K, es), _pitch(K, es),
                                      _pitch(N, es), _pitch(K, 2))
        self._desc = ctypes.byref(self.desc)
        self.workspace = torch.empty(flexmoe_grouped_workspace_bytes(self.desc, max_rows), dtype=torch.uint8, device=device)
        self._ws = (self.workspace.data_ptr(), self.workspace.numel())
        self._lock = threading.Lock()  # holds the descriptor's strides: the library's calls run without the interpreter's lock

    def _groups(self, offsets, keep):
        return (_vector(offsets, self.groups + 1, self._i32, "offsets"),
                None if keep is None else _vector(keep, self.groups, self._i32, "keep"))

    def forward(self, x, w, offsets, keep=None, y=None, stream=None):
        """y_r = x_r W_e^T for x [R, K], w [groups, N, K]."""
        R, d, dt = x.shape[0], self.desc, self.dtype
        if y is None:
            y = _padded((R, self.N), dt, x.device, stream)
        with self._lock:
            d.ldx, d.ldw = _matrix(x, (R, self.K), dt, "x"), _matrix(w, self._w_shape, dt, "w")
            d.ldy = _matrix(y, (R, self.N), dt, "y")
            _check(lib().flexmoe_grouped_forward(self._desc, R, x.data_ptr(), w.data_ptr(), *self._groups(offsets, keep),
                                                 y.data_ptr(), *self._ws, _stream(stream)))
        return y

    def input_grad(self, dy, w, offsets, keep=None, dx=None, stream=None):
        """dx_r = dy_r W_e for dy [R, N]."""
        R, d, dt = dy.shape[0], self.desc, self.dtype
        if dx is None:
            dx = _padded((R, self.K), dt, dy.device, stream)
        with self._lock:
            d.ldy, d.ldw = _matrix(dy, (R, self.N), dt, "dy"), _matrix(w, self._w_shape, dt, "w")
            d.ldx = _matrix(dx, (R, self.K), dt, "dx")
            _check(lib().flexmoe_grouped_input_grad(self._desc, R, dy.data_ptr(), w.data_ptr(), *self._groups(offsets, keep),
                                                    dx.data_ptr(), *self._ws, _stream(stream)))
        return dx

    def weight_grad(self, dy, x, offsets, keep=None, dw=None, accumulate=False, dw_dtype=None, stream=None):
        """dW_e = dy^T x over e's rows, written to (or with accumulate added to) dw [groups, N, K]."""
        R, d, dt = dy.shape[0], self.desc, self.dtype
        if dw is None:
            if accumulate:
                raise ValueError("accumulate needs dw")
            dw = _padded(self._w_shape, self._f32 if dw_dtype is None else dw_dtype, dy.device, stream)
        elif dw_dtype is not None and dw.dtype != dw_dtype:
            raise ValueError("dw is %s, not %s" % (dw.dtype, dw_dtype))
        with self._lock:
            d.dw_dtype = _dtype_code(dw.dtype)
            d.ldy, d.ldx = _matrix(dy, (R, self.N), dt, "dy"), _matrix(x, (R, self.K), dt, "x")
            d.lddw = _matrix(dw, self._w_shape, dw.dtype, "dw")
            _check(lib().flexmoe_grouped_weight_grad(self._desc, R, dy.data_ptr(), x.data_ptr(), *self._groups(offsets, keep),
                                                     dw.data_ptr(), int(accumulate), *self._ws, _stream(stream)))
        return dw


def quantize_rows(x, gate=None, q=None, scale=None, stream=None):
    """Rows of x [..., rows, cols] (or silu(gate) * x) as whole numbers up to 127 and a scale each: (q int8 like x, scale)."""
    import torch
    shape = x.shape
    if len(shape) < 2:
        raise ValueError("x must have rows and columns, got %s" % (tuple(shape),))
    cols = shape[-1]
    rows = shape[0] if len(shape) == 2 else math.prod(shape[:-1])
    ldx = _matrix(x, shape, x.dtype, "x")
    if gate is not None and _matrix(gate, shape, x.dtype, "gate") != ldx:
        raise ValueError("x and gate must have the same strides")
    if q is None:
        q = _padded(shape, torch.int8, x.device, stream)
    if scale is None:
        scale = _new(shape[:-1], torch.float32, x.device, stream)
    _check(lib().flexmoe_quantize_rows(rows, cols, _dtype_code(x.dtype), x.data_ptr(), None if gate is None else gate.data_ptr(), ldx,
                                       q.data_ptr(), _matrix(q, shape, torch.int8, "q"), _vector(scale, rows, torch.float32, "scale"),
                                       _stream(stream)))
    return q, scale


class Int8Product:
    """8-bit experts (one group: a plain matrix): y_r = x_r W_e^T with W_e in whole numbers and a scale per channel.

    w [groups, N, K] int8 and w_scale [groups, N] (quantize_rows of the weights).  Calling it rounds the rows of x and
    multiplies; `product` takes rows that are rounded already.  It keeps the workspace and the rounded rows' buffers for
    up to max_rows rows: calls on different streams need holders of their own; threads may share one.
    """

    def __init__(self, w, w_scale, max_rows, keep_axis="none", out_dtype=None):
        import torch
        self.groups, self.N, self.K = w.shape
        self.w, self.w_scale, self.max_rows = w, w_scale, max_rows
        self._i8, self._i32, self._f32 = torch.int8, torch.int32, torch.float32
        _vector(w_scale, self.groups * self.N, torch.float32, "w_scale")
        self.out_dtype = torch.bfloat16 if out_dtype is None else out_dtype
        self.desc = make_grouped_desc(self.groups, self.N, self.K, _dtype_code(self.out_dtype), FLEXMOE_F32, keep_axis, max_rows,
                                      _pitch(self.K, 1), _matrix(w, w.shape, torch.int8, "w"), _pitch(self.N, self.out_dtype.itemsize))
        self._desc = ctypes.byref(self.desc)
        self.workspace = torch.empty(flexmoe_quantized_workspace_bytes(self.desc, max_rows), dtype=torch.uint8, device=w.device)
        self._ws = (self.workspace.data_ptr(), self.workspace.numel())
        self.q = _padded((max_rows, self.K), torch.int8, w.device)
        self.q_scale = torch.empty(max_rows, dtype=torch.float32, device=w.device)
        self._lock = threading.Lock()  # holds the descriptor's strides, and q from its rounding to the product's launch
        # all rows of any call, for one group: the kernels cut offsets to [0, R]
        self._all_rows = torch.tensor([0, 2 ** 31 - 1], dtype=torch.int32, device=w.device) if self.groups == 1 else None

    @classmethod
    def from_weights(cls, w, max_rows, keep_axis="none", out_dtype=None):
        """From bf16 or fp32 weights [groups, N, K]."""
        return cls(*quantize_rows(w), max_rows, keep_axis, out_dtype)

    def __call__(self, x, offsets=None, keep=None, gate=None, y=None, stream=None):
        """x [R, K] bf16 or fp32 (with gate: silu(gate) * x); offsets may be left out for one group.

        A row's scale is that of its whole length: with keep_axis "K" what lies past a width should be zeros, as the
        products write it.
        """
        R = x.shape[0]
        if x.shape != (R, self.K) or R > self.max_rows:
            raise ValueError("x must be [R, %d] with at most %d rows, got %s" % (self.K, self.max_rows, tuple(x.shape)))
        ldx = _matrix(x, x.shape, x.dtype, "x")
        if gate is not None and _matrix(gate, x.shape, x.dtype, "gate") != ldx:
            raise ValueError("x and gate must have the same strides")
        q, scale, d = self.q.data_ptr(), self.q_scale.data_ptr(), self.desc
        ldq = self.q.stride(0) if self.max_rows > 1 else _pitch(self.K, 1)
        with self._lock:
            _check(lib().flexmoe_quantize_rows(R, self.K, _dtype_code(x.dtype), x.data_ptr(), None if gate is None else gate.data_ptr(), ldx,
                                               q, ldq, scale, _stream(stream)))
            d.ldx = ldq
            return self._product(R, q, scale, offsets, keep, y, x.device, stream)

    def product(self, q, q_scale, offsets=None, keep=None, y=None, stream=None):
        R = q.shape[0]
        with self._lock:
            self.desc.ldx = _matrix(q, (R, self.K), self._i8, "q")
            return self._product(R, q.data_ptr(), _vector(q_scale, R, self._f32, "q_scale"), offsets, keep, y, q.device, stream)

    def _product(self, R, q, q_scale, offsets, keep, y, device, stream):
        if offsets is None:
            if self.groups != 1:
                raise ValueError("offsets are needed for %d groups" % self.groups)
            offsets = self._all_rows.data_ptr()
        else:
            offsets = _vector(offsets, self.groups + 1, self._i32, "offsets")
        if y is None:
            y = _padded((R, self.N), self.out_dtype, device, stream)
        self.desc.ldy = _matrix(y, (R, self.N), self.out_dtype, "y")
        _check(lib().flexmoe_quantized_forward(self._desc, R, q, q_scale, self.w.data_ptr(), self.w_scale.data_ptr(), offsets,
                                               None if keep is None else _vector(keep, self.groups, self._i32, "keep"),
                                               y.data_ptr(), *self._ws, _stream(stream)))
        return y


class AdamW:
    """AdamW over a list of contiguous tensors, states in 32 or in 8 bits (one launch per 56 tensors).

    params: bf16 or fp32, all alike.  masters: fp32 copies that the step works on (bf16 parameters).  states: (m, v) or,
    with 8 bits, (m, v, m_scale, v_scale) lists to continue from; zeros otherwise.  step(grads) takes one gradient per
    parameter.  Every step reads the tensors' addresses again: their storages may be replaced between steps.

    In a graph: addresses, lr and the step's number are fixed by the capture, so that every replay is the same step again,
    its bias corrections and (8 bits) its random bits.  With device_step the number is counted on the device instead
    (clock[0], the steps done; t stays what it was): every call and every replay is the next step.
    """

    def __init__(self, params, masters=None, states=None, state_bits=32, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0,
                 step=0, seed=0, device_step=False):
        import torch
        self.params, self.state_bits = list(params), state_bits
        self.betas, self.eps, self.weight_decay, self.t, self.seed = betas, eps, weight_decay, step, seed
        if not self.params:
            raise ValueError("no parameters")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32, got %s" % (state_bits,))
        # a flexmoe_adamw_clock
        self.clock = torch.tensor([step, 0, 0], dtype=torch.int64, device=self.params[0].device) if device_step else None
        dt = self.params[0].dtype
        sizes = [p.numel() for p in self.params]
        blocks = [-(-n // STATE_BLOCK) for n in sizes]
        st = torch.uint8 if state_bits == 8 else torch.float32
        if states is None:
            def zeros(n, dtype):
                return torch.zeros(n, dtype=dtype, device=self.params[0].device)

            states = ([zeros(n, st) for n in sizes], [zeros(n, st) for n in sizes])
            if state_bits == 8:
                states += ([zeros(n, torch.float32) for n in blocks], [zeros(n, torch.float32) for n in blocks])
        self.m, self.v = (self._list(t) for t in states[:2])
        self.m_scale, self.v_scale = (self._list(t) for t in states[2:]) if state_bits == 8 else (None, None)
        self.masters = None if masters is None else self._list(masters)
        self.sizes, self._param_code = sizes, _dtype_code(dt)
        self._table = (flexmoe_adamw_tensor * len(sizes))()
        self._table_at = ctypes.addressof(self._table)
        self._lock = threading.Lock()  # holds the table and t
        self._n, self._blocks = np.array(sizes, dtype=np.int64), np.array(blocks, dtype=np.int64)
        np.frombuffer(self._table, dtype=np.int64)[flexmoe_adamw_tensor.n.offset // 8::_TENSOR_BYTES // 8] = self._n
        # the table's columns, filled by every step, since a tensor's storage may have been replaced since the last one
        # (p.data = ..., module.to()): states and masters may hold more values than the parameter
        kept = [("param", self.params, self._n, dt, 0), ("m", self.m, self._n, st, 1), ("v", self.v, self._n, st, 1)]
        if state_bits == 8:
            kept += [("m_scale", self.m_scale, self._blocks, torch.float32, 1), ("v_scale", self.v_scale, self._blocks, torch.float32, 1)]
        if masters is not None:
            kept.append(("master", self.masters, self._n, torch.float32, 1))
        self._fields = [(name, n) for name, _, n, _, _ in kept] + [("gradient", self._n)]
        self._columns = tuple((ts, n.ctypes.data, 2 if t == torch.uint8 else _dtype_code(t), self._at(name), longer)
                              for name, ts, n, t, longer in kept)
        self._sizes_at, self._grad_at = self._n.ctypes.data, self._at("grad")
        bad = tensors().columns(self._columns, len(sizes), _TENSOR_BYTES)
        if bad >= 0:
            self._refuse(self._columns, bad)

    @staticmethod
    def _list(tensors_):
        return tensors_ if type(tensors_) is list else list(tensors_)

    def _at(self, field):
        return self._table_at + getattr(flexmoe_adamw_tensor, field).offset

    def _refuse(self, columns, bad):
        c, i = divmod(bad, len(self.sizes) + 1)
        (name, n), (ts, _, code, _, _) = self._fields[c], columns[c]
        if i == len(self.sizes):
            raise ValueError("%s: %d tensors for %d parameters" % (name, len(ts), i))
        raise ValueError("%s %d: need %d contiguous %s values on the GPU, got %s %s"
                         % (name, i, n[i], ("float32", "bfloat16", "uint8")[code], getattr(ts[i], "dtype", type(ts[i])),
                            tuple(getattr(ts[i], "shape", ()))))

    def step(self, grads, lr, grad_scale=1.0, stream=None):
        """One step with the gradients `grads` (bf16 or fp32, all alike, contiguous)."""
        grads = grads if type(grads) is list else list(grads)
        if len(grads) != len(self.sizes):
            raise ValueError("%d gradients for %d parameters" % (len(grads), len(self.sizes)))
        code = _dtype_code(grads[0].dtype)
        with self._lock:
            columns = (*self._columns, (grads, self._sizes_at, code, self._grad_at, 0))
            bad = tensors().columns(columns, len(grads), _TENSOR_BYTES)
            if bad >= 0:
                self._refuse(columns, bad)
            d = flexmoe_adamw_desc(self._param_code, code, self.state_bits, self.seed & 0xffffffff, self.t + 1, lr,
                                   self.betas[0], self.betas[1], self.eps, self.weight_decay, grad_scale)
            if self.clock is not None:
                d.clock = self.clock.data_ptr()
            elif _capturing():
                warnings.warn("the captured AdamW step repeats itself on every replay; AdamW(..., device_step=True) counts steps on the device",
                              stacklevel=2)
            _check(lib().flexmoe_adamw_step(ctypes.byref(d), self._table_at, len(self.sizes), _stream(stream)))
            if self.clock is None:
                self.t += 1


def adamw_state_values(m, v, m_scale, v_scale, dtype=None, stream=None):
    """What 8-bit states stand for: (m, v) as fp32 or bf16."""
    import torch
    dtype = torch.float32 if dtype is None else dtype
    mo, vo = (_new(m.numel(), dtype, m.device, stream) for _ in range(2))
    blocks = -(-m.numel() // STATE_BLOCK)
    flexmoe_adamw_read_state(m.numel(), _vector(m, m.numel(), torch.uint8, "m"), _vector(v, m.numel(), torch.uint8, "v"),
                             _vector(m_scale, blocks, torch.float32, "m_scale"), _vector(v_scale, blocks, torch.float32, "v_scale"),
                             _dtype_code(dtype), mo, vo, stream)
    return mo, vo


class ClippedWeights:
    """The packed weights of one exported budget (offline clipping) and its
    device keep table."""

    def __init__(self, keep_host, w_gate_c, w_up_c, w_down_c, packed_channels, keep_dev):
        self.keep_host = np.asarray(keep_host, dtype=np.int32).copy()
        self.w_gate_c, self.w_up_c, self.w_down_c = w_gate_c, w_up_c, w_down_c
        self.packed_channels = packed_channels
        self.keep_dev = keep_dev


def _packed(t, n, name):
    """The layer's calls take addresses alone: t must hold n values one after another (an expanded gradient holds fewer)."""
    if t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be %d contiguous values, got %s with strides %s" % (name, n, tuple(t.shape), t.stride()))


class Layer:
    """Device-resident masked MoE layer: weights, keep table, workspace.

    A thin holder around the C calls (no arithmetic): it allocates torch
    buffers once and forwards with the library.
    """

    def __init__(self, d, E, I, top_k, I_shared=0, dtype=FLEXMOE_BF16, norm_topk=1,
                 max_tokens=1, device="cuda"):
        import torch
        self.desc = make_desc(d, E, I, top_k, I_shared, dtype, norm_topk, max_tokens)
        self.tdtype = torch.bfloat16 if dtype == FLEXMOE_BF16 else torch.float32
        self.device = device
        self.keep = torch.full((E,), I, dtype=torch.int32, device=device)
        nbytes = flexmoe_workspace_bytes(self.desc, max_tokens)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.w_gate = self.w_up = self.w_down = None
        self.ws_gate = self.ws_up = self.ws_down = None

    def set_weights(self, w_gate, w_up, w_down, ws_gate=None, ws_up=None, ws_down=None):
        self.w_gate, self.w_up, self.w_down = w_gate, w_up, w_down
        self.ws_gate, self.ws_up, self.ws_down = ws_gate, ws_up, ws_down

    def set_budget(self, keep_host, stream=None):
        flexmoe_set_budget(self.desc, self.keep, keep_host, stream)

    def export_clipped(self, keep_host, stream=None) -> ClippedWeights:
        """Pack the current ranked weights for the budget keep_host."""
        import torch
        P = flexmoe_clipped_channels(self.desc, keep_host)
        bufs = [_new((max(P, 1) * self.desc.d,), self.tdtype, self.device, stream) for _ in range(3)]
        flexmoe_export_clipped(self.desc, keep_host, self.w_gate, self.w_up, self.w_down, *bufs,
                               stream=stream)
        keep_dev = torch.from_numpy(np.asarray(keep_host, dtype=np.int32).copy()).to(self.device)
        return ClippedWeights(keep_host, *bufs, P, keep_dev)

    def forward(self, x, logits, y=None, keep=None, dbg=None, stream=None, clipped=None,
                bucketed=None):
        """clipped: a ClippedWeights of this layer -> the offline-clipped path;
        bucketed: (keep_host, k_align) -> the bucketed ablation."""
        T = x.shape[0]
        if y is None:
            y = _new((T, self.desc.d), self.tdtype, self.device, stream)
        D = self.desc
        _packed(x, T * D.d, "x")
        _packed(logits, T * D.E, "logits")
        _packed(y, T * D.d, "y")
        if bucketed is not None:
            flexmoe_layer_forward_bucketed(self.desc, T, x, logits, self.w_gate, self.w_up, self.w_down,
                                           bucketed[0], bucketed[1], self.ws_gate, self.ws_up,
                                           self.ws_down, y, self.workspace, dbg=dbg, stream=stream)
            return y
        if clipped is not None:
            flexmoe_layer_forward_clipped(self.desc, T, x, logits, clipped.w_gate_c, clipped.w_up_c,
                                          clipped.w_down_c, clipped.keep_dev if keep is None else keep,
                                          clipped.packed_channels, self.ws_gate, self.ws_up,
                                          self.ws_down, y, self.workspace, dbg=dbg, stream=stream)
            return y
        flexmoe_layer_forward(self.desc, T, x, logits, self.w_gate, self.w_up, self.w_down,
                              self.keep if keep is None else keep, self.ws_gate, self.ws_up,
                              self.ws_down, y, self.workspace, dbg=dbg, stream=stream)
        return y


class Saliency:
    """Channel ranking on the device (Sec. 3.1): the running Eq. 2 scores of
    one layer over calibration batches, then the reorder of Eq. 3.

    Holds the score table and a saliency workspace for up to max_tokens
    tokens per batch; the weights are those of `layer` (original order).
    """

    def __init__(self, layer: "Layer", max_tokens: int, transpose_once: bool = True):
        import torch
        self.layer = layer
        D = layer.desc
        self.desc = make_desc(D.d, D.E, D.I, D.top_k, D.I_shared, D.dtype, D.norm_topk, max_tokens)
        nbytes = flexmoe_saliency_workspace_bytes(self.desc, max_tokens)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=layer.device)
        self.scores = torch.zeros((D.E, D.I), dtype=torch.float32, device=layer.device)
        self.w_down_t = None
        if transpose_once:   # W_down^T made once for the whole ranking set
            self.w_down_t = torch.empty((D.E, D.I, D.d), dtype=layer.tdtype, device=layer.device)
            flexmoe_transpose_weights(self.desc, None, None, layer.w_down, None, None, None,
                                      None, None, self.w_down_t, None, None, None)

    def add_batch(self, x, logits, y_target, scale=1.0, stream=None):
        L, T = self.layer, x.shape[0]
        _packed(x, T * self.desc.d, "x")
        _packed(logits, T * self.desc.E, "logits")
        _packed(y_target, T * self.desc.d, "y_target")
        flexmoe_channel_saliency(self.desc, T, x, logits, L.w_gate, L.w_up, L.w_down, self.w_down_t,
                                 L.ws_gate, L.ws_up, L.ws_down, y_target, scale, self.scores, self.workspace,
                                 stream=stream)

    def rank_reorder(self, stream=None):
        """Ranked copies of the layer's weights and the permutation (Eq. 3)."""
        import torch
        L = self.layer
        out = [_new(w.shape, w.dtype, w.device, stream) for w in (L.w_gate, L.w_up, L.w_down)]
        perm = _new((L.desc.E, L.desc.I), torch.int32, L.device, stream)
        flexmoe_rank_reorder(L.desc, self.scores, L.w_gate, L.w_up, L.w_down, *out, perm, stream=stream)
        return (*out, perm)


class ActionLearner:
    """One layer's action-learning step on the device (Sec. 3.2): sample the
    per-expert widths (Eq. 5), run the sampled subnet forward, backward for
    an upstream gradient, and the action-logit gradient (Eqs. 6-8).

    Holds the transposed weight copies (made once: the weights are frozen),
    the sampled keep table and a training workspace for up to max_tokens.
    """

    def __init__(self, layer: "Layer", max_tokens: int, ratios):
        import torch
        self.layer = layer
        D = layer.desc
        self.desc = make_desc(D.d, D.E, D.I, D.top_k, D.I_shared, D.dtype, D.norm_topk, max_tokens)
        self.actions = make_actions(ratios)
        dev = layer.device
        nbytes = flexmoe_train_workspace_bytes(self.desc, max_tokens)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        bf = layer.tdtype
        self.wt = [torch.empty((D.E, D.d, D.I), dtype=bf, device=dev),
                   torch.empty((D.E, D.d, D.I), dtype=bf, device=dev),
                   torch.empty((D.E, D.I, D.d), dtype=bf, device=dev)]
        if D.I_shared:
            self.wst = [torch.empty((D.d, D.I_shared), dtype=bf, device=dev),
                        torch.empty((D.d, D.I_shared), dtype=bf, device=dev),
                        torch.empty((D.I_shared, D.d), dtype=bf, device=dev)]
        else:
            self.wst = [None, None, None]
        self.keep = torch.zeros((D.E,), dtype=torch.int32, device=dev)
        self.action = torch.zeros((D.E,), dtype=torch.int32, device=dev)
        self.T = 0

    def transpose_weights(self, stream=None):
        L = self.layer
        flexmoe_transpose_weights(self.desc, L.w_gate, L.w_up, L.w_down, L.ws_gate, L.ws_up, L.ws_down,
                                  *self.wt, *self.wst, stream=stream)

    def sample(self, alpha, gumbel, stream=None):
        _packed(alpha, self.desc.E * self.actions.K, "alpha")
        _packed(gumbel, self.desc.E * self.actions.K, "gumbel")
        flexmoe_sample_actions(self.desc, self.actions, alpha, gumbel, self.keep, self.action, stream=stream)

    def forward(self, x, logits, y=None, keep=None, stream=None):
        L = self.layer
        self.T = x.shape[0]
        if y is None:
            y = _new((self.T, self.desc.d), L.tdtype, L.device, stream)
        _packed(x, self.T * self.desc.d, "x")
        _packed(logits, self.T * self.desc.E, "logits")
        _packed(y, self.T * self.desc.d, "y")
        flexmoe_train_forward(self.desc, self.T, x, logits, L.w_gate, L.w_up, L.w_down,
                              self.keep if keep is None else keep, L.ws_gate, L.ws_up, L.ws_down, y,
                              self.workspace, stream=stream)
        return y

    def backward(self, logits, dy, stream=None):
        import torch
        D, dev = self.desc, self.layer.device
        _packed(logits, self.T * D.E, "logits")
        _packed(dy, self.T * D.d, "dy")
        dx, dl, dm = (_new(shape, torch.float32, dev, stream) for shape in ((self.T, D.d), (self.T, D.E), (D.E, D.I)))
        flexmoe_train_backward(D, self.T, logits, dy, *self.wt, *self.wst, dx, dl, dm, self.workspace,
                               stream=stream)
        return dx, dl, dm

    def action_grad(self, alpha, gumbel, tau, lambda_cost, beta, dmask, stream=None):
        import torch
        _packed(alpha, self.desc.E * self.actions.K, "alpha")
        _packed(gumbel, self.desc.E * self.actions.K, "gumbel")
        _packed(dmask, self.desc.E * self.desc.I, "dmask")
        dalpha = _new(alpha.shape, alpha.dtype, alpha.device, stream)
        stats = _new((2,), torch.float32, alpha.device, stream)
        flexmoe_action_grad(self.desc, self.T, self.actions, alpha, gumbel, tau, lambda_cost, beta, dmask, dalpha,
                            stats, self.workspace, stream=stream)
        return dalpha, stats


def to_device(a: np.ndarray, device="cuda"):
    """NumPy array (fp32, int32, or uint16 bf16 bits) -> torch CUDA tensor."""
    import torch
    if a.dtype == np.uint16:
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(a)).to(device)


def to_host(t) -> np.ndarray:
    """torch tensor -> NumPy (bf16 becomes uint16 bits)."""
    import torch
    t = t.detach().cpu()
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).numpy().view(np.uint16)
    return t.numpy()
