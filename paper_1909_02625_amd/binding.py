"""ctypes binding of libdsp_hip.so: same names as the C ABI, argument marshalling only.

PyTorch appears here solely as the owner of device memory and streams (``tensor.data_ptr()``,
``torch.cuda.current_stream().cuda_stream``); no arithmetic of the method runs in Python.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

__all__ = [
    "DSP_FP32", "DSP_BF16", "DSPError", "lib", "lib_path", "check",
    "dsp_layer_desc", "dsp_block_desc", "make_block_desc",
    "DSP_NORM_NONE", "DSP_NORM_RMS", "DSP_NORM_LAYER", "DSP_GATE_IDENTITY", "DSP_GATE_SIGMOID", "DSP_GATE_TANH",
    "dsp_adamw_tensor", "dsp_adamw_init", "dsp_adamw_destroy", "dsp_adamw_step", "dsp_adamw_get_steps", "dsp_adamw_set_steps",
    "dsp_block_set_adamw", "dsp_param_update_adamw", "dsp_block_adamw_state_bytes", "dsp_block_get_adamw_state",
    "dsp_block_set_adamw_state", "dsp_pipeline_set_adamw",
    "dsp_norm_residual_desc", "make_norm_residual_desc", "dsp_norm_residual_forward", "dsp_norm_residual_workspace_bytes",
    "dsp_norm_residual_backward",
    "DSP_ACT_IDENTITY", "DSP_ACT_RELU", "DSP_ACT_GELU", "DSP_ACT_SILU", "DSP_DECAY_SIGMOID", "DSP_DECAY_EXP",
    "dsp_dense_desc", "make_dense_desc", "dsp_dense_workspace_bytes", "dsp_dense_forward", "dsp_dense_backward",
    "dsp_recurrence_desc", "make_recurrence_desc", "dsp_recurrence_workspace_bytes", "dsp_recurrence_forward", "dsp_recurrence_backward",
    "dsp_policy_loss_desc", "make_policy_loss_desc", "dsp_token_logprob", "dsp_policy_loss",
    "dsp_schedule_validate", "dsp_schedule_index", "dsp_schedule_queue_elems", "dsp_schedule_waits",
    "dsp_block_init", "dsp_block_destroy", "dsp_block_forward", "dsp_block_recompute_backward",
    "dsp_param_update", "dsp_param_update_sum", "dsp_pipeline_set_optimizer", "dsp_block_input_slot",
    "dsp_pipeline_attach_gradient_probe", "dsp_pipeline_gradient_difference", "dsp_block_query", "dsp_block_output_shape",
    "dsp_block_input_shape", "dsp_block_memory", "dsp_block_get_params", "dsp_block_set_params",
    "dsp_block_get_momentum", "dsp_block_set_momentum", "dsp_block_get_grads",
    "dsp_pipeline_init", "dsp_pipeline_destroy", "dsp_pipeline_step", "dsp_pipeline_set_delay",
    "dsp_pipeline_set_graph_replay", "dsp_pipeline_set_launch_threads", "dsp_pipeline_set_single_stream", "dsp_pipeline_set_forward_streams",
    "dsp_block_enable_forward_lane", "dsp_block_step", "dsp_pipeline_set_twin_launches",
    "dsp_pipeline_sync", "dsp_pipeline_losses", "dsp_pipeline_ticks",
    "dsp_conv_forward", "dsp_conv_backward_data", "dsp_conv_backward_weight", "dsp_conv_workspace_bytes",
    "dsp_grouped_conv_forward", "dsp_grouped_conv_backward_data", "dsp_grouped_conv_backward_weight",
    "dsp_grouped_conv_workspace_bytes",
    "dsp_conv_backward_weight_static", "dsp_conv_backward_weight_static_bytes",
    "dsp_bn_workspace_bytes", "dsp_bn_forward", "dsp_bn_backward", "dsp_bn_relu_maxpool_forward", "dsp_bn_relu_backward_from_x", "dsp_bn_relu_maxpool_backward", "dsp_bn_relu_bits_bytes", "dsp_bn_forward_bits",
    "dsp_bn_backward_bits", "dsp_maxpool_forward", "dsp_maxpool_backward",
    "dsp_add_forward", "dsp_add_backward", "dsp_gap_forward", "dsp_gap_backward", "dsp_linear_forward",
    "dsp_linear_backward", "dsp_softmax_ce", "dsp_block_get_activation", "dsp_block_get_pool_argmax",
    "dsp_profile_start", "dsp_profile_stop", "dsp_profile_get",
    "dsp_strerror", "dsp_last_error", "dsp_build_id", "EXPORTED_SYMBOLS",
]

DSP_FP32, DSP_BF16 = 0, 1
DSP_NORM_NONE, DSP_NORM_RMS, DSP_NORM_LAYER = 0, 1, 2
DSP_GATE_IDENTITY, DSP_GATE_SIGMOID, DSP_GATE_TANH = 0, 1, 2
DSP_ACT_IDENTITY, DSP_ACT_RELU, DSP_ACT_GELU, DSP_ACT_SILU = 0, 1, 2, 3
DSP_DECAY_SIGMOID, DSP_DECAY_EXP = 0, 1
_OPS = {"conv": 0, "bn": 1, "maxpool": 2, "gap": 3, "linear": 4, "softmax_ce": 5, "add": 6}

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None


class DSPError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = lib().dsp_last_error().decode()
        super().__init__("%s: %s%s" % (where, lib().dsp_strerror(status).decode(), (" -- " + msg) if msg else ""))


class dsp_layer_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("op", "in0", "in1", "cin", "cout", "r", "s", "stride", "pad", "relu", "groups")]


class dsp_block_desc(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("layers", C.POINTER(dsp_layer_desc)),
                ("N", C.c_int32), ("C", C.c_int32), ("H", C.c_int32), ("W", C.c_int32),
                ("dtype", C.c_int32), ("k", C.c_int32), ("K", C.c_int32), ("m_k", C.c_int32),
                ("p_prev", C.c_int32), ("needs_input_grad", C.c_int32), ("bn_eps", C.c_float)]


class dsp_adamw_tensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("d_param", "d_grad", "d_copy", "d_m", "d_v", "d_m_exp", "d_v_exp")] + \
               [("n", C.c_int64), ("grad_dtype", C.c_int32), ("decay", C.c_int32)]


class dsp_norm_residual_desc(C.Structure):
    _fields_ = [("M", C.c_int64)] + [(n, C.c_int32) for n in ("C", "dtype", "post", "pre", "gate_act", "gate_dtype")] + \
               [("gate_rows", C.c_int64)] + [(n, C.c_float) for n in ("alpha", "beta", "eps")] + \
               [(n, C.c_int64) for n in ("x_stride", "z_stride", "y_stride", "h_stride", "gate_stride")]


class dsp_dense_desc(C.Structure):
    _fields_ = [("M", C.c_int64)] + [(n, C.c_int32) for n in ("cin", "cout", "dtype", "act")] + \
               [(n, C.c_int64) for n in ("x_stride", "y_stride")]


class dsp_recurrence_desc(C.Structure):
    _fields_ = [("rows", C.c_int64)] + [(n, C.c_int32) for n in ("sequences", "steps", "C", "dtype", "decay", "coupled")] + \
               [(n, C.c_int64) for n in ("x_stride", "f_stride", "h_stride")]


class dsp_policy_loss_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "vocab", "dtype")] + \
               [(n, C.c_float) for n in ("clip_low", "clip_high", "kl_coef", "entropy_coef", "temperature")] + \
               [(n, C.c_int64) for n in ("logits_stride", "grad_stride")]


def lib_path():
    return os.path.join(_HERE, "libdsp_hip.so")


def lib():
    """Loads the built library (building it first only if no binary exists at all)."""
    global _LIB
    if _LIB is None:
        # PyTorch owns the device memory and streams handed to the library, so both must talk to ONE
        # HIP runtime: importing torch first makes the loader bind libamdhip64.so.7 to the copy torch
        # ships (two runtimes in a process do not see each other's devices or allocations).
        import torch  # noqa: F401
        path = lib_path()
        if not os.path.exists(path):
            from . import build as _build
            _build.build(force=True)
        _LIB = C.CDLL(path)
        _declare(_LIB)
        from . import build as _build
        have, want = _LIB.dsp_build_id().decode(), _build.source_hash()
        if have != want:
            _LIB = None
            raise RuntimeError("%s was built from other sources (id %s, csrc/ + include/dsp.h now hash to %s): rebuild it "
                               "with `python -m paper_1909_02625_amd.build`" % (path, have, want))
    return _LIB


_vp, _i32, _i64, _sz, _f = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
_pi32, _pi64, _pf = C.POINTER(C.c_int32), C.POINTER(C.c_int64), C.POINTER(C.c_float)

_SIGNATURES = {
    "dsp_schedule_validate": [_i32, _pi32, _pi32, _pi32],
    "dsp_schedule_index": [_i32, _pi32, _pi32, _i32, _i64, _pi64],
    "dsp_schedule_queue_elems": [_i32, _pi32, _pi32, _pi64, _pi64],
    "dsp_schedule_waits": [_i32, _pi32, _pi32, _pi32, _pi32, _pi32, _pi32],
    "dsp_block_init": [C.POINTER(dsp_block_desc), _pf, _sz, C.POINTER(_vp)],
    "dsp_block_destroy": [_vp],
    "dsp_block_forward": [_vp, _i64, _vp, _vp, _vp, _vp, _vp],
    "dsp_block_recompute_backward": [_vp, _i64, _vp, _vp, _vp],
    "dsp_param_update": [_vp, _f, _f, _f, _vp],
    "dsp_param_update_sum": [_vp, _f, _f, _i32, _f, _vp],
    "dsp_pipeline_set_optimizer": [_vp, _f, _f, _i32, _f],
    "dsp_pipeline_attach_gradient_probe": [_vp, _vp],
    "dsp_pipeline_gradient_difference": [_vp, C.POINTER(C.c_int64), C.POINTER(C.c_double), C.POINTER(C.c_double)],
    "dsp_block_input_slot": [_vp, _i64, C.POINTER(_vp)],
    "dsp_block_query": [_vp, _pi64],
    "dsp_block_output_shape": [_vp, _pi32],
    "dsp_block_input_shape": [_vp, _pi32],
    "dsp_block_memory": [_vp, C.POINTER(_sz), C.POINTER(_sz), C.POINTER(_sz)],
    "dsp_block_get_params": [_vp, _pf, _sz],
    "dsp_block_set_params": [_vp, _pf, _sz],
    "dsp_block_get_momentum": [_vp, _pf, _sz],
    "dsp_block_set_momentum": [_vp, _pf, _sz],
    "dsp_block_get_grads": [_vp, _pf, _sz],
    "dsp_pipeline_init": [_i32, C.POINTER(_vp), _pi32, _pi32, _f, _f, _f, _i64, C.POINTER(_vp)],
    "dsp_pipeline_destroy": [_vp],
    "dsp_pipeline_step": [_vp, _vp, _vp, _pf, _pi64, _vp],
    "dsp_pipeline_set_delay": [_vp, _i32, _i32],
    "dsp_pipeline_set_graph_replay": [_vp, _i32],
    "dsp_pipeline_set_launch_threads": [_vp, _i32],
    "dsp_pipeline_set_single_stream": [_vp, _i32],
    "dsp_pipeline_set_forward_streams": [_vp, _i32],
    "dsp_block_enable_forward_lane": [_vp],
    "dsp_pipeline_set_twin_launches": [_vp, _i32],
    "dsp_block_step": [_vp, _i64, _vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp],
    "dsp_pipeline_sync": [_vp],
    "dsp_pipeline_losses": [_vp, _pf, _i64, _pi64],
    "dsp_pipeline_ticks": [_vp, _pi64],
    "dsp_conv_forward": [_i32, _vp, _vp, _vp] + [_i32] * 9 + [_vp],
    "dsp_conv_backward_data": [_i32, _vp, _vp, _vp] + [_i32] * 10 + [_vp],
    "dsp_conv_backward_weight": [_i32, _vp, _vp, _vp] + [_i32] * 9 + [_vp, _sz, _vp],
    "dsp_conv_workspace_bytes": [_i32] * 9 + [C.POINTER(_sz)],
    "dsp_grouped_conv_forward": [_i32, _vp, _vp, _vp] + [_i32] * 10 + [_vp],
    "dsp_grouped_conv_backward_data": [_i32, _vp, _vp, _vp] + [_i32] * 11 + [_vp],
    "dsp_grouped_conv_backward_weight": [_i32, _vp, _vp, _vp] + [_i32] * 10 + [_vp, _sz, _vp],
    "dsp_grouped_conv_workspace_bytes": [_i32] * 10 + [C.POINTER(_sz)],
    "dsp_conv_backward_weight_static": [_i32, _vp, _vp, _vp] + [_i32] * 9 + [_vp],
    "dsp_bn_workspace_bytes": [_i32, C.POINTER(_sz)],
    "dsp_bn_forward": [_i32, _vp, _vp, _vp, _vp, _vp, _f, _i64, _i32, _i32, _vp, _vp, _vp, _sz, _vp],
    "dsp_bn_backward": [_i32, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _vp, _sz, _vp],
    "dsp_bn_relu_maxpool_forward": [_i32, _vp, _vp, _vp, _f] + [_i32] * 7 + [_vp] * 6 + [_sz, _vp],
    "dsp_bn_relu_backward_from_x": [_i32, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _i64, _i32, _vp, _sz, _vp],
    "dsp_bn_relu_maxpool_backward": [_i32, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp] + [_i32] * 7 + [_vp, _sz, _vp],
    "dsp_bn_relu_bits_bytes": [_i32, _i64, _i32, C.POINTER(C.c_size_t)],
    "dsp_bn_forward_bits": [_i32, _vp, _vp, _vp, _vp, _vp, _f, _i64, _i32, _vp, _vp, _vp, _vp, _sz, _vp],
    "dsp_bn_backward_bits": [_i32, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _i64, _i32, _vp, _sz, _vp],
    "dsp_maxpool_forward": [_i32, _vp, _vp, _vp] + [_i32] * 7 + [_vp],
    "dsp_maxpool_backward": [_i32, _vp, _vp, _vp] + [_i32] * 8 + [_vp],
    "dsp_add_forward": [_i32, _vp, _vp, _vp, _i64, _vp],
    "dsp_add_backward": [_i32, _vp, _vp, _i32, _vp, _i32, _i64, _vp],
    "dsp_gap_forward": [_i32, _vp, _vp, _i32, _i32, _i32, _vp],
    "dsp_gap_backward": [_i32, _vp, _vp, _i32, _i32, _i32, _i32, _vp],
    "dsp_linear_forward": [_vp, _vp, _vp, _vp, _i32, _i32, _i32, _vp],
    "dsp_linear_backward": [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _vp],
    "dsp_softmax_ce": [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _vp],
    "dsp_adamw_init": [_i32, C.POINTER(dsp_adamw_tensor), _i32, C.c_uint64, C.POINTER(_vp)],
    "dsp_adamw_destroy": [_vp],
    "dsp_adamw_step": [_vp] + [C.c_double] * 6 + [_vp, _vp],
    "dsp_adamw_get_steps": [_vp, _pi64],
    "dsp_adamw_set_steps": [_vp, _i64, C.c_double, C.c_double],
    "dsp_block_set_adamw": [_vp, _i32, C.c_uint64],
    "dsp_param_update_adamw": [_vp] + [C.c_double] * 6 + [_vp],
    "dsp_block_adamw_state_bytes": [_vp, C.POINTER(_sz)],
    "dsp_block_get_adamw_state": [_vp, _vp, _sz],
    "dsp_block_set_adamw_state": [_vp, _vp, _sz],
    "dsp_pipeline_set_adamw": [_vp] + [C.c_double] * 6,
    "dsp_norm_residual_forward": [C.POINTER(dsp_norm_residual_desc)] + [_vp] * 12,
    "dsp_norm_residual_workspace_bytes": [C.POINTER(dsp_norm_residual_desc), C.POINTER(_sz)],
    "dsp_norm_residual_backward": [C.POINTER(dsp_norm_residual_desc)] + [_vp] * 18 + [_sz, _vp],
    "dsp_dense_workspace_bytes": [C.POINTER(dsp_dense_desc), _i32, C.POINTER(_sz)],
    "dsp_dense_forward": [C.POINTER(dsp_dense_desc)] + [_vp] * 7 + [_sz, _vp],
    "dsp_dense_backward": [C.POINTER(dsp_dense_desc)] + [_vp] * 8 + [_sz, _vp],
    "dsp_recurrence_workspace_bytes": [C.POINTER(dsp_recurrence_desc), C.POINTER(_sz)],
    "dsp_recurrence_forward": [C.POINTER(dsp_recurrence_desc)] + [_vp] * 7 + [_sz, _vp],
    "dsp_recurrence_backward": [C.POINTER(dsp_recurrence_desc)] + [_vp] * 11 + [_sz, _vp],
    "dsp_token_logprob": [C.POINTER(dsp_policy_loss_desc)] + [_vp] * 5,
    "dsp_policy_loss": [C.POINTER(dsp_policy_loss_desc)] + [_vp] * 11,
    "dsp_block_get_activation": [_vp, _i32, _vp, _sz],
    "dsp_block_get_pool_argmax": [_vp, _i32, _vp, _sz],
    "dsp_conv_backward_weight_static_bytes": [C.POINTER(_sz)],
    "dsp_profile_start": [_i32],
    "dsp_profile_stop": [_pi32],
    "dsp_profile_get": [_i32, C.c_char_p, _sz, _pi64, C.POINTER(C.c_double), C.POINTER(C.c_double), _pi32],
}
EXPORTED_SYMBOLS = sorted(list(_SIGNATURES) + ["dsp_strerror", "dsp_last_error", "dsp_build_id"])


def _declare(L):
    for name, args in _SIGNATURES.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = C.c_int
    L.dsp_strerror.argtypes = [C.c_int]
    L.dsp_strerror.restype = C.c_char_p
    L.dsp_last_error.argtypes = []
    L.dsp_last_error.restype = C.c_char_p
    L.dsp_build_id.argtypes = []
    L.dsp_build_id.restype = C.c_char_p


def check(status, where):
    if status != 0:
        raise DSPError(status, where)


def _ptr(x):
    """Device/host address of a torch tensor, numpy array, int or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    return x.ctypes.data


def _stream(s):
    if s is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # 0.3 us; a Stream object costs 2.7
        return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())
    return s if isinstance(s, int) else s.cuda_stream


def _i32arr(v):
    return (C.c_int32 * len(v))(*[int(a) for a in v])


def make_block_desc(layers, in_shape, dtype, k, K, m_k, p_prev=0, needs_input_grad=True, bn_eps=1e-5):
    """Marshals a layer list (dicts, see workloads.configs) and an NCHW input shape into dsp_block_desc.
    Returns (desc, keepalive)."""
    arr = (dsp_layer_desc * len(layers))()
    for d, L in zip(arr, layers):
        d.op, d.in0, d.in1 = _OPS[L["op"]], L["in"], -2
        d.cin = L.get("cin", L.get("c", 0))
        d.cout = L.get("cout", 0)
        d.r, d.s = L.get("r", L.get("k", 0)), L.get("s", L.get("k", 0))
        d.stride, d.pad = L.get("stride", 1), L.get("pad", 0)
        d.relu = int(bool(L.get("relu", False)))
        d.groups = int(L.get("groups", 1))
        if L["op"] in ("bn", "add") and L.get("res") is not None:
            d.in1 = L["res"]
    n, c, h, w = in_shape
    desc = dsp_block_desc(len(layers), arr, n, c, h, w, dtype, k, K, m_k, p_prev, int(bool(needs_input_grad)), bn_eps)
    return desc, arr


# ---- schedule ------------------------------------------------------------------------------------
def dsp_schedule_validate(p, m):
    K = len(m)
    q = (C.c_int32 * K)()
    check(lib().dsp_schedule_validate(K, _i32arr(p), _i32arr(m), q), "dsp_schedule_validate")
    return list(q)


def dsp_schedule_index(p, m, k, tau):
    out = (C.c_int64 * 7)()
    check(lib().dsp_schedule_index(len(m), _i32arr(p), _i32arr(m), k, tau, out), "dsp_schedule_index")
    return dict(zip(("a", "b", "version", "slot_fwd", "slot_bwd", "q_write", "q_read"), list(out)))


def dsp_schedule_queue_elems(p, m, h_elems):
    tot = C.c_int64()
    arr = (C.c_int64 * len(h_elems))(*h_elems)
    check(lib().dsp_schedule_queue_elems(len(m), _i32arr(p), _i32arr(m), arr, C.byref(tot)), "dsp_schedule_queue_elems")
    return tot.value


def dsp_schedule_waits(p, m, spare=None):
    """Returns (wait_down[K], wait_up[K], label_slots)."""
    K = len(m)
    dn, up, lab = (C.c_int32 * K)(), (C.c_int32 * K)(), C.c_int32()
    check(lib().dsp_schedule_waits(K, _i32arr(p), _i32arr(m), None if spare is None else _i32arr(spare), dn, up,
                                   C.byref(lab)), "dsp_schedule_waits")
    return list(dn), list(up), lab.value


# ---- block -----------------------------------------------------------------------------------------
def dsp_block_init(desc, h_params):
    hp = np.ascontiguousarray(h_params, dtype=np.float32)
    out = C.c_void_p()
    check(lib().dsp_block_init(C.byref(desc), hp.ctypes.data_as(_pf), hp.size, C.byref(out)), "dsp_block_init")
    return out.value


def dsp_block_destroy(b):
    check(lib().dsp_block_destroy(b), "dsp_block_destroy")


def dsp_block_forward(b, batch_id, d_in, d_out=None, d_labels=None, d_loss=None, stream=None):
    check(lib().dsp_block_forward(b, batch_id, _ptr(d_in), _ptr(d_out), _ptr(d_labels), _ptr(d_loss), _stream(stream)),
          "dsp_block_forward")


def dsp_block_recompute_backward(b, batch_id, d_grad_out=None, d_grad_in=None, stream=None):
    check(lib().dsp_block_recompute_backward(b, batch_id, _ptr(d_grad_out), _ptr(d_grad_in), _stream(stream)),
          "dsp_block_recompute_backward")


def dsp_block_step(b, batch_fwd, d_in, d_out=None, d_labels=None, d_loss=None, batch_bwd=0, d_grad_out=None,
                   d_grad_in=None, stream=None):
    check(lib().dsp_block_step(b, batch_fwd, _ptr(d_in), _ptr(d_out), _ptr(d_labels), _ptr(d_loss), batch_bwd,
                               _ptr(d_grad_out), _ptr(d_grad_in), _stream(stream)), "dsp_block_step")


def dsp_param_update(b, lr, momentum, weight_decay=0.0, stream=None):
    check(lib().dsp_param_update(b, lr, momentum, weight_decay, _stream(stream)), "dsp_param_update")


def dsp_param_update_sum(b, lr, momentum, s=0, weight_decay=0.0, stream=None):
    check(lib().dsp_param_update_sum(b, lr, momentum, int(s), weight_decay, _stream(stream)), "dsp_param_update_sum")


def dsp_pipeline_set_optimizer(pl, lr, momentum, s=0, weight_decay=0.0):
    check(lib().dsp_pipeline_set_optimizer(pl, lr, momentum, int(s), weight_decay), "dsp_pipeline_set_optimizer")


def dsp_pipeline_attach_gradient_probe(pl, probe):
    check(lib().dsp_pipeline_attach_gradient_probe(pl, probe), "dsp_pipeline_attach_gradient_probe")


def dsp_pipeline_gradient_difference(pl, K):
    """(batch_id, diff_sumsq[K], bp_sumsq[K]) of the latest step; batch_id = -1 while there is none."""
    bid = C.c_int64(-1)
    diff, ref = (C.c_double * K)(), (C.c_double * K)()
    check(lib().dsp_pipeline_gradient_difference(pl, C.byref(bid), diff, ref), "dsp_pipeline_gradient_difference")
    return bid.value, np.array(diff[:], np.float64), np.array(ref[:], np.float64)


# ---- AdamW ---------------------------------------------------------------------------------------------
def dsp_adamw_init(tensors, state_bits=32, seed=0):
    """``tensors``: dicts of contiguous device tensors param (float32), grad (float32 or bfloat16), m, v (float32; with states of 8 bits
    uint8, or float8_e4m3fn and float8_e5m2) and, as they apply, copy (bfloat16), m_exp, v_exp (uint8 or float8_e8m0fnu); decay
    (default True).  They have to outlive the object."""
    import torch
    arr = (dsp_adamw_tensor * max(1, len(tensors)))()
    eight = state_bits == 8
    types = {"param": (torch.float32,), "grad": (torch.float32, torch.bfloat16), "copy": (torch.bfloat16,),
             "m": (torch.uint8, torch.float8_e4m3fn) if eight else (torch.float32,),
             "v": (torch.uint8, torch.float8_e5m2) if eight else (torch.float32,),
             "m_exp": (torch.uint8, torch.float8_e8m0fnu), "v_exp": (torch.uint8, torch.float8_e8m0fnu)}
    for a, t in zip(arr, tensors):
        n = t["param"].numel()
        for name, dtypes in types.items():
            x = t.get(name)
            count = -(-n // 256) if name.endswith("_exp") else n
            if x is not None and (x.dtype not in dtypes or x.numel() != count or not x.is_contiguous()):
                raise ValueError("dsp_adamw_init: %s: %d contiguous elements of %s are wanted" % (name, count, " or ".join(map(str, dtypes))))
            setattr(a, "d_" + name, _ptr(x))
        a.n, a.decay = n, int(bool(t.get("decay", True)))
        a.grad_dtype = DSP_BF16 if t["grad"].dtype == torch.bfloat16 else DSP_FP32
    out = C.c_void_p()
    check(lib().dsp_adamw_init(len(tensors), arr, state_bits, seed, C.byref(out)), "dsp_adamw_init")
    return out.value


def dsp_adamw_destroy(o):
    check(lib().dsp_adamw_destroy(o), "dsp_adamw_destroy")


def dsp_adamw_step(o, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, max_norm=0.0, d_norm=None, stream=None):
    check(lib().dsp_adamw_step(o, lr, beta1, beta2, eps, weight_decay, max_norm, _ptr(d_norm), _stream(stream)), "dsp_adamw_step")


def dsp_adamw_get_steps(o):
    out = C.c_int64()
    check(lib().dsp_adamw_get_steps(o, C.byref(out)), "dsp_adamw_get_steps")
    return out.value


def dsp_adamw_set_steps(o, steps, beta1=0.9, beta2=0.999):
    check(lib().dsp_adamw_set_steps(o, steps, beta1, beta2), "dsp_adamw_set_steps")


def dsp_block_set_adamw(b, state_bits=32, seed=0):
    check(lib().dsp_block_set_adamw(b, state_bits, seed), "dsp_block_set_adamw")


def dsp_param_update_adamw(b, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, max_norm=0.0, stream=None):
    check(lib().dsp_param_update_adamw(b, lr, beta1, beta2, eps, weight_decay, max_norm, _stream(stream)), "dsp_param_update_adamw")


def dsp_block_adamw_state_bytes(b):
    out = C.c_size_t()
    check(lib().dsp_block_adamw_state_bytes(b, C.byref(out)), "dsp_block_adamw_state_bytes")
    return out.value


def dsp_block_get_adamw_state(b):
    """Moments and step number as they lie (numpy uint8)."""
    out = np.empty(dsp_block_adamw_state_bytes(b), np.uint8)
    check(lib().dsp_block_get_adamw_state(b, out.ctypes.data, out.size), "dsp_block_get_adamw_state")
    return out


def dsp_block_set_adamw_state(b, h_src):
    src = np.ascontiguousarray(h_src, np.uint8)
    check(lib().dsp_block_set_adamw_state(b, src.ctypes.data, src.size), "dsp_block_set_adamw_state")


def dsp_pipeline_set_adamw(pl, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, max_norm=0.0):
    check(lib().dsp_pipeline_set_adamw(pl, lr, beta1, beta2, eps, weight_decay, max_norm), "dsp_pipeline_set_adamw")


def dsp_block_input_slot(b, batch_id):
    out = C.c_void_p()
    check(lib().dsp_block_input_slot(b, batch_id, C.byref(out)), "dsp_block_input_slot")
    return out.value


def dsp_block_query(b):
    out = (C.c_int64 * 8)()
    check(lib().dsp_block_query(b, out), "dsp_block_query")
    return dict(zip(("version", "next_fwd", "next_bwd", "ring_entries", "pending", "n_params", "fwd_version_of_next_bwd",
                     "slot_of_next_bwd"), list(out)))


def dsp_block_output_shape(b):
    out = (C.c_int32 * 5)()
    check(lib().dsp_block_output_shape(b, out), "dsp_block_output_shape")
    return tuple(out[:4]), bool(out[4])


def dsp_block_input_shape(b):
    out = (C.c_int32 * 5)()
    check(lib().dsp_block_input_shape(b, out), "dsp_block_input_shape")
    return tuple(out[:4]), out[4]


def dsp_block_memory(b):
    r, w, p = C.c_size_t(), C.c_size_t(), C.c_size_t()
    check(lib().dsp_block_memory(b, C.byref(r), C.byref(w), C.byref(p)), "dsp_block_memory")
    return {"ring": r.value, "workspace": w.value, "params": p.value}


def _get(fn, name, b):
    n = dsp_block_query(b)["n_params"]
    out = np.empty(n, np.float32)
    check(fn(b, out.ctypes.data_as(_pf), n), name)
    return out


def _set(fn, name, b, h):
    h = np.ascontiguousarray(h, dtype=np.float32)
    check(fn(b, h.ctypes.data_as(_pf), h.size), name)


def dsp_block_get_params(b):
    return _get(lib().dsp_block_get_params, "dsp_block_get_params", b)


def dsp_block_set_params(b, h):
    _set(lib().dsp_block_set_params, "dsp_block_set_params", b, h)


def dsp_block_get_momentum(b):
    return _get(lib().dsp_block_get_momentum, "dsp_block_get_momentum", b)


def dsp_block_set_momentum(b, h):
    _set(lib().dsp_block_set_momentum, "dsp_block_set_momentum", b, h)


def dsp_block_get_grads(b):
    return _get(lib().dsp_block_get_grads, "dsp_block_get_grads", b)


# ---- pipeline --------------------------------------------------------------------------------------
def dsp_pipeline_init(blocks, p, m, lr, momentum, weight_decay, max_ticks):
    K = len(blocks)
    arr = (C.c_void_p * K)(*blocks)
    out = C.c_void_p()
    check(lib().dsp_pipeline_init(K, arr, _i32arr(p), _i32arr(m), lr, momentum, weight_decay, max_ticks, C.byref(out)),
          "dsp_pipeline_init")
    return out.value


def dsp_pipeline_destroy(pl):
    check(lib().dsp_pipeline_destroy(pl), "dsp_pipeline_destroy")


def dsp_pipeline_step(pl, d_batch, d_labels, want_loss=False, stream=None):
    """Returns (loss or None, loss_batch_id)."""
    bid = C.c_int64(-1)
    loss = C.c_float(0.0)
    check(lib().dsp_pipeline_step(pl, _ptr(d_batch), _ptr(d_labels), C.byref(loss) if want_loss else None, C.byref(bid),
                                  _stream(stream)), "dsp_pipeline_step")
    return (loss.value if (want_loss and bid.value >= 0) else None), bid.value


def dsp_pipeline_set_delay(pl, k, microseconds):
    check(lib().dsp_pipeline_set_delay(pl, k, microseconds), "dsp_pipeline_set_delay")


def dsp_pipeline_set_graph_replay(pl, enable):
    check(lib().dsp_pipeline_set_graph_replay(pl, int(bool(enable))), "dsp_pipeline_set_graph_replay")


def dsp_pipeline_set_launch_threads(pl, enable):
    check(lib().dsp_pipeline_set_launch_threads(pl, int(bool(enable))), "dsp_pipeline_set_launch_threads")


def dsp_pipeline_set_single_stream(pl, enable):
    check(lib().dsp_pipeline_set_single_stream(pl, int(bool(enable))), "dsp_pipeline_set_single_stream")


def dsp_pipeline_set_forward_streams(pl, enable):
    check(lib().dsp_pipeline_set_forward_streams(pl, int(bool(enable))), "dsp_pipeline_set_forward_streams")


def dsp_pipeline_set_twin_launches(pl, enable):
    check(lib().dsp_pipeline_set_twin_launches(pl, int(bool(enable))), "dsp_pipeline_set_twin_launches")


def dsp_block_enable_forward_lane(b):
    check(lib().dsp_block_enable_forward_lane(b), "dsp_block_enable_forward_lane")


def dsp_pipeline_sync(pl):
    check(lib().dsp_pipeline_sync(pl), "dsp_pipeline_sync")


def dsp_pipeline_losses(pl):
    avail = C.c_int64()
    check(lib().dsp_pipeline_losses(pl, None, 0, C.byref(avail)), "dsp_pipeline_losses")
    out = np.empty(avail.value, np.float32)
    if avail.value:
        check(lib().dsp_pipeline_losses(pl, out.ctypes.data_as(_pf), avail.value, None), "dsp_pipeline_losses")
    return out


def dsp_pipeline_ticks(pl):
    t = C.c_int64()
    check(lib().dsp_pipeline_ticks(pl, C.byref(t)), "dsp_pipeline_ticks")
    return t.value


# ---- single layers ---------------------------------------------------------------------------------
def dsp_grouped_conv_forward(dtype, d_x, d_w, d_y, N, H, W, cin, cout, r, s, stride, pad, groups, stream=None):
    check(lib().dsp_grouped_conv_forward(dtype, _ptr(d_x), _ptr(d_w), _ptr(d_y), N, H, W, cin, cout, r, s, stride, pad, groups,
                                         _stream(stream)), "dsp_grouped_conv_forward")


def dsp_grouped_conv_backward_data(dtype, d_dy, d_wt, d_dx, N, H, W, cin, cout, r, s, stride, pad, groups, accumulate=False,
                                   stream=None):
    check(lib().dsp_grouped_conv_backward_data(dtype, _ptr(d_dy), _ptr(d_wt), _ptr(d_dx), N, H, W, cin, cout, r, s, stride, pad,
                                               groups, int(accumulate), _stream(stream)), "dsp_grouped_conv_backward_data")


def dsp_grouped_conv_backward_weight(dtype, d_x, d_dy, d_dw, N, H, W, cin, cout, r, s, stride, pad, groups, d_workspace,
                                     workspace_bytes, stream=None):
    check(lib().dsp_grouped_conv_backward_weight(dtype, _ptr(d_x), _ptr(d_dy), _ptr(d_dw), N, H, W, cin, cout, r, s, stride, pad,
                                                 groups, _ptr(d_workspace), workspace_bytes, _stream(stream)),
          "dsp_grouped_conv_backward_weight")


def dsp_grouped_conv_workspace_bytes(N, H, W, cin, cout, r, s, stride, pad, groups):
    out = C.c_size_t()
    check(lib().dsp_grouped_conv_workspace_bytes(N, H, W, cin, cout, r, s, stride, pad, groups, C.byref(out)),
          "dsp_grouped_conv_workspace_bytes")
    return out.value


def dsp_conv_forward(dtype, d_x, d_w, d_y, N, H, W, cin, cout, r, s, stride, pad, stream=None):
    check(lib().dsp_conv_forward(dtype, _ptr(d_x), _ptr(d_w), _ptr(d_y), N, H, W, cin, cout, r, s, stride, pad,
                                 _stream(stream)), "dsp_conv_forward")


def dsp_conv_backward_data(dtype, d_dy, d_wt, d_dx, N, H, W, cin, cout, r, s, stride, pad, accumulate=False, stream=None):
    check(lib().dsp_conv_backward_data(dtype, _ptr(d_dy), _ptr(d_wt), _ptr(d_dx), N, H, W, cin, cout, r, s, stride, pad,
                                       int(accumulate), _stream(stream)), "dsp_conv_backward_data")


def dsp_conv_backward_weight(dtype, d_x, d_dy, d_dw, N, H, W, cin, cout, r, s, stride, pad, d_workspace, workspace_bytes,
                             stream=None):
    check(lib().dsp_conv_backward_weight(dtype, _ptr(d_x), _ptr(d_dy), _ptr(d_dw), N, H, W, cin, cout, r, s, stride, pad,
                                         _ptr(d_workspace), workspace_bytes, _stream(stream)), "dsp_conv_backward_weight")


def dsp_conv_workspace_bytes(N, H, W, cin, cout, r, s, stride, pad):
    out = C.c_size_t()
    check(lib().dsp_conv_workspace_bytes(N, H, W, cin, cout, r, s, stride, pad, C.byref(out)), "dsp_conv_workspace_bytes")
    return out.value


def dsp_conv_backward_weight_static(dtype, d_x, d_dy, d_dw, N, H, W, cin, cout, r, s, stride, pad, stream=None):
    check(lib().dsp_conv_backward_weight_static(dtype, _ptr(d_x), _ptr(d_dy), _ptr(d_dw), N, H, W, cin, cout, r, s, stride, pad,
                                                _stream(stream)), "dsp_conv_backward_weight_static")


def dsp_conv_backward_weight_static_bytes():
    out = C.c_size_t()
    check(lib().dsp_conv_backward_weight_static_bytes(C.byref(out)), "dsp_conv_backward_weight_static_bytes")
    return out.value


def dsp_bn_workspace_bytes(C_):
    out = C.c_size_t()
    check(lib().dsp_bn_workspace_bytes(C_, C.byref(out)), "dsp_bn_workspace_bytes")
    return out.value


def dsp_bn_forward(dtype, d_x, d_res, d_y, d_gamma, d_beta, eps, M, C_, relu, d_mean, d_invstd, d_workspace, workspace_bytes,
                   stream=None):
    check(lib().dsp_bn_forward(dtype, _ptr(d_x), _ptr(d_res), _ptr(d_y), _ptr(d_gamma), _ptr(d_beta), eps, M, C_, int(relu),
                               _ptr(d_mean), _ptr(d_invstd), _ptr(d_workspace), workspace_bytes, _stream(stream)),
          "dsp_bn_forward")


def dsp_bn_backward(dtype, d_dy, d_x, d_y, d_dx, d_dres, dres_accumulate, dx_accumulate, d_gamma, d_mean, d_invstd, d_dgamma,
                    d_dbeta, M, C_, relu, d_workspace, workspace_bytes, stream=None):
    check(lib().dsp_bn_backward(dtype, _ptr(d_dy), _ptr(d_x), _ptr(d_y), _ptr(d_dx), _ptr(d_dres), int(dres_accumulate),
                                int(dx_accumulate), _ptr(d_gamma), _ptr(d_mean), _ptr(d_invstd), _ptr(d_dgamma),
                                _ptr(d_dbeta), M, C_, int(relu), _ptr(d_workspace), workspace_bytes, _stream(stream)),
          "dsp_bn_backward")


def dsp_bn_relu_maxpool_forward(dtype, d_x, d_gamma, d_beta, eps, N, H, W, C_, k, stride, pad, d_pool, d_argmax, d_mean, d_invstd,
                                d_scale_shift, d_workspace, workspace_bytes, stream=None):
    check(lib().dsp_bn_relu_maxpool_forward(dtype, _ptr(d_x), _ptr(d_gamma), _ptr(d_beta), eps, N, H, W, C_, k, stride, pad,
                                            _ptr(d_pool), _ptr(d_argmax), _ptr(d_mean), _ptr(d_invstd), _ptr(d_scale_shift),
                                            _ptr(d_workspace), workspace_bytes, _stream(stream)), "dsp_bn_relu_maxpool_forward")


def dsp_bn_relu_backward_from_x(dtype, d_dy, d_x, d_scale_shift, d_dx, dx_accumulate, d_gamma, d_mean, d_invstd, d_dgamma, d_dbeta,
                                M, C_, d_workspace, workspace_bytes, stream=None):
    check(lib().dsp_bn_relu_backward_from_x(dtype, _ptr(d_dy), _ptr(d_x), _ptr(d_scale_shift), _ptr(d_dx), int(dx_accumulate),
                                            _ptr(d_gamma), _ptr(d_mean), _ptr(d_invstd), _ptr(d_dgamma), _ptr(d_dbeta), M, C_,
                                            _ptr(d_workspace), workspace_bytes, _stream(stream)), "dsp_bn_relu_backward_from_x")


def dsp_bn_relu_bits_bytes(dtype, M, C_):
    n = C.c_size_t(0)
    check(lib().dsp_bn_relu_bits_bytes(dtype, M, C_, C.byref(n)), "dsp_bn_relu_bits_bytes")
    return int(n.value)


def dsp_bn_forward_bits(dtype, d_x, d_res, d_y, d_gamma, d_beta, eps, M, C_, d_mean, d_invstd, d_relu_bits, d_workspace,
                        workspace_bytes, stream=None):
    check(lib().dsp_bn_forward_bits(dtype, _ptr(d_x), _ptr(d_res), _ptr(d_y), _ptr(d_gamma), _ptr(d_beta), eps, M, C_, _ptr(d_mean),
                                    _ptr(d_invstd), _ptr(d_relu_bits), _ptr(d_workspace), workspace_bytes, _stream(stream)),
          "dsp_bn_forward_bits")


def dsp_bn_backward_bits(dtype, d_dy, d_x, d_relu_bits, d_dx, d_dres, dres_accumulate, dx_accumulate, d_gamma, d_mean, d_invstd,
                         d_dgamma, d_dbeta, M, C_, d_workspace, workspace_bytes, stream=None):
    check(lib().dsp_bn_backward_bits(dtype, _ptr(d_dy), _ptr(d_x), _ptr(d_relu_bits), _ptr(d_dx), _ptr(d_dres), int(dres_accumulate),
                                     int(dx_accumulate), _ptr(d_gamma), _ptr(d_mean), _ptr(d_invstd), _ptr(d_dgamma), _ptr(d_dbeta),
                                     M, C_, _ptr(d_workspace), workspace_bytes, _stream(stream)), "dsp_bn_backward_bits")


def dsp_bn_relu_maxpool_backward(dtype, d_dpool, d_argmax, d_x, d_scale_shift, d_dx, dx_accumulate, d_gamma, d_mean, d_invstd,
                                 d_dgamma, d_dbeta, N, H, W, C_, k, stride, pad, d_workspace, workspace_bytes, stream=None):
    check(lib().dsp_bn_relu_maxpool_backward(dtype, _ptr(d_dpool), _ptr(d_argmax), _ptr(d_x), _ptr(d_scale_shift), _ptr(d_dx),
                                             int(dx_accumulate), _ptr(d_gamma), _ptr(d_mean), _ptr(d_invstd), _ptr(d_dgamma),
                                             _ptr(d_dbeta), N, H, W, C_, k, stride, pad, _ptr(d_workspace), workspace_bytes,
                                             _stream(stream)), "dsp_bn_relu_maxpool_backward")


def dsp_maxpool_forward(dtype, d_x, d_y, d_argmax, N, H, W, C_, k, stride, pad, stream=None):
    check(lib().dsp_maxpool_forward(dtype, _ptr(d_x), _ptr(d_y), _ptr(d_argmax), N, H, W, C_, k, stride, pad, _stream(stream)),
          "dsp_maxpool_forward")


def dsp_maxpool_backward(dtype, d_dy, d_argmax, d_dx, accumulate, N, H, W, C_, k, stride, pad, stream=None):
    check(lib().dsp_maxpool_backward(dtype, _ptr(d_dy), _ptr(d_argmax), _ptr(d_dx), int(accumulate), N, H, W, C_, k, stride,
                                     pad, _stream(stream)), "dsp_maxpool_backward")


def dsp_add_forward(dtype, d_a, d_b, d_y, n, stream=None):
    check(lib().dsp_add_forward(dtype, _ptr(d_a), _ptr(d_b), _ptr(d_y), n, _stream(stream)), "dsp_add_forward")


def dsp_add_backward(dtype, d_dy, d_da, da_accumulate, d_db, db_accumulate, n, stream=None):
    check(lib().dsp_add_backward(dtype, _ptr(d_dy), _ptr(d_da), int(da_accumulate), _ptr(d_db), int(db_accumulate), n,
                                 _stream(stream)), "dsp_add_backward")


def dsp_gap_forward(dtype, d_x, d_y, N, HW, C_, stream=None):
    check(lib().dsp_gap_forward(dtype, _ptr(d_x), _ptr(d_y), N, HW, C_, _stream(stream)), "dsp_gap_forward")


def dsp_gap_backward(dtype, d_dy, d_dx, accumulate, N, HW, C_, stream=None):
    check(lib().dsp_gap_backward(dtype, _ptr(d_dy), _ptr(d_dx), int(accumulate), N, HW, C_, _stream(stream)), "dsp_gap_backward")


def dsp_linear_forward(d_x, d_w, d_bias, d_z, N, cin, cout, stream=None):
    check(lib().dsp_linear_forward(_ptr(d_x), _ptr(d_w), _ptr(d_bias), _ptr(d_z), N, cin, cout, _stream(stream)),
          "dsp_linear_forward")


def dsp_linear_backward(d_x, d_w, d_dz, d_dx, d_dw, d_dbias, N, cin, cout, stream=None):
    check(lib().dsp_linear_backward(_ptr(d_x), _ptr(d_w), _ptr(d_dz), _ptr(d_dx), _ptr(d_dw), _ptr(d_dbias), N, cin, cout,
                                    _stream(stream)), "dsp_linear_backward")


def dsp_softmax_ce(d_z, d_labels, d_loss, d_dz, d_row_loss, N, C_, stream=None):
    check(lib().dsp_softmax_ce(_ptr(d_z), _ptr(d_labels), _ptr(d_loss), _ptr(d_dz), _ptr(d_row_loss), N, C_, _stream(stream)),
          "dsp_softmax_ce")


# ---- norms, gate and residual sum between two blocks --------------------------------------------------
def make_norm_residual_desc(M, C_, dtype, post=0, pre=0, alpha=1.0, beta=1.0, eps=1e-5, gate_rows=0, gate_act=0, gate_dtype=None,
                            x_stride=0, z_stride=0, y_stride=0, h_stride=0, gate_stride=0):
    return dsp_norm_residual_desc(M, C_, dtype, post, pre, gate_act, dtype if gate_dtype is None else gate_dtype, gate_rows, alpha,
                                  beta, eps, x_stride, z_stride, y_stride, h_stride, gate_stride)


def dsp_norm_residual_forward(desc, d_x, d_z=None, d_gate=None, d_post_gain=None, d_post_bias=None, d_pre_gain=None, d_pre_bias=None,
                              d_y=None, d_h=None, d_post_stats=None, d_pre_stats=None, stream=None):
    check(lib().dsp_norm_residual_forward(C.byref(desc), _ptr(d_x), _ptr(d_z), _ptr(d_gate), _ptr(d_post_gain), _ptr(d_post_bias),
                                          _ptr(d_pre_gain), _ptr(d_pre_bias), _ptr(d_y), _ptr(d_h), _ptr(d_post_stats),
                                          _ptr(d_pre_stats), _stream(stream)), "dsp_norm_residual_forward")


def dsp_norm_residual_workspace_bytes(desc):
    out = C.c_size_t()
    check(lib().dsp_norm_residual_workspace_bytes(C.byref(desc), C.byref(out)), "dsp_norm_residual_workspace_bytes")
    return out.value


def dsp_norm_residual_backward(desc, d_dh, d_dy, d_y, d_z, d_gate, d_post_gain, d_post_bias, d_pre_gain, d_post_stats, d_pre_stats, d_dx,
                               d_dz, d_dgate=None, d_dpost_gain=None, d_dpost_bias=None, d_dpre_gain=None, d_dpre_bias=None,
                               d_workspace=None, workspace_bytes=0, stream=None):
    check(lib().dsp_norm_residual_backward(C.byref(desc), _ptr(d_dh), _ptr(d_dy), _ptr(d_y), _ptr(d_z), _ptr(d_gate),
                                           _ptr(d_post_gain), _ptr(d_post_bias), _ptr(d_pre_gain), _ptr(d_post_stats),
                                           _ptr(d_pre_stats), _ptr(d_dx), _ptr(d_dz), _ptr(d_dgate), _ptr(d_dpost_gain),
                                           _ptr(d_dpost_bias), _ptr(d_dpre_gain), _ptr(d_dpre_bias), _ptr(d_workspace),
                                           workspace_bytes, _stream(stream)), "dsp_norm_residual_backward")


# ---- products, recurrence and policy loss of residual blocks ------------------------------------------
def make_dense_desc(M, cin, cout, dtype, act=0, x_stride=0, y_stride=0):
    return dsp_dense_desc(M, cin, cout, dtype, act, x_stride, y_stride)


def dsp_dense_workspace_bytes(desc, backward=False):
    out = C.c_size_t()
    check(lib().dsp_dense_workspace_bytes(C.byref(desc), int(backward), C.byref(out)), "dsp_dense_workspace_bytes")
    return out.value


def dsp_dense_forward(desc, d_x, d_w, d_bias, d_residual, d_y, d_pre=None, d_workspace=None, workspace_bytes=0, stream=None):
    check(lib().dsp_dense_forward(C.byref(desc), _ptr(d_x), _ptr(d_w), _ptr(d_bias), _ptr(d_residual), _ptr(d_y), _ptr(d_pre),
                                  _ptr(d_workspace), workspace_bytes, _stream(stream)), "dsp_dense_forward")


def dsp_dense_backward(desc, d_dy, d_x, d_w, d_pre, d_dx, d_dw, d_dbias, d_workspace, workspace_bytes, stream=None):
    check(lib().dsp_dense_backward(C.byref(desc), _ptr(d_dy), _ptr(d_x), _ptr(d_w), _ptr(d_pre), _ptr(d_dx), _ptr(d_dw), _ptr(d_dbias),
                                   _ptr(d_workspace), workspace_bytes, _stream(stream)), "dsp_dense_backward")


def make_recurrence_desc(sequences, steps, rows, C_, dtype, decay=0, coupled=True, x_stride=0, f_stride=0, h_stride=0):
    return dsp_recurrence_desc(rows, sequences, steps, C_, dtype, decay, int(bool(coupled)), x_stride, f_stride, h_stride)


def dsp_recurrence_workspace_bytes(desc):
    out = C.c_size_t()
    check(lib().dsp_recurrence_workspace_bytes(C.byref(desc), C.byref(out)), "dsp_recurrence_workspace_bytes")
    return out.value


def dsp_recurrence_forward(desc, d_x, d_f, d_offsets, d_state_in, d_h, d_state_out=None, d_workspace=None, workspace_bytes=0, stream=None):
    check(lib().dsp_recurrence_forward(C.byref(desc), _ptr(d_x), _ptr(d_f), _ptr(d_offsets), _ptr(d_state_in), _ptr(d_h), _ptr(d_state_out),
                                       _ptr(d_workspace), workspace_bytes, _stream(stream)), "dsp_recurrence_forward")


def dsp_recurrence_backward(desc, d_dh, d_dstate_out, d_x, d_f, d_h, d_offsets, d_state_in, d_dx, d_df, d_dstate_in=None, d_workspace=None,
                            workspace_bytes=0, stream=None):
    check(lib().dsp_recurrence_backward(C.byref(desc), _ptr(d_dh), _ptr(d_dstate_out), _ptr(d_x), _ptr(d_f), _ptr(d_h), _ptr(d_offsets),
                                        _ptr(d_state_in), _ptr(d_dx), _ptr(d_df), _ptr(d_dstate_in), _ptr(d_workspace), workspace_bytes,
                                        _stream(stream)), "dsp_recurrence_backward")


def make_policy_loss_desc(rows, vocab, dtype, clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0, temperature=1.0, logits_stride=0,
                          grad_stride=0):
    return dsp_policy_loss_desc(rows, vocab, dtype, clip_low, clip_high, kl_coef, entropy_coef, temperature, logits_stride, grad_stride)


def dsp_token_logprob(desc, d_logits, d_labels, d_logp, d_entropy=None, stream=None):
    check(lib().dsp_token_logprob(C.byref(desc), _ptr(d_logits), _ptr(d_labels), _ptr(d_logp), _ptr(d_entropy), _stream(stream)),
          "dsp_token_logprob")


def dsp_policy_loss(desc, d_logits, d_labels, d_old_logp, d_ref_logp, d_advantage, d_weight, d_loss, d_logp, d_terms, d_dlogits=None,
                    stream=None):
    check(lib().dsp_policy_loss(C.byref(desc), _ptr(d_logits), _ptr(d_labels), _ptr(d_old_logp), _ptr(d_ref_logp), _ptr(d_advantage),
                                _ptr(d_weight), _ptr(d_loss), _ptr(d_logp), _ptr(d_terms), _ptr(d_dlogits), _stream(stream)),
          "dsp_policy_loss")


def dsp_block_get_activation(b, layer, nbytes):
    """Raw bytes (numpy uint8) of the output layer ``layer`` left in the buffers the backward sweep reads."""
    out = np.empty(nbytes, np.uint8)
    check(lib().dsp_block_get_activation(b, layer, out.ctypes.data, nbytes), "dsp_block_get_activation")
    return out


def dsp_block_get_pool_argmax(b, layer, nbytes):
    out = np.empty(nbytes, np.uint8)
    check(lib().dsp_block_get_pool_argmax(b, layer, out.ctypes.data, nbytes), "dsp_block_get_pool_argmax")
    return out


def dsp_profile_start(max_launches):
    check(lib().dsp_profile_start(max_launches), "dsp_profile_start")


def dsp_profile_stop():
    """Returns the per-kernel table: list of dicts (name, launches, ms, units, unit_kind)."""
    n = C.c_int32()
    check(lib().dsp_profile_stop(C.byref(n)), "dsp_profile_stop")
    return [dsp_profile_get(i) for i in range(n.value)]


def dsp_profile_get(i):
    name = C.create_string_buffer(128)
    launches, ms, units, kind = C.c_int64(), C.c_double(), C.c_double(), C.c_int32()
    check(lib().dsp_profile_get(i, name, 128, C.byref(launches), C.byref(ms), C.byref(units), C.byref(kind)),
          "dsp_profile_get")
    return {"name": name.value.decode(), "launches": launches.value, "ms": ms.value, "units": units.value,
            "unit_kind": "flop" if kind.value == 0 else "byte"}


def dsp_strerror(status):
    return lib().dsp_strerror(status).decode()


def dsp_last_error():
    return lib().dsp_last_error().decode()


def dsp_build_id():
    return lib().dsp_build_id().decode()
