"""ctypes binding of liblamp.so: argument marshalling only.

Every function has the name of the C entry point it wraps (see include/lamp.h)
and does nothing but build descriptors and pass device pointers of torch
tensors; all arithmetic runs in the library's CUDA kernels.  There is no CPU
path: loading fails loudly when the library is missing.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblamp.so")

LAMP_BF16, LAMP_F32 = 0, 1
PASS_FWD, PASS_DGRAD, PASS_WGRAD = 0, 1, 2
MODE_INFER, MODE_TRAIN = 0, 1


class LampError(RuntimeError):
    def __init__(self, status, what):
        self.status = int(status)
        super().__init__(f"{what}: lamp status {int(status)} ({lib().lamp_status_string(int(status)).decode()})")


class Tensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("dtype", C.c_int32), ("n", C.c_int32), ("d", C.c_int32), ("h", C.c_int32),
                ("w", C.c_int32), ("c", C.c_int32), ("c_pitch", C.c_int64), ("c_offset", C.c_int32)]


class ConvDesc(C.Structure):
    _fields_ = [("c_in", C.c_int32), ("c_out", C.c_int32), ("ksize", C.c_int32), ("stride", C.c_int32),
                ("pad", C.c_int32), ("transposed", C.c_int32)]


class UNetSpec(C.Structure):
    _fields_ = [("levels", C.c_int32), ("channels", C.c_int32 * 8), ("convs_per_level", C.c_int32),
                ("in_channels", C.c_int32), ("num_classes", C.c_int32), ("in_eps", C.c_float), ("se_ratio", C.c_int32)]


class Fp8Operand(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_pitch", C.c_int64), ("scale", C.c_void_p), ("scale_pitch", C.c_int64),
                ("rows", C.c_int64), ("k", C.c_int64), ("tile_scale", C.c_int32)]


class BlockNorm(C.Structure):
    _fields_ = [("rms", C.c_int32), ("eps", C.c_float), ("post_w", C.c_void_p), ("post_b", C.c_void_p), ("pre_w", C.c_void_p),
                ("pre_b", C.c_void_p), ("gate", C.c_void_p), ("gate_logits", C.POINTER(Tensor)), ("res_scale", C.c_void_p)]


class BlockNormGrads(C.Structure):
    _fields_ = [("post_w", C.c_void_p), ("post_b", C.c_void_p), ("pre_w", C.c_void_p), ("pre_b", C.c_void_p),
                ("gate", C.c_void_p), ("res_scale", C.c_void_p)]


class TeacherTopk(C.Structure):
    _fields_ = [("idx", C.c_void_p), ("logits", C.c_void_p), ("lse", C.c_void_p), ("k", C.c_int32), ("temperature", C.c_float)]


class Fp4Operand(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_pitch", C.c_int64), ("scale", C.c_void_p), ("tensor_scale", C.c_void_p), ("rows", C.c_int64),
                ("k", C.c_int64), ("block", C.c_int32)]


class GroupNorm(C.Structure):
    _fields_ = [("groups", C.c_int32), ("act", C.c_int32), ("slope", C.c_float), ("eps", C.c_float), ("w", C.c_void_p), ("b", C.c_void_p)]


class Grad(C.Structure):
    _fields_ = [("g", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32)]


_lib = None


def lib():
    """Loads liblamp.so (built in-tree by build.py).  Raises if it is absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not found: build it with `python -m paper_2006_12575_b200.build`")
        L = C.CDLL(LIB_PATH)
        vp, sz, i32, f32 = C.c_void_p, C.c_size_t, C.c_int32, C.c_float
        TP, DP, SP = C.POINTER(Tensor), C.POINTER(ConvDesc), C.POINTER(UNetSpec)
        I3 = C.POINTER(C.c_int32)
        FP, NP, GP, KP = C.POINTER(Fp8Operand), C.POINTER(BlockNorm), C.POINTER(BlockNormGrads), C.POINTER(TeacherTopk)
        QP, UP, RP = C.POINTER(Fp4Operand), C.POINTER(GroupNorm), C.POINTER(Grad)
        sig = {
            "lamp_conv3d_workspace_bytes": (sz, [DP, TP, C.c_int]),
            "lamp_conv3d_workspace_min_bytes": (sz, [DP, TP, C.c_int]),
            "lamp_conv3d_fwd": (C.c_int, [DP, TP, vp, vp, TP, vp, vp, sz, vp]),
            "lamp_conv3d_dgrad": (C.c_int, [DP, TP, vp, TP, vp, sz, vp]),
            "lamp_conv3d_dgrad_static_scratch": (C.c_int, [DP, TP, vp, TP, vp]),
            "lamp_conv3d_wgrad": (C.c_int, [DP, TP, TP, vp, vp, vp, sz, vp]),
            "lamp_instnorm_relu_fwd": (C.c_int, [TP, vp, f32, vp, TP, vp]),
            "lamp_instnorm_relu_bwd": (C.c_int, [TP, TP, TP, vp, vp, TP, vp]),
            "lamp_se_squeeze": (C.c_int, [TP, vp, vp, vp]),
            "lamp_se_excite": (C.c_int, [vp, C.c_int64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]),
            "lamp_se_apply_fwd": (C.c_int, [TP, vp, vp, TP, TP, vp]),
            "lamp_se_bwd_reduce": (C.c_int, [TP, TP, vp, vp, vp]),
            "lamp_se_excite_bwd": (C.c_int, [vp, C.c_int64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]),
            "lamp_se_apply_bwd": (C.c_int, [TP, vp, vp, TP, vp]),
            "lamp_fp8_quantize": (C.c_int, [TP, i32, FP, vp]),
            "lamp_gemm_fp8": (C.c_int, [FP, FP, vp, TP, vp]),
            "lamp_fp4_scale_bytes": (sz, [C.c_int64, C.c_int64, i32]),
            "lamp_fp4_quantize": (C.c_int, [TP, i32, QP, vp]),
            "lamp_fp4_dequantize": (C.c_int, [QP, i32, TP, vp]),
            "lamp_gemm_fp4": (C.c_int, [QP, QP, vp, TP, vp]),
            "lamp_group_norm_workspace_bytes": (sz, [UP, TP]),
            "lamp_group_norm_act_fwd": (C.c_int, [UP, TP, vp, TP, vp, vp, sz, vp]),
            "lamp_group_norm_act_bwd": (C.c_int, [UP, TP, TP, vp, TP, vp, vp, vp, sz, vp]),
            "lamp_block_norm_fwd": (C.c_int, [NP, TP, TP, TP, TP, FP, vp]),
            "lamp_block_norm_bwd_workspace_bytes": (sz, [TP, NP]),
            "lamp_block_norm_bwd": (C.c_int, [NP, TP, TP, TP, TP, TP, TP, TP, GP, vp, sz, vp]),
            "lamp_distill_topk_workspace_bytes": (sz, [TP]),
            "lamp_distill_topk_fwd": (C.c_int, [TP, KP, vp, vp, vp, vp, vp, sz, vp]),
            "lamp_distill_topk_bwd": (C.c_int, [TP, KP, vp, vp, TP, vp]),
            "lamp_distill_topk_fwd_bwd": (C.c_int, [TP, KP, vp, vp, vp, TP, vp, sz, vp]),
            "lamp_unet_create": (C.c_int, [SP, C.POINTER(vp)]),
            "lamp_unet_se_layout": (C.c_int, [vp, i32, C.POINTER(sz), C.POINTER(i32)]),
            "lamp_unet_destroy": (None, [vp]),
            "lamp_unet_num_layers": (i32, [vp]),
            "lamp_unet_weight_count": (sz, [vp]),
            "lamp_unet_bias_count": (sz, [vp]),
            "lamp_unet_param_layout": (C.c_int, [vp, i32, C.POINTER(sz), C.POINTER(sz), DP]),
            "lamp_unet_workspace_bytes": (sz, [vp, i32, i32, i32, i32, i32]),
            "lamp_unet_tensor_layout": (C.c_int, [vp, i32, i32, i32, i32, i32, i32, i32, TP, C.POINTER(sz)]),
            "lamp_unet_forward": (C.c_int, [vp, vp, vp, TP, vp, vp, vp, sz, vp]),
            "lamp_unet_forward_layers": (C.c_int, [vp, vp, vp, TP, i32, i32, vp, vp, vp, sz, vp]),
            "lamp_unet_train_step": (C.c_int, [vp, vp, vp, TP, vp, vp, vp, vp, vp, vp, sz, vp]),
            "lamp_unet_train_step_buckets": (C.c_int, [vp, vp, vp, TP, vp, vp, vp, vp, vp, vp, sz, vp,
                                                       C.POINTER(C.c_int64), i32, C.POINTER(vp)]),
            "lamp_sliding_window_num_patches": (i32, [i32, i32, i32, I3, f32]),
            "lamp_sliding_window_partial": (C.c_int, [vp, vp, vp, TP, I3, f32, i32, i32, i32, i32, vp, vp, vp, sz, vp]),
            "lamp_sliding_window_finish": (C.c_int, [vp, vp, i32, C.c_int64, i32, vp, vp]),
            "lamp_sliding_window_workspace_bytes": (sz, [vp, i32, i32, i32, I3, f32, i32]),
            "lamp_sliding_window_infer": (C.c_int, [vp, vp, vp, TP, I3, f32, i32, i32, vp, vp, vp, sz, vp]),
            "lamp_overlap_add": (C.c_int, [vp, i32, i32, i32, i32, I3, f32, i32, vp, vp, vp]),
            "lamp_rmsprop_step": (C.c_int, [C.c_int64, vp, vp, vp, vp, f32, f32, f32, vp]),
            "lamp_rmsprop_step_scaled": (C.c_int, [C.c_int64, vp, vp, vp, vp, vp, f32, f32, f32, vp]),
            "lamp_grad_norm_workspace_bytes": (sz, [RP, i32]),
            "lamp_grad_norm": (C.c_int, [RP, i32, f32, vp, vp, vp, sz, vp]),
            "lamp_grad_clip": (C.c_int, [RP, i32, f32, vp, vp, vp, sz, vp]),
            "lamp_get_async_status": (C.c_int, [vp]),
            "lamp_selftest_wait_timeout": (C.c_int, [vp]),
            "lamp_status_string": (C.c_char_p, [C.c_int]),
            "lamp_version": (C.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


EXPORTS = ["lamp_conv3d_workspace_bytes", "lamp_conv3d_workspace_min_bytes", "lamp_conv3d_fwd", "lamp_conv3d_dgrad", "lamp_conv3d_dgrad_static_scratch",
           "lamp_conv3d_wgrad",
           "lamp_instnorm_relu_fwd", "lamp_instnorm_relu_bwd",
           "lamp_se_squeeze", "lamp_se_excite", "lamp_se_apply_fwd", "lamp_se_bwd_reduce", "lamp_se_excite_bwd", "lamp_se_apply_bwd",
           "lamp_fp8_quantize", "lamp_gemm_fp8", "lamp_fp4_scale_bytes", "lamp_fp4_quantize", "lamp_fp4_dequantize", "lamp_gemm_fp4",
           "lamp_group_norm_workspace_bytes", "lamp_group_norm_act_fwd", "lamp_group_norm_act_bwd", "lamp_block_norm_fwd", "lamp_block_norm_bwd_workspace_bytes", "lamp_block_norm_bwd",
           "lamp_distill_topk_workspace_bytes", "lamp_distill_topk_fwd", "lamp_distill_topk_bwd", "lamp_distill_topk_fwd_bwd",
           "lamp_unet_create", "lamp_unet_se_layout", "lamp_unet_destroy",
           "lamp_unet_num_layers", "lamp_unet_weight_count", "lamp_unet_bias_count", "lamp_unet_param_layout",
           "lamp_unet_workspace_bytes", "lamp_unet_tensor_layout", "lamp_unet_forward", "lamp_unet_forward_layers", "lamp_unet_train_step",
           "lamp_unet_train_step_buckets", "lamp_sliding_window_num_patches", "lamp_sliding_window_partial",
           "lamp_sliding_window_finish",
           "lamp_sliding_window_workspace_bytes", "lamp_sliding_window_infer", "lamp_overlap_add",
           "lamp_rmsprop_step", "lamp_rmsprop_step_scaled", "lamp_grad_norm_workspace_bytes", "lamp_grad_norm", "lamp_grad_clip", "lamp_get_async_status", "lamp_selftest_wait_timeout", "lamp_status_string", "lamp_version"]


def _check(st, what):
    if st != 0:
        raise LampError(st, what)


# handle of the current stream of a device, without the Stream object around it (3 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


# the current device without torch.cuda's check that CUDA is up: whoever passes a CUDA tensor has brought it up
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream():
    return _raw_stream(torch.cuda.current_device())


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else None


def tensor(t: torch.Tensor, c=None, c_offset=0) -> Tensor:
    """Descriptor of a channel slice [c_offset, c_offset + c) of an NDHWC torch tensor [n,d,h,w,pitch]."""
    assert t.dim() == 5 and t.is_contiguous()
    dt = {torch.bfloat16: LAMP_BF16, torch.float32: LAMP_F32}[t.dtype]
    n, d, h, w, pitch = t.shape
    o = Tensor(t.data_ptr(), dt, n, d, h, w, pitch - c_offset if c is None else c, pitch, c_offset)
    o.keep, o.dev = t, t.get_device()                               # the memory lives as long as its descriptor
    return o


def _td(x):
    return x if isinstance(x, Tensor) else tensor(x)


def conv_desc(c_in, c_out, ksize=3, stride=1, pad=1, transposed=0) -> ConvDesc:
    return ConvDesc(c_in, c_out, ksize, stride, pad, transposed)


def lamp_conv3d_workspace_bytes(desc, x, pass_):
    return lib().lamp_conv3d_workspace_bytes(C.byref(desc), C.byref(_td(x)), pass_)


def lamp_conv3d_workspace_min_bytes(desc, x, pass_):
    return lib().lamp_conv3d_workspace_min_bytes(C.byref(desc), C.byref(_td(x)), pass_)


def _ws(ws):
    return (_ptr(ws), ws.numel() * ws.element_size()) if ws is not None else (None, 0)


def lamp_conv3d_fwd(desc, x, w, bias, y, stats=None, ws=None):
    p, nbytes = _ws(ws)
    _check(lib().lamp_conv3d_fwd(C.byref(desc), C.byref(_td(x)), _ptr(w), _ptr(bias), C.byref(_td(y)), _ptr(stats),
                                 p, nbytes, _stream()), "lamp_conv3d_fwd")


def lamp_conv3d_dgrad(desc, dy, w, dx, ws=None):
    p, nbytes = _ws(ws)
    _check(lib().lamp_conv3d_dgrad(C.byref(desc), C.byref(_td(dy)), _ptr(w), C.byref(_td(dx)), p, nbytes, _stream()),
           "lamp_conv3d_dgrad")


STATIC_SCRATCH_BYTES = 4 * 1024 * 1024


def lamp_conv3d_dgrad_static_scratch(desc, dy, w, dx):
    """lamp_conv3d_dgrad without a caller workspace: the scratch is a fixed array inside the library
    (for callers that cannot allocate device memory at call time).  Raises LampError with status 7
    when the layer needs more than STATIC_SCRATCH_BYTES."""
    _check(lib().lamp_conv3d_dgrad_static_scratch(C.byref(desc), C.byref(_td(dy)), _ptr(w), C.byref(_td(dx)), _stream()),
           "lamp_conv3d_dgrad_static_scratch")


def lamp_conv3d_wgrad(desc, x, dy, dw, dbias=None, ws=None):
    p, nbytes = _ws(ws)
    _check(lib().lamp_conv3d_wgrad(C.byref(desc), C.byref(_td(x)), C.byref(_td(dy)), _ptr(dw), _ptr(dbias), p, nbytes,
                                   _stream()), "lamp_conv3d_wgrad")


def lamp_instnorm_relu_fwd(y, stats, eps, mu_rstd, z):
    _check(lib().lamp_instnorm_relu_fwd(C.byref(_td(y)), _ptr(stats), eps, _ptr(mu_rstd), C.byref(_td(z)), _stream()),
           "lamp_instnorm_relu_fwd")


def lamp_instnorm_relu_bwd(dz_a, dz_b, y, mu_rstd, sums, dy):
    b = C.byref(_td(dz_b)) if dz_b is not None else None
    _check(lib().lamp_instnorm_relu_bwd(C.byref(_td(dz_a)), b, C.byref(_td(y)), _ptr(mu_rstd), _ptr(sums),
                                        C.byref(_td(dy)), _stream()), "lamp_instnorm_relu_bwd")


def unet_spec(levels, channels, convs_per_level=2, in_channels=1, num_classes=4, eps=1e-5, se_ratio=0) -> UNetSpec:
    ch = (C.c_int32 * 8)(*(list(channels) + [0] * (8 - len(channels))))
    return UNetSpec(levels, ch, convs_per_level, in_channels, num_classes, eps, se_ratio)


def lamp_unet_create(spec: UNetSpec):
    h = C.c_void_p()
    _check(lib().lamp_unet_create(C.byref(spec), C.byref(h)), "lamp_unet_create")
    return h


def lamp_unet_destroy(net):
    lib().lamp_unet_destroy(net)


def lamp_unet_num_layers(net):
    return lib().lamp_unet_num_layers(net)


def lamp_unet_weight_count(net):
    return lib().lamp_unet_weight_count(net)


def lamp_unet_bias_count(net):
    return lib().lamp_unet_bias_count(net)


def lamp_unet_param_layout(net, layer):
    wo, bo, d = C.c_size_t(), C.c_size_t(), ConvDesc()
    _check(lib().lamp_unet_param_layout(net, layer, C.byref(wo), C.byref(bo), C.byref(d)), "lamp_unet_param_layout")
    return wo.value, bo.value, d


def lamp_unet_se_layout(net, layer):
    off, cr = C.c_size_t(), C.c_int32()
    _check(lib().lamp_unet_se_layout(net, layer, C.byref(off), C.byref(cr)), "lamp_unet_se_layout")
    return off.value, cr.value


def lamp_unet_workspace_bytes(net, n, d, h, w, mode):
    return lib().lamp_unet_workspace_bytes(net, n, d, h, w, mode)


T_IN, T_Y, T_OUT, T_STATS, T_MU_RSTD, T_DY, T_DIN, T_DOUT, T_DOUT2, T_PROBS = range(10)


def lamp_unet_tensor_layout(net, n, d, h, w, mode, layer, which):
    """Returns (descriptor, byte offset into the workspace), or None if the layer has no such tensor."""
    t, off = Tensor(), C.c_size_t()
    st = lib().lamp_unet_tensor_layout(net, n, d, h, w, mode, layer, which, C.byref(t), C.byref(off))
    if st == 2:
        return None
    _check(st, "lamp_unet_tensor_layout")
    return t, off.value


def lamp_unet_forward(net, weights, biases, x, probs, argmax, ws):
    p, nbytes = _ws(ws)
    _check(lib().lamp_unet_forward(net, _ptr(weights), _ptr(biases), C.byref(_td(x)), _ptr(probs), _ptr(argmax),
                                   p, nbytes, _stream()), "lamp_unet_forward")


def lamp_unet_forward_layers(net, weights, biases, x, first_layer, last_layer, probs, argmax, ws):
    p, nbytes = _ws(ws)
    _check(lib().lamp_unet_forward_layers(net, _ptr(weights), _ptr(biases), C.byref(_td(x)), first_layer, last_layer,
                                          _ptr(probs), _ptr(argmax), p, nbytes, _stream()), "lamp_unet_forward_layers")


def lamp_unet_train_step(net, weights, biases, x, labels, loss, grad_w, grad_b, probs, ws):
    p, nbytes = _ws(ws)
    _check(lib().lamp_unet_train_step(net, _ptr(weights), _ptr(biases), C.byref(_td(x)), _ptr(labels), _ptr(loss),
                                      _ptr(grad_w), _ptr(grad_b), _ptr(probs), p, nbytes, _stream()),
           "lamp_unet_train_step")


def lamp_unet_train_step_buckets(net, weights, biases, x, labels, loss, grad_w, grad_b, probs, ws, bucket_start, bucket_events):
    """bucket_start: ascending element offsets into grad_w (first 0); bucket_events: one torch.cuda.Event per bucket,
    recorded by the library when that range of grad_w is final."""
    p, nbytes = _ws(ws)
    n = len(bucket_start)
    for e in bucket_events:
        if not e.cuda_event:                 # torch creates the CUDA event lazily, on the first record
            e.record()
    starts = (C.c_int64 * n)(*[int(v) for v in bucket_start])
    events = (C.c_void_p * n)(*[int(e.cuda_event) for e in bucket_events])
    _check(lib().lamp_unet_train_step_buckets(net, _ptr(weights), _ptr(biases), C.byref(_td(x)), _ptr(labels), _ptr(loss),
                                              _ptr(grad_w), _ptr(grad_b), _ptr(probs), p, nbytes, _stream(), starts, n, events),
           "lamp_unet_train_step_buckets")


def _i3(v):
    return (C.c_int32 * 3)(*v)


def lamp_sliding_window_num_patches(d, h, w, patch, overlap):
    return lib().lamp_sliding_window_num_patches(d, h, w, _i3(patch), overlap)


def lamp_sliding_window_partial(net, weights, biases, volume, patch, overlap, sw_batch, window, first_patch, num_patches,
                                sums_planar, weight_sums, ws):
    p, nbytes = _ws(ws)
    _check(lib().lamp_sliding_window_partial(net, _ptr(weights), _ptr(biases), C.byref(_td(volume)), _i3(patch), overlap,
                                             sw_batch, window, first_patch, num_patches, _ptr(sums_planar),
                                             _ptr(weight_sums), p, nbytes, _stream()), "lamp_sliding_window_partial")


def lamp_sliding_window_finish(sums_planar, weight_sums, k, voxels, write_probs, argmax):
    _check(lib().lamp_sliding_window_finish(_ptr(sums_planar), _ptr(weight_sums), k, voxels, 1 if write_probs else 0,
                                            _ptr(argmax), _stream()), "lamp_sliding_window_finish")


def lamp_sliding_window_workspace_bytes(net, d, h, w, patch, overlap, sw_batch):
    return lib().lamp_sliding_window_workspace_bytes(net, d, h, w, _i3(patch), overlap, sw_batch)


def lamp_sliding_window_infer(net, weights, biases, volume, patch, overlap, sw_batch, window, probs_planar, argmax, ws):
    p, nbytes = _ws(ws)
    _check(lib().lamp_sliding_window_infer(net, _ptr(weights), _ptr(biases), C.byref(_td(volume)), _i3(patch), overlap,
                                           sw_batch, window, _ptr(probs_planar), _ptr(argmax), p, nbytes, _stream()),
           "lamp_sliding_window_infer")


def lamp_overlap_add(patch_probs, k, d, h, w, patch, overlap, window, probs_planar, argmax):
    _check(lib().lamp_overlap_add(_ptr(patch_probs), k, d, h, w, _i3(patch), overlap, window, _ptr(probs_planar),
                                  _ptr(argmax), _stream()), "lamp_overlap_add")


def lamp_se_squeeze(y, mu_rstd, sums):
    _check(lib().lamp_se_squeeze(C.byref(_td(y)), _ptr(mu_rstd), _ptr(sums), _stream()), "lamp_se_squeeze")


def lamp_se_excite(sums, voxels_per_sample, n, c, cr, w1, b1, w2, b2, e, hidden, mean):
    _check(lib().lamp_se_excite(_ptr(sums), voxels_per_sample, n, c, cr, _ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2), _ptr(e),
                                _ptr(hidden), _ptr(mean), _stream()), "lamp_se_excite")


def lamp_se_apply_fwd(y, mu_rstd, e, residual, out):
    _check(lib().lamp_se_apply_fwd(C.byref(_td(y)), _ptr(mu_rstd), _ptr(e), C.byref(_td(residual)) if residual is not None else None,
                                   C.byref(_td(out)), _stream()), "lamp_se_apply_fwd")


def lamp_se_bwd_reduce(dout, y, mu_rstd, de_sums):
    _check(lib().lamp_se_bwd_reduce(C.byref(_td(dout)), C.byref(_td(y)), _ptr(mu_rstd), _ptr(de_sums), _stream()),
           "lamp_se_bwd_reduce")


def lamp_se_excite_bwd(de_sums, voxels_per_sample, n, c, cr, e, hidden, mean, w1, w2, ds_over_v, dw1, db1, dw2, db2):
    _check(lib().lamp_se_excite_bwd(_ptr(de_sums), voxels_per_sample, n, c, cr, _ptr(e), _ptr(hidden), _ptr(mean), _ptr(w1),
                                    _ptr(w2), _ptr(ds_over_v), _ptr(dw1), _ptr(db1), _ptr(dw2), _ptr(db2), _stream()),
           "lamp_se_excite_bwd")


def lamp_se_apply_bwd(dout, e, ds_over_v, dz):
    _check(lib().lamp_se_apply_bwd(C.byref(_td(dout)), _ptr(e), _ptr(ds_over_v), C.byref(_td(dz)), _stream()), "lamp_se_apply_bwd")


# --- 8-bit layers, block norms, distillation -----------------------------------------------------------------------
# The descriptors below hold the tensors they point at, and the calls refuse (ValueError) tensors of another type, size or
# device than the entry point reads: a pointer alone would not show it.
_FP8_TYPES = (torch.uint8, torch.float8_e4m3fn)


def _vec(t, n, what, dev, dtype=torch.float32):
    """Device pointer of a contiguous vector of n elements (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{what}: want a contiguous {dtype} tensor of {n} elements on cuda:{dev}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


_VIEW_TYPES = {torch.bfloat16: LAMP_BF16, torch.float32: LAMP_F32}


def _view(x, dev, what):
    """Descriptor of a tensor argument (torch tensor on the current device, or a Tensor); None stays None."""
    if x is None:
        return x
    if isinstance(x, Tensor):
        if getattr(x, "dev", dev) != dev:
            raise ValueError(f"{what}: descriptor of a tensor on device {x.dev}, the current device is cuda:{dev}")
        return x
    s, dt = x.shape, _VIEW_TYPES.get(x.dtype)
    if dt is None or len(s) != 5 or x.get_device() != dev or not x.is_contiguous():
        raise ValueError(f"{what}: want a contiguous bf16 or fp32 tensor [n, d, h, w, c] on cuda:{dev}, got {tuple(s)} {x.dtype} on {x.device}")
    n, d, h, w, c = s
    return Tensor(x.data_ptr(), dt, n, d, h, w, c, c, 0)


def _byref(s):
    return None if s is None else C.byref(s)


def fp8_operand(q, scale, rows=None, k=None, tile_scale=False) -> Fp8Operand:
    """Operand [rows][k] of lamp_gemm_fp8: q uint8 or float8_e4m3fn [rows, pitch], scale fp32 [ceil(k/128), pitch]."""
    dev = q.get_device()
    if q.dtype not in _FP8_TYPES or scale.dtype is not torch.float32 or dev < 0 or scale.get_device() != dev:
        raise ValueError("fp8_operand: q is a CUDA uint8 or float8_e4m3fn matrix, scale an fp32 matrix on the same device")
    (qr, qc), (sr, sc), (qp, q1), (sp, s1) = q.shape, scale.shape, q.stride(), scale.stride()
    if rows is None:
        rows = qr
    if k is None:
        k = qc
    if rows > qr or k > qc or q1 != 1 or s1 != 1 or sr * 128 < k or sc < ((rows + 127) // 128 if tile_scale else rows):
        raise ValueError(f"fp8_operand: [{rows}, {k}] does not fit q {tuple(q.shape)} and scale {tuple(scale.shape)}")
    # the stride of an axis of one element says nothing: the pitch only has to cover the row
    if qr <= 1:
        qp = (max(qp, qc) + 15) // 16 * 16
    if sr <= 1:
        sp = max(sp, sc)
    o = Fp8Operand(q.data_ptr(), qp, scale.data_ptr(), sp, rows, k, 1 if tile_scale else 0)
    o.keep, o.dev = (q, scale), dev
    return o


def _operand(o, dev, what):
    if getattr(o, "dev", dev) != dev:
        raise ValueError(f"{what}: on cuda:{o.dev}, the current device is cuda:{dev}")
    return C.byref(o)


def lamp_fp8_quantize(x, out: Fp8Operand, transpose=False):
    dev = torch.cuda.current_device()
    _check(lib().lamp_fp8_quantize(_byref(_view(x, dev, "x")), 1 if transpose else 0, _operand(out, dev, "out"), _raw_stream(dev)), "lamp_fp8_quantize")


def lamp_gemm_fp8(a: Fp8Operand, b: Fp8Operand, y, bias=None):
    dev = torch.cuda.current_device()
    _check(lib().lamp_gemm_fp8(_operand(a, dev, "a"), _operand(b, dev, "b"), _vec(bias, b.rows, "bias", dev), _byref(_view(y, dev, "y")),
                               _raw_stream(dev)), "lamp_gemm_fp8")


def block_norm(rms=False, eps=1e-5, post_w=None, post_b=None, pre_w=None, pre_b=None, gate=None, gate_logits=None,
               res_scale=None) -> BlockNorm:
    """Parameters of lamp_block_norm_fwd / _bwd: fp32 vectors [c] (gate: [n, c]), gate_logits a tensor like y."""
    c = dev = None                                                  # of the vectors, for the calls to check
    ptr = []
    for v in (post_w, post_b, pre_w, pre_b, res_scale):
        if v is None:
            ptr.append(None)
            continue
        if c is None:
            c, dev = v.numel(), v.get_device()
        ptr.append(_vec(v, c, "block_norm", dev))
    g = view = gate_shape = None
    if gate is not None:
        gate_shape = (tuple(gate.shape), gate.get_device())
        g = _vec(gate, gate.numel(), "gate", gate_shape[1])
    if gate_logits is not None:
        view = _view(gate_logits, gate_logits.get_device() if torch.is_tensor(gate_logits) else getattr(gate_logits, "dev", None), "gate_logits")
    p = BlockNorm(1 if rms else 0, eps, ptr[0], ptr[1], ptr[2], ptr[3], g, None if view is None else C.pointer(view), ptr[4])
    p.c, p.dev, p.gate_shape, p.logits = c, dev, gate_shape, gate_logits
    p.keep = (post_w, post_b, pre_w, pre_b, res_scale, gate, view)
    return p


def _norm_params(p, shape, dev):
    """The parameters, checked against the shape of the call's tensors."""
    if p.c is not None and (p.c != shape.c or p.dev != dev):
        raise ValueError(f"block_norm: vectors of {p.c} on cuda:{p.dev}, the tensors have {shape.c} channels on cuda:{dev}")
    if p.gate_shape is not None and (p.gate_shape[1] != dev or not _per_sample(p.gate_shape[0], shape)):
        raise ValueError(f"block_norm: gate {p.gate_shape[0]} on cuda:{p.gate_shape[1]}, want [{shape.n}, {shape.c}] on cuda:{dev}")
    if p.logits is not None and (p.logits.get_device() if torch.is_tensor(p.logits) else getattr(p.logits, "dev", dev)) != dev:
        raise ValueError(f"block_norm: gate_logits on another device than the current one, cuda:{dev}")
    return C.byref(p)


def _per_sample(s, shape):
    """Whether s is [n, c], with axes of one element left out or added between the two."""
    n, c = shape.n, shape.c
    return s == (n, c) or (len(s) > 0 and s[-1] == c and [i for i in s[:-1] if i != 1] == ([n] if n != 1 else []))


def lamp_block_norm_fwd(p: BlockNorm, y, x, out, h=None, h_fp8=None):
    dev = torch.cuda.current_device()
    vx = _view(x, dev, "x")
    _check(lib().lamp_block_norm_fwd(_norm_params(p, vx, dev), _byref(_view(y, dev, "y")), C.byref(vx), _byref(_view(out, dev, "out")),
                                     _byref(_view(h, dev, "h")), None if h_fp8 is None else _operand(h_fp8, dev, "h_fp8"), _raw_stream(dev)),
           "lamp_block_norm_fwd")


def lamp_block_norm_bwd_workspace_bytes(t, p: BlockNorm):
    dev = torch.cuda.current_device()
    vt = _view(t, dev, "t")
    return lib().lamp_block_norm_bwd_workspace_bytes(C.byref(vt), _norm_params(p, vt, dev))


def lamp_block_norm_bwd(p: BlockNorm, y, t, dout, dh, dx, dy, ws=None, dgate_logits=None, dpost_w=None, dpost_b=None, dpre_w=None,
                        dpre_b=None, dgate=None, dres_scale=None):
    dev = torch.cuda.current_device()
    vt = _view(t, dev, "t")
    c = vt.c
    if dgate is not None and not _per_sample(dgate.shape, vt):
        raise ValueError(f"dgate: want [{vt.n}, {c}], got {tuple(dgate.shape)}")
    g = BlockNormGrads(_vec(dpost_w, c, "dpost_w", dev), _vec(dpost_b, c, "dpost_b", dev), _vec(dpre_w, c, "dpre_w", dev),
                       _vec(dpre_b, c, "dpre_b", dev), _vec(dgate, vt.n * c, "dgate", dev), _vec(dres_scale, c, "dres_scale", dev))
    if ws is not None and ws.get_device() != dev:
        raise ValueError(f"ws: on {ws.device}, the current device is cuda:{dev}")
    w, nbytes = _ws(ws)
    _check(lib().lamp_block_norm_bwd(_norm_params(p, vt, dev), _byref(_view(y, dev, "y")), C.byref(vt), _byref(_view(dout, dev, "dout")),
                                     _byref(_view(dh, dev, "dh")), _byref(_view(dx, dev, "dx")), _byref(_view(dy, dev, "dy")),
                                     _byref(_view(dgate_logits, dev, "dgate_logits")), C.byref(g), w, nbytes, _raw_stream(dev)),
           "lamp_block_norm_bwd")


def teacher_topk(idx, logits, temperature=1.0, lse=None) -> TeacherTopk:
    """The teacher's k listed classes per row: idx int32 [rows, k], logits fp32 [rows, k], lse fp32 [rows] or None."""
    t = TeacherTopk()
    if idx.dim() != 2 or logits.shape != idx.shape or (lse is not None and lse.numel() != idx.shape[0]):
        raise ValueError(f"teacher_topk: idx and logits are matrices [rows, k], lse a vector [rows]; got {tuple(idx.shape)}, {tuple(logits.shape)}"
                         + ("" if lse is None else f", {tuple(lse.shape)}"))
    t.k, t.temperature = idx.shape[1], temperature
    t.keep = (idx, logits, lse)
    return t


def _teacher(t, z, dev):
    rows = z.n * z.d * z.h * z.w
    idx, logits, lse = t.keep
    t.idx = _vec(idx, rows * t.k, "idx", dev, torch.int32)
    t.logits = _vec(logits, rows * t.k, "logits", dev)
    t.lse = _vec(lse, rows, "lse", dev)
    return C.byref(t), rows


def lamp_distill_topk_workspace_bytes(z):
    return lib().lamp_distill_topk_workspace_bytes(C.byref(_td(z)))


def _scratch(ws, dev):
    if ws is not None and ws.get_device() != dev:
        raise ValueError(f"ws: on {ws.device}, the current device is cuda:{dev}")
    return _ws(ws)


def lamp_distill_topk_fwd(z, teacher: TeacherTopk, row_weight=None, loss_rows=None, lse=None, loss=None, ws=None):
    dev = torch.cuda.current_device()
    vz = _view(z, dev, "z")
    t, rows = _teacher(teacher, vz, dev)
    w, nbytes = _scratch(ws, dev)
    _check(lib().lamp_distill_topk_fwd(C.byref(vz), t, _vec(row_weight, rows, "row_weight", dev), _vec(loss_rows, rows, "loss_rows", dev),
                                       _vec(lse, rows, "lse", dev), _vec(loss, 1, "loss", dev), w, nbytes, _raw_stream(dev)), "lamp_distill_topk_fwd")


def lamp_distill_topk_bwd(z, teacher: TeacherTopk, row_grad, lse, dz):
    dev = torch.cuda.current_device()
    vz = _view(z, dev, "z")
    t, rows = _teacher(teacher, vz, dev)
    _check(lib().lamp_distill_topk_bwd(C.byref(vz), t, _vec(row_grad, rows, "row_grad", dev), _vec(lse, rows, "lse", dev),
                                       _byref(_view(dz, dev, "dz")), _raw_stream(dev)), "lamp_distill_topk_bwd")


def lamp_distill_topk_fwd_bwd(z, teacher: TeacherTopk, row_weight, loss_rows, loss, dz, ws=None):
    dev = torch.cuda.current_device()
    vz = _view(z, dev, "z")
    t, rows = _teacher(teacher, vz, dev)
    w, nbytes = _scratch(ws, dev)
    _check(lib().lamp_distill_topk_fwd_bwd(C.byref(vz), t, _vec(row_weight, rows, "row_weight", dev), _vec(loss_rows, rows, "loss_rows", dev),
                                           _vec(loss, 1, "loss", dev), _byref(_view(dz, dev, "dz")), w, nbytes, _raw_stream(dev)),
           "lamp_distill_topk_fwd_bwd")


def lamp_rmsprop_step(grad, master, v, param_bf16=None, lr=1e-3, alpha=0.99, eps=1e-8):
    _check(lib().lamp_rmsprop_step(grad.numel(), _ptr(grad), _ptr(master), _ptr(v), _ptr(param_bf16), lr, alpha, eps,
                                   _stream()), "lamp_rmsprop_step")


# --- group norm with an activation ---------------------------------------------------------------------------------
ACTIVATIONS = {"none": 0, "leaky_relu": 1, "silu": 2, "gelu": 3}


def _space(ws, dev):
    """Address and bytes of a scratch tensor (None: none)."""
    if ws is None:
        return None, 0
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError(f"ws: want a contiguous tensor on cuda:{dev}, got {tuple(ws.shape)} on {ws.device}")
    return ws.data_ptr(), ws.nbytes


def group_norm(groups, w=None, b=None, act="none", slope=0.0, eps=1e-5) -> GroupNorm:
    """Parameters of lamp_group_norm_act_fwd / _bwd: w, b fp32 [c]; act a name of ACTIVATIONS ("leaky_relu" with slope 0 is ReLU)."""
    c = dev = None
    v = b if w is None else w
    if v is not None:
        c, dev = v.numel(), v.get_device()
    a = ACTIVATIONS.get(act)
    if a is None:
        raise ValueError(f"group_norm: act is one of {', '.join(ACTIVATIONS)}, got {act!r}")
    p = GroupNorm(groups, a, slope, eps, _vec(w, c, "group_norm", dev), _vec(b, c, "group_norm", dev))
    p.c, p.dev, p.keep = c, dev, (w, b)
    return p


def _group_params(p, shape, dev):
    if getattr(p, "c", None) is not None and (p.c != shape.c or p.dev != dev):
        raise ValueError(f"group_norm: vectors of {p.c} on cuda:{p.dev}, the tensors have {shape.c} channels on cuda:{dev}")
    return C.byref(p)


def lamp_group_norm_workspace_bytes(p: GroupNorm, x):
    return lib().lamp_group_norm_workspace_bytes(C.byref(p), C.byref(_td(x)))


def lamp_group_norm_act_fwd(p: GroupNorm, x, z, mean_rstd, ws=None, stats=None):
    dev = _device()
    vx = _view(x, dev, "x")
    w, nbytes = _space(ws, dev)
    _check(lib().lamp_group_norm_act_fwd(_group_params(p, vx, dev), C.byref(vx), _vec(stats, 2 * vx.n * vx.c, "stats", dev, torch.float64),
                                         _byref(_view(z, dev, "z")), _vec(mean_rstd, 2 * vx.n * p.groups, "mean_rstd", dev), w, nbytes,
                                         _raw_stream(dev)), "lamp_group_norm_act_fwd")


def lamp_group_norm_act_bwd(p: GroupNorm, dz, x, mean_rstd, dx, dw=None, db=None, ws=None):
    dev = _device()
    vx = _view(x, dev, "x")
    w, nbytes = _space(ws, dev)
    _check(lib().lamp_group_norm_act_bwd(_group_params(p, vx, dev), _byref(_view(dz, dev, "dz")), C.byref(vx),
                                         _vec(mean_rstd, 2 * vx.n * p.groups, "mean_rstd", dev), _byref(_view(dx, dev, "dx")),
                                         _vec(dw, vx.c, "dw", dev), _vec(db, vx.c, "db", dev), w, nbytes, _raw_stream(dev)), "lamp_group_norm_act_bwd")


# --- 4-bit layers --------------------------------------------------------------------------------------------------
_U8 = torch.uint8


def lamp_fp4_scale_bytes(rows, k, block=32):
    return lib().lamp_fp4_scale_bytes(rows, k, block)


def fp4_operand(q, scale, rows=None, k=None, block=32, tensor_scale=None) -> Fp4Operand:
    """Operand [rows][k] of lamp_gemm_fp4: q uint8 [rows, pitch], two codes a byte; scale uint8, lamp_fp4_scale_bytes(rows, k, block) of them in
    their tiles; tensor_scale fp32 scalar on the device or None."""
    dev = q.get_device()
    if q.dtype is not _U8 or scale.dtype is not _U8 or dev < 0 or scale.get_device() != dev or q.dim() != 2 or not scale.is_contiguous():
        raise ValueError("fp4_operand: q is a CUDA uint8 matrix, scale a contiguous uint8 tensor on the same device")
    (qr, qc), (qp, q1) = q.shape, q.stride()
    if rows is None:
        rows = qr
    if k is None:
        k = 2 * qc
    if block != 32 and block != 16:
        raise ValueError(f"fp4_operand: blocks of 16 or 32, got {block}")
    if rows < 0 or k < 0 or rows > qr or k > 2 * qc or (q1 != 1 and qc > 1) or scale.numel() < (rows + 127) // 128 * ((k + 4 * block - 1) // (4 * block)) * 512:
        raise ValueError(f"fp4_operand: [{rows}, {k}] in blocks of {block} does not fit q {tuple(q.shape)} and {scale.numel()} scales")
    # the stride of an axis of one element says nothing: the pitch only has to cover the row
    if qr <= 1:
        qp = (max(qp, qc) + 15) // 16 * 16
    o = Fp4Operand(q.data_ptr(), qp, scale.data_ptr(), None if tensor_scale is None else _vec(tensor_scale, 1, "tensor_scale", dev), rows, k, block)
    o.keep, o.dev = (q, scale, tensor_scale), dev
    return o


def lamp_fp4_quantize(x, out: Fp4Operand, transpose=False):
    dev = _device()
    _check(lib().lamp_fp4_quantize(_byref(_view(x, dev, "x")), 1 if transpose else 0, _operand(out, dev, "out"), _raw_stream(dev)), "lamp_fp4_quantize")


def lamp_fp4_dequantize(op: Fp4Operand, y, transpose=False):
    dev = _device()
    _check(lib().lamp_fp4_dequantize(_operand(op, dev, "op"), 1 if transpose else 0, _byref(_view(y, dev, "y")), _raw_stream(dev)), "lamp_fp4_dequantize")


def lamp_gemm_fp4(a: Fp4Operand, b: Fp4Operand, y, bias=None):
    dev = _device()
    _check(lib().lamp_gemm_fp4(_operand(a, dev, "a"), _operand(b, dev, "b"), _vec(bias, b.rows, "bias", dev), _byref(_view(y, dev, "y")),
                               _raw_stream(dev)), "lamp_gemm_fp4")


# --- gradient clipping ---------------------------------------------------------------------------------------------
class GradList:
    """The tensors of lamp_grad_norm / lamp_grad_clip, described once and used for many steps; holds them."""

    def __init__(self, tensors, outs):
        self.keep = (tensors, outs)
        self.count, self.dev = len(tensors), tensors[0].get_device() if tensors else None
        self.array = (Grad * max(1, self.count))()
        for i, (g, o) in enumerate(zip(tensors, outs)):
            dt = _VIEW_TYPES.get(g.dtype)
            if dt is None or not g.is_contiguous() or g.get_device() != self.dev or self.dev < 0:
                raise ValueError(f"grad_list: tensor {i}: want a contiguous bf16 or fp32 tensor on one CUDA device, got {tuple(g.shape)} {g.dtype} on {g.device}")
            if o is not g and (o.dtype is not g.dtype or o.numel() != g.numel() or not o.is_contiguous() or o.get_device() != self.dev):
                raise ValueError(f"grad_list: output {i}: want a contiguous {g.dtype} tensor of {g.numel()} elements on {g.device}, got {tuple(o.shape)} {o.dtype} on {o.device}")
            self.array[i] = Grad(g.data_ptr(), o.data_ptr(), g.numel(), dt)
        # what is written must not be part of anything else: sorted by address, each range against the furthest one in front of it
        ranges = []
        for i, (g, o) in enumerate(zip(tensors, outs)):
            if g.numel():
                size = g.numel() * g.element_size()
                a, b = g.data_ptr(), o.data_ptr()
                ranges.append((a, a + size, a == b, i))
                if a != b:
                    ranges.append((b, b + size, True, i))
        end, written_end = 0, 0                                       # of all ranges so far, of the written ones
        for a, b, written, i in sorted(ranges):
            if a < written_end or (written and a < end):
                raise ValueError(f"grad_list: tensor {i} or its output overlaps another one that is written")
            end = max(end, b)
            if written:
                written_end = max(written_end, b)


def grad_list(tensors, outs=None) -> GradList:
    """tensors: gradients (bf16 or fp32, contiguous); outs: where lamp_grad_clip writes, None for in place.

    Made once for buffers that stay from step to step: the checks and the search for overlaps run on the host, about 2 us a tensor (0.13 ms for 62,
    0.5 ms for 301), and the list holds the memory it was made of.  Gradients that are freed and made anew need a new list every step."""
    tensors = list(tensors)
    outs = tensors if outs is None else list(outs)
    if len(outs) != len(tensors):
        raise ValueError(f"grad_list: {len(tensors)} tensors and {len(outs)} outputs")
    return GradList(tensors, outs)


def _grads(g, dev):
    if g.dev is not None and g.dev != dev:
        raise ValueError(f"grads: on cuda:{g.dev}, the current device is cuda:{dev}")
    return g.array


def lamp_grad_norm_workspace_bytes(grads: GradList):
    return lib().lamp_grad_norm_workspace_bytes(grads.array, grads.count)


def lamp_grad_norm(grads: GradList, max_norm, norm, factor=None, ws=None):
    dev = _device()
    w, nbytes = _space(ws, dev)
    _check(lib().lamp_grad_norm(_grads(grads, dev), grads.count, max_norm, _vec(norm, 1, "norm", dev), _vec(factor, 1, "factor", dev), w, nbytes,
                                _raw_stream(dev)), "lamp_grad_norm")


def lamp_grad_clip(grads: GradList, max_norm, norm, factor, ws=None):
    dev = _device()
    w, nbytes = _space(ws, dev)
    _check(lib().lamp_grad_clip(_grads(grads, dev), grads.count, max_norm, _vec(norm, 1, "norm", dev), _vec(factor, 1, "factor", dev), w, nbytes,
                                _raw_stream(dev)), "lamp_grad_clip")


def lamp_rmsprop_step_scaled(grad, grad_scale, master, v, param_bf16=None, lr=1e-3, alpha=0.99, eps=1e-8):
    """lamp_rmsprop_step with the gradients times grad_scale (fp32 scalar on the device, as lamp_grad_norm leaves it in factor)."""
    dev = _device()
    n = grad.numel()
    _check(lib().lamp_rmsprop_step_scaled(n, _vec(grad, n, "grad", dev), _vec(grad_scale, 1, "grad_scale", dev), _vec(master, n, "master", dev),
                                          _vec(v, n, "v", dev), _vec(param_bf16, n, "param_bf16", dev, torch.bfloat16), lr, alpha, eps,
                                          _raw_stream(dev)), "lamp_rmsprop_step_scaled")


def lamp_get_async_status():
    return lib().lamp_get_async_status(_stream())


def lamp_selftest_wait_timeout():
    _check(lib().lamp_selftest_wait_timeout(_stream()), "lamp_selftest_wait_timeout")


def lamp_version():
    return lib().lamp_version().decode()
