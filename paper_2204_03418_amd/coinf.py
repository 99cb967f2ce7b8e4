"""ctypes binding of libcoinf.so (include/coinf.h).

Argument marshalling only: every step of the computation runs in the HIP
kernels behind the C ABI.  Tensors are PyTorch device tensors (the caller's
memory); the stream is PyTorch's current stream.  Importing this module loads
the library and raises ImportError when it has not been built; there is no
fallback path.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcoinf.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"libcoinf.so is not built ({LIB_PATH}); run __graft_entry__.build()")
lib = ctypes.CDLL(LIB_PATH)

# ---------------------------------------------------------------- constants
CO_OK, CO_EMPTY, CO_EINVAL, CO_ENOTSUP, CO_ESTATE, CO_EHIP = 0, 1, -1, -2, -3, -4
CO_ESCRATCH = -5
CO_F32, CO_BF16 = 0, 1
CO_ALGO_AUTO, CO_ALGO_DIRECT, CO_ALGO_GEMM, CO_ALGO_DEPTHWISE, CO_ALGO_GEMM_REG = 0, 1, 2, 3, 4
CO_ALGO_GEMM_WS = 5
CO_ACT_NONE, CO_ACT_RELU, CO_ACT_SILU = 0, 1, 2
CO_NORM_NONE, CO_NORM_BEFORE, CO_NORM_AFTER = 0, 1, 2
CO_POOL_AVG, CO_POOL_MAX = 0, 1
CO_ROTARY_HALF, CO_ROTARY_INTERLEAVED = 0, 1
CO_ROTARY_PLAIN, CO_ROTARY_LINEAR, CO_ROTARY_BASE, CO_ROTARY_PARTS = 0, 1, 2, 3
CO_MAX_TAPS = 64
CO_TAP_NONE, CO_TAP_START, CO_TAP_ACC, CO_TAP_EMIT, CO_TAP_EMIT_FRESH = 0, 1, 2, 3, 4

ALGOS = {"auto": CO_ALGO_AUTO, "direct": CO_ALGO_DIRECT, "gemm": CO_ALGO_GEMM,
         "depthwise": CO_ALGO_DEPTHWISE, "gemm_reg": CO_ALGO_GEMM_REG,
         "gemm_ws": CO_ALGO_GEMM_WS}
DTYPES = {torch.float32: CO_F32, torch.bfloat16: CO_BF16}

i32, i64, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
I32x2, I32x3 = i32 * 2, i32 * 3


class ConvDesc(ctypes.Structure):
    _fields_ = [("spatial_dims", i32), ("batch", i32), ("in_channels", i32),
                ("out_channels", i32), ("groups", i32), ("in_size", I32x2),
                ("kernel", I32x3), ("stride", I32x3), ("padding", I32x3),
                ("dilation", I32x3), ("has_bias", i32), ("dtype", i32), ("algo", i32)]


class ConvInfo(ctypes.Structure):
    _fields_ = [("receptive_field", i32), ("delay", i32), ("out_size", I32x2),
                ("ring_slots", i32), ("algo", i32), ("state_bytes", i64)]


class StepPlan(ctypes.Structure):
    _fields_ = [("emit", i32), ("n_taps", i32), ("out_index", i64),
                ("action", ctypes.c_int8 * CO_MAX_TAPS), ("slot", i32 * CO_MAX_TAPS),
                ("target", i64 * CO_MAX_TAPS)]


class PoolDesc(ctypes.Structure):
    _fields_ = [("kind", i32), ("spatial_dims", i32), ("batch", i32), ("channels", i32),
                ("in_size", I32x2), ("kernel", I32x3), ("stride", I32x3), ("padding", I32x3),
                ("dilation", I32x3), ("count_include_pad", i32), ("dtype", i32)]


class PoolInfo(ctypes.Structure):
    _fields_ = [("receptive_field", i32), ("delay", i32), ("out_size", I32x2),
                ("fifo_slots", i32), ("reserved", i32), ("state_bytes", i64)]


class DelayDesc(ctypes.Structure):
    _fields_ = [("batch", i32), ("channels", i32), ("frame_elems", i32), ("delay", i32),
                ("dtype", i32)]


class PoolPlan(ctypes.Structure):
    _fields_ = [("emit", i32), ("n_taps", i32), ("out_index", i64), ("write_slot", i32),
                ("reserved", i32), ("src", i32 * CO_MAX_TAPS)]


def _sig(name, res, args):
    f = getattr(lib, name)
    f.restype = res
    f.argtypes = args
    return f


CD, CI, PD, PI = (ctypes.POINTER(ConvDesc), ctypes.POINTER(ConvInfo),
                  ctypes.POINTER(PoolDesc), ctypes.POINTER(PoolInfo))
pi32, pi64, pvp = ctypes.POINTER(i32), ctypes.POINTER(i64), ctypes.POINTER(vp)

co_status_str = _sig("co_status_str", ctypes.c_char_p, [i32])
co_conv_query = _sig("co_conv_query", i32, [CD, CI])
co_conv_plan_step = _sig("co_conv_plan_step", i32, [CD, i64, i32, ctypes.POINTER(StepPlan)])
co_conv_init_state = _sig("co_conv_init_state", i32, [CD, vp, vp, vp, i64, vp, pvp])
co_conv_forward_step = _sig("co_conv_forward_step", i32, [vp, vp, vp, i32, vp])
co_conv_forward_steps = _sig("co_conv_forward_steps", i32,
                             [vp, vp, i32, vp, i32, i32, i32, vp, pi32])
co_conv_forward = _sig("co_conv_forward", i32, [CD, vp, vp, vp, i32, vp, vp])
co_conv_clip_frames = _sig("co_conv_clip_frames", i32, [CD, i32, pi32])
co_conv_clean_state = _sig("co_conv_clean_state", i32, [vp, vp])
co_conv_get_steps = _sig("co_conv_get_steps", i32, [vp, pi64])
co_conv_attach_state = _sig("co_conv_attach_state", i32, [CD, vp, i64, i64, vp, pvp])
co_conv_destroy = _sig("co_conv_destroy", i32, [vp])
co_conv_algo_name = _sig("co_conv_algo_name", ctypes.c_char_p, [vp])
co_conv_steps_fused = _sig("co_conv_steps_fused", i32, [vp, i32, i32, pi32])
co_conv_steps_route = _sig("co_conv_steps_route", i32, [CD, i32, i32, i32, pi32])
co_conv_forward_steps_noalloc = _sig("co_conv_forward_steps_noalloc", i32,
                                     [vp, vp, i32, vp, i32, i32, i32, vp, pi32])
co_conv_scratch_bytes = _sig("co_conv_scratch_bytes", i32, [pi64])
co_conv_out_frames = _sig("co_conv_out_frames", i32, [CD, i64, i32, i32, pi32])
co_pool_query = _sig("co_pool_query", i32, [PD, PI])
co_pool_plan_step = _sig("co_pool_plan_step", i32, [PD, i64, ctypes.POINTER(PoolPlan)])
co_pool_init_state = _sig("co_pool_init_state", i32, [PD, vp, i64, vp, pvp])
co_pool_forward_step = _sig("co_pool_forward_step", i32, [vp, vp, vp, i32, vp])
co_pool_forward_steps = _sig("co_pool_forward_steps", i32,
                             [vp, vp, i32, vp, i32, i32, i32, vp, pi32])
co_pool_forward = _sig("co_pool_forward", i32, [PD, vp, i32, vp, vp])
co_pool_steps_fused = _sig("co_pool_steps_fused", i32, [vp, i32, i32, pi32])
co_pool_out_frames = _sig("co_pool_out_frames", i32, [PD, i64, i32, i32, pi32])
co_pool_clip_frames = _sig("co_pool_clip_frames", i32, [PD, i32, pi32])
co_pool_clean_state = _sig("co_pool_clean_state", i32, [vp, vp])
co_pool_get_steps = _sig("co_pool_get_steps", i32, [vp, pi64])
co_pool_attach_state = _sig("co_pool_attach_state", i32, [PD, vp, i64, i64, vp, pvp])
co_pool_destroy = _sig("co_pool_destroy", i32, [vp])
DD = ctypes.POINTER(DelayDesc)
co_delay_query = _sig("co_delay_query", i32, [DD, pi64])
co_delay_init_state = _sig("co_delay_init_state", i32, [DD, vp, i64, vp, pvp])
co_delay_forward_step = _sig("co_delay_forward_step", i32, [vp, vp, vp, i32, vp])
co_delay_add_step = _sig("co_delay_add_step", i32, [vp, vp, vp, vp, i32, vp])
co_delay_forward_steps = _sig("co_delay_forward_steps", i32,
                              [vp, vp, i32, vp, i32, i32, vp, pi32])
co_delay_add_steps = _sig("co_delay_add_steps", i32, [vp, vp, i32, vp, i32, vp, i32, vp])
co_add_frames = _sig("co_add_frames", i32, [vp, vp, vp, i32, i32, i32, i32, i32, i32, vp])
co_delay_clean_state = _sig("co_delay_clean_state", i32, [vp, vp])
co_delay_get_steps = _sig("co_delay_get_steps", i32, [vp, pi64])
co_delay_destroy = _sig("co_delay_destroy", i32, [vp])
co_chain_delay = _sig("co_chain_delay", i32, [i32, pi32, pi32, pi32, pi64, pi64, pi64, pi64])
co_convpool_bind = _sig("co_convpool_bind", i32, [vp, vp, pvp])
co_convpool_forward_step = _sig("co_convpool_forward_step", i32, [vp, vp, vp, i32, vp])
co_convpool_forward_steps = _sig("co_convpool_forward_steps", i32,
                                 [vp, vp, i32, vp, i32, i32, vp, pi32])
co_convpool_destroy = _sig("co_convpool_destroy", i32, [vp])
pf32, f32 = ctypes.POINTER(ctypes.c_float), ctypes.c_float
co_conv_init_state_bn = _sig("co_conv_init_state_bn", i32,
                             [CD, vp, vp, vp, vp, vp, vp, f32, vp, i64, vp, pvp])
co_conv_fold_bn = _sig("co_conv_fold_bn", i32, [CD, vp, vp, vp, vp, vp, vp, f32, vp, vp, vp])
co_act_forward = _sig("co_act_forward", i32, [vp, vp, i64, i32, i32, vp])


class BnParams(ctypes.Structure):
    _fields_ = [("gamma", vp), ("beta", vp), ("mean", vp), ("var", vp), ("eps", ctypes.c_float)]


co_conv_forward_ws = _sig("co_conv_forward_ws", i32,
                          [CD, vp, vp, ctypes.POINTER(BnParams), vp, i32, vp, vp, i64, vp])
co_bneck_bind = _sig("co_bneck_bind", i32, [vp, i32, vp, i32, vp, pvp])
co_bneck_forward_step = _sig("co_bneck_forward_step", i32, [vp, vp, vp, i32, vp])
co_bneck_forward_steps = _sig("co_bneck_forward_steps", i32,
                              [vp, vp, i32, vp, i32, i32, vp, pi32])
co_bneck_workspace_bytes = _sig("co_bneck_workspace_bytes", i32, [vp, i32, pi64])
co_bneck_forward_steps_ws = _sig("co_bneck_forward_steps_ws", i32,
                                 [vp, vp, i32, vp, i32, i32, vp, i64, vp, pi32])
co_bneck_destroy = _sig("co_bneck_destroy", i32, [vp])
co_residual_align = _sig("co_residual_align", i32, [i64, i64, i64, i64, pi64, pi64, pi64])


class Tokens(ctypes.Structure):
    _fields_ = [("data", vp), ("batch_stride", i64), ("token_stride", i64)]


class ShortConvDesc(ctypes.Structure):
    _fields_ = [("batch", i32), ("channels", i32), ("kernel", i32), ("has_bias", i32),
                ("act", i32), ("dtype", i32)]


class ScanDesc(ctypes.Structure):
    _fields_ = [("batch", i32), ("heads", i32), ("head_dim", i32), ("state_size", i32),
                ("groups", i32), ("dt_softplus", i32), ("dtype", i32), ("dt_dtype", i32)]


class ShortConvCall(ctypes.Structure):
    _fields_ = [("weight", vp), ("bias", vp), ("x", Tokens), ("y", Tokens), ("lengths", vp),
                ("state", vp), ("T", i32), ("update_state", i32)]


class ScanCall(ctypes.Structure):
    _fields_ = [("A", vp), ("D", vp), ("dt_bias", vp), ("x", Tokens), ("dt", Tokens),
                ("b", Tokens), ("c", Tokens), ("y", Tokens), ("lengths", vp), ("state", vp),
                ("workspace", vp), ("workspace_bytes", i64), ("T", i32), ("update_state", i32)]


class NormDesc(ctypes.Structure):
    _fields_ = [("batch", i32), ("tokens", i32), ("dim", i32), ("groups", i32), ("gate", i32),
                ("residual", i32), ("dtype", i32), ("residual_dtype", i32), ("eps", f32)]


class NormCall(ctypes.Structure):
    _fields_ = [("x", Tokens), ("gate", Tokens), ("residual", Tokens), ("y", Tokens),
                ("residual_out", Tokens), ("weight", vp), ("scale", vp)]


co_shortconv_query = _sig("co_shortconv_query", i32, [ctypes.POINTER(ShortConvDesc), pi64])
co_shortconv_forward_steps = _sig("co_shortconv_forward_steps", i32,
                                  [ctypes.POINTER(ShortConvDesc), ctypes.POINTER(ShortConvCall),
                                   vp])
co_scan_query = _sig("co_scan_query", i32, [ctypes.POINTER(ScanDesc), pi64])
co_scan_workspace_bytes = _sig("co_scan_workspace_bytes", i32,
                               [ctypes.POINTER(ScanDesc), i32, pi64])
co_scan_forward_steps = _sig("co_scan_forward_steps", i32,
                             [ctypes.POINTER(ScanDesc), ctypes.POINTER(ScanCall), vp])
co_norm_forward = _sig("co_norm_forward", i32,
                       [ctypes.POINTER(NormDesc), ctypes.POINTER(NormCall), vp])
co_norm_forward_lengths = _sig("co_norm_forward_lengths", i32,
                               [ctypes.POINTER(NormDesc), ctypes.POINTER(NormCall), vp, vp])


class RotaryScaling(ctypes.Structure):
    _fields_ = [("kind", i32), ("factor", ctypes.c_double), ("original", ctypes.c_double),
                ("low", ctypes.c_double), ("high", ctypes.c_double)]


class RotaryDesc(ctypes.Structure):
    _fields_ = [("batch", i32), ("heads", I32x2), ("head_dim", i32), ("rotary_dim", i32),
                ("layout", i32), ("dtype", i32), ("magnitude", f32)]


class RotaryCall(ctypes.Structure):
    _fields_ = [("turns", vp), ("positions", vp), ("position_batch_stride", i64),
                ("position_token_stride", i64), ("position_each", i32), ("T", i32),
                ("lengths", vp), ("x", Tokens * 2), ("y", Tokens * 2)]


class PagesDesc(ctypes.Structure):
    _fields_ = [("batch", i32), ("pages", i32), ("page_tokens", i32), ("stream_pages", i32),
                ("layers", i32), ("kv_heads", i32), ("head_dim", i32)]


class PagesInfo(ctypes.Structure):
    _fields_ = [("page_bytes", i64), ("pool_bytes", i64), ("workspace_bytes", i64)]


class Pages(ctypes.Structure):
    _fields_ = [(k, vp) for k in ("pool", "table", "tokens", "first", "refs", "base", "granted",
                                  "refused", "workspace")]


class AttnDesc(ctypes.Structure):
    _fields_ = [("batch", i32), ("heads", i32), ("kv_heads", i32), ("head_dim", i32),
                ("pages", i32), ("page_tokens", i32), ("stream_pages", i32), ("window", i32),
                ("dtype", i32), ("scale", f32)]


class AttnCache(ctypes.Structure):
    _fields_ = [(k, vp) for k in ("pool", "table", "base", "granted", "first")]


_pages_args = [ctypes.POINTER(PagesDesc), ctypes.POINTER(Pages)]
_attn_args = [ctypes.POINTER(AttnDesc), ctypes.POINTER(AttnCache)]
_pTokens = ctypes.POINTER(Tokens)
co_rotary_turns = _sig("co_rotary_turns", i32, [i32, ctypes.c_double,
                                                ctypes.POINTER(RotaryScaling), vp])
co_rotary_forward = _sig("co_rotary_forward", i32,
                         [ctypes.POINTER(RotaryDesc), ctypes.POINTER(RotaryCall), vp])
co_pages_query = _sig("co_pages_query", i32,
                      [ctypes.POINTER(PagesDesc), ctypes.POINTER(PagesInfo)])
co_pages_reserve = _sig("co_pages_reserve", i32, _pages_args + [i32, vp, i32, vp])
co_pages_truncate = _sig("co_pages_truncate", i32, _pages_args + [vp, vp])
co_pages_select = _sig("co_pages_select", i32, _pages_args + [vp, vp])
co_pages_compact = _sig("co_pages_compact", i32, _pages_args + [vp])
co_attn_append = _sig("co_attn_append", i32, _attn_args + [_pTokens, _pTokens, i32, vp])
co_attn_read = _sig("co_attn_read", i32, _attn_args + [vp, _pTokens, _pTokens, i32, vp])
co_attn_workspace_bytes = _sig("co_attn_workspace_bytes", i32,
                               [ctypes.POINTER(AttnDesc), i32, pi64])
co_attn_forward_steps = _sig("co_attn_forward_steps", i32,
                             _attn_args + [_pTokens, _pTokens, i32, vp, i64, vp])


class CoinfError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: {co_status_str(status).decode()} ({status})")


def check(status, what):
    if status < 0:
        raise CoinfError(status, what)
    return status


def _axes(v, nd, fill):
    """Per-axis 3-tuple (time first) from an int or sequence of nd values."""
    v = (int(v),) * nd if isinstance(v, int) else tuple(int(e) for e in v)
    assert len(v) == nd, v
    return v + (fill,) * (3 - nd)


def conv_desc(batch, in_channels, out_channels, kernel, in_size=(), stride=1, padding=0,
              dilation=1, groups=1, has_bias=True, dtype=CO_F32, algo="auto"):
    """Build a ConvDesc; kernel/stride/padding/dilation are time first."""
    sd = len(in_size)
    nd = sd + 1
    d = ConvDesc()
    d.spatial_dims = sd
    d.batch, d.in_channels, d.out_channels, d.groups = batch, in_channels, out_channels, groups
    d.in_size = I32x2(*(tuple(in_size) + (1,) * (2 - sd)))
    d.kernel = I32x3(*_axes(kernel, nd, 1))
    d.stride = I32x3(*_axes(stride, nd, 1))
    d.padding = I32x3(*_axes(padding, nd, 0))
    d.dilation = I32x3(*_axes(dilation, nd, 1))
    d.has_bias = 1 if has_bias else 0
    d.dtype = dtype
    d.algo = ALGOS[algo] if isinstance(algo, str) else int(algo)
    return d


def pool_desc(kind, batch, channels, kernel, in_size=(), stride=None, padding=0, dilation=1,
              count_include_pad=True, dtype=CO_F32):
    sd = len(in_size)
    nd = sd + 1
    d = PoolDesc()
    d.kind = CO_POOL_MAX if kind == "max" else CO_POOL_AVG
    d.spatial_dims = sd
    d.batch, d.channels = batch, channels
    d.in_size = I32x2(*(tuple(in_size) + (1,) * (2 - sd)))
    d.kernel = I32x3(*_axes(kernel, nd, 1))
    d.stride = I32x3(*_axes(kernel if stride is None else stride, nd, 1))
    d.padding = I32x3(*_axes(padding, nd, 0))
    d.dilation = I32x3(*_axes(dilation, nd, 1))
    d.count_include_pad = 1 if count_include_pad else 0
    d.dtype = dtype
    return d


def conv_query(desc):
    info = ConvInfo()
    check(co_conv_query(ctypes.byref(desc), ctypes.byref(info)), "co_conv_query")
    return info


def conv_plan(desc, n, update_state=True):
    p = StepPlan()
    check(co_conv_plan_step(ctypes.byref(desc), n, 1 if update_state else 0, ctypes.byref(p)),
          "co_conv_plan_step")
    return p


def pool_query(desc):
    info = PoolInfo()
    check(co_pool_query(ctypes.byref(desc), ctypes.byref(info)), "co_pool_query")
    return info


def pool_plan(desc, n):
    p = PoolPlan()
    check(co_pool_plan_step(ctypes.byref(desc), n, ctypes.byref(p)), "co_pool_plan_step")
    return p


# A step is a kernel of a few microseconds: what the binding does around it is
# most of a small layer's time.  The handle of the current stream is read
# without building a Stream object (2.9 -> 0.3 us), pointers are plain integers, a
# frame that fits takes one chain of comparisons, and an output the binding
# has just made is not checked (together 9.6 -> 6.1 us a step, 4 -> 8
# channels, one stream).
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    """The HIP stream handle: of the current device's current stream, or of stream."""
    if stream is not None:
        return stream.cuda_stream
    if _current_raw_stream is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _current_raw_stream(_current_device())


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _need(t, dtype, shape, what):
    if t.is_cuda and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return
    if t.device.type != "cuda":
        raise ValueError(f"{what} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{what} has dtype {t.dtype}, expected {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")


class CoConv:
    """A continual ConvNd layer over a device state buffer (co_conv_* ABI).

    weight (C_out, C_in/groups, kT, *kS) and bias (C_out,) are device tensors
    of one dtype (float32 or bfloat16); batch and in_size fix the frame shape
    (B, C_in, *in_size).  kernel geometry comes from weight.shape.  bn =
    (gamma, beta, running_mean, running_var, eps), float32 device tensors of
    C_out and a float, folds an evaluation-mode batch normalisation of the
    output into the layer (co_conv_init_state_bn): every step emits
    BN(conv(x)).
    """

    def __init__(self, weight, bias=None, *, batch, in_size=(), stride=1, padding=0,
                 dilation=1, groups=1, algo="auto", state=None, attach_steps=None, bn=None):
        dt = DTYPES[weight.dtype]
        self.torch_dtype = weight.dtype
        self.desc = conv_desc(batch, weight.shape[1] * groups, weight.shape[0],
                              tuple(weight.shape[2:]), tuple(in_size), stride, padding, dilation,
                              groups, bias is not None, dt, algo)
        self.info = conv_query(self.desc)
        self.batch, self.in_size = batch, tuple(in_size)
        self.in_channels, self.out_channels = weight.shape[1] * groups, weight.shape[0]
        self.out_size = tuple(self.info.out_size[:len(in_size)])
        self._frames = (self.frame_shape(), self.out_frame_shape())
        self.weight, self.bias, self.bn = weight, bias, bn
        dev = weight.device
        if state is None:
            state = torch.empty(self.info.state_bytes, dtype=torch.uint8, device=dev)
        self.state = state
        h = ctypes.c_void_p()
        if attach_steps is None:
            _need(weight, weight.dtype, weight.shape, "weight")
            if bias is not None:
                _need(bias, weight.dtype, (weight.shape[0],), "bias")
            if bn is None:
                check(co_conv_init_state(ctypes.byref(self.desc), _ptr(weight), _ptr(bias),
                                         _ptr(state), state.numel(), _stream(),
                                         ctypes.byref(h)), "co_conv_init_state")
            else:
                check(co_conv_init_state_bn(ctypes.byref(self.desc), _ptr(weight), _ptr(bias),
                                            *self._bn_args(), _ptr(state), state.numel(),
                                            _stream(), ctypes.byref(h)),
                      "co_conv_init_state_bn")
        else:
            check(co_conv_attach_state(ctypes.byref(self.desc), _ptr(state), state.numel(),
                                       int(attach_steps), _stream(), ctypes.byref(h)),
                  "co_conv_attach_state")
        self.handle = h

    def _bn_args(self):
        gamma, beta, mean, var, eps = self.bn
        for t, what in ((gamma, "gamma"), (beta, "beta"), (mean, "running_mean"),
                        (var, "running_var")):
            _need(t, torch.float32, (self.out_channels,), what)
        return _ptr(gamma), _ptr(beta), _ptr(mean), _ptr(var), float(eps)

    # the destroy function is bound as a default so that objects collected
    # during interpreter shutdown, after the module globals are cleared, still
    # release their handles
    def __del__(self, _destroy=co_conv_destroy):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            _destroy(h)
            self.handle = None

    @property
    def delay(self):
        return self.info.delay

    @property
    def receptive_field(self):
        return self.info.receptive_field

    @property
    def t_stride(self):
        return self.desc.stride[0]

    @property
    def t_padding(self):
        return self.desc.padding[0]

    @property
    def algo(self):
        return co_conv_algo_name(self.handle).decode()

    @property
    def steps(self):
        n = i64()
        check(co_conv_get_steps(self.handle, ctypes.byref(n)), "co_conv_get_steps")
        return n.value

    def frame_shape(self):
        return (self.batch, self.in_channels) + self.in_size

    def out_frame_shape(self):
        return (self.batch, self.out_channels) + self.out_size

    def new_output(self):
        return torch.empty(self.out_frame_shape(), dtype=self.torch_dtype, device=self.state.device)

    def forward_step(self, x_t, update_state=True, out=None):
        """Principle 2 forward_step; returns the output frame or None (empty)."""
        shape, out_shape = self._frames
        _need(x_t, self.torch_dtype, shape, "x_t")
        if out is None:
            out = torch.empty(out_shape, dtype=self.torch_dtype, device=self.state.device)
        else:
            _need(out, self.torch_dtype, out_shape, "out")
        st = co_conv_forward_step(self.handle, x_t.data_ptr(), out.data_ptr(),
                                  1 if update_state else 0, _stream())
        if st == CO_OK:
            return out
        check(st, "co_conv_forward_step")
        return None

    def forward_step_raw(self, x_ptr, y_ptr, update_state=True, stream=None):
        """forward_step on raw device pointers (no checks); returns the status."""
        return co_conv_forward_step(self.handle, x_ptr, y_ptr, 1 if update_state else 0,
                                    _stream(stream))

    def forward_steps(self, x, pad_end=False, update_state=True):
        """Principle 2 forward_steps over x (B, C_in, T, *S); None when empty.
        The result is contiguous, sized to the frames the call emits."""
        T = x.shape[2]
        _need(x, self.torch_dtype, (self.batch, self.in_channels, T) + self.in_size, "x")
        cap = self.out_frames(T, pad_end)
        y = torch.empty((self.batch, self.out_channels, cap) + self.out_size,
                        dtype=self.torch_dtype, device=x.device)
        n = i32()
        check(co_conv_forward_steps(self.handle, _ptr(x), T, _ptr(y), cap,
                                    1 if pad_end else 0, 1 if update_state else 0, _stream(),
                                    ctypes.byref(n)), "co_conv_forward_steps")
        if n.value == 0:
            return None
        return y[:, :, :n.value]

    def out_frames(self, T, pad_end=False):
        """Frames forward_steps over T frames emits from the current step."""
        return conv_out_frames(self.desc, self.steps, T, pad_end)

    def steps_fused(self, T, pad_end=False):
        """True when forward_steps over T frames runs as one launch."""
        f = i32()
        check(co_conv_steps_fused(self.handle, T, self.out_frames(T, pad_end), ctypes.byref(f)),
              "co_conv_steps_fused")
        return bool(f.value)

    def steps_route(self, T, pad_end=False, update_state=True):
        """How forward_steps over T frames runs (STEPS_ROUTES)."""
        return conv_steps_route(self.desc, T, self.out_frames(T, pad_end), update_state)

    def folded(self):
        """(weight, bias) with the batch normalisation folded in, in the io
        dtype (co_conv_fold_bn); the layer's own when it has none."""
        if self.bn is None:
            return self.weight, self.bias
        w = torch.empty_like(self.weight)
        b = torch.empty(self.out_channels, dtype=self.torch_dtype, device=self.weight.device)
        check(co_conv_fold_bn(ctypes.byref(self.desc), _ptr(self.weight), _ptr(self.bias),
                              *self._bn_args(), _ptr(w), _ptr(b), _stream()), "co_conv_fold_bn")
        return w, b

    def forward(self, x):
        """Principle 2 forward (clip mode), stateless: on the step kernels
        from a clean state in a scratch workspace (co_conv_forward_ws), with
        the batch normalisation folded in as the steps have it."""
        bn = None
        if self.bn is not None:
            gamma, beta, mean, var, eps = self._bn_args()
            bn = BnParams(gamma, beta, mean, var, eps)
        return conv_forward(self.desc, self.weight, self.bias, x, bn=bn)

    def clean_state(self):
        check(co_conv_clean_state(self.handle, _stream()), "co_conv_clean_state")


STEPS_ROUTES = ("loop", "depthwise", "direct_mma", "direct", "gemm", "reg", "clip")


def conv_steps_route(desc, T, y_cap_frames, update_state=True):
    """How forward_steps over T frames of such a layer runs (co_conv_steps_route)."""
    r = i32()
    check(co_conv_steps_route(ctypes.byref(desc), T, y_cap_frames, 1 if update_state else 0,
                              ctypes.byref(r)), "co_conv_steps_route")
    return STEPS_ROUTES[r.value]


def conv_out_frames(desc, n0, T, pad_end=False):
    """Frames forward_steps over T frames emits from step counter n0
    (co_conv_out_frames)."""
    n = i32()
    check(co_conv_out_frames(ctypes.byref(desc), int(n0), int(T), 1 if pad_end else 0,
                             ctypes.byref(n)), "co_conv_out_frames")
    return n.value


def pool_out_frames(desc, n0, T, pad_end=False):
    """Frames a pool's forward_steps over T frames emits from step counter n0
    (co_pool_out_frames)."""
    n = i32()
    check(co_pool_out_frames(ctypes.byref(desc), int(n0), int(T), 1 if pad_end else 0,
                             ctypes.byref(n)), "co_pool_out_frames")
    return n.value


def residual_align(f, s, p, module_delay):
    """(residual delay, clip shrink, delay of the whole) of a centred residual
    (co_residual_align); None when the clip shapes cannot be joined."""
    d_res, shrink, delay = i64(), i64(), i64()
    st = co_residual_align(int(f), int(s), int(p), int(module_delay), ctypes.byref(d_res),
                           ctypes.byref(shrink), ctypes.byref(delay))
    if st != CO_OK:
        return None
    return d_res.value, shrink.value, delay.value


def conv_forward(desc, weight, bias, x, bn=None, direct=False):
    """Clip-mode forward: on the step kernels AUTO picks, from a clean state
    in a scratch workspace (co_conv_forward_ws), or with direct=True on the
    direct clip kernel (co_conv_forward)."""
    T = x.shape[2]
    t_out = i32()
    check(co_conv_clip_frames(ctypes.byref(desc), T, ctypes.byref(t_out)), "co_conv_clip_frames")
    sd = desc.spatial_dims
    info = conv_query(desc)
    y = torch.empty((desc.batch, desc.out_channels, t_out.value) + tuple(info.out_size[:sd]),
                    dtype=x.dtype, device=x.device)
    if direct:
        if bn is not None:
            raise ValueError("the direct clip kernel takes no batch normalisation")
        check(co_conv_forward(ctypes.byref(desc), _ptr(weight), _ptr(bias), _ptr(x), T, _ptr(y),
                              _stream()), "co_conv_forward")
        return y
    ws = torch.empty(info.state_bytes, dtype=torch.uint8, device=x.device)
    check(co_conv_forward_ws(ctypes.byref(desc), _ptr(weight), _ptr(bias),
                             ctypes.byref(bn) if bn is not None else None, _ptr(x), T, _ptr(y),
                             _ptr(ws), ws.numel(), _stream()), "co_conv_forward_ws")
    return y


class CoPool:
    """A continual AvgPoolNd / MaxPoolNd layer over a device state buffer."""

    def __init__(self, kind, *, batch, channels, kernel, in_size=(), stride=None, padding=0,
                 dilation=1, count_include_pad=True, dtype=torch.float32, device="cuda",
                 state=None, attach_steps=None):
        self.torch_dtype = dtype
        self.desc = pool_desc(kind, batch, channels, kernel, tuple(in_size), stride, padding,
                              dilation, count_include_pad, DTYPES[dtype])
        self.info = pool_query(self.desc)
        self.batch, self.channels, self.in_size = batch, channels, tuple(in_size)
        self.out_size = tuple(self.info.out_size[:len(in_size)])
        self._frames = (self.frame_shape(), self.out_frame_shape())
        if state is None:
            state = torch.empty(self.info.state_bytes, dtype=torch.uint8, device=device)
        self.state = state
        h = ctypes.c_void_p()
        if attach_steps is None:
            check(co_pool_init_state(ctypes.byref(self.desc), _ptr(state), state.numel(),
                                     _stream(), ctypes.byref(h)), "co_pool_init_state")
        else:
            check(co_pool_attach_state(ctypes.byref(self.desc), _ptr(state), state.numel(),
                                       int(attach_steps), _stream(), ctypes.byref(h)),
                  "co_pool_attach_state")
        self.handle = h

    # the destroy function is bound as a default so that objects collected
    # during interpreter shutdown, after the module globals are cleared, still
    # release their handles
    def __del__(self, _destroy=co_pool_destroy):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            _destroy(h)
            self.handle = None

    @property
    def delay(self):
        return self.info.delay

    @property
    def receptive_field(self):
        return self.info.receptive_field

    @property
    def t_stride(self):
        return self.desc.stride[0]

    @property
    def t_padding(self):
        return self.desc.padding[0]

    @property
    def steps(self):
        n = i64()
        check(co_pool_get_steps(self.handle, ctypes.byref(n)), "co_pool_get_steps")
        return n.value

    def frame_shape(self):
        return (self.batch, self.channels) + self.in_size

    def out_frame_shape(self):
        return (self.batch, self.channels) + self.out_size

    def forward_step(self, x_t, update_state=True, out=None):
        shape, out_shape = self._frames
        _need(x_t, self.torch_dtype, shape, "x_t")
        if out is None:
            out = torch.empty(out_shape, dtype=self.torch_dtype, device=x_t.device)
        else:
            _need(out, self.torch_dtype, out_shape, "out")
        st = co_pool_forward_step(self.handle, x_t.data_ptr(), out.data_ptr(),
                                  1 if update_state else 0, _stream())
        if st == CO_OK:
            return out
        check(st, "co_pool_forward_step")
        return None

    def forward_step_raw(self, x_ptr, y_ptr, update_state=True, stream=None):
        return co_pool_forward_step(self.handle, x_ptr, y_ptr, 1 if update_state else 0,
                                    _stream(stream))

    def forward_steps(self, x, pad_end=False, update_state=True):
        T = x.shape[2]
        _need(x, self.torch_dtype, (self.batch, self.channels, T) + self.in_size, "x")
        cap = self.out_frames(T, pad_end)
        y = torch.empty((self.batch, self.channels, cap) + self.out_size,
                        dtype=self.torch_dtype, device=x.device)
        n = i32()
        check(co_pool_forward_steps(self.handle, _ptr(x), T, _ptr(y), cap,
                                    1 if pad_end else 0, 1 if update_state else 0, _stream(),
                                    ctypes.byref(n)), "co_pool_forward_steps")
        if n.value == 0:
            return None
        return y[:, :, :n.value]

    def out_frames(self, T, pad_end=False):
        """Frames forward_steps over T frames emits from the current step."""
        return pool_out_frames(self.desc, self.steps, T, pad_end)

    def steps_fused(self, T, pad_end=False):
        """True when forward_steps over T frames runs as one persistent launch."""
        f = i32()
        check(co_pool_steps_fused(self.handle, T, self.out_frames(T, pad_end), ctypes.byref(f)),
              "co_pool_steps_fused")
        return bool(f.value)

    def forward(self, x):
        T = x.shape[2]
        t_out = i32()
        check(co_pool_clip_frames(ctypes.byref(self.desc), T, ctypes.byref(t_out)),
              "co_pool_clip_frames")
        y = torch.empty((self.batch, self.channels, t_out.value) + self.out_size,
                        dtype=x.dtype, device=x.device)
        check(co_pool_forward(ctypes.byref(self.desc), _ptr(x), T, _ptr(y), _stream()),
              "co_pool_forward")
        return y

    def clean_state(self):
        check(co_pool_clean_state(self.handle, _stream()), "co_pool_clean_state")


def chain_delay(layers):
    """Principle 6 over a chain of layers (anything with receptive_field,
    t_stride and t_padding): (f_acc, p_acc, s_acc, delay) of the last one."""
    n = len(layers)
    arr = i32 * n
    f = arr(*[m.receptive_field for m in layers])
    st = arr(*[m.t_stride for m in layers])
    p = arr(*[m.t_padding for m in layers])
    out = [i64() for _ in range(4)]
    check(co_chain_delay(n, f, st, p, *[ctypes.byref(o) for o in out]), "co_chain_delay")
    return tuple(o.value for o in out)


class CoDelay:
    """co.Delay: step n outputs frame n - delay (empty before); clip mode is
    the identity.  Frames are (batch, channels, *in_size)."""

    def __init__(self, delay, *, batch, channels, in_size=(), dtype=torch.float32,
                 device="cuda"):
        self.torch_dtype = dtype
        self.batch, self.channels, self.in_size = batch, channels, tuple(in_size)
        self.out_channels, self.out_size = channels, tuple(in_size)
        E = 1
        for v in in_size:
            E *= int(v)
        self.E = E
        self.desc = DelayDesc(batch, channels, E, int(delay), DTYPES[dtype])
        nb = i64()
        check(co_delay_query(ctypes.byref(self.desc), ctypes.byref(nb)), "co_delay_query")
        self.state = torch.empty(max(nb.value, 1), dtype=torch.uint8, device=device)
        h = ctypes.c_void_p()
        check(co_delay_init_state(ctypes.byref(self.desc), _ptr(self.state), self.state.numel(),
                                  _stream(), ctypes.byref(h)), "co_delay_init_state")
        self.handle = h

    # the destroy function is bound as a default so that objects collected
    # during interpreter shutdown, after the module globals are cleared, still
    # release their handles
    def __del__(self, _destroy=co_delay_destroy):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            _destroy(h)
            self.handle = None

    delay = property(lambda self: self.desc.delay)
    receptive_field = property(lambda self: self.desc.delay + 1)
    t_stride = property(lambda self: 1)
    t_padding = property(lambda self: 0)

    @property
    def steps(self):
        n = i64()
        check(co_delay_get_steps(self.handle, ctypes.byref(n)), "co_delay_get_steps")
        return n.value

    def frame_shape(self):
        return (self.batch, self.channels) + self.in_size

    def forward_step(self, x_t, update_state=True, out=None, emit=True):
        """x_{n - delay}, or None while empty; emit=False only advances."""
        _need(x_t, self.torch_dtype, self.frame_shape(), "x_t")
        y = None
        if emit:
            y = torch.empty_like(x_t) if out is None else out
        st = check(co_delay_forward_step(self.handle, _ptr(x_t), _ptr(y),
                                         1 if update_state else 0, _stream()),
                   "co_delay_forward_step")
        return y if (st == CO_OK and emit) else None

    def add_step(self, x_t, a_t, update_state=True, out=None):
        """a_t + x_{n - delay} (the residual merge), or None while empty."""
        _need(x_t, self.torch_dtype, self.frame_shape(), "x_t")
        _need(a_t, self.torch_dtype, self.frame_shape(), "a_t")
        y = torch.empty_like(a_t) if out is None else out
        st = check(co_delay_add_step(self.handle, _ptr(x_t), _ptr(a_t), _ptr(y),
                                     1 if update_state else 0, _stream()), "co_delay_add_step")
        return y if st == CO_OK else None

    def forward_steps(self, x, update_state=True):
        T = x.shape[2]
        _need(x, self.torch_dtype, (self.batch, self.channels, T) + self.in_size, "x")
        y = torch.empty_like(x)
        n = i32()
        check(co_delay_forward_steps(self.handle, _ptr(x), T, _ptr(y), T,
                                     1 if update_state else 0, _stream(), ctypes.byref(n)),
              "co_delay_forward_steps")
        return y[:, :, :n.value] if n.value else None

    def add_steps(self, x, a, update_state=True):
        """a (the last a.shape[2] steps' module outputs) + the delayed x."""
        T = x.shape[2]
        _need(x, self.torch_dtype, (self.batch, self.channels, T) + self.in_size, "x")
        na = 0 if a is None else a.shape[2]
        y = None
        if na:
            _need(a, self.torch_dtype, (self.batch, self.channels, na) + self.in_size, "a")
            y = torch.empty_like(a)
        check(co_delay_add_steps(self.handle, _ptr(x), T, _ptr(a) if na else None, na,
                                 _ptr(y) if na else None, 1 if update_state else 0, _stream()),
              "co_delay_add_steps")
        return y

    def forward(self, x):
        return x

    def clean_state(self):
        check(co_delay_clean_state(self.handle, _stream()), "co_delay_clean_state")


def add_frames(a, x, x_offset=0):
    """y[:, :, i] = a[:, :, i] + x[:, :, i + x_offset] (clip-mode merge)."""
    rows = a.shape[0] * a.shape[1]
    E = 1
    for v in a.shape[3:]:
        E *= int(v)
    y = torch.empty_like(a)
    check(co_add_frames(_ptr(a), _ptr(x), _ptr(y), rows, E, a.shape[2], x.shape[2],
                        int(x_offset), DTYPES[a.dtype], _stream()), "co_add_frames")
    return y


ACTS = {"none": CO_ACT_NONE, "relu": CO_ACT_RELU}


def act_forward(x, act="relu", out=None):
    """Elementwise activation of any contiguous tensor (co_act_forward)."""
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    y = torch.empty_like(x) if out is None else out
    _need(y, x.dtype, x.shape, "out")
    check(co_act_forward(_ptr(x), _ptr(y), x.numel(), DTYPES[x.dtype], ACTS[act], _stream()),
          "co_act_forward")
    return y


class CoReLU:
    """ReLU as a continual module: stateless and elementwise, so it has delay
    0 and receptive field 1 (section 3.2's composition of per-frame
    layers); every step emits."""

    delay, receptive_field, t_stride, t_padding = 0, 1, 1, 0
    act = "relu"

    def forward_step(self, x_t, update_state=True):
        return act_forward(x_t)

    def forward_steps(self, x, update_state=True):
        return act_forward(x.contiguous())

    def forward(self, x):
        return act_forward(x.contiguous())

    def clean_state(self):
        pass


class Bottleneck:
    """The X3D bottleneck front (pointwise CoConv -> optional ReLU ->
    depthwise CoConv -> optional ReLU -> CoPool over its whole output plane,
    batch normalisations folded into the convolutions) stepped as one launch
    per frame (co_bneck_*).  The three modules keep their states and step
    counters, and the outputs equal stepping them separately bit for bit.
    The pointwise layer must be a 1x1x1 CoConv on the register-GEMM kernel
    (algo "gemm_reg", AUTO's choice for such layers)."""

    def __init__(self, pw, relu1, dw, relu2, pool):
        h = ctypes.c_void_p()
        check(co_bneck_bind(pw.handle, CO_ACT_RELU if relu1 else CO_ACT_NONE, dw.handle,
                            CO_ACT_RELU if relu2 else CO_ACT_NONE, pool.handle,
                            ctypes.byref(h)), "co_bneck_bind")
        self.pw, self.relu1, self.dw, self.relu2, self.pool = pw, relu1, dw, relu2, pool
        self.handle = h

    @staticmethod
    def fits(pw, dw, pool):
        h = ctypes.c_void_p()
        if co_bneck_bind(pw.handle, CO_ACT_NONE, dw.handle, CO_ACT_NONE, pool.handle,
                         ctypes.byref(h)) != CO_OK:
            return False
        co_bneck_destroy(h)
        return True

    # the destroy function is bound as a default so that objects collected
    # during interpreter shutdown, after the module globals are cleared, still
    # release their handles
    def __del__(self, _destroy=co_bneck_destroy):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            _destroy(h)
            self.handle = None

    def _chain(self):
        return [self.pw, self.dw, self.pool]

    delay = property(lambda self: chain_delay(self._chain())[3])
    receptive_field = property(lambda self: chain_delay(self._chain())[0])
    t_stride = property(lambda self: chain_delay(self._chain())[2])
    t_padding = property(lambda self: chain_delay(self._chain())[1])

    def forward_step(self, x_t, update_state=True):
        _need(x_t, self.pw.torch_dtype, self.pw.frame_shape(), "x_t")
        z = torch.empty(self.pool.out_frame_shape(), dtype=self.pool.torch_dtype,
                        device=x_t.device)
        st = check(co_bneck_forward_step(self.handle, _ptr(x_t), _ptr(z),
                                         1 if update_state else 0, _stream()),
                   "co_bneck_forward_step")
        return z if st == CO_OK else None

    def forward_steps(self, x, update_state=True):
        T = x.shape[2]
        w, c, p = self.pw, self.dw, self.pool
        _need(x, w.torch_dtype, (w.batch, w.in_channels, T) + w.in_size, "x")
        # the pointwise layer emits every frame; the pool once per depthwise frame
        cap = pool_out_frames(p.desc, p.steps, conv_out_frames(c.desc, c.steps, T))
        z = torch.empty((p.batch, p.channels, cap) + p.out_size, dtype=p.torch_dtype,
                        device=x.device)
        n, nb = i32(), i64()
        check(co_bneck_workspace_bytes(self.handle, T, ctypes.byref(nb)),
              "co_bneck_workspace_bytes")
        ws = torch.empty(nb.value, dtype=torch.uint8, device=x.device) if nb.value else None
        check(co_bneck_forward_steps_ws(self.handle, _ptr(x), T, _ptr(z), cap,
                                        1 if update_state else 0, _ptr(ws), nb.value, _stream(),
                                        ctypes.byref(n)), "co_bneck_forward_steps_ws")
        return z if n.value else None

    def forward(self, x):
        y = self.pw.forward(x)
        if self.relu1:
            y = act_forward(y)
        y = self.dw.forward(y)
        if self.relu2:
            y = act_forward(y)
        return self.pool.forward(y)

    def clean_state(self):
        for m in self._chain():
            m.clean_state()


class ConvPool:
    """A depthwise CoConv followed by a CoPool over its whole output plane,
    stepped as one launch (co_convpool_*).  Both modules keep their states and
    step counters, and the outputs equal stepping them separately."""

    def __init__(self, conv, pool):
        h = ctypes.c_void_p()
        check(co_convpool_bind(conv.handle, pool.handle, ctypes.byref(h)), "co_convpool_bind")
        self.conv, self.pool, self.handle = conv, pool, h

    @staticmethod
    def fits(conv, pool):
        h = ctypes.c_void_p()
        if co_convpool_bind(conv.handle, pool.handle, ctypes.byref(h)) != CO_OK:
            return False
        co_convpool_destroy(h)
        return True

    # the destroy function is bound as a default so that objects collected
    # during interpreter shutdown, after the module globals are cleared, still
    # release their handles
    def __del__(self, _destroy=co_convpool_destroy):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            _destroy(h)
            self.handle = None

    delay = property(lambda self: chain_delay([self.conv, self.pool])[3])
    receptive_field = property(lambda self: chain_delay([self.conv, self.pool])[0])
    t_stride = property(lambda self: chain_delay([self.conv, self.pool])[2])
    t_padding = property(lambda self: chain_delay([self.conv, self.pool])[1])

    def _out(self, frames, device):
        return torch.empty((self.pool.batch, self.pool.channels, frames) + self.pool.out_size,
                           dtype=self.pool.torch_dtype, device=device)

    def forward_step(self, x_t, update_state=True):
        _need(x_t, self.conv.torch_dtype, self.conv.frame_shape(), "x_t")
        z = torch.empty(self.pool.out_frame_shape(), dtype=self.pool.torch_dtype,
                        device=x_t.device)
        st = check(co_convpool_forward_step(self.handle, _ptr(x_t), _ptr(z),
                                            1 if update_state else 0, _stream()),
                   "co_convpool_forward_step")
        return z if st == CO_OK else None

    def forward_steps(self, x, update_state=True):
        T = x.shape[2]
        c, p = self.conv, self.pool
        _need(x, c.torch_dtype, (c.batch, c.in_channels, T) + c.in_size, "x")
        # the pool steps once per emitted convolution frame
        cap = pool_out_frames(p.desc, p.steps, conv_out_frames(c.desc, c.steps, T))
        z = self._out(cap, x.device)
        n = i32()
        check(co_convpool_forward_steps(self.handle, _ptr(x), T, _ptr(z), cap,
                                        1 if update_state else 0, _stream(), ctypes.byref(n)),
              "co_convpool_forward_steps")
        return z if n.value else None

    def forward(self, x):
        return self.pool.forward(self.conv.forward(x))

    def clean_state(self):
        self.conv.clean_state()
        self.pool.clean_state()


class Sequential:
    """Section 3.3's Sequential: modules in a chain; an empty step output
    ends the step (downstream modules do not advance), and the chain's delay
    follows Principle 6.  With fuse (the default) a pointwise CoConv, an
    optional CoReLU, a depthwise CoConv, an optional CoReLU and a CoPool
    over its whole output plane run as one Bottleneck launch per step, and
    a depthwise CoConv directly followed by such a CoPool as one ConvPool
    launch, with identical results."""

    def __init__(self, *modules, fuse=True):
        mods = list(modules)
        if fuse:
            mods = self._fuse(mods)
        self.modules = mods

    @staticmethod
    def _bottleneck_at(mods, i):
        """(Bottleneck, modules consumed) starting at mods[i], or None."""
        j = i
        parts = []
        for kind in ("conv", "relu", "conv", "relu", "pool"):
            m = mods[j] if j < len(mods) else None
            if kind == "relu":
                parts.append(isinstance(m, CoReLU))
                j += 1 if isinstance(m, CoReLU) else 0
                continue
            want = CoConv if kind == "conv" else CoPool
            if not isinstance(m, want):
                return None
            parts.append(m)
            j += 1
        pw, r1, dw, r2, pool = parts
        if not Bottleneck.fits(pw, dw, pool):
            return None
        return Bottleneck(pw, r1, dw, r2, pool), j - i

    def _fuse(self, mods):
        out, i = [], 0
        while i < len(mods):
            a = mods[i]
            b = mods[i + 1] if i + 1 < len(mods) else None
            bn = self._bottleneck_at(mods, i)
            if bn is not None:
                out.append(bn[0])
                i += bn[1]
            elif isinstance(a, CoConv) and isinstance(b, CoPool) and ConvPool.fits(a, b):
                out.append(ConvPool(a, b))
                i += 2
            else:
                out.append(a)
                i += 1
        return out

    @property
    def delay(self):
        return chain_delay(self.modules)[3]

    @property
    def receptive_field(self):
        return chain_delay(self.modules)[0]

    @property
    def t_stride(self):
        return chain_delay(self.modules)[2]

    @property
    def t_padding(self):
        return chain_delay(self.modules)[1]

    def forward_step(self, x_t, update_state=True):
        for m in self.modules:
            x_t = m.forward_step(x_t, update_state=update_state)
            if x_t is None:
                return None
        return x_t

    def forward_steps(self, x, update_state=True):
        for m in self.modules:
            x = m.forward_steps(x, update_state=update_state)
            if x is None:
                return None
        return x

    def forward(self, x):
        for m in self.modules:
            x = m.forward(x)
        return x

    def clean_state(self):
        for m in self.modules:
            m.clean_state()


class Residual:
    """Section 3.1.1's residual connection around a module with equal input
    and output frames (stride 1): the input joins the module's output aligned
    on the centre of its receptive field, so the residual branch is delayed by
    (f - 1) // 2 steps (Principle 7: the whole has the module's delay, and a
    step is empty while either branch is).  With equal temporal padding
    ((f - 1) / 2) clip mode adds the input as is; a module with less padding
    needs residual_shrink=True, which drops the border frames of the input in
    clip mode (the centred residual)."""

    def __init__(self, module, residual_shrink=False):
        if module.t_stride != 1:
            raise ValueError("residual connections need temporal stride 1")
        al = residual_align(module.receptive_field, module.t_stride, module.t_padding,
                            module.delay)
        if al is None:
            raise ValueError("clip shapes differ: the module's temporal padding exceeds "
                             "(f - 1) / 2")
        self.module = module
        self.d_res, self.shrink, self._delay = al
        if self.shrink > 0 and not residual_shrink:
            raise ValueError("clip shapes differ: give the module padding (f - 1) / 2 or "
                             "residual_shrink=True")
        self.line = CoDelay(self.d_res, batch=module.batch, channels=module.out_channels,
                            in_size=module.out_size, dtype=module.torch_dtype,
                            device=module.state.device)

    delay = property(lambda self: self._delay)
    receptive_field = property(lambda self: self.module.receptive_field)
    t_stride = property(lambda self: 1)
    t_padding = property(lambda self: self.module.t_padding)
    batch = property(lambda self: self.module.batch)
    out_channels = property(lambda self: self.module.out_channels)
    out_size = property(lambda self: self.module.out_size)
    torch_dtype = property(lambda self: self.module.torch_dtype)

    def forward_step(self, x_t, update_state=True):
        a = self.module.forward_step(x_t, update_state=update_state)
        if a is None:
            self.line.forward_step(x_t, update_state=update_state, emit=False)
            return None
        return self.line.add_step(x_t, a, update_state=update_state, out=a)

    def forward_steps(self, x, update_state=True):
        a = self.module.forward_steps(x, update_state=update_state)
        return self.line.add_steps(x, a, update_state=update_state)

    def forward(self, x):
        a = self.module.forward(x)
        return add_frames(a, x, self.shrink)

    def clean_state(self):
        self.module.clean_state()
        self.line.clean_state()


# ------------------------------------------------------------ token layers
# Layers over token sequences (B, T, values), time-major as the projections
# around them write it.  Their state is a plain device tensor (self.state): it
# may be read, copied, zeroed or indexed by stream between calls.  Delay 0.


# A single token's call is a few microseconds.  A layer keeps the structure that
# describes its call; shapes, strides and dtypes are checked and filled in when
# they differ from the last call's, and a like call sets the pointers alone (conv
# 7.7 -> 5.1 us, scan 10.8 -> 6.2 us, pre-norm 13.6 -> 6.8 us a call).  Like a
# handle, a layer is one thread's.
_like = torch.empty_like  # 1.2 us; new_empty, for inputs that are slices, 1.5


def _on(t, device, what):
    if t.device.type != "cuda":
        raise ValueError(f"{what} must be a device tensor")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, expected {device}")


def _tokens(t, dtype, shape, what, into, device):
    """Checks that t is a tensor on that device, of that dtype and shape (B, T, ...),
    or (B, ...) for single tokens, whose values of one token are contiguous, and
    fills `into` with its strides."""
    _on(t, device, what)
    if t.dtype is not dtype:
        raise ValueError(f"{what} has dtype {t.dtype}, expected {dtype}")
    if t.shape not in (shape, shape[:1] + shape[2:] if shape[1] == 1 else shape):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    st = t.stride()
    run, lead = 1, t.dim() - len(shape) + 2
    for i in range(t.dim() - 1, lead - 1, -1):
        if t.shape[i] != 1:
            if st[i] != run:
                raise ValueError(f"{what}: the values of a token must be contiguous")
            run *= t.shape[i]
    into.batch_stride, into.token_stride = st[0], st[1] if lead == 2 else 0


def _lengths(lengths, batch, device):
    _need(lengths, torch.int32, (batch,), "lengths")
    if lengths.device != device:
        _on(lengths, device, "lengths")
    return lengths.data_ptr()


class _TokenState:
    """The state of a token layer: a tensor that another one of its kind may replace."""

    def _keep_state(self, state, dtype, shape, device):
        self._state_kind = dtype, shape, device
        if state is None:
            state = torch.zeros(shape, dtype=dtype, device=device)
        self.state = state

    @property
    def state(self):
        return self._state

    @state.setter
    def state(self, state):
        dtype, shape, device = self._state_kind
        _need(state, dtype, shape, "state")
        _on(state, device, "state")
        self._state = state

    def clean_state(self):
        self._state.zero_()


def _vector(t, n, what, device):
    """A float32 device vector of n parameters, or None."""
    if t is None:
        return None
    if tuple(t.shape) != (n,) or t.device != device:
        raise ValueError(f"{what} must be ({n},) on {device}")
    return t.detach().to(torch.float32).contiguous()


class CoShortConv(_TokenState):
    """Short causal depthwise convolution over tokens with its activation
    (co_shortconv_* ABI).

    weight (C, K) or (C, 1, K) with K <= 8 and bias (C,): device tensors of one
    dtype (float32 or bfloat16).  act: "none", "relu" or "silu".  The state
    (B, K - 1, C) holds the newest inputs, oldest first; state: a tensor to keep
    it in (continued from), default a new clean one.

    lengths (int32 (B,) on the device): how many of a call's tokens each stream
    has.  Outputs past them are 0, whatever the tokens there hold.
    """

    delay, t_stride = 0, 1

    def __init__(self, weight, bias=None, *, batch, act="silu", state=None):
        if weight.dim() == 3 and weight.shape[1] == 1:
            weight = weight[:, 0]
        if weight.dim() != 2:
            raise ValueError("weight must be (C, K) or (C, 1, K)")
        self.batch, self.torch_dtype = batch, weight.dtype
        self.channels, self.kernel = weight.shape
        _need(weight, weight.dtype, weight.shape, "weight")
        self.device = weight.device
        if bias is not None:
            _need(bias, weight.dtype, (self.channels,), "bias")
            _on(bias, self.device, "bias")
        self._weight, self._bias = weight, bias
        acts = {"none": CO_ACT_NONE, "relu": CO_ACT_RELU, "silu": CO_ACT_SILU}
        self.desc = ShortConvDesc(batch, self.channels, self.kernel, 1 if bias is not None else 0,
                                  acts[act], DTYPES[weight.dtype])
        nb = i64()
        check(co_shortconv_query(ctypes.byref(self.desc), ctypes.byref(nb)), "co_shortconv_query")
        self._keep_state(state, weight.dtype, (batch, self.kernel - 1, self.channels), self.device)
        self._call = ShortConvCall(_ptr(weight), _ptr(bias))
        self._x, self._y = self._call.x, self._call.y
        self._args = ctypes.byref(self.desc), ctypes.byref(self._call)
        self._sig = None

    # parameters: a call takes those that the layer was made with
    weight = property(lambda self: self._weight)
    bias = property(lambda self: self._bias)
    receptive_field = property(lambda self: self.kernel)
    t_padding = property(lambda self: self.kernel - 1)

    def _check(self, x, out, step, state, update):
        B, C, call = self.batch, self.channels, self._call
        T = 1 if step else x.shape[1] if x.dim() == 3 else -1
        if x.dim() != 3 - step:
            raise ValueError(f"x has shape {tuple(x.shape)}, expected "
                             f"{(B, C) if step else (B, 'T', C)}")
        _tokens(x, self.torch_dtype, (B, T, C), "x", self._x, self.device)
        self._y.batch_stride, self._y.token_stride = T * C, C
        if out is not None:
            if out.dim() != x.dim():
                raise ValueError(f"out has shape {tuple(out.shape)}, expected {tuple(x.shape)}")
            _tokens(out, self.torch_dtype, (B, T, C), "out", self._y, self.device)
        call.T, call.state, call.update_state = T, state, update
        self._dense = x.is_contiguous()

    def _run(self, x, lengths, state, update, out, step=False):
        sig = (step, x.shape, x.stride(), x.dtype, x.get_device(), state, update,
               None if out is None else (out.shape, out.stride(), out.dtype, out.get_device()))
        if sig != self._sig:
            self._sig = None
            self._check(x, out, step, state, update)
            self._sig = sig
        if out is None:
            out = _like(x) if self._dense else x.new_empty(x.shape)
        self._x.data, self._y.data = x.data_ptr(), out.data_ptr()
        self._call.lengths = None if lengths is None else _lengths(lengths, self.batch, self.device)
        pd, pc = self._args
        st = co_shortconv_forward_steps(pd, pc, _stream())
        if st != CO_OK:
            check(st, "co_shortconv_forward_steps")
        return out

    def forward_steps(self, x, lengths=None, update_state=True, out=None):
        """The next T tokens x (B, T, C) of the streams -> (B, T, C)."""
        return self._run(x, lengths, self._state.data_ptr(), 1 if update_state else 0, out)

    def forward_step(self, x_t, lengths=None, update_state=True, out=None):
        """The next token x_t (B, C) of each stream (of those with length 1) -> (B, C)."""
        return self._run(x_t, lengths, self._state.data_ptr(), 1 if update_state else 0, out, True)

    def forward(self, x, lengths=None, out=None):
        """Whole sequences from a clean state, which the layer's own is not touched by."""
        return self._run(x, lengths, None, 0, out)


class CoScan(_TokenState):
    """Selective state space scan (co_scan_* ABI): heads of head_dim values with
    a head_dim x state_size state each, a decay a head and token, and B and C
    shared by the heads of a group.

    A (H,): the decay of a head is exp(dt A), so A <= 0.  D (H,): skip weight.
    dt_bias (H,) is added to dt, then with dt_softplus softplus is taken of it.
    dtype: of x, b, c and the output; dt has it or is float32.  state
    (B, H, head_dim, state_size) float32, continued from; default a new clean
    one.  lengths: as CoShortConv's.
    """

    delay, receptive_field, t_stride, t_padding = 0, 1, 1, 0

    def __init__(self, A, *, batch, head_dim, state_size, groups=1, D=None, dt_bias=None,
                 dt_softplus=False, dtype=torch.bfloat16, state=None):
        if A.device.type != "cuda":
            raise ValueError("A must be a device tensor")
        H = self.heads = A.shape[0]
        self.batch, self.head_dim, self.state_size = batch, head_dim, state_size
        self.groups, self.torch_dtype = groups, dtype
        self.device = A.device
        self._A = _vector(A, H, "A", A.device)
        self._D = _vector(D, H, "D", A.device)
        self._dt_bias = _vector(dt_bias, H, "dt_bias", A.device)
        self.desc = ScanDesc(batch, H, head_dim, state_size, groups, 1 if dt_softplus else 0,
                             DTYPES[dtype], DTYPES[dtype])
        nb = i64()
        check(co_scan_query(ctypes.byref(self.desc), ctypes.byref(nb)), "co_scan_query")
        self._keep_state(state, torch.float32, (batch, H, head_dim, state_size), self.device)
        call = self._call = ScanCall(_ptr(self._A), _ptr(self._D), _ptr(self._dt_bias))
        self._parts = call.x, call.dt, call.b, call.c, call.y
        self._args = ctypes.byref(self.desc), ctypes.byref(call)
        self._sig = None

    # parameters: a call takes those that the layer was made with
    A = property(lambda self: self._A)
    D = property(lambda self: self._D)
    dt_bias = property(lambda self: self._dt_bias)

    def workspace_bytes(self, T):
        """Device workspace of a call over T tokens."""
        nb = i64()
        check(co_scan_workspace_bytes(ctypes.byref(self.desc), T, ctypes.byref(nb)),
              "co_scan_workspace_bytes")
        return nb.value

    def _check(self, x, dt, b, c, out, step, state, update):
        B, H, P, call = self.batch, self.heads, self.head_dim, self._call
        T = 1 if step else x.shape[1] if x.dim() == 4 else -1
        dtype = self.torch_dtype
        dt_dtype = torch.float32 if dt.dtype is torch.float32 else dtype
        bc = (B, T, self.groups, self.state_size)
        for t, kind, shape, what, into in ((x, dtype, (B, T, H, P), "x", call.x),
                                           (dt, dt_dtype, (B, T, H), "dt", call.dt),
                                           (b, dtype, bc, "b", call.b),
                                           (c, dtype, bc, "c", call.c),
                                           (out, dtype, (B, T, H, P), "out", call.y)):
            if t is None:
                into.batch_stride, into.token_stride = T * H * P, H * P
                continue
            if t.dim() != len(shape) - step:
                raise ValueError(f"{what} has shape {tuple(t.shape)}, expected "
                                 f"{shape[:1] + shape[2:] if step else shape}")
            _tokens(t, kind, shape, what, into, self.device)
        self.desc.dt_dtype = DTYPES[dt_dtype]
        call.T, call.state, call.update_state = T, state, update
        self._dense = x.is_contiguous()
        self._nws = call.workspace_bytes = self.workspace_bytes(T)

    def _run(self, x, dt, b, c, lengths, state, update, out, step=False):
        sig = (step, x.shape, x.stride(), x.dtype, x.get_device(), dt.shape, dt.stride(), dt.dtype,
               dt.get_device(), b.shape, b.stride(), b.dtype, b.get_device(), c.shape, c.stride(),
               c.dtype, c.get_device(), state, update,
               None if out is None else (out.shape, out.stride(), out.dtype, out.get_device()))
        if sig != self._sig:
            self._sig = None
            self._check(x, dt, b, c, out, step, state, update)
            self._sig = sig
        if out is None:
            out = _like(x) if self._dense else x.new_empty(x.shape)
        ix, idt, ib, ic, iy = self._parts
        ix.data, idt.data, ib.data = x.data_ptr(), dt.data_ptr(), b.data_ptr()
        ic.data, iy.data = c.data_ptr(), out.data_ptr()
        call = self._call
        call.lengths = None if lengths is None else _lengths(lengths, self.batch, self.device)
        ws = None
        if self._nws:
            ws = torch.empty(self._nws, dtype=torch.uint8, device=x.device)
            call.workspace = ws.data_ptr()
        pd, pc = self._args
        st = co_scan_forward_steps(pd, pc, _stream())
        if st != CO_OK:
            check(st, "co_scan_forward_steps")
        return out

    def forward_steps(self, x, dt, b, c, lengths=None, update_state=True, out=None):
        """The next T tokens: x (B, T, H, P), dt (B, T, H), b and c (B, T, G, N) -> (B, T, H, P)."""
        return self._run(x, dt, b, c, lengths, self._state.data_ptr(), 1 if update_state else 0,
                         out)

    def forward_step(self, x_t, dt_t, b_t, c_t, lengths=None, update_state=True, out=None):
        """The next token of each stream (of those with length 1): the same without T."""
        return self._run(x_t, dt_t, b_t, c_t, lengths, self._state.data_ptr(),
                         1 if update_state else 0, out, True)

    def forward(self, x, dt, b, c, lengths=None, out=None):
        """Whole sequences from a clean state, which the layer's own is not touched by."""
        return self._run(x, dt, b, c, lengths, None, 0, out)


class CoNorm:
    """Root-mean-square norm of the last axis, in `groups` equal parts, with a
    gate and a residual sum in the same pass (co_norm_forward).

    weight (D,) and scale (D,), the residual's: parameters, taken as float32,
    either may be None (1; then dim says D).  gate "before" norms x silu(gate),
    "after" multiplies the normed values.  residual "before" (a pre-norm) adds
    scale x to the residual and norms the sum; "after" (a post-norm) adds the
    normed values times scale.  Stateless, delay 0: forward, forward_step and
    forward_steps are one (update_state, which chains pass on, says nothing here).
    """

    delay, receptive_field, t_stride, t_padding = 0, 1, 1, 0
    MODES = {None: CO_NORM_NONE, "before": CO_NORM_BEFORE, "after": CO_NORM_AFTER}

    def __init__(self, weight=None, *, dim=None, eps=1e-5, groups=1, gate=None, residual=None,
                 scale=None):
        given = weight if weight is not None else scale
        if given is None and dim is None:
            raise ValueError("weight, scale or dim must be given")
        self.dim = dim if dim is not None else given.shape[0]
        if groups < 1 or self.dim % groups:
            raise ValueError(f"groups {groups} does not divide dim {self.dim}")
        if scale is not None and residual is None:
            raise ValueError("scale is the residual's")
        for t, what in ((weight, "weight"), (scale, "scale")):
            if t is not None and t.device.type != "cuda":
                raise ValueError(f"{what} must be a device tensor")
        self.device = given.device if given is not None else None  # None: any input's
        self._weight = _vector(weight, self.dim, "weight", self.device)
        self._scale = _vector(scale, self.dim, "scale", self.device)
        self.gate, self.residual = gate, residual
        self.desc = NormDesc(0, 0, self.dim, groups, self.MODES[gate], self.MODES[residual], CO_F32,
                             CO_F32, eps)
        call = self._call = NormCall(weight=_ptr(self._weight), scale=_ptr(self._scale))
        self._x, self._z, self._r, self._y, self._o = (call.x, call.gate, call.residual, call.y,
                                                       call.residual_out)
        self._args = ctypes.byref(self.desc), ctypes.byref(call)
        self._sig = None

    # parameters: a call takes those that the layer was made with
    weight = property(lambda self: self._weight)
    scale = property(lambda self: self._scale)

    def _rows(self, t, dtype, shape, tokens, what, into, device):
        _on(t, device, what)
        if t.dtype is not dtype:
            raise ValueError(f"{what} has dtype {t.dtype}, expected {dtype}")
        if t.shape != shape:
            raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if t.numel() == 0:
            into.batch_stride = into.token_stride = 0
            return
        try:
            v = t if t.dim() == 3 else t.view(-1, tokens, self.dim)
        except RuntimeError:
            raise ValueError(f"{what}: the leading axes must be evenly spaced") from None
        if self.dim != 1 and v.stride(2) != 1:
            raise ValueError(f"{what}: the values of a row must be contiguous")
        into.batch_stride, into.token_stride = v.stride(0), v.stride(1)

    def forward(self, x, gate=None, residual=None, out=None, residual_out=None, lengths=None):
        """x (..., D), gate of its shape and dtype, residual of its shape (float32 or
        bfloat16) -> y; (y, new residual) with residual "before"; the new residual
        with "after".  out may be x, residual_out may be residual.  lengths (of x
        (B, T, D), or (B, D) for single tokens): as CoShortConv's."""
        sig = (lengths is None, x.shape, x.stride(), x.dtype, x.get_device(),
               None if gate is None else (gate.shape, gate.stride(), gate.dtype, gate.get_device()),
               None if residual is None else (residual.shape, residual.stride(), residual.dtype,
                                              residual.get_device()),
               None if out is None else (out.shape, out.stride(), out.dtype, out.get_device()),
               None if residual_out is None else (residual_out.shape, residual_out.stride(),
                                                  residual_out.dtype, residual_out.get_device()))
        if sig != self._sig:
            self._sig = None
            self._check(x, gate, residual, out, residual_out, lengths is not None)
            self._sig = sig
        form = self.residual
        self._x.data = x.data_ptr()
        if gate is not None:
            self._z.data = gate.data_ptr()
        if form is not None:
            if residual_out is None:
                residual_out = _like(residual) if self._dense[1] else residual.new_empty(x.shape)
            self._r.data, self._o.data = residual.data_ptr(), residual_out.data_ptr()
        if form != "after":
            if out is None:
                out = _like(x) if self._dense[0] else x.new_empty(x.shape)
            self._y.data = out.data_ptr()
        pd, pc = self._args
        if lengths is None:
            st = co_norm_forward(pd, pc, _stream())
        else:
            st = co_norm_forward_lengths(pd, pc, _lengths(lengths, x.shape[0], x.device), _stream())
        if st != CO_OK:
            check(st, "co_norm_forward")
        if form is None:
            return out
        return residual_out if form == "after" else (out, residual_out)

    def _check(self, x, gate, residual, out, residual_out, ragged):
        if (gate is None) != (self.gate is None) or (residual is None) != (self.residual is None):
            raise ValueError("gate and residual are given to the layers that have them")
        shape, d = x.shape, self.desc
        if x.dim() == 0 or shape[-1] != self.dim:
            raise ValueError(f"x has shape {tuple(shape)}, expected (..., {self.dim})")
        if x.dtype not in DTYPES:
            raise ValueError(f"x has dtype {x.dtype}")
        if ragged and x.dim() not in (2, 3):
            raise ValueError(f"x has shape {tuple(shape)}, expected (B, T, {self.dim}) or "
                             f"(B, {self.dim}) beside lengths")
        tokens = shape[-2] if x.dim() > (2 if ragged else 1) else 1
        d.tokens, d.dtype = tokens, DTYPES[x.dtype]
        d.batch = x.numel() // (tokens * self.dim) if tokens else 0
        dev = x.device if self.device is None else self.device
        self._rows(x, x.dtype, shape, tokens, "x", self._x, dev)
        if gate is not None:
            self._rows(gate, x.dtype, shape, tokens, "gate", self._z, dev)
        if residual is not None:
            if residual.dtype not in DTYPES:
                raise ValueError(f"residual has dtype {residual.dtype}")
            d.residual_dtype = DTYPES[residual.dtype]
            self._rows(residual, residual.dtype, shape, tokens, "residual", self._r, dev)
            self._o.batch_stride, self._o.token_stride = tokens * self.dim, self.dim
            if residual_out is not None:
                self._rows(residual_out, residual.dtype, shape, tokens, "residual_out", self._o,
                           dev)
        self._y.batch_stride, self._y.token_stride = tokens * self.dim, self.dim
        if out is not None:
            self._rows(out, x.dtype, shape, tokens, "out", self._y, dev)
        self._dense = x.is_contiguous(), residual is not None and residual.is_contiguous()

    def forward_steps(self, x, gate=None, residual=None, out=None, residual_out=None,
                      lengths=None, update_state=True):
        return self.forward(x, gate, residual, out, residual_out, lengths)

    forward_step = forward_steps

    def clean_state(self):
        pass


class Mixer:
    """A selective state space mixer between its two projections: a CoShortConv
    over the columns x, B and C, a CoScan over its output and dt, and a CoNorm
    gated by z.  Inputs u (B, T, W) are a projection's columns [z | x | B | C | dt]
    of H P, H P, G N, G N and H values; outputs (B, T, H P).  Call modes, lengths
    and states as its layers'; delay 0."""

    delay, receptive_field, t_stride, t_padding = 0, 1, 1, 0

    def __init__(self, conv, scan, norm):
        self.inner = scan.heads * scan.head_dim
        shared = scan.groups * scan.state_size
        if conv.channels != self.inner + 2 * shared or norm.dim != self.inner:
            raise ValueError(f"the convolution has {conv.channels} channels and the norm "
                             f"{norm.dim} values, expected {self.inner + 2 * shared} and "
                             f"{self.inner}")
        if norm.gate is None or norm.residual is not None:
            raise ValueError("the mixer's norm has a gate and no residual")
        if conv.batch != scan.batch or conv.torch_dtype != scan.torch_dtype:
            raise ValueError("the layers' batches and dtypes differ")
        self.conv, self.scan, self.norm = conv, scan, norm
        self.batch, self.torch_dtype = scan.batch, scan.torch_dtype
        self._columns = (self.inner, conv.channels, scan.heads)
        self._split = (self.inner, shared, shared)
        self.width = sum(self._columns)

    def _run(self, u, lengths, conv, scan):
        z, xbc, dt = u.split(self._columns, -1)
        s = self.scan
        x, b, c = conv(xbc).split(self._split, -1)
        lead = u.shape[:-1]
        bc = lead + (s.groups, s.state_size)
        y = scan(x.view(lead + (s.heads, s.head_dim)), dt, b.view(bc), c.view(bc))
        return self.norm.forward(y.view(z.shape), gate=z, lengths=lengths)

    def forward_steps(self, u, lengths=None, update_state=True):
        """The next T tokens u (B, T, W) of the streams -> (B, T, H P)."""
        return self._run(u, lengths, lambda v: self.conv.forward_steps(v, lengths, update_state),
                         lambda *v: self.scan.forward_steps(*v, lengths, update_state))

    def forward_step(self, u_t, lengths=None, update_state=True):
        """The next token u_t (B, W) of each stream (of those with length 1) -> (B, H P)."""
        return self._run(u_t, lengths, lambda v: self.conv.forward_step(v, lengths, update_state),
                         lambda *v: self.scan.forward_step(*v, lengths, update_state))

    def forward(self, u, lengths=None):
        """Whole sequences from a clean state, which the mixer's own is not touched by."""
        return self._run(u, lengths, lambda v: self.conv.forward(v, lengths),
                         lambda *v: self.scan.forward(*v, lengths))

    def clean_state(self):
        self.conv.clean_state()
        self.scan.clean_state()


# ------------------------------------------------- attention over token streams
# Rotary positions, pages of a cache in 4 bits, and attention over it.  As the
# token layers: plain device tensors as state, argument checks kept between like
# calls, one thread a layer.


def _enqueue(index, what, fn, *args):
    """Calls an entry point on the current stream of a layer's GPU."""
    if _current_raw_stream is not None and _current_device() == index:
        st = fn(*args, _current_raw_stream(index))
    else:
        with torch.cuda.device(index):
            st = fn(*args, torch.cuda.current_stream(index).cuda_stream)
    if st != CO_OK:
        check(st, what)


def _device(device):
    """A GPU with its index."""
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError(f"device is {device}, expected a GPU")
    return device if device.index is not None else torch.device("cuda",
                                                                torch.cuda.current_device())


def _key(t):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


class CoRotary:
    """Rotary positions (co_rotary_forward): the first rotary_dim values of each head
    are pairs that turn with the position, base^(-2 i / rotary_dim) radians of it.

    layout: "half" (values i and i + rotary_dim / 2 are a pair) or "interleaved"
    (2 i and 2 i + 1).  scaling, for contexts longer than trained ones: None, or a dict
    of kind "linear" (all angles divided by factor), "base" (a base so much larger that the
    slowest angle is divided by it) or "parts" (angles that make less than low turns
    in `original` positions are divided, those that make more than high stay, those
    between in part), with factor and, for "parts", original, low and high.  magnitude
    multiplies what turns.  Stateless, delay 0.
    """

    delay, receptive_field, t_stride, t_padding = 0, 1, 1, 0
    LAYOUTS = {"half": CO_ROTARY_HALF, "interleaved": CO_ROTARY_INTERLEAVED}
    SCALINGS = {"linear": (CO_ROTARY_LINEAR, ()), "base": (CO_ROTARY_BASE, ()),
                "parts": (CO_ROTARY_PARTS, ("original", "low", "high"))}

    def __init__(self, head_dim, *, rotary_dim=None, base=10000.0, layout="half", scaling=None,
                 magnitude=1.0, device="cuda"):
        self.head_dim = head_dim
        self.rotary_dim = head_dim if rotary_dim is None else rotary_dim
        if layout not in self.LAYOUTS:
            raise ValueError(f"layout {layout!r}, expected one of {sorted(self.LAYOUTS)}")
        if not 2 <= self.rotary_dim <= head_dim or self.rotary_dim % 2:
            raise ValueError(f"rotary_dim {self.rotary_dim} of {head_dim} values: expected an even "
                             f"part of them")
        how = None
        if scaling is not None:
            kind = scaling.get("kind")
            if kind not in self.SCALINGS:
                raise ValueError(f"scaling kind {kind!r}, expected one of {sorted(self.SCALINGS)}")
            number, more = self.SCALINGS[kind]
            want = {"kind", "factor", *more}
            if set(scaling) != want:
                raise ValueError(f"scaling {kind!r} has {sorted(want)}")
            how = RotaryScaling(number, *(float(scaling[k]) if k in scaling else 0.0
                                          for k in ("factor", "original", "low", "high")))
        turns = (ctypes.c_uint64 * (self.rotary_dim // 2))()
        check(co_rotary_turns(self.rotary_dim, float(base),
                              None if how is None else ctypes.byref(how), turns),
              "co_rotary_turns")
        self.device = _device(device)
        self._turns = torch.tensor([ctypes.c_int64(v).value for v in turns],
                                   dtype=torch.int64).to(self.device)
        self.desc = RotaryDesc(0, I32x2(0, 0), head_dim, self.rotary_dim, self.LAYOUTS[layout],
                               CO_F32, float(magnitude))
        self._call = RotaryCall(turns=_ptr(self._turns))
        self._x, self._y = tuple(self._call.x), tuple(self._call.y)
        self._args = ctypes.byref(self.desc), ctypes.byref(self._call)
        self._sig = None

    def _check(self, x, k, positions, out, k_out, step):
        d, call = self.desc, self._call
        if x.dtype not in DTYPES:
            raise ValueError(f"x has dtype {x.dtype}")
        d.dtype = DTYPES[x.dtype]
        if k is None and k_out is not None:
            raise ValueError("k_out is k's")
        if x.dim() != 4 - step:
            raise ValueError(f"x has shape {tuple(x.shape)}, expected "
                             f"{('B', 'H', 'D') if step else ('B', 'T', 'H', 'D')}")
        B, T = x.shape[0], 1 if step else x.shape[1]
        d.batch, call.T = B, T
        d.heads[1] = 0
        self._dense = []
        for i, (t, o, what) in enumerate(((x, out, "x"), (k, k_out, "k"))):
            if t is None:
                continue
            if t.dim() != x.dim():
                raise ValueError(f"{what} has shape {tuple(t.shape)}, expected as x's")
            shape = torch.Size((B, T, t.shape[-2], self.head_dim))
            _tokens(t, x.dtype, shape, what, self._x[i], self.device)
            d.heads[i] = t.shape[-2]
            width = t.shape[-2] * self.head_dim
            self._y[i].batch_stride, self._y[i].token_stride = T * width, width
            if o is not None:
                if o.dim() != x.dim():
                    raise ValueError(f"out has shape {tuple(o.shape)}, expected as {what}'s")
                _tokens(o, x.dtype, shape, "out", self._y[i], self.device)
            self._dense.append(t.is_contiguous())
        if positions is not None:
            _on(positions, self.device, "positions")
            if positions.dtype is not torch.int32:
                raise ValueError(f"positions has dtype {positions.dtype}, expected torch.int32")
            each = positions.dim() == 2
            if positions.shape not in ((B,), (B, T)):
                raise ValueError(f"positions has shape {tuple(positions.shape)}, expected ({B},) or "
                                 f"({B}, {T})")
            call.position_batch_stride = positions.stride(0)
            call.position_token_stride = positions.stride(1) if each else 0
            call.position_each = 1 if each else 0

    def _run(self, x, k, positions, lengths, out, k_out, step):
        sig = (step, _key(x), _key(k), _key(positions), _key(out), _key(k_out))
        if sig != self._sig:
            self._sig = None
            self._check(x, k, positions, out, k_out, step)
            self._sig = sig
        call, d = self._call, self.desc
        if out is None:
            out = _like(x) if self._dense[0] else x.new_empty(x.shape)
        self._x[0].data, self._y[0].data = x.data_ptr(), out.data_ptr()
        if k is not None:
            if k_out is None:
                k_out = _like(k) if self._dense[1] else k.new_empty(k.shape)
            self._x[1].data, self._y[1].data = k.data_ptr(), k_out.data_ptr()
        call.positions = None if positions is None else positions.data_ptr()
        call.lengths = None if lengths is None else _lengths(lengths, x.shape[0], self.device)
        if call.T and d.batch:
            _enqueue(self.device.index, "co_rotary_forward", co_rotary_forward, *self._args)
        return out if k is None else (out, k_out)

    def forward(self, x, k=None, *, positions=None, lengths=None, out=None, k_out=None):
        """x (B, T, H, D), and k (B, T, H', D) in the same launch -> x, or (x, k), turned.
        positions, int32 on the device: (B,) of each stream's first token, or (B, T); default 0,
        1, ...  out may be x, k_out may be k.  lengths: as CoShortConv's."""
        return self._run(x, k, positions, lengths, out, k_out, 0)

    forward_steps = forward

    def forward_step(self, x_t, k_t=None, *, positions=None, lengths=None, out=None, k_out=None):
        """The same of single tokens, (B, H, D)."""
        return self._run(x_t, k_t, positions, lengths, out, k_out, 1)

    def clean_state(self):
        pass


class CoPages:
    """Pages of a cache of keys and values in 4 bits (co_pages_* ABI), for all layers of a
    model: which stream holds which tokens where.

    A pool of `pages` pages of page_tokens tokens (16 to 256) in each of the layers; a
    stream holds at most stream_pages of them at once, as many as its length or, with
    reserve's keep, its window needs.  Everything is a plain device tensor, and no call
    waits for the device:

    pool (layers, pages, page_bytes) uint8; table (batch, stream_pages) int32, position p of
    stream b in page table[b, p // page_tokens % stream_pages]; tokens, first (batch,), a
    stream's length and the lowest position it still holds; refs (pages,), how many streams hold
    a page; base, granted (batch,), the length before the newest reserve and what it
    gave; refused (batch,), what reserves refused, summed.  state: a dict of any of them
    to keep and continue from; default clean ones.
    """

    def __init__(self, *, batch, pages, stream_pages, kv_heads, head_dim, page_tokens=64, layers=1,
                 device=None, state=None):
        self.batch, self.pages, self.stream_pages = batch, pages, stream_pages
        self.kv_heads, self.head_dim = kv_heads, head_dim
        self.page_tokens, self.layers = page_tokens, layers
        self.desc = PagesDesc(batch, pages, page_tokens, stream_pages, layers, kv_heads, head_dim)
        info = PagesInfo()
        check(co_pages_query(ctypes.byref(self.desc), ctypes.byref(info)), "co_pages_query")
        self.page_bytes = info.page_bytes
        state = {} if state is None else dict(state)
        if device is None:
            given = next(iter(state.values()), None)
            device = "cuda" if given is None else given.device
        self.device = _device(device)
        shapes = dict(pool=(layers, pages, self.page_bytes), table=(batch, stream_pages),
                      tokens=(batch,), first=(batch,), refs=(pages,), base=(batch,),
                      granted=(batch,), refused=(batch,))
        if not set(state) <= set(shapes):
            raise ValueError(f"state has {sorted(state)}, expected some of {sorted(shapes)}")
        self._state = {}
        for name, shape in shapes.items():
            dtype = torch.uint8 if name == "pool" else torch.int32
            t = state.get(name)
            if t is None:
                t = (torch.empty if name == "pool" else torch.zeros)(shape, dtype=dtype,
                                                                     device=self.device)
                if name == "table":
                    t.fill_(-1)
            _need(t, dtype, shape, name)
            _on(t, self.device, name)
            self._state[name] = t
        self._call = Pages(*(_ptr(self._state[k]) for k in shapes))
        # as the state, one call's at a time
        self._ws = torch.empty(info.workspace_bytes, dtype=torch.uint8, device=self.device)
        self._call.workspace = self._ws.data_ptr()
        self._args = ctypes.byref(self.desc), ctypes.byref(self._call)
        self._T = None  # tokens of the newest reserve

    pool = property(lambda self: self._state["pool"])
    table = property(lambda self: self._state["table"])
    tokens = property(lambda self: self._state["tokens"])
    first = property(lambda self: self._state["first"])
    refs = property(lambda self: self._state["refs"])
    base = property(lambda self: self._state["base"])
    granted = property(lambda self: self._state["granted"])
    refused = property(lambda self: self._state["refused"])

    def _run(self, what, fn, *args):
        _enqueue(self.device.index, what, fn, *self._args, *args)

    def reserve(self, T, lengths=None, keep=0):
        """Pages for the next T tokens of each stream (lengths, as CoShortConv's, of
        them), which its layers then append and attend to -> granted: how many each stream got, all
        it asked for or none where pages are short.  keep > 0: positions that no
        window of `keep` tokens sees any more are given up first.  Pages that other streams
        hold too are copied, not written."""
        self._run("co_pages_reserve", co_pages_reserve, T,
                  None if lengths is None else _lengths(lengths, self.batch, self.device), keep)
        self._T = T
        return self.granted

    def truncate(self, tokens):
        """Gives up each stream's tokens from position tokens[b] (int32 on the device) on; with
        tokens=self.base those of the newest reserve, as after rejected drafts."""
        self._run("co_pages_truncate", co_pages_truncate,
                  _lengths(tokens, self.batch, self.device))
        self._T = None

    def select(self, source):
        """Every stream b at once becomes what stream source[b] (int32 on the device) was, and shares
        its pages: itself, another one (a fork), or with -1 an empty stream, whose pages
        are free where nobody else holds them."""
        self._run("co_pages_select", co_pages_select, _lengths(source, self.batch, self.device))
        self._T = None

    def compact(self):
        """Moves the pages in use to the lowest indexes of the pool, in every layer."""
        self._run("co_pages_compact", co_pages_compact)

    def clean_state(self):
        for name, t in self._state.items():
            if name == "table":
                t.fill_(-1)
            elif name != "pool":
                t.zero_()
        self._T = None


class CoAttention:
    """Causal attention over token streams (co_attn_* ABI): keys and values go into
    one layer of a CoPages in 4 bits, and each token attends to what its stream
    holds up to itself, or to the newest `window` tokens of that.

    heads: query heads, a multiple of the pages' kv_heads, which neighbouring ones share.
    scale: of the products, default head_dim ** -0.5.  dtype: of q, k, v and the output.
    A step of a model: pages.reserve(T, lengths), then each layer's forward_steps; tokens that
    the reserve did not grant give 0.  Delay 0; the state is the pages'.
    """

    delay, t_stride, t_padding = 0, 1, 0

    def __init__(self, pages, layer=0, *, heads, window=None, scale=None, dtype=torch.bfloat16):
        if not 0 <= layer < pages.layers:
            raise ValueError(f"layer {layer} of {pages.layers}")
        if window is not None and window < 1:
            raise ValueError(f"window {window}")
        if dtype not in DTYPES:
            raise ValueError(f"dtype {dtype}")
        self.pages, self.layer, self.heads, self.window = pages, layer, heads, window
        self.batch, self.kv_heads, self.head_dim = pages.batch, pages.kv_heads, pages.head_dim
        self.torch_dtype, self.device = dtype, pages.device
        self.scale = self.head_dim ** -0.5 if scale is None else float(scale)
        self.desc = self._desc(pages.pages, pages.stream_pages)
        check(co_attn_workspace_bytes(ctypes.byref(self.desc), 0, ctypes.byref(i64())),
              "co_attn_workspace_bytes")
        pool = pages.pool[layer]
        self._cache = AttnCache(_ptr(pool), _ptr(pages.table), _ptr(pages.base),
                                _ptr(pages.granted), _ptr(pages.first))
        self._q, self._k, self._v, self._y, self._rk, self._rv = (Tokens() for _ in range(6))
        self._ref = {t: ctypes.byref(getattr(self, t))
                     for t in ("_q", "_k", "_v", "_y", "_rk", "_rv")}
        self._args = ctypes.byref(self.desc), ctypes.byref(self._cache)
        self._append_sig = self._attend_sig = None

    receptive_field = property(lambda self: self.window)  # None: all that a stream holds

    def _desc(self, pages, stream_pages):
        return AttnDesc(self.batch, self.heads, self.kv_heads, self.head_dim, pages,
                        self.pages.page_tokens, stream_pages, self.window or 0,
                        DTYPES[self.torch_dtype], self.scale)

    def _tokens(self, t, heads, what, into, step):
        shape = (self.batch, 1 if step else t.shape[1] if t.dim() == 4 else -1, heads,
                 self.head_dim)
        if t.dim() != 4 - step:
            raise ValueError(f"{what} has shape {tuple(t.shape)}, expected "
                             f"{shape[:1] + shape[2:] if step else shape[:1] + ('T',) + shape[2:]}")
        _tokens(t, self.torch_dtype, torch.Size(shape), what, into, self.device)
        return shape[1]

    def _reserved(self, T):
        if self.pages._T is not None and T != self.pages._T:
            raise ValueError(f"{T} tokens, but the newest reserve was for {self.pages._T}")

    def _append(self, k, v, step, args):
        sig = step, _key(k), _key(v)
        if sig != self._append_sig:
            self._append_sig = None
            T = self._tokens(k, self.kv_heads, "k", self._k, step)
            if self._tokens(v, self.kv_heads, "v", self._v, step) != T:
                raise ValueError(f"k has {T} tokens, v {v.shape[1]}")
            self._append_T = T
            self._append_sig = sig
        self._k.data, self._v.data = k.data_ptr(), v.data_ptr()
        if self._append_T:
            _enqueue(self.device.index, "co_attn_append", co_attn_append, *args, self._ref["_k"],
                     self._ref["_v"], self._append_T)
        return self._append_T

    def _attend(self, q, out, step, desc, args):
        sig = step, _key(q), _key(out), desc.stream_pages
        if sig != self._attend_sig:
            self._attend_sig = None
            T = self._tokens(q, self.heads, "q", self._q, step)
            width = self.heads * self.head_dim
            self._y.batch_stride, self._y.token_stride = T * width, width
            if out is not None and self._tokens(out, self.heads, "out", self._y, step) != T:
                raise ValueError(f"q has {T} tokens, out {out.shape[1]}")
            nb = i64()
            check(co_attn_workspace_bytes(ctypes.byref(desc), T, ctypes.byref(nb)),
                  "co_attn_workspace_bytes")
            self._attend_T, self._nws, self._dense = T, nb.value, q.is_contiguous()
            self._attend_sig = sig
        if out is None:
            out = _like(q) if self._dense else q.new_empty(q.shape)
        ws = None
        if self._nws:
            ws = torch.empty(self._nws, dtype=torch.uint8, device=self.device)
        self._q.data, self._y.data = q.data_ptr(), out.data_ptr()
        if self._attend_T:
            _enqueue(self.device.index, "co_attn_forward_steps", co_attn_forward_steps, *args,
                     self._ref["_q"], self._ref["_y"], self._attend_T, _ptr(ws), self._nws)
        return out

    def append(self, k, v):
        """Puts k and v (B, T, kv_heads, D) of the newest reserve's tokens into the cache."""
        self._reserved(k.shape[1] if k.dim() == 4 else 1)
        self._append(k, v, 0, self._args)

    def attend(self, q, out=None):
        """The newest reserve's tokens q (B, T, heads, D), appended before, over the cache ->
        (B, T, heads, D)."""
        self._reserved(q.shape[1] if q.dim() == 4 else 1)
        return self._attend(q, out, 0, self.desc, self._args)

    def forward_steps(self, q, k, v, out=None):
        """append and attend."""
        self.append(k, v)
        return self.attend(q, out)

    def forward_step(self, q_t, k_t, v_t, out=None):
        """The same of single tokens, (B, heads, D) and (B, kv_heads, D)."""
        self._reserved(1)
        self._append(k_t, v_t, 1, self._args)
        return self._attend(q_t, out, 1, self.desc, self._args)

    def forward(self, q, k, v, lengths=None, out=None):
        """Whole sequences from their start, through a cache of the call's own: the layer's pages are
        not touched.  lengths: as CoShortConv's."""
        P, B = self.pages.page_tokens, self.batch
        T = q.shape[1] if q.dim() == 4 else 0
        if k.dim() == 4 and k.shape[1] != T:
            raise ValueError(f"q has {T} tokens, k {k.shape[1]}")
        each = max(1, -(-T // P))
        desc = self._desc(B * each, each)
        pool = torch.empty(B * each * self.pages.page_bytes, dtype=torch.uint8, device=self.device)
        table = torch.arange(B * each, dtype=torch.int32, device=self.device)
        base = torch.zeros(B, dtype=torch.int32, device=self.device)
        cache = AttnCache(_ptr(pool), _ptr(table), _ptr(base),
                          None if lengths is None else _lengths(lengths, B, self.device), None)
        args = ctypes.byref(desc), ctypes.byref(cache)
        self._append(k, v, 0, args)
        return self._attend(q, out, 0, desc, args)

    def read(self, first, T):
        """What the cache holds at positions first[b] .. first[b] + T - 1 (first int32 on the device) of
        each stream -> keys and values (B, T, kv_heads, D), 0 where it holds nothing."""
        shape = self.batch, T, self.kv_heads, self.head_dim
        k = torch.empty(shape, dtype=self.torch_dtype, device=self.device)
        v = _like(k)
        width = self.kv_heads * self.head_dim
        for t, into in ((k, self._rk), (v, self._rv)):
            into.data, into.batch_stride, into.token_stride = t.data_ptr(), T * width, width
        if T:
            _enqueue(self.device.index, "co_attn_read", co_attn_read, *self._args,
                     _lengths(first, self.batch, self.device), self._ref["_rk"], self._ref["_rv"],
                     T)
        return k, v
