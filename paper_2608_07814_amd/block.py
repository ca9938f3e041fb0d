"""The operators around the expert layer and the experts in 4 bits
(include/lorex_block.h), bound like ``lorex``: argument marshalling only.

* :func:`block_norm`, :func:`block_norm_backward`: the norms before and after a
  block with its gate and residual scale;
* :func:`block_norm_dropout`, :func:`block_norm_dropout_backward`: the same with the
  block's output dropped out;
* :func:`block_norm_mx8`: the same with the next block's input in 8 bits;
* :func:`route_topk_logits`: the router with its logits;
* :func:`balance_loss`, :func:`balance_loss_backward`: the router's balance
  loss, the tokens per expert, the gradient of the logits;
* :func:`mx4_quantize`, :func:`mx4_dequantize`, :func:`mx4_gemm`: microscaled
  4-bit values, and products of them per group of rows;
* :func:`mx8_quantize`, :func:`mx8_dequantize`, :func:`mx8_gemm`: microscaled 8-bit
  values, and products of 8-bit activations and 4-bit weights with a bias, an
  activation and a residual;
* :class:`Mx4Experts`, :func:`mx4_moe_block`: a MoE block whose experts are held
  in 4 bits, built from these and the library's router and bucketing;
* :func:`mx4_moe_few`: the experts' layer for a few tokens in two launches.

Tensors are contiguous and on one GPU, which need not be the current one. Calls
are asynchronous on ``stream`` (a ``torch.cuda.Stream`` of that GPU; default: its
current one). Outputs can be given; those that are not are allocated, as are
workspaces, in the order of the call's stream: with ``stream`` the caller has
that stream wait for inputs that another one makes, and its own stream wait for
that one before it uses the outputs. Autograd does not record these calls: their
outputs have no graph, whatever requires gradients; the gradients are the
``_backward`` calls.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import lorex as lx
from .lorex import LX_BF16, LX_F32, _check

MX4_NONE, MX4_SWIGLU = 0, 1
ACT_NONE, ACT_SILU, ACT_GELU, ACT_SWIGLU = 0, 1, 2, 3
NORM_MAX_D = 32768
MOE_FEW_MAX_T = 64

_c_void, _c_i32, _c_i64, _c_f32, _c_size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


class LxNormLayer(ctypes.Structure):
    _fields_ = [("d", _c_i32), ("h_dtype", _c_i32), ("y_dtype", _c_i32), ("x_dtype", _c_i32), ("w_dtype", _c_i32),
                ("residual_scale", _c_f32), ("eps", _c_f32), ("w_pre", _c_void), ("w_post", _c_void),
                ("scale", _c_void), ("gate", _c_void)]


class LxDropout(ctypes.Structure):
    _fields_ = [("p", _c_f32), ("rng", _c_void)]


class LxEpilogue(ctypes.Structure):
    _fields_ = [("act", _c_i32), ("bias_dtype", _c_i32), ("residual_dtype", _c_i32), ("bias", _c_void), ("residual", _c_void)]


EXPORTS = {
    "lx_mx8_gemm_workspace_bytes": (_c_size, [_c_i32] * 5),
    "lx_mx8_gemm": (_c_i32, [_c_void, _c_void, _c_i32, _c_void, _c_void, _c_void, _c_void, _c_i32, _c_i32, _c_i32, _c_i32,
                             _c_void, _c_void, _c_i32, _c_void, _c_void, _c_size, _c_void]),
    "lx_mx4_moe_few_workspace_bytes": (_c_size, [_c_i32] * 5),
    "lx_mx4_moe_few": (_c_i32, [_c_void, _c_i32, _c_i32, _c_i32, _c_void, _c_void, _c_i32, _c_i32, _c_i32] + [_c_void] * 5
                       + [_c_i32, _c_void, _c_size, _c_void]),
    "lx_block_norm_mx8": (_c_i32, [_c_void, _c_i32, _c_void, _c_void, _c_i32, _c_i32] + [_c_void] * 7),
    "lx_block_norm_dropout": (_c_i32, [_c_void, _c_void, _c_i32] + [_c_void] * 5),
    "lx_block_norm_dropout_backward": (_c_i32, [_c_void, _c_void, _c_i32] + [_c_void] * 11 + [_c_size, _c_void]),
    "lx_mx8_quantize": (_c_i32, [_c_void, _c_i32, _c_i64, _c_i32, _c_i32, _c_void, _c_void, _c_void]),
    "lx_mx8_dequantize": (_c_i32, [_c_void, _c_void, _c_i64, _c_i32, _c_void, _c_i32, _c_void]),
    "lx_block_norm": (_c_i32, [_c_void, _c_i32, _c_void, _c_void, _c_i32, _c_i32] + [_c_void] * 5),
    "lx_block_norm_backward_workspace_bytes": (_c_size, [_c_i32, _c_i32]),
    "lx_block_norm_backward": (_c_i32, [_c_void, _c_i32] + [_c_void] * 11 + [_c_size, _c_void]),
    "lx_route_topk_logits": (_c_i32, [_c_void, _c_void, _c_i32, _c_i32, _c_i32, _c_i32, _c_i32] + [_c_void] * 4
                             + [_c_size, _c_void]),
    "lx_balance_loss_workspace_bytes": (_c_size, [_c_i32, _c_i32]),
    "lx_balance_loss": (_c_i32, [_c_void, _c_i32, _c_i32, _c_i32, _c_void, _c_i32, _c_void, _c_f32] + [_c_void] * 5
                        + [_c_size, _c_void]),
    "lx_balance_loss_backward": (_c_i32, [_c_void, _c_i32, _c_i32, _c_i32, _c_i32, _c_void, _c_void, _c_void, _c_f32,
                                          _c_void, _c_void, _c_void]),
    "lx_mx4_quantize": (_c_i32, [_c_void, _c_i32, _c_i64, _c_i32, _c_i32, _c_void, _c_void, _c_void]),
    "lx_mx4_dequantize": (_c_i32, [_c_void, _c_void, _c_i64, _c_i32, _c_void, _c_i32, _c_void]),
    "lx_mx4_gemm_workspace_bytes": (_c_size, [_c_i32] * 4),
    "lx_mx4_gemm": (_c_i32, [_c_void, _c_void, _c_i32, _c_void, _c_void, _c_void, _c_void, _c_i32, _c_i32, _c_i32,
                             _c_i32, _c_void, _c_i32, _c_void, _c_size, _c_void]),
}

_LIB: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """liblorex.so with this header's entry points declared."""
    global _LIB
    if _LIB is None:
        L = lx.lib()
        for name, (res, args) in EXPORTS.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = L
    return _LIB


# stands for the address of an empty tensor, which has none: NULL would mean
# that the argument is not given, and nothing is read there
_EMPTY = 256

_DTYPES = {torch.float32: LX_F32, torch.bfloat16: LX_BF16}


def _dtype(name: str, t: torch.Tensor) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise ValueError(f"{name} must be fp32 or bf16")
    return dt


def _gpu(name: str, t: torch.Tensor) -> int:
    """The index of the GPU that a call's tensors are on."""
    i = t.get_device()
    if i < 0:
        raise ValueError(f"{name} must be on a GPU")
    return i


def _arg(name: str, t: Optional[torch.Tensor], shape: tuple, dtype, gpu: int) -> Optional[int]:
    """Address of an argument after its checks (None stays None)."""
    if t is None:
        return None
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.get_device() != gpu:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{gpu}")
    return t.data_ptr() or _EMPTY


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr() or _EMPTY


# (torch.cuda.current_stream builds an object, 1.7 us of a call of 6)
_current_raw_stream = torch._C._cuda_getCurrentRawStream


_current_device = torch._C._cuda_getDevice
# (torch.cuda.stream's own way in and out takes 8 us)
_current_stream, _set_stream = torch._C._cuda_getCurrentStream, torch._C._cuda_setStream


def _there(fn, gpu: int, stream, args: dict):
    """``fn`` again, of the same arguments (its locals(), ``gpu`` among them), with the
    GPU of its tensors as the current one, where the library launches (the default
    stream's handle is the same on every GPU), and with the call's stream as the
    current one, so that what the call allocates is memory of that stream's order:
    memory of another stream's pool may still be in use by that stream's pending
    work."""
    del args["gpu"]
    if gpu != _current_device():
        with torch.cuda.device(gpu):
            return fn(**args)
    if stream.device_index != gpu:
        raise ValueError(f"stream is on cuda:{stream.device_index}, the tensors on cuda:{gpu}")
    args["stream"] = None
    number, device, kind = _current_stream(gpu)
    _set_stream(stream_id=stream.stream_id, device_index=gpu, device_type=stream.device_type)
    try:
        out = fn(**args)
    finally:
        _set_stream(stream_id=number, device_index=device, device_type=kind)
    _record(out, torch.Stream(stream_id=number, device_index=device, device_type=kind))
    return out


def _record(out, stream):
    """The memory of ``out``'s tensors, once they are freed, is not reused before
    ``stream`` has done the work that it has by then."""
    if isinstance(out, tuple):
        for v in out:
            _record(v, stream)
    elif hasattr(out, "record_stream"):
        out.record_stream(stream)


def _workspace(given: Optional[torch.Tensor], need: int, like: torch.Tensor):
    """(tensor to keep during the call, address, bytes)"""
    if given is None:
        if not need:
            return None, None, 0
        given = like.new_empty((need,), dtype=torch.uint8)
    elif given.dtype != torch.uint8 or not given.is_contiguous() or given.get_device() != like.get_device():
        raise ValueError(f"workspace must be contiguous uint8 on {like.device}")
    return given, given.data_ptr(), given.numel()


class Mx8(NamedTuple):
    """8-bit values: codes uint8 [..., Kp], scales uint8 [..., Kp / 32], and the K
    values of a row (Kp: :func:`mx4_padded`)."""
    codes: torch.Tensor
    scales: torch.Tensor
    K: int


# ------------------------------------------------------------ block norms
def _norm_layer(h, y, x_dtype, w_pre, w_post, scale, gate, residual_scale, eps, T, d, gpu) -> LxNormLayer:
    w = w_pre if w_pre is not None else w_post if w_post is not None else scale
    wt = None if w is None else w.dtype
    return LxNormLayer(d, _dtype("h", h), LX_F32 if y is None else _dtype("y", y), x_dtype,
                       LX_F32 if w is None else _dtype("weights", w), residual_scale, eps,
                       _arg("w_pre", w_pre, (d,), wt, gpu), _arg("w_post", w_post, (d,), wt, gpu),
                       _arg("scale", scale, (d,), wt, gpu), _arg("gate", gate, (T,), torch.float32, gpu))


def block_norm(h: torch.Tensor, y: Optional[torch.Tensor] = None, *, w_pre: Optional[torch.Tensor] = None,
               w_post: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
               gate: Optional[torch.Tensor] = None, slot_row: Optional[torch.Tensor] = None,
               slot_weights: Optional[torch.Tensor] = None, residual_scale: float = 1.0, eps: float = 1e-6,
               h_out: Optional[torch.Tensor] = None, x: Optional[torch.Tensor] = None,
               x_dtype: torch.dtype = torch.bfloat16, stream=None):
    """The norms around a block (lx_block_norm): the residual stream h [T][d]
    and the block's output y ([T][d], or rows [n][d] gathered by slot_row [T][k]
    and summed with slot_weights [T][k]) -> (h_out, x). Without y only x = h
    rms(h) w_pre is computed and h_out is h; without w_pre x is None. gate [T]
    fp32; w_pre, w_post, scale [d] of one dtype. x takes ``x_dtype`` unless it is
    given; h_out may be h."""
    if h.dim() != 2:
        raise ValueError("h must be [T][d]")
    gpu = _gpu("h", h)
    if stream is not None or gpu != _current_device():
        return _there(block_norm, gpu, stream, locals())
    return _block_norm(h, y, w_pre, w_post, scale, gate, slot_row, slot_weights, residual_scale, eps, h_out, x, x_dtype, None, gpu)


def _block_norm(h, y, w_pre, w_post, scale, gate, slot_row, slot_weights, residual_scale, eps, h_out, x, x_dtype, dropout, gpu,
                x_values=None):
    T, d = shape = h.shape
    k = y_rows = 0
    yp = None
    if y is not None:
        y_rows = y.shape[0]
        if slot_row is None:
            yp = _arg("y", y, shape, None, gpu)
        else:
            if slot_row.dim() != 2:
                raise ValueError("slot_row must be [T][k]")
            k = slot_row.shape[1]
            yp = _arg("y", y, (y_rows, d), None, gpu)
        if h_out is None:
            h_out = h.new_empty(shape, dtype=h.dtype)
    else:
        if h_out is not None or slot_row is not None or slot_weights is not None or any(v is not None for v in (w_post, scale, gate)):
            raise ValueError("h_out, slots, w_post, scale and gate go with y")
    if w_pre is None:
        if x is not None:
            raise ValueError("x goes with w_pre")
    elif x is None and x_dtype is not Mx8:
        x = h.new_empty(shape, dtype=x_dtype)
    plain = x_values if x_dtype is Mx8 else x  # x as a tensor
    s = _norm_layer(h, y, LX_BF16 if plain is None else _dtype("x", plain), w_pre, w_post, scale, gate, residual_scale, eps, T, d, gpu)
    hp, op = _arg("h", h, shape, None, gpu), _arg("h_out", h_out, shape, h.dtype, gpu)
    if x_dtype is Mx8:
        Kp = mx4_padded(d)
        if x is None:
            x = Mx8(h.new_empty((T, Kp), dtype=torch.uint8), h.new_empty((T, Kp // 32), dtype=torch.uint8), d)
            xp = _arg("x_values", x_values, shape, None, gpu), _ptr(x.codes), _ptr(x.scales)
        elif x.K != d:
            raise ValueError("x.K does not fit h")
        else:
            xp = (_arg("x_values", x_values, shape, None, gpu), _arg("x codes", x.codes, (T, Kp), torch.uint8, gpu),
                  _arg("x scales", x.scales, (T, Kp // 32), torch.uint8, gpu))
    else:
        xp = (_arg("x", x, shape, None, gpu),)
    if dropout is not None:
        st = lib().lx_block_norm_dropout(ctypes.byref(s), ctypes.byref(dropout), T, hp, yp, op, *xp, _current_raw_stream(gpu))
    else:
        fn = lib().lx_block_norm_mx8 if x_dtype is Mx8 else lib().lx_block_norm
        st = fn(ctypes.byref(s), T, hp, yp, y_rows, k, _arg("slot_row", slot_row, (T, k), torch.int32, gpu),
                _arg("slot_weights", slot_weights, (T, k), torch.float32, gpu), op, *xp, _current_raw_stream(gpu))
    if st:
        _check(st)
    return (h if y is None else h_out), x


def block_norm_mx8(h: torch.Tensor, y: Optional[torch.Tensor] = None, *, w_pre: torch.Tensor,
                   w_post: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                   gate: Optional[torch.Tensor] = None, slot_row: Optional[torch.Tensor] = None,
                   slot_weights: Optional[torch.Tensor] = None, residual_scale: float = 1.0, eps: float = 1e-6,
                   h_out: Optional[torch.Tensor] = None, x: Optional["Mx8"] = None,
                   x_values: Optional[torch.Tensor] = None, stream=None):
    """:func:`block_norm` with x in 8 bits (lx_block_norm_mx8) -> (h_out, x): what
    :func:`mx8_gemm` reads. ``x_values`` [T][d] (fp32 or bf16), if given, gets x as
    :func:`block_norm` writes it (for a router). In training its gradients are those
    of :func:`block_norm_backward`, from the gradient of the values that x stands for."""
    if h.dim() != 2:
        raise ValueError("h must be [T][d]")
    if w_pre is None:
        raise ValueError("w_pre must be given")
    gpu = _gpu("h", h)
    if stream is not None or gpu != _current_device():
        return _there(block_norm_mx8, gpu, stream, locals())
    return _block_norm(h, y, w_pre, w_post, scale, gate, slot_row, slot_weights, residual_scale, eps, h_out, x, Mx8, None, gpu, x_values)


def _dropout(p: float, rng: torch.Tensor, y, gpu) -> LxDropout:
    if not 0 <= p < 1 - 2 ** -17:
        raise ValueError("p must be in [0, 1 - 2^-17)")
    if y is None:
        raise ValueError("y must be given")
    return LxDropout(p, _arg("rng", rng, (2,), torch.int64, gpu))


def block_norm_dropout(h: torch.Tensor, y: torch.Tensor, p: float, rng: torch.Tensor, *, w_pre: Optional[torch.Tensor] = None,
                       w_post: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                       gate: Optional[torch.Tensor] = None, residual_scale: float = 1.0, eps: float = 1e-6,
                       h_out: Optional[torch.Tensor] = None, x: Optional[torch.Tensor] = None,
                       x_dtype: torch.dtype = torch.bfloat16, stream=None):
    """:func:`block_norm` without slots, the (normalised) block's output dropped out with
    probability p before gate and scale (lx_block_norm_dropout). rng: int64 [2] on the
    GPU, the generator's seed and offset, read when the kernel runs. Every layer, step
    and rank takes an offset or a seed of its own (``rng[1] += 1`` between the replays of
    a captured graph draws anew); the backward takes the same values."""
    if h.dim() != 2:
        raise ValueError("h must be [T][d]")
    gpu = _gpu("h", h)
    if stream is not None or gpu != _current_device():
        return _there(block_norm_dropout, gpu, stream, locals())
    return _block_norm(h, y, w_pre, w_post, scale, gate, None, None, residual_scale, eps, h_out, x, x_dtype,
                       _dropout(p, rng, y, gpu), gpu)


class BlockNormGrads(NamedTuple):
    dh: torch.Tensor
    dy: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dw_pre: Optional[torch.Tensor]
    dw_post: Optional[torch.Tensor]
    dscale: Optional[torch.Tensor]


def block_norm_backward(h_out: torch.Tensor, y: Optional[torch.Tensor], dx: Optional[torch.Tensor],
                        dh_out: Optional[torch.Tensor] = None, *, w_pre: Optional[torch.Tensor] = None,
                        w_post: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                        gate: Optional[torch.Tensor] = None, residual_scale: float = 1.0, eps: float = 1e-6,
                        dh: Optional[torch.Tensor] = None, dy: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None) -> BlockNormGrads:
    """Gradients of :func:`block_norm` without slots (lx_block_norm_backward),
    from h_out as it was stored (without a block: the stream h), y, the gradient
    dx of x and dh_out of h_out (None: zero). The gradients of gate and weights
    are fp32."""
    if h_out.dim() != 2:
        raise ValueError("h_out must be [T][d]")
    gpu = _gpu("h_out", h_out)
    if stream is not None or gpu != _current_device():
        return _there(block_norm_backward, gpu, stream, locals())
    return _block_norm_backward(h_out, y, dx, dh_out, w_pre, w_post, scale, gate, residual_scale, eps, dh, dy, workspace, None, gpu)


def _block_norm_backward(h_out, y, dx, dh_out, w_pre, w_post, scale, gate, residual_scale, eps, dh, dy, workspace, dropout, gpu):
    T, d = shape = h_out.shape
    if (dx is None) != (w_pre is None):
        raise ValueError("dx goes with w_pre")
    if y is None and (dy is not None or any(v is not None for v in (w_post, scale, gate))):
        raise ValueError("dy, w_post, scale and gate go with y")
    s = _norm_layer(h_out, y, LX_BF16 if dx is None else _dtype("dx", dx), w_pre, w_post, scale, gate, residual_scale,
                    eps, T, d, gpu)
    if dh is None:
        dh = h_out.new_empty(shape, dtype=h_out.dtype)
    if dy is None and y is not None:
        dy = h_out.new_empty(shape, dtype=y.dtype)
    dgate = None if gate is None else h_out.new_empty((T,), dtype=torch.float32)
    given = [v is not None for v in (w_pre, w_post, scale)]
    rows = iter(h_out.new_empty((sum(given), d), dtype=torch.float32).unbind(0) if any(given) else ())
    dw_pre, dw_post, dscale = (next(rows) if g else None for g in given)
    L = lib()
    keep, ws, n = _workspace(workspace, L.lx_block_norm_backward_workspace_bytes(T, d), h_out)
    fn, s = (L.lx_block_norm_backward, (ctypes.byref(s),)) if dropout is None else (
        L.lx_block_norm_dropout_backward, (ctypes.byref(s), ctypes.byref(dropout)))
    st = fn(
        *s, T, _arg("h_out", h_out, shape, None, gpu), _arg("y", y, shape, None, gpu),
        _arg("dx", dx, shape, None, gpu), _arg("dh_out", dh_out, shape, h_out.dtype, gpu),
        _arg("dh", dh, shape, h_out.dtype, gpu), _arg("dy", dy, shape, None if y is None else y.dtype, gpu),
        _ptr(dgate), _ptr(dw_pre), _ptr(dw_post), _ptr(dscale), ws, n, _current_raw_stream(gpu))
    if st:
        _check(st)
    return BlockNormGrads(dh, dy, dgate, dw_pre, dw_post, dscale)


def block_norm_dropout_backward(h_out: torch.Tensor, y: torch.Tensor, dx: Optional[torch.Tensor],
                                dh_out: Optional[torch.Tensor], p: float, rng: torch.Tensor, *,
                                w_pre: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
                                scale: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                                residual_scale: float = 1.0, eps: float = 1e-6, dh: Optional[torch.Tensor] = None,
                                dy: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                stream=None) -> BlockNormGrads:
    """Gradients of :func:`block_norm_dropout` (lx_block_norm_dropout_backward), with the
    p and the values of rng that it took; the other arguments as in
    :func:`block_norm_backward`."""
    if h_out.dim() != 2:
        raise ValueError("h_out must be [T][d]")
    gpu = _gpu("h_out", h_out)
    if stream is not None or gpu != _current_device():
        return _there(block_norm_dropout_backward, gpu, stream, locals())
    return _block_norm_backward(h_out, y, dx, dh_out, w_pre, w_post, scale, gate, residual_scale, eps, dh, dy, workspace,
                                _dropout(p, rng, y, gpu), gpu)


# ------------------------------------------------------------ balance loss
def route_topk_logits(x: torch.Tensor, w_r: torch.Tensor, k: int, *, workspace: Optional[torch.Tensor] = None,
                      stream=None):
    """The router with its logits (lx_route_topk_logits): bf16 x [T][d], w_r [E][d]
    -> (int32 ids [T][k], fp32 weights [T][k], fp32 logits [T][E])."""
    if x.dim() != 2 or w_r.dim() != 2:
        raise ValueError("x must be [T][d] and w_r [E][d]")
    gpu = _gpu("x", x)
    if stream is not None or gpu != _current_device():
        return _there(route_topk_logits, gpu, stream, locals())
    T, d = x.shape
    E = w_r.shape[0]
    ids, weights = x.new_empty((T, k), dtype=torch.int32), x.new_empty((T, k), dtype=torch.float32)
    logits = x.new_empty((T, E), dtype=torch.float32)
    L = lib()
    keep, ws, n = _workspace(workspace, L.lx_route_workspace_bytes(T, d, E), x)
    st = L.lx_route_topk_logits(_arg("x", x, (T, d), torch.bfloat16, gpu), _arg("w_r", w_r, (E, d), torch.bfloat16, gpu),
                                LX_BF16, T, d, E, k, ids.data_ptr(), weights.data_ptr(), logits.data_ptr(), ws, n,
                                _current_raw_stream(gpu))
    if st:
        _check(st)
    return ids, weights, logits


class BalanceLoss(NamedTuple):
    loss: torch.Tensor      # [1] fp32
    counts: torch.Tensor    # [E] int32: slots of unmasked tokens on each expert
    prob: torch.Tensor      # [E] fp32: mean router probability
    n_tokens: torch.Tensor  # [1] int32: unmasked tokens


def _mask_arg(mask, T, gpu):
    if mask is not None and mask.dtype == torch.bool:
        mask = mask.view(torch.uint8)
    return _arg("mask", mask, (T,), torch.uint8, gpu)


def balance_loss(logits: torch.Tensor, topk_ids: torch.Tensor, *, mask: Optional[torch.Tensor] = None,
                 coef: float = 1.0, workspace: Optional[torch.Tensor] = None, stream=None) -> BalanceLoss:
    """The balance loss of router logits [T][E] (fp32 or bf16) and the chosen
    experts topk_ids [T][k] (lx_balance_loss), over the tokens whose mask (uint8
    or bool [T], None: all) is set."""
    if logits.dim() != 2 or topk_ids.dim() != 2:
        raise ValueError("logits must be [T][E] and topk_ids [T][k]")
    gpu = _gpu("logits", logits)
    if stream is not None or gpu != _current_device():
        return _there(balance_loss, gpu, stream, locals())
    T, E = logits.shape
    k = topk_ids.shape[1]
    r = BalanceLoss(logits.new_empty((1,), dtype=torch.float32), logits.new_empty((E,), dtype=torch.int32),
                    logits.new_empty((E,), dtype=torch.float32), logits.new_empty((1,), dtype=torch.int32))
    L = lib()
    keep, ws, n = _workspace(workspace, L.lx_balance_loss_workspace_bytes(T, E), logits)
    st = L.lx_balance_loss(_arg("logits", logits, (T, E), None, gpu), _dtype("logits", logits), T, E,
                           _arg("topk_ids", topk_ids, (T, k), torch.int32, gpu), k, _mask_arg(mask, T, gpu), coef,
                           r.loss.data_ptr(), r.counts.data_ptr(), r.prob.data_ptr(), r.n_tokens.data_ptr(), ws, n,
                           _current_raw_stream(gpu))
    if st:
        _check(st)
    return r


def balance_loss_backward(logits: torch.Tensor, counts: torch.Tensor, n_tokens: torch.Tensor, k: int, *,
                          mask: Optional[torch.Tensor] = None, coef: float = 1.0,
                          dloss: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                          stream=None) -> torch.Tensor:
    """The gradient of the logits (lx_balance_loss_backward), from counts and
    n_tokens as :func:`balance_loss` returned them or summed over micro-batches
    or ranks; dloss: fp32 scalar tensor (None: 1)."""
    if logits.dim() != 2:
        raise ValueError("logits must be [T][E]")
    gpu = _gpu("logits", logits)
    if stream is not None or gpu != _current_device():
        return _there(balance_loss_backward, gpu, stream, locals())
    T, E = shape = logits.shape
    if dlogits is None:
        dlogits = logits.new_empty(shape, dtype=logits.dtype)
    if dloss is not None and dloss.dim() != 1:
        dloss = dloss.view(1)
    st = lib().lx_balance_loss_backward(
        _arg("logits", logits, shape, None, gpu), _dtype("logits", logits), T, E, k, _mask_arg(mask, T, gpu),
        _arg("counts", counts, (E,), torch.int32, gpu), _arg("n_tokens", n_tokens, (1,), torch.int32, gpu), coef,
        _arg("dloss", dloss, (1,), torch.float32, gpu), _arg("dlogits", dlogits, shape, logits.dtype, gpu),
        _current_raw_stream(gpu))
    if st:
        _check(st)
    return dlogits


# ------------------------------------------------------------ 4-bit values
def mx4_padded(K: int) -> int:
    """Values of a row of K after its padding (LX_MX4_KP)."""
    return -(-K // 128) * 128


class Mx4(NamedTuple):
    """4-bit values: codes uint8 [..., Kp / 2], scales uint8 [..., Kp / 32], and
    the K values of a row."""
    codes: torch.Tensor
    scales: torch.Tensor
    K: int


def mx4_quantize(x: torch.Tensor, *, act: int = MX4_NONE, out: Optional[Mx4] = None, stream=None) -> Mx4:
    """x [..., K] fp32 or bf16 -> 4-bit values (lx_mx4_quantize). With
    ``act=MX4_SWIGLU`` x is [..., 2K], the gate and up projections of a SwiGLU
    expert, and silu(gate) * up is rounded."""
    gpu = _gpu("x", x)
    if stream is not None or gpu != _current_device():
        return _there(mx4_quantize, gpu, stream, locals())
    if x.dim() < 1 or not x.is_contiguous():
        raise ValueError("x must be contiguous with at least one dimension")
    lead, K = x.shape[:-1], x.shape[-1]
    if act == MX4_SWIGLU:
        if K % 2:
            raise ValueError("rows of gate and up projections have an even length")
        K //= 2
    rows = lead.numel()
    Kp = mx4_padded(K)
    cs, ss = (*lead, Kp // 2), (*lead, Kp // 32)
    if out is None:
        out = Mx4(x.new_empty(cs, dtype=torch.uint8), x.new_empty(ss, dtype=torch.uint8), K)
    elif out.K != K:
        raise ValueError("out.K does not fit x")
    st = lib().lx_mx4_quantize(x.data_ptr(), _dtype("x", x), rows, K, act, _arg("codes", out.codes, cs, torch.uint8, gpu),
                               _arg("scales", out.scales, ss, torch.uint8, gpu), _current_raw_stream(gpu))
    if st:
        _check(st)
    return out


def mx4_dequantize(q: Mx4, dtype: torch.dtype = torch.bfloat16, *, out: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """The values [..., K] of 4-bit codes (lx_mx4_dequantize), exact in both types."""
    gpu = _gpu("codes", q.codes)
    if stream is not None or gpu != _current_device():
        return _there(mx4_dequantize, gpu, stream, locals())
    lead, K = q.codes.shape[:-1], q.K
    Kp = mx4_padded(K)
    shape = (*lead, K)
    if out is None:
        out = q.codes.new_empty(shape, dtype=dtype)
    st = lib().lx_mx4_dequantize(_arg("codes", q.codes, (*lead, Kp // 2), torch.uint8, gpu),
                                 _arg("scales", q.scales, (*lead, Kp // 32), torch.uint8, gpu), lead.numel(), K,
                                 _arg("out", out, shape, None, gpu), _dtype("out", out), _current_raw_stream(gpu))
    if st:
        _check(st)
    return out


def mx4_gemm(a: Mx4, b: Mx4, *, offsets: Optional[torch.Tensor] = None, row_map: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
             workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[m] = A[row(m)] B[g]^T for the rows m of group g (lx_mx4_gemm): a
    [rows][K]; b [G][N][K] (or [N][K]: one group); offsets int32 [G + 1] (None: one
    group of all rows); row_map int32 [M] (None: row m of a). Rows past
    offsets[G] are left as they are."""
    gpu = _gpu("a", a.codes)
    if stream is not None or gpu != _current_device():
        return _there(mx4_gemm, gpu, stream, locals())
    ac, bc, K = a.codes, b.codes, a.K
    if ac.dim() != 2 or bc.dim() not in (2, 3):
        raise ValueError("a must be [rows][K] and b [G][N][K] or [N][K]")
    if K != b.K:
        raise ValueError(f"a has {K} values in a row and b {b.K}")
    Kp = mx4_padded(K)
    rows = ac.shape[0]
    *lead, _ = bc.shape
    G, N = lead if len(lead) == 2 else (1, lead[0])
    M = rows if row_map is None else row_map.shape[0]
    if out is None:
        out = ac.new_empty((M, N), dtype=out_dtype)
    L = lib()
    keep, ws, n = _workspace(workspace, L.lx_mx4_gemm_workspace_bytes(M, N, K, G), ac)
    st = L.lx_mx4_gemm(_arg("a codes", ac, (rows, Kp // 2), torch.uint8, gpu),
                       _arg("a scales", a.scales, (rows, Kp // 32), torch.uint8, gpu), rows,
                       _arg("row_map", row_map, (M,), torch.int32, gpu),
                       _arg("b codes", bc, (*lead, Kp // 2), torch.uint8, gpu),
                       _arg("b scales", b.scales, (*lead, Kp // 32), torch.uint8, gpu),
                       _arg("offsets", offsets, (G + 1,), torch.int32, gpu), G, M, N, K,
                       _arg("out", out, (M, N), None, gpu), _dtype("out", out), ws, n, _current_raw_stream(gpu))
    if st:
        _check(st)
    return out


# ------------------------------------------------------------ 8-bit values
def mx8_quantize(x: torch.Tensor, *, act: int = MX4_NONE, out: Optional[Mx8] = None, stream=None) -> Mx8:
    """x [..., K] fp32 or bf16 -> 8-bit values (lx_mx8_quantize). With
    ``act=MX4_SWIGLU`` x is [..., 2K], the gate and up projections of a SwiGLU
    expert, and silu(gate) * up is rounded."""
    gpu = _gpu("x", x)
    if stream is not None or gpu != _current_device():
        return _there(mx8_quantize, gpu, stream, locals())
    if x.dim() < 1 or not x.is_contiguous():
        raise ValueError("x must be contiguous with at least one dimension")
    lead, K = x.shape[:-1], x.shape[-1]
    if act == MX4_SWIGLU:
        if K % 2:
            raise ValueError("rows of gate and up projections have an even length")
        K //= 2
    Kp = mx4_padded(K)
    cs, ss = (*lead, Kp), (*lead, Kp // 32)
    if out is None:
        codes, scales = x.new_empty(cs, dtype=torch.uint8), x.new_empty(ss, dtype=torch.uint8)
        out, cp, sp = Mx8(codes, scales, K), codes.data_ptr() or _EMPTY, scales.data_ptr() or _EMPTY
    elif out.K != K:
        raise ValueError("out.K does not fit x")
    else:
        cp, sp = _arg("codes", out.codes, cs, torch.uint8, gpu), _arg("scales", out.scales, ss, torch.uint8, gpu)
    st = lib().lx_mx8_quantize(x.data_ptr(), _dtype("x", x), lead.numel(), K, act, cp, sp, _current_raw_stream(gpu))
    if st:
        _check(st)
    return out


def mx8_dequantize(q: Mx8, dtype: torch.dtype = torch.bfloat16, *, out: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """The values [..., K] of 8-bit codes (lx_mx8_dequantize)."""
    gpu = _gpu("codes", q.codes)
    if stream is not None or gpu != _current_device():
        return _there(mx8_dequantize, gpu, stream, locals())
    lead, K = q.codes.shape[:-1], q.K
    Kp = mx4_padded(K)
    shape = (*lead, K)
    if out is None:
        out = q.codes.new_empty(shape, dtype=dtype)
    st = lib().lx_mx8_dequantize(_arg("codes", q.codes, (*lead, Kp), torch.uint8, gpu),
                                 _arg("scales", q.scales, (*lead, Kp // 32), torch.uint8, gpu), lead.numel(), K,
                                 _arg("out", out, shape, None, gpu), _dtype("out", out), _current_raw_stream(gpu))
    if st:
        _check(st)
    return out


def mx8_gemm(a: Mx8, b: Mx4, *, offsets: Optional[torch.Tensor] = None, row_map: Optional[torch.Tensor] = None,
             bias: Optional[torch.Tensor] = None, act: int = ACT_NONE, residual: Optional[torch.Tensor] = None,
             out=None, out_dtype=torch.float32, workspace: Optional[torch.Tensor] = None, stream=None):
    """out[m] = act(A[row(m)] B[g]^T + bias[g]) + residual[m] for the rows m of group g
    (lx_mx8_gemm): a [rows][K] in 8 bits; b [G][N][K] (or [N][K]: one group) in 4; bias
    [G][N] ([N] for one group) and residual [M][columns] fp32 or bf16; ``ACT_SWIGLU``
    takes N / 2 gate and N / 2 up rows and gives N / 2 columns. offsets, row_map and
    rows past offsets[G] as in :func:`mx4_gemm`. The result is a tensor of
    ``out_dtype``, or with ``out_dtype="mx8"`` (or an :class:`Mx8` given as out) 8-bit
    values."""
    gpu = _gpu("a", a.codes)
    if stream is not None or gpu != _current_device():
        return _there(mx8_gemm, gpu, stream, locals())
    ac, bc, K = a.codes, b.codes, a.K
    if ac.dim() != 2 or bc.dim() not in (2, 3):
        raise ValueError("a must be [rows][K] and b [G][N][K] or [N][K]")
    if K != b.K:
        raise ValueError(f"a has {K} values in a row and b {b.K}")
    Kp = mx4_padded(K)
    rows = ac.shape[0]
    *lead, _ = bc.shape
    G, N = lead if len(lead) == 2 else (1, lead[0])
    M = rows if row_map is None else row_map.shape[0]
    if act == ACT_SWIGLU and N % 2:
        raise ValueError("SwiGLU needs an even number of weight rows")
    cols = N // 2 if act == ACT_SWIGLU else N
    mx8 = isinstance(out, Mx8) or (out is None and out_dtype == "mx8")
    if mx8:
        cp = mx4_padded(cols)
        if out is None:
            out = Mx8(ac.new_empty((M, cp), dtype=torch.uint8), ac.new_empty((M, cp // 32), dtype=torch.uint8), cols)
        elif out.K != cols:
            raise ValueError(f"out has {out.K} values in a row, the result {cols}")
        to = _arg("out codes", out.codes, (M, cp), torch.uint8, gpu), 0, _arg("out scales", out.scales, (M, cp // 32), torch.uint8, gpu)
    else:
        if out is None:
            out = ac.new_empty((M, cols), dtype=out_dtype)
        to = _arg("out", out, (M, cols), None, gpu), _dtype("out", out), None
    if bias is not None and bias.dim() == 1 and G == 1:
        bias = bias.view(1, -1)
    e = LxEpilogue(act, 0 if bias is None else _dtype("bias", bias), 0 if residual is None else _dtype("residual", residual),
                   _arg("bias", bias, (G, N), None, gpu), _arg("residual", residual, (M, cols), None, gpu))
    # (lx_mx8_gemm_workspace_bytes is 0 for all sizes: the question takes half a microsecond)
    keep, ws, n = (None, None, 0) if workspace is None else _workspace(workspace, 0, ac)
    st = lib().lx_mx8_gemm(_arg("a codes", ac, (rows, Kp), torch.uint8, gpu),
                       _arg("a scales", a.scales, (rows, Kp // 32), torch.uint8, gpu), rows,
                       _arg("row_map", row_map, (M,), torch.int32, gpu),
                       _arg("b codes", bc, (*lead, Kp // 2), torch.uint8, gpu),
                       _arg("b scales", b.scales, (*lead, Kp // 32), torch.uint8, gpu),
                       _arg("offsets", offsets, (G + 1,), torch.int32, gpu), G, M, N, K, ctypes.byref(e), *to, ws, n,
                       _current_raw_stream(gpu))
    if st:
        _check(st)
    return out


# ------------------------------------------------------------ a MoE block in 4 bits
class Mx4Experts(NamedTuple):
    """The E experts of a layer in 4 bits: the gate and up projections as one
    weight [E][2f][d] (gate rows first), the down projection [E][d][f]."""
    gate_up: Mx4
    down: Mx4


def mx4_experts(w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, stream=None) -> Mx4Experts:
    """Experts w_gate, w_up [E][f][d], w_down [E][d][f] rounded to 4 bits, once
    when a model is loaded; all of it in ``stream``, the joining of the projections
    too."""
    gpu = _gpu("w_gate", w_gate)
    if stream is not None or gpu != _current_device():
        return _there(mx4_experts, gpu, stream, locals())
    return Mx4Experts(mx4_quantize(torch.cat([w_gate, w_up], dim=1)), mx4_quantize(w_down.contiguous()))


def mx4_moe_few(x: torch.Tensor, topk_ids: torch.Tensor, topk_weights: torch.Tensor, experts: Mx4Experts, *,
                out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
                workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The experts' layer for up to ``MOE_FEW_MAX_T`` tokens in two launches
    (lx_mx4_moe_few): x [T][d] (fp32 or bf16, not rounded), topk_ids and topk_weights
    [T][k] as the router gives them -> the weighted sum of the experts' outputs
    [T][d]."""
    if x.dim() != 2 or topk_ids.dim() != 2:
        raise ValueError("x must be [T][d] and topk_ids [T][k]")
    gpu = _gpu("x", x)
    if stream is not None or gpu != _current_device():
        return _there(mx4_moe_few, gpu, stream, locals())
    T, d = x.shape
    k = topk_ids.shape[1]
    gu, down = experts
    E, f = down.codes.shape[0], down.K
    if gu.K != d:
        raise ValueError(f"x has {d} values in a row, the experts {gu.K}")
    dp, fp = mx4_padded(d), mx4_padded(f)
    if out is None:
        out = x.new_empty((T, d), dtype=out_dtype)
    L = lib()
    keep, ws, n = _workspace(workspace, L.lx_mx4_moe_few_workspace_bytes(T, k, E, d, f), x)
    u8 = torch.uint8
    st = L.lx_mx4_moe_few(_arg("x", x, (T, d), None, gpu), _dtype("x", x), T, d, _arg("topk_ids", topk_ids, (T, k), torch.int32, gpu),
                          _arg("topk_weights", topk_weights, (T, k), torch.float32, gpu), k, E, f,
                          _arg("gate_up codes", gu.codes, (E, 2 * f, dp // 2), u8, gpu),
                          _arg("gate_up scales", gu.scales, (E, 2 * f, dp // 32), u8, gpu),
                          _arg("down codes", down.codes, (E, d, fp // 2), u8, gpu),
                          _arg("down scales", down.scales, (E, d, fp // 32), u8, gpu),
                          _arg("out", out, (T, d), None, gpu), _dtype("out", out), ws, n, _current_raw_stream(gpu))
    if st:
        _check(st)
    return out


class Mx4BlockOut(NamedTuple):
    h_out: torch.Tensor              # [T][d] the stream after the block
    x_next: Optional[torch.Tensor]   # [T][d] the next block's input (w_next given)
    x: torch.Tensor                  # [T][d] this block's input
    topk_ids: torch.Tensor
    topk_weights: torch.Tensor
    logits: Optional[torch.Tensor]   # [T][E] fp32, as the router chose by (balance_coef given)
    balance: Optional[BalanceLoss]


def mx4_moe_block(h: torch.Tensor, w_pre: torch.Tensor, w_r: torch.Tensor, experts: Mx4Experts, k: int, *,
                  w_post: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                  gate: Optional[torch.Tensor] = None, residual_scale: float = 1.0, eps: float = 1e-6,
                  w_next: Optional[torch.Tensor] = None, balance_coef: Optional[float] = None,
                  mask: Optional[torch.Tensor] = None, activations: str = "mx4") -> Mx4BlockOut:
    """One MoE block with its experts in 4 bits, on the current stream: norm,
    router (lx_route_topk), bucketing (lx_bucket), the experts' products per
    group of rows with SwiGLU and rounding between them, then the experts' sum,
    norm, gate, residual and the next block's norm in one kernel. h [T][d], w_r
    [E][d] bf16 (d a multiple of 64, E of 4); the other arguments as in
    :func:`block_norm`. With ``balance_coef`` the router's logits and balance
    loss too (tokens whose ``mask`` is 0 left out). ``activations`` says how the
    products see theirs: "mx4" in 4 bits, "mx8" in 8 (the norm rounds them, SwiGLU and
    its rounding are the first product's epilogue), "full" not rounded (at most
    ``MOE_FEW_MAX_T`` tokens, :func:`mx4_moe_few`)."""
    if activations not in ("mx4", "mx8", "full"):
        raise ValueError('activations must be "mx4", "mx8" or "full"')
    if activations == "full" and h.shape[0] > MOE_FEW_MAX_T:
        raise ValueError(f'activations="full" takes at most {MOE_FEW_MAX_T} tokens')
    gpu = _gpu("h", h)
    if gpu != _current_device():
        return _there(mx4_moe_block, gpu, None, locals())
    T, d = h.shape
    E = experts.gate_up.codes.shape[0]
    f = experts.down.K
    if w_r.shape != (E, d) or experts.down.codes.shape[:2] != (E, d) or experts.gate_up.codes.shape[1] != 2 * f:
        raise ValueError("w_r must be [E][d], the experts [E][2f][d] and [E][d][f] for h [T][d]")
    if w_r.get_device() != gpu:
        raise ValueError(f"w_r is on {w_r.device}, h on {h.device}")
    if activations == "mx8":
        x = h.new_empty((T, d), dtype=torch.bfloat16)
        _, x8 = block_norm_mx8(h, w_pre=w_pre, eps=eps, x_values=x)
    else:
        _, x = block_norm(h, w_pre=w_pre, eps=eps)
    logits = balance = None
    if not T:  # nothing to route
        ids, weights = h.new_empty((0, k), dtype=torch.int32), h.new_empty((0, k), dtype=torch.float32)
        if balance_coef is not None:
            logits = h.new_empty((0, E), dtype=torch.float32)
    elif balance_coef is not None:
        ids, weights, logits = route_topk_logits(x, w_r, k)
    else:
        ids, weights = lx.route_topk(x, w_r, k)
    if balance_coef is not None:
        balance = balance_loss(logits, ids, mask=mask, coef=balance_coef)
    if not T:
        h_out, x_next = block_norm(h, h.new_empty((0, d), dtype=torch.float32), w_pre=w_next, w_post=w_post, scale=scale,
                                   gate=gate, residual_scale=residual_scale, eps=eps)
        return Mx4BlockOut(h_out, x_next, x, ids, weights, logits, balance)
    if activations == "full":
        y = mx4_moe_few(x, ids, weights, experts)
        h_out, x_next = block_norm(h, y, w_pre=w_next, w_post=w_post, scale=scale, gate=gate, residual_scale=residual_scale, eps=eps)
        return Mx4BlockOut(h_out, x_next, x, ids, weights, logits, balance)
    # rows of the experts: a tree without levels, whose weights bucketing does not read.
    # It takes a forward's workspace, so the tree is given small sizes: with the experts'
    # own that is 2.9 GiB for 8192 tokens on 8 experts of 14336, with 64 (the smallest for
    # which a decode batch has one table of tiles to build, not two) 16 MiB
    tree = lx.LxTreeLayer()
    tree.E, tree.d, tree.f, tree.dtype, tree.n_anchors = E, 64, 64, LX_BF16, E
    tree.anchor_gate = tree.anchor_up = tree.anchor_down = experts.gate_up.codes.data_ptr()
    L = lib()
    n = L.lx_moe_tree_workspace_bytes(ctypes.byref(tree), T, k)
    if not n:
        raise lx.LorexError(lx.LX_ERR_UNSUPPORTED, L.lx_last_error().decode())
    ws = h.new_empty(n, dtype=torch.uint8)
    row_token = h.new_empty(T * min(k, E), dtype=torch.int32)
    offsets = h.new_empty(E + 1, dtype=torch.int32)
    slot_row = h.new_empty((T, k), dtype=torch.int32)
    _check(L.lx_bucket(ctypes.byref(tree), T, k, ids.data_ptr(), 0, row_token.data_ptr(), offsets.data_ptr(),
                       slot_row.data_ptr(), ws.data_ptr(), n, _current_raw_stream(gpu)))
    if activations == "mx8":
        hidden = mx8_gemm(x8, experts.gate_up, offsets=offsets, row_map=row_token, act=ACT_SWIGLU, out_dtype="mx8")
        y = mx8_gemm(hidden, experts.down, offsets=offsets, out_dtype=torch.float32)
    else:
        # (gate and up projections are kept in bf16 on their way into SwiGLU: half of fp32's
        # bytes of the block's widest rows, and their 2^-9 is small next to what follows,
        # a rounding to 4 bits, whose steps are a quarter of a value and more)
        gate_up = mx4_gemm(mx4_quantize(x), experts.gate_up, offsets=offsets, row_map=row_token, out_dtype=torch.bfloat16)
        y = mx4_gemm(mx4_quantize(gate_up, act=MX4_SWIGLU), experts.down, offsets=offsets, out_dtype=torch.float32)
    h_out, x_next = block_norm(h, y, w_pre=w_next, w_post=w_post, scale=scale, gate=gate, slot_row=slot_row,
                               slot_weights=weights, residual_scale=residual_scale, eps=eps)
    return Mx4BlockOut(h_out, x_next, x, ids, weights, logits, balance)
