"""The operators around the expert layer and the experts in 4 bits
(include/lorex_block.h), bound like ``lorex``: argument marshalling only.

* :func:`block_norm`, :func:`block_norm_backward`: the norms before and after a
  block with its gate and residual scale;
* :func:`balance_loss`, :func:`balance_loss_backward`: the router's balance
  loss, the tokens per expert, the gradient of the logits;
* :func:`mx4_quantize`, :func:`mx4_dequantize`, :func:`mx4_gemm`: microscaled
  4-bit values, and products of them per group of rows;
* :class:`Mx4Experts`, :func:`mx4_moe_block`: a MoE block whose experts are held
  in 4 bits, built from these and the library's router and bucketing.

Tensors are contiguous and on one GPU. Calls are asynchronous on ``stream`` (a
``torch.cuda.Stream``; default: the current one). Outputs can be given; those
that are not are allocated, as are workspaces.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import lorex as lx
from .lorex import LX_BF16, LX_F32, LX_ERR_UNSUPPORTED, LorexError, _check

MX4_NONE, MX4_SWIGLU = 0, 1
NORM_MAX_D = 32768

_c_void, _c_i32, _c_i64, _c_f32, _c_size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


class LxNormLayer(ctypes.Structure):
    _fields_ = [("d", _c_i32), ("h_dtype", _c_i32), ("y_dtype", _c_i32), ("x_dtype", _c_i32), ("w_dtype", _c_i32),
                ("residual_scale", _c_f32), ("eps", _c_f32), ("w_pre", _c_void), ("w_post", _c_void),
                ("scale", _c_void), ("gate", _c_void)]


EXPORTS = {
    "lx_block_norm": (_c_i32, [_c_void, _c_i32, _c_void, _c_void, _c_i32, _c_i32] + [_c_void] * 5),
    "lx_block_norm_backward_workspace_bytes": (_c_size, [_c_i32, _c_i32]),
    "lx_block_norm_backward": (_c_i32, [_c_void, _c_i32] + [_c_void] * 11 + [_c_size, _c_void]),
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


def _arg(name: str, t: Optional[torch.Tensor], shape: tuple, dtype, device) -> Optional[int]:
    """Address of an argument after its checks (None stays None)."""
    if t is None:
        return None
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    return t.data_ptr() or _EMPTY


def _need_gpu(name: str, t: torch.Tensor):
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU")


class _On:
    """The stream of a call and the tensors the call allocates: those stay
    reserved until that stream is done with them."""

    def __init__(self, stream, device):
        cur = torch.cuda.current_stream(device)
        self.other = stream if stream is not None and stream != cur else None
        self.handle = (cur if stream is None else stream).cuda_stream
        self.device = device

    def empty(self, shape, dtype):
        t = torch.empty(shape, dtype=dtype, device=self.device)
        if self.other is not None:
            t.record_stream(self.other)
        return t

    def workspace(self, given: Optional[torch.Tensor], need: int):
        """(address, bytes) of a workspace; the tensor is kept by the caller's frame."""
        if given is None and need:
            given = self.empty(need, torch.uint8)
        return given


# ------------------------------------------------------------ block norms
def _norm_layer(h, y, x_dtype, w_pre, w_post, scale, gate, residual_scale, eps, T, d, dev) -> LxNormLayer:
    ws = [w for w in (w_pre, w_post, scale) if w is not None]
    if any(w.dtype != ws[0].dtype for w in ws):
        raise ValueError("w_pre, w_post and scale must have one dtype")
    s = LxNormLayer()
    s.d = d
    s.h_dtype = _dtype("h", h)
    s.y_dtype = s.h_dtype if y is None else _dtype("y", y)
    s.x_dtype = x_dtype
    s.w_dtype = _dtype("weights", ws[0]) if ws else LX_F32
    s.residual_scale, s.eps = residual_scale, eps
    s.w_pre = _arg("w_pre", w_pre, (d,), None, dev)
    s.w_post = _arg("w_post", w_post, (d,), None, dev)
    s.scale = _arg("scale", scale, (d,), None, dev)
    s.gate = _arg("gate", gate, (T,), torch.float32, dev)
    return s


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
    _need_gpu("h", h)
    T, d = h.shape
    dev = h.device
    on = _On(stream, dev)
    k = y_rows = 0
    if y is not None:
        y_rows = y.shape[0]
        if slot_row is None:
            yp = _arg("y", y, (T, d), None, dev)
        else:
            if slot_row.dim() != 2:
                raise ValueError("slot_row must be [T][k]")
            k = slot_row.shape[1]
            yp = _arg("y", y, (y_rows, d), None, dev)
        if h_out is None:
            h_out = on.empty((T, d), h.dtype)
    else:
        yp = None
        if h_out is not None or slot_row is not None or slot_weights is not None or any(v is not None for v in (w_post, scale, gate)):
            raise ValueError("h_out, slots, w_post, scale and gate go with y")
    if w_pre is None:
        if x is not None:
            raise ValueError("x goes with w_pre")
    elif x is None:
        x = on.empty((T, d), x_dtype)
    s = _norm_layer(h, y, LX_BF16 if x is None else _dtype("x", x), w_pre, w_post, scale, gate, residual_scale, eps, T, d, dev)
    _check(lib().lx_block_norm(ctypes.byref(s), T, _arg("h", h, (T, d), None, dev), yp, y_rows, k,
                               _arg("slot_row", slot_row, (T, k), torch.int32, dev),
                               _arg("slot_weights", slot_weights, (T, k), torch.float32, dev),
                               _arg("h_out", h_out, (T, d), h.dtype, dev), _arg("x", x, (T, d), None, dev), on.handle))
    return (h if y is None else h_out), x


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
    _need_gpu("h_out", h_out)
    T, d = h_out.shape
    dev = h_out.device
    on = _On(stream, dev)
    if (dx is None) != (w_pre is None):
        raise ValueError("dx goes with w_pre")
    if y is None and (dy is not None or any(v is not None for v in (w_post, scale, gate))):
        raise ValueError("dy, w_post, scale and gate go with y")
    s = _norm_layer(h_out, y, LX_BF16 if dx is None else _dtype("dx", dx), w_pre, w_post, scale, gate, residual_scale,
                    eps, T, d, dev)
    if dh is None:
        dh = on.empty((T, d), h_out.dtype)
    if dy is None and y is not None:
        dy = on.empty((T, d), y.dtype)
    grad = lambda v, n: None if v is None else on.empty((n,), torch.float32)  # noqa: E731
    dgate, dw_pre, dw_post, dscale = grad(gate, T), grad(w_pre, d), grad(w_post, d), grad(scale, d)
    L = lib()
    workspace = on.workspace(workspace, L.lx_block_norm_backward_workspace_bytes(T, d))
    p = lambda v: None if v is None else v.data_ptr() or _EMPTY  # noqa: E731
    _check(L.lx_block_norm_backward(
        ctypes.byref(s), T, _arg("h_out", h_out, (T, d), None, dev), _arg("y", y, (T, d), None, dev),
        _arg("dx", dx, (T, d), None, dev), _arg("dh_out", dh_out, (T, d), h_out.dtype, dev),
        _arg("dh", dh, (T, d), h_out.dtype, dev), _arg("dy", dy, (T, d), None if y is None else y.dtype, dev),
        p(dgate), p(dw_pre), p(dw_post), p(dscale), p(workspace), 0 if workspace is None else workspace.numel(),
        on.handle))
    return BlockNormGrads(dh, dy, dgate, dw_pre, dw_post, dscale)


# ------------------------------------------------------------ balance loss
class BalanceLoss(NamedTuple):
    loss: torch.Tensor      # [1] fp32
    counts: torch.Tensor    # [E] int32: slots of unmasked tokens on each expert
    prob: torch.Tensor      # [E] fp32: mean router probability
    n_tokens: torch.Tensor  # [1] int32: unmasked tokens


def _mask_arg(mask, T, dev):
    if mask is not None and mask.dtype == torch.bool:
        mask = mask.view(torch.uint8)
    return _arg("mask", mask, (T,), torch.uint8, dev)


def balance_loss(logits: torch.Tensor, topk_ids: torch.Tensor, *, mask: Optional[torch.Tensor] = None,
                 coef: float = 1.0, workspace: Optional[torch.Tensor] = None, stream=None) -> BalanceLoss:
    """The balance loss of router logits [T][E] (fp32 or bf16) and the chosen
    experts topk_ids [T][k] (lx_balance_loss), over the tokens whose mask (uint8
    or bool [T], None: all) is set."""
    if logits.dim() != 2 or topk_ids.dim() != 2:
        raise ValueError("logits must be [T][E] and topk_ids [T][k]")
    _need_gpu("logits", logits)
    T, E = logits.shape
    k = topk_ids.shape[1]
    dev = logits.device
    on = _On(stream, dev)
    r = BalanceLoss(on.empty((1,), torch.float32), on.empty((E,), torch.int32), on.empty((E,), torch.float32),
                    on.empty((1,), torch.int32))
    L = lib()
    workspace = on.workspace(workspace, L.lx_balance_loss_workspace_bytes(T, E))
    _check(L.lx_balance_loss(_arg("logits", logits, (T, E), None, dev), _dtype("logits", logits), T, E,
                             _arg("topk_ids", topk_ids, (T, k), torch.int32, dev), k, _mask_arg(mask, T, dev), coef,
                             r.loss.data_ptr(), r.counts.data_ptr(), r.prob.data_ptr(), r.n_tokens.data_ptr(),
                             None if workspace is None else workspace.data_ptr(),
                             0 if workspace is None else workspace.numel(), on.handle))
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
    _need_gpu("logits", logits)
    T, E = logits.shape
    dev = logits.device
    on = _On(stream, dev)
    if dlogits is None:
        dlogits = on.empty((T, E), logits.dtype)
    if dloss is not None:
        dloss = dloss.view(1)
    _check(lib().lx_balance_loss_backward(
        _arg("logits", logits, (T, E), None, dev), _dtype("logits", logits), T, E, k, _mask_arg(mask, T, dev),
        _arg("counts", counts, (E,), torch.int32, dev), _arg("n_tokens", n_tokens, (1,), torch.int32, dev), coef,
        _arg("dloss", dloss, (1,), torch.float32, dev), _arg("dlogits", dlogits, (T, E), logits.dtype, dev), on.handle))
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
    _need_gpu("x", x)
    if x.dim() < 1 or not x.is_contiguous():
        raise ValueError("x must be contiguous with at least one dimension")
    lead, K = tuple(x.shape[:-1]), x.shape[-1]
    if act == MX4_SWIGLU:
        if K % 2:
            raise ValueError("rows of gate and up projections have an even length")
        K //= 2
    rows = 1
    for v in lead:
        rows *= v
    Kp = mx4_padded(K)
    on = _On(stream, x.device)
    if out is None:
        out = Mx4(on.empty(lead + (Kp // 2,), torch.uint8), on.empty(lead + (Kp // 32,), torch.uint8), K)
    elif out.K != K:
        raise ValueError("out.K does not fit x")
    _check(lib().lx_mx4_quantize(x.data_ptr(), _dtype("x", x), rows, K, act,
                                 _arg("codes", out.codes, lead + (Kp // 2,), torch.uint8, x.device),
                                 _arg("scales", out.scales, lead + (Kp // 32,), torch.uint8, x.device), on.handle))
    return out


def mx4_dequantize(q: Mx4, dtype: torch.dtype = torch.bfloat16, *, out: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """The values [..., K] of 4-bit codes (lx_mx4_dequantize), exact in both types."""
    _need_gpu("codes", q.codes)
    lead, K, dev = tuple(q.codes.shape[:-1]), q.K, q.codes.device
    Kp = mx4_padded(K)
    rows = 1
    for v in lead:
        rows *= v
    on = _On(stream, dev)
    if out is None:
        out = on.empty(lead + (K,), dtype)
    _check(lib().lx_mx4_dequantize(_arg("codes", q.codes, lead + (Kp // 2,), torch.uint8, dev),
                                   _arg("scales", q.scales, lead + (Kp // 32,), torch.uint8, dev), rows, K,
                                   _arg("out", out, lead + (K,), None, dev), _dtype("out", out), on.handle))
    return out


def mx4_gemm(a: Mx4, b: Mx4, *, offsets: Optional[torch.Tensor] = None, row_map: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
             workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[m] = A[row(m)] B[g]^T for the rows m of group g (lx_mx4_gemm): a
    [rows][K]; b [G][N][K] (or [N][K]: one group); offsets int32 [G + 1] (None: one
    group of all rows); row_map int32 [M] (None: row m of a). Rows past
    offsets[G] are left as they are."""
    _need_gpu("a", a.codes)
    if a.codes.dim() != 2 or b.codes.dim() not in (2, 3):
        raise ValueError("a must be [rows][K] and b [G][N][K] or [N][K]")
    if a.K != b.K:
        raise ValueError(f"a has {a.K} values in a row and b {b.K}")
    dev, K = a.codes.device, a.K
    Kp = mx4_padded(K)
    rows = a.codes.shape[0]
    lead = tuple(b.codes.shape[:-1])
    G, N = lead if len(lead) == 2 else (1, lead[0])
    M = rows if row_map is None else row_map.shape[0]
    on = _On(stream, dev)
    if out is None:
        out = on.empty((M, N), out_dtype)
    L = lib()
    workspace = on.workspace(workspace, L.lx_mx4_gemm_workspace_bytes(M, N, K, G))
    _check(L.lx_mx4_gemm(_arg("a codes", a.codes, (rows, Kp // 2), torch.uint8, dev),
                         _arg("a scales", a.scales, (rows, Kp // 32), torch.uint8, dev), rows,
                         _arg("row_map", row_map, (M,), torch.int32, dev),
                         _arg("b codes", b.codes, lead + (Kp // 2,), torch.uint8, dev),
                         _arg("b scales", b.scales, lead + (Kp // 32,), torch.uint8, dev),
                         _arg("offsets", offsets, (G + 1,), torch.int32, dev), G, M, N, K,
                         _arg("out", out, (M, N), None, dev), _dtype("out", out),
                         None if workspace is None else workspace.data_ptr(),
                         0 if workspace is None else workspace.numel(), on.handle))
    return out
