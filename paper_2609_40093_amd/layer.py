"""Python binding of the layer operators (include/ep_layer.h), marshalling only.

Norm, router, experts' products, adapters, dropout and the gradients run in the library's HIP kernels; outputs
and workspaces are torch tensors of the current device.  Without a tensor to write to, a call
allocates its outputs; with `stream`, allocations belong to that stream.

No call takes part in torch's autograd: outputs come detached, also of inputs that require grad,
and the ..._grad calls are what a backward pass is made of (examples/moe_layer.py, or the
backward of a torch.autograd.Function of the caller's).
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
from dataclasses import dataclass
from typing import Optional, Tuple, Union

import torch

from . import _lib
from ._lib import EP_OUT_BF16, EP_OUT_F32, EP_ROWS8_EXTRA, EP_ROWS_8BIT, EP_ROWS_BF16
from .api import _check, _current_stream, _get_device, _lib_handle, _need, _ptr

__all__ = ["Norm", "rmsnorm", "rmsnorm_grad", "rows8_empty", "rows8_values", "Routing", "route", "route_grad",
           "combine_grad", "Product", "expert_product", "ProductGrad", "expert_product_grad",
           "AdapterRows", "adapter_rows", "AdapterProduct", "adapter_product", "AdapterGrad", "adapter_product_grad",
           "dropout", "dropout_rmsnorm", "dropout_rmsnorm_grad"]

_BF16 = (torch.bfloat16,)
_F32 = (torch.float32,)
_I32 = (torch.int32,)
_I64 = (torch.int64,)
_F8 = (torch.float8_e4m3fn,)
_NO_STREAM = contextlib.nullcontext()


def _on(stream):
    """Allocations of a call on `stream` are made on it, so that their memory is not handed out
    again before that stream has used it."""
    if stream is None:
        return _NO_STREAM
    return torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream)


def _shape(t: torch.Tensor, name: str, shape):
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _optional(t: Optional[torch.Tensor], name: str, dtypes, shape):
    """Checks an argument that may be None.  One expression for a tensor that fits."""
    if t is None or (t.is_cuda and t.dtype in dtypes and t.shape == shape and t.is_contiguous()
                     and t.get_device() == _get_device()):
        return
    _need(t, name, dtypes)
    _shape(t, name, shape)


def _given(t: Optional[torch.Tensor], name: str) -> torch.Tensor:
    if t is None:
        raise ValueError(f"{name} is required")
    return t


def _output(want: Union[bool, torch.Tensor, None], name: str, dtype, shape, device) -> Optional[torch.Tensor]:
    """An output to write: the tensor given, a new one for True, none for False or None."""
    if want is True:
        return torch.empty(*shape, dtype=dtype, device=device)
    if want is False or want is None:
        return None
    _optional(want, name, (dtype,), shape)
    return want


def _workspace(n: int, device) -> Optional[torch.Tensor]:
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


@functools.lru_cache(maxsize=4096)
def _bytes(name: str, *args) -> int:
    """Workspace bytes of a call: a pure function of the sizes."""
    n = ctypes.c_size_t()
    _check(getattr(_lib_handle(), name)(*args, ctypes.byref(n)), name)
    return n.value


# ------------------------------------------------------------------------- 8-bit rows

def rows8_empty(num_rows: int, hidden: int, device="cuda") -> torch.Tensor:
    """A buffer for 8-bit rows: uint8 [num_rows, hidden + 16]."""
    return torch.empty((num_rows, hidden + EP_ROWS8_EXTRA), dtype=torch.uint8, device=device)


def rows8_values(rows8: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """Views of 8-bit rows: the e4m3 values [n, hidden] and the fp32 scales [n, 1]; a row's
    numbers are values * scale."""
    h = rows8.shape[1] - EP_ROWS8_EXTRA
    return rows8[:, :h].view(torch.float8_e4m3fn), rows8[:, h:h + 4].view(torch.float32)


# ------------------------------------------------------------------------------- norm

@dataclass
class Norm:
    total: Optional[torch.Tensor]
    out: Optional[torch.Tensor]
    rows8: Optional[torch.Tensor]


def rmsnorm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, *, residual: Optional[torch.Tensor] = None,
            eps: float = 1e-6, total: Union[bool, torch.Tensor, None] = None, out: Union[bool, torch.Tensor] = True,
            rows8: Union[bool, torch.Tensor] = False, stream=None) -> Norm:
    """ep_rmsnorm on bf16 rows [T, H]: total = x + residual (written when there is a residual,
    or on request), out = its RMS norm times weight, rows8 = the same as 8-bit rows.  Outputs
    are wanted (True), not wanted (False), or tensors to write."""
    _need(x, "x", _BF16, 2)
    T, H = x.shape
    _optional(residual, "residual", _BF16, x.shape)
    _optional(weight, "weight", _BF16, (H,))
    with _on(stream):
        got = Norm(_output(residual is not None if total is None else total, "total", torch.bfloat16, x.shape, x.device),
                   _output(out, "out", torch.bfloat16, x.shape, x.device),
                   _output(rows8, "rows8", torch.uint8, (T, H + EP_ROWS8_EXTRA), x.device))
    _check(_lib_handle().ep_rmsnorm(_ptr(x), _ptr(residual), _ptr(weight), T, H, eps, _ptr(got.total), _ptr(got.out),
                                    _ptr(got.rows8), _current_stream(stream)), "ep_rmsnorm")
    return got


def rmsnorm_grad(total: torch.Tensor, weight: Optional[torch.Tensor], d_out: torch.Tensor, *,
                 d_total: Optional[torch.Tensor] = None, eps: float = 1e-6, dx: Optional[torch.Tensor] = None,
                 d_weight: Union[bool, torch.Tensor] = True,
                 stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """ep_rmsnorm_grad: (dx bf16 [T, H], d_weight fp32 [H] or None) at the norm's `total`."""
    _need(total, "total", _BF16, 2)
    T, H = total.shape
    _optional(_given(d_out, "d_out"), "d_out", _BF16, total.shape)
    _optional(d_total, "d_total", _BF16, total.shape)
    _optional(weight, "weight", _BF16, (H,))
    lib = _lib_handle()
    with _on(stream):
        dx = _output(True if dx is None else dx, "dx", torch.bfloat16, total.shape, total.device)
        d_weight = _output(d_weight, "d_weight", torch.float32, (H,), total.device)
        n = _bytes("ep_rmsnorm_grad_workspace_bytes", T, H) if d_weight is not None else 0
        ws = _workspace(n, total.device)
    _check(lib.ep_rmsnorm_grad(_ptr(total), _ptr(weight), _ptr(d_out), _ptr(d_total), T, H, eps, _ptr(dx),
                               _ptr(d_weight), _ptr(ws), n, _current_stream(stream)), "ep_rmsnorm_grad")
    return dx, d_weight


# ----------------------------------------------------------------------------- router

@dataclass
class Routing:
    topk_idx: torch.Tensor                 # int32 [T, k]
    topk_w: torch.Tensor                   # fp32 [T, k]
    expert_counts: Optional[torch.Tensor]  # int32 [E]
    prob_sums: Optional[torch.Tensor]      # fp32 [E]
    loss: Optional[torch.Tensor]           # fp32 [1]
    mask: Optional[torch.Tensor]
    normalize: bool
    balance: float


def _logits(logits: torch.Tensor) -> Tuple[int, int]:
    _need(logits, "logits", (torch.float32, torch.bfloat16), 2)
    return logits.shape


def route(logits: torch.Tensor, k: int, *, mask: Optional[torch.Tensor] = None, normalize: bool = True,
          balance: float = 0.0, counts: bool = True, out: Optional[Routing] = None, stream=None) -> Routing:
    """ep_route on logits [T, E]: the k best experts, their gates, and with `counts` the slots
    per expert, the probability sums and the balance loss.  mask: bool or uint8 [T], False for
    tokens that are not live.  `out` (of an earlier call of the same sizes) is written again."""
    T, E = _logits(logits)
    _optional(mask, "mask", (torch.bool, torch.uint8), (T,))
    lib, dev = _lib_handle(), logits.device
    with _on(stream):
        if out is None:
            f32 = torch.float32
            out = Routing(torch.empty(T, k, dtype=torch.int32, device=dev), torch.empty(T, k, dtype=f32, device=dev),
                          *((torch.empty(E, dtype=torch.int32, device=dev), torch.empty(E, dtype=f32, device=dev),
                             torch.empty(1, dtype=f32, device=dev)) if counts else (None, None, None)), None, True, 0.0)
        else:
            _optional(out.topk_idx, "out.topk_idx", _I32, (T, k))
            _optional(out.topk_w, "out.topk_w", _F32, (T, k))
            _optional(out.expert_counts, "out.expert_counts", _I32, (E,))
            _optional(out.prob_sums, "out.prob_sums", _F32, (E,))
            _optional(out.loss, "out.loss", _F32, (1,))
        n = 0
        if out.expert_counts is not None:
            n = _bytes("ep_route_workspace_bytes", T, E)
        ws = _workspace(n, dev)
    _check(lib.ep_route(_ptr(logits), logits.dtype == torch.bfloat16, _ptr(mask), T, E, k, normalize, balance,
                        _ptr(out.topk_idx), _ptr(out.topk_w), _ptr(out.expert_counts), _ptr(out.prob_sums),
                        _ptr(out.loss), _ptr(ws), n, _current_stream(stream)), "ep_route")
    out.mask, out.normalize, out.balance = mask, normalize, balance
    return out


def route_grad(logits: torch.Tensor, routing: Routing, d_topk_w: Optional[torch.Tensor] = None,
               d_loss: Optional[torch.Tensor] = None, *, counts: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """ep_route_grad: the logits' gradient from the gates' (d_topk_w [T, k]) and the loss's
    (d_loss [1]).  counts: the slots per expert of the loss, those of `routing` by default."""
    T, E = _logits(logits)
    k = routing.topk_idx.shape[1]
    _optional(routing.topk_idx, "routing.topk_idx", _I32, (T, k))
    _optional(routing.mask, "routing.mask", (torch.bool, torch.uint8), (T,))
    _optional(d_topk_w, "d_topk_w", _F32, (T, k))
    _optional(d_loss, "d_loss", _F32, (1,))
    counts = routing.expert_counts if counts is None else counts
    _optional(counts, "counts", _I32, (E,))
    with _on(stream):
        out = _output(True if out is None else out, "out", logits.dtype, logits.shape, logits.device)
    _check(_lib_handle().ep_route_grad(
        _ptr(logits), logits.dtype == torch.bfloat16, _ptr(routing.mask), _ptr(routing.topk_idx), _ptr(counts),
        _ptr(d_topk_w), _ptr(d_loss), T, E, k, routing.normalize, routing.balance, _ptr(out), _current_stream(stream)),
        "ep_route_grad")
    return out


# ---------------------------------------------------------------------------- combine

def combine_grad(d_out: torch.Tensor, y: torch.Tensor, slot_pos: torch.Tensor, topk_w: torch.Tensor, *,
                 dy: Union[bool, torch.Tensor] = True, d_topk_w: Union[bool, torch.Tensor] = True,
                 stream=None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """ep_combine_grad of combine_rows(y, slot_pos, topk_w): (dy bf16 like y, d_topk_w fp32
    [T, k]).  Rows that no slot names keep what dy holds.  A new dy holds zeros there if y has
    more rows than there are slots; with as many or fewer its memory is not cleared, so where
    slots are without a row (a slot_pos outside y) and the rows left over are read, give a
    zeroed `dy`."""
    _need(topk_w, "topk_w", _F32, 2)
    _need(y, "y", _BF16, 2)
    T, k = topk_w.shape
    H = y.shape[1]
    _optional(_given(d_out, "d_out"), "d_out", _BF16, (T, H))
    _optional(_given(slot_pos, "slot_pos"), "slot_pos", _I32, (T * k,))
    with _on(stream):
        if dy is True and y.shape[0] > T * k:
            dy = torch.zeros_like(y)
        else:
            dy = _output(dy, "dy", torch.bfloat16, y.shape, y.device)
        d_topk_w = _output(d_topk_w, "d_topk_w", torch.float32, (T, k), y.device)
    _check(_lib_handle().ep_combine_grad(_ptr(d_out), _ptr(y), y.shape[0], _ptr(slot_pos), _ptr(topk_w), T, H, k,
                                         _ptr(dy), _ptr(d_topk_w), _current_stream(stream)), "ep_combine_grad")
    return dy, d_topk_w


# ------------------------------------------------------------------- experts' product

@dataclass
class Product:
    out: torch.Tensor
    pre: Optional[torch.Tensor]


def _act(act: str) -> int:
    if act not in _lib.EP_ACTIVATIONS:
        raise ValueError(f"act must be one of {list(_lib.EP_ACTIVATIONS)}")
    return _lib.EP_ACTIVATIONS[act]


def _weights(w: torch.Tensor, act: str, dtypes) -> Tuple[int, int, int, int]:
    """(E, weight rows, N, K) of [E, rows, K] weights."""
    _need(w, "w", dtypes, 3)
    E, wide, K = w.shape
    if act == "swiglu" and wide % 2:
        raise ValueError("swiglu needs an even number of weight rows: the gates', then the ups'")
    return E, wide, wide // 2 if act == "swiglu" else wide, K


def _offsets(offsets: Optional[torch.Tensor], E: int):
    if offsets is None:
        if E != 1:
            raise ValueError("more than one expert needs offsets")
    else:
        _optional(offsets, "offsets", _I32, (E + 1,))


def expert_product(x: torch.Tensor, w: torch.Tensor, offsets: Optional[torch.Tensor] = None, *,
                   w_scale: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, act: str = "none",
                   residual: Optional[torch.Tensor] = None, keep_pre: Union[bool, torch.Tensor] = False,
                   out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16,
                   stream=None) -> Product:
    """ep_expert_product: act(x w[e]^T + bias[e]) + residual for the rows of each expert.

    x: bf16 [rows, K] with bf16 w [E, N, K], or 8-bit rows (uint8 [rows, K + 16]) with
    float8_e4m3fn w and w_scale fp32 [E, N].  offsets: int32 [E + 1] of a layout, none for one
    expert.  act: none, relu, silu, gelu, or swiglu (w [E, 2N, K]: gates, then ups).  keep_pre:
    also the values before the activation, as the gradient reads them.  Rows outside the offsets
    keep what the outputs hold (new ones are not cleared)."""
    bits8 = x.dtype == torch.uint8
    _need(x, "x", (torch.uint8,) if bits8 else _BF16, 2)
    E, wide, N, K = _weights(w, act, _F8 if bits8 else _BF16)
    rows = x.shape[0]
    _shape(x, "x", (rows, K + EP_ROWS8_EXTRA if bits8 else K))
    _offsets(offsets, E)
    if bits8 and w_scale is None:
        raise ValueError("8-bit weights need w_scale")
    _optional(w_scale, "w_scale", _F32, (E, wide))
    _optional(bias, "bias", _BF16, (E, wide))
    _optional(residual, "residual", _BF16, (rows, N))
    code = _act(act)
    if out is not None:
        out_dtype = out.dtype
    if out_dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"out has dtype {out_dtype}, expected bfloat16 or float32")
    lib = _lib_handle()
    kind = EP_ROWS_8BIT if bits8 else EP_ROWS_BF16
    with _on(stream):
        got = Product(_output(True if out is None else out, "out", out_dtype, (rows, N), x.device),
                      _output(keep_pre, "pre", torch.bfloat16, (rows, wide), x.device))
        n = _bytes("ep_expert_product_workspace_bytes", rows, E, K, N, kind, code)
        ws = _workspace(n, x.device)
    _check(lib.ep_expert_product(
        _ptr(x), kind, rows, _ptr(offsets), E, _ptr(w), _ptr(w_scale), K, N, _ptr(bias), code, _ptr(residual),
        _ptr(got.pre), _ptr(got.out), EP_OUT_F32 if out_dtype == torch.float32 else EP_OUT_BF16, _ptr(ws), n,
        _current_stream(stream)), "ep_expert_product")
    return got


@dataclass
class ProductGrad:
    dx: Optional[torch.Tensor]
    dw: Optional[torch.Tensor]
    dbias: Optional[torch.Tensor]


def expert_product_grad(x: torch.Tensor, w: torch.Tensor, d_y: torch.Tensor, offsets: Optional[torch.Tensor] = None, *,
                        pre: Optional[torch.Tensor] = None, act: str = "none", with_bias: bool = False,
                        dx: Union[bool, torch.Tensor] = True, dw: Union[bool, torch.Tensor] = True,
                        dbias: Optional[torch.Tensor] = None, stream=None) -> ProductGrad:
    """ep_expert_product_grad of a bf16 product: dx [rows, K], dw [E, N, K], and with_bias dbias
    fp32 [E, N].  pre: what the forward kept, needed with an activation.  Rows outside the
    offsets keep what dx holds (a new one is not cleared)."""
    _need(x, "x", _BF16, 2)
    E, wide, N, K = _weights(w, act, _BF16)
    rows = x.shape[0]
    _shape(x, "x", (rows, K))
    _offsets(offsets, E)
    _optional(_given(d_y, "d_y"), "d_y", _BF16, (rows, N))
    code = _act(act)
    if act != "none" and pre is None:
        raise ValueError("an activation's gradient needs pre")
    _optional(pre, "pre", _BF16, (rows, wide))
    lib = _lib_handle()
    with _on(stream):
        got = ProductGrad(_output(dx, "dx", torch.bfloat16, (rows, K), x.device),
                          _output(dw, "dw", torch.bfloat16, (E, wide, K), x.device),
                          _output(dbias if dbias is not None else with_bias, "dbias", torch.float32, (E, wide), x.device))
        n = _bytes("ep_expert_product_grad_workspace_bytes", rows, E, K, N, code,
                   (_lib.EP_GRAD_DBIAS if got.dbias is not None else 0) | (_lib.EP_GRAD_WITHOUT_DX if got.dx is None else 0)
                   | (_lib.EP_GRAD_WITHOUT_DW if got.dw is None else 0))
        ws = _workspace(n, x.device)
    _check(lib.ep_expert_product_grad(
        _ptr(x), rows, _ptr(offsets), E, _ptr(w), K, N, code, _ptr(pre), _ptr(d_y), _ptr(got.dx), _ptr(got.dw),
        _ptr(got.dbias), _ptr(ws), n, _current_stream(stream)), "ep_expert_product_grad")
    return got


# ------------------------------------------------------------------ low-rank adapters

@dataclass
class AdapterRows:
    """A batch's rows by adapter.  order: int32 [rows], none where the rows come by adapter already;
    offsets: int32 [A + 1], where each adapter's rows begin in that order."""
    order: Optional[torch.Tensor]
    offsets: Optional[torch.Tensor]


def adapter_rows(row_adapter: torch.Tensor, num_adapters: int, *, out: Optional[AdapterRows] = None,
                 stream=None) -> AdapterRows:
    """ep_adapter_rows: the rows sorted by adapter from each row's adapter, int32 [rows] (an id
    outside [0, num_adapters): none).  Made once for all the projections of a batch."""
    _need(row_adapter, "row_adapter", _I32, 1)
    n, dev = row_adapter.shape[0], row_adapter.device
    if out is None:
        with _on(stream):
            out = AdapterRows(torch.empty(n, dtype=torch.int32, device=dev),
                              torch.empty(max(num_adapters, 0) + 1, dtype=torch.int32, device=dev))
    else:
        _optional(_given(out.order, "out.order"), "out.order", _I32, (n,))
        _optional(_given(out.offsets, "out.offsets"), "out.offsets", _I32, (num_adapters + 1,))
    _check(_lib_handle().ep_adapter_rows(_ptr(row_adapter), n, num_adapters, _ptr(out.order), _ptr(out.offsets),
                                         _current_stream(stream)), "ep_adapter_rows")
    return out


@dataclass
class AdapterProduct:
    out: torch.Tensor
    pre: Optional[torch.Tensor]
    low: Optional[torch.Tensor]


def _adapters(x, a, b, rows, w, scale, act):
    """(rows, A, R, K, weight rows, N) of the adapters' arguments, checked."""
    _need(x, "x", _BF16, 2)
    _need(a, "a", _BF16, 3)
    _need(b, "b", _BF16, 3)
    (n, K), (A, wide, R) = x.shape, b.shape
    _shape(a, "a", (A, R, K))
    if act == "swiglu" and wide % 2:
        raise ValueError("swiglu needs an even number of weight rows: the gates', then the ups'")
    _optional(w, "w", _BF16, (wide, K))
    _optional(scale, "scale", _F32, (A,))
    if rows.offsets is None:
        if A != 1:
            raise ValueError("more than one adapter needs the rows' offsets")
    else:
        _optional(rows.offsets, "rows.offsets", _I32, (A + 1,))
    _optional(rows.order, "rows.order", _I32, (n,))
    return n, A, R, K, wide, wide // 2 if act == "swiglu" else wide


_ALL_ROWS = AdapterRows(None, None)


def adapter_product(x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, rows: AdapterRows = _ALL_ROWS, *,
                    w: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                    bias: Optional[torch.Tensor] = None, act: str = "none", residual: Optional[torch.Tensor] = None,
                    keep_pre: Union[bool, torch.Tensor] = False, keep_low: Union[bool, torch.Tensor] = False,
                    out: Optional[torch.Tensor] = None, stream=None) -> AdapterProduct:
    """ep_adapter_product: act(x w^T + scale (x a[i]^T) b[i]^T + bias) + residual, i the row's adapter, if any.

    x bf16 [rows, K]; a bf16 [A, R, K], b bf16 [A, N, R]; w bf16 [N, K], or none for the adapters
    alone; scale fp32 [A]; bias bf16 [N].  rows: adapter_rows of the batch; AdapterRows(None, offsets) for
    rows that come by adapter; left out, one adapter has every row.  act: as expert_product (swiglu:
    w and b with 2N rows).  keep_pre, keep_low: also the values before the activation, and the
    low-rank values [rows, R], as the gradient reads them.  `out` may be the residual itself."""
    n, A, R, K, wide, N = _adapters(x, a, b, rows, w, scale, act)
    _optional(bias, "bias", _BF16, (wide,))
    _optional(residual, "residual", _BF16, (n, N))
    code, lib = _act(act), _lib_handle()
    with _on(stream):
        got = AdapterProduct(_output(True if out is None else out, "out", torch.bfloat16, (n, N), x.device),
                             _output(keep_pre, "pre", torch.bfloat16, (n, wide), x.device),
                             _output(keep_low, "low", torch.bfloat16, (n, R), x.device))
        size = _bytes("ep_adapter_product_workspace_bytes", n, A, R, K, N, w is not None, code)
        ws = _workspace(size, x.device)
    _check(lib.ep_adapter_product(
        _ptr(x), n, _ptr(rows.order), _ptr(rows.offsets), A, R, _ptr(a), _ptr(b), _ptr(scale), _ptr(w), K, N, _ptr(bias),
        code, _ptr(residual), _ptr(got.pre), _ptr(got.low), _ptr(got.out), _ptr(ws), size, _current_stream(stream)),
        "ep_adapter_product")
    return got


@dataclass
class AdapterGrad:
    dx: Optional[torch.Tensor]
    da: Optional[torch.Tensor]
    db: Optional[torch.Tensor]


def adapter_product_grad(x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, low: torch.Tensor, d_y: torch.Tensor,
                         rows: AdapterRows = _ALL_ROWS, *, w: Optional[torch.Tensor] = None,
                         scale: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None, act: str = "none",
                         dx: Union[bool, torch.Tensor] = True, da: Union[bool, torch.Tensor] = True,
                         db: Union[bool, torch.Tensor] = True, stream=None) -> AdapterGrad:
    """ep_adapter_product_grad, with w held fast: dx bf16 [rows, K], da like a, db like b.  low, pre:
    what the forward kept (pre is needed with an activation).  Without w, dx is the adapters' part.  A trained
    bias's gradient: expert_product_grad(x, w[None], d_y, pre=pre, act=act, dx=False, dw=False, with_bias=True).dbias[0]
    (and w's: its dw)."""
    n, A, R, K, wide, N = _adapters(x, a, b, rows, w, scale, act)
    _optional(_given(low, "low"), "low", _BF16, (n, R))
    _optional(_given(d_y, "d_y"), "d_y", _BF16, (n, N))
    code = _act(act)
    if act != "none" and pre is None:
        raise ValueError("an activation's gradient needs pre")
    _optional(pre, "pre", _BF16, (n, wide))
    lib = _lib_handle()
    with _on(stream):
        got = AdapterGrad(_output(dx, "dx", torch.bfloat16, (n, K), x.device),
                          _output(da, "da", torch.bfloat16, (A, R, K), x.device),
                          _output(db, "db", torch.bfloat16, (A, wide, R), x.device))
        size = _bytes("ep_adapter_product_grad_workspace_bytes", n, A, R, K, N, w is not None, code, rows.order is not None,
                      (_lib.EP_ADAPTER_DX if got.dx is not None else 0) | (_lib.EP_ADAPTER_DA if got.da is not None else 0)
                      | (_lib.EP_ADAPTER_DB if got.db is not None else 0))
        ws = _workspace(size, x.device)
    _check(lib.ep_adapter_product_grad(
        _ptr(x), n, _ptr(rows.order), _ptr(rows.offsets), A, R, _ptr(a), _ptr(b), _ptr(scale), _ptr(w), K, N, _ptr(low),
        code, _ptr(pre), _ptr(d_y), _ptr(got.dx), _ptr(got.da), _ptr(got.db), _ptr(ws), size, _current_stream(stream)),
        "ep_adapter_product_grad")
    return got


# ---------------------------------------------------------------------------- dropout

def dropout(x: torch.Tensor, p: float, rng: torch.Tensor, *, site: int = 0, residual: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """ep_dropout: residual + dropout(x), bf16 of any shape with a multiple of 8 values.

    rng: int64 [2] on the device, the seed and the step; site: which of the program's dropouts this is.
    The same rng and site give the same mask, so the gradient of x is dropout(d_out, p, rng, site=site).
    `out` may be x or the residual itself."""
    _need(x, "x", _BF16)
    _optional(residual, "residual", _BF16, x.shape)
    _rng(rng, site)
    with _on(stream):
        out = _output(True if out is None else out, "out", torch.bfloat16, x.shape, x.device)
    _check(_lib_handle().ep_dropout(_ptr(x), _ptr(residual), x.numel(), p, _ptr(rng), site, _ptr(out),
                                    _current_stream(stream)), "ep_dropout")
    return out


def _rng(rng: torch.Tensor, site: int):
    _optional(_given(rng, "rng"), "rng", _I64, (2,))
    if not 0 <= site < 1 << 32:
        raise ValueError(f"site must be a number of 32 bits, not {site}")


def dropout_rmsnorm(x: torch.Tensor, p: float, rng: torch.Tensor, weight: Optional[torch.Tensor] = None, *, site: int = 0,
                    residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
                    total: Union[bool, torch.Tensor, None] = None, out: Union[bool, torch.Tensor] = True,
                    rows8: Union[bool, torch.Tensor] = False, stream=None) -> Norm:
    """ep_dropout_rmsnorm: rmsnorm of dropout(x) + residual; total = that sum (written where there is a
    residual, or on request).  The rest as rmsnorm and dropout."""
    _need(x, "x", _BF16, 2)
    T, H = x.shape
    _optional(residual, "residual", _BF16, x.shape)
    _optional(weight, "weight", _BF16, (H,))
    _rng(rng, site)
    with _on(stream):
        got = Norm(_output(residual is not None if total is None else total, "total", torch.bfloat16, x.shape, x.device),
                   _output(out, "out", torch.bfloat16, x.shape, x.device),
                   _output(rows8, "rows8", torch.uint8, (T, H + EP_ROWS8_EXTRA), x.device))
    _check(_lib_handle().ep_dropout_rmsnorm(_ptr(x), _ptr(residual), _ptr(weight), T, H, eps, p, _ptr(rng), site,
                                            _ptr(got.total), _ptr(got.out), _ptr(got.rows8), _current_stream(stream)),
           "ep_dropout_rmsnorm")
    return got


def dropout_rmsnorm_grad(total: torch.Tensor, weight: Optional[torch.Tensor], d_out: torch.Tensor, p: float,
                         rng: torch.Tensor, *, site: int = 0, d_total: Optional[torch.Tensor] = None, eps: float = 1e-6,
                         dx: Union[bool, torch.Tensor] = True, d_residual: Union[bool, torch.Tensor] = True,
                         d_weight: Union[bool, torch.Tensor] = True, stream=None
                         ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor], Optional[torch.Tensor]]:
    """ep_dropout_rmsnorm_grad: (dx bf16 [T, H], d_residual bf16 [T, H], d_weight fp32 [H]) at the norm's
    `total`; each may be left out, but one of the first two is wanted."""
    _need(total, "total", _BF16, 2)
    T, H = total.shape
    _optional(_given(d_out, "d_out"), "d_out", _BF16, total.shape)
    _optional(d_total, "d_total", _BF16, total.shape)
    _optional(weight, "weight", _BF16, (H,))
    _rng(rng, site)
    lib = _lib_handle()
    with _on(stream):
        dx = _output(dx, "dx", torch.bfloat16, total.shape, total.device)
        d_residual = _output(d_residual, "d_residual", torch.bfloat16, total.shape, total.device)
        d_weight = _output(d_weight, "d_weight", torch.float32, (H,), total.device)
        n = _bytes("ep_rmsnorm_grad_workspace_bytes", T, H) if d_weight is not None else 0
        ws = _workspace(n, total.device)
    _check(lib.ep_dropout_rmsnorm_grad(_ptr(total), _ptr(weight), _ptr(d_out), _ptr(d_total), T, H, eps, p, _ptr(rng), site,
                                       _ptr(dx), _ptr(d_residual), _ptr(d_weight), _ptr(ws), n, _current_stream(stream)),
           "ep_dropout_rmsnorm_grad")
    return dx, d_residual, d_weight
