"""The operators around the integer inner product in a transformer block (pwlq_block.h): rows of activations in 8 bits,
the norms before and after a block with its gate and residual scale, and low-rank adapters beside a projection with
frozen, packed weights; each with what training takes.

A projection with packed weights, its adapters and the norm in front of it, for rows x of the residual stream and the
last block's output f:

    x, codes, step = norm_block(x, f, pre_weight=w, post_weight=v, pack=True)
    y, _ = pwlq.linear_i8(codes, 1.0, 0.0, packed_codes, packed_flags, N, bits, p, m)
    y, h = adapter(codes, down, up, ids, scale, base=y, x_step=step, base_step=step, dtype=torch.bfloat16)

In training `codes` and `step` are the activation checkpoint that adapter_backward reads, and pack_rows makes those of
norm_block_backward.  Argument marshalling only: the work is the library's, on the current stream.
"""
from __future__ import annotations

import ctypes
from typing import Dict, Optional, Tuple

import torch

from .pwlq import _check, _pwlq_call, _stream, _workspace, lib

Tensor = torch.Tensor

_TYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2, torch.int8: 3}
_FLOATS = (torch.float32, torch.bfloat16, torch.float16)
_PACK, _UNPACK, _NORM, _NORM_BACKWARD, _ADAPTER, _ADAPTER_BACKWARD = (
    ctypes.cast(f, ctypes.c_void_p).value
    for f in (lib.pwlq_pack_rows, lib.pwlq_unpack_rows, lib.pwlq_norm_block, lib.pwlq_norm_block_backward, lib.pwlq_adapter,
              lib.pwlq_adapter_backward))
_NONE = (None, 0, 0, None)


def _rows(name: str, t: Optional[Tensor], T: int, cols: int, device, dtypes, step: Optional[Tensor] = None, factors: bool = False):
    """The four arguments that rows take; `factors`: steps may go with a float type too."""
    if t is None:
        if step is not None:
            raise ValueError(f"{name} is left out and has steps")
        return _NONE
    if not (t.device == device and t.dtype in dtypes and t.dim() == 2 and t.shape[0] == T and t.shape[1] == cols):
        raise ValueError(f"{name} must be a [{T}, {cols}] tensor of {' or '.join(str(d) for d in dtypes)} on {device}")
    stride = t.stride(0)
    if (cols > 1 and t.stride(1) != 1) or (stride < cols and T > 1):
        raise ValueError(f"{name} must have its columns next to each other, and rows that do not overlap")
    if (t.dtype == torch.int8) != (step is not None) and not (factors and t.dtype != torch.int8):
        raise ValueError(f"{name} needs its steps where it is int8, and has none else")
    if step is not None:
        _vector(name + "'s steps", step, (T,), device)
    return t, _TYPE[t.dtype], stride if T > 1 else cols, step


def _vector(name: str, t: Optional[Tensor], shape: Tuple[int, ...], device, dtype=torch.float32) -> None:
    if t is not None and not (t.device == device and t.dtype == dtype and t.shape == shape and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {list(shape)} on {device}")


def _on_gpu(name: str, t: Tensor) -> torch.device:
    if not (t.is_cuda and t.dim() == 2):
        raise ValueError(f"{name} must be a matrix on the GPU")
    return t.device


def pack_rows(x: Tensor, out: Optional[Tuple[Tensor, Tensor]] = None) -> Tuple[Tensor, Tensor]:
    """pwlq_pack_rows: rows [T, K] of float32, bfloat16 or float16 in 8 bits.
    Returns (codes int8 [T, K], step f32 [T]); a value is code * step[row]."""
    device = _on_gpu("x", x)
    T, K = x.shape
    rows = _rows("x", x, T, K, device, _FLOATS)
    if out is None:
        out = torch.empty(T, K, dtype=torch.int8, device=device), torch.empty(T, dtype=torch.float32, device=device)
    codes, step = out
    _check(_pwlq_call.pack_rows(_PACK, *rows, T, K, codes, step, _stream()))
    return codes, step


def unpack_rows(codes: Tensor, step: Tensor, dtype: torch.dtype = torch.float32, out: Optional[Tensor] = None) -> Tensor:
    """pwlq_unpack_rows: the values that packed rows stand for."""
    device = _on_gpu("codes", codes)
    T, K = codes.shape
    _vector("codes", codes, (T, K), device, torch.int8)
    _vector("step", step, (T,), device)
    if out is None:
        out = torch.empty(T, K, dtype=dtype, device=device)
    _check(_pwlq_call.unpack_rows(_UNPACK, codes, step, T, K, *_rows("out", out, T, K, device, _FLOATS), _stream()))
    return out


def norm_block(x: Tensor, f: Optional[Tensor] = None, *, pre_weight: Tensor, post_weight: Optional[Tensor] = None,
               gate: Optional[Tensor] = None, alpha: float = 1.0, eps: float = 1e-6, pack: bool = False):
    """pwlq_norm_block: x_out = x + alpha * gate * norm(f), u = norm(x_out), for rows of D columns.

    x residual stream [T, D]; f the block's output [T, D], or None for the norm alone; pre_weight and post_weight f32 [D]
    (post_weight None: f as it is); gate [G, D] of f's type, G a divisor of T.  Returns (x_out, u), or with `pack`
    (x_out, codes, step); x_out is x where f is None."""
    device = _on_gpu("x", x)
    T, D = x.shape
    dtype = x.dtype if f is None else f.dtype
    x_rows = _rows("x", x, T, D, device, _FLOATS)
    f_rows = _rows("f", f, T, D, device, _FLOATS)
    _vector("pre_weight", pre_weight, (D,), device)
    _vector("post_weight", post_weight, (D,), device)
    gate_rows = 0
    if gate is not None:
        gate_rows = gate.shape[0]
        _vector("gate", gate, (gate_rows, D), device, dtype)
    x_out, out_rows = x, _NONE
    if f is not None:
        x_out = torch.empty(T, D, dtype=x.dtype, device=device)
        out_rows = x_out, x_rows[1], D, None
    u = torch.empty(T, D, dtype=torch.int8 if pack else dtype, device=device)
    step = torch.empty(T, dtype=torch.float32, device=device) if pack else None
    _check(_pwlq_call.norm_block(_NORM, T, D, *x_rows, *f_rows, *out_rows, u, _TYPE[u.dtype], D, step, post_weight, pre_weight, gate,
                                 gate_rows, alpha, eps, _stream()))
    return (x_out, u, step) if pack else (x_out, u)


def norm_block_backward(du: Optional[Tensor], dx_out: Optional[Tensor], x_out: Tensor, f: Optional[Tensor] = None, *,
                        pre_weight: Tensor, post_weight: Optional[Tensor] = None, gate: Optional[Tensor] = None,
                        alpha: float = 1.0, eps: float = 1e-6, x_step: Optional[Tensor] = None,
                        f_step: Optional[Tensor] = None, workspace: Optional[Tensor] = None) -> Dict[str, Optional[Tensor]]:
    """pwlq_norm_block_backward: gradients of norm_block's inputs from those of its outputs, du of u and dx_out of x_out
    (one of them may be None).  x_out and f as the forward pass had them, or both int8 with their steps.
    Returns dx, df, d_pre, d_post and d_gate (None where there is no such input)."""
    device = _on_gpu("x_out", x_out)
    T, D = x_out.shape
    if du is None and dx_out is None:
        raise ValueError("du and dx_out are both None")
    if f is None and f_step is not None:
        raise ValueError("f is left out and has steps")
    kept = x_out.dtype == torch.int8
    stream = dx_out.dtype if dx_out is not None else du.dtype if kept else x_out.dtype
    dtype = du.dtype if du is not None else stream if f is None or kept else f.dtype
    du_rows = _rows("du", du, T, D, device, (dtype,))
    dxo_rows = _rows("dx_out", dx_out, T, D, device, (stream,))
    x_rows = _rows("x_out", x_out, T, D, device, (torch.int8 if kept else stream,), x_step)
    f_rows = _rows("f", f, T, D, device, (torch.int8 if kept else dtype,), f_step)
    _vector("pre_weight", pre_weight, (D,), device)
    _vector("post_weight", post_weight, (D,), device)
    gate_rows = 0
    if gate is not None:
        gate_rows = gate.shape[0]
        _vector("gate", gate, (gate_rows, D), device, dtype)
    if stream not in _FLOATS or dtype not in _FLOATS:
        raise ValueError("gradients of rows must be of a float type")
    f32 = torch.float32
    dx = torch.empty(T, D, dtype=stream, device=device)
    df = None if f is None else torch.empty(T, D, dtype=dtype, device=device)
    d_pre = torch.empty(D, dtype=f32, device=device)
    d_post = None if post_weight is None else torch.empty(D, dtype=f32, device=device)
    d_gate = None if gate is None else torch.empty(gate_rows, D, dtype=f32, device=device)
    if workspace is None:
        workspace = _workspace(lib.pwlq_norm_block_backward_workspace_bytes(T, D, gate_rows), device)
    _check(_pwlq_call.norm_block_backward(
        _NORM_BACKWARD, T, D, *du_rows, *dxo_rows, *x_rows, *f_rows, dx, _TYPE[stream], D, None,
        *(_NONE if df is None else (df, _TYPE[dtype], D, None)), post_weight, pre_weight, gate, gate_rows, alpha, eps, d_pre, d_post,
        d_gate, workspace, workspace.numel(), _stream()))
    return dict(dx=dx, df=df, d_pre=d_pre, d_post=d_post, d_gate=d_gate)


def _adapters(down: Tensor, up: Tensor, ids: Tensor, scale: Tensor, T: int, K: int, device):
    """Checks of what every adapter call takes; (adapters, R, N)."""
    if not (down.dim() == 3 and up.dim() == 3 and down.dtype in _FLOATS):
        raise ValueError("down [adapters, R, K] and up [adapters, R, N] must be float32, bfloat16 or float16")
    n, R, N = up.shape
    _vector("down", down, (n, R, K), device, down.dtype)
    _vector("up", up, (n, R, N), device, down.dtype)
    _vector("ids", ids, (T,), device, torch.int32)
    _vector("scale", scale, (n,), device)
    return n, R, N


def adapter(x: Tensor, down: Tensor, up: Tensor, ids: Tensor, scale: Tensor, *, base: Optional[Tensor] = None,
            x_step: Optional[Tensor] = None, base_step: Optional[Tensor] = None, dtype: Optional[torch.dtype] = None,
            out: Optional[Tensor] = None, workspace: Optional[Tensor] = None) -> Tuple[Tensor, Tensor]:
    """pwlq_adapter: out[t] = base_step[t] * base[t] + h[t] up[a], h[t] = scale[a] * x[t] down[a]^T, a = ids[t].

    x [T, K] of the adapters' type, or int8 with x_step; down [n, R, K], up [n, R, N]; ids int32 [T] (outside 0..n-1: no
    adapter); scale f32 [n]; base [T, N] float32 or of the adapters' type, or None.  Returns (out [T, N] of `dtype`,
    h f32 [T, R]); `dtype` is float32 or the adapters' type, which is the default."""
    device = _on_gpu("x", x)
    T, K = x.shape
    n, R, N = _adapters(down, up, ids, scale, T, K, device)
    own = (down.dtype, torch.float32)
    x_rows = _rows("x", x, T, K, device, (down.dtype, torch.int8), x_step)
    base_rows = _rows("base", base, T, N, device, own, base_step, True)
    if out is None:
        out = torch.empty(T, N, dtype=dtype or down.dtype, device=device)
    h = torch.empty(T, R, dtype=torch.float32, device=device)
    if workspace is None:
        workspace = _workspace(lib.pwlq_adapter_workspace_bytes(T, K, R), device)
    _check(_pwlq_call.adapter(_ADAPTER, T, K, N, R, n, _TYPE[down.dtype], down, up, ids, scale, *x_rows, *base_rows,
                              *_rows("out", out, T, N, device, own), h, workspace, workspace.numel(), _stream()))
    return out, h


def adapter_backward(dy: Tensor, x: Tensor, down: Tensor, up: Tensor, ids: Tensor, scale: Tensor, h: Tensor, *,
                     x_step: Optional[Tensor] = None, dx_base: Optional[Tensor] = None, dtype: Optional[torch.dtype] = None,
                     workspace: Optional[Tensor] = None) -> Dict[str, Tensor]:
    """pwlq_adapter_backward: gradients from dy [T, N] (the adapters' type), with x as adapter had it or an 8-bit checkpoint
    of it, and its h.  dx = dx_base + what the adapters pass on, dx_base [T, K] float32 or of the adapters' type, or
    None.  Returns d_down and d_up (float32) and dx (of dx_base's type, else of `dtype`, the adapters' by default)."""
    device = _on_gpu("x", x)
    T, K = x.shape
    n, R, N = _adapters(down, up, ids, scale, T, K, device)
    own = (down.dtype, torch.float32)
    dy_rows = _rows("dy", dy, T, N, device, (down.dtype,))
    x_rows = _rows("x", x, T, K, device, (down.dtype, torch.int8), x_step)
    base_rows = _rows("dx_base", dx_base, T, K, device, own)
    _vector("h", h, (T, R), device)
    dx = torch.empty(T, K, dtype=dx_base.dtype if dx_base is not None else dtype or down.dtype, device=device)
    d_down = torch.empty(n, R, K, dtype=torch.float32, device=device)
    d_up = torch.empty(n, R, N, dtype=torch.float32, device=device)
    if workspace is None:
        workspace = _workspace(lib.pwlq_adapter_backward_workspace_bytes(T, K, N, R, n), device)
    _check(_pwlq_call.adapter_backward(
        _ADAPTER_BACKWARD, T, K, N, R, n, _TYPE[down.dtype], down, up, ids, scale, *dy_rows, *x_rows, *base_rows,
        *_rows("dx", dx, T, K, device, own), h, d_down, d_up, workspace, workspace.numel(), _stream()))
    return dict(d_down=d_down, d_up=d_up, dx=dx)
