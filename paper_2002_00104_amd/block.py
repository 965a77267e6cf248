"""The operators around the integer inner product in a transformer block (pwlq_block.h): rows of activations in 8 bits,
the norms before and after a block with its gate and residual scale, and low-rank adapters beside a projection with
frozen, packed weights; each with what training takes.

A projection with packed weights, its adapters and the norm in front of it, for rows x of the residual stream and the
last block's output f:

    x, codes, step = norm_block(x, f, pre_weight=w, post_weight=v, pack=True)
    y, _ = pwlq.linear_i8(codes, 1.0, 0.0, packed_codes, packed_flags, N, bits, p, m)
    y, h = adapter(codes, down, up, ids, scale, base=y, x_step=step, base_step=step, dtype=torch.bfloat16)

In training `codes` and `step` are the activation checkpoint that adapter_backward reads, and pack_rows makes those of
norm_block_backward.  Autograd sees none of it: norm_block and adapter refuse tensors that require gradients unless they are
called under torch.no_grad(), as in the forward pass of a torch.autograd.Function whose backward calls theirs.

Argument marshalling only: the work is the library's, on the current stream of the current device, where all tensors are.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import torch

from .pwlq import PwlqError, _stream

try:
    from . import _pwlq_block
except ImportError as e:
    raise ImportError(f"the module _pwlq_block is missing: build it with `python -m paper_2002_00104_amd.build` ({e})") from e
_pwlq_block.raises(PwlqError)

Tensor = torch.Tensor


def pack_rows(x: Tensor, out: Optional[Tuple[Tensor, Tensor]] = None) -> Tuple[Tensor, Tensor]:
    """pwlq_pack_rows: rows [T, K] of float32, bfloat16 or float16 in 8 bits.
    Returns (codes int8 [T, K], step f32 [T]); a value is code * step[row]."""
    codes, step = out or (None, None)
    return _pwlq_block.pack_rows(x, codes, step, _stream())


def unpack_rows(codes: Tensor, step: Tensor, dtype: torch.dtype = torch.float32, out: Optional[Tensor] = None) -> Tensor:
    """pwlq_unpack_rows: the values that packed rows stand for."""
    return _pwlq_block.unpack_rows(codes, step, dtype, out, _stream())


def norm_block(x: Tensor, f: Optional[Tensor] = None, *, pre_weight: Tensor, post_weight: Optional[Tensor] = None,
               gate: Optional[Tensor] = None, alpha: float = 1.0, eps: float = 1e-6, pack: bool = False) -> Tuple[Tensor, ...]:
    """pwlq_norm_block: x_out = x + alpha * gate * norm(f), u = norm(x_out), for rows of D columns.

    x residual stream [T, D]; f the block's output [T, D], or None for the norm alone; pre_weight and post_weight f32 [D]
    (post_weight None: f as it is); gate [G, D] of f's type, G a divisor of T.  Returns (x_out, u), or with `pack`
    (x_out, codes, step); x_out is x where f is None."""
    return _pwlq_block.norm_block(x, f, pre_weight, post_weight, gate, alpha, eps, pack, _stream())


def norm_block_backward(du: Optional[Tensor], dx_out: Optional[Tensor], x_out: Tensor, f: Optional[Tensor] = None, *,
                        pre_weight: Tensor, post_weight: Optional[Tensor] = None, gate: Optional[Tensor] = None,
                        alpha: float = 1.0, eps: float = 1e-6, x_step: Optional[Tensor] = None,
                        f_step: Optional[Tensor] = None, dtype: Optional[torch.dtype] = None,
                        workspace: Optional[Tensor] = None) -> Dict[str, Optional[Tensor]]:
    """pwlq_norm_block_backward: gradients of norm_block's inputs from those of its outputs, du of u and dx_out of x_out
    (one of them may be None).  x_out and f as the forward pass had them, or both int8 with their steps.  dx has dx_out's type,
    without it x_out's, or du's where x_out is int8; df has du's, without it f's, or where f is int8 the gate's, else `dtype` (dx's
    type by default).  Returns dx, df, d_pre, d_post and d_gate (None where there is no such input)."""
    dx, df, d_pre, d_post, d_gate = _pwlq_block.norm_block_backward(
        du, dx_out, x_out, f, pre_weight, post_weight, gate, alpha, eps, x_step, f_step, dtype, workspace, _stream())
    return dict(dx=dx, df=df, d_pre=d_pre, d_post=d_post, d_gate=d_gate)


def adapter(x: Tensor, down: Tensor, up: Tensor, ids: Tensor, scale: Tensor, *, base: Optional[Tensor] = None,
            x_step: Optional[Tensor] = None, base_step: Optional[Tensor] = None, dtype: Optional[torch.dtype] = None,
            out: Optional[Tensor] = None, workspace: Optional[Tensor] = None) -> Tuple[Tensor, Tensor]:
    """pwlq_adapter: out[t] = base_step[t] * base[t] + h[t] up[a], h[t] = scale[a] * x[t] down[a]^T, a = ids[t].

    x [T, K] of the adapters' type, or int8 with x_step; down [n, R, K], up [n, R, N]; ids int32 [T] (outside 0..n-1: no
    adapter); scale f32 [n]; base [T, N] float32 or of the adapters' type, or None.  Returns (out [T, N] of `dtype`,
    h f32 [T, R]); `dtype` is float32 or the adapters' type, which is the default.  `out` may be base."""
    return _pwlq_block.adapter(x, down, up, ids, scale, base, x_step, base_step, dtype, out, workspace, _stream())


def adapter_backward(dy: Tensor, x: Tensor, down: Tensor, up: Tensor, ids: Tensor, scale: Tensor, h: Tensor, *,
                     x_step: Optional[Tensor] = None, dx_base: Optional[Tensor] = None, dtype: Optional[torch.dtype] = None,
                     workspace: Optional[Tensor] = None) -> Dict[str, Tensor]:
    """pwlq_adapter_backward: gradients from dy [T, N] (the adapters' type), with x as adapter had it or an 8-bit checkpoint
    of it, and its h.  dx = dx_base + what the adapters pass on, dx_base [T, K] float32 or of the adapters' type, or
    None.  Returns d_down and d_up (float32) and dx (of dx_base's type, else of `dtype`, the adapters' by default)."""
    d_down, d_up, dx = _pwlq_block.adapter_backward(dy, x, down, up, ids, scale, h, x_step, dx_base, dtype, workspace, _stream())
    return dict(d_down=d_down, d_up=d_up, dx=dx)
