"""What a transformer block has between its projections (pwlq_attention.h): a paged cache of keys and values, in 16 bits or in
8-bit rows, new rows that enter it with their position's rotation on the way, and attention over it for single tokens, trees of
drafted tokens and prompts.

A block that decodes, with the projections and norms of `block` around it:

    cache = make_cache(pages, heads, page, D, torch.int8)
    q = append(cache, table, lengths, k, v, q, frequencies=f)
    y = attend(q, cache, table, lengths)
    codes, step = block.pack_rows(y.view(T, -1))                    for the output projection

A batch is S sequences: table int32 [S, n], the pages of each; lengths int32 [S], their rows with those of the call; starts int32
[S + 1], the first of the call's rows of each and their end, or None for one row each.  The call's rows are the last ones of
their sequences; rows from starts[S] on belong to none, and an output has there what it had (nothing in particular where a call makes it).

Argument marshalling only: the work is the library's, on the current stream of the current device, where all tensors are.
Autograd sees none of it: tensors that require gradients are refused unless a call is made under torch.no_grad().
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

import torch

from .pwlq import PwlqError, _stream

try:
    from . import _pwlq_attention
except ImportError as e:
    raise ImportError(f"the module _pwlq_attention is missing: build it with `python -m paper_2002_00104_amd.build` ({e})") from e
_pwlq_attention.raises(PwlqError)

Tensor = torch.Tensor


class Cache(NamedTuple):
    """Pages of keys and values, [pages, heads, page, D] of bfloat16 or float16, or int8 with a float32 step for each row of a
    head, [pages, heads, page].  page is a power of two from 16 on, D a multiple of 16 up to 256."""
    keys: Tensor
    values: Tensor
    key_step: Optional[Tensor] = None
    value_step: Optional[Tensor] = None


def make_cache(pages: int, heads: int, page: int, D: int, dtype: torch.dtype = torch.bfloat16, device="cuda") -> Cache:
    """An empty cache; with dtype int8 one of 8-bit rows."""
    shape = (pages, heads, page, D)
    keys, values = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
    if dtype != torch.int8:
        return Cache(keys, values)
    return Cache(keys, values, *(torch.zeros(shape[:3], dtype=torch.float32, device=device) for _ in range(2)))


def append(cache: Cache, table: Tensor, lengths: Tensor, k: Tensor, v: Tensor, q: Optional[Tensor] = None, *,
           starts: Optional[Tensor] = None, positions: Optional[Tensor] = None, frequencies: Optional[Tensor] = None,
           interleaved: bool = False, out: Optional[Tensor] = None) -> Optional[Tensor]:
    """pwlq_append: rows k and v [T, heads, D] into the cache; k and q [T, H, D] turned by their positions.

    positions int32 [T], by default each row's place in its sequence; frequencies float32 [R / 2] of the first R channels, R a
    multiple of 16 (None: no rotation), whose pairs are (i, i + R/2), or (2i, 2i + 1) with `interleaved`.  All rows of one type,
    the cache's if that is not int8; k, v and q may be columns of one matrix.  Returns the turned q (None without q)."""
    return _pwlq_attention.append(*cache, table, lengths, starts, k, v, q, positions, frequencies, interleaved, out, _stream())


def read(cache: Cache, table: Tensor, lengths: Tensor, *, starts: Optional[Tensor] = None, rows: Optional[int] = None,
         dtype: Optional[torch.dtype] = None, out: Optional[Tuple[Tensor, Tensor]] = None) -> Tuple[Tensor, Tensor]:
    """pwlq_read: the last rows of each sequence, [rows, heads, D] of keys and of values; `rows` goes with starts.  dtype is the
    cache's, or bfloat16 (the default) or float16 from int8."""
    k, v = out or (None, None)
    return _pwlq_attention.read(*cache, table, lengths, starts, rows, dtype, k, v, _stream())


def attend(q: Tensor, cache: Cache, table: Tensor, lengths: Tensor, *, starts: Optional[Tensor] = None, longest: Optional[int] = None,
           scale: Optional[float] = None, cap: float = 0.0, slopes: Optional[Tensor] = None, window: int = 0,
           prefix: Optional[Tensor] = None, tree: Optional[Tensor] = None, out: Optional[Tensor] = None,
           workspace: Optional[Tensor] = None) -> Tensor:
    """pwlq_attend: softmax(scores) v for q [T, H, D] over the cache; H is a multiple of the cache's heads.

    scores are scale (default D^-0.5) * q.k, capped by cap * tanh(./cap) where cap > 0, less slopes[h] * distance (float32 [H]).
    A row sees its sequence up to itself, the last `window` rows of that if it is not 0, and the first prefix[s] rows (int32 [S])
    in any case.  With tree, int64 [T, words], it sees what the sequence held before the call, and of the call's rows of its
    sequence those whose bit is set: row j's is bit j % 64 of word j // 64.  A row that sees nothing is zeros.  longest: the most
    rows of a sequence, where known; it chooses the kernel.  workspace: bytes for calls that take turns on one stream, else one is made; it
    holds up to 69 MB, by the sizes.  Returns [T, H, D] of q's type."""
    return _pwlq_attention.attend(*cache, table, lengths, starts, q, longest, scale, cap, slopes, window, prefix, tree, out, workspace, _stream())
