"""The operators of pwlq_attention.h from their formulas, in binary64 on the CPU, and what a result may be off.

u = 2^-24, U(t) half a unit in the last place of t relative to a value.  An attention output is sum w v / sum w with w = exp(s - m):
  - a score is a sum of D products in binary32, then at most eight operations: off by e = (D + 8) u (scale sum |q||k| + |bias|), where it
    is capped by 2^-19 cap more (its two forms' error, below 4e-7 of cap, and the reciprocal's and exponential's); a change of all scores by at most e
    moves the output by at most 2 e sum p |v|;
  - a weight is rounded once to the elements' type for the product with the values: U(t) sum p |v|.  With 8-bit values in bfloat16 that is the weight
    times the row's step, still one rounding; in binary16 the value is rounded too: U(t) more.  Weights of binary16 below its normal range
    are off by up to 2^-24 of a weight of 1, and the sum of weights is at least 1: 2^-24 sum |v|;
  - sums over n keys in binary32, of the weights and of the products, are off by at most n u each, and the exponential by 2 u.
The output is rounded once.
"""
import math

import torch

U = 2.0 ** -24
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


class Batch:
    """Sequences of the sizes [(new rows, length)], their pages drawn from `pages` in no order, on the CPU."""

    def __init__(self, g, sizes, page, spare=3, extra_columns=0):
        self.sizes, self.page = sizes, page
        need = [-(-max(n, 0) // page) for _, n in sizes]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=g).tolist()
        width = max(need + [1]) + extra_columns
        self.table = torch.full((len(sizes), width), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.lengths = torch.tensor([n for _, n in sizes], dtype=torch.int32)
        starts = [0]
        for n, _ in sizes:
            starts.append(starts[-1] + n)
        self.starts = torch.tensor(starts, dtype=torch.int32)
        self.rows = starts[-1]

    def slots(self, s):
        n, length = self.sizes[s]
        return range(length - n, length)

    def where(self, s, slot, pages):
        """(page, row), or None where there is none."""
        if not 0 <= slot < self.table.shape[1] * self.page:
            return None
        p = int(self.table[s, slot // self.page])
        return (p, slot % self.page) if 0 <= p < pages else None


def wide(rows, step):
    x = rows.double()
    return x if step is None else x * step.double()[..., None]


def sequence_rows(batch, cache, s):
    """Keys and values [length, heads, D] in binary64, and whether each row exists."""
    keys, values, key_step, value_step = cache
    length, P = batch.sizes[s][1], batch.page
    pages = batch.table[s, :-(-length // P)].long()
    there = ((pages >= 0) & (pages < keys.shape[0])).repeat_interleave(P)[:length]
    pages = pages.clamp(0, keys.shape[0] - 1)

    def rows(pool, step):
        x = wide(pool[pages], None if step is None else step[pages]).transpose(1, 2)
        return x.reshape(-1, *x.shape[2:])[:length]
    return rows(keys, key_step), rows(values, value_step), there


def seen_by(batch, s, window, prefix, tree):
    n, length = batch.sizes[s]
    own, slot = torch.arange(length - n, length)[:, None], torch.arange(length)
    if tree is not None:
        kept = length - n
        j = slot - kept
        first = int(batch.starts[s])
        word = tree[first:first + n].gather(1, (j // 64).clamp(0, tree.shape[1] - 1).expand(n, length))
        bit = ((word >> (j.clamp(min=0) % 64)) & 1).bool() & (j // 64 < tree.shape[1])
        seen = (j < 0) | bit
    else:
        seen = slot <= own
        if window:
            seen = seen & (own - slot < window)
        if prefix is not None:
            seen = seen | (slot < int(prefix[s]))
    return seen & (own >= 0)


def attend(q, batch, cache, scale, cap=0.0, slopes=None, window=0, prefix=None, tree=None):
    """Output and slack [T, H, D] in binary64; rows of no sequence are NaN."""
    T, H, D = q.shape
    G = cache[0].shape[1]
    out, slack = (torch.full((T, H, D), math.nan, dtype=torch.float64) for _ in range(2))
    coded = cache[2] is not None
    unit = UNIT[q.dtype] * (2 if coded and q.dtype == torch.float16 else 1)
    for s, (n, length) in enumerate(batch.sizes):
        first = int(batch.starts[s])
        if not n:
            continue
        if not length:
            out[first:first + n] = slack[first:first + n] = 0.0
            continue
        keys, values, there = sequence_rows(batch, cache, s)
        seen = seen_by(batch, s, window, prefix, tree) & there
        away = (torch.arange(length - n, length)[:, None] - torch.arange(length)).abs().double()
        for h in range(H):
            k, v = keys[:, h * G // H], values[:, h * G // H]
            x = q[first:first + n, h].double()
            score = scale * (x @ k.T)
            off = (D + 8) * U * abs(scale) * (x.abs() @ k.abs().T)
            if cap:
                score = cap * torch.tanh(score / cap)
                off = off + 2.0 ** -19 * cap
            if slopes is not None:
                score = score - float(slopes[h]) * away
                off = off + (D + 8) * U * float(slopes[h]) * away
            score = score.masked_fill(~seen, -math.inf)
            top = score.amax(1, keepdim=True)
            weight = (score - torch.where(top == -math.inf, torch.zeros_like(top), top)).exp().masked_fill(~seen, 0.0)
            total = weight.sum(1, keepdim=True)
            p = weight / torch.where(total == 0, torch.ones_like(total), total)
            # what a row does not see is left out, not multiplied with 0
            keep = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
            y, size = p @ keep, p @ keep.abs()
            bad = (~torch.isfinite(v)).any(1)
            for j in bad.nonzero().flatten().tolist():
                hurt = seen[:, j:j + 1] & ~torch.isfinite(v[j])
                y = torch.where(hurt, y + p[:, j:j + 1] * v[j], y)
            y = torch.where(total == 0, torch.zeros_like(y), y)
            e = off.masked_fill(~seen, 0.0).nan_to_num(0.0, 0.0, 0.0).amax(1, keepdim=True)
            out[first:first + n, h] = y
            slack[first:first + n, h] = size * (unit + 2 * e + (2 * length + 8) * U) + U * keep.abs().sum(0)
    return out, slack


def check(name, got, want, slack):
    """|got - want| <= slack + half a unit, wherever want is not NaN for being no sequence's (slack NaN); NaN and infinities alike."""
    unit, got = UNIT[got.dtype], got.detach().cpu().double()
    assert got.shape == want.shape
    told = ~torch.isnan(slack)
    got, want, slack = got[told], want[told], slack[told]
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{name}: NaN in other places"
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), name
    # one rounding, of the value with its slack; below binary16's normal range in steps of 2^-24
    room = slack * (1 + unit) + unit * want.abs() + 2.0 ** -25
    over = ((got - want).abs() - room)[fine]
    if over.numel() and float(over.max()) > 0:
        at = int(over.argmax())
        raise AssertionError(f"{name}: {got[fine][at]} for {want[fine][at]}, {room[fine][at]:.3g} allowed; {int((over > 0).sum())} of {over.numel()} over")


def rotate(x, positions, frequencies, interleaved):
    """x [T, heads, D] and how far a turned channel may be off: the angle's fraction of a turn and its functions in binary32."""
    x = x.double()
    off = torch.zeros_like(x)
    if frequencies is None:
        return x, off
    angle = positions.double()[:, None] * frequencies.double()
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    R = 2 * frequencies.numel()
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    u, w, size = a * cos - b * sin, b * cos + a * sin, (a.abs() + b.abs()) * 2.0 ** -21
    y = x.clone()
    if interleaved:
        y[..., 0:R:2], y[..., 1:R:2], off[..., 0:R:2], off[..., 1:R:2] = u, w, size, size
    else:
        y[..., :R // 2], y[..., R // 2:R], off[..., :R // 2], off[..., R // 2:R] = u, w, size, size
    return y, off
