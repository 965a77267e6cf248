"""The operators of pwlq_block.h from their formulas, in binary64 on the CPU, and what a result may be off.

A sum of n terms that the kernels form in binary32 in chains of at most n/32 additions, joined by a tree of at most 16
levels, is off by at most (n/32 + 16) u times the sum of the terms' magnitudes, u = 2^-24; each function returns that sum
of magnitudes beside the value.  A result stored in bfloat16 or binary16 is rounded once more, by half a unit in its last place.
"""
import torch

U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def chain(n):
    return (n / 32 + 16) * U


def wide(x, step=None):
    x = x.detach().cpu().double()
    return x if step is None else x * step.cpu().double()[:, None]


def check(name, got, want, slack):
    """|got - want| <= slack + half a unit of got's type, everywhere; NaN and infinities in the same places."""
    unit = UNIT[got.dtype]
    got = wide(got) if got.dim() != 1 else got.cpu().double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{name}: NaN in other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), name
    least = 2.0 ** -24 if unit == UNIT[torch.float16] else 2.0 ** -126     # what underflows
    room = torch.as_tensor(slack).expand_as(want) + unit * want.abs() + least
    over = ((got - want).abs() - room)[fine]
    if over.numel() and float(over.max()) > 0:
        at = int(over.argmax())
        raise AssertionError(f"{name}: {got[fine][at]} for {want[fine][at]}, {(got - want).abs()[fine][at]:.3g} off, "
                             f"{room[fine][at]:.3g} allowed; {int((over > 0).sum())} of {over.numel()} over")


def pack(x):
    """Codes and steps, in the binary32 arithmetic that defines them."""
    x = x.detach().cpu().float()
    bits = x.abs().view(torch.int32).amax(1)
    a = bits.view(torch.float32)
    bad, small = bits >= 0x7f800000, a < 2.0 ** -100
    one = torch.ones_like(a)
    factor = torch.where(bad | small, 0 * one, torch.full_like(a, 127.0) / torch.where(small | bad, one, a))
    step = torch.where(small, 0 * one, torch.where(bad, one * float("nan"), a / torch.full_like(a, 127.0)))
    codes = torch.where((bad | small)[:, None], torch.zeros_like(x), torch.round(x * factor[:, None]))
    return codes.to(torch.int8), step


def norm(x, w, eps):
    return x * w / (x.square().mean(1, keepdim=True) + eps).sqrt()


def gate_rows(gate, T):
    return gate.repeat_interleave(T // gate.shape[0], 0) if gate.shape[0] else gate


def norm_block(x, f, pre, post, gate, alpha, eps):
    """x_out, u and the slack of each: the norms' factors are off by chain(D), every product and sum by u."""
    x, pre = wide(x), pre.cpu().double()
    D = x.shape[1]
    mag = x.abs()
    if f is not None:
        v = wide(f)
        if post is not None:
            v = norm(v, post.cpu().double(), eps)
        if gate is not None:
            v = v * gate_rows(wide(gate), x.shape[0])
        x = x + alpha * v
        mag = mag + (alpha * v).abs()
    slack_x = (chain(D) + 8 * U) * mag
    b = 1 / (x.square().mean(1, keepdim=True) + eps).sqrt()
    # an error of x_out reaches u itself, and through b by at most as much of the row's mean
    row = (slack_x.square().mean(1, keepdim=True)).sqrt() * b
    u = x * b * pre
    slack_u = (slack_x * b + x.abs() * b * row) * pre.abs() + (chain(D) + 8 * U) * u.abs()
    return x, u, slack_x, slack_u


def norm_backward(du, dxo, x, f, pre, post, gate, alpha, eps):
    """The gradients by their formulas, and slacks from the magnitudes of what they sum."""
    T, D = x.shape
    pre = pre.cpu().double()
    zero = torch.zeros(T, D, dtype=torch.float64)
    dx, out, slack = (dxo if dxo is not None else zero).clone(), {}, {}
    mag = dx.abs()
    d_pre = torch.zeros(D, dtype=torch.float64)
    s_pre = d_pre.clone()
    if du is not None:
        b = 1 / (x.square().mean(1, keepdim=True) + eps).sqrt()
        xh, wdu = x * b, du * pre
        dx = dx + b * (wdu - xh * (wdu * xh).mean(1, keepdim=True))
        mag = mag + b * (wdu.abs() + xh.abs() * (wdu * xh).abs().mean(1, keepdim=True))
        d_pre, s_pre = (du * xh).sum(0), (du * xh).abs().sum(0)
    c = 4 * chain(D) + 16 * U
    out["dx"], slack["dx"] = dx, c * mag
    out["d_pre"], slack["d_pre"] = d_pre, (chain(T) + c) * s_pre
    if f is not None:
        a = torch.ones(T, 1, dtype=torch.float64) if post is None else 1 / (f.square().mean(1, keepdim=True) + eps).sqrt()
        fh, p = f * a, torch.ones(D, dtype=torch.float64) if post is None else post.cpu().double()
        g = torch.ones(T, D, dtype=torch.float64) if gate is None else gate_rows(wide(gate), T)
        dv, mv = alpha * g * dx, abs(alpha) * g.abs() * mag
        if gate is not None:
            G = gate.shape[0]
            out["d_gate"] = (alpha * dx * fh * p).view(G, T // G, D).sum(1)
            slack["d_gate"] = (chain(T // G) + 2 * c) * (abs(alpha) * mag * (fh * p).abs()).view(G, T // G, D).sum(1)
        if post is None:
            out["df"], slack["df"] = dv, 2 * c * mv
        else:
            out["d_post"], slack["d_post"] = (dv * fh).sum(0), (chain(T) + 2 * c) * (mv * fh.abs()).sum(0)
            w = dv * p
            out["df"] = a * (w - fh * (w * fh).mean(1, keepdim=True))
            slack["df"] = 3 * c * a * (mv * p.abs() + fh.abs() * (mv * (p * fh).abs()).mean(1, keepdim=True))
    return out, slack


def first(x, w, ids, scale):
    """H and its sums of magnitudes."""
    T, R = x.shape[0], w.shape[1]
    h = torch.zeros(T, R, dtype=torch.float64)
    m = h.clone()
    for t in range(T):
        a = int(ids[t])
        if 0 <= a < w.shape[0]:
            h[t] = float(scale[a]) * (w[a] @ x[t])
            m[t] = abs(float(scale[a])) * (w[a].abs() @ x[t].abs())
    return h, m


def second(h, hm, w, ids, base):
    y, m = base.clone(), base.abs()
    for t in range(h.shape[0]):
        a = int(ids[t])
        if 0 <= a < w.shape[0]:
            y[t] += h[t] @ w[a]
            m[t] += hm[t] @ w[a].abs()
    return y, m


def outer(h, hm, x, ids, n):
    g = torch.zeros(n, h.shape[1], x.shape[1], dtype=torch.float64)
    m = g.clone()
    for a in range(n):
        mine = (ids == a).nonzero().flatten()
        g[a], m[a] = h[mine].t() @ x[mine], hm[mine].t() @ x[mine].abs()
    return g, m
