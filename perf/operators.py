"""Timed cases of the operators around an inner product with packed weights in a transformer block.

Rows of activations are packed to 8 bits with a step each, as the integer product takes them and as a training
program keeps them for its backward pass; the norms before and after a block come with its gate and residual
scale, forward and backward; low-rank adapters of many requests stand beside a shared projection, in serving
and in training.  With `own` false `run` computes them by elementary torch operations in 32 bits, otherwise by
the framework's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1}
_EPS = 1e-6


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _pack(name, T, K, dtype):
    return dict(name=name, kind="pack", T=T, K=K, dtype=dtype)


def _norm(name, T, D, dtype, residual, gates=0, post=True, packed=False, backward=False):
    """`gates`: rows of the gate (0: none); `packed`: a forward pass emits its output in 8 bits, a backward
    pass reads the block's output and the residual from 8-bit checkpoints."""
    return dict(name=name, kind="norm", T=T, D=D, dtype=dtype, residual=residual, gates=gates, post=post,
                packed=packed, backward=backward)


def _adapter(name, T, K, N, R, adapters, dtype, order="runs", packed=True, base="f32", out="bf16", backward=False):
    """`order`: tokens of a request side by side ("runs"), or a token of each in turn ("mixed")."""
    return dict(name=name, kind="adapter", T=T, K=K, N=N, R=R, adapters=adapters, dtype=dtype, order=order,
                packed=packed, base=base, out=out, backward=backward)


def listed():
    return [
        # the activations of one small layer, of no round size, checkpointed and read back in binary32
        _pack("pack_ragged_layer", 515, 1155, "f32"),
        # the input of a transformer block's last projection for a prompt, kept for the backward pass
        _pack("pack_prompt", 4096, 11008, "bf16"),
        # between two blocks while a batch of eight decodes: norm, residual, norm, 8-bit activations
        _norm("norm_decode", 8, 4096, "bf16", "bf16", packed=True),
        # the same for a prompt, with a gate per channel and the residual stream in binary32
        _norm("norm_prompt", 4096, 4096, "bf16", "f32", gates=1, packed=True),
        # a training step's backward pass from 8-bit checkpoints
        _norm("norm_backward", 4096, 4096, "bf16", "bf16", gates=1, packed=True, backward=True),
        # a width of no vector size, a gate for each of five sequences, all in binary32
        _norm("norm_backward_ragged", 515, 1155, "f32", "f32", gates=5, backward=True),
        # one request, one token
        _adapter("adapter_one_token", 1, 4096, 4096, 16, 8, "bf16"),
        # decoding of eight requests, each with an adapter of its own, beside an 11008-wide projection
        _adapter("adapter_decode", 8, 4096, 11008, 16, 32, "bf16", order="mixed"),
        # prompts of several requests in one batch
        _adapter("adapter_prompts", 4096, 4096, 4096, 16, 8, "bf16"),
        # a classifier head: odd rank, half precision, activations not packed, binary32 output
        _adapter("adapter_head", 250, 2048, 1000, 5, 3, "f16", packed=False, out="f32"),
        # a training step of four adapters at once, from 8-bit checkpoints
        _adapter("adapter_backward", 4096, 4096, 11008, 16, 4, "bf16", base="bf16", backward=True),
        # one adapter of high rank
        _adapter("adapter_backward_wide", 2048, 4096, 4096, 64, 1, "bf16", base="f32", out="f32", backward=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("pack", "norm", "norm", "adapter", "adapter", "adapter"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if kind == "pack":
        K = _log(rng, 16, 11008)
        return dict(kind=kind, T=_log(rng, 1, min(16384, 20_000_000 // K)), K=K, dtype=dtype)
    if kind == "norm":
        D = _log(rng, 64, 8192)
        T = _log(rng, 1, min(8192, 8_000_000 // D))
        gates = rng.choice((0, 1, 1, T, next(g for g in range(min(T, 6), 0, -1) if T % g == 0)))
        # binary32 outputs show a code that a sum's order put on the other side of a tie: packed in 16 bits only
        backward = rng.random() < 0.5
        return dict(kind=kind, T=T, D=D, dtype=dtype, residual=rng.choice((dtype, "f32")), gates=gates,
                    post=rng.random() < 0.7, packed=rng.random() < 0.5 and (backward or dtype != "f32"), backward=backward)
    K, N, R = _log(rng, 64, 11008), _log(rng, 64, 11008), _log(rng, 1, 64)
    T = _log(rng, 1, min(4096, 26_000_000 // (K + N), 1_000_000_000 // (R * (K + N))))
    return dict(kind=kind, T=T, K=K, N=N, R=R, adapters=_log(rng, 1, 32), dtype=dtype,
                order=rng.choice(("runs", "mixed")), packed=rng.random() < 0.7, base=rng.choice(("f32", dtype)),
                out=rng.choice(("f32", dtype)), backward=rng.random() < 0.4)


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _pack_plain(x):
    """Codes and step of each row: rne(x * (127 / absmax)), absmax / 127."""
    x = x.float()
    a = x.abs().amax(1, keepdim=True)
    most = torch.full_like(a, 127.0)
    codes = torch.round(x * torch.where(a > 0, most / a, torch.zeros_like(a)))
    return codes.to(torch.int8), (a / most).squeeze(1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale)

    def activations(rows, cols):
        """Bell-shaped, with a size of its own for each channel and a few channels that stand out."""
        size = torch.randn((cols,), generator=gen, device="cuda").mul_(0.4).exp_()
        size[torch.rand((cols,), generator=gen, device="cuda") < 0.003] *= 8.0
        return normal(rows, cols).mul_(size)

    T, dtype = case["T"], _TYPES[case["dtype"]]
    if case["kind"] == "pack":
        return dict(kind="pack", x=activations(T, case["K"]).to(dtype))
    if case["kind"] == "norm":
        D, G, stream = case["D"], case["gates"], _TYPES[case["residual"]]
        s = dict(kind="norm", backward=case["backward"], packed=case["packed"], dtype=dtype, stream=stream, alpha=0.5,
                 pre=1.0 + normal(D, scale=0.1), post=1.0 + normal(D, scale=0.1) if case["post"] else None,
                 gate=(0.7 + normal(G, D, scale=0.3)).to(dtype) if G else None,
                 x=activations(T, D).to(stream), f=normal(T, D, scale=0.3).to(dtype), x_step=None, f_step=None)
        if case["backward"]:
            s["du"], s["dx_out"] = normal(T, D, scale=1e-2).to(dtype), normal(T, D, scale=1e-2).to(stream)
            if case["packed"]:
                s["x"], s["x_step"] = _pack_plain(s["x"])
                s["f"], s["f_step"] = _pack_plain(s["f"])
        return s
    K, N, R, n = case["K"], case["N"], case["R"], case["adapters"]
    s = dict(kind="adapter", backward=case["backward"], dtype=dtype, out=_TYPES[case["out"]],
             down=normal(n, R, K, scale=K ** -0.5).to(dtype), up=normal(n, R, N, scale=0.05).to(dtype),
             scale=1.0 + torch.rand((n,), generator=gen, device="cuda"), x_step=None, base_step=None)
    # requests of one to many tokens, one in eight without an adapter
    of = torch.randint(0, n, (T,), generator=gen, device="cuda", dtype=torch.int32)
    if T > 1:
        of[torch.rand((T,), generator=gen, device="cuda") < 0.125] = -1
    if case["order"] == "runs":
        first = torch.rand((T,), generator=gen, device="cuda") < 2.0 * n / T
        of = of[first.cumsum(0).clamp_(max=T - 1)]
    s["ids"] = of.contiguous()
    s["x"] = activations(T, K).to(dtype)
    if case["packed"]:
        s["x"], s["x_step"] = _pack_plain(s["x"])
    if case["backward"]:
        s["dy"] = normal(T, N, scale=1e-2).to(dtype)
        s["dx_base"] = normal(T, K, scale=1e-2).to(_TYPES[case["base"]])
        s["h"] = _first_product(s["x"], s["x_step"], s["down"], s["ids"], s["scale"])[0]
    else:
        # the integer product of packed activations has each row in units of its step
        s["base_step"] = s["x_step"]
        s["base"] = (normal(T, N) / s["base_step"][:, None] if case["packed"] else normal(T, N)).to(_TYPES[case["base"]])
    return s


# --------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------
def _wide(x, step):
    x = x.float()
    return x if step is None else x * step[:, None]


def _norm_plain(s):
    f, v = s["f"].float(), s["f"].float()
    if s["post"] is not None:
        v = f * torch.rsqrt(f.square().mean(1, keepdim=True) + _EPS) * s["post"]
    if s["gate"] is not None:
        v = v * s["gate"].float().repeat_interleave(v.shape[0] // s["gate"].shape[0], 0)
    x = s["x"].float() + s["alpha"] * v
    u = x * torch.rsqrt(x.square().mean(1, keepdim=True) + _EPS) * s["pre"]
    if s["packed"]:
        u = _wide(*_pack_plain(u))
    return x.to(s["stream"]), u.to(s["dtype"])


def _norm_backward_plain(s):
    x, f, du = _wide(s["x"], s["x_step"]), _wide(s["f"], s["f_step"]), s["du"].float()
    T, D = x.shape
    b = torch.rsqrt(x.square().mean(1, keepdim=True) + _EPS)
    xh, wdu = x * b, du * s["pre"]
    dx = s["dx_out"].float() + b * (wdu - xh * (wdu * xh).mean(1, keepdim=True))
    out = dict(dx=dx.to(s["stream"]), d_pre=(du * xh).sum(0))
    fh = f
    if s["post"] is not None:
        a = torch.rsqrt(f.square().mean(1, keepdim=True) + _EPS)
        fh = f * a
    dv = s["alpha"] * dx
    if s["gate"] is not None:
        G = s["gate"].shape[0]
        v = fh if s["post"] is None else fh * s["post"]
        out["d_gate"] = (dv * v).view(G, T // G, D).sum(1)
        dv = dv * s["gate"].float().repeat_interleave(T // G, 0)
    if s["post"] is None:
        out["df"] = dv.to(s["dtype"])
    else:
        out["d_post"] = (dv * fh).sum(0)
        wdv = dv * s["post"]
        out["df"] = (a * (wdv - fh * (wdv * fh).mean(1, keepdim=True))).to(s["dtype"])
    return out


def _first_product(x, step, weight, ids, scale):
    """[T, R] of each row with its own adapter's [R, K], and the same spread over all adapters, [T, n R]:
    one product with the adapters side by side, of which a row keeps its own."""
    n, R, K = weight.shape
    mine = ids[:, None] == torch.arange(n, device=ids.device, dtype=ids.dtype)
    all_of = _wide(x, step) @ weight.view(n * R, K).float().t()
    spread = all_of.view(-1, n, R) * torch.where(mine, scale, torch.zeros_like(scale))[:, :, None]
    return spread.sum(1), spread.view(-1, n * R)


def _adapter_plain(s):
    h, spread = _first_product(s["x"], s["x_step"], s["down"], s["ids"], s["scale"])
    n, R, N = s["up"].shape
    return (_wide(s["base"], s["base_step"]) + spread @ s["up"].view(n * R, N).float()).to(s["out"]), h


def _adapter_backward_plain(s):
    n, R, N = s["up"].shape
    K = s["down"].shape[2]
    dy, x = s["dy"].float(), _wide(s["x"], s["x_step"])
    _, spread = _first_product(dy, None, s["up"], s["ids"], s["scale"])
    dx = s["dx_base"].float() + spread @ s["down"].view(n * R, K).float()
    mine = s["ids"][:, None] == torch.arange(n, device=dy.device, dtype=s["ids"].dtype)
    h = torch.where(mine[:, :, None], s["h"][:, None, :], torch.zeros_like(s["scale"])[None, :, None]).reshape(-1, n * R)
    return dict(d_down=(spread.t() @ x).view(n, R, K), d_up=(h.t() @ dy).view(n, R, N), dx=dx.to(s["dx_base"].dtype))


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    s = state
    if own:
        from paper_2002_00104_amd import block
        if s["kind"] == "pack":
            codes, step = block.pack_rows(s["x"])
            return block.unpack_rows(codes, step, s["x"].dtype), step
        if s["kind"] == "norm" and s["backward"]:
            got = block.norm_block_backward(s["du"], s["dx_out"], s["x"], s["f"], post_weight=s["post"], pre_weight=s["pre"],
                                            gate=s["gate"], alpha=s["alpha"], eps=_EPS, x_step=s["x_step"], f_step=s["f_step"])
            return {k: v for k, v in got.items() if v is not None}
        if s["kind"] == "norm":
            got = block.norm_block(s["x"], s["f"], post_weight=s["post"], pre_weight=s["pre"], gate=s["gate"],
                                   alpha=s["alpha"], eps=_EPS, pack=s["packed"])
            return (got[0], block.unpack_rows(got[1], got[2], s["dtype"])) if s["packed"] else got
        if s["backward"]:
            return block.adapter_backward(s["dy"], s["x"], s["down"], s["up"], s["ids"], s["scale"], s["h"],
                                          x_step=s["x_step"], dx_base=s["dx_base"])
        return block.adapter(s["x"], s["down"], s["up"], s["ids"], s["scale"], base=s["base"], x_step=s["x_step"],
                             base_step=s["base_step"], dtype=s["out"])
    if s["kind"] == "pack":
        codes, step = _pack_plain(s["x"])
        return _wide(codes, step).to(s["x"].dtype), step
    if s["kind"] == "norm":
        return _norm_backward_plain(s) if s["backward"] else _norm_plain(s)
    return _adapter_backward_plain(s) if s["backward"] else _adapter_plain(s)


def work(case):
    T, e = case["T"], _SIZE[case["dtype"]]
    if case["kind"] == "pack":                  # x in; codes out and in again; the values out
        n = T * case["K"]
        return {"bytes": n * (2 * e + 2) + 12 * T, "flops": 5 * n}
    if case["kind"] == "norm":
        D, r = case["D"], _SIZE[case["residual"]]
        gate, weights = case["gates"] * D * e, 4 * D * (1 + case["post"])
        if case["backward"]:                    # du, dx_out, x, f in; dx, df and the parameters' gradients out
            kept = 2 if case["packed"] else e + r
            return {"bytes": T * D * (2 * e + 2 * r + kept) + gate + 2 * weights + 4 * case["gates"] * D, "flops": 25 * T * D}
        # f, x in; x, u out (in 8 bits: out, in again, and the values)
        return {"bytes": T * D * (e + 2 * r + (2 + e if case["packed"] else e)) + gate + weights, "flops": 12 * T * D}
    K, N, R = case["K"], case["N"], case["R"]
    used = min(case["adapters"], T)             # at most so many adapters have a token
    weights, x = used * R * (K + N), T * K * (1 if case["packed"] else e)
    if case["backward"]:                        # x, dy, h, dx_base in; dx and the adapters' gradients out
        return {"bytes": x + T * N * e + 4 * T * R + 2 * T * K * _SIZE[case["base"]] + weights * e +
                4 * case["adapters"] * R * (K + N), "flops": 4 * T * R * (K + N)}
    return {"bytes": x + weights * e + T * N * (_SIZE[case["base"]] + _SIZE[case["out"]]) + 4 * T * R,
            "flops": 2 * T * R * (K + N)}


# --------------------------------------------------------------------------
# the definitions in binary64
# --------------------------------------------------------------------------
def _pack_exact(x):
    a = x.abs().max(dim=1).values
    step = a / 127.0
    return (x / torch.where(a > 0, step, torch.ones_like(step))[:, None]).round() * step[:, None], step


def _rms_norm(x, weight):
    return x / (x.pow(2).sum(1, keepdim=True) / x.shape[1] + _EPS).sqrt() * weight


def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() if isinstance(v, torch.Tensor) and k != "ids" else v for k, v in s.items()}
    if s["kind"] == "pack":
        return _pack_exact(d["x"])
    for name in ("x", "f", "base"):
        if d.get(name + "_step") is not None:
            d[name] = d[name] * d[name + "_step"].unsqueeze(1)
    if s["kind"] == "norm":
        with torch.enable_grad():
            leaves = {k: d[k].requires_grad_() for k in ("x", "f", "pre", "post", "gate") if d[k] is not None}
            v = d["f"] if d["post"] is None else _rms_norm(d["f"], d["post"])
            if d["gate"] is not None:
                rows = torch.arange(v.shape[0], device=v.device) // (v.shape[0] // d["gate"].shape[0])
                v = v * d["gate"][rows]
            v = d["alpha"] * v
            if not s["backward"]:
                x = d["x"] + v
                u = _rms_norm(x, d["pre"]).detach()
                return x.detach(), _pack_exact(u)[0] if s["packed"] else u
            # the residual given is the one after the sum: its gradient is the sum's
            (_rms_norm(d["x"], d["pre"]) * d["du"]).sum().backward()
            dx = d["x"].grad + d["dx_out"]
            (v * dx).sum().backward()
        names = dict(f="df", pre="d_pre", post="d_post", gate="d_gate")
        return dict({names[k]: t.grad for k, t in leaves.items() if k != "x"}, dx=dx)
    n = s["down"].shape[0]
    rows = [(s["ids"] == a).nonzero().flatten() for a in range(n)]
    if not s["backward"]:
        y, h = d["base"].clone(), torch.zeros_like(d["x"][:, :1]).repeat(1, s["down"].shape[1])
        for a in range(n):
            h[rows[a]] = d["scale"][a] * d["x"][rows[a]] @ d["down"][a].t()
            y[rows[a]] += h[rows[a]] @ d["up"][a]
        return y, h
    dx, d_down, d_up = d["dx_base"].clone(), torch.zeros_like(d["down"]), torch.zeros_like(d["up"])
    for a in range(n):
        dh = d["scale"][a] * d["dy"][rows[a]] @ d["up"][a].t()
        dx[rows[a]] += dh @ d["down"][a]
        d_down[a], d_up[a] = dh.t() @ d["x"][rows[a]], d["h"][rows[a]].t() @ d["dy"][rows[a]]
    return dict(d_down=d_down, d_up=d_up, dx=dx)
