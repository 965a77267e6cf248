"""The operators of pwlq_block.h against their formulas in binary64: packed rows, the norms around a block, adapters, and the
gradients.  The slacks are derived in block_ref.py."""
import math
import zlib

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_2002_00104_amd import block
    return block


def gen(*key):
    g = torch.Generator()
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def normal(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def spread(t, how):
    """The same values on the GPU: as they are, as columns of a wider matrix, or off the alignment of vectors."""
    t = t.cuda()
    if how == "whole":
        return t
    pad = 8 if how == "columns" else 3
    wide = torch.full((t.shape[0], t.shape[1] + 2 * pad), float("nan") if t.is_floating_point() else 77, dtype=t.dtype, device="cuda")
    wide[:, pad:pad + t.shape[1]] = t
    return wide[:, pad:pad + t.shape[1]]


# --------------------------------------------------------------------------
# packed rows
# --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,K", [(1, 1), (1, 4096), (3, 7), (5, 8), (64, 576), (33, 1155), (2, 513), (2, 16384), (3, 16385), (2, 65536)])
@pytest.mark.parametrize("how", ["whole", "columns", "odd"])
def test_pack_and_unpack(B, dtype, T, K, how):
    print(f"[case] pack {dtype} {T}x{K} {how}", flush=True)
    x = normal(gen(T, K), T, K, dtype=dtype, scale=3.0)
    codes, step = B.pack_rows(spread(x, how))
    want = ref.pack(x)
    assert torch.equal(codes.cpu(), want[0]) and torch.equal(step.cpu(), want[1])
    for out in (F32, BF16, F16):
        y = B.unpack_rows(codes, step, out)
        assert torch.equal(y.cpu(), (want[0].float() * want[1][:, None]).to(out))


def test_pack_odd_rows(B):
    """Rows of zeros, of one value, with NaN or an infinity, tiny and huge ones, and ties to even."""
    inf, nan = math.inf, math.nan
    rows = [[0.0] * 9, [-0.0] * 9, [5.0] + [0.0] * 8, [nan] + [1.0] * 8, [1.0] * 8 + [-inf], [nan, inf] + [0.0] * 7,
            [2.0 ** -101] * 9, [2.0 ** -100] * 9, [2.0 ** -140] * 9, [3.0e38, -3.0e38, 1.0] + [0.0] * 6,
            [127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5, -126.5]]
    x = torch.tensor(rows)
    codes, step = B.pack_rows(x.cuda())
    want = ref.pack(x)
    assert torch.equal(codes.cpu(), want[0])
    assert torch.equal(torch.isnan(step.cpu()), torch.isnan(want[1]))
    fine = ~torch.isnan(want[1])
    assert torch.equal(step.cpu()[fine], want[1][fine])
    assert codes.cpu()[-1].tolist() == [127, 0, 2, 2, 0, -2, -2, 126, -126]
    assert torch.isnan(B.unpack_rows(codes, step)[3:6]).all()


# --------------------------------------------------------------------------
# norms
# --------------------------------------------------------------------------
NORM_SHAPES = [(1, 1), (1, 4096), (7, 8), (6, 577), (130, 72), (12, 1155), (4, 8192), (2, 8200), (2, 16384), (600, 64)]
TYPES = [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]


def gates(T):
    return sorted({0, 1, T} | {g for g in (2, 3, 5) if T % g == 0})


def norm_inputs(T, D, dtype, stream, post, G, key):
    g = gen("norm", T, D, G, key)
    return dict(x=normal(g, T, D, dtype=stream, scale=2.0), f=normal(g, T, D, dtype=dtype, scale=0.5),
                pre=1 + normal(g, D, scale=0.2), post=1 + normal(g, D, scale=0.2) if post else None,
                gate=normal(g, G, D, dtype=dtype) if G else None, alpha=0.75, eps=1e-5)


def cuda(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("T,D", NORM_SHAPES)
@pytest.mark.parametrize("post", [True, False])
def test_norm_block(B, dtype, stream, T, D, post):
    for G in gates(T):
        for how in ("whole", "columns", "odd")[:3 if G == 1 else 1]:
            print(f"[case] norm {dtype} {stream} {T}x{D} post={post} G={G} {how}", flush=True)
            s = norm_inputs(T, D, dtype, stream, post, G, 0)
            x, u, sx, su = ref.norm_block(**s)
            kw = dict(pre_weight=s["pre"].cuda(), post_weight=cuda(s["post"]), gate=cuda(s["gate"]), alpha=s["alpha"], eps=s["eps"])
            got = B.norm_block(spread(s["x"], how), spread(s["f"], how), **kw)
            assert got[0].dtype == stream and got[1].dtype == dtype
            ref.check("x_out", got[0], x, sx)
            ref.check("u", got[1], u, su)
            xo, codes, step = B.norm_block(spread(s["x"], how), spread(s["f"], how), pack=True, **kw)
            assert torch.equal(xo, got[0])
            most = u.abs().amax(1)
            ref.check("step", step, most / 127, su.amax(1) / 127 + 2 * ref.U * most)
            # a code is at most half a step off, and what u is off
            off = (ref.wide(codes, step) - u).abs()
            assert (off <= 0.5001 * step.cpu().double()[:, None] + su + 1e-30).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,D", [(1, 8), (9, 577), (3, 4096)])
def test_norm_alone(B, dtype, T, D):
    g = gen(T, D)
    x, pre = normal(g, T, D, dtype=dtype), 1 + normal(g, D, scale=0.2)
    _, u, _, su = ref.norm_block(x, None, pre, None, None, 1.0, 1e-6)
    xd = x.cuda()
    got = B.norm_block(xd, pre_weight=pre.cuda())
    assert got[0] is xd
    ref.check("u", got[1], u, su)
    du = normal(g, T, D, dtype=dtype)
    out, slack = ref.norm_backward(ref.wide(du), None, ref.wide(x), None, pre, None, None, 1.0, 1e-6)
    got = B.norm_block_backward(du.cuda(), None, xd, pre_weight=pre.cuda())
    for k in out:
        ref.check(k, got[k], out[k], slack[k])
    assert got["df"] is None and got["d_post"] is None and got["d_gate"] is None


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("T,D", NORM_SHAPES)
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("kept", [True, False])
def test_norm_backward(B, dtype, stream, T, D, post, kept):
    for G in gates(T):
        for how in ("whole", "columns", "odd")[:3 if G == 1 else 1]:
            for left in ("", "du", "dx_out")[:3 if G == 0 else 1]:
                print(f"[case] norm backward {dtype} {stream} {T}x{D} post={post} kept={kept} G={G} {how} without {left}", flush=True)
                s = norm_inputs(T, D, dtype, stream, post, G, 1)
                g = gen("grad", T, D)
                du, dxo = normal(g, T, D, dtype=dtype), normal(g, T, D, dtype=stream)
                xs = fs = None
                x, f = s["x"], s["f"]
                if kept:
                    (x, xs), (f, fs) = ref.pack(x), ref.pack(f)
                if left == "du":
                    du = None
                if left == "dx_out":
                    dxo = None
                    if kept:
                        stream = dtype
                want, slack = ref.norm_backward(None if du is None else ref.wide(du), None if dxo is None else ref.wide(dxo),
                                                ref.wide(x, xs), ref.wide(f, fs), s["pre"], s["post"], s["gate"], s["alpha"], s["eps"])
                if left == "du" and kept and dtype != stream:
                    continue                               # df then has dx_out's type, and the gate too
                got = B.norm_block_backward(None if du is None else spread(du, how), None if dxo is None else spread(dxo, how),
                                            spread(x, how), spread(f, how), pre_weight=s["pre"].cuda(), post_weight=cuda(s["post"]),
                                            gate=cuda(s["gate"]), alpha=s["alpha"], eps=s["eps"], x_step=cuda(xs), f_step=cuda(fs))
                assert got["dx"].dtype == stream and got["df"].dtype == dtype
                assert {k for k, v in got.items() if v is not None} == set(want)
                for k in want:
                    ref.check(k, got[k], want[k], slack[k])


def test_norm_gradient_against_differences(B):
    """d(loss)/d(input) by central differences of the forward pass itself, in binary32."""
    T, D = 4, 40
    s = norm_inputs(T, D, F32, F32, True, 2, 5)
    g = gen("diff")
    cu, cx = normal(g, T, D), normal(g, T, D)

    def loss(**change):
        v = dict(s, **change)
        x, u, _, _ = ref.norm_block(**v)
        return float((x * cx).sum() + (u * cu).sum())

    xo, _ = B.norm_block(s["x"].cuda(), s["f"].cuda(), pre_weight=s["pre"].cuda(), post_weight=s["post"].cuda(), gate=s["gate"].cuda(),
                         alpha=s["alpha"], eps=s["eps"])
    got = B.norm_block_backward(cu.cuda(), cx.cuda(), xo, s["f"].cuda(), pre_weight=s["pre"].cuda(), post_weight=s["post"].cuda(),
                                gate=s["gate"].cuda(), alpha=s["alpha"], eps=s["eps"])
    for name, key in (("x", "dx"), ("f", "df"), ("pre", "d_pre"), ("post", "d_post"), ("gate", "d_gate")):
        direction = normal(g, *s[name].shape)
        e = 2.0 ** -12
        up, down = loss(**{name: s[name].double() + e * direction.double()}), loss(**{name: s[name].double() - e * direction.double()})
        numeric = (up - down) / (2 * e)
        analytic = float((got[key].cpu().double() * direction.double()).sum())
        size = float((got[key].cpu().double() * direction.double()).abs().sum())
        # the difference quotient is off by e^2/6 of a third derivative of order the sum's size
        assert abs(numeric - analytic) <= 1e-5 * size, (name, numeric, analytic)


def test_norm_rows_of_zeros_and_poison(B):
    """A row of zeros divides by sqrt(eps); a NaN or an infinity stays in its row."""
    T, D = 5, 96
    s = norm_inputs(T, D, BF16, BF16, True, 1, 6)
    s["x"][1] = 0
    s["f"][1] = 0
    s["x"][3, 7] = float("nan")
    s["f"][4, 2] = float("inf")
    x, u, sx, su = ref.norm_block(**s)
    kw = dict(pre_weight=s["pre"].cuda(), post_weight=s["post"].cuda(), gate=s["gate"].cuda(), alpha=s["alpha"], eps=s["eps"])
    xo, un = B.norm_block(s["x"].cuda(), s["f"].cuda(), **kw)
    for t in (0, 1, 2):
        ref.check("x_out", xo[t:t + 1], x[t:t + 1], sx[t:t + 1])
        ref.check("u", un[t:t + 1], u[t:t + 1], su[t:t + 1])
    assert (un[1] == 0).all() and torch.isnan(un[3]).all() and torch.isnan(un[4]).any()
    _, codes, step = B.norm_block(s["x"].cuda(), s["f"].cuda(), pack=True, **kw)
    assert torch.isnan(step[3:]).all() and (codes[3:] == 0).all() and step[1] == 0 and (codes[1] == 0).all()


# --------------------------------------------------------------------------
# adapters
# --------------------------------------------------------------------------
# rows, columns in, columns out, rank, adapters
ADAPTER_SHAPES = [(1, 4096, 512, 16, 3), (1, 1, 1, 1, 1), (8, 640, 1000, 16, 9), (16, 100, 72, 5, 2), (17, 100, 72, 5, 2), (33, 577, 131, 3, 4),
                  (70, 1096, 264, 16, 5), (129, 136, 1032, 40, 2), (40, 520, 136, 130, 3), (300, 64, 64, 8, 1), (95, 2112, 640, 64, 40)]
ORDERS = ["runs", "mixed", "none"]


def adapter_inputs(T, K, N, R, n, dtype, packed, order, key):
    g = gen("adapter", T, K, N, R, n, key)
    ids = torch.randint(0, n, (T,), generator=g, dtype=torch.int32)
    ids[torch.rand((T,), generator=g) < 0.2] = -1
    if T > 3:
        ids[1], ids[T - 1] = n, 1 << 30                   # beyond the last adapter: none either
    if order == "runs":
        ids = ids.sort().values
    if order == "none":
        ids[:] = -1
    x, step = normal(g, T, K, dtype=dtype, scale=2.0), None
    if packed:
        x, step = ref.pack(x)
    return dict(x=x, x_step=step, down=normal(g, n, R, K, dtype=dtype, scale=K ** -0.5), up=normal(g, n, R, N, dtype=dtype, scale=0.1),
                ids=ids, scale=normal(g, n).abs() + 0.5, base=normal(g, T, N))


@pytest.mark.parametrize("T,K,N,R,n", ADAPTER_SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("packed", [True, False])
def test_adapter(B, T, K, N, R, n, dtype, packed):
    for order, how, base, out in (("runs", "whole", F32, dtype), ("mixed", "columns", dtype, F32), ("none", "whole", F32, F32),
                                  ("mixed", "odd", F32, dtype), ("runs", "whole", None, dtype)):
        print(f"[case] adapter {T}x{K}x{N} R={R} n={n} {dtype} packed={packed} {order} {how} base={base} out={out}", flush=True)
        s = adapter_inputs(T, K, N, R, n, dtype, packed, order, 0)
        bt = None if base is None else s["base"].to(base)
        factor = s["x_step"] if packed and base is not None else None
        b64 = torch.zeros(T, N, dtype=torch.float64) if bt is None else ref.wide(bt, factor)
        x64 = ref.wide(s["x"], s["x_step"])
        h, hm = ref.first(x64, s["down"].double(), s["ids"], s["scale"])
        y, ym = ref.second(h, hm, s["up"].double(), s["ids"], b64)
        got, gh = B.adapter(spread(s["x"], how), s["down"].cuda(), s["up"].cuda(), s["ids"].cuda(), s["scale"].cuda(),
                            base=None if bt is None else spread(bt, how), x_step=cuda(s["x_step"]), base_step=cuda(factor), dtype=out)
        assert got.dtype == out and gh.dtype == F32
        ref.check("h", gh, h, (ref.chain(K) + 4 * ref.U) * hm)
        ref.check("out", got, y, (ref.chain(K) + ref.chain(R) + 8 * ref.U) * ym)


@pytest.mark.parametrize("T,K,N,R,n", ADAPTER_SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("packed", [True, False])
def test_adapter_backward(B, T, K, N, R, n, dtype, packed):
    for order, how, base in (("runs", "whole", F32), ("mixed", "columns", dtype), ("none", "whole", F32), ("mixed", "odd", None)):
        print(f"[case] adapter backward {T}x{K}x{N} R={R} n={n} {dtype} packed={packed} {order} {how} base={base}", flush=True)
        s = adapter_inputs(T, K, N, R, n, dtype, packed, order, 1)
        g = gen("dy", T, N)
        dy, h = normal(g, T, N, dtype=dtype, scale=0.5), normal(g, T, R)
        bt = None if base is None else normal(g, T, K, dtype=base)
        x64, dy64 = ref.wide(s["x"], s["x_step"]), ref.wide(dy)
        dh, dhm = ref.first(dy64, s["up"].double(), s["ids"], s["scale"])
        dx, dxm = ref.second(dh, dhm, s["down"].double(), s["ids"], torch.zeros(T, K, dtype=torch.float64) if bt is None else ref.wide(bt))
        d_down, ddm = ref.outer(dh, dhm, x64, s["ids"], n)
        d_up, dum = ref.outer(h.double(), h.double().abs(), dy64, s["ids"], n)
        got = B.adapter_backward(spread(dy, how), spread(s["x"], how), s["down"].cuda(), s["up"].cuda(), s["ids"].cuda(), s["scale"].cuda(),
                                 h.cuda(), x_step=cuda(s["x_step"]), dx_base=None if bt is None else spread(bt, how))
        assert got["dx"].dtype == (base or dtype) and got["d_down"].dtype == got["d_up"].dtype == F32
        ref.check("dx", got["dx"], dx, (ref.chain(N) + ref.chain(R) + 8 * ref.U) * dxm)
        ref.check("d_down", got["d_down"], d_down, (ref.chain(N) + ref.chain(T) + 8 * ref.U) * ddm)
        ref.check("d_up", got["d_up"], d_up, (ref.chain(T) + 4 * ref.U) * dum)


@pytest.mark.parametrize("T", [5, 40])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_an_adapter_s_infinities_stay_with_its_rows(B, T, dtype):
    """Rows without the poisoned adapter are bit for bit what they are beside a sound one; its own rows may be anything."""
    K, N, R, n = 96, 144, 6, 3
    s = adapter_inputs(T, K, N, R, n, dtype, False, "mixed", 2)
    g = gen("poison")
    dy, h = normal(g, T, N, dtype=dtype), normal(g, T, R)
    of = s["ids"]
    clean = ~(of == 1)

    def both(down, up, x, dyv):
        y, hh = B.adapter(x.cuda(), down.cuda(), up.cuda(), of.cuda(), s["scale"].cuda(), base=s["base"].cuda())
        return (y, hh), B.adapter_backward(dyv.cuda(), x.cuda(), down.cuda(), up.cuda(), of.cuda(), s["scale"].cuda(), h.cuda())

    (y0, h0), b0 = both(s["down"], s["up"], s["x"], dy)
    down, up, x, dyv = s["down"].clone(), s["up"].clone(), s["x"].clone(), dy.clone()
    down[1], up[1] = float("nan"), float("inf")
    x[~clean], dyv[~clean] = float("inf"), float("nan")
    (y1, h1), b1 = both(down, up, x, dyv)
    keep = clean.cuda()
    for a, b in ((y0, y1), (h0, h1), (b0["dx"], b1["dx"])):
        assert torch.equal(a[keep], b[keep])
    for name in ("d_down", "d_up"):
        for a in (0, 2):
            assert torch.equal(b0[name][a], b1[name][a]), name
    assert not torch.isfinite(y1[~keep]).any()


def test_adapter_gradients_against_differences(B):
    T, K, N, R, n = 40, 72, 56, 4, 3
    s = adapter_inputs(T, K, N, R, n, F32, False, "runs", 3)
    g = gen("adapter diff")
    c = normal(g, T, N)
    _, h = B.adapter(s["x"].cuda(), s["down"].cuda(), s["up"].cuda(), s["ids"].cuda(), s["scale"].cuda())
    got = B.adapter_backward(c.cuda(), s["x"].cuda(), s["down"].cuda(), s["up"].cuda(), s["ids"].cuda(), s["scale"].cuda(), h)

    def loss(**change):
        v = {k: (change[k] if k in change else s[k].double()) for k in ("x", "down", "up")}
        hh, hm = ref.first(v["x"], v["down"], s["ids"], s["scale"])
        return float((ref.second(hh, hm, v["up"], s["ids"], torch.zeros(T, N, dtype=torch.float64))[0] * c).sum())

    for name, key in (("x", "dx"), ("down", "d_down"), ("up", "d_up")):
        d = normal(g, *s[name].shape).double()
        e = 2.0 ** -10                                     # the loss is linear in each: no error of the quotient but rounding
        numeric = (loss(**{name: s[name].double() + e * d}) - loss(**{name: s[name].double() - e * d})) / (2 * e)
        prod = got[key].cpu().double() * d
        assert abs(numeric - float(prod.sum())) <= 4e-6 * float(prod.abs().sum()) + 1e-9, name


def test_results_repeat_and_other_streams_agree(B):
    """No result depends on timing: every gradient is the same bits again, on another stream too."""
    T, K, N, R, n = 700, 1024, 768, 16, 4
    s = adapter_inputs(T, K, N, R, n, BF16, True, "mixed", 4)
    g = gen("repeat")
    dy = normal(g, T, N, dtype=BF16).cuda()
    args = [s["x"].cuda(), s["down"].cuda(), s["up"].cuda(), s["ids"].cuda(), s["scale"].cuda()]
    step = s["x_step"].cuda()
    nb = norm_inputs(T, K, BF16, BF16, True, 1, 9)
    du, dxo = normal(g, T, K, dtype=BF16).cuda(), normal(g, T, K, dtype=BF16).cuda()
    nx, nf, kw = nb["x"].cuda(), nb["f"].cuda(), dict(pre_weight=nb["pre"].cuda(), post_weight=nb["post"].cuda(), gate=nb["gate"].cuda())

    def all_of():
        y, h = B.adapter(*args, x_step=step)
        out = [y, h, *B.adapter_backward(dy, *args, h, x_step=step).values()]
        return out + list(B.norm_block(nx, nf, pack=True, **kw)) + list(B.norm_block_backward(du, dxo, nx, nf, **kw).values())

    one = [t.clone() for t in all_of()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        two = all_of()
    side.synchronize()
    for a, b, c in zip(one, two, all_of()):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_replay_from_a_graph(B):
    """The calls only launch kernels: recorded once, replayed on new contents, every replay against the eager result."""
    T, K, N, R, n = 96, 256, 384, 8, 3
    s = adapter_inputs(T, K, N, R, n, BF16, False, "runs", 7)
    g = gen("graph")
    x, dy = s["x"].cuda(), normal(g, T, N, dtype=BF16).cuda()
    args = [s["down"].cuda(), s["up"].cuda(), s["ids"].cuda(), s["scale"].cuda()]
    pre, post, gate = (1 + normal(g, K, scale=0.1)).cuda(), (1 + normal(g, K, scale=0.1)).cuda(), normal(g, 1, K, dtype=BF16).cuda()
    kw = dict(pre_weight=pre, post_weight=post, gate=gate)

    def step():
        xo, codes, st = B.norm_block(x, x, pack=True, **kw)
        y, h = B.adapter(codes, *args, x_step=st)
        back = B.adapter_backward(dy, codes, *args, h, x_step=st)
        nb = B.norm_block_backward(back["dx"], x, xo, x, **kw)
        return [xo, codes, st, y, h, *back.values(), *nb.values(), B.unpack_rows(*B.pack_rows(y), BF16)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    torch.cuda.synchronize()
    for rep in range(4):
        x.copy_(normal(g, T, K, dtype=BF16))
        dy.copy_(normal(g, T, N, dtype=BF16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), f"replay {rep}"
        torch.cuda.synchronize()


# --------------------------------------------------------------------------
# empty batches and refusals
# --------------------------------------------------------------------------
def test_empty_batches(B):
    K, N, R, n = 64, 40, 4, 2
    x = torch.empty(0, K, dtype=BF16, device="cuda")
    codes, step = B.pack_rows(x)
    assert codes.shape == (0, K) and B.unpack_rows(codes, step, BF16).shape == (0, K)
    w = torch.ones(K, device="cuda")
    assert B.norm_block(x, x, pre_weight=w)[1].shape == (0, K)
    got = B.norm_block_backward(x, x, x, x, pre_weight=w, post_weight=w, gate=torch.ones(2, K, dtype=BF16, device="cuda"))
    assert got["dx"].shape == (0, K)
    for k in ("d_pre", "d_post", "d_gate"):
        assert (got[k] == 0).all()
    down, up = torch.ones(n, R, K, dtype=BF16, device="cuda"), torch.ones(n, R, N, dtype=BF16, device="cuda")
    ids, scale = torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(n, device="cuda")
    y, h = B.adapter(x, down, up, ids, scale)
    assert y.shape == (0, N) and h.shape == (0, R)
    got = B.adapter_backward(y, x, down, up, ids, scale, h)
    assert (got["d_down"] == 0).all() and (got["d_up"] == 0).all() and got["dx"].shape == (0, K)


def test_what_is_refused(B):
    def f(*shape, dtype=BF16):
        return torch.ones(*shape, dtype=dtype, device="cuda")

    x, w = f(4, 64), f(64, dtype=F32)
    with pytest.raises(ValueError):
        B.pack_rows(x.cpu())
    with pytest.raises(ValueError):
        B.pack_rows(x.t())
    with pytest.raises(ValueError):
        B.pack_rows(x.to(torch.float64))
    with pytest.raises(ValueError):
        B.norm_block(x, f(4, 63), pre_weight=w)
    with pytest.raises(ValueError):
        B.norm_block(x, x, pre_weight=f(64))
    from paper_2002_00104_amd import pwlq
    with pytest.raises(pwlq.PwlqError):
        B.norm_block(x, x, pre_weight=w, gate=f(3, 64))            # 3 gate rows do not divide 4 rows
    with pytest.raises(pwlq.PwlqError):
        B.norm_block(x, pre_weight=w, post_weight=w)               # a post norm of nothing
    with pytest.raises(pwlq.PwlqError):
        B.norm_block(x, x.float(), pre_weight=w)                   # a residual narrower than the block's output
    with pytest.raises(pwlq.PwlqError):
        B.norm_block(f(1, 16392), f(1, 16392), pre_weight=f(16392, dtype=F32))
    with pytest.raises(pwlq.PwlqError):
        B.pack_rows(f(1, 65537))
    codes, step = B.pack_rows(x)
    down, up = f(2, 4, 64), f(2, 4, 48)
    ids, scale = torch.zeros(4, dtype=torch.int32, device="cuda"), f(2, dtype=F32)
    with pytest.raises(ValueError):
        B.adapter(codes, down, up, ids, scale)                     # codes without steps
    with pytest.raises(ValueError):
        B.adapter(x, down, up, ids.long(), scale)
    with pytest.raises(ValueError):
        B.adapter(x, down, up.half(), ids, scale)
    with pytest.raises(ValueError):
        B.adapter(x.half(), down, up, ids, scale)
    with pytest.raises(ValueError):
        B.adapter(x, down.transpose(0, 1), up, ids, scale)
    with pytest.raises(pwlq.PwlqError):
        B.adapter(x, f(2, 257, 64), f(2, 257, 48), ids, scale)
    with pytest.raises(pwlq.PwlqError):
        B.adapter(f(40, 1024), f(2, 4, 1024), up, torch.zeros(40, dtype=torch.int32, device="cuda"), scale,
                  workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        B.norm_block_backward(None, None, x, x, pre_weight=w)
    with pytest.raises(ValueError):
        B.norm_block_backward(x, x, codes, x, pre_weight=w, x_step=step)       # one checkpoint in 8 bits, the other not
    torch.cuda.synchronize()
