"""The operators of pwlq_block.h where adapters alternate over many rows, in place, and beyond 2^32 elements."""
import pytest
import torch

import block_ref as ref
from test_gpu_block import B, BF16, F16, F32, adapter_inputs, cuda, gen, norm_inputs, normal  # noqa: F401

pytestmark = pytest.mark.gpu

# rows, columns in, columns out, rank, adapters: on both sides of the rule by which rows are collected, T * n * sixteens of ranks >= 2048;
# rows of one adapter that fill no tile, one more than a span, as many adapters as rows and more
MANY = [(255, 136, 72, 16, 8), (256, 136, 72, 16, 8), (257, 200, 200, 3, 8), (513, 65, 129, 33, 3), (65, 264, 520, 100, 5),
        (300, 72, 1160, 17, 300), (770, 520, 40, 8, 1000),
        # few rows: in one launch or two, by the ranks, the columns and the rows
        (5, 264, 520, 64, 3), (5, 264, 520, 48, 3), (12, 4100, 600, 40, 4), (20, 5000, 700, 16, 4), (200, 600, 1400, 16, 6), (200, 600, 400, 16, 6)]


def ids_of(order, T, n, g):
    t = torch.arange(T)
    if order == "turn":                                  # one of each adapter after the other
        return t % n
    if order == "one":                                   # all rows of one, which is not the first
        return torch.full((T,), n - 1)
    if order == "ends":                                  # a span's first and last row apart from the others
        return torch.where((t % 256 == 0) | (t % 256 == 255), n // 2, -1)
    return torch.where(torch.rand((T,), generator=g) < 0.5, torch.randint(0, n, (T,), generator=g), 0)       # half of the rows the first's


@pytest.mark.parametrize("T,K,N,R,n", MANY)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("order", ["turn", "one", "ends", "half"])
def test_alternating_adapters(B, T, K, N, R, n, dtype, order):  # noqa: F811
    print(f"[case] alternating {T}x{K}x{N} R={R} n={n} {dtype} {order}", flush=True)
    s = adapter_inputs(T, K, N, R, n, dtype, True, "mixed", 7)
    s["ids"] = ids_of(order, T, n, gen("ids", T, n)).to(torch.int32)
    base = s["base"].to(dtype)
    x64 = ref.wide(s["x"], s["x_step"])
    h, hm = ref.first(x64, s["down"].double(), s["ids"], s["scale"])
    y, ym = ref.second(h, hm, s["up"].double(), s["ids"], ref.wide(base, s["x_step"]))
    args = [s[k].cuda() for k in ("x", "down", "up", "ids", "scale")]
    step, out = s["x_step"].cuda(), base.cuda()
    got, gh = B.adapter(*args, base=out, x_step=step, base_step=step)
    ref.check("h", gh, h, (ref.chain(K) + 4 * ref.U) * hm)
    ref.check("out", got, y, (ref.chain(K) + ref.chain(R) + 8 * ref.U) * ym)
    again, _ = B.adapter(*args, base=out, x_step=step, base_step=step, out=out)          # in the place of its base
    assert again.data_ptr() == out.data_ptr() and torch.equal(again, got)
    dy = normal(gen("dy", T, N), T, N, dtype=dtype, scale=0.5)
    dh, dhm = ref.first(dy.double(), s["up"].double(), s["ids"], s["scale"])
    dx, dxm = ref.second(dh, dhm, s["down"].double(), s["ids"], torch.zeros(T, K, dtype=torch.float64))
    d_down, ddm = ref.outer(dh, dhm, x64, s["ids"], n)
    d_up, dum = ref.outer(gh.cpu().double(), gh.cpu().double().abs(), dy.double(), s["ids"], n)
    got = B.adapter_backward(dy.cuda(), *args[:5], gh, x_step=step)
    ref.check("dx", got["dx"], dx, (ref.chain(N) + ref.chain(R) + 8 * ref.U) * dxm)
    ref.check("d_down", got["d_down"], d_down, (ref.chain(N) + ref.chain(T) + 8 * ref.U) * ddm)
    ref.check("d_up", got["d_up"], d_up, (ref.chain(T) + 4 * ref.U) * dum)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_stay_with_their_rows_where_adapters_alternate(B, dtype):  # noqa: F811
    T, K, N, R, n = 530, 96, 144, 6, 8
    s = adapter_inputs(T, K, N, R, n, dtype, False, "mixed", 8)
    clean = s["ids"] != 1
    other = [s[k].cuda() for k in ("ids", "scale", "base")]
    y0, h0 = B.adapter(s["x"].cuda(), s["down"].cuda(), s["up"].cuda(), *other[:2], base=other[2])
    down, up, x = s["down"].clone(), s["up"].clone(), s["x"].clone()
    down[1], up[1] = float("nan"), float("inf")
    x[~clean] = float("inf")
    y1, h1 = B.adapter(x.cuda(), down.cuda(), up.cuda(), *other[:2], base=other[2])
    keep = clean.cuda()
    assert torch.equal(y0[keep], y1[keep]) and torch.equal(h0[keep], h1[keep])
    assert not torch.isfinite(y1[~keep]).any()


def test_more_than_2_32_elements(B):  # noqa: F811
    """The last rows, beyond 2^32 elements, are what they are by themselves."""
    T, D = (1 << 20) + 5, 4104
    tail = normal(gen("far"), 7, D, dtype=BF16)
    x = torch.zeros((T, D), dtype=BF16, device="cuda")
    x[-7:] = tail.cuda()
    print("[case] far pack", flush=True)
    codes, step = B.pack_rows(x)
    want = ref.pack(tail)
    assert torch.equal(codes[-7:].cpu(), want[0]) and torch.equal(step[-7:].cpu(), want[1])
    assert torch.equal(B.unpack_rows(codes, step, BF16)[-7:].cpu(), (want[0].float() * want[1][:, None]).to(BF16))
    print("[case] far norm", flush=True)
    s = norm_inputs(7, D, BF16, BF16, True, 1, 9)
    kw = dict(pre_weight=s["pre"].cuda(), post_weight=s["post"].cuda(), gate=s["gate"].cuda(), alpha=s["alpha"], eps=s["eps"])
    got = B.norm_block(x, x, **kw)
    near = B.norm_block(x[-7:].clone(), x[-7:].clone(), **kw)
    assert all(torch.equal(a[-7:], b) for a, b in zip(got, near))
    del got
    print("[case] far norm backward", flush=True)
    back = B.norm_block_backward(x, None, x, x, **kw)
    near = B.norm_block_backward(x[-7:].clone(), None, x[-7:].clone(), x[-7:].clone(), **kw)
    assert torch.equal(back["dx"][-7:], near["dx"]) and torch.equal(back["df"][-7:], near["df"])


def test_strides_that_pass_2_32_elements(B):  # noqa: F811
    T, K, N, R, n = 4200, 64, 80, 8, 4
    stride = 1 << 20
    g = gen("strides")
    x = torch.empty((T, stride), dtype=torch.int8, device="cuda")[:, :K]
    out = torch.empty((T, stride), dtype=BF16, device="cuda")[:, :N]
    ids = (torch.arange(T, device="cuda") % n).to(torch.int32)
    codes, step = ref.pack(normal(g, T, K))
    x.copy_(codes.cuda())
    base = normal(g, T, N, dtype=BF16)
    out.copy_(base.cuda())
    down, up = normal(g, n, R, K, dtype=BF16).cuda(), normal(g, n, R, N, dtype=BF16).cuda()
    scale = torch.ones(n, device="cuda")
    print("[case] far strides", flush=True)
    near, nh = B.adapter(codes.cuda(), down, up, ids, scale, base=base.cuda(), x_step=step.cuda())
    got, gh = B.adapter(x, down, up, ids, scale, base=out, x_step=step.cuda(), out=out)
    assert torch.equal(got, near) and torch.equal(gh, nh)
    from paper_2002_00104_amd.pwlq import PwlqError
    with pytest.raises((ValueError, PwlqError)):
        B.adapter(torch.empty((2, stride + 16), dtype=torch.int8, device="cuda")[:, :K], down, up, ids[:2], scale, x_step=step[:2].cuda())
