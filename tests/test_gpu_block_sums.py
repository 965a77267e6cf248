"""Gradients that are sums over many rows, where the rows are split: norms whose walks have more than two rows and leave more than 128
partial rows, with gate rows that end inside a walk, straddle walks and are longer than one; rows of no whole vectors at every width;
8-bit checkpoints beside a binary32 residual stream; adapters' gradients in more than 64 parts."""
import pytest
import torch

import block_ref as ref
from test_gpu_block import B, BF16, F16, F32, TYPES, adapter_inputs, cuda, gates, gen, norm_inputs, normal, spread  # noqa: F401

pytestmark = pytest.mark.gpu


def norm_both_ways(B, T, D, dtype, stream, post, kept, G, how="whole", forward=True):  # noqa: F811
    print(f"[case] norm {dtype} {stream} {T}x{D} post={post} kept={kept} G={G} {how}", flush=True)
    s = norm_inputs(T, D, dtype, stream, post, G, 11)
    kw = dict(pre_weight=s["pre"].cuda(), post_weight=cuda(s["post"]), gate=cuda(s["gate"]), alpha=s["alpha"], eps=s["eps"])
    if forward:
        x, u, sx, su = ref.norm_block(**s)
        got = B.norm_block(spread(s["x"], how), spread(s["f"], how), **kw)
        ref.check("x_out", got[0], x, sx)
        ref.check("u", got[1], u, su)
        _, codes, step = B.norm_block(spread(s["x"], how), spread(s["f"], how), pack=True, **kw)
        assert ((ref.wide(codes, step) - u).abs() <= 0.5001 * step.cpu().double()[:, None] + su + 1e-30).all()
    g = gen("sums", T, D)
    du, dxo, x, f, xs, fs = normal(g, T, D, dtype=dtype), normal(g, T, D, dtype=stream), s["x"], s["f"], None, None
    if kept:
        (x, xs), (f, fs) = ref.pack(x), ref.pack(f)
    want, slack = ref.norm_backward(ref.wide(du), ref.wide(dxo), ref.wide(x, xs), ref.wide(f, fs), s["pre"], s["post"], s["gate"], s["alpha"], s["eps"])
    got = B.norm_block_backward(spread(du, how), spread(dxo, how), spread(x, how), spread(f, how), x_step=cuda(xs), f_step=cuda(fs), **kw)
    assert got["dx"].dtype == stream and got["df"].dtype == dtype
    assert {k for k, v in got.items() if v is not None} == set(want)
    for k in want:
        ref.check(k, got[k], want[k], slack[k])


# 2048 wavefronts walk the rows: 4 walks of a wavefront to a workgroup up to 512 columns, else a walk of one wavefront for each
# 512 columns up to 2048 and for each 1024 beyond.  Spans of 3, 5, 5 and 9 rows.
LONG = [(6000, 296, BF16, F32), (6000, 301, F32, F32), (5000, 520, F16, F16), (3000, 2050, BF16, BF16), (4100, 4096, BF16, BF16)]


@pytest.mark.parametrize("T,D,dtype,stream,G", [(T, *how, G) for T, *how in LONG
                                                for G in [0, 1] + [T // per for per in (1, 2, 3, 4, 5, 9, 100) if T % per == 0]])
def test_long_walks(B, T, D, dtype, stream, G):  # noqa: F811
    norm_both_ways(B, T, D, dtype, stream, True, dtype != F32, G, forward=False)


@pytest.mark.parametrize("T,G", [(8193, 1), (8193, 3), (12289, 1)])
def test_long_walks_without_a_post_norm(B, T, G):  # noqa: F811
    norm_both_ways(B, T, 200, F32, F32, False, False, G, forward=False)


@pytest.mark.parametrize("D", [2050, 4090, 4100, 8191, 8201, 12288, 16383])
@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("kept", [True, False])
def test_wide_rows(B, D, dtype, stream, kept):  # noqa: F811
    for post in (True, False):
        norm_both_ways(B, 9, D, dtype, stream, post, kept, 3, "odd" if post else "columns")


@pytest.mark.parametrize("T,D", [(6, 577), (12, 1155), (130, 72), (4, 8192), (10, 2050)])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("post", [True, False])
def test_checkpoints_beside_a_binary32_residual(B, T, D, dtype, post):  # noqa: F811
    for G in gates(T):
        for how in ("whole", "columns", "odd"):
            norm_both_ways(B, T, D, dtype, F32, post, True, G, how, forward=False)


@pytest.mark.parametrize("T,K,N,R,n", [(6000, 64, 72, 5, 1), (4200, 129, 40, 40, 1), (14000, 64, 72, 16, 3)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("packed", [True, False])
def test_adapters_gradients_in_many_parts(B, T, K, N, R, n, dtype, packed):  # noqa: F811
    print(f"[case] parts {T}x{K}x{N} R={R} n={n} {dtype} packed={packed}", flush=True)
    s = adapter_inputs(T, K, N, R, n, dtype, packed, "mixed", 12)
    g = gen("parts", T, N)
    dy, h = normal(g, T, N, dtype=dtype, scale=0.5), normal(g, T, R)
    x64, dy64 = ref.wide(s["x"], s["x_step"]), ref.wide(dy)
    dh, dhm = ref.first(dy64, s["up"].double(), s["ids"], s["scale"])
    dx, dxm = ref.second(dh, dhm, s["down"].double(), s["ids"], torch.zeros(T, K, dtype=torch.float64))
    d_down, ddm = ref.outer(dh, dhm, x64, s["ids"], n)
    d_up, dum = ref.outer(h.double(), h.double().abs(), dy64, s["ids"], n)
    got = B.adapter_backward(dy.cuda(), s["x"].cuda(), s["down"].cuda(), s["up"].cuda(), s["ids"].cuda(), s["scale"].cuda(), h.cuda(),
                             x_step=cuda(s["x_step"]))
    ref.check("dx", got["dx"], dx, (ref.chain(N) + ref.chain(R) + 8 * ref.U) * dxm)
    ref.check("d_down", got["d_down"], d_down, (ref.chain(N) + ref.chain(T) + 8 * ref.U) * ddm)
    ref.check("d_up", got["d_up"], d_up, (ref.chain(T) + 4 * ref.U) * dum)
