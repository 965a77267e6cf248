"""Gradients of a few adapters of a large bank: the rows are split although most adapters have none."""
import pytest
import torch

import block_ref as ref
from test_gpu_block import B, BF16, F32, adapter_inputs, gen, normal  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,K,N,R,n", [(9000, 64, 72, 16, 512), (12300, 136, 40, 20, 300)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", ["one", "eight", "all"])
def test_few_of_many_adapters(B, T, K, N, R, n, dtype, order):  # noqa: F811
    print(f"[case] bank {T}x{K}x{N} R={R} n={n} {dtype} {order}", flush=True)
    s = adapter_inputs(T, K, N, R, n, dtype, True, "mixed", 14)
    t = torch.arange(T)
    s["ids"] = {"one": torch.full((T,), n - 2), "eight": t % 8 * (n // 8), "all": t * n // T}[order].to(torch.int32)
    g = gen("bank", T, N)
    dy, h = normal(g, T, N, dtype=dtype, scale=0.5), normal(g, T, R)
    x64, dy64 = ref.wide(s["x"], s["x_step"]), ref.wide(dy)
    dh, dhm = ref.first(dy64, s["up"].double(), s["ids"], s["scale"])
    d_down, ddm = ref.outer(dh, dhm, x64, s["ids"], n)
    d_up, dum = ref.outer(h.double(), h.double().abs(), dy64, s["ids"], n)
    got = B.adapter_backward(dy.cuda(), s["x"].cuda(), s["down"].cuda(), s["up"].cuda(), s["ids"].cuda(), s["scale"].cuda(), h.cuda(),
                             x_step=s["x_step"].cuda())
    ref.check("d_down", got["d_down"], d_down, (ref.chain(N) + ref.chain(T) + 8 * ref.U) * ddm)
    ref.check("d_up", got["d_up"], d_up, (ref.chain(T) + 4 * ref.U) * dum)
