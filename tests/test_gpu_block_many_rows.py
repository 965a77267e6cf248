"""Adapters over millions of rows: rows of the beginning, the middle and the end by the formulas, gradients summed in binary64."""
import pytest
import torch

import block_ref as ref
from test_gpu_block import B, BF16  # noqa: F401

pytestmark = pytest.mark.gpu


def test_five_million_rows(B):  # noqa: F811
    T, K, N, R, n = 5_000_003, 64, 64, 8, 4
    print(f"[case] {T} rows", flush=True)
    g = torch.Generator(device="cuda").manual_seed(5)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(BF16)

    x, dy, base = normal(T, K), normal(T, N, scale=0.5), normal(T, N)
    down, up = normal(n, R, K, scale=K ** -0.5), normal(n, R, N, scale=0.1)
    scale = torch.rand((n,), generator=g, device="cuda") + 0.5
    ids = torch.arange(T, device="cuda").div(1000, rounding_mode="floor").remainder(n + 1).sub(1).to(torch.int32)
    y, h = B.adapter(x, down, up, ids, scale, base=base)
    got = B.adapter_backward(dy, x, down, up, ids, scale, h)
    at = torch.cat([torch.arange(0, 200), torch.arange(T // 2, T // 2 + 200), torch.arange(T - 200, T)]).cuda()
    at[150:200] += 900                                    # a change of adapters
    a = {k: v[at].cpu() for k, v in dict(x=x, dy=dy, base=base, ids=ids, y=y, h=h, dx=got["dx"]).items()}
    wide = dict(down=ref.wide(down), up=ref.wide(up))
    want, mag = ref.first(a["x"].double(), wide["down"], a["ids"], scale.cpu())
    ref.check("h", a["h"], want, (ref.chain(K) + 4 * ref.U) * mag)
    want, mag = ref.second(want, mag, wide["up"], a["ids"], a["base"].double())
    ref.check("out", a["y"], want, (ref.chain(K) + ref.chain(R) + 8 * ref.U) * mag)
    want, mag = ref.first(a["dy"].double(), wide["up"], a["ids"], scale.cpu())
    want, mag = ref.second(want, mag, wide["down"], a["ids"], torch.zeros(len(at), K, dtype=torch.float64))
    ref.check("dx", a["dx"], want, (ref.chain(N) + ref.chain(R) + 8 * ref.U) * mag)
    for k in range(n):
        print(f"[case] {T} rows, gradients of adapter {k}", flush=True)
        mine = (ids == k).nonzero().flatten()
        x64, dy64, h64 = x[mine].double(), dy[mine].double(), h[mine].double()
        dh = scale[k].double() * (dy64 @ up[k].double().t().contiguous())
        dhm = scale[k].double() * (dy64.abs() @ up[k].double().abs().t().contiguous())
        ref.check("d_up", got["d_up"][k], (h64.t() @ dy64).cpu(), ((ref.chain(T) + 4 * ref.U) * (h64.t().abs() @ dy64.abs())).cpu())
        ref.check("d_down", got["d_down"][k], (dh.t() @ x64).cpu(),
                  ((ref.chain(N) + ref.chain(T) + 8 * ref.U) * (dhm.t() @ x64.abs())).cpu())
