"""The gradient of the residual stream alone, from 8-bit checkpoints of a binary32 stream and a 16-bit block output: the
checkpoints do not say the output's type, the gate or the caller does."""
import pytest
import torch

import block_ref as ref
from test_gpu_block import B, BF16, F16, F32, cuda, gen, norm_inputs, normal  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,D,G", [(12, 577, 3), (6, 72, 6), (4, 2050, 1), (5, 96, 0)])
@pytest.mark.parametrize("post", [True, False])
def test_block_output_type_without_du(B, dtype, T, D, G, post):  # noqa: F811
    print(f"[case] kept {dtype} {T}x{D} G={G} post={post}", flush=True)
    s = norm_inputs(T, D, dtype, F32, post, G, 13)
    dxo = normal(gen("kept", T, D), T, D)
    (x, xs), (f, fs) = ref.pack(s["x"]), ref.pack(s["f"])
    want, slack = ref.norm_backward(None, ref.wide(dxo), ref.wide(x, xs), ref.wide(f, fs), s["pre"], s["post"], s["gate"], s["alpha"], s["eps"])
    kw = dict(pre_weight=s["pre"].cuda(), post_weight=cuda(s["post"]), gate=cuda(s["gate"]), alpha=s["alpha"], eps=s["eps"], x_step=xs.cuda(),
              f_step=fs.cuda())
    if not G:                                              # nothing has the type: as it is asked for, else that of dx
        assert B.norm_block_backward(None, dxo.cuda(), x.cuda(), f.cuda(), **kw)["df"].dtype == F32
        kw["dtype"] = dtype
    got = B.norm_block_backward(None, dxo.cuda(), x.cuda(), f.cuda(), **kw)
    assert got["dx"].dtype == F32 and got["df"].dtype == dtype
    assert {k for k, v in got.items() if v is not None} == set(want)
    for k in want:
        ref.check(k, got[k], want[k], slack[k])


def test_types_that_do_not_go_together(B):  # noqa: F811
    x, w = torch.ones(4, 64, dtype=BF16, device="cuda"), torch.ones(64, device="cuda")
    codes, step = B.pack_rows(x)
    kw = dict(pre_weight=w, x_step=step, f_step=step)
    from paper_2002_00104_amd.pwlq import PwlqError
    with pytest.raises(PwlqError):                         # a residual narrower than the block's output
        B.norm_block_backward(None, x, codes, codes, gate=torch.ones(1, 64, device="cuda"), **kw)
    with pytest.raises(ValueError):
        B.norm_block_backward(None, x, codes, codes, dtype=torch.float64, **kw)
    with pytest.raises(TypeError):
        B.norm_block_backward(None, x, codes, codes, dtype="bfloat16", **kw)
    with pytest.raises(ValueError):                        # du's type it is
        B.norm_block_backward(x, x, codes, codes, gate=torch.ones(1, 64, device="cuda"), **kw)
