"""The forward calls record nothing for autograd, so they do not take what autograd would have to follow."""
import pytest
import torch

from test_gpu_block import B, BF16  # noqa: F401

pytestmark = pytest.mark.gpu


def inputs():
    norm = dict(x=torch.ones(4, 64, dtype=BF16), f=torch.ones(4, 64, dtype=BF16), pre_weight=torch.ones(64), post_weight=torch.ones(64),
                gate=torch.ones(1, 64, dtype=BF16))
    adapter = dict(x=torch.ones(4, 64, dtype=BF16), down=torch.ones(2, 8, 64, dtype=BF16), up=torch.ones(2, 8, 48, dtype=BF16),
                   ids=torch.zeros(4, dtype=torch.int32), scale=torch.ones(2), base=torch.ones(4, 48), base_step=torch.ones(4))
    return {"norm_block": {k: v.cuda() for k, v in norm.items()}, "adapter": {k: v.cuda() for k, v in adapter.items()}}


@pytest.mark.parametrize("name", ["norm_block", "adapter"])
def test_tensors_that_require_gradients(B, name):  # noqa: F811
    call = getattr(B, name)
    sound = inputs()[name]
    want = call(**sound)
    for key, value in sound.items():
        if not value.is_floating_point():
            continue
        tracked = dict(sound, **{key: value.clone().requires_grad_()})
        with pytest.raises(ValueError, match=f"^{key} requires gradients.*{name}_backward"):
            call(**tracked)
        with pytest.raises(ValueError, match="requires gradients"):          # a result of such a tensor, as a network has it
            call(**dict(sound, **{key: tracked[key] * 1}))
        for mode in (torch.no_grad, torch.inference_mode):
            with mode():
                assert all(torch.equal(a, b) for a, b in zip(call(**tracked), want))
        assert all(torch.equal(a, b) for a, b in zip(call(**dict(tracked, **{key: tracked[key].detach()})), want))


def test_steps_that_require_gradients(B):  # noqa: F811
    s = inputs()["adapter"]
    codes, step = B.pack_rows(s.pop("x"))
    with pytest.raises(ValueError, match="^x_step requires gradients"):
        B.adapter(codes, x_step=step.requires_grad_(), **s)
    with pytest.raises(ValueError, match="^out requires gradients"):
        B.adapter(codes, x_step=step.detach(), out=torch.ones(4, 48, dtype=BF16, device="cuda", requires_grad=True), **s)
