"""The operators together, as the example uses them: fine-tuning from 8-bit checkpoints, then serving."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "adapters_beside_packed_weights.py")
    spec = importlib.util.spec_from_file_location("adapters_beside_packed_weights", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def setting(example, T=90, width=256, adapters=3):
    stack = example.Stack(width, blocks=2, rank=6, adapters=adapters)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((T, width), generator=g, device="cuda").to(torch.bfloat16)
    ids = (torch.arange(T, device="cuda") % (adapters + 1) - 1).to(torch.int32)
    return stack, x, ids, g


def test_training_lowers_the_loss(example):
    stack, x, ids, g = setting(example)
    target = stack.forward(x, ids).float() + 0.5 * torch.randn((4, 256), generator=g, device="cuda")[ids.long() + 1]
    optimizer = torch.optim.Adam(stack.parameters(), lr=5e-3)
    losses = [stack.step(x, ids, target, optimizer).item() for _ in range(30)]
    print(losses)
    assert losses[-1] < 0.5 * losses[0]


def test_an_untouched_adapter_does_not_learn(example):
    stack, x, ids, g = setting(example)
    ids = torch.where(ids == 1, torch.full_like(ids, -1), ids)
    before = [b.master["up"].clone() for b in stack.blocks]
    optimizer = torch.optim.Adam(stack.parameters(), lr=5e-3)
    stack.step(x, ids, torch.randn((90, 256), generator=g, device="cuda"), optimizer)
    for b, up in zip(stack.blocks, before):
        assert torch.equal(b.master["up"][1], up[1]) and not torch.equal(b.master["up"][0], up[0])


def test_rows_are_served_as_they_were_in_the_prompt(example):
    """A batch of single tokens takes other kernels than a prompt.  Sums in another order move an 8-bit code by one step
    now and then and a bfloat16 output by a unit: together far below a tenth of the outputs' size, which is 1."""
    stack, x, ids, g = setting(example)
    for b in stack.blocks:
        b.master["up"].copy_(0.05 * torch.randn(b.master["up"].shape, generator=g, device="cuda"))
        b.cast()
    prompt = stack.forward(x, ids).float()
    for rows in ([7], [0, 1, 2, 3], list(range(40, 80))):
        at = torch.tensor(rows, device="cuda")
        assert (stack.forward(x[at].contiguous(), ids[at].contiguous()).float() - prompt[at]).abs().max() < 0.1
