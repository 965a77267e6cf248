"""The work is launched on the current device: tensors of another one are refused.  One GPU is enough: the tensors of the other are
shells without memory."""
import pytest
import torch

from test_gpu_block import B, BF16, F32  # noqa: F401

pytestmark = pytest.mark.gpu


class Shell(torch.Tensor):
    @staticmethod
    def __new__(cls, *shape, dtype=BF16):
        other = f"cuda:{torch.cuda.current_device() + 1}"
        return torch.Tensor._make_wrapper_subclass(cls, shape, dtype=dtype, device=other)

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise AssertionError(f"{func} of a tensor that is not there")


CALLS = {
    "pack_rows": lambda B: B.pack_rows(Shell(4, 64)),
    "unpack_rows": lambda B: B.unpack_rows(Shell(4, 64, dtype=torch.int8), Shell(4, dtype=F32)),
    "norm_block": lambda B: B.norm_block(Shell(4, 64), Shell(4, 64), pre_weight=Shell(64, dtype=F32)),
    "norm_block_backward": lambda B: B.norm_block_backward(Shell(4, 64), None, Shell(4, 64), pre_weight=Shell(64, dtype=F32)),
    "adapter": lambda B: B.adapter(Shell(4, 64), Shell(2, 8, 64), Shell(2, 8, 48), Shell(4, dtype=torch.int32), Shell(2, dtype=F32)),
    "adapter_backward": lambda B: B.adapter_backward(Shell(4, 48), Shell(4, 64), Shell(2, 8, 64), Shell(2, 8, 48), Shell(4, dtype=torch.int32),
                                                     Shell(2, dtype=F32), Shell(4, 8, dtype=F32)),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_tensors_of_another_device(B, name):  # noqa: F811
    with pytest.raises(ValueError, match="current device"):
        CALLS[name](B)
