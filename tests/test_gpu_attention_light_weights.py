"""A key of a score far above those of many others: what these weigh together is not lost, though each is next to nothing."""
import pytest
import torch

import attention_ref as ref
from test_gpu_attention import A, BF16, F16, I8, gen  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("longest", [1, 8, 1000])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype,packed", [(BF16, False), (F16, False), (BF16, True), (F16, True)], ids=["bf16", "f16", "bf16 codes", "f16 codes"])
def test_values_that_are_all_one(A, dtype, packed, D, longest):  # noqa: F811
    """The first key's weight is 1, that of 2^20 others 2^-25.2 to 2^-24.8: 2^-5 together.  Where all values are 1, so is the output."""
    page, n = 65536, 1 << 20
    many = longest == 1000 or (longest == 8 and D == 256)   # tiles of 128 rows
    most = 8.0
    keys = torch.zeros(2, 1, page, D)
    keys[0, 0, 0, 0] = most
    values = torch.ones(2, 1, page, D)
    if packed:
        step = torch.ones(2, 1, page)
        cache = (keys.to(I8), values.to(I8), step, step)
    else:
        cache = (keys.to(dtype), values.to(dtype), None, None)
    cache = A.Cache(*(None if t is None else t.cuda() for t in cache))
    # sequences of no rows beside it, so many that the long one is a workgroup's whole; alone it is cut
    for S in (1, 2048):
        table = torch.full((S, n // page), 1, dtype=torch.int32)
        table[0, 0] = 0
        lengths, starts = torch.zeros(S, dtype=torch.int32), torch.full((S + 1,), 2, dtype=torch.int32)
        lengths[0], starts[0] = n, 0
        q = torch.zeros(2, 4, D, dtype=dtype)
        q[..., 0] = 1.0
        for gap in (24.8, 25.0, 25.2):
            got = A.attend(q.cuda(), cache, table.cuda(), lengths.cuda(), starts=starts.cuda(), longest=longest, scale=gap / 1.4426950408889634 / most)
            # the sums of weights and of products are of the same numbers but for each weight's rounding: half a unit of what it is, or in binary16 2^-25 of
            # weights that are multiples of 2^-7; both sums take at most so many steps after the first key, each off by half a unit of the sum; then the
            # output's rounding
            steps = n / 16 + n / 32 if many else 2 * n / 128
            room = 2 * ref.UNIT[dtype] + (n * 2.0 ** -32 if dtype == F16 else 0.0) + 2.0 * steps * 2.0 ** -24
            worst = float((got.double() - 1.0).abs().max())
            print(f"[case] {dtype} {packed} {D} {longest} S={S} gap {gap}: {worst:.3g} of {room:.3g}", flush=True)
            assert worst <= room
