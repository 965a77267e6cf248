"""Scores so large that a rounding of theirs is more than a weight can bear, and products so large that a scale of next to nothing matters.  Queries
and keys are whole numbers whose products are exact, so what comes out is known: one value, the mean of two, or the mean of all."""
import pytest
import torch

import attention_ref as ref
from test_gpu_attention import A, BF16, F16, gen, normal  # noqa: F401

pytestmark = pytest.mark.gpu
LONGEST = [1, 8, 1000]                                      # tiles of 16, 32 and 128 rows, at 4 heads of queries for one
SIZES = [(1, 90), (3, 700), (40, 120)]


def integers(g, dtype, packed, D, factor):
    """A cache of which channel 0 of the keys is a whole number times `factor`, no two of a sequence's on the same page alike by more than chance, and
    the values are whole numbers; the codes' steps are 1 and `factor`."""
    batch = ref.Batch(g, SIZES, 16)
    shape = (batch.pages, 1, batch.page)
    keys, values = torch.zeros(*shape, D), torch.randint(-100, 101, (*shape, D), generator=g).float()
    keys[..., 0] = torch.randint(-100, 101, shape, generator=g)
    if packed:
        one = torch.ones(shape)
        return batch, (keys.to(torch.int8), values.to(torch.int8), one * factor, one)
    return batch, ((keys * factor).to(dtype), values.to(dtype), None, None)


def expected(batch, cache, sign, T):
    """Of each row the mean of the values whose key is the largest (sign 1), the smallest (-1) or any (0), of those that the row sees."""
    out = torch.zeros(T, cache[0].shape[3], dtype=torch.float64)
    counts = torch.zeros(T, 1)
    for s, (n, length) in enumerate(batch.sizes):
        keys, values, _ = ref.sequence_rows(batch, cache, s)
        for j, own in enumerate(range(length - n, length)):
            k, v = sign * keys[:own + 1, 0, 0], values[:own + 1, 0]
            best = k == k.max()
            out[int(batch.starts[s]) + j] = v[best].mean(0)
            counts[int(batch.starts[s]) + j] = best.sum()
    return out, counts


def call(A, q, batch, cache, **kw):  # noqa: F811
    return A.attend(q.cuda(), A.Cache(*(None if t is None else t.cuda() for t in cache)), batch.table.cuda(), batch.lengths.cuda(), starts=batch.starts.cuda(),
                    **kw).cpu().double()


def mean_of_few(got, want, counts, unit):
    """Weights are 1 and 0, their sums are whole numbers: a product with the sum's reciprocal (2^-23) and the output's rounding."""
    want = want[:, None].expand_as(got)
    assert ((got - want).abs() <= (unit + 2.0 ** -22) * want.abs() + 2.0 ** -22 * counts[:, :, None]).all()


@pytest.mark.parametrize("longest", LONGEST)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype,packed", [(BF16, False), (F16, False), (BF16, True), (F16, True)], ids=["bf16", "f16", "bf16 codes", "f16 codes"])
def test_the_largest_score_takes_all(A, dtype, packed, D, longest):  # noqa: F811
    g = gen("far", D)
    batch, cache = integers(g, dtype, packed, D, 1.0)
    q = torch.zeros(batch.rows, 4, D, dtype=dtype)
    q[..., 0] = 1.0
    # one unit of a key is 2^8 at least: every other weight is 0
    for scale in (2.0 ** 8, 2.0 ** 18, 2.0 ** 21, 2.0 ** 24, 2.0 ** 27, 2.0 ** 32, 2.0 ** 60):
        for sign in (1, -1):
            got = call(A, q, batch, cache, scale=sign * scale, longest=longest)
            print(f"[case] {dtype} {packed} {D} {longest} scale {sign * scale}", flush=True)
            mean_of_few(got, *expected(batch, cache, sign, batch.rows), ref.UNIT[dtype])


@pytest.mark.parametrize("longest", LONGEST)
@pytest.mark.parametrize("dtype,packed", [(BF16, False), (BF16, True)], ids=["bf16", "bf16 codes"])
def test_large_products(A, dtype, packed, longest):  # noqa: F811
    """Queries and keys whose products are 2^40 and more, with a scale of 1, and 2^100 and more with scales that leave nothing of them."""
    g = gen("products")
    batch, cache = integers(g, dtype, packed, 64, 2.0 ** 20)
    q = torch.zeros(batch.rows, 4, 64, dtype=dtype)
    q[..., 0] = 2.0 ** 20
    mean_of_few(call(A, q, batch, cache, scale=1.0, longest=longest), *expected(batch, cache, 1, batch.rows), ref.UNIT[dtype])
    batch, cache = integers(g, dtype, packed, 64, 2.0 ** 60)
    q[..., 0] = 2.0 ** 58
    want, counts = expected(batch, cache, 0, batch.rows)
    for scale in (0.0, -0.0, 2.0 ** -148, -2.0 ** -148):    # scores are 0, or below 2^-23
        got = call(A, q, batch, cache, scale=scale, longest=longest)
        # with all weights 1 nothing but the sums is rounded, and the weights that differ from 1 by 2^-22
        room = 2.0 ** -21 * 100 + 2.0 ** -24 * 700 * 100
        assert ((got - want[:, None]).abs() <= ref.UNIT[dtype] * want[:, None].abs() + room).all(), scale
