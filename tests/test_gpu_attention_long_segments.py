"""Tiles of 128 rows over 8-bit caches of more than 128 channels, where a workgroup goes through more than 1024 keys of one item: the pages it has
looked up are then more than half of a wavefront's lanes hold.  Rows' steps differ by large factors, so that another row's step is seen."""
import math

import pytest
import torch

import attention_ref as ref
import block_ref
from test_gpu_attention import A, BF16, F16, gen, normal, run_attend  # noqa: F401

pytestmark = pytest.mark.gpu


def packed_cache(g, batch, G, D):
    """Rows of sizes from 1/8 to 8; page 0, which no sequence has, is NaN."""
    shape = (batch.pages, G, batch.page)
    cache = []
    for scale in (0.5, 0.7):
        x = normal(g, *shape, D, scale=scale) * 2.0 ** torch.randint(-3, 4, shape, generator=g)[..., None]
        codes, step = block_ref.pack(x.view(-1, D))
        cache.append((codes.view(*shape, D), step.view(shape)))
    (keys, key_step), (values, value_step) = cache
    keys[0], values[0], key_step[0], value_step[0] = 77, 77, math.nan, math.nan
    return keys, values, key_step, value_step


def without_page_0(batch):
    spare = next(p for p in range(batch.pages) if not (batch.table == p).any())
    batch.table[batch.table == 0] = spare
    return batch


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("D", [128, 144, 192, 256])
def test_whole_items(A, D, dtype):  # noqa: F811
    """128 sequences of 4 heads, most of which have no rows: items enough to stay whole."""
    g = gen("whole", D)
    for page in (16, 64):
        batch = without_page_0(ref.Batch(g, [(3, 2600), (0, 0), (40, 1531), (1, 1100), (2, 513)] + [(0, 0)] * 123, page))
        cache = packed_cache(g, batch, 4, D)
        q = normal(g, batch.rows, 4, D, dtype=dtype)
        for kw in ({}, dict(window=1500), dict(cap=5.0)):
            print(f"[case] whole D={D} {dtype} page {page} {kw}", flush=True)
            run_attend(A, q, batch, cache, name=f"page {page} {kw}", longest=1024, **kw)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("D", [128, 144, 192, 256])
def test_long_parts(A, D, dtype):  # noqa: F811
    """Nine sequences on the same pages, whose line is cut into parts of about 30 units."""
    g = gen("parts", D)
    batch = without_page_0(ref.Batch(g, [(2, 8191)], 32))
    n = 9
    batch.sizes, batch.rows = [(2, 8191 - 700 * s) for s in range(n)], 2 * n
    batch.table = batch.table.repeat(n, 1)
    batch.lengths = torch.tensor([length for _, length in batch.sizes], dtype=torch.int32)
    batch.starts = torch.arange(n + 1, dtype=torch.int32) * 2
    cache = packed_cache(g, batch, 4, D)
    q = normal(g, batch.rows, 8, D, dtype=dtype)
    for kw in ({}, dict(tree=torch.tensor([[1], [3]] * n))):
        print(f"[case] parts D={D} {dtype} {sorted(kw)}", flush=True)
        run_attend(A, q, batch, cache, name=str(sorted(kw)), longest=1024, **kw)


@pytest.mark.parametrize("dtype,packed", [(BF16, False), (F16, False), (BF16, True), (F16, True)], ids=["bf16", "f16", "bf16 codes", "f16 codes"])
@pytest.mark.parametrize("longest", [1, 8, 1024])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_not_finite_far_from_the_start(A, D, longest, dtype, packed):  # noqa: F811
    """Infinities and NaN among values thousands of keys into an item, seen by some of its rows, by all, and by none; whole and cut."""
    g = gen("far from the start", D)
    for empty in (0, 2100):
        batch = without_page_0(ref.Batch(g, [(3, 4200), (40, 2531), (1, 1100)] + [(0, 0)] * empty, 16))
        if packed:
            cache = packed_cache(g, batch, 2, D)
        else:
            shape = (batch.pages, 2, 16, D)
            cache = (normal(g, *shape, dtype=dtype), normal(g, *shape, dtype=dtype), None, None)
        for s, slot, what in ((0, 4198, math.inf), (0, 3600, math.nan), (0, 100, math.inf), (1, 2510, -math.inf), (1, 2500, math.inf), (1, 2100, math.nan),
                              (2, 400, math.nan)):
            page, row = batch.where(s, slot, batch.pages)
            if packed:
                cache[1][page, 0, row], cache[3][page, 0, row] = 0, math.nan
            else:
                cache[1][page, 0, row, D - 3] = what
        q = normal(g, batch.rows, 4, D, dtype=dtype, scale=0.3)
        for window in (0, 420, 699):
            print(f"[case] far from the start {D} {longest} {dtype} {packed} {empty} {window}", flush=True)
            run_attend(A, q, batch, cache, name=f"window {window}", longest=longest, window=window)
