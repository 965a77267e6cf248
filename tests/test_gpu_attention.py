"""The operators of pwlq_attention.h against their formulas in binary64.  The slacks are derived in attention_ref.py."""
import math
import zlib

import pytest
import torch

import attention_ref as ref
import block_ref

pytestmark = pytest.mark.gpu

BF16, F16, I8 = torch.bfloat16, torch.float16, torch.int8


@pytest.fixture(scope="module")
def A():
    assert torch.cuda.is_available()
    from paper_2002_00104_amd import attention
    return attention


def gen(*key):
    g = torch.Generator()
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def make_cache(g, batch, G, D, dtype, packed):
    """Keys and values of all pages, what belongs to no sequence included; steps where packed."""
    shape = (batch.pages, G, batch.page, D)
    keys, values = normal(g, *shape), normal(g, *shape, scale=0.7) + 0.3
    if not packed:
        return keys.to(dtype), values.to(dtype), None, None
    (k, ks), (v, vs) = (block_ref.pack(x.view(-1, D)) for x in (keys, values))
    return k.view(shape), v.view(shape), ks.view(shape[:3]), vs.view(shape[:3])


def on_gpu(A, cache):
    return A.Cache(*(None if t is None else t.cuda() for t in cache))


def spread(t, how):
    """The same [T, heads, D] on the GPU: as it is, as columns of a wider matrix, heads first in memory, or off any alignment."""
    t = t.cuda()
    T, H, D = t.shape
    if how == "whole":
        return t
    if how == "heads first":
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    pad = 8 if how == "columns" else 3
    wide = torch.full((T, H * D + 2 * pad), math.nan, dtype=t.dtype, device="cuda")
    wide[:, pad:pad + H * D] = t.reshape(T, H * D)
    return wide[:, pad:pad + H * D].unflatten(1, (H, D))


def run_attend(A, q, batch, cache, *, how="whole", starts=True, name="", **kw):
    scale = kw.pop("scale", q.shape[2] ** -0.5)
    put = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
    if starts:
        put["starts"] = batch.starts.cuda()
    got = A.attend(spread(q, how), on_gpu(A, cache), batch.table.cuda(), batch.lengths.cuda(), scale=scale, **put)
    kw.pop("longest", None)
    want, slack = ref.attend(q, batch, cache, scale, **kw)
    ref.check(name, got, want, slack)
    # the same with a table that has room for more, for which keys are cut into parts
    roomy = torch.nn.functional.pad(batch.table, (0, 20000 // batch.page + 1), value=2 ** 31 - 1).cuda()
    ref.check(name + " roomy", A.attend(spread(q, how), on_gpu(A, cache), roomy, batch.lengths.cuda(), scale=scale, **put), want, slack)
    return got


# --------------------------------------------------------------------------
# attention
# --------------------------------------------------------------------------
SIZES = {
    "one": [(1, 1)],
    "tokens": [(1, 1), (1, 17), (1, 128), (1, 129), (1, 700), (1, 33)],
    "pairs": [(2, 2), (2, 65), (2, 300), (2, 31)],
    "mixed": [(1, 90), (40, 40), (7, 200), (130, 257), (1, 1)],
    "prompt": [(259, 259)],
    "part": [(65, 400), (33, 97)],
    "gaps": [(0, 50), (3, 0), (5, 3), (1, 64), (0, 0), (2, 130)],
}
HEADS = [(1, 1), (8, 2), (5, 5), (12, 1), (20, 1), (33, 3)]


@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("sizes", sorted(SIZES))
@pytest.mark.parametrize("D", [16, 64, 80, 96, 112, 128, 160, 192, 240, 256])
def test_attend(A, sizes, D, dtype, packed):
    H, G = HEADS[zlib.crc32(repr((sizes, D)).encode()) % len(HEADS)]
    print(f"[case] attend {sizes} D={D} H={H} G={G} {dtype} {packed}", flush=True)
    g = gen("attend", sizes, D)
    batch = ref.Batch(g, SIZES[sizes], 16 if D % 64 else 64)
    cache = make_cache(g, batch, G, D, dtype, packed)
    q = normal(g, batch.rows, H, D, dtype=dtype, scale=1.5)
    run_attend(A, q, batch, cache, name=sizes)
    # what the caller says of the longest decides which kernel runs: all of them are right for all rows
    for longest in (1, max(2, 32 * G // H), 1000):
        run_attend(A, q, batch, cache, name=f"{sizes}, longest {longest}", longest=longest)


@pytest.mark.parametrize("H,G", HEADS)
@pytest.mark.parametrize("page", [16, 32, 256, 1024])
@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
def test_heads_and_pages(A, H, G, page, packed):
    g = gen("heads", H, G, page)
    batch = ref.Batch(g, [(1, 40), (1, 513), (1, 1500)], page, extra_columns=2)
    cache = make_cache(g, batch, G, 64, BF16, packed)
    q = normal(g, 3, H, 64, dtype=BF16)
    for how in ("whole", "columns", "heads first", "odd"):
        run_attend(A, q, batch, cache, starts=False, how=how, name=how)
    batch = ref.Batch(g, [(30, 300), (20, 20)], page)
    cache = make_cache(g, batch, G, 64, BF16, packed)
    q = normal(g, 50, H, 64, dtype=BF16)
    for how in ("whole", "columns", "heads first", "odd"):
        run_attend(A, q, batch, cache, how=how, name=how)


@pytest.mark.parametrize("dtype,packed", [(BF16, False), (BF16, True), (F16, True)], ids=["bf16", "bf16 codes", "f16 codes"])
@pytest.mark.parametrize("sizes", ["tokens", "mixed", "gaps", "part"])
@pytest.mark.parametrize("D", [80, 128, 256])
def test_scores(A, sizes, D, dtype, packed):
    """Caps, slopes, windows and prefixes, alone and together."""
    H, G = 6, 2
    g = gen("scores", sizes, D)
    batch = ref.Batch(g, SIZES[sizes], 32)
    cache = make_cache(g, batch, G, D, dtype, packed)
    q = normal(g, batch.rows, H, D, dtype=dtype, scale=3.0)
    S = len(batch.sizes)
    slopes = 2.0 ** -torch.arange(1, H + 1).float()
    prefix = torch.tensor([(0, 5, 40, 1000, 129, -3)[s % 6] for s in range(S)], dtype=torch.int32)
    for kw in (dict(cap=2.0), dict(cap=1e6), dict(slopes=slopes), dict(window=1), dict(window=20), dict(window=2 ** 40), dict(prefix=prefix),
               dict(cap=30.0, slopes=slopes, window=33, prefix=prefix), dict(scale=0.0), dict(scale=-0.25)):
        print(f"[case] {sizes} D={D} {dtype} {packed} {sorted(kw)}", flush=True)
        for longest in (1, 1000):
            run_attend(A, q, batch, cache, name=str(sorted(kw)), longest=longest, **kw)


def make_tree(g, batch, words):
    """Each drafted token continues one before it or the last kept one."""
    bits = torch.zeros(batch.rows, 64 * words, dtype=torch.bool)
    for s, (n, _) in enumerate(batch.sizes):
        at = int(batch.starts[s])
        for j in range(n):
            parent = int(torch.randint(0, j + 1, (1,), generator=g))
            if parent:
                bits[at + j] = bits[at + parent - 1]
            if j < 64 * words:
                bits[at + j, j] = True
    return (bits.view(batch.rows, words, 64).long() * (torch.ones(64, dtype=torch.long) << torch.arange(64))).sum(2)


@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
@pytest.mark.parametrize("new", [[1, 3], [4, 8], [63, 64, 65], [100, 7], [130]])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_tree(A, new, D, packed):
    g = gen("tree", new, D)
    batch = ref.Batch(g, [(n, n + 37 * i + (200 if i else 0)) for i, n in enumerate(new)] + [(2, 1)], 16)
    cache = make_cache(g, batch, 2, D, BF16, packed)
    q = normal(g, batch.rows, 8, D, dtype=BF16)
    for words in {1, (max(new) + 63) // 64}:
        tree = make_tree(g, batch, words)
        for cap in (0.0, 5.0):
            for longest in (1, max(new)):
                run_attend(A, q, batch, cache, name=f"{words} words", tree=tree, cap=cap, longest=longest)
    # rows that see what was kept only, and nothing at all where nothing was
    none = torch.zeros(batch.rows, 1, dtype=torch.long)
    got = run_attend(A, q, batch, cache, tree=none)
    assert not got[:new[0]].any()


def test_tree_of_a_chain_is_a_prompt(A):
    """A tree in which each token continues the one before it sees what the prompt sees."""
    g = gen("chain")
    batch = ref.Batch(g, [(60, 200), (17, 17)], 16)
    cache = make_cache(g, batch, 2, 128, BF16, False)
    q = normal(g, batch.rows, 8, 128, dtype=BF16)
    chain = torch.tensor([(1 << (j + 1)) - 1 for n, _ in batch.sizes for j in range(n)], dtype=torch.long)[:, None]
    for s in range(2):
        assert torch.equal(ref.seen_by(batch, s, 0, None, chain), ref.seen_by(batch, s, 0, None, None))
    run_attend(A, q, batch, cache, tree=chain)
    run_attend(A, q, batch, cache)


@pytest.mark.parametrize("dtype,packed", [(BF16, False), (F16, False), (BF16, True), (F16, True)])
@pytest.mark.parametrize("longest", [1, 8, 1000])
@pytest.mark.parametrize("D", [48, 80, 128, 192, 256])
def test_not_finite(A, dtype, packed, longest, D):
    """Infinities and NaN in keys and values reach the rows that see them, and no others."""
    g = gen("not finite", D)
    batch = ref.Batch(g, [(70, 100), (1, 77), (3, 61), (1, 50)], 16)
    inf, nan = math.inf, math.nan
    for kind in ("values", "keys"):
        cache = list(make_cache(g, batch, 2, D, dtype, packed))
        # past the ends there is anything
        for s, (_, length) in enumerate(batch.sizes):
            if length % 16:
                page = int(batch.table[s, length // 16])
                for i, t in enumerate(cache):
                    if t is not None and t.dtype != I8:
                        t[page, :, length % 16:] = nan if i % 2 else -inf
        for s, slot, what in ((0, 64, nan), (0, 80, inf), (0, 99, -inf), (2, 60, nan), (2, 59, inf)):
            page, row = batch.where(s, slot, batch.pages)
            if packed:
                t = cache[2 if kind == "keys" else 3]
                t[page, 0, row] = nan                   # a row with an infinity or NaN, as it is packed
                cache[0 if kind == "keys" else 1][page, 0, row] = 0
            else:
                t = cache[0 if kind == "keys" else 1]
                t[page, 0, row, D - 3] = what
        q = normal(g, batch.rows, 4, D, dtype=dtype)
        if kind == "keys":
            q[..., D - 3] = q[..., D - 3].abs().clamp(min=0.1)
        # a key's infinity makes a score of infinity (whose softmax is NaN) or of minus infinity (whose weight is 0)
        print(f"[case] not finite {kind} {dtype} {packed} {longest} {D}", flush=True)
        run_attend(A, q, batch, cache, name=kind, longest=longest)
        run_attend(A, q, batch, cache, name=kind + ", window", longest=longest, window=15)


@pytest.mark.parametrize("longest", [1, 8, 1000])
def test_nothing_but_minus_infinity(A, longest):
    """A row whose scores are all minus infinity is zeros."""
    g = gen("minus")
    batch = ref.Batch(g, [(3, 40)], 16)
    keys, values, _, _ = make_cache(g, batch, 1, 64, BF16, False)
    keys[..., 5] = -math.inf
    q = normal(g, 3, 2, 64, dtype=BF16)
    q[..., 5] = 1.0
    got = A.attend(q.cuda(), A.Cache(keys.cuda(), values.cuda()), batch.table.cuda(), batch.lengths.cuda(), starts=batch.starts.cuda(), longest=longest)
    assert not got.any()


@pytest.mark.parametrize("longest", [1, 8, 1000])
@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
def test_pages_that_are_none(A, packed, longest):
    """Rows on a page outside the cache are not seen; what lies there otherwise (page 0) is full of NaN here."""
    g = gen("none")
    batch = ref.Batch(g, [(5, 100), (1, 200), (70, 90), (1, 16)], 16)
    cache = list(make_cache(g, batch, 2, 128, BF16, packed))
    table = batch.table
    table[table == 0] = batch.pages - 1 if not (table == batch.pages - 1).any() else -1
    table[0, 3], table[1, 0], table[1, 5], table[2, 4], table[3, 0] = -1, batch.pages, 2 ** 31 - 1, -2 ** 31, -7
    for t in cache:
        if t is not None:
            t[0] = 77 if t.dtype == I8 else math.nan
    q = normal(g, batch.rows, 4, 128, dtype=BF16)
    got = run_attend(A, q, batch, cache, longest=longest)
    assert not got[-1].any()


def test_odd_starts_and_lengths(A):
    """Whatever the device's arrays hold, no row outside the call and no page outside the cache is touched."""
    g = gen("odd starts")
    batch = ref.Batch(g, [(4, 40), (4, 40), (4, 40)], 16)
    cache = on_gpu(A, make_cache(g, batch, 2, 64, BF16, False))
    q = normal(g, 12, 4, 64, dtype=BF16).cuda()
    for starts, lengths in (([0, 4, 2, 12], [40, 40, 40]), ([-5, 4, 8, 99], [40, 2 ** 31 - 1, -9]), ([9, 3, 3, 1], [0, 0, 0]),
                            ([2 ** 31 - 1] * 4, [40] * 3), ([-2 ** 31] * 4, [40] * 3)):
        for longest in (1, 8, 1000):
            A.attend(q, cache, batch.table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(),
                     starts=torch.tensor(starts, dtype=torch.int32).cuda(), longest=longest)
        torch.cuda.synchronize()


@pytest.mark.parametrize("S,T", [(3, 12), (70, 200), (2100, 2500)])
def test_rows_before_the_first_sequence(A, S, T):
    """Starts that begin behind the first rows, fall, or are any numbers: what lies before a sequence's first row belongs to none."""
    g = gen("no first", S)
    batch = ref.Batch(g, [(1, 40)] * S, 16)
    kept = make_cache(g, batch, 2, 64, BF16, False)
    cache, table, lengths = on_gpu(A, kept), batch.table.cuda(), batch.lengths.cuda()
    q, k = normal(g, T, 4, 64, dtype=BF16), normal(g, T, 2, 64, dtype=BF16)
    for first in (1, 5, T, 2 ** 31 - 1):
        starts = torch.full((S + 1,), first, dtype=torch.int32)
        starts[-1] = max(first, T)                          # the last sequence has all rows from `first` on
        for longest in (1, 8, 1000):
            out = torch.full_like(q, 7.0).cuda()
            A.attend(q.cuda(), cache, table, lengths, starts=starts.cuda(), longest=longest, out=out)
            assert (out[:first] == 7.0).all()
        to = tuple(torch.full_like(k, 7.0).cuda() for _ in range(2))
        A.read(cache, table, lengths, starts=starts.cuda(), rows=T, out=to)
        assert all((t[:first] == 7.0).all() for t in to)
        turned = torch.full_like(q, 7.0).cuda()
        A.append(cache, table, lengths, k.cuda(), k.cuda(), q.cuda(), starts=starts.cuda(), out=turned)
        assert (turned[:first] == 7.0).all() and torch.equal(turned[first:].cpu(), q[first:])
    for i in range(4):
        starts = torch.randint(-5, T + 5, (S + 1,), generator=g, dtype=torch.int32) if i < 3 else torch.arange(S, -1, -1, dtype=torch.int32)
        for longest in (1, 8, 1000):
            A.attend(q.cuda(), cache, table, lengths, starts=starts.cuda(), longest=longest)
        A.read(cache, table, lengths, starts=starts.cuda(), rows=T)
        A.append(cache, table, lengths, k.cuda(), k.cuda(), q.cuda(), starts=starts.cuda())
        torch.cuda.synchronize()


@pytest.mark.parametrize("longest", [1, 8, 1000])
def test_rows_behind_the_last_sequence(A, longest):
    g = gen("behind")
    batch = ref.Batch(g, [(3, 40), (70, 90)], 16)
    cache = make_cache(g, batch, 2, 64, BF16, False)
    q = normal(g, batch.rows + 9, 4, 64, dtype=BF16)
    out = torch.full(q.shape, 7.0, dtype=BF16, device="cuda")
    A.attend(q.cuda(), on_gpu(A, cache), batch.table.cuda(), batch.lengths.cuda(), starts=batch.starts.cuda(), longest=longest, out=out)
    want, slack = ref.attend(q, batch, cache, 0.125)
    ref.check("behind", out, want, slack)
    assert (out[batch.rows:] == 7.0).all()
    k = normal(g, batch.rows + 9, 2, 64, dtype=BF16).cuda()
    turned = torch.full(q.shape, 7.0, dtype=BF16, device="cuda")
    A.append(on_gpu(A, cache), batch.table.cuda(), batch.lengths.cuda(), k, k, q.cuda(), starts=batch.starts.cuda(), out=turned)
    assert torch.equal(turned[:batch.rows].cpu(), q[:batch.rows]) and (turned[batch.rows:] == 7.0).all()
    to = tuple(torch.full(k.shape, 7.0, dtype=BF16, device="cuda") for _ in range(2))
    A.read(on_gpu(A, cache), batch.table.cuda(), batch.lengths.cuda(), starts=batch.starts.cuda(), rows=k.shape[0], out=to)
    assert all((t[batch.rows:] == 7.0).all() for t in to)


@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
def test_many_sequences(A, packed):
    """More sequences than a call is cut for, and none of them long."""
    g = gen("many")
    batch = ref.Batch(g, [(1 + s % 3 // 2, 2 + s * 7 % 40) for s in range(2100)], 16)
    cache = make_cache(g, batch, 1, 64, BF16, packed)
    q = normal(g, batch.rows, 2, 64, dtype=BF16)
    run_attend(A, q, batch, cache, longest=2)
    batch = ref.Batch(g, [(1, 2 + s * 7 % 40) for s in range(2040)], 16)
    cache = make_cache(g, batch, 1, 64, BF16, packed)
    q = normal(g, batch.rows, 2, 64, dtype=BF16)
    run_attend(A, q, batch, cache, starts=False)
    run_attend(A, q, batch, cache)


@pytest.mark.parametrize("dtype,packed", [(BF16, False), (F16, True)])
def test_long(A, dtype, packed):
    """Keys split among many workgroups, of one sequence and of sequences of very different lengths."""
    g = gen("long")
    for sizes, longest in (([(1, 20000)], 1), ([(1, 9000), (1, 3), (1, 70), (1, 5000)], 1), ([(9, 9000), (40, 70)], 40), ([(64, 4000)], 64)):
        batch = ref.Batch(g, sizes, 64)
        cache = make_cache(g, batch, 2, 128, dtype, packed)
        q = normal(g, batch.rows, 4, 128, dtype=dtype, scale=2.0)
        run_attend(A, q, batch, cache, name=str(sizes), longest=longest)


def test_scores_that_grow(A):
    """The reference of a row's weights moves again and again, and falls behind by less than a step."""
    g = gen("grow")
    batch = ref.Batch(g, [(1, 1500), (40, 1500)], 64)
    keys, values, _, _ = make_cache(g, batch, 1, 64, BF16, False)
    for s, (_, length) in enumerate(batch.sizes):
        for slot in range(length):
            page, row = batch.where(s, slot, batch.pages)
            keys[page, :, row, 0] = slot / 16.0
    q = normal(g, 41, 2, 64, dtype=BF16)
    for scale, first in ((0.1, 1.0), (0.1, -1.0), (0.02, 4.0), (1.0, 16.0)):
        q[..., 0] = first
        for longest in (1, 1000):
            run_attend(A, q, batch, (keys, values, None, None), scale=scale, longest=longest)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_much_larger_scores_that_are_not_seen(A, D, packed, dtype):
    """What a row does not see has scores beside which its own weights would be nothing."""
    g = gen("larger", D)
    batch = ref.Batch(g, [(150, 300), (1, 77), (9, 40)], 16)
    cache = list(make_cache(g, batch, 1, D, dtype, packed))
    q = normal(g, batch.rows, 3, D, dtype=dtype, scale=60.0)
    for longest in (1, 10, 1000):
        for kw in (dict(window=1), dict(window=2), dict(window=40), {}, dict(tree=make_tree(g, batch, 3))):
            run_attend(A, q, batch, cache, name=str(sorted(kw)), longest=longest, **kw)


def test_beyond_32_bits(A):
    """Pages that lie more than 4 GiB into the cache."""
    pages, G, P, D = 20000, 8, 128, 128
    for dtype in (BF16, I8):
        cache = A.make_cache(pages, G, P, D, dtype)
        assert cache.keys.numel() * cache.keys.element_size() > (1 << 31 if dtype == I8 else 1 << 32)
        g = gen("far")
        batch = ref.Batch(g, [(3, 300), (150, 150)], P)
        far = torch.where(batch.table >= 0, pages - 1 - batch.table, batch.table)
        k, v, q = (normal(g, n, h, D, dtype=BF16) for n, h in ((450, G), (450, G), (450, 16)))
        whole = ref.Batch(g, [(300, 300), (150, 150)], P)
        A.append(cache, far.cuda(), batch.lengths.cuda(), k.cuda(), v.cuda(), starts=whole.starts.cuda())
        near = [torch.zeros(batch.pages, G, P, D, dtype=dtype), torch.zeros(batch.pages, G, P, D, dtype=dtype), None, None]
        if dtype == I8:
            near[2:] = [torch.zeros(batch.pages, G, P), torch.zeros(batch.pages, G, P)]
        row = 0
        for s, (_, length) in enumerate(whole.sizes):
            for slot in range(length):
                p, at = batch.where(s, slot, batch.pages)
                for i, x in ((0, k), (1, v)):
                    if dtype == I8:
                        near[i][p, :, at], near[2 + i][p, :, at] = block_ref.pack(x[row])
                    else:
                        near[i][p, :, at] = x[row]
                row += 1
        at = torch.cat([torch.arange(297, 300), torch.arange(300, 450)])
        got = A.attend(q[at].cuda(), cache, far.cuda(), batch.lengths.cuda(), starts=batch.starts.cuda())
        want, slack = ref.attend(q[at], batch, near, D ** -0.5)
        ref.check("far", got, want, slack)
        back = A.read(cache, far.cuda(), batch.lengths.cuda(), starts=whole.starts.cuda(), rows=450, dtype=BF16)
        for x, y in zip((k, v), back):
            if dtype == I8:
                codes, step = block_ref.pack(x.view(-1, D))
                x = (codes.float() * step[:, None]).to(BF16).view(x.shape)
            assert torch.equal(y.cpu(), x)
        del cache


# --------------------------------------------------------------------------
# appending and reading
# --------------------------------------------------------------------------
@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("D,R", [(16, 16), (48, 32), (64, 64), (80, 80), (128, 128), (128, 48), (192, 0), (256, 256)])
@pytest.mark.parametrize("sizes", ["one", "tokens", "mixed", "gaps"])
def test_append_and_read(A, sizes, D, R, dtype, packed):
    H, G = HEADS[zlib.crc32(repr((sizes, D)).encode()) % len(HEADS)]
    g = gen("append", sizes, D)
    batch = ref.Batch(g, SIZES[sizes], 16)
    T = batch.rows
    k, v, q = (normal(g, T, n, D, dtype=dtype, scale=2.0) for n in (G, G, H))
    frequencies = 10000.0 ** (-torch.arange(0, R, 2).float() / R) if R else None
    slots = torch.tensor([slot for s in range(len(batch.sizes)) for slot in batch.slots(s)], dtype=torch.int32)
    far = torch.randint(-5, 2 ** 31 - 1, (T,), generator=g, dtype=torch.int32)
    for how, interleaved, positions in (("whole", False, None), ("columns", True, None), ("odd", False, far), ("heads first", True, far)):
        print(f"[case] append {sizes} D={D} R={R} H={H} G={G} {dtype} {packed} {how} {interleaved}", flush=True)
        cache = make_cache(g, batch, G, D, dtype, packed)
        dev = on_gpu(A, cache)
        args = dict(starts=batch.starts.cuda(), frequencies=None if frequencies is None else frequencies.cuda(), interleaved=interleaved,
                    positions=None if positions is None else positions.cuda())
        got = A.append(dev, batch.table.cuda(), batch.lengths.cuda(), spread(k, how), spread(v, how), spread(q, how), **args)
        at = slots if positions is None else positions
        want, off = ref.rotate(q, at, frequencies, interleaved)
        ref.check("q", got, want, off)
        want_k, off_k = ref.rotate(k, at, frequencies, interleaved)
        kept = [None if t is None else t.cpu().clone() for t in dev]
        row = 0
        for s in range(len(batch.sizes)):
            for slot in batch.slots(s):
                place = batch.where(s, slot, batch.pages)
                if place:
                    p, r = place
                    for i, (want, off) in ((0, (want_k[row], off_k[row])), (1, (v[row].double(), torch.zeros(G, D, dtype=torch.float64)))):
                        if packed:
                            codes, step = kept[i][p, :, r], kept[2 + i][p, :, r].double()
                            # half a step, what the turn is off, and the quotient's and the factor's rounding of up to 127
                            room = (0.5 + 127 * 4 * ref.U) * step[:, None] + 2 * off + off.amax(1, keepdim=True)
                            assert ((codes.double() * step[:, None] - want).abs() <= room).all()
                            assert (codes.abs().amax(1) == 127).all()
                            if i == 1 or R == 0:
                                exact = block_ref.pack((v if i else k)[row])
                                assert torch.equal(codes, exact[0]) and torch.equal(step.float(), exact[1])
                        else:
                            ref.check("cache", kept[i][p, :, r][None], want[None], off[None])
                        # so that what is left can be compared
                        kept[i][p, :, r] = cache[i][p, :, r]
                        if packed:
                            kept[2 + i][p, :, r] = cache[2 + i][p, :, r]
                row += 1
        assert all(a is None or torch.equal(a, b) for a, b in zip(kept, cache)), "rows of the cache that were not given changed"
        # read back
        rows = A.read(dev, batch.table.cuda(), batch.lengths.cuda(), starts=batch.starts.cuda(), rows=T, dtype=dtype)
        row = 0
        for s in range(len(batch.sizes)):
            for slot in batch.slots(s):
                place = batch.where(s, slot, batch.pages)
                for i in range(2):
                    want = torch.zeros(G, D, dtype=dtype)
                    if place:
                        x = dev[i][place[0], :, place[1]].cpu()
                        want = (x.float() * dev[2 + i][place[0], :, place[1]].cpu()[:, None]).to(dtype) if packed else x
                    assert torch.equal(rows[i][row].cpu(), want)
                row += 1


def test_append_many_rows(A):
    """Several rows to a workgroup, with more heads than it has groups of lanes, and no whole number of rows."""
    g = gen("many rows")
    batch = ref.Batch(g, [(1000, 1000), (0, 5), (301, 400)], 64)
    k, v, q = (normal(g, batch.rows, n, 64, dtype=BF16) for n in (5, 5, 40))
    dev = A.make_cache(batch.pages, 5, 64, 64, BF16)
    f = 10000.0 ** (-torch.arange(32).float() / 32)
    got = A.append(dev, batch.table.cuda(), batch.lengths.cuda(), k.cuda(), v.cuda(), q.cuda(), starts=batch.starts.cuda(), frequencies=f.cuda())
    at = torch.tensor([slot for s in range(3) for slot in batch.slots(s)])
    want, off = ref.rotate(q, at, f, False)
    ref.check("q", got, want, off)
    rows = A.read(dev, batch.table.cuda(), batch.lengths.cuda(), starts=batch.starts.cuda(), rows=batch.rows)
    want, off = ref.rotate(k, at, f, False)
    ref.check("k", rows[0], want, off)
    assert torch.equal(rows[1].cpu(), v)


def test_append_rows_that_are_not_finite(A):
    """A row of a head with an infinity or a NaN is a row of NaN in 8 bits, one of next to nothing is zeros."""
    g = gen("rows")
    cache = A.make_cache(1, 2, 16, 64, I8)
    k = normal(g, 3, 2, 64, dtype=BF16)
    k[0, 0, 3], k[1, 1, 9], k[2, 0] = math.inf, math.nan, 2.0 ** -110
    table, lengths = torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.tensor([3], dtype=torch.int32).cuda()
    starts = torch.tensor([0, 3], dtype=torch.int32).cuda()
    A.append(cache, table, lengths, k.cuda(), k.cuda(), starts=starts)
    rows = A.read(cache, table, lengths, starts=starts, rows=3)
    for t in rows:
        t = t.cpu()
        assert torch.isnan(t[0, 0]).all() and torch.isnan(t[1, 1]).all() and not t[2, 0].any()
        assert torch.isfinite(t[0, 1]).all() and torch.isfinite(t[1, 0]).all()
    for step, x in ((cache.key_step, cache.keys), (cache.value_step, cache.values)):
        assert not x[0, 0, 0].any() and torch.isnan(step[0, 0, 0])


def test_append_skips_pages_that_are_none(A):
    g = gen("skip")
    cache = A.make_cache(4, 1, 16, 64, BF16)
    table = torch.tensor([[1, -1, 4, 2]], dtype=torch.int32).cuda()
    lengths, starts = torch.tensor([64], dtype=torch.int32).cuda(), torch.tensor([0, 64], dtype=torch.int32).cuda()
    k = normal(g, 64, 1, 64, dtype=BF16)
    A.append(cache, table, lengths, k.cuda(), k.cuda(), starts=starts)
    for pool in cache[:2]:
        assert torch.equal(pool[1, 0].cpu(), k[:16, 0]) and torch.equal(pool[2, 0].cpu(), k[48:, 0])
        assert not pool[0].any() and not pool[3].any()
    rows = A.read(cache, table, lengths, starts=starts, rows=64)
    assert not rows[0][16:48].any() and torch.equal(rows[1][48:].cpu(), k[48:])


# --------------------------------------------------------------------------
# together, and how they are called
# --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, I8], ids=["16 bits", "8 bits"])
def test_a_block_decodes(A, dtype):
    """Prompts, then tokens one by one, as a program runs them: projected, appended, attended to, packed and projected again; each step as
    if the whole sequences had come at once."""
    from paper_2002_00104_amd import block, pwlq
    g = gen("decodes")
    H, G, D, page = 4, 2, 64, 16
    prompts, steps = [5, 33, 16], 4
    batch = ref.Batch(g, [(n, n + steps) for n in prompts], page)
    cache, table = A.make_cache(batch.pages, G, page, D, dtype), batch.table.cuda()
    f = (10000.0 ** (-torch.arange(D // 2).float() / (D // 2))).cuda()
    whole = [normal(g, n + steps, (H + 2 * G) * D, dtype=BF16).cuda() for n in prompts]

    def call(rows, lengths, starts=None):
        q, k, v = (t.unflatten(1, (-1, D)) for t in rows.split((H * D, G * D, G * D), 1))
        q = A.append(cache, table, lengths, k, v, q, starts=starts, frequencies=f)
        return A.attend(q, cache, table, lengths, starts=starts, longest=None if starts is None else max(prompts))

    def counts(*n):
        return torch.tensor(n, dtype=torch.int32).cuda()

    first = call(torch.cat([w[:n] for w, n in zip(whole, prompts)]), counts(*prompts), counts(0, *torch.tensor(prompts).cumsum(0).tolist()))
    outs = [list(t) for t in first.split(prompts)]
    for i in range(steps):
        y = call(torch.stack([w[n + i] for w, n in zip(whole, prompts)]), counts(*(n + i + 1 for n in prompts)))
        for o, t in zip(outs, y):
            o.append(t)
    full = [n + steps for n in prompts]
    again = call(torch.cat(whole), counts(*full), counts(0, *torch.tensor(full).cumsum(0).tolist()))
    kept = [None if t is None else t.cpu() for t in cache]
    batch.sizes = [(n, n) for n in full]
    batch.starts = torch.tensor([0, *torch.tensor(full).cumsum(0).tolist()], dtype=torch.int32)
    q = torch.cat(whole)[:, :H * D].unflatten(1, (-1, D))
    at = torch.cat([torch.arange(n) for n in full])
    turned = A.append(cache, table, counts(*full), torch.cat(whole)[:, H * D:(H + G) * D].unflatten(1, (-1, D)),
                      torch.cat(whole)[:, (H + G) * D:].unflatten(1, (-1, D)), q, starts=batch.starts.cuda(), positions=at.to(torch.int32).cuda(), frequencies=f)
    want, slack = ref.attend(turned.cpu(), batch, kept, D ** -0.5)
    ref.check("at once", again, want, slack)
    ref.check("step by step", torch.cat([torch.stack(o) for o in outs]), want, slack)
    # what comes next takes it as it is
    codes, step = block.pack_rows(again.view(again.shape[0], -1))
    weight = normal(g, 32, H * D, scale=0.1).cuda()
    found = pwlq.search(weight, 4, 50)
    packed_codes, flags, w_hat = pwlq.quantize_packed(weight, 4, found["p_star"], found["m"])
    y = pwlq.linear_i8(codes, 1.0, 0.0, packed_codes, flags, 32, 4, found["p_star"], found["m"])[0]
    value = codes.double() * step.double()[:, None] @ w_hat.double().T
    assert torch.allclose(y.double() * step.double()[:, None], value, rtol=1e-4, atol=1e-4 * float(value.abs().max()))


def test_repeats_bit_for_bit(A):
    g = gen("bits")
    batch = ref.Batch(g, [(1, 9000), (1, 50), (1, 4000)], 64)
    cache = on_gpu(A, make_cache(g, batch, 2, 128, BF16, False))
    q, table, lengths = normal(g, 3, 8, 128, dtype=BF16).cuda(), batch.table.cuda(), batch.lengths.cuda()
    first = A.attend(q, cache, table, lengths)
    for _ in range(5):
        assert torch.equal(A.attend(q, cache, table, lengths), first)


def test_another_stream(A):
    g = gen("stream")
    batch = ref.Batch(g, [(1, 3000), (1, 50)], 64)
    kept = make_cache(g, batch, 2, 128, BF16, False)
    cache, table, lengths = on_gpu(A, kept), batch.table.cuda(), batch.lengths.cuda()
    q = normal(g, 2, 8, 128, dtype=BF16)
    want, slack = ref.attend(q, batch, kept, 128 ** -0.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = A.attend(q.cuda(), cache, table, lengths)
    side.synchronize()
    ref.check("side", got, want, slack)


@pytest.mark.parametrize("dtype", [BF16, I8], ids=["16 bits", "8 bits"])
def test_captured_and_replayed(A, dtype):
    """A decoding step in a graph: lengths, tables and rows change between replays, with eager work between them."""
    g = gen("graph")
    H, G, D, page, S = 8, 2, 128, 16, 3
    lengths0 = [1, 40, 333]
    batch = ref.Batch(g, [(1, n + 20) for n in lengths0], page)
    cache, other = (A.make_cache(batch.pages, G, page, D, dtype) for _ in range(2))
    table, f = batch.table.cuda(), (10000.0 ** (-torch.arange(D // 2).float() / (D // 2))).cuda()
    lengths = torch.tensor(lengths0, dtype=torch.int32).cuda()
    fill = normal(g, sum(lengths0), 2 * G, D, dtype=BF16).cuda()
    starts = torch.tensor([0, 1, 41, 374], dtype=torch.int32).cuda()
    for c in (cache, other):
        A.append(c, table, lengths, fill[:, :G], fill[:, G:], starts=starts)
    rows = torch.empty(S, (H + 2 * G) * D, dtype=BF16, device="cuda")

    def step(c):
        q, k, v = (t.unflatten(1, (-1, D)) for t in rows.split((H * D, G * D, G * D), 1))
        return A.attend(A.append(c, table, lengths, k, v, q, frequencies=f), c, table, lengths)

    rows.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache)                                         # writes rows: both caches get the same calls
        step(other)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(cache))
        graphs.append(graph)
    for i in range(6):
        lengths += 1
        rows.copy_(normal(g, S, (H + 2 * G) * D, dtype=BF16))
        eager = step(other)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i % 2], eager)
        assert all(a is None or torch.equal(a, b) for a, b in zip(cache, other))


def test_refusals(A):
    g = gen("refusals")
    batch = ref.Batch(g, [(1, 40), (1, 50)], 16)
    cache, table, lengths = on_gpu(A, make_cache(g, batch, 2, 64, BF16, False)), batch.table.cuda(), batch.lengths.cuda()
    q, k = normal(g, 2, 4, 64, dtype=BF16).cuda(), normal(g, 2, 2, 64, dtype=BF16).cuda()
    packed = on_gpu(A, make_cache(g, batch, 2, 64, BF16, True))
    starts = torch.tensor([0, 1, 2], dtype=torch.int32).cuda()
    ok = A.attend(q, cache, table, lengths)
    from paper_2002_00104_amd.pwlq import PwlqError
    grad = q.float().requires_grad_().to(BF16)
    for call in (lambda: A.attend(q.cpu(), cache, table, lengths), lambda: A.attend(q.float(), cache, table, lengths),
                 lambda: A.attend(q.half(), cache, table, lengths), lambda: A.attend(q[:1], cache, table, lengths, starts=starts[:2]),
                 lambda: A.attend(q, cache, table.long(), lengths), lambda: A.attend(q, cache, table, lengths.long()),
                 lambda: A.attend(q, cache, table, lengths[:1]), lambda: A.attend(q, cache, table, lengths, starts=starts[:2]),
                 lambda: A.attend(q[..., ::2], cache, table, lengths), lambda: A.attend(q, cache._replace(values=cache.values[:2]), table, lengths),
                 lambda: A.attend(q, packed._replace(key_step=None), table, lengths), lambda: A.attend(q, cache._replace(key_step=packed.key_step), table, lengths),
                 lambda: A.attend(q, cache, table, lengths, slopes=torch.ones(2, device="cuda")),
                 lambda: A.attend(q, cache, table, lengths, tree=torch.ones(2, 1, device="cuda")),
                 lambda: A.attend(q, cache, table, lengths, out=ok[:1]), lambda: A.attend(grad, cache, table, lengths),
                 lambda: A.append(cache, table, lengths, k, k, grad), lambda: A.append(cache, table, lengths, k, k[:, :1]),
                 lambda: A.append(cache, table, lengths, k, k, out=ok), lambda: A.append(cache, table, lengths, k.half(), k.half()),
                 lambda: A.append(cache, table, lengths, k, k, frequencies=torch.ones(65, device="cuda")),
                 lambda: A.append(cache, table, lengths, k, k, positions=torch.ones(2, device="cuda")),
                 lambda: A.read(cache, table, lengths, starts=starts), lambda: A.read(cache, table, lengths, rows=-1),
                 lambda: A.read(cache, table, lengths, dtype=F16), lambda: A.read(packed, table, lengths, dtype=torch.float32)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: A.attend(q, cache, table, lengths, cap=-1.0), lambda: A.attend(q, cache, table, lengths, cap=math.nan),
                 lambda: A.attend(q, cache, table, lengths, window=-1), lambda: A.attend(q[:1], cache, table, lengths),
                 lambda: A.attend(normal(g, 2, 3, 64, dtype=BF16).cuda(), cache, table, lengths),
                 lambda: A.attend(q, cache, table, lengths, window=3, tree=torch.ones(2, 1, dtype=torch.long, device="cuda")),
                 lambda: A.attend(q, cache, torch.nn.functional.pad(table, (0, 300)), lengths, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")),
                 lambda: A.append(cache, table, lengths, k, k, frequencies=torch.ones(12, device="cuda")),
                 lambda: A.append(cache, table, lengths, k, k, normal(g, 2, 3, 64, dtype=BF16).cuda()),
                 lambda: A.read(cache, table, lengths, rows=1)):
        with pytest.raises(PwlqError):
            call()
    with torch.no_grad():
        A.attend(grad, cache, table, lengths)
    none = torch.empty(0, 4, 64, dtype=BF16, device="cuda")
    empty = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    assert A.attend(none, cache, empty, lengths[:0]).shape == (0, 4, 64)
    assert A.read(cache, empty, lengths[:0])[0].shape == (0, 2, 64)
    assert torch.equal(A.attend(q, cache, table, lengths), ok)
