"""Calls of the operators of pwlq_attention.h that a program makes and one test of sizes does not: two at once, graphs that share a workspace,
outputs of other strides, pages and sequences used twice, the largest pages, the ends of the range of scale and cap, and what the binding refuses."""
import math

import pytest
import torch

import attention_ref as ref
from test_gpu_attention import A, BF16, F16, I8, gen, make_cache, normal, on_gpu, run_attend, spread  # noqa: F401
from test_gpu_block_device import Shell

pytestmark = pytest.mark.gpu
LONGEST = [1, 8, 1000]                                      # tiles of 16, 32 and 128 rows, at 4 heads of queries for one


def shells(dtype):
    cache = [Shell(3, 2, 16, 64, dtype=dtype), Shell(3, 2, 16, 64, dtype=dtype)]
    return cache + ([Shell(3, 2, 16, dtype=torch.float32) for _ in range(2)] if dtype == I8 else [None, None])


@pytest.mark.parametrize("dtype", [BF16, I8], ids=["16 bits", "8 bits"])
@pytest.mark.parametrize("name", ["append", "read", "attend"])
def test_tensors_of_another_device(A, name, dtype):  # noqa: F811
    table, lengths = Shell(2, 3, dtype=torch.int32), Shell(2, dtype=torch.int32)
    cache, rows = A.Cache(*shells(dtype)), Shell(2, 2, 64)
    call = {"append": lambda: A.append(cache, table, lengths, rows, rows), "read": lambda: A.read(cache, table, lengths),
            "attend": lambda: A.attend(rows, cache, table, lengths)}[name]
    with pytest.raises(ValueError, match="current device"):
        call()


def sound(A, dtype=BF16):  # noqa: F811
    g = gen("sound")
    batch = ref.Batch(g, [(1, 40), (1, 50)], 16)
    cache = on_gpu(A, make_cache(g, batch, 2, 64, BF16, dtype == I8))
    return cache, batch.table.cuda(), batch.lengths.cuda(), *(normal(g, 2, n, 64, dtype=BF16).cuda() for n in (4, 2, 2))


@pytest.mark.parametrize("one", ["table", "lengths", "k", "q", "keys"])
def test_one_tensor_of_another_device(A, one):  # noqa: F811
    cache, table, lengths, q, k, v = sound(A)
    if one == "keys":
        cache = cache._replace(values=Shell(*cache.values.shape))
    args = dict(table=table, lengths=lengths, q=q, k=k)
    if one in args:
        args[one] = Shell(*args[one].shape, dtype=args[one].dtype)
    calls = [lambda: A.append(cache, args["table"], args["lengths"], args["k"], v, args["q"])]
    if one != "k":
        calls.append(lambda: A.attend(args["q"], cache, args["table"], args["lengths"]))
    if one not in ("k", "q"):
        calls.append(lambda: A.read(cache, args["table"], args["lengths"]))
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_tensors_that_require_gradients(A):  # noqa: F811
    cache, table, lengths, q, k, v = sound(A)
    packed = sound(A, I8)[0]
    f, slopes = torch.ones(32, device="cuda"), torch.ones(4, device="cuda")
    out, rows = torch.empty_like(q), torch.empty_like(k)

    def tracked(t):
        return t.clone().requires_grad_()

    calls = {
        "q": [lambda: A.attend(tracked(q), cache, table, lengths), lambda: A.append(cache, table, lengths, k, v, tracked(q))],
        "k": [lambda: A.append(cache, table, lengths, tracked(k), v), lambda: A.read(cache, table, lengths, out=(tracked(k), rows))],
        "v": [lambda: A.append(cache, table, lengths, k, tracked(v)), lambda: A.read(cache, table, lengths, out=(rows, tracked(v)))],
        "frequencies": [lambda: A.append(cache, table, lengths, k, v, frequencies=tracked(f))],
        "slopes": [lambda: A.attend(q, cache, table, lengths, slopes=tracked(slopes))],
        "out": [lambda: A.attend(q, cache, table, lengths, out=tracked(out)), lambda: A.append(cache, table, lengths, k, v, q, out=tracked(out))],
    }
    for field in ("keys", "values", "key_step", "value_step"):
        from_ = packed if "step" in field else cache
        other = from_._replace(**{field: tracked(getattr(from_, field))})
        calls[field] = [lambda c=other: A.append(c, table, lengths, k, v), lambda c=other: A.read(c, table, lengths),
                        lambda c=other: A.attend(q, c, table, lengths)]
    for name, of in calls.items():
        for call in of:
            with pytest.raises(ValueError, match=f"^{name} requires gradients"):
                call()
            with torch.no_grad():
                call()


@pytest.mark.parametrize("longest", LONGEST)
@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
def test_ends_of_scale_and_cap(A, packed, longest):  # noqa: F811
    g = gen("ends")
    batch = ref.Batch(g, [(2, 90), (5, 300)], 16)
    cache = make_cache(g, batch, 1, 64, BF16, packed)
    q = normal(g, batch.rows, 4, 64, dtype=BF16)
    for kw in (dict(cap=2.0 ** 60), dict(cap=2.0 ** -60), dict(scale=2.0 ** -60), dict(scale=2.0 ** 60, cap=2.0 ** -60), dict(scale=2.0 ** 60, cap=3.0),
               dict(scale=-2.0 ** -60, cap=2.0 ** 60)):
        run_attend(A, q, batch, cache, longest=longest, name=str(kw), **kw)


@pytest.mark.parametrize("longest", LONGEST)
def test_the_largest_pages(A, longest):  # noqa: F811
    g = gen("large pages")
    batch = ref.Batch(g, [(1, 65536), (3, 65538), (40, 60)], 65536)
    cache = make_cache(g, batch, 1, 16, BF16, False)
    q = normal(g, batch.rows, 4, 16, dtype=BF16)
    run_attend(A, q, batch, cache, longest=longest, window=700)
    k = normal(g, batch.rows, 2, 16, dtype=BF16)[:, :1]
    on, table, lengths, starts = on_gpu(A, cache), batch.table.cuda(), batch.lengths.cuda(), batch.starts.cuda()
    A.append(on, table, lengths, k.cuda(), -k.cuda(), starts=starts)
    got = A.read(on, table, lengths, starts=starts, rows=batch.rows)
    assert torch.equal(got[0].cpu(), k) and torch.equal(got[1].cpu(), -k)


@pytest.mark.parametrize("how", ["heads first", "columns", "odd"])
@pytest.mark.parametrize("longest", LONGEST)
@pytest.mark.parametrize("D", [80, 128])
def test_outputs_of_other_strides(A, D, longest, how):  # noqa: F811
    g = gen("strided")
    batch = ref.Batch(g, [(1, 90), (9, 500), (2, 2)], 32)
    cache = make_cache(g, batch, 2, D, BF16, False)
    q = normal(g, batch.rows, 8, D, dtype=BF16)
    put = (on_gpu(A, cache), batch.table.cuda(), batch.lengths.cuda())
    starts = batch.starts.cuda()
    want = A.attend(q.cuda(), *put, starts=starts, longest=longest)
    out = spread(torch.full_like(q, 9.0), how)
    A.attend(spread(q, how), *put, starts=starts, longest=longest, out=out)
    assert torch.equal(out, want)
    if how != "heads first":                                # what lies beside the columns is as it was
        base = out._base if out._base is not None else out
        assert base.isnan().sum() == (16 if how == "columns" else 6) * batch.rows
    k = normal(g, batch.rows, 2, D, dtype=BF16)
    turned = spread(torch.full_like(q, 9.0), how)
    f = torch.rand(D // 2, generator=g).cuda()
    plain = A.append(*put, k.cuda(), k.cuda(), q.cuda(), starts=starts, frequencies=f)
    A.append(*put, spread(k, how), spread(k, how), spread(q, how), starts=starts, frequencies=f, out=turned)
    assert torch.equal(turned, plain)
    to = tuple(spread(torch.full_like(k, 9.0), how) for _ in range(2))
    for got, same in zip(A.read(*put, starts=starts, rows=batch.rows, out=to), A.read(*put, starts=starts, rows=batch.rows)):
        assert torch.equal(got, same)


@pytest.mark.parametrize("longest", LONGEST)
def test_rows_and_heads_that_are_one_in_memory(A, longest):  # noqa: F811
    g = gen("expanded")
    batch = ref.Batch(g, [(1, 90), (9, 500)], 32)
    cache = make_cache(g, batch, 2, 64, BF16, False)
    put = (on_gpu(A, cache), batch.table.cuda(), batch.lengths.cuda())
    starts = batch.starts.cuda()
    for q in (normal(g, 1, 8, 64, dtype=BF16).cuda().expand(batch.rows, 8, 64), normal(g, batch.rows, 1, 64, dtype=BF16).cuda().expand(batch.rows, 8, 64)):
        assert torch.equal(A.attend(q, *put, starts=starts, longest=longest), A.attend(q.contiguous(), *put, starts=starts, longest=longest))
        with pytest.raises(Exception, match="overlap"):
            A.attend(q, *put, starts=starts, longest=longest, out=torch.empty_like(q[:1]).expand(q.shape))


@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
@pytest.mark.parametrize("longest", LONGEST)
def test_shared_pages(A, longest, packed):  # noqa: F811
    """Sequences with the same first pages, one whose pages are one page, and a sequence twice."""
    g = gen("shared")
    batch = ref.Batch(g, [(2, 200), (3, 180), (1, 130), (2, 200)], 16)
    batch.table[1, :10] = batch.table[0, :10]
    batch.table[2] = batch.table[2, 0]
    batch.table[3] = batch.table[0]
    cache = make_cache(g, batch, 2, 128, BF16, packed)
    q = normal(g, batch.rows, 8, 128, dtype=BF16)
    run_attend(A, q, batch, cache, longest=longest)


@pytest.mark.parametrize("longest", LONGEST)
def test_lengths_beyond_the_table(A, longest):  # noqa: F811
    g = gen("beyond")
    batch = ref.Batch(g, [(2, 160), (3, 160)], 16)
    cache = make_cache(g, batch, 2, 64, BF16, False)
    q = normal(g, batch.rows, 4, 64, dtype=BF16).cuda()
    put = (on_gpu(A, cache), batch.table[:, :10].contiguous().cuda())
    starts = batch.starts.cuda()
    a, b = (A.attend(q, *put, torch.tensor(n, dtype=torch.int32).cuda(), starts=starts, longest=longest) for n in ([160, 160], [161, 2 ** 31 - 1]))
    assert torch.equal(a, b)


def test_two_at_once(A):  # noqa: F811
    """Calls on two streams that may overlap, each with a workspace of its own, as calls without one have."""
    g = gen("at once")
    batch = ref.Batch(g, [(1, 9000), (1, 3000), (1, 50)], 64)
    cache = make_cache(g, batch, 2, 128, BF16, False)
    on, table, lengths = on_gpu(A, cache), batch.table.cuda(), batch.lengths.cuda()
    qs = [normal(g, 3, 8, 128, dtype=BF16) for _ in range(2)]
    gpu = [q.cuda() for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(A.attend(gpu[i], on, table, lengths))
    torch.cuda.synchronize()
    for q, of in zip(qs, got):
        want, slack = ref.attend(q, batch, cache, 128 ** -0.5)
        ref.check("at once", of[0], want, slack)
        assert all(torch.equal(o, of[0]) for o in of)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
def test_graphs_that_share_a_workspace(A, dtype):  # noqa: F811
    """Single tokens, a tree and a prompt in three graphs with one workspace, replayed in turn on one stream with eager calls between."""
    g = gen("one workspace")
    batch = ref.Batch(g, [(1, 3000), (1, 900)], 32)
    wide = ref.Batch(g, [(6, 3000), (6, 900)], 32)
    long = ref.Batch(g, [(300, 3000), (80, 900)], 32)
    workspace = torch.full((1 << 28,), 255, dtype=torch.uint8, device="cuda")
    calls = []
    for b, kw in ((batch, {}), (wide, dict(tree=torch.randint(0, 64, (12, 1), generator=g).cuda(), longest=6)), (long, {})):
        cache, q = on_gpu(A, make_cache(g, b, 2, 128, dtype, False)), normal(g, b.rows, 8, 128, dtype=dtype).cuda()
        put = (cache, b.table.cuda(), b.lengths.cuda())
        calls.append(lambda q=q, put=put, starts=b.starts.cuda(), kw=kw, **more: A.attend(q, *put, starts=starts, **kw, **more))
    want = [call() for call in calls]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for call in calls:
            call(workspace=workspace)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for call in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call(workspace=workspace))
        graphs.append(graph)
    for order in ((0, 1, 2), (2, 0, 1), (1, 1, 0, 2), (0, 2, 2, 1)):
        for i in order:
            outs[i].fill_(math.nan)
            graphs[i].replay()
            again = calls[i](workspace=workspace)
            assert torch.equal(again, want[i])
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
@pytest.mark.parametrize("longest", LONGEST)
def test_the_longest_sequences(A, longest, packed):  # noqa: F811
    """2^30 rows on one page: the last ones through a window as where the sequence is short, and all of them with equal weights."""
    g = gen("longest")
    page, D, most = 65536, 64, 1 << 30
    keys, values, key_step, value_step = make_cache(g, ref.Batch(g, [(1, page)], page, spare=0), 1, D, BF16, packed)
    cache = on_gpu(A, (keys, values, key_step, value_step))
    q = normal(g, 9, 4, D, dtype=BF16).cuda()
    starts = torch.tensor([0, 4, 9], dtype=torch.int32).cuda()
    table = torch.zeros(2, most // page, dtype=torch.int32).cuda()
    none = torch.zeros(2, dtype=torch.int32).cuda()
    long, short = (torch.tensor([n, n - 70000], dtype=torch.int32).cuda() for n in (most, 4 * page))
    for window in (1, 700):
        for prefix in (None, none):                         # with one the window says nothing about how much is seen
            a = A.attend(q, cache, table, long, starts=starts, longest=longest, window=window, prefix=prefix)
            b = A.attend(q, cache, table[:, :4].contiguous(), short, starts=starts, longest=longest, window=window, prefix=prefix)
            # sums in another order: a rounding of the output and of each weight, and n roundings of each of two sums
            assert ((a.double() - b.double()).abs() <= (4 * 2.0 ** -8 + 2 * window * 2.0 ** -24) * values_of(values, value_step).abs().max()).all()
    got = A.attend(torch.zeros_like(q[:1]), cache, table[:1], long[:1], starts=starts[:2].clamp(max=1), longest=longest)
    mean = values_of(values, value_step).mean(0)
    # at most 2^30 / 512 keys are summed one after the other, and the weight times a step is rounded once
    slack = mean.abs() * 2.0 ** -8 + (2.0 ** -8 + 2.0 ** 21 * 2.0 ** -24) * values_of(values, value_step).abs().mean(0)
    assert ((got.double().cpu() - mean).abs() <= slack).all()


def values_of(values, step):
    """[rows, D] in binary64 of a page of one head."""
    v = values[0, 0].double()
    return v if step is None else v * step[0, 0].double()[:, None]


@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
def test_the_most_rows(A, packed):  # noqa: F811
    """2^20 rows of a call: a sequence's, of which each sees itself only, and of as many sequences of one row."""
    most, D = 1 << 20, 16
    g = torch.Generator("cuda").manual_seed(7)
    k, v, q = (torch.randn(most, n, D, generator=g, device="cuda").to(BF16) for n in (1, 1, 2))
    for S, page in ((1, 4096), (most, 16)):
        pages = most // page if S == 1 else 1024
        cache = A.make_cache(pages, 1, page, D, I8 if packed else BF16)
        n = most // S
        starts = (torch.arange(S + 1, dtype=torch.int32) * n).cuda()
        lengths = torch.full((S,), n, dtype=torch.int32).cuda()
        if S == 1:
            table = torch.randperm(pages, generator=g, device="cuda").int()[None].contiguous()
            assert torch.equal(A.append(cache, table, lengths, k, v, q, starts=starts), q)
        else:                                               # pages are shared, so they are written through a table of their own
            table = (torch.arange(S, device="cuda") % pages).int()[:, None].contiguous()
            A.append(cache, table[:pages].contiguous(), lengths[:pages], k[:pages].contiguous(), v[:pages].contiguous())
        own = A.read(cache, table, lengths, starts=starts, rows=most, dtype=BF16)[1].expand(most, 2, D)
        for longest in (n, 1):
            got = A.attend(q, cache, table, lengths, starts=starts, longest=longest, window=1)
            # one weight of 1 times the row's step, or a value times its step: rounded, and the output too
            assert ((got.double() - own.double()).abs() <= 2.0 ** -7 * own.double().abs() + 1e-30).all()
    assert torch.equal(A.attend(q, cache, table, lengths), A.attend(q, cache, table, lengths, starts=starts, longest=1))
