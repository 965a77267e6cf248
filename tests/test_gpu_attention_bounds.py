"""What the slacks of the general tests leave open: capped scores to within a rounding of their own size, at the ends of the range too, and what lies around
the tensors of a call whose arrays on the device hold anything."""
import math

import pytest
import torch

import attention_ref as ref
from test_gpu_attention import A, BF16, F16, HEADS, gen, make_cache, normal, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu
LONGEST = [1, 8, 1000]                                      # tiles of 16, 32 and 128 rows, at 4 heads of queries for one


def capped(q, batch, cache, scale, cap, exact):
    """Output and slack in binary64.  A capped score is off by what the product is off (nothing where `exact`: small whole numbers), and by no more than
    twice the cap for that; by 2^-20 of itself for the cap's two forms; and by 2^-22 of the uncapped one, as far as that is below the cap, for two factors."""
    T, H, D = q.shape
    G = cache[0].shape[1]
    out, slack = (torch.zeros(T, H, D, dtype=torch.float64) for _ in range(2))
    unit = ref.UNIT[q.dtype] * (2 if cache[2] is not None and q.dtype == F16 else 1)
    for s, (n, length) in enumerate(batch.sizes):
        first = int(batch.starts[s])
        keys, values, _ = ref.sequence_rows(batch, cache, s)
        seen = ref.seen_by(batch, s, 0, None, None)
        for h in range(H):
            k, v, x = keys[:, h * G // H], values[:, h * G // H], q[first:first + n, h].double()
            plain = scale * (x @ k.T)
            score = cap * torch.tanh(plain / cap)
            off = torch.zeros_like(score) if exact else ((D + 8) * ref.U * abs(scale) * (x.abs() @ k.abs().T)).clamp(max=2 * cap)
            off = off + 2.0 ** -20 * score.abs() + 2.0 ** -22 * plain.abs().clamp(max=cap)
            p = torch.softmax(score.masked_fill(~seen, -math.inf), 1)
            out[first:first + n, h] = p @ v
            # a change of each score by at most e moves a weight's share by a factor of exp(2 e) at most
            e = off.masked_fill(~seen, 0.0).amax(1, keepdim=True)
            slack[first:first + n, h] = (p @ v.abs()) * (unit + torch.expm1(2 * e) + (2 * length + 8) * ref.U) + 2.0 ** -31 * v.abs().sum(0)
    return out, slack


def run(A, q, batch, cache, scale, cap, exact, name, longest):  # noqa: F811
    want, slack = capped(q, batch, cache, scale, cap, exact)
    starts, lengths = batch.starts.cuda(), batch.lengths.cuda()
    for table in (batch.table, torch.nn.functional.pad(batch.table, (0, 1250), value=-1)):
        got = A.attend(q.cuda(), on_gpu(A, cache), table.cuda(), lengths, starts=starts, scale=scale, cap=cap, longest=longest)
        ref.check(name, got, want, slack)
    return got, want


@pytest.mark.parametrize("longest", LONGEST)
@pytest.mark.parametrize("dtype,packed", [(BF16, False), (F16, False), (BF16, True), (F16, True)], ids=["bf16", "f16", "bf16 codes", "f16 codes"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_capped_scores(A, D, dtype, packed, longest):  # noqa: F811
    """From caps that almost all scores reach to caps that none comes near."""
    g = gen("capped", D)
    batch = ref.Batch(g, [(1, 300), (7, 200), (40, 60)], 16)
    cache = make_cache(g, batch, 2, D, dtype, packed)
    q = normal(g, batch.rows, 4, D, dtype=dtype, scale=2.0)
    for cap in (0.3, 2.0, 30.0, 1e6):
        run(A, q, batch, cache, D ** -0.5, cap, False, f"cap {cap}", longest)


@pytest.mark.parametrize("longest", LONGEST)
@pytest.mark.parametrize("dtype,packed", [(BF16, False), (F16, False), (BF16, True), (F16, True)], ids=["bf16", "f16", "bf16 codes", "f16 codes"])
def test_known_products(A, dtype, packed, longest):  # noqa: F811
    """Whole numbers, whose products are exact: both ends of scale and cap, where scores are two values and zero, or as without a cap."""
    g = gen("known")
    batch = ref.Batch(g, [(1, 300), (7, 200), (40, 60)], 16)
    D, shape = 64, (batch.pages, 1, 16)
    keys, values = (torch.randint(-3, 4, (*shape, D), generator=g).float() for _ in range(2))
    one = torch.ones(shape)
    cache = (keys.to(torch.int8), values.to(torch.int8), one, one) if packed else (keys.to(dtype), values.to(dtype), None, None)
    q = torch.randint(-2, 3, (batch.rows, 4, D), generator=g).to(dtype)
    results = []
    for scale, cap in ((2.0 ** 60, 3.0), (-2.0 ** 60, 3.0), (2.0 ** 60, 2.0 ** -60), (2.0 ** -60, 2.0 ** 60), (2.0 ** -5, 2.0 ** 60), (2.0 ** -5, 2.0 ** 20),
                       (2.0 ** -5, 0.5)):
        results.append(run(A, q, batch, cache, scale, cap, True, f"scale {scale} cap {cap}", longest))
    # these differ by more than their slacks: what is tested is seen
    assert (results[0][1] - results[1][1]).abs().max() > 0.5 and (results[0][1] - results[2][1]).abs().max() > 0.5


class Around:
    """A tensor within a larger one of which all else has one value."""

    def __init__(self, t, value, front=4096):
        size = t.numel()
        self.whole = torch.full((front + size + 4096,), value, dtype=t.dtype, device="cuda")
        self.t = self.whole[front:front + size].view(t.shape)
        self.t.copy_(t)
        self.front, self.value = front, value

    def check(self, name):
        n = self.t.numel()
        assert (self.whole[:self.front] == self.value).all() and (self.whole[self.front + n:] == self.value).all(), name


# starts and lengths of three sequences in 12 rows of a call, with tables of three pages of 16; and what rows these
# come to, (first, end, length), where no two sequences have the same
WILD = [([0, 4, 2, 12], [40, 40, 40], {}),
        ([-5, 4, 8, 99], [40, 2 ** 31 - 1, -9], {0: (0, 4, 40), 1: (4, 8, 48), 2: (8, 12, 0)}),
        ([9, 3, 3, 1], [0, 0, 0], {}),
        ([2 ** 31 - 1] * 4, [40] * 3, {}),
        ([-2 ** 31] * 4, [40] * 3, {}),
        ([-2 ** 31, 0, 12, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1, 1], {1: (0, 12, 48)})]


@pytest.mark.parametrize("longest", LONGEST)
@pytest.mark.parametrize("packed", [False, True], ids=["16 bits", "8 bits"])
@pytest.mark.parametrize("case", range(len(WILD)))
def test_around_the_tensors(A, case, packed, longest):  # noqa: F811
    starts, lengths, told = WILD[case]
    g = gen("around", case)
    batch = ref.Batch(g, [(4, 48)] * 3, 16)
    kept = make_cache(g, batch, 2, 64, BF16, packed)
    q, k = normal(g, 12, 4, 64, dtype=BF16), normal(g, 12, 2, 64, dtype=BF16)
    starts_on, lengths_on = (torch.tensor(t, dtype=torch.int32).cuda() for t in (starts, lengths))
    table = Around(batch.table, 2 ** 31 - 1)
    pools = [None if t is None else Around(t, 77) for t in kept]
    cache = A.Cache(*(None if p is None else p.t for p in pools))
    queries, out = Around(q, 9.0), Around(torch.full_like(q, 7.0), 9.0)
    A.attend(queries.t, cache, table.t, lengths_on, starts=starts_on, longest=longest, out=out.t)
    rows = [Around(torch.full_like(k, 7.0), 9.0) for _ in range(2)]
    A.read(cache, table.t, lengths_on, starts=starts_on, rows=12, out=tuple(r.t for r in rows))
    turned = Around(torch.full_like(q, 7.0), 9.0)
    new = Around(k, 9.0)
    before = [None if p is None else p.t.clone() for p in pools]
    for name, a in (("q", queries), ("out", out), ("k", rows[0]), ("v", rows[1]), ("table", table)):
        a.check(name)
    assert torch.equal(queries.t.cpu(), q) and all(b is None or torch.equal(b.cpu(), t) for b, t in zip(before, kept))
    batch.sizes = [(0, 0)] * 3
    for s, (a, b, length) in told.items():
        batch.sizes[s] = (b - a, length)
        batch.starts[s] = a
        # rows that are in the cache, as they are read from it
        for j in range(a, b):
            place = batch.where(s, length - (b - j), batch.pages)
            for i, r in enumerate(rows):
                want = torch.zeros(2, 64)
                if place:
                    want = kept[i][place[0], :, place[1]].float()
                    if packed:
                        want = want * kept[2 + i][place[0], :, place[1]][:, None]
                assert torch.equal(r.t[j].cpu(), want.to(BF16))
    if told:
        want, slack = ref.attend(q, batch, kept, 0.125)
        ref.check("out", out.t, want, slack)
    A.append(cache, table.t, lengths_on, new.t, new.t, queries.t, starts=starts_on, out=turned.t)
    for name, a in (("q", queries), ("turned", turned), ("new", new), ("table", table), *((f"pool {i}", p) for i, p in enumerate(pools) if p)):
        a.check(name)
    if case == 1:                                           # its first sequence's rows are on its third page
        page = int(batch.table[0, 0])
        assert all(b is None or torch.equal(b[page], p.t[page]) for b, p in zip(before, pools))
    assert torch.equal(queries.t.cpu(), q)
