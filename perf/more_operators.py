"""Timed cases of the operators around a paged cache of keys and values, in the elements' own type or in 8-bit rows.

New rows of a batch of sequences are appended to the cache with their position's rotation on the way, and read back;
queries attend over the cache: one token of each sequence, a tree of drafted tokens, and prompts, with scores capped by a
tanh, a bias that grows with the distance, a window and a prefix that everything sees.  With `own` false `run` computes
them by elementary torch operations in 32 bits over a padded batch, otherwise by the framework's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _append(name, S, new, context, H, G, D, page, dtype, packed=False, rotated=None, interleaved=False, far=0, ragged=False):
    """S sequences of up to `new` new rows each after up to `context` kept ones (`ragged`: fewer in all but the first);
    `rotated` channels of a head turn by their position (None: all); `far`: positions begin there, not at the row's place."""
    return dict(name=name, kind="append", S=S, new=new, context=context, H=H, G=G, D=D, page=page, dtype=dtype, packed=packed,
                rotated=D if rotated is None else rotated, interleaved=interleaved, far=far, ragged=ragged)


def _attend(name, S, new, context, H, G, D, page, dtype, packed=False, cap=0.0, slopes=False, window=0, prefix=0, tree=False,
            ragged=False):
    """`prefix`: so many first rows of each sequence are seen by all of its rows."""
    return dict(name=name, kind="attend", S=S, new=new, context=context, H=H, G=G, D=D, page=page, dtype=dtype, packed=packed,
                cap=cap, slopes=slopes, window=window, prefix=prefix, tree=tree, ragged=ragged)


def listed():
    return [
        # one request decodes: its token's key and value enter the cache, its query is rotated
        _append("append_token", 1, 1, 1000, 32, 8, 128, 64, "bf16"),
        # a batch that decodes, with an 8-bit cache; the rows are read back
        _append("append_decode_packed", 64, 1, 2047, 32, 8, 128, 64, "bf16", packed=True, ragged=True),
        # prompts of three requests, of no round length, into an 8-bit cache, and read back
        _append("append_prompts_packed", 3, 2047, 0, 32, 8, 128, 64, "bf16", packed=True, ragged=True),
        # one request decodes after a short prompt
        _attend("attend_token", 1, 1, 1000, 32, 8, 128, 64, "bf16"),
        # a batch that decodes, sequences of very different lengths
        _attend("attend_decode", 64, 1, 8191, 32, 8, 128, 64, "bf16", ragged=True),
        # one long document, 8-bit cache
        _attend("attend_long_packed", 1, 1, 131071, 32, 8, 128, 256, "bf16", packed=True),
        # wide heads with capped scores and a window, half precision, small pages
        _attend("attend_capped_window", 16, 1, 8000, 16, 8, 256, 16, "f16", cap=50.0, window=1024, ragged=True),
        # a tree of drafted tokens of one request
        _attend("tree_one", 1, 63, 4000, 32, 8, 128, 64, "bf16", tree=True),
        # trees of a batch, of different sizes, 8-bit cache
        _attend("tree_batch_packed", 16, 26, 4095, 32, 8, 128, 64, "bf16", packed=True, tree=True, ragged=True),
        # one prompt of a fresh request
        _attend("prompt", 1, 4096, 0, 32, 8, 128, 64, "bf16"),
        # prompts of three requests of odd lengths, a bias by distance and heads of 80 channels
        _attend("prompts_sloped", 3, 1155, 515, 12, 12, 80, 32, "f16", slopes=True, ragged=True),
        # a part of a long prompt after what the cache holds in 8 bits; capped, and half of the part is a prefix
        _attend("prompt_part_packed", 1, 1024, 7169, 32, 8, 128, 64, "bf16", packed=True, cap=30.0, prefix=7681),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    D = rng.choice((16, 32, 48, 64, 64, 80, 96, 112, 128, 128, 128, 160, 192, 256))
    G = _log(rng, 1, 16)
    H = G * rng.choice((1, 1, 2, 3, 4, 4, 5, 7, 8))
    page, dtype, packed = rng.choice((16, 32, 64, 128, 256)), rng.choice(("bf16", "bf16", "f16")), rng.random() < 0.5
    kind = rng.choice(("append", "append", "token", "token", "token", "tree", "tree", "prompt", "prompt"))
    ragged = rng.random() < 0.7
    if kind == "append":
        T = _log(rng, 1, max(1, min(4096, 16_000_000 // ((H + 2 * G) * D))))
        S = _log(rng, 1, min(T, 64))
        c = _append("", S, max(1, T // S), _log(rng, 1, 2000), H, G, D, page, dtype, packed, rng.choice((D, D, D // 32 * 16, 0)),
                    rng.random() < 0.3, rng.choice((0, 0, 1_000_003)), ragged)
    else:
        shape = dict(cap=rng.choice((0.0, 0.0, 0.0, 30.0)), ragged=ragged)
        if kind != "tree":
            shape.update(slopes=rng.random() < 0.3, window=rng.choice((0, 0, 0, _log(rng, 1, 4096))))
        if kind == "token":
            S = _log(rng, 1, 64)
            new, context = 1, _log(rng, 1, min(131071, 250_000_000 // (S * G * D)))
        elif kind == "tree":
            S, new = _log(rng, 1, 16), rng.randint(2, 100)
            context = _log(rng, 1, min(32768, 100_000_000 // (S * G * D), 400_000_000 // (S * new * H)))
            shape.update(tree=True)
        else:
            S, new = rng.choice((1, 1, 2, 3, 5)), _log(rng, 2, 2048)
            context = _log(rng, 1, max(1, min(16384, 100_000_000 // (S * G * D), 400_000_000 // (S * new * H) - new)))
            shape.update(prefix=rng.choice((0, 0, new // 2, context + new // 2)))
        c = _attend("", S, new, context, H, G, D, page, dtype, packed, **shape)
    del c["name"]
    return c


def _sizes(case):
    """(new rows, all rows) of each sequence: those of the first as the case says, of the others spread below where ragged."""
    def spread(most, i):
        return most if i == 0 or not case["ragged"] else int(most * ((i * 0.6180339887) % 1.0))

    new = [max(1, spread(case["new"], i)) for i in range(case["S"])]
    return [(n, n + spread(case["context"], i + 1 if i else 0)) for i, n in enumerate(new)]


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _pack_plain(x):
    """Codes and step of each row of the last dimension: rne(x * (127 / absmax)), absmax / 127."""
    a = x.abs().amax(-1, keepdim=True)
    most = torch.full_like(a, 127.0)
    return torch.round(x * torch.where(a > 0, most / a, torch.zeros_like(a))).to(torch.int8), (a / most).squeeze(-1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale)

    def channels(*shape):
        """Sizes of channels, a few of which stand out, as keys have them."""
        size = normal(*shape, scale=0.4).exp_()
        size[torch.rand(shape, generator=gen, device="cuda") < 0.02] *= 5.0
        return size

    H, G, D, P, dtype = case["H"], case["G"], case["D"], case["page"], _TYPES[case["dtype"]]
    sizes = _sizes(case)
    T, S = sum(n for n, _ in sizes), len(sizes)
    used = [-(-length // P) for _, length in sizes]
    # pages lie in no order; what a sequence does not need of its table is not set
    pages = sum(used) + 3
    order = torch.randperm(pages, generator=host, dtype=torch.int64).to(torch.int32)
    table = torch.full((S, max(used)), -1, dtype=torch.int32)
    at = 0
    for i, u in enumerate(used):
        table[i, :u] = order[at:at + u]
        at += u
    starts = torch.zeros(S + 1, dtype=torch.int64)
    starts[1:] = torch.tensor([n for n, _ in sizes]).cumsum(0)
    s = dict(kind=case["kind"], dtype=dtype, page=P, D=D, packed=case["packed"], table=table.cuda(),
             lengths=torch.tensor([length for _, length in sizes], dtype=torch.int32).cuda(),
             starts=starts.to(torch.int32).cuda(), longest=max(n for n, _ in sizes), most=max(length for _, length in sizes),
             one_each=all(n == 1 for n, _ in sizes), key_step=None, value_step=None)
    key_size = channels(G, D)
    keys = normal(pages, G, P, D).mul_(key_size[:, None])
    values = normal(pages, G, P, D).mul_(0.5).add_(normal(G, 1, D, scale=0.5))
    if case["packed"]:
        (keys, s["key_step"]), (values, s["value_step"]) = _pack_plain(keys), _pack_plain(values)
    else:
        keys, values = keys.to(dtype), values.to(dtype)
    s["keys"], s["values"] = keys, values
    if case["kind"] == "append":
        # q, k and v as one projection leaves them: columns of one matrix
        rows = normal(T, (H + 2 * G) * D)
        rows[:, H * D:(H + G) * D] *= key_size.view(-1)
        rows = rows.to(dtype)
        s["q"], s["k"], s["v"] = (t.view(T, -1, D) for t in rows.split((H * D, G * D, G * D), 1))
        R = case["rotated"]
        s["frequencies"] = (10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).float().cuda() if R else None
        s["interleaved"], s["positions"] = case["interleaved"], None
        if case["far"]:
            s["positions"] = (case["far"] + torch.randint(0, 4096, (T,), generator=gen, device="cuda")).to(torch.int32)
        return s
    # scores of about unit size times 1.5, whatever the heads' width
    s["scale"] = D ** -0.5
    norm = key_size.square().mean(1).sqrt().repeat_interleave(H // G)
    s["q"] = normal(T, H, D).mul_(1.5 / norm[:, None]).to(dtype)
    s["cap"], s["window"] = case["cap"], case["window"]
    s["slopes"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H) if case["slopes"] else None
    s["prefix"] = torch.full((S,), case["prefix"], dtype=torch.int32, device="cuda") if case["prefix"] else None
    s["tree"] = None
    if case["tree"]:
        # each drafted token continues one before it, or the last kept token, and sees those that it continues and itself
        words = -(-case["new"] // 64)
        bits = torch.zeros(T, 64 * words, dtype=torch.bool)
        at = 0
        for n, _ in sizes:
            for j, parent in enumerate(torch.rand(n, generator=host).mul_(torch.arange(n) + 1).long().tolist()):
                if parent:
                    bits[at + j] = bits[at + parent - 1]
                bits[at + j, j] = True
            at += n
        power = torch.ones(64, dtype=torch.int64) << torch.arange(64)
        s["tree"] = (bits.view(T, words, 64).long() * power).sum(2).cuda()
    return s


# --------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------
def _places(s, T):
    """Sequence, number among its sequence's new rows, and slot of each row."""
    row = torch.arange(T, device=s["starts"].device)
    of = torch.searchsorted(s["starts"].long(), row, right=True) - 1
    among = row - s["starts"].long()[of]
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    return of, among, (s["lengths"].long() - new)[of] + among


def _rotate_plain(x, cos, sin, interleaved):
    """x [T, heads, D] in 32 bits, cos and sin [T, R / 2]: pairs of the first R channels turn."""
    half = cos.shape[1]
    turning, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (turning[..., 0::2], turning[..., 1::2]) if interleaved else (turning[..., :half], turning[..., half:])
    cos, sin = cos[:, None], sin[:, None]
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((turned, rest), -1)


def _append_plain(s):
    of, _, slot = _places(s, s["k"].shape[0])
    page, place = s["table"][of, slot // s["page"]].long(), slot % s["page"]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if s["frequencies"] is not None:
        where = slot if s["positions"] is None else s["positions"]
        angle = where.double()[:, None] * s["frequencies"].double()
        cos, sin = angle.cos().float(), angle.sin().float()
        q, k = _rotate_plain(q, cos, sin, s["interleaved"]), _rotate_plain(k, cos, sin, s["interleaved"])
    q = q.to(s["dtype"])
    if not s["packed"]:
        s["keys"][page, :, place] = k.to(s["dtype"])
        s["values"][page, :, place] = v.to(s["dtype"])
        return q, s["keys"], s["values"]
    (k, k_step), (v, v_step) = _pack_plain(k), _pack_plain(v)
    s["keys"][page, :, place], s["key_step"][page, :, place] = k, k_step
    s["values"][page, :, place], s["value_step"][page, :, place] = v, v_step
    read = (s["keys"], s["key_step"]), (s["values"], s["value_step"])
    return q, *((c[page, :, place].float() * step[page, :, place][..., None]).to(s["dtype"]) for c, step in read)


def _attend_plain(s):
    """All sequences as long as the longest, with as many rows as the one with most: what is too much is masked."""
    T, H, D = s["q"].shape
    S, P, most, longest = s["lengths"].shape[0], s["page"], s["most"], s["longest"]
    G = s["keys"].shape[1]
    slot = torch.arange(most, device=s["q"].device)
    page = s["table"][:, slot // P].long().clamp_(min=0)

    def cached(rows, step):
        x = rows[page, :, slot % P].float()
        if step is not None:
            x = x * step[page, :, slot % P][..., None]
        return x.transpose(1, 2)                                     # [S, G, most, D]

    first = s["starts"][:-1].long()
    new = s["starts"][1:].long() - first
    among = torch.arange(longest, device=slot.device)
    row = (first[:, None] + among).clamp_(max=T - 1)                 # [S, longest]
    q = s["q"].float()[row].view(S, longest, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(S, G, -1, D)
    score = (q @ cached(s["keys"], s["key_step"]).transpose(2, 3)).mul_(s["scale"]).view(S, H, longest, most)
    if s["cap"]:
        score = score.div_(s["cap"]).tanh_().mul_(s["cap"])
    kept = s["lengths"].long() - new
    mine = (kept[:, None] + among)[:, :, None]                       # [S, longest, 1]
    if s["tree"] is not None:
        drafted = (slot - kept[:, None])[:, None, :]                 # [S, 1, most]
        word = (drafted // 64).clamp(0, s["tree"].shape[1] - 1).expand(S, longest, most)
        bit = s["tree"][row].gather(2, word) >> drafted.clamp(min=0).remainder(64) & 1
        seen = (drafted < 0) | (bit != 0)
    else:
        seen = slot <= mine
        if s["window"]:
            seen = seen & (mine - slot < s["window"])
        if s["prefix"] is not None:
            seen = seen | (slot < s["prefix"][:, None, None])
    seen = seen & (slot < s["lengths"][:, None, None])
    if s["slopes"] is not None:
        score = score.sub_(s["slopes"][:, None, None] * (mine - slot).abs().float()[:, None])
    score = score.masked_fill_(~seen[:, None], -math.inf)
    top = score.amax(3, keepdim=True)
    weight = score.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = weight.sum(3, keepdim=True)
    out = (weight.view(S, G, -1, most) @ cached(s["values"], s["value_step"])).view(S, H, longest, D)
    out = out / torch.where(total > 0, total, torch.ones_like(total))
    of, among, _ = _places(s, T)
    return out[of, :, among].to(s["dtype"])


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    s = state
    if own:
        from paper_2002_00104_amd import attention
        cache = attention.Cache(s["keys"], s["values"], s["key_step"], s["value_step"])
        starts = None if s["one_each"] else s["starts"]
        if s["kind"] == "append":
            q = attention.append(cache, s["table"], s["lengths"], s["k"], s["v"], s["q"], starts=starts,
                                 positions=s["positions"], frequencies=s["frequencies"], interleaved=s["interleaved"])
            if not s["packed"]:
                return q, s["keys"], s["values"]
            return q, *attention.read(cache, s["table"], s["lengths"], starts=starts, rows=q.shape[0], dtype=s["dtype"])
        return attention.attend(s["q"], cache, s["table"], s["lengths"], starts=starts, longest=s["longest"],
                                scale=s["scale"], cap=s["cap"], slopes=s["slopes"], window=s["window"],
                                prefix=s["prefix"], tree=s["tree"])
    return _append_plain(s) if s["kind"] == "append" else _attend_plain(s)


def _seen(case, n, length):
    """Pairs of a query row and a key that it sees, and the first key that any row sees, for one sequence."""
    kept = length - n
    if case["tree"]:
        return n * kept + n * (n + 1) // 4, 0           # a drafted token sees less than half of the others
    pairs, first = 0, length
    for j in range(n):
        own_slot = kept + j
        lo = max(0, own_slot - case["window"] + 1) if case["window"] else 0
        prefix = min(case["prefix"], length)
        pairs += own_slot + 1 - lo + min(prefix, lo) + max(0, prefix - own_slot - 1)
        first = min(first, 0 if prefix else lo)
    return pairs, first


def work(case):
    sizes = _sizes(case)
    T, H, G, D = sum(n for n, _ in sizes), case["H"], case["G"], case["D"]
    kept = D + 4 if case["packed"] else 2 * D            # a row of one head in the cache
    if case["kind"] == "append":                         # q, k, v in; q and the cache's rows out (8 bits: read, and out again)
        again = 2 * G * (kept + 2 * D) if case["packed"] else 0
        return {"bytes": T * (4 * H * D + 4 * G * D + 2 * G * kept + again), "flops": T * (3 * (H + G) + 4 * G) * D}
    seen = [_seen(case, n, length) for n, length in sizes]
    rows = sum(length - first for (_, first), (_, length) in zip(seen, sizes))
    tree = T * 8 * -(-case["new"] // 64) if case["tree"] else 0
    return {"bytes": 4 * T * H * D + 2 * G * rows * kept + tree, "flops": 4 * H * D * sum(p for p, _ in seen)}


# --------------------------------------------------------------------------
# the definitions in binary64
# --------------------------------------------------------------------------
def _pack_exact(x):
    step = x.abs().max(dim=-1, keepdim=True).values / 127.0
    return (x / torch.where(step > 0, step, torch.ones_like(step))).round() * step


def _turn_exact(x, angle, interleaved):
    """Each pair of channels as a complex number."""
    R = 2 * angle.shape[1]
    order = torch.arange(R, device=x.device).view(-1, 2) if interleaved else torch.arange(R, device=x.device).view(2, -1).t()
    y = x.clone()
    pair = torch.complex(x[:, :, order[:, 0]], x[:, :, order[:, 1]]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    y[:, :, order[:, 0]], y[:, :, order[:, 1]] = pair.real, pair.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    sizes = [(n, length) for n, length in _sizes(case)]
    P, H, G, D = case["page"], case["H"], case["G"], case["D"]
    table = s["table"].tolist()
    if case["kind"] == "append":
        slots = [(i, slot) for i, (n, length) in enumerate(sizes) for slot in range(length - n, length)]
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        if s["frequencies"] is not None:
            at = s["positions"].double() if case["far"] else torch.tensor([slot for _, slot in slots], dtype=torch.float64, device=q.device)
            angle = torch.outer(at, s["frequencies"].double())
            q, k = _turn_exact(q, angle, case["interleaved"]), _turn_exact(k, angle, case["interleaved"])
        if case["packed"]:
            return q, _pack_exact(k), _pack_exact(v)
        keys, values = s["keys"].double(), s["values"].double()
        page = torch.tensor([table[i][slot // P] for i, slot in slots], device=q.device)
        place = torch.tensor([slot % P for _, slot in slots], device=q.device)
        keys[page, :, place], values[page, :, place] = k, v
        return q, keys, values
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    row = 0
    for i, (n, length) in enumerate(sizes):
        if length == 0:
            row += n
            continue
        pages = torch.tensor(table[i][:-(-length // P)], device=out.device)
        slot = torch.arange(length, device=out.device)
        own_slot = torch.arange(length - n, length, device=out.device)[:, None]
        if case["tree"]:
            word = s["tree"][row:row + n]
            seen = torch.ones(n, length, dtype=torch.bool, device=out.device)
            for j in range(n):
                seen[:, length - n + j] = (word[:, j // 64] >> (j % 64)) % 2 != 0
        else:
            seen = slot <= own_slot
            if case["window"]:
                seen = seen & (slot > own_slot - case["window"])
            if case["prefix"]:
                seen[:, :case["prefix"]] = True
        for g in range(G):
            k, v = s["keys"][pages, g].double(), s["values"][pages, g].double()
            if case["packed"]:
                k, v = k * s["key_step"][pages, g].double()[..., None], v * s["value_step"][pages, g].double()[..., None]
            k, v = k.reshape(-1, D)[:length], v.reshape(-1, D)[:length]
            for h in range(g * (H // G), (g + 1) * (H // G)):
                score = torch.mm(s["q"][row:row + n, h].double(), k.t()) * s["scale"]
                if case["cap"]:
                    score = torch.tanh(score / case["cap"]) * case["cap"]
                if case["slopes"]:
                    score = score - float(s["slopes"][h]) * (own_slot - slot).abs()
                score[~seen] = -math.inf
                out[row:row + n, h] = torch.mm(torch.softmax(score, 1).nan_to_num(0.0), v)
        row += n
    return out
