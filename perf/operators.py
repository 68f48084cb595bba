"""The operators of an instance's prefix cache, their sizes and their plain forms.

The router sends a request to an instance because that instance holds the
keys and values of the request's prefix.  What the instance then does with
them is measured here: sequences fork from the cached prefix, grow and are
freed, pages are compacted, new tokens' queries and keys are normed, rotated
and appended, and attention reads the pages, a shared prefix once for all the
sequences that start with it.

Every case is a dict of plain values.  Lengths follow from the case alone (its
`lens` seeds them); values and the places of pages follow from prepare()'s
seed.  Copies are compared bit by bit, so they are returned as whole numbers.
"""

import math
import random

import torch

own = False
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}

ATTEND = dict(kind="attend", dtype="bf16", q_heads=32, kv_heads=8, dim=128, page=16, layout="heads", layers=1,
              seqs=4, groups=1, prefix_lo=256, prefix_hi=1024, own_lo=16, own_hi=1024, new_lo=1, new_hi=1, lens=1)
APPEND = dict(ATTEND, kind="append", groups=0, prefix_lo=0, prefix_hi=0, rot=128, interleaved=False)
STEP = dict(ATTEND, kind="step", rot=128, interleaved=False)
FORK = dict(kind="fork", dtype="bf16", kv_heads=8, dim=128, page=16, layout="heads", layers=4, pages=1024,
            parents=2, children=8, len_lo=256, len_hi=1024, add_lo=1, add_hi=64, lens=1)
COMPACT = dict(kind="compact", dtype="bf16", kv_heads=8, dim=128, page=16, layout="heads", layers=4, pages=512,
               seqs=8, shared=8, live=0.5, lens=1)


def listed():
    return [
        # Four requests of the tiny workload decode one token each behind a
        # common prefix: latency and launches.
        dict(ATTEND, name="attend_few", lens=11),
        # A decode step of the agent workload: 256 sequences behind 12
        # templates of 2,048-8,192 tokens, 100-1,000 tokens of their own.
        dict(ATTEND, name="attend_templates", dtype="f16", q_heads=64, seqs=256, groups=12, prefix_lo=2048,
             prefix_hi=8192, own_lo=100, own_hi=1000, lens=12),
        # Long contexts: a 16k prefix shared by eight sequences each, up to
        # 100k tokens of their own, few key heads: bandwidth.
        dict(ATTEND, name="attend_long", q_heads=16, kv_heads=2, seqs=16, groups=2, prefix_lo=16384,
             prefix_hi=16384, own_lo=16384, own_hi=100_000, lens=13),
        # Drafts of 0-8 tokens checked at once, a head of its own for every
        # query head, 64-token pages laid out token by token.
        dict(ATTEND, name="attend_drafts", dtype="f16", q_heads=12, kv_heads=12, dim=64, page=64, layout="tokens",
             seqs=96, groups=5, prefix_lo=1000, prefix_hi=4000, own_lo=0, own_hi=700, new_lo=0, new_hi=8, lens=14),
        # The uncached parts of 16 agent prompts, 100-1,000 tokens each,
        # behind cached templates: tensor work.
        dict(ATTEND, name="attend_prompts", seqs=16, groups=3, prefix_lo=2048, prefix_hi=8192, own_lo=0, own_hi=0,
             new_lo=100, new_hi=1000, lens=15),
        # Two layers of a decode step as a program runs it: one plan, then
        # norm, rotation and append, and attention in each layer.
        dict(STEP, name="step_decode", layers=2, seqs=128, groups=8, prefix_lo=2048, prefix_hi=8192, own_lo=100,
             own_hi=1000, lens=16),
        # The tokens of one decode step enter the cache: latency.
        dict(APPEND, name="append_tokens", seqs=61, own_lo=100, own_hi=8192, lens=17),
        # Prompts enter the cache: bandwidth; half of each head rotated, pairs
        # side by side.
        dict(APPEND, name="append_prompts", dtype="f16", seqs=16, own_lo=0, own_hi=2048, new_lo=1000, new_hi=5000,
             rot=64, interleaved=True, lens=18),
        # Two prompts sampled eight times: fork, grow by some tokens, free.
        dict(FORK, name="fork_few", lens=19),
        # 512 requests start from 32 cached prompts in eight layers.
        dict(FORK, name="fork_many", layers=8, pages=16384, parents=32, children=512, len_hi=2048, lens=20),
        # A small cache with every other page free.
        dict(COMPACT, name="compact_few", lens=21),
        # An instance's cache after many requests have left.
        dict(COMPACT, name="compact_many", layers=8, pages=8192, seqs=96, shared=64, live=0.6, lens=22),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tokens", "tokens", "drafts", "prompts", "step", "append", "fork", "compact"])
    shape = dict(dtype=rng.choice(["bf16", "f16"]), dim=rng.choice([64, 128]), page=rng.choice([8, 16, 32, 64]),
                 layout=rng.choice(["heads", "tokens"]), lens=rng.randrange(1 << 30))
    kv = rng.choice([1, 2, 4, 8])
    shape["kv_heads"] = kv
    heads = kv * rng.choice([1, 2, 3, 4, 7, 8])
    if kind in ("tokens", "drafts", "step"):
        seqs = _log_between(rng, 1, 192)
        top = _log_between(rng, 256, 12_000)
        c = dict(STEP if kind == "step" else ATTEND, **shape, q_heads=heads, seqs=seqs,
                 groups=rng.randint(0, min(8, seqs)), prefix_lo=top // 4, prefix_hi=top, own_lo=rng.choice([0, 1, 100]),
                 own_hi=_log_between(rng, 101, 4000))
        if kind == "drafts":
            c.update(new_lo=0, new_hi=rng.randint(2, 16))
    elif kind == "prompts":
        top = _log_between(rng, 64, 6000)
        hi = _log_between(rng, 17, 700)
        c = dict(ATTEND, **shape, q_heads=heads, seqs=rng.randint(1, 12), groups=rng.randint(0, 1), prefix_lo=top // 2,
                 prefix_hi=top, own_lo=0, own_hi=rng.randint(0, 500), new_lo=rng.randint(1, hi), new_hi=hi)
    elif kind == "append":
        hi = _log_between(rng, 1, 2000)
        c = dict(APPEND, **shape, q_heads=heads, seqs=_log_between(rng, 1, 32), own_hi=_log_between(rng, 20, 4000),
                 new_lo=rng.randint(0, hi), new_hi=hi)
    elif kind == "fork":
        hi = _log_between(rng, 20, 3000)
        c = dict(FORK, **shape, layers=rng.randint(1, 8), parents=rng.randint(1, 16), children=_log_between(rng, 1, 300),
                 len_lo=rng.randint(1, hi), len_hi=hi, add_lo=0, add_hi=rng.randint(1, 100))
        blocks = -(-(hi + 1 + c["add_hi"]) // c["page"])
        c["pages"] = c["parents"] * blocks + c["children"] * (2 + -(-c["add_hi"] // c["page"])) + rng.randint(1, 500)
    else:
        pages = _log_between(rng, 40, 6000)
        c = dict(COMPACT, **shape, layers=rng.randint(1, 6), pages=pages, seqs=rng.randint(1, 64),
                 shared=rng.randint(0, 32), live=round(rng.uniform(0.1, 0.95), 3))
    if kind in ("step", "append"):
        c.update(rot=rng.choice([32, c["dim"]]), interleaved=rng.choice([False, True]))
    return c


# -- lengths and the places of pages ------------------------------------------------

def _lengths(c):
    """Per sequence: its group (-1: none), shared prefix, length with the new tokens, new tokens."""
    rng = random.Random(c["lens"])
    page, n, g = c["page"], c["seqs"], c["groups"]
    prefix = [max(page, _log_between(rng, max(1, c["prefix_lo"]), max(1, c["prefix_hi"])) // page * page)
              for _ in range(g)]
    weights = [1 / (k + 1) for k in range(g)]   # few templates take most requests
    of = sorted(rng.choices(range(g), weights, k=n)) if g else [-1] * n
    got = []
    for s in range(n):
        p = prefix[of[s]] if g else 0
        new = rng.randint(c["new_lo"], c["new_hi"])
        if s == n - 1 and not any(x[3] for x in got):
            new = max(1, new)   # a batch has a token
        got.append((of[s], p, p + rng.randint(c["own_lo"], c["own_hi"]) + new, new))
    return got


def _blocks(tokens, page):
    return -(-tokens // page)


def _dev():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _ints(values, dev):
    return torch.tensor(values, dtype=torch.int32, device=dev)


def _pools(c, pages, gen, dev):
    shape = (c["layers"], pages) + ((c["kv_heads"], c["page"]) if c["layout"] == "heads" else (c["page"], c["kv_heads"]))
    k = torch.randn(shape + (c["dim"],), generator=gen, device=dev, dtype=TYPES[c["dtype"]])
    v = torch.randn(shape + (c["dim"],), generator=gen, device=dev, dtype=TYPES[c["dtype"]])
    return k, v


def _batch_state(c, seed):
    """A batch of sequences in pages: what attend, append and step cases start from."""
    dev = _dev()
    gen = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    seqs, page = _lengths(c), c["page"]
    widest = max(_blocks(length, page) for _, _, length, _ in seqs) + 1
    need, first = 0, {}
    for g, p, length, _ in seqs:
        need += _blocks(length, page) - (p // page if g in first else 0)
        if g >= 0:
            first[g] = True
    pages = need + 3
    free = list(range(pages))
    rng.shuffle(free)
    rows, shared = [], {}
    for g, p, length, _ in seqs:
        if g >= 0 and g not in shared:
            shared[g] = [free.pop() for _ in range(p // page)]
        row = list(shared[g]) if g >= 0 else []
        row += [free.pop() for _ in range(_blocks(length, page) - len(row))]
        rows.append(row + [-1] * (widest - len(row)))
    place = list(range(len(seqs)))   # the batch's order is not the tables' order
    rng.shuffle(place)
    tables = torch.full((len(seqs), widest), -1, dtype=torch.int32)
    tables[torch.tensor(place)] = torch.tensor(rows, dtype=torch.int32)
    lengths = [0] * len(seqs)
    for at, (_, _, length, _) in zip(place, seqs):
        lengths[at] = length
    refs = torch.bincount(tables[tables >= 0].long(), minlength=pages).to(torch.int32)
    offsets, group_offsets, group_prefix = [0], [0], []
    for g, p, _, new in seqs:
        offsets.append(offsets[-1] + new)
    for g in sorted({g for g, _, _, _ in seqs if g >= 0}):
        members = [p for h, p, _, _ in seqs if h == g]
        group_offsets.append(group_offsets[-1] + len(members))
        group_prefix.append(members[0])
    k, v = _pools(c, pages, gen, dev)
    s = dict(case=c, k=k, v=v, tables=tables.to(dev), lengths=_ints(lengths, dev), refs=refs.to(dev),
             seqs=_ints(place, dev), offsets=_ints(offsets, dev), tokens=offsets[-1], host=seqs, place=place,
             group_offsets=_ints(group_offsets, dev) if group_prefix else None,
             group_prefix=_ints(group_prefix, dev) if group_prefix else None,
             most=max(length for _, _, length, _ in seqs), newest=max(1, max(new for _, _, _, new in seqs)),
             scale=c["dim"] ** -0.5)
    T, hq, hk, d, t = s["tokens"], c["q_heads"], c["kv_heads"], c["dim"], TYPES[c["dtype"]]
    if c["kind"] == "attend":
        s["q"] = torch.randn(T, hq, d, generator=gen, device=dev, dtype=t) * 1.5
        for at, (_, _, length, _) in zip(place, seqs):   # the slots behind a sequence's end hold what was left there
            if length % page:
                last = int(tables[at, _blocks(length, page) - 1])
                tail = (slice(None), last, slice(None), slice(length % page, None)) if c["layout"] == "heads" else (
                    slice(None), last, slice(length % page, None))
                k[tail], v[tail] = float("nan"), float("inf")
    else:
        # what the projections of each layer leave: queries, keys and values of a token side by side
        s["qkv"] = torch.randn(c["layers"], T, (hq + 2 * hk) * d, generator=gen, device=dev, dtype=t) * 2
        s["q_weight"] = (1 + 0.2 * torch.randn(d, generator=gen, device=dev)).to(t)
        s["k_weight"] = (1 + 0.2 * torch.randn(d, generator=gen, device=dev)).to(t)
        inv = 10_000.0 ** (-torch.arange(0, c["rot"], 2, device=dev, dtype=torch.float64) / c["rot"])
        angle = torch.arange(s["most"], device=dev, dtype=torch.float64)[:, None] * inv
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


def _layer_inputs(s, layer):
    c = s["case"]
    hq, hk, d = c["q_heads"], c["kv_heads"], c["dim"]
    x = s["qkv"][layer].view(s["tokens"], hq + 2 * hk, d)
    return x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]


def _fork_lengths(c):
    """(lengths of the parents, per child its parent, the length it keeps and what it grows by)"""
    rng = random.Random(c["lens"])
    parents = [rng.randint(c["len_lo"], c["len_hi"]) for _ in range(c["parents"])]
    kids = []
    for _ in range(c["children"]):
        p = rng.randrange(len(parents))
        kids.append((p, rng.randint((parents[p] + 1) // 2, parents[p]), rng.randint(c["add_lo"], c["add_hi"])))
    return parents, kids


def _fork_state(c, seed):
    dev = _dev()
    gen = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    parents, kids = _fork_lengths(c)
    n, page = len(parents) + len(kids), c["page"]
    widest = max([_blocks(x, page) for x in parents] + [_blocks(x + a, page) for _, x, a in kids]) + 1
    place = list(range(n))
    rng.shuffle(place)
    free = list(range(c["pages"]))
    rng.shuffle(free)
    tables = torch.full((n, widest), -1, dtype=torch.int32)
    lengths = [0] * n
    for at, x in zip(place, parents):
        tables[at, :_blocks(x, page)] = torch.tensor([free.pop() for _ in range(_blocks(x, page))], dtype=torch.int32)
        lengths[at] = x
    refs = torch.bincount(tables[tables >= 0].long(), minlength=c["pages"]).to(torch.int32)
    k, v = _pools(c, c["pages"], gen, dev)
    return dict(case=c, k=k, v=v, tables=tables.to(dev), lengths=_ints(lengths, dev), refs=refs.to(dev),
                parents=_ints([place[p] for p, _, _ in kids], dev),
                children=_ints(place[len(parents):], dev),
                keep=_ints([x for _, x, _ in kids], dev), add=_ints([a for _, _, a in kids], dev))


def _compact_places(c):
    """The ids of the live pages, and how many of them the sequences share from their start."""
    rng = random.Random(c["lens"])
    live = max(1, int(c["live"] * c["pages"]))
    return sorted(rng.sample(range(c["pages"]), live)), min(c["shared"], live // 2)


def _compact_state(c, seed):
    dev = _dev()
    gen = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    ids, shared = _compact_places(c)
    rng.shuffle(ids)
    n, page = c["seqs"], c["page"]
    rows = [ids[:shared] for _ in range(n)]
    deal = random.Random(c["lens"] + 1)
    for i, p in enumerate(ids[shared:]):   # the rest dealt out, ragged
        at = deal.randrange(n) if i >= n else i
        rows[at] = rows[at] + [p]
    widest = max(map(len, rows)) + 1
    tables = torch.tensor([r + [-1] * (widest - len(r)) for r in rows], dtype=torch.int32)
    lengths = [max(0, len(r) * page - rng.randrange(page)) for r in rows]
    refs = torch.bincount(tables[tables >= 0].long(), minlength=c["pages"]).to(torch.int32)
    k, v = _pools(c, c["pages"], gen, dev)
    return dict(case=c, k=k, v=v, tables=tables.to(dev), lengths=_ints(lengths, dev), refs=refs.to(dev),
                tables_out=torch.full_like(tables, -1).to(dev), refs_out=torch.zeros_like(refs).to(dev))


def prepare(case, seed):
    s = {"fork": _fork_state, "compact": _compact_state}.get(case["kind"], _batch_state)(case, seed)
    if own:   # the handle that a program keeps for its cache: the same tensors
        from paper_2602_06502_gb300.cache import PagedCache
        s["cache"] = PagedCache(s["k"], s["v"], s["tables"], s["lengths"], s["refs"], layout=case["layout"])
    return s


# -- the plain forms -------------------------------------------------------------------

def _positions(s):
    """Per new token: its sequence in the batch, its row of the tables, its position."""
    dev = s["offsets"].device
    t = torch.arange(s["tokens"], device=dev)
    of = torch.searchsorted(s["offsets"][1:].long(), t, right=True)
    row = s["seqs"].long()[of]
    return t, of, row, s["lengths"].long()[row] - (s["offsets"].long()[of + 1] - t)


def _plain_append(s, layer):
    c = s["case"]
    q, k, v = _layer_inputs(s, layer)
    _, _, row, pos = _positions(s)
    half = c["rot"] // 2
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]

    def turn(x, w):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        r, rest = x[..., :c["rot"]], x[..., c["rot"]:]
        if c["interleaved"]:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = r[..., :half], r[..., half:]
            r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([r, rest], -1)

    q, k = turn(q, s["q_weight"]).to(s["k"].dtype), turn(k, s["k_weight"]).to(s["k"].dtype)
    page, slot = s["tables"][row, pos // c["page"]].long(), pos % c["page"]
    if c["layout"] == "heads":
        s["k"][layer][page, :, slot] = k
        s["v"][layer][page, :, slot] = v
    else:
        s["k"][layer][page, slot] = k
        s["v"][layer][page, slot] = v
    return q


def _plain_attend(s, q, layer):
    c = s["case"]
    n, hq, hk, d, page = c["seqs"], c["q_heads"], c["kv_heads"], c["dim"], c["page"]
    L, new, dev = s["most"], s["newest"], q.device
    t, of, row, pos = _positions(s)
    at = t - s["offsets"].long()[of]
    seq_len = s["lengths"].long()[s["seqs"].long()]
    counts = s["offsets"].long()[1:] - s["offsets"].long()[:-1]
    pages = s["tables"][s["seqs"].long(), :_blocks(L, page)].long().clamp(min=0)
    there = (torch.arange(L, device=dev) < seq_len[:, None])[:, None, :, None]

    def read(pool):   # [n, kv heads, L, dim], nothing behind a sequence's end
        x = pool[layer][pages]
        x = (x.permute(0, 2, 1, 3, 4) if c["layout"] == "heads" else x.permute(0, 3, 1, 2, 4)).flatten(2, 3)[:, :, :L]
        return torch.where(there, x.float(), 0.0)

    qp = torch.zeros(n, new, hq, d, device=dev)
    qp[of, at] = q.float()
    qp = qp.view(n, new, hk, hq // hk, d).permute(0, 2, 3, 1, 4).flatten(2, 3)
    scores = (qp @ read(s["k"]).transpose(-1, -2)).mul_(s["scale"]).view(n, hk, hq // hk, new, L)
    where = (seq_len - counts)[:, None] + torch.arange(new, device=dev)          # a query's position
    hidden = torch.arange(L, device=dev) > where[:, :, None]
    scores.masked_fill_(hidden[:, None, None], -torch.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(top == -torch.inf, 0.0, top)).exp_()
    total = scores.sum(-1, keepdim=True)
    o = (scores.view(n, hk, hq // hk * new, L) @ read(s["v"])).view(n, hk, hq // hk, new, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n, new, hq, d)
    return o[of, at].to(q.dtype)


def _plain_fork(s):
    c = s["case"]
    page, dev = c["page"], s["tables"].device
    parents, children, keep = s["parents"].long(), s["children"].long(), s["keep"].long()
    col = torch.arange(s["tables"].shape[1], device=dev)
    blocks, tail = (keep + page - 1) // page, keep % page
    rows = s["tables"][parents]
    shared = col < (keep // page)[:, None]
    s["refs"].index_add_(0, rows[shared], torch.ones_like(rows[shared]))
    part = torch.nonzero(tail).flatten()                       # a last page that is not full is copied
    fresh = torch.nonzero(s["refs"] == 0).flatten()[:part.numel()]
    old = rows[part, blocks[part] - 1].long()
    rows[part, blocks[part] - 1] = fresh.to(torch.int32)
    s["refs"][fresh] = 1
    live = torch.arange(page, device=dev) < tail[part][:, None]
    live = live[None, :, None, :, None] if c["layout"] == "heads" else live[None, :, :, None, None]
    for pool in (s["k"], s["v"]):
        pool[:, fresh] = torch.where(live, pool[:, old], pool[:, fresh])
    s["tables"][children] = torch.where(col < blocks[:, None], rows, s["tables"][children])
    s["lengths"][children] = s["keep"]


def _plain_extend(s):
    page, dev = s["case"]["page"], s["tables"].device
    children, add = s["children"].long(), s["add"].long()
    have = s["lengths"][children].long()
    col = torch.arange(s["tables"].shape[1], device=dev)
    wanted = (col >= ((have + page - 1) // page)[:, None]) & (col < ((have + add + page - 1) // page)[:, None])
    rows = s["tables"][children]
    fresh = torch.nonzero(s["refs"] == 0).flatten()[:int(wanted.sum())]
    rows[wanted] = fresh.to(torch.int32)
    s["refs"][fresh] = 1
    s["tables"][children] = rows
    s["lengths"][children] = (have + add).to(torch.int32)


def _plain_free(s):
    page, dev = s["case"]["page"], s["tables"].device
    children = s["children"].long()
    blocks = (s["lengths"][children].long() + page - 1) // page
    used = s["tables"][children][torch.arange(s["tables"].shape[1], device=dev) < blocks[:, None]]
    s["refs"].index_add_(0, used, -torch.ones_like(used))
    s["lengths"][children] = 0


def _plain_compact(s):
    page, dev = s["case"]["page"], s["tables"].device
    used = s["refs"] > 0
    ids = torch.arange(used.numel(), device=dev)
    live = used.sum()
    src, dst = torch.nonzero(used & (ids >= live)).flatten(), torch.nonzero(~used & (ids < live)).flatten()
    for pool in (s["k"], s["v"]):
        pool[:, dst] = pool[:, src]
    to = ids.to(torch.int32)
    to[src] = dst.to(torch.int32)
    refs = torch.where(ids < live, s["refs"], 0)
    refs[dst] = s["refs"][src]
    s["refs_out"].copy_(refs)
    blocks = (s["lengths"].long() + page - 1) // page
    mine = torch.arange(s["tables"].shape[1], device=dev) < blocks[:, None]
    s["tables_out"].copy_(torch.where(mine, to[s["tables"].clamp(min=0).long()], s["tables_out"]))


def run(s):
    c = s["case"]
    if c["kind"] == "fork":
        if own:
            s["cache"].fork(s["parents"], s["children"], s["keep"])
            s["cache"].extend(s["children"], s["add"])
            s["cache"].free(s["children"])
        else:
            _plain_fork(s)
            _plain_extend(s)
            _plain_free(s)
        return {"k": s["k"].view(torch.int16), "v": s["v"].view(torch.int16), "tables": s["tables"],
                "lengths": s["lengths"], "refs": s["refs"]}
    if c["kind"] == "compact":
        if own:
            s["cache"].compact(s["tables_out"], s["refs_out"])
        else:
            _plain_compact(s)
        return {"k": s["k"].view(torch.int16), "v": s["v"].view(torch.int16), "tables": s["tables_out"],
                "refs": s["refs_out"]}

    def append(layer):
        if not own:
            return _plain_append(s, layer)
        q, k, v = _layer_inputs(s, layer)
        return s["cache"].append(s["seqs"], s["offsets"], q, k, v, s["cos"], s["sin"], layer=layer,
                                 q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, interleaved=c["interleaved"])

    if c["kind"] == "append":
        q = append(0)
        return {"q": q, "k": s["k"], "v": s["v"].view(torch.int16)}
    if own:
        plan = s["cache"].plan(s["seqs"], s["offsets"], s["tokens"], c["q_heads"], s["group_offsets"],
                               s["group_prefix"])

    def attend(q, layer):
        return s["cache"].attend(plan, q, layer=layer, scale=s["scale"]) if own else _plain_attend(s, q, layer)

    if c["kind"] == "attend":
        return {"o": attend(s["q"], 0)}
    out = {}
    for layer in range(c["layers"]):
        q = append(layer)
        out["q%d" % layer], out["o%d" % layer] = q, attend(q, layer)
    return dict(out, k=s["k"], v=s["v"].view(torch.int16))


# -- what a pass cannot do without --------------------------------------------------------

def work(case):
    c = case
    page = c["page"]
    row = c["kv_heads"] * c["dim"] * 2   # bytes of a token's keys, or values, in one layer
    if c["kind"] == "fork":
        parents, kids = _fork_lengths(c)
        copied = sum(x % page for _, x, _ in kids) * row * 2 * c["layers"]
        entries = sum(_blocks(x, page) for _, x, _ in kids)
        grown = sum(_blocks(x + a, page) - _blocks(x, page) for _, x, a in kids)
        # copied tokens read and written; table entries read and written, their counts raised and lowered
        return {"bytes": 2 * copied + entries * (8 + 16) + grown * (4 + 16) + len(kids) * 28, "flops": 0}
    if c["kind"] == "compact":
        ids, shared = _compact_places(c)
        moved = sum(i >= len(ids) for i in ids)
        entries = len(ids) - shared + shared * c["seqs"]
        return {"bytes": 2 * moved * page * row * 2 * c["layers"] + entries * 8 + c["pages"] * 8, "flops": 0}
    seqs = _lengths(c)
    tokens = sum(new for _, _, _, new in seqs)
    q = tokens * c["q_heads"] * c["dim"] * 2
    total = {"bytes": 0, "flops": 0}
    if c["kind"] != "attend":
        rows = len({p for _, _, length, new in seqs for p in range(length - new, length)})
        heads = c["q_heads"] + c["kv_heads"]
        total["bytes"] += c["layers"] * (2 * q + 4 * tokens * row) + rows * c["rot"] * 4 + 4 * c["dim"]
        total["flops"] += c["layers"] * tokens * heads * c["dim"] * 7
    if c["kind"] != "append":
        prefix = {g: p for g, p, _, _ in seqs if g >= 0}
        held = sum(prefix.values()) + sum(length - p for _, p, length, new in seqs if new)
        pairs = sum(new * (length - new) + new * (new + 1) // 2 for _, _, length, new in seqs)
        total["bytes"] += c["layers"] * (2 * q + held * row * 2) + held // page * 4
        total["flops"] += c["layers"] * pairs * c["q_heads"] * c["dim"] * 4
    return total


# -- in 64 bits --------------------------------------------------------------------------

def _exact_append(s, layer, k_pool):
    """Token by token of each sequence, a pair of a head's values turned as a complex number."""
    c = s["case"]
    rot, done = c["rot"], []
    q_all, k_all, _ = _layer_inputs(s, layer)
    begin = 0
    for (_, _, length, new), at in zip(s["host"], s["place"]):
        pos = torch.arange(length - new, length, device=q_all.device)
        turn = torch.complex(s["cos"][pos].double(), s["sin"][pos].double())[:, None]
        out = []
        for x, w in ((q_all[begin:begin + new], s["q_weight"]), (k_all[begin:begin + new], s["k_weight"])):
            x = x.double()
            x = x / ((x ** 2).sum(-1, keepdim=True) / c["dim"] + EPS).sqrt() * w.double()
            r = x[..., :rot]
            r = r.unflatten(-1, (rot // 2, 2)) if c["interleaved"] else r.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.complex(r[..., 0], r[..., 1]) * turn)
            z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
            out.append(torch.cat([z, x[..., rot:]], -1))
        done.append(out[0])
        where = s["tables"][at].long()[pos // c["page"]]
        for h in range(c["kv_heads"]):
            if c["layout"] == "heads":
                k_pool[where, h, pos % c["page"]] = out[1][:, h]
            else:
                k_pool[where, pos % c["page"], h] = out[1][:, h]
        begin += new
    return torch.cat(done)


def _exact_attend(s, q, k_pool, v_pool):
    """Sequence by sequence, key head by key head: weights exp(score - log of the sum)."""
    c = s["case"]
    group, page, out, begin = c["q_heads"] // c["kv_heads"], c["page"], torch.zeros_like(q, dtype=torch.float64), 0
    for (_, _, length, new), at in zip(s["host"], s["place"]):
        if not new:
            continue
        key = torch.arange(length, device=q.device)
        where, slot = s["tables"][at].long()[key // page], key % page
        ahead = key[None] > torch.arange(length - new, length, device=q.device)[:, None]
        for h in range(c["kv_heads"]):
            at_h = (where, h, slot) if c["layout"] == "heads" else (where, slot, h)
            mine = q[begin:begin + new, h * group:(h + 1) * group].double().transpose(0, 1)
            score = torch.matmul(mine, k_pool[at_h].double().T) * s["scale"]
            score = score.masked_fill(ahead, -torch.inf)
            weight = torch.exp(score - torch.logsumexp(score, -1, keepdim=True))
            out[begin:begin + new, h * group:(h + 1) * group] = torch.matmul(weight, v_pool[at_h].double()).transpose(0, 1)
        begin += new
    return out


def exact(case, seed):
    c = case
    if c["kind"] in ("fork", "compact"):
        return None   # copies and whole numbers
    s = _batch_state(c, seed)
    if c["kind"] == "attend":
        return {"o": _exact_attend(s, s["q"], s["k"][0], s["v"][0])}
    k = s["k"].double()
    if c["kind"] == "append":
        return {"q": _exact_append(s, 0, k[0]), "k": k, "v": None}
    out = {}
    for layer in range(c["layers"]):
        q = _exact_append(s, layer, k[layer])
        # attention's own inputs are the rounded queries, keys and values
        _, _, v = _layer_inputs(s, layer)
        held_k = k[layer].to(s["k"].dtype)
        _, _, row, pos = _positions(s)
        where, slot = s["tables"][row, pos // c["page"]].long(), pos % c["page"]
        if c["layout"] == "heads":
            s["v"][layer][where, :, slot] = v
        else:
            s["v"][layer][where, slot] = v
        out["q%d" % layer], out["o%d" % layer] = q, _exact_attend(s, q.to(held_k.dtype), held_k, s["v"][layer])
    return dict(out, k=k, v=None)
