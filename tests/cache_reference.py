"""Plain models of the paged cache for its tests: bookkeeping in Python lists,
attention and the appended keys in float64."""

import random

import numpy as np
import torch


class Pages:
    """Bookkeeping of a cache: what extend, fork, free and compact do."""

    def __init__(self, pages, page_tokens, max_seqs):
        self.B, self.refs, self.tables, self.lengths = page_tokens, [0] * pages, [[] for _ in range(max_seqs)], [0] * max_seqs

    def _take(self, n):
        free = [p for p, r in enumerate(self.refs) if r == 0][:n]
        assert len(free) == n
        for p in free:
            self.refs[p] = 1
        return free

    def extend(self, seqs, add):
        for s, a in zip(seqs, add):
            n = -(-(self.lengths[s] + a) // self.B) - len(self.tables[s])
            self.tables[s] = self.tables[s] + self._take(n)
            self.lengths[s] += a

    def fork(self, parents, children, lengths):
        """Returns (old page, new page, tokens) of each copy."""
        copies = []
        for p, c, n in zip(parents, children, lengths):
            full, tail = divmod(n, self.B)
            row = self.tables[p][:full]
            for x in row:
                self.refs[x] += 1
            if tail:
                new, = self._take(1)
                copies.append((self.tables[p][full], new, tail))
                row = row + [new]
            self.tables[c], self.lengths[c] = row, n
        return copies

    def free(self, seqs):
        for s in seqs:
            for x in self.tables[s]:
                self.refs[x] -= 1
            self.tables[s], self.lengths[s] = [], 0

    def compact(self):
        """Returns (old page, new page) of each move."""
        live = sum(r > 0 for r in self.refs)
        src = [p for p, r in enumerate(self.refs) if r and p >= live]
        dst = [p for p, r in enumerate(self.refs) if not r and p < live]
        to = dict(zip(src, dst))
        self.tables = [[to.get(x, x) for x in row] for row in self.tables]
        for s, d in to.items():
            self.refs[d], self.refs[s] = self.refs[s], 0
        return list(to.items())


def ints(values, device="cuda"):
    return torch.tensor(list(values), dtype=torch.int32, device=device)


def make_batch(rng_seed, *, page, kv_heads, dim, dtype, layout="heads", prefix=(), own, new, groups=None, layers=1, junk=True,
               spare=5, extra_row=0):
    """A PagedCache of len(own) sequences with random contents.

    groups: sequences per group, in order (the rest have none); prefix: tokens
    each group shares; own[i]: cached tokens of sequence i besides its prefix
    and its new[i] new tokens (negative: the sequence is shorter than its new
    tokens).  Returns a dict."""
    from paper_2602_06502_gb300.cache import PagedCache
    rng = random.Random(rng_seed)
    gen = torch.Generator(device="cuda").manual_seed(rng_seed)
    n = len(own)
    group_of, at = [-1] * n, 0
    for g, m in enumerate(groups or []):
        for _ in range(m):
            group_of[at] = g
            at += 1
    length = [max(0, (prefix[g] if g >= 0 else 0) + o + w) for g, o, w in zip(group_of, own, new)]
    need = sum(-(-x // page) for x in length)
    free = list(range(need + spare))
    rng.shuffle(free)
    shared = [[free.pop() for _ in range(p // page)] for p in prefix]
    widest = max([1] + [-(-x // page) for x in length]) + extra_row
    rows = []
    for g, x in zip(group_of, length):
        row = list(shared[g]) if g >= 0 else []
        row = row[:-(-x // page)]
        row += [free.pop() for _ in range(-(-x // page) - len(row))]
        rows.append(row)
    place = list(range(n + 2))
    rng.shuffle(place)
    place = place[:n]
    tables = torch.full((n + 2, widest), -7, dtype=torch.int32)
    lengths = [0] * (n + 2)
    refs = [0] * (need + spare)
    for s, row, x in zip(place, rows, length):
        if row:
            tables[s, :len(row)] = torch.tensor(row, dtype=torch.int32)
        lengths[s] = x
        for p in row:
            refs[p] += 1
    inner = (kv_heads, page) if layout == "heads" else (page, kv_heads)
    shape = (layers, need + spare) + inner + (dim,)
    k = torch.randn(shape, generator=gen, device="cuda").to(dtype)
    v = torch.randn(shape, generator=gen, device="cuda").to(dtype)
    if junk:   # free pages, and slots behind a sequence's end
        for p, r in enumerate(refs):
            if not r:
                k[:, p], v[:, p] = float("nan"), float("inf")
        for row, x in zip(rows, length):
            if x % page:
                tail = (slice(None), row[-1], slice(None), slice(x % page, None)) if layout == "heads" else \
                    (slice(None), row[-1], slice(x % page, None))
                k[tail], v[tail] = float("inf"), float("nan")
    offsets = [0]
    for w in new:
        offsets.append(offsets[-1] + w)
    go = [0]
    for m in groups or []:
        go.append(go[-1] + m)
    cache = PagedCache(k, v, tables.cuda(), ints(lengths), ints(refs), layout)
    return dict(cache=cache, rows=rows, length=length, place=place, seqs=ints(place), offsets=ints(offsets), host_offsets=offsets,
                new=list(new), tokens=offsets[-1], group_offsets=ints(go) if groups else None,
                group_prefix=ints(prefix) if groups else None, page=page, layout=layout, gen=gen)


def read_seq(b, pool, i, layer=0):
    """[length, kv heads, dim] of sequence i."""
    x = pool[layer][torch.tensor(b["rows"][i], dtype=torch.long, device=pool.device)]
    if b["layout"] == "heads":
        x = x.transpose(1, 2)
    return x.flatten(0, 1)[:b["length"][i]]


def attend_reference(b, q, scale, layer=0):
    """(output, logarithm of the sum, sum of weight * |v|) in float64; rows that see nothing give zeros, -inf."""
    T, hq, d = q.shape
    hk = b["cache"].kv_heads
    o = torch.zeros(T, hq, d, dtype=torch.float64, device=q.device)
    mass = torch.zeros_like(o)
    lse = torch.full((T, hq), -torch.inf, dtype=torch.float64, device=q.device)
    for i, w in enumerate(b["new"]):
        n, t0 = b["length"][i], b["host_offsets"][i]
        if not w or not n:
            continue
        k, v = read_seq(b, b["cache"].k, i, layer).double(), read_seq(b, b["cache"].v, i, layer).double()
        x = q[t0:t0 + w].double().view(w, hk, hq // hk, d)
        s = torch.einsum("thgd,phd->thgp", x, k) * scale
        pos = n - w + torch.arange(w, device=q.device)
        s = s.masked_fill((torch.arange(n, device=q.device) > pos[:, None])[:, None, None], -torch.inf)
        z = torch.logsumexp(s, -1)
        p = torch.exp(s - torch.where(z == -torch.inf, 0.0, z)[..., None])
        o[t0:t0 + w] = torch.einsum("thgp,phd->thgd", p, v).reshape(w, hq, d)
        mass[t0:t0 + w] = torch.einsum("thgp,phd->thgd", p, v.abs()).reshape(w, hq, d)
        lse[t0:t0 + w] = z.reshape(w, hq)
    return o, lse, mass


def attend_bound(ref, mass, dtype, longest, vmax):
    """How far an output may be from the reference.

    u: unit roundoff of the type.  Each weight is rounded once (u mass), the
    output once (u |o|); scores in 32 bits (products of 64-128 terms, one
    scaling, exp2 to 2^-22) move a weight by less than 2^-14; float16 weights
    below 2^-14 of the running maximum round by up to 2^-25 each."""
    u = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    small = longest * 2.0 ** -25 * vmax if dtype == torch.float16 else 0.0
    tiny = 2.0 ** -24   # the output may be a subnormal float16
    return (u + 2.0 ** -14) * mass + u * ref.abs() * 1.01 + small + tiny


def numpy(x):
    return np.asarray(x.cpu())
