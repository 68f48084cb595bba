"""A prefix cache on the CPU with the calls of cache.PagedCache that the
instance example makes: bookkeeping of cache_reference.Pages, appended keys and
attention sequence by sequence in the tensors' own type."""

import torch

from cache_reference import Pages
from paper_2602_06502_gb300 import dualmap as D


class CpuCache:
    def __init__(self, books, shape, max_blocks, dtype):
        self.books, self.page_tokens, self.max_blocks = books, books.B, max_blocks
        self.k, self.v = torch.zeros(shape, dtype=dtype), torch.zeros(shape, dtype=dtype)   # layers, pages, heads, tokens, dim
        self.error = D.DM_OK

    @classmethod
    def empty(cls, *, pages, kv_heads, head_dim, max_seqs, max_tokens, page_tokens=16, layers=1, dtype=torch.float32,
              layout="heads", device="cpu"):
        return cls(Pages(pages, page_tokens, max_seqs), (layers, pages, kv_heads, page_tokens, head_dim),
                   -(-max_tokens // page_tokens), dtype)

    @property
    def refs(self):
        return torch.tensor(self.books.refs, dtype=torch.int32)

    @property
    def lengths(self):
        return torch.tensor(self.books.lengths, dtype=torch.int32)

    def last_error(self):
        e, self.error = self.error, D.DM_OK
        return e

    def extend(self, seqs, add):
        if self.error:
            return
        seqs, add, m = seqs.tolist(), add.tolist(), self.books
        blocks = [-(-(m.lengths[s] + a) // m.B) for s, a in zip(seqs, add)]
        if max(blocks) > self.max_blocks or sum(blocks) - sum(len(m.tables[s]) for s in seqs) > m.refs.count(0):
            self.error = D.DM_ERR_CAPACITY
            return
        m.extend(seqs, add)

    def fork(self, parents, children, lengths):
        if self.error:
            return
        for old, new, tail in self.books.fork(parents.tolist(), children.tolist(), lengths.tolist()):
            for pool in (self.k, self.v):
                pool[:, new, :, :tail] = pool[:, old, :, :tail]

    def free(self, seqs):
        if not self.error:
            self.books.free(seqs.tolist())

    def compact(self):
        if not self.error:
            for old, new in self.books.compact():
                self.k[:, new], self.v[:, new] = self.k[:, old], self.v[:, old]

    def append(self, seqs, offsets, q, k, v, cos, sin, *, layer=0, q_weight=None, k_weight=None, eps=1e-6):
        if self.error:
            return torch.full_like(q, torch.nan)
        out, off = torch.empty(q.shape, dtype=q.dtype), offsets.tolist()
        for i, s in enumerate(seqs.tolist()):
            a, b = off[i], off[i + 1]
            p = torch.arange(self.books.lengths[s] - (b - a), self.books.lengths[s])
            c, n = cos[p][:, None], sin[p][:, None]

            def turn(x, w):
                x = x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + eps) * w.float()
                lo, hi = x.chunk(2, -1)
                return torch.cat([lo * c - hi * n, hi * c + lo * n], -1).to(q.dtype)

            out[a:b] = turn(q[a:b], q_weight)
            page, slot = torch.tensor(self.books.tables[s], dtype=torch.long)[p // self.page_tokens], p % self.page_tokens
            self.k[layer][page, :, slot], self.v[layer][page, :, slot] = turn(k[a:b], k_weight), v[a:b]
        return out

    def plan(self, seqs, offsets, tokens, q_heads, group_offsets, group_prefix):
        seqs, off, go = seqs.tolist(), offsets.tolist(), group_offsets.tolist()
        for g, p in enumerate(group_prefix.tolist()):
            rows = [self.books.tables[s][:p // self.page_tokens] for s in seqs[go[g]:go[g + 1]]]
            if any(r != rows[0] for r in rows):
                self.error = self.error or D.DM_ERR_INVALID_ARG
        return None if self.error else (seqs, off)

    def attend(self, plan, q, *, layer=0):
        if plan is None or self.error:
            return torch.full_like(q, torch.nan)
        out = torch.empty_like(q)
        for s, a, b in zip(plan[0], plan[1], plan[1][1:]):
            n, rows = self.books.lengths[s], torch.tensor(self.books.tables[s], dtype=torch.long)
            k, v = (x[layer][rows].transpose(1, 2).flatten(0, 1)[:n].float() for x in (self.k, self.v))
            g = q.shape[1] // k.shape[1]
            score = torch.einsum("thd,phd->htp", q[a:b].float(), k.repeat_interleave(g, 1)) * q.shape[-1] ** -0.5
            hidden = torch.arange(n) > torch.arange(n - (b - a), n)[:, None]
            out[a:b] = torch.einsum("htp,phd->thd", score.masked_fill(hidden, -torch.inf).softmax(-1),
                                    v.repeat_interleave(g, 1)).to(q.dtype)
        return out
