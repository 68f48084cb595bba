"""One instance behind the router: a small random transformer on the prefix
cache, fed with the requests of a synthetic trace that the router sends there.

    python -m paper_2602_06502_gb300.instance --workload tiny --batches 4 --decode 16

Each batch is routed (scheduler.Scheduler); the instance's requests fork from
what it holds of their prefixes, their other tokens run through the layers
(append, then attention that reads a shared prefix once), some tokens are
decoded greedily, and the sequences stay as prefixes for later requests until
their pages are needed.  One JSON line per batch.

    ... --experts 8 --top-k 2 --eight-bits

adds a layer of experts after each attention, and keeps the projections' and the
experts' weights in 8 bits.
"""

import argparse
import hashlib
import json
import os
import sys
import time

import numpy as np
import torch

from . import dualmap as D
from .cache import PagedCache
from .experts import Experts, Linear, Weights, last_error


class Instance:
    """A decoder of `layers` attention layers with random weights over a
    PagedCache: admit() prompts, decode() greedily, keep or drop().  experts: a
    layer of so many of width `expert_width` (default: the model's) after each
    attention, top_k a token; eight_bits: projections and experts in 8 bits."""

    def __init__(self, *, pages, max_tokens, max_seqs=512, page_tokens=16, layers=2, q_heads=16, kv_heads=4, head_dim=64,
                 vocab=32000, dtype=torch.bfloat16, seed=0, device="cuda", experts=0, top_k=2, expert_width=None, eight_bits=False):
        self.cache = PagedCache.empty(pages=pages, kv_heads=kv_heads, head_dim=head_dim, max_seqs=max_seqs, max_tokens=max_tokens,
                                      page_tokens=page_tokens, layers=layers, dtype=dtype, device=device)
        self.device, self.layers, self.q_heads, self.kv_heads, self.dim = device, layers, q_heads, kv_heads, head_dim
        width = q_heads * head_dim
        gen = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=gen, device=device) * shape[0] ** -0.5).to(dtype)

        self.embedding = (torch.randn(vocab, width, generator=gen, device=device)).to(dtype)
        self.qkv = [weight(width, (q_heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.out = [weight(width, width) for _ in range(layers)]
        self.norms = [(1 + 0.1 * torch.randn(2, head_dim, generator=gen, device=device)).to(dtype) for _ in range(layers)]
        angle = torch.arange(max_tokens, device=device, dtype=torch.float64)[:, None] * \
            10_000.0 ** (-torch.arange(0, head_dim, 2, device=device, dtype=torch.float64) / head_dim)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        self.status, self.gates, self.experts, self.linears = None, [], [], []
        if experts or eight_bits:
            self.status = torch.zeros(1, dtype=torch.int32, device=device)   # of all products, asked once a step
        if eight_bits:   # (queries, keys and values; output) of each layer
            self.linears = [[Linear(Weights.quantized(w.T.contiguous(), status=self.status)) for w in pair]
                            for pair in zip(self.qkv, self.out)]
            self.qkv, self.out = [], []
        for _ in range(layers if experts else 0):
            m = expert_width or width
            self.gates.append(weight(width, experts))
            pair = []
            for n, k in ((2 * m, width), (width, m)):
                w = (torch.randn(experts, n, k, generator=gen, device=device) * k ** -0.5).to(dtype)
                pair.append(Weights.quantized(w, status=self.status) if eight_bits else Weights(w, status=self.status))
            self.experts.append(Experts(*pair, top_k))
        self.tokens = {}        # sequence -> its tokens, oldest first
        self.serial = {}        # sequence -> its number among all that were ever admitted (ids are given out again)
        self.origin = {}        # sequence -> (serial of the sequence it forked from or -1, tokens it kept)
        self.blocks = {}        # (block before, the block's tokens) -> sequences that hold it, oldest first
        self.max_tokens, self.max_seqs = max_tokens, max_seqs
        self.free_seqs = list(range(max_seqs - 1, -1, -1))
        self.reused = self.computed = self.admitted = 0

    def _ints(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.device)

    def _chain(self, tokens):
        """Keys of the full blocks of `tokens`: each names its whole prefix."""
        key, B = b"", self.cache.page_tokens
        for i in range(0, len(tokens) - B + 1, B):
            key = hashlib.blake2b(key + tokens[i:i + B].tobytes(), digest_size=16).digest()
            yield key

    def _held(self, tokens, most):
        """(sequence, tokens): the longest prefix of full blocks that is held, up to `most` tokens."""
        seq, n, B = -1, 0, self.cache.page_tokens
        for key in self._chain(tokens):
            if key not in self.blocks or n + B > most:
                break
            seq, n = next(reversed(self.blocks[key])), n + B
        return seq, n

    def _short(self, pages, seqs):
        return len(self.free_seqs) < seqs or int((self.cache.refs == 0).sum()) < pages

    def _make_room(self, pages, seqs):
        """Drops the oldest sequences until `pages` pages and `seqs` sequence ids are free, and packs the rest."""
        dropped = False
        while self.tokens and self._short(pages, seqs):
            self.drop([next(iter(self.tokens))])
            dropped = True
        if dropped:
            self.cache.compact()
        if self._short(pages, seqs):
            raise ValueError(f"no room for {seqs} sequences in {pages} pages")

    def admit(self, prompts, hits=None, room=0):
        """Starts a sequence per prompt (uint32 arrays) and runs the tokens that
        no held prefix covers; hits: the router's cached-prefix tokens, which
        bound what is reused; room: tokens that each will be decoded.  Returns (sequences, logits of their last tokens),
        in the order in which the sequences run: those of one prefix together.
        A batch that the cache could not hold even by itself is refused, and nothing changes."""
        B = self.cache.page_tokens
        if not prompts or not all(1 <= len(t) <= self.max_tokens - room for t in prompts):
            raise ValueError(f"prompts have 1 to {self.max_tokens - room} tokens")
        pages = sum(-(-(len(t) + room) // B) for t in prompts)
        if len(prompts) > self.max_seqs or pages > self.cache.refs.shape[0]:
            raise ValueError(f"a batch of {len(prompts)} sequences in {pages} pages: more than the cache has")
        self._make_room(pages, len(prompts))
        found = [self._held(t, min(len(t) - 1, len(t) if hits is None else int(h)))
                 for t, h in zip(prompts, hits if hits is not None else [0] * len(prompts))]
        order = sorted(range(len(prompts)), key=lambda i: found[i])
        seqs = [self.free_seqs.pop() for _ in order]
        forked = [(found[i], s) for i, s in zip(order, seqs) if found[i][0] >= 0]
        if forked:
            self.cache.fork(self._ints([f[0] for f, _ in forked]), self._ints([s for _, s in forked]),
                            self._ints([f[1] for f, _ in forked]))
        news = []
        for i, s in zip(order, seqs):
            self.tokens[s] = np.ascontiguousarray(prompts[i], dtype=np.uint32)
            self.origin[s] = self.serial.get(found[i][0], -1), found[i][1]
            self.serial[s] = self.admitted
            self.admitted += 1
            news.append(self.tokens[s][found[i][1]:])
        try:
            logits = self._forward(seqs, news)
        except D.DualMapError:
            self.drop(seqs)
            raise
        self.reused += sum(found[i][1] for i in order)
        for s in seqs:
            for key in self._chain(self.tokens[s]):
                self.blocks.setdefault(key, {})[s] = None
        return seqs, logits

    def decode(self, seqs, logits, steps):
        """Greedy tokens [steps, len(seqs)]."""
        out = []
        for _ in range(steps):
            token = logits.argmax(-1)
            out.append(token)
            host = token.cpu().numpy().astype(np.uint32)
            logits = self._forward(seqs, [t[None] for t in host])
            for s, t in zip(seqs, host):
                self.tokens[s] = np.append(self.tokens[s], t)
        return torch.stack(out) if out else torch.empty(0, len(seqs), dtype=torch.int64, device=self.device)

    def drop(self, seqs):
        """Gives the sequences' pages up."""
        self.cache.free(self._ints(seqs))
        for s in seqs:
            for key in self._chain(self.tokens[s]):
                holders = self.blocks.get(key, {})
                holders.pop(s, None)
                if not holders:
                    self.blocks.pop(key, None)
            del self.tokens[s], self.origin[s], self.serial[s]
            self.free_seqs.append(s)

    def groups(self, seqs):
        """(offsets, prefixes): runs of sequences that forked from one sequence at one length."""
        offsets, prefix, last = [0], [], None
        for i, s in enumerate(seqs):
            if self.origin[s] != last or self.origin[s][0] < 0:
                if i:
                    offsets.append(i)
                prefix.append(self.origin[s][1])
                last = self.origin[s]
        return self._ints(offsets + [len(seqs)]), self._ints(prefix)

    @staticmethod
    def _normed(x):
        return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def _forward(self, seqs, news):
        """Appends the new tokens of each sequence and returns the logits of its last one.
        A step that the cache refused raises DualMapError (synchronises)."""
        counts = [len(t) for t in news]
        offsets = np.concatenate([[0], np.cumsum(counts)])
        T, hq, hk, d = int(offsets[-1]), self.q_heads, self.kv_heads, self.dim
        ids, at = self._ints(seqs), self._ints(offsets.tolist())
        self.cache.extend(ids, self._ints(counts))
        plan = self.cache.plan(ids, at, T, hq, *self.groups(seqs))   # once for all layers
        x = self.embedding[torch.from_numpy(np.concatenate(news).astype(np.int64)).to(self.device)]
        for layer in range(self.layers):
            if self.linears:   # their rows are divided by their root mean square when they are quantised
                qkv = self.linears[layer][0](x, eps=1e-6).view(T, hq + 2 * hk, d)
            else:
                qkv = (self._normed(x) @ self.qkv[layer]).view(T, hq + 2 * hk, d)
            qw, kw = self.norms[layer]
            q = self.cache.append(ids, at, qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], self.cos, self.sin, layer=layer,
                                  q_weight=qw, k_weight=kw)
            o = self.cache.attend(plan, q, layer=layer).view(T, hq * d)
            x = x + (self.linears[layer][1](o) if self.linears else o @ self.out[layer])
            if self.experts:
                h = self._normed(x)
                x = self.experts[layer](h, h @ self.gates[layer], residual=x)
        err = self.cache.last_error()
        if self.status is not None:
            err = last_error(self.status) or err
        if err:
            raise D.DualMapError(err, "instance")
        self.computed += T
        return x[at[1:].long() - 1] @ self.embedding.T


def run(workload_name, instance=0, batches=4, decode=16, overrides=None, pages=8192, device="cuda:0", **model):
    """Yields one dict per batch of the trace.  model: of Instance."""
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    from tracegen import Trace, workload

    from .scheduler import Scheduler

    w = workload(workload_name, **(overrides or {}))
    tr = Trace(w)
    longest = int(max(tr.L)) + decode
    node = Instance(pages=pages, max_tokens=longest, max_seqs=w["batch"] + 256, page_tokens=w["block_tokens"], vocab=w["vocab"],
                    device=device, **model)
    g = Scheduler(block_tokens=w["block_tokens"], route_prefix_blocks=w["route_prefix_blocks"], vnodes=w["vnodes"],
                  max_instances=tr.max_instance_id() + 1, capacity=w["capacity"], slo_us=w["slo_us"], cost_us=w["cost_us"],
                  max_batch=w["batch"], max_batch_tokens=max(int(tr.batch_layout(b)[4]) for b in range(len(tr.batches))) + (1 << 16),
                  seed=w["seed"], device=device)
    for i in range(w["n_instances"]):
        rc = g.add_instance(i)
        if rc:
            raise D.DualMapError(rc, "dm_add_instance")
    dev = torch.device(device)
    for b in range(min(batches, len(tr.batches))):
        s, e, off, lens, nt = tr.batch_layout(b)
        tok = tr.batch_tokens(b)
        g.route(torch.from_numpy(tok.view(np.int32)).to(dev), torch.from_numpy(off.view(np.int64)).to(dev),
                torch.from_numpy(lens.view(np.int32)).to(dev), e - s, nt, tr.batch_time(b))
        r = g.results(e - s)
        g.commit()
        mine = np.nonzero(r["chosen"] == instance)[0]
        hits = np.where(r["cand1"][mine] == instance, r["hit1"][mine], r["hit2"][mine])
        before = node.reused, node.computed
        out = {"batch": b, "requests": len(mine), "router_hit_tokens": int(hits.sum())}
        if len(mine):
            prompts = [tok[int(off[i]):int(off[i]) + int(lens[i])] for i in mine]
            torch.cuda.synchronize(dev)
            t0 = time.perf_counter()
            seqs, logits = node.admit(prompts, hits, room=decode)
            torch.cuda.synchronize(dev)
            t1 = time.perf_counter()
            node.decode(seqs, logits, decode)
            torch.cuda.synchronize(dev)
            t2 = time.perf_counter()
            out.update(prompt_tokens=int(lens[mine].sum()), reused_tokens=node.reused - before[0],
                       computed_tokens=node.computed - before[1], prefill_ms=1e3 * (t1 - t0),
                       decode_ms_per_step=1e3 * (t2 - t1) / max(decode, 1))
        out.update(held_sequences=len(node.tokens), pages_in_use=int((node.cache.refs > 0).sum()),
                   pages_unshared=int(node.cache.refs.sum()))
        err = node.cache.last_error() or g.last_error()
        if err:
            raise D.DualMapError(err, "instance")
        yield out
    g.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--workload", default="tiny")
    ap.add_argument("--instance", type=int, default=0)
    ap.add_argument("--batches", type=int, default=4)
    ap.add_argument("--decode", type=int, default=16, help="tokens decoded per request")
    ap.add_argument("--pages", type=int, default=8192)
    ap.add_argument("--experts", type=int, default=0, help="experts of a layer after each attention")
    ap.add_argument("--top-k", type=int, default=2, help="experts that a token goes to")
    ap.add_argument("--eight-bits", action="store_true", help="projections and experts in 8 bits")
    ap.add_argument("--set", action="append", default=[], metavar="KEY=VALUE", help="override a workload field")
    args = ap.parse_args()
    over = {}
    for kv in args.set:
        k, v = kv.split("=", 1)
        over[k] = float(v) if "." in v else int(v)
    for row in run(args.workload, args.instance, args.batches, args.decode, over, args.pages, experts=args.experts,
                   top_k=args.top_k, eight_bits=args.eight_bits):
        print(json.dumps(row), flush=True)


if __name__ == "__main__":
    main()
