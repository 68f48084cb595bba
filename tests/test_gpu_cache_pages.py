"""Pages of an instance's prefix cache (dm_cache_extend, _fork, _free,
_compact) against a plain model: which pages are given out, counts, tables,
and the copied values bit by bit."""

import random

import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    lib_ready()
    import torch
    return torch


def make(torch, *, pages, page_tokens=16, max_seqs=40, max_blocks=40, layers=2, kv_heads=3, dim=64, layout="heads", seed=0,
         dtype=None):
    from cache_reference import Pages
    from paper_2602_06502_gb300.cache import PagedCache
    inner = (kv_heads, page_tokens) if layout == "heads" else (page_tokens, kv_heads)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randint(-30000, 30000, (layers, pages) + inner + (dim,), generator=gen, device="cuda", dtype=torch.int16)
            .view(dtype or torch.bfloat16) for _ in range(2))
    z = dict(dtype=torch.int32, device="cuda")
    c = PagedCache(k, v, torch.full((max_seqs, max_blocks), -1, **z), torch.zeros(max_seqs, **z), torch.zeros(pages, **z), layout)
    return c, Pages(pages, page_tokens, max_seqs)


def same_books(c, m, tables=None, refs=None):
    refs = (c.refs if refs is None else refs).cpu().tolist()
    tables = (c.tables if tables is None else tables).cpu().tolist()
    assert refs == m.refs
    assert c.lengths.cpu().tolist() == m.lengths
    for s, row in enumerate(m.tables):
        assert tables[s][:len(row)] == row, s


def copy_tail(pool, layout, old, new, tail):
    if layout == "heads":
        pool[:, new, :, :tail] = pool[:, old, :, :tail]
    else:
        pool[:, new, :tail] = pool[:, old, :tail]


@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("page_tokens,pages,seed", [(16, 300, 1), (4, 1000, 2), (64, 129, 3), (8, 5000, 4), (32, 40_000, 5)])
def test_random_calls(torch, layout, page_tokens, pages, seed):
    """Grow, fork, free and compact at random; everything equals the model after each call."""
    from cache_reference import ints
    rng = random.Random(seed)
    c, m = make(torch, pages=pages, page_tokens=page_tokens, layout=layout, seed=seed)
    k, v = c.k.clone(), c.v.clone()
    bits = torch.int16
    for step in range(40):
        empty = [s for s in range(40) if m.lengths[s] == 0]
        live = [s for s in range(40) if m.lengths[s] > 0]
        free = m.refs.count(0)
        act = rng.choice(["extend", "extend", "fork", "fork", "free", "compact"])
        if act == "extend":
            seqs, add = [], []
            for s in rng.sample(range(40), rng.randint(1, 12)):
                a = rng.choice([0, 1, page_tokens, rng.randint(0, 6 * page_tokens)])
                need = -(-(m.lengths[s] + a) // page_tokens) - len(m.tables[s])
                if need <= free and m.lengths[s] + a <= 40 * page_tokens:
                    seqs.append(s)
                    add.append(a)
                    free -= need
            m.extend(seqs, add)
            c.extend(ints(seqs), ints(add))
        elif act == "fork" and live and empty:
            kids = rng.sample(empty, min(len(empty), rng.randint(1, 10), free))
            par = [rng.choice(live) for _ in kids]
            keep = [rng.choice([0, m.lengths[p], rng.randint(0, m.lengths[p]), m.lengths[p] // page_tokens * page_tokens]) for p in par]
            for old, new, tail in m.fork(par, kids, keep):
                for pool in (k, v):
                    copy_tail(pool, layout, old, new, tail)
            c.fork(ints(par), ints(kids), ints(keep))
        elif act == "free" and live:
            gone = rng.sample(range(40), rng.randint(1, 8))
            m.free(gone)
            c.free(ints(gone + gone[:1]))   # twice is once
        elif act == "compact":
            moves = m.compact()
            old = torch.tensor([a for a, _ in moves], dtype=torch.long, device="cuda")
            new = torch.tensor([b for _, b in moves], dtype=torch.long, device="cuda")
            for pool in (k, v):
                pool[:, new] = pool[:, old]
            count = ints([-1])
            if step % 2:
                c.compact(moved=count)
            else:
                tables, refs = torch.full_like(c.tables, -3), torch.zeros_like(c.refs)
                before = c.tables.clone(), c.refs.clone()
                c.compact(tables, refs, count)
                assert torch.equal(before[0], c.tables) and torch.equal(before[1], c.refs)
                same_books(c, m, tables, refs)
                c.tables.copy_(tables)
                c.refs.copy_(refs)
            assert count.item() == len(moves)
        assert c.last_error() == 0
        same_books(c, m)
        assert torch.equal(c.k.view(bits), k.view(bits)) and torch.equal(c.v.view(bits), v.view(bits)), (step, act)


@pytest.mark.parametrize("pages", [1, 3, 4, 127, 128, 129, 32767, 32768, 32769, 100_001])
def test_pool_sizes(torch, pages):
    """Every page can be given out, at sizes around a warp's and a cluster's runs; ids ascend over the holes."""
    from cache_reference import ints
    c, m = make(torch, pages=pages, page_tokens=4, max_seqs=3, max_blocks=pages, layers=1, kv_heads=1)
    holes = sorted(random.Random(pages).sample(range(pages), pages // 3))
    c.refs[torch.tensor(holes, dtype=torch.long, device="cuda")] = 1
    free = sorted(set(range(pages)) - set(holes))
    half = len(free) // 2
    c.extend(ints([2, 0]), ints([4 * half, 4 * (len(free) - half)]))
    assert c.last_error() == 0
    assert c.tables[2, :half].tolist() == free[:half]
    assert c.tables[0, :len(free) - half].tolist() == free[half:]
    assert bool((c.refs == 1).all())
    c.extend(ints([1]), ints([1]))
    from paper_2602_06502_gb300 import dualmap as D
    assert c.last_error() == D.DM_ERR_CAPACITY and c.lengths.tolist()[1] == 0
    c.free(ints([2, 0]))
    moved = ints([0])
    c.compact(moved=moved)
    assert c.last_error() == 0
    low = [h for h in holes if h < len(holes)]
    assert moved.item() == len(holes) - len(low)
    assert c.refs.tolist() == [1] * len(holes) + [0] * (pages - len(holes))


def test_page_and_layer_strides(torch):
    """Keys and values side by side in a page, layers outermost."""
    from cache_reference import ints
    from paper_2602_06502_gb300.cache import PagedCache
    both = torch.randint(-30000, 30000, (3, 50, 2, 2, 16, 64), device="cuda", dtype=torch.int16).view(torch.float16)
    z = dict(dtype=torch.int32, device="cuda")
    c = PagedCache(both[:, :, 0], both[:, :, 1], torch.zeros(4, 8, **z), torch.zeros(4, **z), torch.zeros(50, **z))
    want = both.clone()
    c.extend(ints([1]), ints([16 * 4 + 5]))
    c.fork(ints([1, 1]), ints([3, 0]), ints([16 + 7, 64 + 5]))
    want[:, 5, :, :, :7] = want[:, 1, :, :, :7]
    want[:, 6, :, :, :5] = want[:, 4, :, :, :5]
    assert c.last_error() == 0 and torch.equal(both.view(torch.int16), want.view(torch.int16))
    c.free(ints([1, 3]))
    c.compact()
    want[:, 4] = want[:, 6]   # pages 0-3 (shared with sequence 0) and 6 are in use
    assert c.last_error() == 0 and torch.equal(both.view(torch.int16), want.view(torch.int16))
    assert c.tables[0, :5].tolist() == [0, 1, 2, 3, 4] and c.refs.tolist() == [1] * 5 + [0] * 45


def test_refusals_change_nothing(torch):
    from cache_reference import ints
    from paper_2602_06502_gb300 import dualmap as D
    c, m = make(torch, pages=64, max_seqs=8, max_blocks=10)
    c.extend(ints([0, 1]), ints([37, 16 * 8]))
    m.extend([0, 1], [37, 16 * 8])
    k = c.k.clone()
    inv, cap = D.DM_ERR_INVALID_ARG, D.DM_ERR_CAPACITY
    for want, call in [
            (inv, lambda: c.extend(ints([2, 8]), ints([1, 1]))), (inv, lambda: c.extend(ints([-1]), ints([1]))),
            (inv, lambda: c.extend(ints([2, 2]), ints([1, 1]))), (inv, lambda: c.extend(ints([2]), ints([-1]))),
            (cap, lambda: c.extend(ints([1]), ints([33]))),          # an eleventh block
            (cap, lambda: c.extend(ints([2]), ints([2 ** 31 - 1]))),
            (cap, lambda: c.extend(ints([2, 3, 4, 5, 6, 7]), ints([160] * 6))),   # 60 of 53 pages
            (inv, lambda: c.fork(ints([0]), ints([1]), ints([5]))),   # not empty
            (inv, lambda: c.fork(ints([0, 0]), ints([2, 2]), ints([5, 5]))),
            (inv, lambda: c.fork(ints([0]), ints([2]), ints([38]))), (inv, lambda: c.fork(ints([0]), ints([2]), ints([-1]))),
            (inv, lambda: c.fork(ints([9]), ints([2]), ints([1]))), (inv, lambda: c.fork(ints([0]), ints([99]), ints([1]))),
            (inv, lambda: c.free(ints([0, 8])))]:
        call()
        c.extend(ints([3]), ints([16]))   # does nothing while the error stands
        assert c.last_error() == want
        assert c.last_error() == 0
        same_books(c, m)
        assert torch.equal(k.view(torch.int16), c.k.view(torch.int16))
    c.extend(ints([]), ints([]))
    c.free(ints([]))
    assert c.last_error() == 0


def test_argument_checks(torch):
    from cache_reference import ints
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300.cache import PagedCache
    c, _ = make(torch, pages=8)
    with pytest.raises(ValueError):
        PagedCache(c.k.float(), c.v.float(), c.tables, c.lengths, c.refs)
    with pytest.raises(ValueError):
        PagedCache(c.k.transpose(2, 3), c.v.transpose(2, 3), c.tables, c.lengths, c.refs)
    with pytest.raises(ValueError):
        PagedCache(c.k, c.v, c.tables.long(), c.lengths, c.refs)
    with pytest.raises(ValueError):
        PagedCache(c.k, c.v, c.tables, c.lengths, c.refs[:7])
    with pytest.raises(D.DualMapError):   # pages of 24 tokens
        PagedCache.empty(pages=4, kv_heads=1, head_dim=64, max_seqs=2, max_tokens=64, page_tokens=24)
    with pytest.raises(D.DualMapError):
        PagedCache.empty(pages=4, kv_heads=1, head_dim=80, max_seqs=2, max_tokens=64)
    with pytest.raises(ValueError):
        c.extend(ints([0, 1]), ints([1]))
    with pytest.raises(ValueError):
        c.free(ints([0]).long())
    with pytest.raises(D.DualMapError):   # more than the sequences there are
        c.free(ints([0] * 41))


def test_many_requests(torch):
    """More requests in a call than are searched in shared memory."""
    from cache_reference import ints
    n = 5000
    c, m = make(torch, pages=30_000, page_tokens=4, max_seqs=2 * n, max_blocks=6, layers=1, kv_heads=1)
    rng = random.Random(8)
    k = c.k.clone()
    seqs, add = rng.sample(range(2 * n), n), [rng.randint(0, 20) for _ in range(n)]
    m.extend(seqs, add)
    c.extend(ints(seqs), ints(add))
    assert c.last_error() == 0
    same_books(c, m)
    live = [s for s in seqs if m.lengths[s]]
    kids = [s for s in range(2 * n) if not m.lengths[s]][:n]
    par = [rng.choice(live) for _ in kids]
    keep = [rng.randint(0, m.lengths[p]) for p in par]
    for old, new, tail in m.fork(par, kids, keep):
        copy_tail(k, "heads", old, new, tail)
    c.fork(ints(par), ints(kids), ints(keep))
    assert c.last_error() == 0
    same_books(c, m)
    assert torch.equal(c.k.view(torch.int16), k.view(torch.int16))
    m.free(live)
    c.free(ints(live))
    m.compact()
    c.compact()
    same_books(c, m)
    m.free(kids)
    c.free(ints(kids))
    assert c.refs.sum().item() == 0
