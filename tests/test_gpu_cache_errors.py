"""What the calls of an instance's prefix cache do around an error that the
device recorded."""

import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    lib_ready()
    import torch
    return torch


def step(torch, **kw):
    import cache_reference as R
    b = R.make_batch(21, **{**dict(page=16, kv_heads=2, dim=64, dtype=torch.bfloat16, own=[30, 200], new=[1, 40]), **kw})
    return b, b["cache"], torch.randn(b["tokens"], 4, 64, generator=b["gen"], device="cuda").bfloat16()


@pytest.mark.parametrize("new", [[1, 2], [1, 40]])   # few rows, many rows
def test_plan_made_while_an_error_stands(torch, new):
    """A plan that an earlier call's error kept from being made is no plan: attention on it is refused, not skipped."""
    import cache_reference as R
    from paper_2602_06502_gb300 import dualmap as D
    b, c, q = step(torch, new=new)
    good = c.attend(c.plan(b["seqs"], b["offsets"], b["tokens"], 4), q)
    c.extend(R.ints([b["place"][0]]), R.ints([1 << 20]))   # more than there is
    plan = c.plan(b["seqs"], b["offsets"], b["tokens"], 4)
    assert c.last_error() == D.DM_ERR_CAPACITY
    out = torch.full_like(q, 5.0)
    c.attend(plan, q, out=out)
    assert c.last_error() == D.DM_ERR_INVALID_ARG and bool((out == 5).all())
    assert torch.equal(c.attend(c.plan(b["seqs"], b["offsets"], b["tokens"], 4), q), good)
    assert c.last_error() == 0


def test_output_of_a_refused_plan(torch):
    """Attention on a plan that was found wrong gives NaN, not what the memory held before."""
    import cache_reference as R
    from paper_2602_06502_gb300 import dualmap as D
    b, c, q = step(torch)
    good = c.plan(b["seqs"], b["offsets"], b["tokens"], 4)
    want = c.attend(good, q)
    plan = c.plan(R.ints([0, 99]), b["offsets"], b["tokens"], 4)
    assert c.last_error() == D.DM_ERR_INVALID_ARG
    assert bool(torch.isnan(c.attend(plan, q)).all())
    assert torch.equal(c.attend(good, q), want)   # a plan from before the error still holds
    assert c.last_error() == 0


@pytest.mark.parametrize("more", [0, 4])
def test_blocks_past_32_bits(torch, more):
    """1,024 sequences that together ask for 2^32 blocks (and one more) of a small pool."""
    import cache_reference as R
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300.cache import PagedCache
    n, blocks = 1024, (1 << 22) + 1
    z = dict(dtype=torch.int32, device="cuda")
    k = torch.zeros(1, 8, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    c = PagedCache(k, k.clone(), torch.empty(n, blocks, **z), torch.zeros(n, **z), torch.zeros(8, **z))
    c.extend(R.ints(range(n)), R.ints([1 << 24] * (n - 1) + [(1 << 24) + more]))
    assert c.last_error() == D.DM_ERR_CAPACITY
    assert not bool(c.lengths.any()) and not bool(c.refs.any())
    c.extend(R.ints([5, 3]), R.ints([9, 20]))
    assert c.last_error() == 0
    assert c.tables[5, :3].tolist() == [0, 1, 2] and c.tables[3, :5].tolist() == [3, 4, 5, 6, 7]


def test_table_entries_that_are_no_pages(torch):
    """fork, free and append record them and write nothing outside the cache; attention reads zeros there."""
    import cache_reference as R
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300.cache import PagedCache
    b, c, q = step(torch, junk=False)
    guard = torch.zeros(c.refs.shape[0] + 8, dtype=torch.int32, device="cuda")
    guard[4:-4] = c.refs
    at, child, inv = b["place"][1], min(set(range(4)) - set(b["place"])), D.DM_ERR_INVALID_ARG
    spare = int((c.refs == 0).nonzero()[0])
    c.k[:, spare], c.v[:, spare] = 0, 0
    c = PagedCache(c.k, c.v, c.tables, c.lengths, guard[4:-4])
    k, v = c.k.clone(), c.v.clone()
    c.tables[at, 2] = spare
    zeros = c.attend(c.plan(b["seqs"], b["offsets"], b["tokens"], 4), q)
    rows = torch.ones(220, 8, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (c.refs.shape[0], -1, 1 << 30):
        c.tables[at, 2] = bad
        got = c.attend(c.plan(b["seqs"], b["offsets"], b["tokens"], 4), q)
        assert c.last_error() == 0 and torch.equal(got, zeros)
        c.append(R.ints([at]), R.ints([0, 220]), rows[:, :4], rows[:, 4:6], rows[:, 6:])
        assert c.last_error() == inv
        assert torch.equal(c.k[:, spare], k[:, spare])
        c.k.copy_(k)
        c.v.copy_(v)
        c.fork(R.ints([at]), R.ints([child]), R.ints([64]))
        assert c.last_error() == inv
        c.free(R.ints([child]))
        c.last_error()
        c.lengths[child] = 0
        assert torch.equal(c.k, k) and torch.equal(c.v, v)
    assert not bool(guard[:4].any()) and not bool(guard[-4:].any())
