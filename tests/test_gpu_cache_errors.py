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
