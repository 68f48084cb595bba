"""Memory that the cache allocates itself is not given out again while a
stream other than its own still uses it."""

import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    lib_ready()
    import torch
    return torch


def given_out_again(torch, size, at):
    """Whether one of some new tensors of the present stream lies at `at` (none of them is written)."""
    new = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
    return any(x.data_ptr() == at for x in new)


def test_plan_dropped_while_another_stream_attends(torch):
    import cache_reference as R
    b = R.make_batch(31, page=16, kv_heads=2, dim=64, dtype=torch.float16, own=[50, 200], new=[1, 40])
    c = b["cache"]
    q = torch.randn(b["tokens"], 4, 64, generator=b["gen"], device="cuda").half()
    side = torch.cuda.Stream()
    want = c.attend(c.plan(b["seqs"], b["offsets"], b["tokens"], 4), q)
    plan = c.plan(b["seqs"], b["offsets"], b["tokens"], 4)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)   # some 0.2 s
        o = c.attend(plan, q)
    at, size = plan.keep[-1].data_ptr(), plan.keep[-1].numel()
    del plan
    assert not given_out_again(torch, size, at)
    assert not side.query()   # the attention had not run by then
    side.synchronize()
    assert torch.equal(o, want) and c.last_error() == 0


def test_cache_dropped_while_another_stream_uses_it(torch):
    import cache_reference as R
    from paper_2602_06502_gb300.cache import PagedCache
    ids, add = R.ints([1, 5]), R.ints([70, 3])
    # a kernel's first launch may wait for the whole device
    PagedCache.empty(pages=30, kv_heads=2, head_dim=64, max_seqs=40, max_tokens=640).extend(ids, add)
    torch.cuda.synchronize()
    c = PagedCache.empty(pages=3000, kv_heads=2, head_dim=64, max_seqs=4000, max_tokens=640)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
        c.extend(ids, add)
    held = [(x.data_ptr(), x.numel() * x.element_size()) for x in (c.work, c.tables, c.k)]
    del c
    for at, size in held:
        assert not given_out_again(torch, size, at)
    assert not side.query()
    side.synchronize()
