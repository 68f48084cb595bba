"""PagedCache on a device that is not the current one: what depends on the
device is asked there.  Runs without a GPU, on stubs."""

import contextlib

import pytest


@pytest.fixture
def cache(monkeypatch):
    import torch

    from paper_2602_06502_gb300 import cache as M
    at = ["another"]

    @contextlib.contextmanager
    def device(d):
        at.append(d)
        yield
        at.pop()

    asked = []
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(M.D, "dm_plan_bytes", lambda struct, *shape: asked.append(at[-1]) or 4096)
    c = M.PagedCache.__new__(M.PagedCache)
    c.device, c.struct, c._plan_bytes, c._errors = torch.device("cpu"), M.D.dm_cache(), {}, 0
    c._call = lambda name, *args: None
    return c, asked


def test_a_plans_size_is_asked_on_the_caches_device(cache):
    """It depends on the device's SMs."""
    import torch
    c, asked = cache
    ints = [torch.zeros(n, dtype=torch.int32) for n in (2, 3)]
    c.plan(ints[0], ints[1], 4, 8)
    c.plan(ints[0], ints[1], 4, 8)
    assert asked == [c.device]
