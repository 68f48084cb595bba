"""The prefix cache serves: its calls give no gradients, and say so where
autograd would miss them.  Runs without a GPU, on a cache whose calls are
stubs."""

import pytest


@pytest.fixture
def call(monkeypatch):
    import torch

    from paper_2602_06502_gb300 import cache as M
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    c = M.PagedCache.__new__(M.PagedCache)
    c.device, c.dtype, c.head_dim, c.kv_heads, c._errors, c._lib = torch.device("cpu"), torch.bfloat16, 64, 1, 0, None
    c.calls = []
    c._call = lambda name, *args: c.calls.append(name)
    x = {n: torch.zeros(3, h, 64, dtype=torch.bfloat16) for n, h in (("q", 2), ("k", 1), ("v", 1), ("out", 2))}
    x.update({n: torch.ones(64, dtype=torch.bfloat16) for n in ("q_weight", "k_weight")})
    x.update({n: torch.ones(5, 32) for n in ("cos", "sin")})
    ints = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    plan = M.Plan(M.D.dm_plan(), (None,), 3, 2, 0, 0)

    def go(name, **kw):
        if name == "append":
            c.append(*ints, **{**x, **kw})
        else:
            c.attend(plan, kw.get("q", x["q"]), out=kw.get("out"))
        return c.calls
    return go, x


@pytest.mark.parametrize("name,which", [("append", w) for w in ("q", "k", "v", "out", "q_weight", "k_weight", "cos", "sin")] +
                         [("attend", w) for w in ("q", "out")])
def test_inputs_that_want_gradients(call, name, which):
    import torch
    go, x = call
    assert go(name) == ["dm_cache_" + name]
    wants = x[which].clone().requires_grad_()
    with pytest.raises(ValueError, match="grad"):
        go(name, **{which: wants})
    with pytest.raises(ValueError, match="grad"):
        go(name, **{which: wants * 1})   # a view or result of one
    with torch.no_grad():
        go(name, **{which: wants})
    with torch.inference_mode():
        go(name, **{which: wants})
    assert go(name, **{which: wants.detach()}) == ["dm_cache_" + name] * 4
