"""Numbers that 32 bits do not hold are refused, not cut off."""

import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    lib_ready()
    import torch
    return torch


@pytest.mark.parametrize("top_k", [(1 << 32) + 1, 1 << 32, (1 << 33) + 2])
def test_choice(torch, top_k):
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300 import experts as X
    with pytest.raises(D.DualMapError):
        X.choose(torch.zeros(0, 8, device="cuda"), top_k)


@pytest.mark.parametrize("per_source", [(1 << 32) + 1, 1 << 32, -(1 << 32) + 1])
def test_sources(torch, per_source):
    from paper_2602_06502_gb300 import experts as X
    w = X.Weights(torch.ones(16, 64, dtype=torch.bfloat16, device="cuda"))
    x = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        X.product(x, w, sources=torch.arange(4, dtype=torch.int32, device="cuda"), per_source=per_source)


def test_matrices(torch):
    """Widths and numbers of rows whose low 32 bits would make a small matrix."""
    from paper_2602_06502_gb300 import experts as X
    wide = torch.empty(1, (1 << 32) + 16, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        X.quantize(wide)
    with pytest.raises(ValueError):
        X.choose(wide, 2)
    with pytest.raises(ValueError):
        X.Weights(wide)
    long = torch.empty((1 << 32) + 16, 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        X.quantize(long)
    with pytest.raises(ValueError):
        X.choose(long, 2)
    with pytest.raises(ValueError):
        X.Linear(X.Weights(torch.ones(16, 8, dtype=torch.bfloat16, device="cuda")))(long)
    with pytest.raises(ValueError):
        X.Weights(long)
