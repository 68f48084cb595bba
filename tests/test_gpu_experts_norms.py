"""Rows that a norm divides by their root mean square, at the ends of the range."""

import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    lib_ready()
    import torch
    return torch


def gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows,k", [(3, 40), (700, 1000), (3, 3000), (700, 4096), (2, 20000)])
def test_rows_of_zeros(torch, rows, k, dtype):
    """Their steps and scale are zeros whatever eps is, and so is a projection of them."""
    from paper_2602_06502_gb300 import experts as X
    x = torch.randn(rows, k, generator=gen(torch, k), device="cuda").to(getattr(torch, dtype))
    x[1] = 0
    for eps in (None, 0.0, 1e-6):
        q, scale = X.quantize(x, eps=eps)
        assert (q[1] == 0).all() and scale[1] == 0 and torch.isfinite(scale).all()
    w = X.Linear(X.Weights.quantized(torch.randn(24, k, generator=gen(torch, 1), device="cuda").bfloat16()))
    for eps in (0.0, 1e-6):
        y = w(x, eps=eps)
        assert (y[1] == 0).all() and torch.isfinite(y).all()
