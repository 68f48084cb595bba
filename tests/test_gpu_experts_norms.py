"""Rows that a norm divides by their root mean square, at the ends of the range."""

import pytest

import experts_reference as R
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


TOPS = [3.3e38, 1e20, 2.0 ** 51, 2.0 ** 49, 1.0, 2.0 ** -47, 2.0 ** -49, 1e-25, 1e-38, 1e-40]


def extreme(torch, rows, k):
    """Rows of bfloat16 whose largest values are TOPS, in turn; one in three with nothing else of that size."""
    x = torch.randn(rows, k, generator=gen(torch, rows + k), device="cuda", dtype=torch.float64)
    x[::3, 1:] *= 1e-3
    top = torch.tensor(TOPS, device="cuda", dtype=torch.float64).repeat(-(-rows // len(TOPS)))[:rows, None]
    return (x / x.abs().amax(-1, keepdim=True) * top).bfloat16()


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6, 1e30])
@pytest.mark.parametrize("rows,k", [(10, 40), (10, 1000), (700, 1000), (10, 2000), (700, 2000), (10, 3000), (700, 4096), (10, 7000), (20, 20000)])
def test_rows_at_the_ends_of_the_range(torch, rows, k, eps):
    from paper_2602_06502_gb300 import experts as X
    x = extreme(torch, rows, k)
    q, scale = X.quantize(x, eps=eps)
    want, ref = R.quantized(x)
    assert torch.equal(q.double(), want)
    ref = ref / (x.double().square().mean(-1) + eps).sqrt()
    # the sum of squares, a division, a reciprocal root and products, as in the tests of ordinary rows; eps is rounded to
    # 32 bits, and what is left of a square below 2^-149 is at most 2^-26 of the sum
    assert bool(((scale.double() - ref).abs() <= ref * (k / 32 + 80) * 2.0 ** -24 + 2.0 ** -149).all())


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("rows", [8, 300])
def test_projections_at_the_ends_of_the_range(torch, rows, eps):
    """Rows that the product quantises itself, and many, as halves."""
    from paper_2602_06502_gb300 import experts as X
    k = 264
    x = extreme(torch, rows, k)
    x = x[(x.abs().amax(-1) > 1e-30) | (x.abs().amax(-1) == 0)]   # a scale that 32 bits hold in full
    real = torch.randn(40, k, generator=gen(torch, 2), device="cuda").bfloat16()
    w = X.Weights.quantized(real)
    y = X.Linear(w)(x, eps=eps, out=torch.empty(x.shape[0], 40, device="cuda"))
    q, scale = X.quantize(x, eps=eps)
    z, off = R.sums(q, w.w, scale, w.scale)
    # and two sums of squares of k terms each
    R.close(y, z, R.round_off(z, off + z.abs() * (k / 16 + 64) * 2.0 ** -24, torch.float32))
    assert (z.abs().amax(-1) > 0).all() and w.last_error() == 0
