"""Every positive finite bfloat16 against tops of every mantissa."""

import pytest

import experts_reference as R
from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shift", [-133, -126, -101, -60, -1, 0, 6, 60, 126])
def test_quantize_every_value_against_every_mantissa(shift):
    lib_ready()
    import torch
    from paper_2602_06502_gb300 import experts as X
    every = torch.arange(0, 0x7F80, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16)
    tops = (torch.arange(128, 256, device="cuda", dtype=torch.float64) * 2.0 ** (shift - 7)).bfloat16()   # subnormal ones lose bits
    x = torch.where(every <= tops[:, None], every, tops[:, None])
    x[:, 0] = -tops
    assert x.shape == (128, 0x7F80)
    q, scale = X.quantize(x)
    want, ref = R.quantized(x)
    assert torch.equal(q.double(), want)
    assert bool(((scale.double() - ref).abs() <= ref * 2.0 ** -24 + 2.0 ** -149).all())
