"""Expert layers on both sides of the sizes at which other kernels take their
products: what lies behind the work buffer stays as it was, and the layer is the
sum of its parts."""

import ctypes as C

import pytest

import test_gpu_experts as E
from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    lib_ready()
    import torch
    return torch


BEHIND = 64 << 20   # bytes; more than any of these layers lays out
SIZES = [(128, 64, 8, 512, 256), (129, 64, 8, 512, 256), (256, 64, 8, 512, 256), (257, 64, 8, 512, 256), (200, 64, 8, 1024, 384),
         (600, 24, 2, 256, 128), (200, 256, 8, 264, 72), (300, 160, 5, 131, 45)]


@pytest.mark.parametrize("skewed", [False, True])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens,experts,top_k,k,m", SIZES)
def test_layer_stays_in_its_buffer(torch, tokens, experts, top_k, k, m, eight, skewed):
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300 import experts as X
    x, up, down, logits, residual, t = E.make_layer(torch, tokens + k, tokens, experts, k, m, "bfloat16", eight)
    if skewed:
        logits[:, 1:1 + top_k] += 9   # nearly all tokens go to the same experts
    size = D.dm_experts_bytes(up.struct, down.struct, tokens, top_k)
    buffer = torch.full((size + BEHIND,), 0xA5, dtype=torch.uint8, device="cuda")
    y = torch.empty(tokens, k, dtype=t, device="cuda")
    a = D.dm_experts_args(x.data_ptr(), logits.data_ptr(), None if residual is None else residual.data_ptr(), y.data_ptr(), up.status_at,
                          buffer.data_ptr(), size, x.stride(0), logits.stride(0), 0 if residual is None else residual.stride(0), y.stride(0),
                          D.DM_BF16, D.DM_F32, tokens, top_k, 1, 0)
    assert D.lib().dm_experts(up.ref, down.ref, C.byref(a), torch.cuda.current_stream().cuda_stream) == D.DM_OK
    assert up.last_error() == D.DM_OK
    assert bool((buffer[size:] == 0xA5).all())
    assert torch.equal(y, X.Experts(up, down, top_k)(x, logits, residual=residual))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("tokens,experts,top_k,k,m", SIZES)
def test_layer_in_8_bits_is_its_parts(torch, tokens, experts, top_k, k, m, dtype):
    E.test_layer_in_8_bits_is_its_parts(torch, tokens, experts, top_k, k, m, dtype)


@pytest.mark.parametrize("tokens,experts,top_k,k,m", [(129, 64, 8, 512, 256), (200, 64, 8, 1024, 384), (300, 160, 5, 131, 45)])
def test_layer(torch, tokens, experts, top_k, k, m):
    E.test_layer(torch, tokens, experts, top_k, k, m, "bfloat16")
