"""A status word that atomics cannot reach is refused before any launch."""

import pytest

import test_experts_args as A
from test_experts_args import D   # noqa: F401 (a fixture)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_status_off_its_alignment(D, off):   # noqa: F811
    at = dict(status=(1 << 25) + off)
    one = A.eight(D, experts=1)
    assert D.dm_product(A.weights(D), A.product(D, **at)) == D.DM_ERR_INVALID_ARG
    assert D.dm_linear(one, A.linear(D, **at)) == D.DM_ERR_INVALID_ARG
    assert D.dm_linear(one, A.linear(D, rows=4, work=None, work_bytes=0, **at)) == D.DM_ERR_INVALID_ARG
    assert D.dm_experts(A.weights(D), A.down(D), A.layer(D, **at)) == D.DM_ERR_INVALID_ARG
    assert D.dm_products_last_error((1 << 25) + off) == D.DM_ERR_INVALID_ARG
