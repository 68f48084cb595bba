"""The work buffer of an expert layer holds what the layer lays out in it: asked
of the library alone, without a GPU."""

import pytest

from test_experts_args import D, eight   # noqa: F401 (D is a fixture)


def layer(D, experts, k, m):
    up = eight(D, experts=experts, n=2 * m, k=k, row=k, expert=2 * m * k)
    down = eight(D, experts=experts, n=k, k=m, row=m, expert=k * m)
    return up, down


def least(D, up, down, tokens, top_k):
    """Bytes that a layer in 8 bits cannot do without.  Rows whose product runs on the tensor cores are there as halves
    (2 bytes a value), laid out by the quantising kernel in a place of their own, or from bytes, which are there too, by
    the product in its own work buffer, which the two products share."""
    slots, k, m = tokens * top_k, up.k, down.k
    same = 4 * 4 * slots + 2 * slots * m + 4 * slots * k + 4 * tokens + 4 * slots   # pairs, h, parts, scales
    halves = [D.dm_product_bytes(up, slots, 1, 1) > 1, D.dm_product_bytes(down, slots, 0, 0) > 1]
    if all(halves):
        return same + min(2 * slots * (k + m), tokens * k + slots * m + 2 * slots * max(k, m))
    if halves[0]:
        return same + 2 * slots * k + slots * m
    return same + tokens * k + (2 if halves[1] else 1) * slots * m


SHAPES = [(64, 8, 512, 256), (64, 8, 1024, 384), (24, 2, 256, 128), (256, 8, 7168, 2048), (160, 8, 2992, 2000),
          (1024, 32, 64, 16), (64, 8, 2048, 1024), (5, 2, 272, 48)]


@pytest.mark.parametrize("experts,top_k,k,m", SHAPES)
def test_layer_holds_its_rows(D, experts, top_k, k, m):   # noqa: F811
    up, down = layer(D, experts, k, m)
    tokens = {1, 4, 127, 128, 129, 200, 256, 257, 512, 513, 600, 1024, 4096}
    for product, limit in ((up, 8), (down, 8), (up, 32), (down, 32), (up, 64), (down, 64)):   # next to each change of kernels
        tokens |= {max(1, product.experts * limit // top_k + i) for i in (-1, 0, 1)}
    for t in sorted(tokens):
        assert D.dm_experts_bytes(up, down, t, top_k) >= least(D, up, down, t, top_k), t
