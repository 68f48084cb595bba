"""Argument checks of the products' and experts' entry points, made before any
CUDA call: they run without a GPU, on a library that is only loaded."""

import ctypes as C
import subprocess

import pytest


@pytest.fixture(scope="module")
def D():
    import __graft_entry__ as g
    g.build()
    from paper_2602_06502_gb300 import dualmap
    return dualmap


def weights(D, **kw):
    """Weights whose pointers are never followed."""
    base = dict(w=1 << 20, scale=None, dtype=D.DM_BF16, experts=4, n=64, k=96, row=96, expert=64 * 96)
    base.update(kw)
    return D.dm_weights(**base)


def eight(D, **kw):
    return weights(D, **dict(dict(dtype=D.DM_I8, scale=1 << 21), **kw))


BAD_WEIGHTS = [dict(w=None), dict(w=(1 << 20) + 8), dict(dtype=3), dict(dtype=9), dict(experts=0), dict(experts=1025), dict(n=0), dict(k=0),
               dict(n=(1 << 24) + 1), dict(k=(1 << 24) + 1), dict(row=92), dict(row=88), dict(row=(1 << 32) + 8), dict(expert=4),
               dict(expert=64), dict(expert=64 * 96 - 8)]


@pytest.mark.parametrize("bad", BAD_WEIGHTS, ids=str)
def test_weights(D, bad):
    w = weights(D, **bad)
    assert D.dm_product_bytes(w, 4) == 0
    assert D.dm_product(w, product(D)) == D.DM_ERR_INVALID_ARG
    assert D.dm_experts_bytes(w, w, 4, 2) == 0
    one = weights(D, **dict(dict(experts=1), **bad))
    assert D.dm_linear_bytes(one, 4) == 0


def test_weights_in_8_bits(D):
    assert D.dm_product_bytes(eight(D), 4) > 0
    for bad in (dict(scale=None), dict(scale=(1 << 21) + 2), dict(row=104, expert=64 * 104)):
        assert D.dm_product_bytes(eight(D, **bad), 4) == 0
    assert D.dm_product_bytes(weights(D, n=63), 4, 1) == 0      # an odd number of channels has no halves
    assert D.dm_product_bytes(weights(D), 4, 2) == 0 and D.dm_product_bytes(weights(D), 4, 0, 2) == 0
    assert D.dm_product_bytes(weights(D), 1 << 31) == 0


def product(D, **kw):
    base = dict(x=1 << 22, y=1 << 23, offsets=1 << 24, status=1 << 25, work=None, work_bytes=0, x_row=96, y_row=64, rows=4, x_rows=4,
                per_source=0, y_dtype=D.DM_BF16)
    base.update(kw)
    return D.dm_product_args(**base)


BAD_PRODUCTS = [dict(x=None), dict(x=(1 << 22) + 8), dict(y=None), dict(y=(1 << 23) + 1), dict(offsets=None), dict(offsets=(1 << 24) + 2),
                dict(status=None), dict(x_row=92), dict(x_row=88), dict(y_row=63), dict(rows=1 << 31), dict(x_rows=3), dict(x_rows=0),
                dict(sources=1 << 26, per_source=0), dict(sources=(1 << 26) + 1, per_source=1), dict(y_dtype=2), dict(y_dtype=4), dict(gated=2),
                dict(reserved0=1), dict(x_row=(1 << 32) + 8), dict(y_row=(1 << 32) + 1)]


@pytest.mark.parametrize("bad", BAD_PRODUCTS, ids=str)
def test_product(D, bad):
    assert D.dm_product(weights(D), product(D, **bad)) == D.DM_ERR_INVALID_ARG


def test_product_more(D):
    inv = D.DM_ERR_INVALID_ARG
    assert D.lib().dm_product(None, C.byref(product(D)), None) == inv and D.lib().dm_product(C.byref(weights(D)), None, None) == inv
    assert D.dm_product(eight(D), product(D)) == inv                          # no scales of the rows
    assert D.dm_product(weights(D), product(D, rows=0)) == D.DM_OK            # nothing to do
    assert D.dm_product(weights(D), product(D, rows=0, x=None, y=None, x_rows=0)) == D.DM_OK
    big = product(D, rows=10_000, x_rows=10_000, sources=1 << 26, per_source=1)
    assert D.dm_product_bytes(weights(D), 10_000, 0, 1) > 1
    assert D.dm_product(weights(D), big) == inv                               # wants a work buffer
    big.work, big.work_bytes = 1 << 27, 512
    assert D.dm_product(weights(D), big) == inv
    big.work, big.work_bytes = (1 << 27) + 16, 1 << 40
    assert D.dm_product(weights(D), big) == inv


def test_last_error(D):
    assert D.dm_products_last_error(None) == D.DM_ERR_INVALID_ARG


def quantize(D, **kw):
    base = dict(x=1 << 20, q=1 << 21, scale=1 << 22, count=None, x_row=96, q_row=96, dtype=D.DM_F16, rows=4, k=96, eps=-1.0)
    base.update(kw)
    return D.dm_quantize_args(**base)


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=(1 << 20) + 2), dict(q=None), dict(q=(1 << 21) + 8), dict(scale=None),
                                 dict(scale=(1 << 22) + 1), dict(count=2), dict(x_row=92), dict(x_row=88), dict(q_row=104), dict(q_row=80),
                                 dict(dtype=2), dict(dtype=3), dict(k=0), dict(k=(1 << 24) + 1), dict(rows=1 << 31), dict(eps=float("nan")),
                                 dict(eps=float("inf"))], ids=str)
def test_quantize(D, bad):
    assert D.dm_quantize(quantize(D, **bad)) == D.DM_ERR_INVALID_ARG


def test_quantize_nothing(D):
    assert D.dm_quantize(quantize(D, rows=0)) == D.DM_OK
    assert D.lib().dm_quantize(None, None) == D.DM_ERR_INVALID_ARG


def choose(D, **kw):
    base = dict(logits=1 << 20, logits_row=64, dtype=D.DM_F32, tokens=100_000, experts=64, top_k=8, renormalize=1, ids=1 << 21,
                weights=1 << 22, offsets=1 << 23, slots=1 << 24, sources=1 << 25, work=1 << 26, work_bytes=1 << 30)
    base.update(kw)
    return D.dm_choose_args(**base)


@pytest.mark.parametrize("bad", [dict(logits=None), dict(logits=2), dict(logits_row=63), dict(logits_row=(1 << 32) + 1), dict(dtype=2), dict(dtype=4),
                                 dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=33), dict(experts=4, top_k=5),
                                 dict(tokens=1 << 31), dict(tokens=1 << 29), dict(renormalize=2), dict(reserved0=1), dict(ids=None),
                                 dict(weights=None), dict(offsets=None), dict(slots=None), dict(sources=None), dict(ids=(1 << 21) + 2),
                                 dict(work=None), dict(work=(1 << 26) + 8), dict(work_bytes=64)], ids=str)
def test_choose(D, bad):
    assert D.dm_choose_experts(choose(D, **bad)) == D.DM_ERR_INVALID_ARG


def test_choose_bytes(D):
    assert D.dm_choose_bytes(4, 8, 2) == 1 and D.dm_choose_bytes(0, 8, 2) == 1
    assert D.dm_choose_bytes(100_000, 64, 8) > 1
    for bad in ((4, 0, 1), (4, 1025, 1), (4, 8, 0), (4, 8, 9), (4, 64, 33), (1 << 30, 64, 2)):
        assert D.dm_choose_bytes(*bad) == 0
    assert D.lib().dm_choose_experts(None, None) == D.DM_ERR_INVALID_ARG


def linear(D, **kw):
    base = dict(x=1 << 22, y=1 << 23, status=1 << 25, work=1 << 26, work_bytes=1 << 30, x_row=96, y_row=64, dtype=D.DM_F16, y_dtype=D.DM_F16,
                rows=40, eps=-1.0)
    base.update(kw)
    return D.dm_linear_args(**base)


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=(1 << 22) + 8), dict(y=None), dict(y=(1 << 23) + 1), dict(status=None), dict(work=None),
                                 dict(work=(1 << 26) + 16), dict(work_bytes=256), dict(x_row=92), dict(x_row=88), dict(y_row=63), dict(dtype=2),
                                 dict(dtype=3), dict(y_dtype=2), dict(rows=1 << 31), dict(eps=float("nan"))], ids=str)
def test_linear(D, bad):
    assert D.dm_linear(eight(D, experts=1), linear(D, **bad)) == D.DM_ERR_INVALID_ARG


def test_linear_more(D):
    inv = D.DM_ERR_INVALID_ARG
    assert D.dm_linear(weights(D, experts=1), linear(D)) == inv     # 16-bit weights
    assert D.dm_linear(eight(D), linear(D)) == inv                  # many experts
    assert D.dm_linear_bytes(weights(D, experts=1), 4) == 0 and D.dm_linear_bytes(eight(D, experts=1), 40) > 1
    assert D.dm_linear_bytes(eight(D, experts=1), 4) == 1           # so few that no work buffer is wanted
    assert D.dm_linear(eight(D, experts=1), linear(D, rows=4, work=None, work_bytes=0, x=None)) == inv
    assert D.dm_linear(eight(D, experts=1), linear(D, rows=0)) == D.DM_OK


def layer(D, **kw):
    base = dict(x=1 << 22, logits=1 << 23, residual=1 << 24, y=1 << 25, status=1 << 26, work=1 << 27, work_bytes=1 << 40, x_row=96,
                logits_row=4, residual_row=96, y_row=96, dtype=D.DM_BF16, logits_dtype=D.DM_F32, tokens=5, top_k=2, renormalize=1)
    base.update(kw)
    return D.dm_experts_args(**base)


def down(D, make=weights, **kw):
    return make(D, **dict(dict(n=96, k=32, row=32, expert=96 * 32), **kw))


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=(1 << 22) + 8), dict(logits=None), dict(logits=(1 << 23) + 2), dict(residual=(1 << 24) + 1),
                                 dict(y=None), dict(y=(1 << 25) + 1), dict(status=None), dict(work=None), dict(work=(1 << 27) + 16),
                                 dict(work_bytes=1024), dict(x_row=92), dict(x_row=88), dict(logits_row=3), dict(residual_row=95),
                                 dict(y_row=95), dict(dtype=1), dict(dtype=2), dict(logits_dtype=2), dict(logits_dtype=4), dict(tokens=1 << 31),
                                 dict(top_k=0), dict(top_k=5), dict(renormalize=2), dict(reserved0=1)], ids=str)
def test_layer(D, bad):
    assert D.dm_experts(weights(D), down(D), layer(D, **bad)) == D.DM_ERR_INVALID_ARG


def test_layer_shapes(D):
    inv = D.DM_ERR_INVALID_ARG
    assert D.dm_experts_bytes(weights(D), down(D), 5, 2) > 0
    for up, dn in ((weights(D), down(D, k=33, row=40, expert=96 * 40)), (weights(D), down(D, n=95)), (weights(D), down(D, experts=3)),
                   (weights(D), down(D, make=eight)), (eight(D), down(D)), (weights(D, n=63), down(D))):
        assert D.dm_experts_bytes(up, dn, 5, 2) == 0
        assert D.dm_experts(up, dn, layer(D)) == inv
    assert D.dm_experts(weights(D), down(D), layer(D, tokens=0)) == D.DM_OK
    assert D.lib().dm_experts(None, None, C.byref(layer(D)), None) == inv
    assert D.lib().dm_experts(C.byref(weights(D)), C.byref(down(D)), None, None) == inv


def test_struct_layouts_match_header(D, tmp_path):
    import os
    hdr = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dualmap.h")
    structs = [D.dm_weights, D.dm_quantize_args, D.dm_choose_args, D.dm_product_args, D.dm_linear_args, D.dm_experts_args]
    lines = ["#include <stdio.h>", "#include <stddef.h>", f'#include "{hdr}"', "int main(void) {"]
    want = []
    for st in structs:
        lines.append(f'printf("%zu\\n", sizeof({st.__name__}));')
        want.append(C.sizeof(st))
        for f, _ in st._fields_:
            lines.append(f'printf("%zu\\n", offsetof({st.__name__}, {f}));')
            want.append(getattr(st, f).offset)
    prog = tmp_path / "layout.c"
    prog.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-o", str(tmp_path / "layout"), str(prog)], check=True)
    got = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == want
