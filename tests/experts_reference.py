"""Plain forms in 64 bits of the products and expert layers, and how far 32-bit
arithmetic may be from them."""

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}   # a rounding, relative
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}   # and next to zero


def padded(gen, rows, width, pad, dtype, values=None):
    """[rows, width] in rows that are `pad` elements longer and hold NaN (or 77) there."""
    x = torch.full((rows, width + pad), 77 if dtype is torch.int8 else float("nan"), dtype=dtype, device="cuda")
    new = torch.randn(rows, width, generator=gen, device="cuda") if values is None else values
    x[:, :width] = new.to(dtype)
    return x[:, :width]


def whole(gen, shape, most):
    """Whole numbers of -most .. most."""
    return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").float()


def pad_of(k, dtype):
    """Elements that make a row of k a multiple of 16 bytes."""
    return -k % (16 if dtype is torch.int8 else 8)


def sums(x, w, x_scale=None, scale=None):
    """(z, how far off 32-bit sums may be): z = x w^T (scaled) of one expert.

    A sum of k products in 32 bits, in whatever order and with roundings that
    may cut off (2^-23 each), is off by at most k 2^-23 of the sum of their
    sizes; 64 more for partial sums and scales."""
    z, size = x.double() @ w.double().T, x.double().abs() @ w.double().abs().T
    if scale is not None:
        f = x_scale.double()[:, None] * scale.double()
        z, size = z * f, size * f.abs()
    return z, (x.shape[1] + 64) * 2.0 ** -23 * size


def gate(z, off):
    """silu(g) u and how far off it may be.  |silu'| <= 1.1; the exponential is
    off by (2 + 1.2 |g|) 2^-23, the division and the products by 2^-22 each."""
    g, u = z.chunk(2, -1)
    dg, du = off.chunk(2, -1)
    s = g * torch.sigmoid(g)
    y = s * u
    return y, 1.1 * dg * (u.abs() + du) + s.abs() * du + y.abs() * (8 + 2 * g.abs()) * 2.0 ** -23


def round_off(y, off, dtype):
    """How far off a value may be that is off by `off` and then rounded."""
    return off + (y.abs() + off) * HALF[dtype] + TINY[dtype]


def close(got, want, off):
    far = (got.double() - want).abs()
    bad = ~(far <= off)
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:3].tolist(), float((far / off.clamp(min=1e-300)).nan_to_num(nan=1e9).max()))


def quantized(x):
    """(q, scale) of a matrix, in 64 bits."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    q = torch.where(top > 0, torch.round(127 * x / torch.where(top > 0, top, 1.0)), 0.0)
    return q, (top / 127)[:, 0]


def chosen(logits, top_k, renormalize):
    """ids and weights, token by token in Python."""
    ids, weights = [], []
    for row in logits.double().tolist():
        order = sorted((e for e in range(len(row)) if row[e] > -float("inf")), key=lambda e: (-row[e], e))[:top_k]
        pick = torch.tensor([row[e] for e in order], dtype=torch.float64)
        base = torch.logsumexp(pick if renormalize else torch.tensor(row, dtype=torch.float64), 0) if order else 0.0
        ids.append(order + [-1] * (top_k - len(order)))
        weights.append(torch.exp(pick - base).tolist() + [0.0] * (top_k - len(order)))
    return ids, torch.tensor(weights, dtype=torch.float64)


def sorted_pairs(ids, experts):
    """(offsets, slots, sources) of ids [tokens][top_k], in Python."""
    pairs = [(e, i) for i, e in enumerate(x for row in ids for x in row)]
    order = [i for e, i in sorted(p for p in pairs if p[0] >= 0)]
    slots = [-1] * len(pairs)
    for s, i in enumerate(order):
        slots[i] = s
    flat = [e for e, _ in pairs]
    offsets = [sum(0 <= e < x for e in flat) for x in range(experts + 1)] if experts <= 64 else None
    return offsets, slots, order + [-1] * (len(pairs) - len(order))
