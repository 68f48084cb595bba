"""Products with 16-bit and 8-bit weights, quantised rows, the choice of experts
and the expert layer, against plain forms in 64 bits."""

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


def ints(torch, x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# -- rows in 8 bits -----------------------------------------------------------------

@pytest.mark.parametrize("rows,k,dtype,norm", [(1, 1, "bfloat16", False), (3, 16, "float16", True), (61, 1024, "bfloat16", True),
                                               (9, 1031, "float16", False), (300, 2048, "bfloat16", False), (7, 2049, "bfloat16", True),
                                               (5, 16384, "float16", False), (4, 16385, "bfloat16", True), (2, 40003, "float16", True),
                                               (3000, 64, "float16", False)])
def test_quantize(torch, rows, k, dtype, norm):
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    t = getattr(torch, dtype)
    x = R.padded(gen(torch, k), rows, k, R.pad_of(k, t) + 8, t)
    if rows > 4:
        x[2] = 0
        x[3] *= 2.0 ** -14 if t is torch.float16 else 1e-33
        x[4, :] = (torch.arange(k, device="cuda") % 255 - 127).to(t)   # and borders: halves of a top of 254
        x[4, 0] = 254
    q, scale = X.quantize(x, eps=1e-6 if norm else None)
    want, ref = R.quantized(x)
    assert torch.equal(q.double(), want)
    # a division's rounding; with a norm also the sum of the squares (up to 8 values of k / 256 vectors one
    # after another and 16 sums of sums), a division and a reciprocal root, whose error is 2 units
    off = 2.0 ** -24
    if norm:
        ref = ref / (x.double().square().mean(-1) + 1e-6).sqrt()
        off = (k / 32 + 80) * 2.0 ** -24
    assert bool(((scale.double() - ref).abs() <= ref * off + 2.0 ** -149).all())


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_quantize_every_value_against_every_top(torch, dtype):
    """All positive finite values below each of many tops, the multiples of 127 among them."""
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    t = getattr(torch, dtype)
    every = torch.arange(0, 0x7F80 if t is torch.bfloat16 else 0x7C00, 16 if t is torch.bfloat16 else 1, dtype=torch.int32, device="cuda")
    every = every.to(torch.int16).view(t)
    tops = [1.0, 127.0, 254.0, 255.0, 1016.0, 3.140625, 0.9921875, 2.0 ** -20, 65504.0 if t is torch.float16 else 3.3e38]
    tops += [1905.0, 889.0, 6.0e-8] if t is torch.float16 else [1.2e-38, 1e-40, 5e37]
    rows = []
    for top in tops:
        top = torch.tensor(top, device="cuda").to(t)
        row = torch.where(every.float() <= top.float(), every, top)
        row[0] = -top
        rows.append(row)
    x = torch.stack(rows)
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % 8))
    q, _ = X.quantize(x)
    want, _ = R.quantized(x)
    assert torch.equal(q.double(), want)


def test_quantize_what_is_not_finite(torch):
    from paper_2602_06502_gb300 import experts as X
    x = torch.ones(5, 300, device="cuda", dtype=torch.bfloat16)[:, :296].contiguous()
    x[1, 7], x[2, 290], x[3, 0] = float("inf"), float("nan"), -float("inf")
    q, scale = X.quantize(x)
    assert (q[1:4] == 0).all() and torch.isnan(scale[1:4]).all() and (q[[0, 4]] == 127).all()
    count = ints(torch, [2])
    out = X.quantize(x, count=count)
    assert torch.equal(out[0][:2], q[:2])


# -- products -----------------------------------------------------------------------

ROWS = {"few": [1, 0, 3, 8], "tiles": [9, 0, 17, 1, 0], "wide": [130, 1, 0, 64], "one": [5], "many": [700], "none": [0, 0, 0],
        "long": [257, 31, 513], "all": [0, 40], "one of many": [900] + [3, 0, 1, 5] * 40 + [64, 65]}


def case(torch, seed, rows, k, n, dtype, gated=False, exact=True, spare=0):
    """Inputs of a grouped product; exact: whole numbers whose sums 32 bits hold."""
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    t, g = getattr(torch, dtype), gen(torch, seed)
    E, total, wide = len(rows), sum(rows) + spare, n * (2 if gated else 1)
    most = 127 if t is torch.int8 else 4
    make = (lambda *s: R.whole(g, s, most)) if exact or t is torch.int8 else (lambda *s: torch.randn(s, generator=g, device="cuda"))
    x = R.padded(g, total, k, R.pad_of(k, t), t, make(total, k))
    w = R.padded(g, E * wide, k, R.pad_of(k, t) + (16 if k % 3 == 0 else 0), t, make(E * wide, k) * (1 if exact or t is torch.int8 else k ** -0.5))
    xs = ws = None
    if t is torch.int8:
        xs = torch.rand(total, generator=g, device="cuda") * 2.0 ** -7 + 2.0 ** -9
        ws = torch.rand(E, wide, generator=g, device="cuda") * 2.0 ** -7 + 2.0 ** -9
    offsets = [0]
    for r in rows:
        offsets.append(offsets[-1] + r)
    return x, xs, X.Weights(w.unflatten(0, (E, wide)), ws), offsets, t


SHAPES = [("few", 64, 16), ("few", 1024, 256), ("tiles", 200, 48), ("tiles", 1000, 129), ("wide", 512, 384), ("wide", 72, 33), ("one", 31, 1),
          ("one", 4096, 100), ("many", 320, 520), ("none", 64, 64), ("long", 1408, 264), ("all", 96, 8),
          ("one of many", 520, 160)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "int8"])
@pytest.mark.parametrize("rows,k,n", SHAPES)
def test_product(torch, rows, k, n, dtype, gated):
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    x, xs, w, offsets, t = case(torch, k + n, ROWS[rows], k, n, dtype, gated, exact=False, spare=3)
    out_t = torch.float16 if dtype == "float16" else torch.bfloat16
    out = torch.full((x.shape[0], n), 7.0, dtype=out_t, device="cuda")
    y = X.product(x, w, ints(torch, offsets), x_scale=xs, gated=gated, out=out)
    assert y is out and w.last_error() == 0
    assert (y[offsets[-1]:] == 7).all()   # rows that are nobody's
    for e, (a, b) in enumerate(zip(offsets, offsets[1:])):
        if a < b:
            z, off = R.sums(x[a:b], w.w[e], None if xs is None else xs[a:b], None if xs is None else w.scale[e])
            if gated:
                z, off = R.gate(z, off)
            R.close(y[a:b], z, R.round_off(z, off, out_t))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "int8"])
@pytest.mark.parametrize("rows,k,n", SHAPES)
def test_product_of_whole_numbers_is_exact(torch, rows, k, n, dtype):
    """Sums that 32 bits hold: nothing but the last rounding, and none in 32 bits."""
    from paper_2602_06502_gb300 import experts as X
    k = min(k, 1040) if dtype == "int8" else k
    x, xs, w, offsets, t = case(torch, k + n, ROWS[rows], k, n, dtype)
    if xs is not None:
        xs.fill_(0.5)
        w.scale.fill_(2.0)
    y = X.product(x, w, ints(torch, offsets), x_scale=xs, dtype=torch.float32)
    for e, (a, b) in enumerate(zip(offsets, offsets[1:])):
        assert torch.equal(y[a:b].double(), x[a:b].double() @ w.w[e].double().T)
    assert w.last_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "int8"])
@pytest.mark.parametrize("rows,k,n,gated", [("few", 264, 40, True), ("wide", 264, 40, False), ("long", 96, 300, True),
                                            ("one of many", 520, 160, False)])
def test_product_of_chosen_rows(torch, rows, k, n, dtype, gated):
    """Rows that name the rows of x they read, several the same one; y in rows of odd width."""
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    x, xs, w, offsets, t = case(torch, k + n, ROWS[rows], k, n, dtype, gated, exact=False)
    total, few = offsets[-1], max(1, offsets[-1] // 3)
    sources = torch.randint(0, 3 * few, (total,), generator=gen(torch, 5), device="cuda").int()
    x, xs = x[:few], None if xs is None else xs[:few].contiguous()
    out = torch.full((total, n + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    X.product(x, w, ints(torch, offsets), x_scale=xs, gated=gated, sources=sources, per_source=3, out=out[:, 1:n + 1])
    assert (out[:, 0] == 7).all() and (out[:, n + 1:] == 7).all()
    for e, (a, b) in enumerate(zip(offsets, offsets[1:])):
        if a < b:
            at = (sources[a:b] // 3).long()
            z, off = R.sums(x[at], w.w[e], None if xs is None else xs[at], None if xs is None else w.scale[e])
            if gated:
                z, off = R.gate(z, off)
            R.close(out[a:b, 1:n + 1], z, R.round_off(z, off, torch.bfloat16))
    assert w.last_error() == 0


@pytest.mark.parametrize("rows", [1, 4, 7, 8, 9, 16, 33, 128, 129, 500])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_linear(torch, rows, dtype):
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    t, g = getattr(torch, dtype), gen(torch, rows)
    k, n = 1024, 392
    x = R.padded(g, rows, k, 0, t)
    real = R.padded(g, n, k, 0, t) * k ** -0.5
    w = X.Weights.quantized(real)
    want, ref = R.quantized(real)
    assert torch.equal(w.w.double(), want)
    for eps in (None, 1e-6):
        y = X.Linear(w)(x, eps=eps)
        q, scale = X.quantize(x, eps=eps)
        z, off = R.sums(q, w.w, scale, w.scale)
        R.close(y, z, R.round_off(z, off, t))
    y = X.Linear(X.Weights(real))(x)
    z, off = R.sums(x, real)
    R.close(y, z, R.round_off(z, off, t))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("k,n", [(16, 1), (31, 40), (72, 24), (1024, 40), (1031, 17), (4100, 200)])
@pytest.mark.parametrize("rows", [1, 3, 8, 9])
def test_linear_steps_are_the_quantised_rows(torch, rows, k, n, dtype):
    """Few rows are quantised within the product: their steps are dm_quantize's, borders and all, so whole numbers as
    scales give the bits of the two calls."""
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    t, g = getattr(torch, dtype), gen(torch, rows + k)
    x = R.padded(g, rows, k, R.pad_of(k, t) + 8, t)
    if rows > 2:
        x[1] = (torch.arange(k, device="cuda") % 255 - 127).to(t)   # halves of a top of 254
        x[1, 0] = 254
        x[2] = 0
    if rows > 3:
        x[3] *= 2.0 ** -14 if t is torch.float16 else 1e-33
        x[4, k // 2] = float("nan")
    pad = R.pad_of(k, torch.int8)
    w = X.Weights(R.padded(g, n, k, pad, torch.int8, R.whole(g, (n, k), 127)), torch.rand(n, generator=g, device="cuda") + 0.5)
    q, scale = X.quantize(x)
    want = X.product(q, w, x_scale=scale, dtype=torch.float32)
    y = X.Linear(w)(x, out=torch.empty(rows, n, device="cuda"))
    if k <= 1024:   # exact sums
        assert torch.equal(y.nan_to_num(nan=7e30), want.nan_to_num(nan=7e30))
    z, off = R.sums(q, w.w, scale, w.scale)
    ok = torch.isfinite(scale)
    R.close(y[ok], z[ok], R.round_off(z[ok], off[ok], torch.float32))
    assert torch.isnan(y[~ok]).all()
    y = X.Linear(w)(x, eps=1e-6, out=torch.empty(rows, n, device="cuda"))
    q, scale = X.quantize(x, eps=1e-6)
    z, off = R.sums(q, w.w, scale, w.scale)
    # and the two sums of squares, each of k terms
    R.close(y[ok], z[ok], R.round_off(z[ok], off[ok] + z[ok].abs() * (k / 16 + 64) * 2.0 ** -24, torch.float32))


# -- the choice of experts -------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("tokens,experts,top_k", [(1, 1, 1), (4, 8, 2), (1, 1024, 32), (33, 33, 7), (128, 64, 8), (129, 64, 8), (600, 100, 3),
                                                  (40, 40, 32), (2000, 257, 1), (0, 8, 2)])
def test_choose(torch, tokens, experts, top_k, dtype):
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    g = gen(torch, tokens + experts)
    logits = (torch.randn(tokens, experts + 5, generator=g, device="cuda") * 3).to(getattr(torch, dtype))[:, :experts]
    if tokens > 30:
        logits[3] = -float("inf")                       # padding
        logits[4, 1:] = -float("inf")                   # one expert
        logits[5] = 1.0                                 # all alike
        logits[6, ::2] = -float("inf")
        logits[:, experts // 2] = -float("inf")         # an expert that is off
        logits[7, 0], logits[7, 1] = 0.0, -0.0
    for renormalize in (True, False):
        c = X.choose(logits, top_k, renormalize=renormalize)
        ids, weights = R.chosen(logits.cpu(), top_k, renormalize)
        assert c.ids.tolist() == ids
        offsets, slots, sources = R.sorted_pairs(ids, experts)
        assert c.slots.flatten().tolist() == slots and c.sources.tolist() == sources
        if offsets is not None:
            assert c.offsets.tolist() == offsets
        # an exponential's two units, a sum of up to 1,024 of them, a division
        if tokens:
            R.close(c.weights.cpu(), weights, weights * (experts / 32 + 16) * 2.0 ** -23 + 2.0 ** -126)


def test_choose_what_is_not_a_number(torch):
    from paper_2602_06502_gb300 import experts as X
    x = torch.zeros(4, 6, device="cuda")
    x[1, 2], x[2, :], x[3, 4] = float("nan"), float("nan"), float("inf")
    c = X.choose(x, 6)
    assert c.ids[1].tolist() == [0, 1, 3, 4, 5, 2] and c.ids[2].tolist() == [0, 1, 2, 3, 4, 5] and c.ids[3, 0] == 4
    assert torch.isnan(c.weights[1:]).all() and not torch.isnan(c.weights[0]).any()


# -- the layer -----------------------------------------------------------------------------

def make_layer(torch, seed, tokens, experts, k, m, dtype, eight):
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    t, g = getattr(torch, dtype), gen(torch, seed)
    x = R.padded(g, tokens, k, R.pad_of(k, t), t)
    up = torch.randn(experts, 2 * m, k, generator=g, device="cuda") * k ** -0.5
    down = torch.randn(experts, k, m, generator=g, device="cuda") * m ** -0.5
    ws = []
    for w in (up, down):
        wide = -(-w.shape[-1] // 16) * 16
        held = torch.zeros(w.shape[:-1] + (wide,), dtype=t, device="cuda")
        held[..., :w.shape[-1]] = w.to(t)
        if eight:
            q, s = X.quantize(held.flatten(0, 1))
            ws.append(X.Weights(q.unflatten(0, w.shape[:2])[..., :w.shape[-1]], s.unflatten(0, w.shape[:2])))
        else:
            ws.append(X.Weights(held[..., :w.shape[-1]]))
    logits = torch.randn(tokens, experts, generator=g, device="cuda")
    if tokens > 5:
        logits[2] = -float("inf")
        logits[:, 0] = -float("inf")
    residual = torch.randn(tokens, k, generator=g, device="cuda").to(t) if k % 8 == 0 else None
    return x, ws[0], ws[1], logits, residual, t


LAYERS = [(1, 4, 2, 64, 32), (4, 8, 2, 1024, 256), (37, 12, 3, 200, 104), (129, 16, 4, 512, 264), (600, 5, 2, 264, 40), (64, 64, 8, 128, 48),
          (9, 3, 3, 61, 27), (2048, 4, 1, 128, 64)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("tokens,experts,top_k,k,m", LAYERS)
def test_layer(torch, tokens, experts, top_k, k, m, dtype):
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    x, up, down, logits, residual, t = make_layer(torch, tokens + k, tokens, experts, k, m, dtype, False)
    for renormalize in (True, False):
        y = X.Experts(up, down, top_k, renormalize=renormalize)(x, logits, residual=residual)
        ids, weights = R.chosen(logits.cpu(), top_k, renormalize)
        ids, weights = torch.tensor(ids, device="cuda"), weights.cuda()
        want = torch.zeros(tokens, k, dtype=torch.float64, device="cuda") if residual is None else residual.double()
        off = torch.zeros_like(want)
        size = want.abs()
        for e in range(experts):
            at, place = torch.nonzero(ids == e, as_tuple=True)
            if not at.numel():
                continue
            h, dh = R.gate(*R.sums(x[at], up.w[e]))
            dh = R.round_off(h, dh, t)                       # h is held in x's type
            z, dz = R.sums(h, down.w[e])
            dz = dz + dh @ down.w[e].double().abs().T
            f = weights[at, place, None]
            want.index_add_(0, at, f * z)
            size.index_add_(0, at, f * z.abs())
            off.index_add_(0, at, f * dz + f * z.abs() * (experts / 32 + 16) * 2.0 ** -23)   # the weights'
        off = off + size * (top_k + 1) * 2.0 ** -23          # the sum of the parts
        R.close(y, want, R.round_off(want, off, t))
    assert up.last_error() == 0 and down.last_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("tokens,experts,top_k,k,m", LAYERS)
def test_layer_in_8_bits_is_its_parts(torch, tokens, experts, top_k, k, m, dtype):
    """The layer's pieces one by one, each tested above, give what the layer gives."""
    from paper_2602_06502_gb300 import experts as X
    import experts_reference as R
    x, up, down, logits, residual, t = make_layer(torch, tokens + m, tokens, experts, k, m, dtype, True)
    y = X.Experts(up, down, top_k)(x, logits, residual=residual)
    c = X.choose(logits, top_k)
    q, scale = X.quantize(x)
    h = torch.empty(tokens * top_k, -(-m // 8) * 8, dtype=t, device="cuda")[:, :m]
    X.product(q, up, c.offsets, x_scale=scale, sources=c.sources, per_source=top_k, gated=True, out=h)
    hq, h_scale = X.quantize(h, count=c.offsets[experts:])
    parts = X.product(hq, down, c.offsets, x_scale=h_scale, dtype=torch.float32)
    parts = torch.where(c.slots[..., None] >= 0, parts[c.slots.long()].double(), 0.0) * c.weights[..., None].double()
    want = parts.sum(1) + (0 if residual is None else residual.double())
    size = parts.abs().sum(1) + (0 if residual is None else residual.double().abs())
    # a residual, top_k products and sums in 32 bits; the pieces are the layer's own kernels
    R.close(y, want, R.round_off(want, size * (top_k + 1) * 2.0 ** -23, t))
    assert up.last_error() == 0 and down.last_error() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "int8"])
@pytest.mark.parametrize("most", [4, 40])
def test_product_of_many_experts(torch, dtype, most):
    """1,024 experts, some without rows, by both kernels: whole numbers, so nothing but the rounding."""
    import random

    from paper_2602_06502_gb300 import experts as X
    rng = random.Random(most)
    rows = [rng.randint(0, most) for _ in range(1024)]
    x, xs, w, offsets, t = case(torch, most, rows, 64, 24, dtype)
    if xs is not None:
        xs.fill_(0.5)
        w.scale.fill_(2.0)
    y = X.product(x, w, ints(torch, offsets), x_scale=xs, dtype=torch.float32)
    of = torch.repeat_interleave(torch.arange(1024, device="cuda"), torch.tensor(rows, device="cuda"))
    assert torch.equal(y.double(), torch.einsum("rk,rnk->rn", x.double(), w.w[of].double())) and w.last_error() == 0


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens", [0, 1, 20, 300])
def test_layer_of_one_expert(torch, tokens, eight):
    """Every token goes to the one expert, with a weight of 1: what its parts give."""
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    x, up, down, _, residual, t = make_layer(torch, tokens + 1, tokens, 1, 512, 96, "bfloat16", eight)
    logits = torch.randn(tokens, 1, generator=gen(torch, 3), device="cuda")
    y = X.Experts(up, down, 1)(x, logits, residual=residual)
    assert y.shape == (tokens, 512)
    off = ints(torch, [0, tokens])
    q, scale = X.quantize(x) if eight else (x, None)
    h = X.product(q, up, off, x_scale=scale, gated=True, dtype=t)
    hq, h_scale = X.quantize(h) if eight else (h, None)
    want = X.product(hq, down, off, x_scale=h_scale, dtype=torch.float32).double() + residual.double()
    R.close(y, want, R.round_off(want, (want.abs() + 2 * residual.double().abs()) * 2.0 ** -22, t))   # one sum and its rounding
    assert up.last_error() == 0 and down.last_error() == 0


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens", [7, 200])
def test_layer_keeps_bad_tokens_apart(torch, tokens, eight):
    """A token whose row or scores are not numbers is NaN, and the others are what they were."""
    from paper_2602_06502_gb300 import experts as X
    x, up, down, logits, residual, t = make_layer(torch, tokens, tokens, 6, 256, 64, "float16", eight)
    logits = torch.randn(tokens, 6, generator=gen(torch, 4), device="cuda")
    e = X.Experts(up, down, 2)
    want = e(x, logits, residual=residual)
    x, logits = x.clone(), logits.clone()
    x[1, 3], x[4, 200], logits[5, 2] = float("nan"), float("inf"), float("nan")
    y = e(x, logits, residual=residual)
    bad = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    bad[[1, 4, 5]] = True
    assert torch.isnan(y[[1, 5]]).all() and not torch.isfinite(y[4]).any()
    assert torch.equal(y[~bad], want[~bad]) and up.last_error() == 0


def test_choose_for_many_tokens(torch):
    """More tokens than 32 bits of threads: 2^27 + 77 in rows of eight scores; the first, the last and the sums."""
    from paper_2602_06502_gb300 import experts as X
    tokens = (1 << 27) + 77
    logits = torch.zeros(tokens, 8, dtype=torch.bfloat16, device="cuda")
    logits[::2, 3] = 1                       # ties go to the lowest id
    logits[1::4, 6] = 2
    logits[-2:] = -float("inf")
    c = X.choose(logits, 1)
    del logits
    want = torch.zeros(tokens, dtype=torch.int32, device="cuda")
    want[::2], want[1::4], want[-2:] = 3, 6, -1
    assert torch.equal(c.ids[:, 0], want)
    counts = torch.stack([(want == e).sum() for e in range(8)])
    assert torch.equal(c.offsets[1:].long(), counts.cumsum(0)) and int(c.offsets[0]) == 0
    total = int(counts.sum())
    for e in (0, 3, 6):
        a, b = int(c.offsets[e]), int(c.offsets[e + 1])
        assert torch.equal(c.sources[a:b].long(), torch.nonzero(want == e)[:, 0])
    assert (c.sources[total:] == -1).all() and (c.slots[-2:] == -1).all()
    assert torch.equal(c.slots[c.sources[:total].long(), 0], torch.arange(total, dtype=torch.int32, device="cuda"))
