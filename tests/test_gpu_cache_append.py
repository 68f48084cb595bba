"""dm_cache_append against the formula in float64: norm per head, rotation,
slots of keys and values, strides, refusals."""

import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    lib_ready()
    import torch
    return torch


def tables(torch, rows, rot):
    inv = 10_000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / max(rot, 1))
    a = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * inv
    return a.cos().float(), a.sin().float()


def reference(torch, x, w, eps, cos, sin, pos, rot, interleaved):
    """(value, sum of the magnitudes that were added) in float64"""
    x = x.double()
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    if not rot:
        return x, x.abs()
    c, s = cos.double()[pos][:, None], sin.double()[pos][:, None]
    r, y, mag = x[..., :rot], x.clone(), x.abs()
    i = torch.arange(0, rot, 2, device=x.device) if interleaved else torch.arange(rot // 2, device=x.device)
    j = i + 1 if interleaved else i + rot // 2
    a, b = r[..., i], r[..., j]
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    mag[..., i], mag[..., j] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, mag


def check(torch, got, want, mag, dtype):
    # one rounding of the result, some 2^-24 steps before it: the mean square of up to 128
    # terms, its root, two products and a sum: less than 2^-19 of the magnitudes
    u = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    far = (got.double() - want).abs() - (u * want.abs() + 2.0 ** -19 * mag + 2.0 ** -25)
    assert bool((far <= 0).all()), far.max().item()


CASES = [
    # page, layout, dtype, dim, kv heads, q heads, new tokens, own tokens, rot, interleaved, norms
    (16, "heads", "bfloat16", 128, 8, 32, [1] * 61, [0, 15, 16, 17, 4000] + [100 + i for i in range(56)], 128, False, True),
    (16, "tokens", "float16", 64, 2, 2, [5, 0, 1, 33], [0, 3, 31, 7], 64, True, True),
    (64, "heads", "float16", 128, 1, 7, [200, 1], [0, 63], 64, False, True),
    (4, "tokens", "bfloat16", 64, 3, 6, [3, 9, 4], [1, 0, 2], 32, True, False),
    (8, "heads", "bfloat16", 128, 5, 15, [1], [0], 16, False, True),
    (32, "heads", "bfloat16", 64, 4, 12, [17, 31, 0, 2], [15, 1, 40, 30], 0, False, True),
    (16, "heads", "float16", 128, 2, 16, [1500, 700], [10, 0], 112, False, True),
]


@pytest.mark.parametrize("page,layout,dtype,dim,hk,hq,new,own,rot,inter,norms", CASES)
@pytest.mark.parametrize("packed", [False, True])
def test_append(torch, page, layout, dtype, dim, hk, hq, new, own, rot, inter, norms, packed):
    import cache_reference as R
    dt = getattr(torch, dtype)
    b = R.make_batch(5, page=page, kv_heads=hk, dim=dim, dtype=dt, layout=layout, own=own, new=new, layers=2, junk=False)
    c, T = b["cache"], b["tokens"]
    x = (torch.randn(T, hq + 2 * hk, dim, generator=b["gen"], device="cuda") * 3).to(dt)
    x[0] = 0     # a zero vector stays one
    if packed:
        q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    else:
        q, k, v = x[:, :hq].contiguous(), x[:, hq:hq + hk].contiguous(), x[:, hq + hk:].transpose(0, 1).contiguous().transpose(0, 1)
    qw = (1 + 0.3 * torch.randn(dim, generator=b["gen"], device="cuda")).to(dt) if norms else None
    kw = (1 + 0.3 * torch.randn(dim, generator=b["gen"], device="cuda")).to(dt)
    cos, sin = tables(torch, max(b["length"]), rot) if rot else (None, None)
    want_k, want_v = c.k.clone(), c.v.clone()
    raw_q, raw_k, raw_v = q.clone(), k.clone(), v.clone()
    out = q if packed else None   # in place
    got = c.append(b["seqs"], b["offsets"], q, k, v, cos, sin, layer=1, q_weight=qw, k_weight=kw, eps=1e-5, interleaved=inter, out=out)
    assert c.last_error() == 0
    pos = torch.cat([torch.arange(n - w, n, device="cuda") for n, w in zip(b["length"], new)])
    ref, mag = reference(torch, raw_q, qw, 1e-5, cos, sin, pos, rot, inter)
    check(torch, got, ref, mag, dt)
    ref_k, mag_k = reference(torch, raw_k, kw, 1e-5, cos, sin, pos, rot, inter)
    t = 0
    for i, (n, w) in enumerate(zip(b["length"], new)):
        for p in range(n - w, n):
            at = (1, b["rows"][i][p // page], slice(None), p % page) if layout == "heads" else (1, b["rows"][i][p // page], p % page)
            if t < 300 or t > T - 50:
                check(torch, c.k[at], ref_k[t], mag_k[t], dt)
                assert torch.equal(c.v[at], raw_v[t])
            want_k[at], want_v[at] = c.k[at], c.v[at]
            t += 1
    assert torch.equal(want_k, c.k) and torch.equal(want_v, c.v)   # nothing else was written


def test_keys_alone(torch):
    """No queries: q of zero heads."""
    import cache_reference as R
    b = R.make_batch(6, page=16, kv_heads=2, dim=64, dtype=torch.bfloat16, own=[3, 20], new=[2, 1])
    c = b["cache"]
    k, v = (torch.randn(3, 2, 64, generator=b["gen"], device="cuda").bfloat16() for _ in range(2))
    c.append(b["seqs"], b["offsets"], k[:, :0], k, v)
    assert c.last_error() == 0
    assert torch.equal(R.read_seq(b, c.k, 0)[3:], k[:2]) and torch.equal(R.read_seq(b, c.v, 1)[20:], v[2:])


def test_rows_outside_the_offsets(torch):
    import cache_reference as R
    b = R.make_batch(7, page=16, kv_heads=1, dim=64, dtype=torch.float16, own=[4], new=[3])
    c = b["cache"]
    x = torch.randn(10, 1, 64, generator=b["gen"], device="cuda").half()
    out = torch.full_like(x, 9.0)
    c.append(b["seqs"], R.ints([2, 5]), x, x, x, out=out)
    assert c.last_error() == 0
    assert bool((out[:2] == 9).all()) and bool((out[5:] == 9).all()) and torch.equal(out[2:5], x[2:5])
    assert torch.equal(R.read_seq(b, c.k, 0)[4:], x[2:5])


def test_refusals(torch):
    import cache_reference as R
    from paper_2602_06502_gb300 import dualmap as D
    b = R.make_batch(8, page=16, kv_heads=2, dim=64, dtype=torch.bfloat16, own=[3, 20], new=[2, 1], junk=False)
    c, T = b["cache"], b["tokens"]
    x = torch.randn(T, 4, 64, generator=b["gen"], device="cuda").bfloat16()
    q, k = x, x[:, :2].contiguous()
    cos, sin = tables(torch, 64, 64)
    before = c.k.clone()
    ok = dict(layer=0)
    for bad in (dict(layer=1), dict(eps=-1.0), dict(eps=float("nan"))):
        with pytest.raises(D.DualMapError):
            c.append(b["seqs"], b["offsets"], q, k, k, cos, sin, **{**ok, **bad})
    with pytest.raises(D.DualMapError):   # three query heads to two key heads
        c.append(b["seqs"], b["offsets"], q[:, :3], k, k, cos, sin)
    with pytest.raises(D.DualMapError):   # 24 dims turn
        c.append(b["seqs"], b["offsets"], q, k, k, *tables(torch, 64, 24))
    odd = torch.empty(T * 4 * 65 + 8, dtype=torch.bfloat16, device="cuda").as_strided((T, 4, 64), (4 * 65, 65, 1))
    with pytest.raises(D.DualMapError):   # heads that do not begin on 16 bytes
        c.append(b["seqs"], b["offsets"], odd, k, k, cos, sin)
    with pytest.raises(ValueError):
        c.append(b["seqs"], b["offsets"], q.half(), k, k, cos, sin)
    with pytest.raises(ValueError):
        c.append(b["seqs"], b["offsets"], q, k[:2], k, cos, sin)
    with pytest.raises(ValueError):
        c.append(b["seqs"], b["offsets"], q, k, k, cos)
    assert torch.equal(before, c.k) and c.last_error() == 0
    inv = D.DM_ERR_INVALID_ARG
    c.append(R.ints([99, 98]), b["offsets"], q, k, k, cos, sin)
    assert c.last_error() == inv
    c.append(b["seqs"], b["offsets"], q, k, k, cos[:4], sin[:4])     # positions beyond the rotation's table
    assert c.last_error() == inv
    c.append(b["seqs"], R.ints([0, 3, 4]), q, k, k, cos, sin)       # more rows than there are
    assert c.last_error() == inv
    c.lengths[b["place"][1]] = 0                                   # more new tokens than the sequence has
    c.append(b["seqs"], b["offsets"], q, k, k, cos, sin)
    assert c.last_error() == inv


def test_a_sequence_named_twice(torch):
    """Two of a call's entries with tokens for one sequence are refused, wherever they stand; other orders of the
    same sequences, one after another, are not."""
    import cache_reference as R
    from paper_2602_06502_gb300 import dualmap as D
    n = 300
    b = R.make_batch(9, page=16, kv_heads=1, dim=64, dtype=torch.float16, own=[20 + i % 7 for i in range(n)], new=[1] * n)
    c, place = b["cache"], b["place"]
    x = torch.randn(n, 1, 64, generator=b["gen"], device="cuda").half()
    once = R.ints(range(n + 1))
    for order in (place, place[::-1], place[7:] + place[:7], place):
        c.append(R.ints(order), once, x, x, x)
        assert c.last_error() == 0
    for i, j in ((0, 1), (3, 299), (120, 121), (0, 299)):
        order = list(place)
        order[j] = order[i]
        for _ in range(3):
            c.append(R.ints(order), once, x, x, x)
            assert c.last_error() == D.DM_ERR_INVALID_ARG
        # without tokens the second is no writer
        gaps = [0]
        for k in range(n):
            gaps.append(gaps[-1] + (k != j))
        c.append(R.ints(order), R.ints(gaps), x[:n - 1], x[:n - 1], x[:n - 1])
        assert c.last_error() == 0
        c.append(b["seqs"], once, x, x, x)
        assert c.last_error() == 0
    for i in (0, 150, 299):
        assert torch.equal(R.read_seq(b, c.k, i)[-1], x[i]) and torch.equal(R.read_seq(b, c.v, i)[-1], x[i])


@pytest.mark.parametrize("page,layout,dtype,dim,hk,hq,new,own,rot,inter,norms", CASES)
def test_every_row_is_stored(torch, page, layout, dtype, dim, hk, hq, new, own, rot, inter, norms):
    """All keys and values of a call, gathered from their slots at once, and all slots that are not theirs."""
    import cache_reference as R
    dt = getattr(torch, dtype)
    b = R.make_batch(15, page=page, kv_heads=hk, dim=dim, dtype=dt, layout=layout, own=own, new=new, layers=2, junk=False)
    c, T = b["cache"], b["tokens"]
    x = (torch.randn(T, hq + 2 * hk, dim, generator=b["gen"], device="cuda") * 3).to(dt)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    qw, kw = ((1 + 0.3 * torch.randn(dim, generator=b["gen"], device="cuda")).to(dt) if norms else None for _ in range(2))
    cos, sin = tables(torch, max(b["length"]), rot) if rot else (None, None)
    held = c.k.clone(), c.v.clone()
    got = c.append(b["seqs"], b["offsets"], q, k, v, cos, sin, layer=1, q_weight=qw, k_weight=kw, eps=1e-5, interleaved=inter)
    assert c.last_error() == 0
    pos = torch.cat([torch.arange(n - w, n, device="cuda") for n, w in zip(b["length"], new)])
    at = torch.tensor([b["rows"][i][p // page] for i, (n, w) in enumerate(zip(b["length"], new)) for p in range(n - w, n)],
                      dtype=torch.long, device="cuda")
    where = (1, at, slice(None), pos % page) if layout == "heads" else (1, at, pos % page)
    check(torch, got, *reference(torch, q, qw, 1e-5, cos, sin, pos, rot, inter), dt)
    check(torch, c.k[where], *reference(torch, k, kw, 1e-5, cos, sin, pos, rot, inter), dt)
    assert torch.equal(c.v[where], v)
    for pool, before in zip((c.k, c.v), held):
        pool[where] = before[where]
        assert torch.equal(pool, before)
