"""Attention over the paged cache (dm_cache_plan, dm_cache_attend) against
float64, at the edges of pages, tiles, units and CTAs; slots behind a
sequence's end and free pages hold infinities and NaN."""

import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    lib_ready()
    import torch
    return torch


def run(torch, seed, *, hq, scale=None, gain=1.0, strided=False, layer=0, **kw):
    import cache_reference as R
    b = R.make_batch(seed, **kw)
    c, T, D = b["cache"], b["tokens"], kw["dim"]
    q = (torch.randn(T, hq + 3, D, generator=b["gen"], device="cuda") * gain).to(kw["dtype"])[:, :hq]
    if not strided:
        q = q.contiguous()
    out = torch.full((T, D, hq + 1) if False else (T, hq + 1, D), 7.0, dtype=kw["dtype"], device="cuda")
    lse = torch.full((T, hq), 7.0, device="cuda")
    plan = c.plan(b["seqs"], b["offsets"], T, hq, b["group_offsets"], b["group_prefix"])
    assert c.last_error() == 0
    o = c.attend(plan, q, layer=layer, scale=scale, out=out[:, :hq], lse=lse)
    assert c.last_error() == 0
    scale = D ** -0.5 if scale is None else scale
    ref, ref_lse, mass = R.attend_reference(b, q, scale, layer)
    far = (o.double() - ref).abs() - R.attend_bound(ref, mass, kw["dtype"], max(b["length"]), 6.0)
    assert not bool(torch.isnan(o).any())
    assert bool((far <= 0).all()), (far.max().item(), (far > 0).nonzero()[:8].tolist())
    hidden = ref_lse == -torch.inf
    assert bool((lse[hidden] == -torch.inf).all()) and bool((o[hidden] == 0).all())
    assert bool(((lse.double() - ref_lse)[~hidden].abs() <= 2.0 ** -14 * (1 + ref_lse[~hidden].abs())).all())
    assert bool((out[:, hq:] == 7).all())
    again = c.attend(plan, q, layer=layer, scale=scale)   # the same bits every time
    assert torch.equal(again, o)
    return b


BF, HF = "bfloat16", "float16"
# name: page, layout, type, dim, key heads, query heads, groups, prefixes, own, new
CASES = {
    "one_token": (16, "heads", BF, 128, 1, 1, None, (), [0], [1]),
    "short": (16, "heads", BF, 128, 2, 8, None, (), [0, 1, 14, 15, 16, 17, 62, 63, 64, 65, 127, 128, 129], [1] * 13),
    "short_64": (4, "tokens", HF, 64, 3, 9, None, (), [0, 2, 3, 4, 5, 31, 32, 33, 63, 64, 200], [1] * 11),
    "many_keys": (64, "heads", HF, 128, 1, 16, None, (), [20_000], [1]),
    "many_keys_split": (16, "tokens", BF, 64, 2, 2, None, (), [70_001, 1, 33], [1, 1, 1]),
    "seventeen_rows": (16, "heads", BF, 128, 1, 17, None, (), [0, 5, 127, 128, 300], [1] * 5),
    "many_heads": (32, "heads", HF, 64, 1, 71, None, (), [9, 1000], [2, 3]),
    "rows_over_a_tile": (8, "heads", BF, 128, 2, 6, None, (), [0, 100], [43, 86]),
    "prompt": (16, "heads", BF, 128, 2, 8, None, (), [0, 77], [300, 513]),
    "prompt_64": (64, "tokens", HF, 64, 3, 3, None, (), [1000, 0], [129, 260]),
    "long_prompt": (16, "heads", HF, 128, 1, 4, None, (), [0], [2500]),
    "shared": (16, "heads", BF, 128, 2, 8, [5, 3], (256, 512), [0, 3, 100, 17, 64, 1, 0, 200], [1] * 8),
    "shared_narrow": (16, "heads", BF, 128, 3, 6, [2, 3], (64, 16), [5, 0, 9, 15, 16], [1] * 5),
    "shared_64": (64, "tokens", HF, 64, 4, 4, [40, 30], (1024, 64), [7 * i for i in range(70)], [1 + i % 3 for i in range(70)]),
    "shared_many_rows": (32, "heads", BF, 128, 1, 8, [90], (640,), [i for i in range(90)], [1 + i % 5 for i in range(90)]),
    "shared_and_not": (16, "heads", HF, 128, 2, 4, [3, 2], (48, 0), [4, 4, 4, 70, 70, 8, 300], [1, 2, 0, 1, 3, 1, 2]),
    "group_with_prompt": (16, "heads", BF, 128, 2, 8, [3], (160,), [0, 5, 2], [1, 90, 2]),
    "group_of_one": (16, "heads", BF, 64, 2, 4, [1, 2], (160, 32), [3, 0, 9], [1, 1, 0]),
    "sees_nothing": (16, "heads", BF, 128, 2, 4, None, (), [-3, -1, -20, 5], [3, 4, 25, 1]),
    "sees_nothing_wide": (16, "heads", HF, 64, 1, 8, None, (), [-40, -300, 2], [90, 290, 40]),
    "no_new": (16, "heads", BF, 128, 1, 2, None, (), [0, 30, 40], [0, 2, 0]),
    "drafts": (64, "tokens", HF, 64, 2, 24, [8, 7], (448, 1984), [37 * i for i in range(15)], [i % 9 for i in range(15)]),
}


@pytest.mark.parametrize("name", CASES)
def test_attend(torch, name):
    page, layout, dtype, dim, hk, hq, groups, prefix, own, new = CASES[name]
    run(torch, sum(map(ord, name)), hq=hq, page=page, layout=layout, dtype=getattr(torch, dtype), dim=dim, kv_heads=hk, groups=groups,
        prefix=prefix, own=own, new=new, strided=len(name) % 2 == 1, layers=2, layer=1)


@pytest.mark.parametrize("page", [4, 8, 16, 32, 64])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("dtype,dim", [(BF, 64), (BF, 128), (HF, 64), (HF, 128)])
def test_pages_and_types(torch, page, layout, dtype, dim):
    """Every page size, layout, type and head size, narrow and wide, shared and not."""
    run(torch, page + dim, hq=6, page=page, layout=layout, dtype=getattr(torch, dtype), dim=dim, kv_heads=2, groups=[4, 2],
        prefix=(192, 64), own=[3, 70, 0, 129, 61, 5, 200, 31], new=[1, 2, 6, 1, 1, 0, 100, 3])


@pytest.mark.parametrize("gain,scale", [(20.0, None), (1.0, 4.0), (0.01, None), (30.0, 1.0)])
def test_steep_and_flat_scores(torch, gain, scale):
    """Maxima that grow along the keys by far more than the rescaling's
    threshold, weights of one key, and nearly equal weights."""
    # float64 keeps the same inputs; a weight moves by 2^-23 of the largest score, which
    # steep scores make more than the bound allows, so keys and queries are small whole numbers
    import cache_reference as R
    b = R.make_batch(3, page=16, kv_heads=2, dim=128, dtype=torch.bfloat16, own=[500, 900, 3], new=[40, 1, 2])
    c = b["cache"]
    c.k.copy_(torch.nan_to_num(c.k.float()).clamp(-3, 3).round().to(c.k.dtype))
    q = (torch.randn(b["tokens"], 8, 128, generator=b["gen"], device="cuda")).round().to(c.k.dtype)
    scale = (128 ** -0.5 if scale is None else scale) * gain
    lse = torch.empty(b["tokens"], 8, device="cuda")
    plan = c.plan(b["seqs"], b["offsets"], b["tokens"], 8)
    o = c.attend(plan, q, scale=scale, lse=lse)
    assert c.last_error() == 0
    ref, ref_lse, mass = R.attend_reference(b, q, scale)
    # scores are exact before scaling; scaling and the subtraction round by 2^-23 of the largest
    # score in base 2, up to 160 * scale * 1.45 here
    top = 160 * scale * 1.45
    bound = R.attend_bound(ref, mass, torch.bfloat16, 1000, 6.0) + top * 2.0 ** -21 * mass
    assert bool(((o.double() - ref).abs() <= bound).all())
    assert bool(((lse.double() - ref_lse).abs() <= 2.0 ** -14 * (1 + ref_lse.abs())).all())


def test_large_pool_offsets(torch):
    """A pool whose last pages lie beyond 2^31 elements and 2^32 bytes."""
    import cache_reference as R
    from paper_2602_06502_gb300.cache import PagedCache
    pages = 140_000   # x 16 x 8 x 128 = 2.29e9 elements
    k = torch.empty(1, pages, 8, 16, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    gen = torch.Generator(device="cuda").manual_seed(9)
    ids = [139_999, 131_073, 2, 139_000, 131_071]
    t = torch.zeros(3, 8, dtype=torch.int32, device="cuda")
    t[1, :5] = R.ints(ids)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[torch.tensor(ids, device="cuda")] = 1
    c = PagedCache(k, v, t, R.ints([0, 70, 0]), refs)
    x = torch.randn(70, 24, 128, generator=gen, device="cuda").bfloat16()
    q, kk, vv = x[:, :8], x[:, 8:16], x[:, 16:]
    c.append(R.ints([1]), R.ints([0, 70]), q, kk, vv)
    b = dict(cache=c, rows=[ids], length=[70], place=[1], host_offsets=[0], new=[70], page=16, layout="heads")
    assert torch.equal(R.read_seq(b, c.k, 0), kk) and torch.equal(R.read_seq(b, c.v, 0), vv)
    plan = c.plan(R.ints([1]), R.ints([0, 70]), 70, 8)
    o = c.attend(plan, q.contiguous())
    assert c.last_error() == 0
    ref, _, mass = R.attend_reference(b, q, 128 ** -0.5)
    assert bool(((o.double() - ref).abs() <= R.attend_bound(ref, mass, torch.bfloat16, 70, 6.0)).all())
    c.fork(R.ints([1]), R.ints([0]), R.ints([69]))
    c.compact()
    assert c.last_error() == 0
    b["rows"] = [c.tables[1, :5].tolist()]
    assert sorted(c.tables[1, :5].tolist() + c.tables[0, 4:5].tolist()) == list(range(6))
    assert torch.equal(R.read_seq(b, c.k, 0), kk) and torch.equal(R.read_seq(b, c.v, 0), vv)


def test_other_stream(torch):
    """The calls run on torch's current stream, in its order."""
    import cache_reference as R
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        b = R.make_batch(31, page=16, kv_heads=2, dim=64, dtype=torch.float16, own=[50, 200], new=[1, 40])
        c = b["cache"]
        q = torch.randn(b["tokens"], 4, 64, generator=b["gen"], device="cuda").half()
        o = c.attend(c.plan(b["seqs"], b["offsets"], b["tokens"], 4), q)
        ref, _, mass = R.attend_reference(b, q, 64 ** -0.5)
        ok = ((o.double() - ref).abs() <= R.attend_bound(ref, mass, torch.float16, 240, 6.0)).all()
    s.synchronize()
    assert bool(ok)


def test_refusals(torch):
    import cache_reference as R
    from paper_2602_06502_gb300 import dualmap as D
    b = R.make_batch(4, page=16, kv_heads=2, dim=64, dtype=torch.bfloat16, groups=[3], prefix=(64,), own=[3, 20, 1], new=[2, 1, 0])
    c, T = b["cache"], b["tokens"]
    q = torch.randn(T, 4, 64, generator=b["gen"], device="cuda").bfloat16()
    inv = D.DM_ERR_INVALID_ARG

    def refused(seqs=b["seqs"], offsets=b["offsets"], go=b["group_offsets"], gp=b["group_prefix"]):
        plan = c.plan(seqs, offsets, T, 4, go, gp)
        assert c.last_error() == inv
        out = torch.full_like(q, 5.0)
        c.attend(plan, q, out=out)   # an empty plan
        assert c.last_error() == 0 and bool((out == 5).all())

    refused(seqs=R.ints([0, 1, 77]))
    refused(seqs=R.ints([0, 1, -1]))
    refused(offsets=R.ints([0, 2, 1, 3]))
    refused(offsets=R.ints([0, 1, 2, T + 1]))
    refused(offsets=R.ints([-1, 1, 2, T]))
    refused(gp=R.ints([40]))             # no multiple of a page
    refused(gp=R.ints([-16]))
    refused(gp=R.ints([80]))             # reaches into the new tokens of the first
    refused(go=R.ints([0, 4]))
    refused(go=R.ints([2, 1]))
    at = b["place"][1]
    old = int(c.tables[at, 2])
    c.tables[at, 2] = b["rows"][1][-1]   # the second does not begin with the group's pages
    refused()
    c.tables[at, 2] = old
    plan = c.plan(b["seqs"], b["offsets"], T, 4, b["group_offsets"], b["group_prefix"])
    assert c.last_error() == 0
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(layer=1)):
        with pytest.raises(D.DualMapError):
            c.attend(plan, q, **bad)
    with pytest.raises(ValueError):
        c.attend(plan, q[:, :2])
    with pytest.raises(ValueError):
        c.attend(plan, q.half())
    with pytest.raises(D.DualMapError):
        c.plan(b["seqs"], b["offsets"], T, 5)
    with pytest.raises(ValueError):
        c.plan(b["seqs"], b["offsets"], T, 4, b["group_offsets"])
    # nothing to do
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    c.attend(c.plan(b["seqs"], R.ints([0, 0, 0, 0]), 0, 4), none)
    c.attend(c.plan(R.ints([]), R.ints([0]), 0, 4), none)
    assert c.last_error() == 0


@pytest.mark.parametrize("groups", [0, 700])
def test_many_sequences(torch, groups):
    """More sequences, groups and blocks than the plan keeps in shared memory."""
    import random
    rng = random.Random(groups)
    n = 2600
    sizes = None
    if groups:
        sizes = [rng.randint(2, 4) for _ in range(groups)]
        while sum(sizes) > n:
            sizes.pop()
    own = [rng.randint(0, 70) for _ in range(n)]
    new = [rng.choice([0, 1, 1, 1, 2, 9, 40]) for _ in range(n)]
    run(torch, 50 + groups, hq=2, page=4, layout="heads", dtype=torch.bfloat16, dim=64, kv_heads=1, groups=sizes,
        prefix=[4 * rng.randint(1, 12) for _ in sizes or []], own=own, new=new)


@pytest.mark.parametrize("kv_heads, hq, dim", [(12, 36, 64), (8, 40, 128), (36, 36, 64), (9, 36, 128)])
def test_many_rows_joined(torch, kv_heads, hq, dim):
    """So many rows of shared groups, and of prompts that CTAs share, that several are joined at a time; groups'
    rows that begin anywhere among them, and behind the first 256."""
    new = [1 + i % 3 for i in range(300)] + [0, 250, 61]
    run(torch, 64 + dim + hq, hq=hq, page=16, layout="heads", dtype=torch.bfloat16 if dim == 64 else torch.float16, dim=dim,
        kv_heads=kv_heads, groups=[150, 3, 40, 2], prefix=(320, 96, 1024, 160), own=[i % 41 for i in range(300)] + [5, 700, 3000],
        new=new)


def test_long_prompt_of_many_blocks(torch):
    """A prompt of more row blocks than threads lay out at once."""
    run(torch, 60, hq=64, page=64, layout="tokens", dtype=torch.float16, dim=64, kv_heads=1, own=[0, 3], new=[4500, 1])


def test_one_sm_each(torch):
    """A little wide work beside much narrow work, and the other way round."""
    run(torch, 61, hq=8, page=16, layout="heads", dtype=torch.bfloat16, dim=128, kv_heads=1, own=[9000] * 20 + [3], new=[1] * 20 + [5])
    run(torch, 62, hq=8, page=16, layout="heads", dtype=torch.bfloat16, dim=128, kv_heads=1, own=[7, 2000, 30], new=[1, 600, 1])


def test_layers_of_one_plan_and_graphs(torch):
    """One plan for several layers, captured into a graph and replayed."""
    import cache_reference as R
    b = R.make_batch(70, page=16, kv_heads=2, dim=128, dtype=torch.bfloat16, layers=3, groups=[6], prefix=(320,),
                     own=[5, 40, 0, 17, 33, 100, 600], new=[1, 1, 2, 1, 1, 1, 130])
    c, T = b["cache"], b["tokens"]
    q = torch.randn(T, 8, 128, generator=b["gen"], device="cuda").bfloat16()
    plan = c.plan(b["seqs"], b["offsets"], T, 8, b["group_offsets"], b["group_prefix"])
    outs = [torch.empty_like(q) for _ in range(3)]
    want = [c.attend(plan, q, layer=i) for i in range(3)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        for i in range(3):
            c.attend(plan, q, layer=i, out=outs[i])
    for _ in range(3):
        for o in outs:
            o.zero_()
        g.replay()
    assert c.last_error() == 0
    for i in range(3):
        ref, _, mass = R.attend_reference(b, q, 128 ** -0.5, i)
        assert torch.equal(outs[i], want[i])
        assert bool(((outs[i].double() - ref).abs() <= R.attend_bound(ref, mass, torch.bfloat16, 700, 6.0)).all())


def test_buffer_without_the_plan(torch):
    """attend on a work buffer that holds no plan, or another step's, writes nothing and says so."""
    import cache_reference as R
    from paper_2602_06502_gb300 import dualmap as D
    b = R.make_batch(6, page=16, kv_heads=2, dim=64, dtype=torch.bfloat16, own=[30, 200], new=[1, 40])
    c, T = b["cache"], b["tokens"]
    q = torch.randn(T, 4, 64, generator=b["gen"], device="cuda").bfloat16()
    out = torch.full_like(q, 5.0)
    other = c.plan(b["seqs"], b["offsets"], T + 1, 4)
    for fill in (0, 255):
        plan = c.plan(b["seqs"], b["offsets"], T, 4)
        assert c.last_error() == 0
        plan.keep[-1].fill_(fill)
        c.attend(plan, q, out=out)
        assert c.last_error() == D.DM_ERR_INVALID_ARG and bool((out == 5).all())
    plan = c.plan(b["seqs"], b["offsets"], T, 4)
    held = plan.struct.work
    plan.struct.work = other.struct.work
    assert plan.struct.work_bytes <= other.struct.work_bytes
    c.attend(plan, q, out=out)
    assert c.last_error() == D.DM_ERR_INVALID_ARG and bool((out == 5).all())
    plan.struct.work = held
    c.attend(plan, q, out=out)
    assert c.last_error() == 0 and not bool((out == 5).all())


@pytest.mark.parametrize("new", [[1, 2], [1, 60]])   # few rows, many rows
def test_a_query_that_is_not_finite(torch, new):
    """NaN in one query stays in its own row, and its logarithm says so too."""
    import cache_reference as R
    b = R.make_batch(8, page=16, kv_heads=2, dim=64, dtype=torch.bfloat16, own=[30, 700], new=new)
    c, T = b["cache"], b["tokens"]
    q = torch.randn(T, 4, 64, generator=b["gen"], device="cuda").bfloat16()
    plan = c.plan(b["seqs"], b["offsets"], T, 4)
    lse, clean = torch.empty(T, 4, device="cuda"), torch.empty(T, 4, device="cuda")
    ref = c.attend(plan, q, lse=clean)
    q[T - 1, 3] = float("nan")
    o = c.attend(plan, q, lse=lse)
    bad = torch.zeros(T, 4, dtype=torch.bool, device="cuda")
    bad[T - 1, 3] = True
    assert torch.equal(torch.isnan(lse), bad) and torch.equal(torch.isnan(o).all(-1), bad)
    assert torch.equal(lse[~bad], clean[~bad]) and torch.equal(o[~bad], ref[~bad])
    assert c.last_error() == 0
