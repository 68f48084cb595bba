"""How products and expert layers are used: what the wrappers refuse, errors that
the device finds, captured graphs, streams, far offsets, the instance."""

import numpy as np
import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    lib_ready()
    import torch
    return torch


def ints(torch, x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def layer(torch, seed, experts=6, k=256, m=96, top_k=2, eight=False, dtype=None):
    from paper_2602_06502_gb300 import experts as X
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = dtype or torch.bfloat16
    up = (torch.randn(experts, 2 * m, k, generator=g, device="cuda") * k ** -0.5).to(t)
    down = (torch.randn(experts, k, m, generator=g, device="cuda") * m ** -0.5).to(t)
    make = X.Weights.quantized if eight else X.Weights
    return X.Experts(make(up), make(down), top_k)


def batch(torch, seed, tokens, k=256, experts=6, dtype=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(tokens, k, generator=g, device="cuda").to(dtype or torch.bfloat16)
    return x, torch.randn(tokens, experts, generator=g, device="cuda")


# -- refusals ------------------------------------------------------------------------

def test_weights_refused(torch):
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300 import experts as X
    w = torch.zeros(4, 32, 64, dtype=torch.bfloat16, device="cuda")
    q, s = torch.zeros(4, 32, 64, dtype=torch.int8, device="cuda"), torch.ones(4, 32, device="cuda")
    X.Weights(w), X.Weights(w[0]), X.Weights(q, s), X.Weights(w[:, :, :61]), X.Weights(w[::2])
    for bad in ((w.float(),), (w[0, 0],), (w.cpu(),), (w.transpose(1, 2),), (q,), (w, s), (q, s[:, :31]), (q, s.double()), (q, s.cpu()),
                (q, s.t().contiguous().t()), (w[:0],), (w.clone().requires_grad_(),)):
        with pytest.raises(ValueError):
            X.Weights(*bad)
    with pytest.raises(D.DualMapError):
        X.Weights(torch.zeros(4, 32, 61, dtype=torch.bfloat16, device="cuda"))      # rows that are no multiple of 16 bytes
    with pytest.raises(D.DualMapError):
        X.Weights(torch.zeros(4 * 32 * 64 + 8, dtype=torch.bfloat16, device="cuda")[1:8193].view(4, 32, 64))
    with pytest.raises(ValueError):
        X.Weights(w, status=torch.zeros(1, device="cuda"))


def test_products_refused(torch):
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300 import experts as X
    w = X.Weights(torch.zeros(4, 32, 64, dtype=torch.bfloat16, device="cuda"))
    q = X.Weights(torch.zeros(32, 64, dtype=torch.int8, device="cuda"), torch.ones(32, device="cuda"))
    x, off = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda"), ints(torch, [0, 2, 4, 6, 8])
    assert X.product(x, w, off).shape == (8, 32) and X.product(x, w, off, gated=True).shape == (8, 16)
    assert X.product(x[:0], w, ints(torch, [0] * 5)).shape == (0, 32)
    bad = [(x, w), (x, w, off[:4]), (x, w, off.long()), (x, w, off.cpu()), (x.half(), w, off), (x.float(), w, off), (x[:, :63], w, off),
           (x[0], w, off), (x.t(), w, off), (x.cpu(), w, off), (x, q)]
    for args in bad:
        with pytest.raises(ValueError):
            X.product(*args)
    out = torch.zeros(8, 32, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(out=out[:, :31]), dict(out=out[:7]), dict(out=out.int()), dict(out=out.t()), dict(sources=off.long()), dict(x_scale=torch.ones(8, device="cuda")),
               dict(sources=off[:1].expand(8)), dict(sources=torch.zeros(8, dtype=torch.int32, device="cuda"), per_source=0),
               dict(out=out.expand(2, 8, 32)[0].as_strided((8, 32), (16, 1)))):
        with pytest.raises(ValueError):
            X.product(x, w, off, **kw)
    with pytest.raises(D.DualMapError):
        X.product(torch.zeros(8 * 64 + 8, dtype=torch.bfloat16, device="cuda")[1:513].view(8, 64), w, off)   # begins off 16 bytes
    odd = X.Weights(torch.zeros(4, 31, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        X.product(x, odd, off, gated=True)
    with pytest.raises(ValueError):
        X.product(x.clone().requires_grad_(), w, off)
    with torch.no_grad():
        X.product(x.clone().requires_grad_(), w, off)


def test_choices_linears_and_layers_refused(torch):
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300 import experts as X
    x, logits = batch(torch, 1, 5)
    for k in (0, 7, -1):
        with pytest.raises(D.DualMapError):
            X.choose(logits, k)
    for bad in (logits.double(), logits[0], logits.cpu(), logits.clone().requires_grad_()):
        with pytest.raises(ValueError):
            X.choose(bad, 2)
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(count=ints(torch, [1, 2]))):
        with pytest.raises(ValueError):
            X.quantize(x, **kw)
    for bad in (x.float(), x.t(), x[0], x.cpu(), x.clone().requires_grad_()):
        with pytest.raises(ValueError):
            X.quantize(bad)
    w16 = X.Weights(torch.zeros(32, 256, dtype=torch.bfloat16, device="cuda"))
    w8 = X.Weights.quantized(torch.ones(32, 256, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        X.Linear(w16)(x, eps=1e-6)
    with pytest.raises(ValueError):
        X.Linear(w8)(x.float())
    with pytest.raises(ValueError):
        X.Linear(w8)(x.clone().requires_grad_())
    e = layer(torch, 2)
    with pytest.raises(ValueError):
        X.Linear(e.up)
    for args in ((e.down, e.up, 2), (e.up, e.down, 0), (e.up, e.down, 7), (w16, w16, 1), (e.up, layer(torch, 2, eight=True).down, 2)):
        with pytest.raises(ValueError):
            X.Experts(*args)
    for args, kw in (((x.half(), logits), {}), ((x[:, :255], logits), {}), ((x, logits[:4]), {}), ((x, logits[:, :5]), {}),
                     ((x, logits), dict(residual=x.float())), ((x, logits), dict(residual=x[:4])), ((x, logits), dict(out=x[:4])),
                     ((x, logits.clone().requires_grad_()), {})):
        with pytest.raises(ValueError):
            e(*args, **kw)


# -- errors that the device finds --------------------------------------------------------

@pytest.mark.parametrize("rows", [12, 700])
def test_offsets_and_sources_out_of_range(torch, rows):
    """Recorded; the products after do nothing until the error has been read."""
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300 import experts as X
    g = torch.Generator(device="cuda").manual_seed(3)
    w = X.Weights((torch.randn(3, 40, 64, generator=g, device="cuda")).bfloat16())
    x = torch.randn(rows, 64, generator=g, device="cuda").bfloat16()
    good = ints(torch, [0, 5, 5, rows])
    want = X.product(x, w, good)
    for bad in ([0, 5, 4, rows], [-1, 0, 5, rows], [0, 5, 5, rows + 1], [0, 1 << 30, 5, rows], [5, 0, 0, 0]):
        X.product(x, w, ints(torch, bad))
        out = torch.full((rows, 40), 7.0, dtype=torch.bfloat16, device="cuda")
        X.product(x, w, good, out=out)
        assert (out == 7).all()
        assert w.last_error() == D.DM_ERR_INVALID_ARG and w.last_error() == D.DM_OK
        assert torch.equal(X.product(x, w, good), want)
    for bad in (-1, rows, 1 << 30):
        sources = torch.arange(rows, device="cuda", dtype=torch.int32)
        sources[rows // 2] = bad
        X.product(x, w, good, sources=sources)
        assert w.last_error() == D.DM_ERR_INVALID_ARG
    sources = torch.arange(rows, device="cuda", dtype=torch.int32)
    assert torch.equal(X.product(x, w, good, sources=sources), want) and w.last_error() == D.DM_OK


def test_weights_that_share_a_status(torch):
    from paper_2602_06502_gb300 import dualmap as D
    from paper_2602_06502_gb300 import experts as X
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    w = torch.ones(2, 16, 32, dtype=torch.bfloat16, device="cuda")
    a, b = X.Weights(w, status=status), X.Weights.quantized(w, status=status)
    x = torch.ones(4, 32, dtype=torch.bfloat16, device="cuda")
    X.product(x, a, ints(torch, [0, 9, 4]))
    out = torch.full((4, 16), 7.0, dtype=torch.bfloat16, device="cuda")
    q, s = X.quantize(x)
    X.product(q, b, ints(torch, [0, 2, 4]), x_scale=s, out=out)
    assert (out == 7).all()
    assert X.last_error(status) == D.DM_ERR_INVALID_ARG and b.last_error() == D.DM_OK


# -- the same inputs, the same outputs ---------------------------------------------------

@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens", [3, 40, 300])
def test_layers_repeat(torch, tokens, eight):
    e = layer(torch, 4, eight=eight)
    x, logits = batch(torch, 5, tokens)
    want = e(x, logits)
    for _ in range(3):
        assert torch.equal(e(x, logits), want)
    out = x.clone()
    assert e(x, logits, residual=out, out=out) is out
    assert torch.equal(out, e(x, logits, residual=x)) and e.last_error() == 0


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens", [4, 200])
def test_captured_and_replayed(torch, tokens, eight):
    """Two graphs of one layer, replayed in turn on new inputs, beside eager calls."""
    e = layer(torch, 6, eight=eight)
    graphs = []
    for seed in (7, 8):
        x, logits = batch(torch, seed, tokens)
        e(x, logits, residual=x)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = e(x, logits, residual=x)
        graphs.append((g, x, logits, y))
    for seed in range(20, 26):
        for i, (g, x, logits, y) in enumerate(graphs):
            nx, nl = batch(torch, seed + 100 * i, tokens)
            x.copy_(nx)
            logits.copy_(nl)
            g.replay()
            want = e(nx, nl, residual=nx)
            assert torch.equal(y, want)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]   # and at once
    for _ in range(20):
        for s, (g, *_) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for g, x, logits, y in graphs:
        assert torch.equal(y, e(x, logits, residual=x))
    assert e.last_error() == 0


def test_projections_on_two_streams(torch):
    from paper_2602_06502_gb300 import experts as X
    g = torch.Generator(device="cuda").manual_seed(9)
    lin = X.Linear(X.Weights.quantized(torch.randn(512, 1024, generator=g, device="cuda").bfloat16()))
    xs = [torch.randn(n, 1024, generator=g, device="cuda").bfloat16() for n in (5, 100, 400)]
    want = [lin(x, eps=1e-6) for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for _ in range(10):
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                got.append(lin(x, eps=1e-6))
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 3])


def test_weights_dropped_while_another_stream_uses_them(torch):
    from test_gpu_cache_streams import given_out_again
    from paper_2602_06502_gb300 import experts as X
    g = torch.Generator(device="cuda").manual_seed(10)
    real = torch.randn(256, 512, generator=g, device="cuda").bfloat16()
    x = torch.randn(3, 512, generator=g, device="cuda").bfloat16()
    want = X.Linear(X.Weights.quantized(real))(x)
    w = X.Weights.quantized(real)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)   # some 0.2 s
        y = X.Linear(w)(x)
    at, size = w.w.data_ptr(), w.w.numel()
    del w
    assert not given_out_again(torch, size, at)
    assert not side.query()   # the product had not run by then
    side.synchronize()
    assert torch.equal(y, want)


# -- far offsets ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bfloat16", "int8"])
@pytest.mark.parametrize("rows", [3, 600])
def test_offsets_past_32_bits(torch, rows, dtype):
    """The last of 40 experts begins behind 2^32 bytes; x and y have rows far apart."""
    import experts_reference as R
    from paper_2602_06502_gb300 import experts as X
    t, g = getattr(torch, dtype), torch.Generator(device="cuda").manual_seed(11)
    E, n, k = 40, 96, 128
    far = 1 << (27 if t is torch.int8 else 26)          # elements from an expert to the next: 2^27 bytes
    w = torch.empty(E * far, dtype=t, device="cuda").as_strided((E, n, k), (far, k, 1))
    w[E - 1] = R.whole(g, (n, k), 4).to(t)
    step = (1 << 32) // rows // 8 * 8                   # of x, elements
    x = torch.empty(rows * step, dtype=t, device="cuda").as_strided((rows, k), (step, 1))
    x.copy_(R.whole(g, (rows, k), 4).to(t))
    y = torch.zeros(rows * step, dtype=torch.bfloat16, device="cuda").as_strided((rows, n), (step, 1))
    eight = t is torch.int8
    w = X.Weights(w, torch.ones(E, n, device="cuda") if eight else None)
    if eight:
        x = x if step % 16 == 0 else x.clone()
    X.product(x, w, ints(torch, [0] * E + [rows]), x_scale=torch.ones(rows, device="cuda") if eight else None, out=y)
    want = x.double() @ w.w[E - 1].double().T
    assert torch.equal(y.double(), want.bfloat16().double()) and w.last_error() == 0   # whole numbers: nothing but the rounding


# -- the instance -----------------------------------------------------------------------------

def node(**kw):
    from paper_2602_06502_gb300.instance import Instance
    return Instance(pages=600, max_tokens=700, max_seqs=40, layers=2, q_heads=8, kv_heads=2, head_dim=64, vocab=500, seed=3, **kw)


@pytest.mark.parametrize("kw", [dict(experts=4, top_k=4, expert_width=320), dict(eight_bits=True), dict(experts=3, top_k=3, eight_bits=True)],
                         ids=str)
def test_instance(torch, kw):
    """Sequences that run together and each alone, fed the same tokens.  Each token goes to all experts: which ones it
    chooses jumps where two scores are close, and sums in another order move them."""
    rng = np.random.default_rng(4)
    together, alone = node(**kw), node(**kw)
    head = rng.integers(0, 500, size=192).astype(np.uint32)
    first = [np.concatenate([head, rng.integers(0, 500, size=9).astype(np.uint32)])]
    together.admit(first)
    prompts = [np.concatenate([head, rng.integers(0, 500, size=n).astype(np.uint32)]) for n in (7, 1, 40)]
    prompts.append(rng.integers(0, 500, size=33).astype(np.uint32))
    steps = 4
    seqs, logits = together.admit(prompts, room=steps)
    assert together.reused == 3 * 192
    start = [together.tokens[s] for s in seqs]
    feed = rng.integers(0, 500, size=(steps, len(seqs))).astype(np.uint32)
    got = [logits] + [together._forward(seqs, [t[None] for t in row]) for row in feed]
    for k, tokens in enumerate(start):
        own, ref = alone.admit([tokens], room=steps)
        refs = [ref] + [alone._forward(own, [row[k][None]]) for row in feed]
        for x, y in zip(got, refs):
            # Both round activations at the same places; sums in another order move one by a unit in its last place (2^-8)
            # here and there over two layers.  In 8 bits that can move any value by a step: a row's steps are 2^-7 of its
            # largest, some four times its root mean square, so the two differ by up to sqrt(2 / 12) 2^-5 = 1.3% for each of
            # eight products, at random 3.6%.
            far = (x[k].float() - y[0].float()).norm() / y[0].float().norm()
            assert float(far) < (2.0 ** -4 if kw.get("eight_bits") else 2.0 ** -5), (k, float(far))
        alone.drop(own)
    assert together.cache.last_error() == 0


def test_instance_against_its_formulas(torch):
    """One prompt through a layer with experts, in 32 bits."""
    n = node(experts=5, top_k=2, expert_width=96)
    tokens = np.arange(1, 60, dtype=np.uint32)
    seqs, logits = n.admit([tokens])
    x = n.embedding[torch.from_numpy(tokens.astype(np.int64)).cuda()].float()
    norm = lambda v: v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6)   # noqa: E731
    T, hq, hk, d = len(tokens), 8, 2, 64
    for i in range(2):
        qkv = (norm(x) @ n.qkv[i].float()).view(T, hq + 2 * hk, d)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        qw, kw = n.norms[i].float()

        def turn(a, w):
            a = norm(a) * w
            lo, hi = a.chunk(2, -1)
            c, s = n.cos[:T, None], n.sin[:T, None]
            return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)

        q, k = turn(q, qw), turn(k, kw).repeat_interleave(4, 1)
        score = torch.einsum("thd,phd->htp", q, k) * d ** -0.5
        score = score.masked_fill(torch.ones(T, T, device="cuda", dtype=torch.bool).triu(1), -torch.inf)
        o = torch.einsum("htp,phd->thd", score.softmax(-1), v.repeat_interleave(4, 1)).reshape(T, hq * d)
        x = x + o @ n.out[i].float()
        h = norm(x)
        up, down = n.experts[i].up.w.float(), n.experts[i].down.w.float()
        w, ids = (h @ n.gates[i].float()).topk(2, -1)
        w = w.softmax(-1)
        every = torch.einsum("tk,enk->ten", h, up)
        act = torch.nn.functional.silu(every[..., :96]) * every[..., 96:]
        y = torch.einsum("tem,ekm->tek", act, down)
        x = x + (y.gather(1, ids[..., None].expand(-1, -1, y.shape[-1])) * w[..., None]).sum(1)
    want = x[-1] @ n.embedding.float().T
    # bfloat16 activations (2^-8 a rounding) through two layers of about eight roundings each, at random
    far = (logits[0].float() - want).norm() / want.norm()
    assert float(far) < 2.0 ** -4, float(far)


@pytest.mark.parametrize("model", [dict(experts=4, top_k=2), dict(experts=8, top_k=2, eight_bits=True)], ids=str)
def test_instance_behind_the_router(torch, model):
    from paper_2602_06502_gb300.instance import run
    rows = list(run("tiny", instance=1, batches=2, decode=3, overrides=dict(n_requests=400, batch=200), pages=4096, **model))
    assert len(rows) == 2 and rows[1]["requests"] > 0
    assert rows[1]["reused_tokens"] + rows[1]["computed_tokens"] == rows[1]["prompt_tokens"] + 3 * rows[1]["requests"]
