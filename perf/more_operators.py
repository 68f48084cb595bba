"""The operators of an instance's projections and expert layers, their sizes and their plain forms.

An instance serves the tokens that the router sends it: a token's row goes
through the projections around attention and, in a layer of experts, through
the few experts that a gate chooses for it.  Measured here are the product
with 8-bit weights (a scale for each token and each output channel), the
quantising of its rows, the choice of experts, the products grouped by expert
over rows of ragged counts, and the whole expert layer.

Every case is a dict of plain values.  The experts' popularity and the ragged
counts follow from the case alone (its `lens` seeds them); values follow from
prepare()'s seed.
"""

import math
import random

import torch

own = False
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# weights: "16" are of the rows' type, "8" are int8 with a scale a channel.
# pad: elements between the rows of x and of the weights beyond their width.
QUANTIZE = dict(kind="quantize", dtype="bf16", rows=61, k=1024, norm=True, pad=0)
LINEAR = dict(kind="linear", dtype="bf16", rows=4, k=1024, n=1536, norm=True, pad=0)
ROUTE = dict(kind="route", dtype="f32", rows=4, experts=8, top_k=2, renormalize=True, masked=0.0, lens=1)
GROUPED = dict(kind="grouped", dtype="bf16", weights="16", rows=16, experts=8, k=1024, n=1024, gated=False, pad=0, spare=0, lens=1)
LAYER = dict(kind="layer", dtype="bf16", weights="16", rows=4, experts=8, top_k=2, k=1024, n=2048, renormalize=True,
             masked=0.0, pad=0, lens=1)


def listed():
    return [
        # A decode step's tokens are quantised, a norm over their width on the way: latency.
        dict(QUANTIZE, name="quantize_tokens"),
        # Prompts' tokens before a projection: bandwidth.
        dict(QUANTIZE, name="quantize_prompts", dtype="f16", rows=8191, k=4096, norm=False),
        # The projection to queries, keys and values of four decoded tokens, at the instance's own width: latency.
        dict(LINEAR, name="linear_few"),
        # The same of a decode step of 128 sequences with 32 and 2 x 8 heads of 128: the weights' bytes.
        dict(LINEAR, name="linear_decode", rows=128, k=4096, n=6144),
        # The same of prompts: tensor work.
        dict(LINEAR, name="linear_prompts", dtype="f16", rows=8191, k=4096, n=6144),
        # Four decoded tokens choose two of eight experts: latency.
        dict(ROUTE, name="route_few"),
        # Prompts choose eight of 128, where some experts are switched off and some rows are padding.
        dict(ROUTE, name="route_many", dtype="bf16", rows=8192, experts=128, top_k=8, masked=0.1, renormalize=False, lens=2),
        # The first product of an expert layer for a few tokens, the gate's half multiplied in: the weights' bytes.
        dict(GROUPED, name="grouped_few", n=2048, gated=True, lens=3),
        # Prompts' rows over 64 experts, some with thousands and some with none, an odd width: tensor work.
        dict(GROUPED, name="grouped_ragged", dtype="f16", rows=16001, experts=64, k=2048, n=1415, spare=100, lens=4),
        # An expert layer of four decoded tokens: launches.
        dict(LAYER, name="layer_few", lens=5),
        # An expert layer of a decode step in 8 bits: nearly all experts are read, for few rows each.
        dict(LAYER, name="layer_decode", weights="8", rows=128, experts=64, top_k=8, k=2048, n=1024, lens=6),
        # An expert layer of prompts: tensor work.
        dict(LAYER, name="layer_prompts", rows=4096, experts=32, top_k=4, k=4096, n=1536, lens=7),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """(width, pad): a multiple of 16, or any number in rows that are padded to 16 bytes and more."""
    k = _log_between(rng, lo, hi)
    if rng.random() < 0.7:
        return -(-k // 16) * 16, 0
    return k, -k % 16 + 16 * rng.randint(0, 2)


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "route", "grouped", "grouped", "layer", "layer"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "f16"]), rows=_log_between(rng, 1, 6000))
    if kind == "quantize":
        k, pad = _width(rng, 16, 8192)
        return dict(c, k=k, pad=pad, norm=rng.choice([False, True]))
    if kind == "linear":
        k, pad = _width(rng, 48, 6000)
        return dict(c, k=k, pad=pad, n=_log_between(rng, 16, 8000), norm=rng.choice([False, True]))
    experts = _log_between(rng, 2, 160)
    c.update(experts=experts, lens=rng.randrange(1 << 30))
    if kind != "grouped":
        c.update(top_k=rng.randint(1, min(8, experts)), renormalize=rng.choice([False, True]),
                 masked=rng.choice([0.0, 0.0, 0.2]))
    if kind == "route":
        return dict(c, dtype=rng.choice(["bf16", "f16", "f32"]))
    k, pad = _width(rng, 64, 3000)
    c.update(k=k, pad=pad, weights=rng.choice(["16", "8"]))
    if kind == "grouped":
        return dict(c, n=_log_between(rng, 16, 2500), gated=rng.choice([False, True]), spare=rng.choice([0, 0, 7]))
    c["n"] = -(-_log_between(rng, 32, 2000) // 16) * 16
    c["experts"] = min(experts, max(2, 150_000_000 // (k * c["n"])))   # weights of a gigabyte
    c["top_k"] = min(c["top_k"], c["experts"])
    return dict(c, rows=min(c["rows"], 12_000 // c["top_k"]))


# -- inputs -------------------------------------------------------------------------

def _dev():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _padded(gen, rows, width, pad, dtype, dev):
    """Rows of normal values, `pad` elements between them that nobody may read as theirs."""
    if not pad:
        return torch.randn(rows, width, generator=gen, device=dev, dtype=dtype)
    x = torch.full((rows, width + pad), float("nan"), device=dev, dtype=dtype)
    x[:, :width] = torch.randn(rows, width, generator=gen, device=dev, dtype=dtype)
    return x[:, :width]


def _counts(c):
    """Rows of each expert: few experts take most, some none."""
    rng = random.Random(c["lens"])
    order = list(range(c["experts"]))
    rng.shuffle(order)
    there = order[:max(1, int(0.85 * len(order)))]
    counts = [0] * c["experts"]
    for e in rng.choices(there, [1 / (i + 3) for i in range(len(there))], k=c["rows"]):
        counts[e] += 1
    return counts


def _logits(c, gen, dev):
    """A gate's scores: experts of unlike popularity; minus infinity where an expert is off or a row is padding."""
    rng = random.Random(c["lens"])
    liking = torch.tensor([rng.gauss(0, 0.7) for _ in range(c["experts"])], device=dev)
    x = torch.randn(c["rows"], c["experts"], generator=gen, device=dev) + liking
    if c["masked"]:
        off = [e for e in range(c["experts"]) if rng.random() < c["masked"]]
        if off:
            x[:, torch.tensor(off, device=dev)] = -torch.inf
        x[torch.rand(c["rows"], generator=gen, device=dev) < 0.02] = -torch.inf
    return x


def _weights(c, gen, experts, n, k, dev):
    """[experts, n, k] in the rows' type, or int8 and their scales [experts, n]."""
    if c["weights"] == "16":
        return (_padded(gen, experts * n, k, c["pad"], TYPES[c["dtype"]], dev).unflatten(0, (experts, n)).mul_(k ** -0.5), None)
    q = torch.empty(experts, n, k + c["pad"], dtype=torch.int8, device=dev)
    scale = torch.empty(experts, n, device=dev)
    for e in range(experts):
        w = torch.randn(n, k, generator=gen, device=dev) * k ** -0.5
        scale[e] = w.abs().amax(-1) / 127
        q[e, :, :k] = (w / scale[e][:, None]).round().to(torch.int8)
    return q[..., :k], scale


def _inputs(c, seed):
    dev = _dev()
    gen = torch.Generator(device=dev).manual_seed(seed)
    s = dict(case=c)
    if c["kind"] == "route":
        s["logits"] = _logits(c, gen, dev).to(TYPES[c["dtype"]])
        return s
    if c["kind"] in ("quantize", "linear", "layer"):
        s["x"] = _padded(gen, c["rows"], c["k"], c["pad"], TYPES[c["dtype"]], dev)
        s["x"] *= 1 + torch.rand(c["rows"], 1, generator=gen, device=dev).to(s["x"].dtype)   # tokens of unlike size
    if c["kind"] == "linear":
        w, scale = _weights(dict(c, weights="8"), gen, 1, c["n"], c["k"], dev)
        s["w"], s["w_scale"] = w[0], scale[0]
    elif c["kind"] == "grouped":
        counts = _counts(c)
        s["offsets_host"] = [0]
        for x in counts:
            s["offsets_host"].append(s["offsets_host"][-1] + x)
        s["offsets"] = torch.tensor(s["offsets_host"], dtype=torch.int32, device=dev)
        rows = c["rows"] + c["spare"]   # the spare rows are nobody's
        x = _padded(gen, rows, c["k"], c["pad"], TYPES[c["dtype"]], dev)
        s["x_scale"] = None
        if c["weights"] == "8":
            s["x_scale"] = x.float().abs().amax(-1) / 127
            q = torch.zeros(rows, c["k"] + c["pad"], dtype=torch.int8, device=dev)
            q[:, :c["k"]] = (x.float() / s["x_scale"][:, None]).round().to(torch.int8)
            x = q[:, :c["k"]]
        s["x"] = x
        s["w"], s["w_scale"] = _weights(c, gen, c["experts"], c["n"] * (2 if c["gated"] else 1), c["k"], dev)
        s["y"] = torch.zeros(rows, c["n"], dtype=TYPES[c["dtype"]], device=dev)
    elif c["kind"] == "layer":
        s["logits"] = _logits(c, gen, dev)
        s["up"] = _weights(c, gen, c["experts"], 2 * c["n"], c["k"], dev)
        s["down"] = _weights(dict(c, pad=0), gen, c["experts"], c["k"], c["n"], dev)
        s["residual"] = torch.randn(c["rows"], c["k"], generator=gen, device=dev, dtype=TYPES[c["dtype"]])
    return s


def prepare(case, seed):
    c, s = case, _inputs(case, seed)
    if own:   # the weights as a program keeps them
        from paper_2602_06502_gb300 import experts as X
        if c["kind"] == "linear":
            s["linear"] = X.Linear(X.Weights(s["w"], s["w_scale"]))
        elif c["kind"] == "grouped":
            s["weights"] = X.Weights(s["w"], s["w_scale"])
        elif c["kind"] == "layer":
            s["layer"] = X.Experts(X.Weights(*s["up"]), X.Weights(*s["down"]), c["top_k"], renormalize=c["renormalize"])
    return s


# -- the plain forms ----------------------------------------------------------------

def _plain_quantize(x, norm):
    """q = x / scale rounded to even, |q| <= 127; a norm over the row is a factor of the scale alone."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    q = torch.where(top > 0, (x.double() * 127 / top.double()).round(), 0.0)   # values next to a border
    scale = top / 127
    if norm:
        scale = scale * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return q.to(torch.int8), scale[:, 0]


def _plain_product(x, x_scale, w, w_scale):
    """Rows times one expert's weights, in 32 bits."""
    y = x.float() @ w.float().T
    return y if w_scale is None else y * x_scale[:, None] * w_scale


def _plain_gate(y):
    g, u = y.chunk(2, -1)
    return g / (1 + torch.exp(-g)) * u


def _plain_route(logits, top_k, renormalize):
    x = logits.float()
    tokens, experts = x.shape
    got, ids = torch.sort(x, dim=-1, descending=True, stable=True)
    got, ids = got[:, :top_k], ids[:, :top_k]
    base = got[:, :1].clamp(min=torch.finfo(torch.float32).min)
    weights = torch.exp(got - base)
    total = (weights if renormalize else torch.exp(x - base)).sum(-1, keepdim=True)
    weights = torch.where(total > 0, weights / total, 0.0)
    there = got > -torch.inf
    ids = torch.where(there, ids, -1)
    flat = torch.where(there, ids, experts).flatten()
    order = torch.argsort(flat, stable=True)
    offsets = torch.searchsorted(flat[order], torch.arange(experts + 1, device=x.device))
    at = torch.arange(flat.numel(), device=x.device)
    sources = torch.where(at < offsets[-1], order, -1)
    slots = torch.empty_like(order)
    slots[order] = at
    slots = torch.where(flat < experts, slots, -1).view(tokens, top_k)
    return dict(ids=ids.int(), weights=weights, offsets=offsets.int(), slots=slots.int(), sources=sources.int())


def _plain_layer(s):
    c = s["case"]
    t = s["x"].dtype
    r = _plain_route(s["logits"], c["top_k"], c["renormalize"])
    x, x_scale = (s["x"], None) if c["weights"] == "16" else _plain_quantize(s["x"], False)
    offsets, sources = r["offsets"].tolist(), r["sources"].long()
    y = s["residual"].float()
    parts = torch.zeros(sources.numel(), c["k"], device=y.device)
    for e in range(c["experts"]):
        a, b = offsets[e], offsets[e + 1]
        if a == b:
            continue
        token = sources[a:b] // c["top_k"]
        up, down = [(w[e], None if scale is None else scale[e]) for w, scale in (s["up"], s["down"])]
        h = _plain_gate(_plain_product(x[token], None if x_scale is None else x_scale[token], *up))
        h_scale = None
        if c["weights"] == "8":
            h, h_scale = _plain_quantize(h.to(t), False)   # what the rows' type holds is quantised
        parts[sources[a:b]] = _plain_product(h, h_scale, *down)
    parts = parts.view(c["rows"], c["top_k"], c["k"])
    return (y + (parts * r["weights"][..., None]).sum(1)).to(t)


def run(s):
    c = s["case"]
    if own:
        from paper_2602_06502_gb300 import experts as X
    if c["kind"] == "quantize":
        q, scale = X.quantize(s["x"], eps=EPS if c["norm"] else None) if own else _plain_quantize(s["x"], c["norm"])
        return {"q": q, "scale": scale}
    if c["kind"] == "linear":
        if own:
            return {"y": s["linear"](s["x"], eps=EPS if c["norm"] else None)}
        q, scale = _plain_quantize(s["x"], c["norm"])
        return {"y": _plain_product(q, scale, s["w"], s["w_scale"]).to(s["x"].dtype)}
    if c["kind"] == "route":
        if not own:
            return _plain_route(s["logits"], c["top_k"], c["renormalize"])
        r = X.choose(s["logits"], c["top_k"], renormalize=c["renormalize"])
        return dict(ids=r.ids, weights=r.weights, offsets=r.offsets, slots=r.slots, sources=r.sources)
    if c["kind"] == "grouped":
        if own:
            return {"y": X.product(s["x"], s["weights"], s["offsets"], x_scale=s["x_scale"], gated=c["gated"], out=s["y"])}
        for e, (a, b) in enumerate(zip(s["offsets_host"], s["offsets_host"][1:])):
            if a < b:
                y = _plain_product(s["x"][a:b], None if s["x_scale"] is None else s["x_scale"][a:b], s["w"][e],
                                   None if s["w_scale"] is None else s["w_scale"][e])
                s["y"][a:b] = (_plain_gate(y) if c["gated"] else y).to(s["y"].dtype)
        return {"y": s["y"]}
    return {"y": s["layer"](s["x"], s["logits"], residual=s["residual"]) if own else _plain_layer(s)}


# -- what a pass cannot do without --------------------------------------------------------

def work(case):
    c = case
    rows, size = c["rows"], 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "quantize":
        return {"bytes": rows * (c["k"] * (size + 1) + 4), "flops": rows * c["k"] * (5 if c["norm"] else 3)}
    if c["kind"] == "linear":
        return {"bytes": rows * (c["k"] + c["n"]) * size + c["n"] * (c["k"] + 4), "flops": 2 * rows * c["n"] * c["k"]}
    if c["kind"] == "route":
        slots = rows * c["top_k"]   # id, weight, slot and source of each
        return {"bytes": rows * c["experts"] * size + slots * 16 + (c["experts"] + 1) * 4, "flops": rows * c["experts"] * 3}
    if c["kind"] == "grouped":
        wide = c["n"] * (2 if c["gated"] else 1)
        each, more = (size, 0) if c["weights"] == "16" else (1, 4)
        active = sum(x > 0 for x in _counts(c))
        return {"bytes": rows * (c["k"] * each + more + c["n"] * size) + active * wide * (c["k"] * each + more),
                "flops": 2 * rows * wide * c["k"]}
    slots = rows * c["top_k"]
    each = size if c["weights"] == "16" else 1
    active = c["experts"] * (1 - (1 - c["top_k"] / c["experts"]) ** rows)   # expected, were all alike
    return {"bytes": int(active * 3 * c["n"] * c["k"] * each) + rows * (3 * c["k"] * size + c["experts"] * 4),
            "flops": 6 * slots * c["n"] * c["k"]}


# -- in 64 bits --------------------------------------------------------------------------

def _exact_quantize(x, norm):
    """Row by row of its definition: the nearest of the 255 steps, even ones at ties."""
    x = x.double()
    top = x.abs().max(-1).values
    step = torch.where(top > 0, top, 1.0)
    q = torch.round(127.0 * x / step[:, None])
    scale = top / 127.0
    if norm:
        scale = scale / torch.sqrt((x ** 2).sum(-1) / x.shape[-1] + EPS)
    return q, scale


def _exact_choice(logits, top_k, renormalize):
    """(ids, weights): the best that is left, one after another; weights exp(score - log of the sum)."""
    x = logits.double()
    left, ids = x.clone(), []
    at = torch.arange(x.shape[1], device=x.device)
    for _ in range(top_k):
        best = left.max(-1, keepdim=True).values
        first = torch.where((left == best) & (best > -torch.inf), at, x.shape[1]).min(-1).values
        ids.append(torch.where(first < x.shape[1], first, -1))
        left = left.masked_fill(at == first[:, None], -torch.inf)
    ids = torch.stack(ids, 1)
    score = torch.where(ids >= 0, x.gather(1, ids.clamp(min=0)), -torch.inf)
    total = torch.logsumexp(score if renormalize else x, -1, keepdim=True)
    return ids, torch.where(ids >= 0, torch.exp(score - total), 0.0)


def _exact_rows(x, w, scale):
    y = torch.matmul(w.double(), x.double().T).T
    return y if scale is None else y * scale.double()


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["kind"] == "quantize":
        q, scale = _exact_quantize(s["x"], c["norm"])
        return {"q": q.to(torch.int8), "scale": scale}
    if c["kind"] == "linear":
        q, scale = _exact_quantize(s["x"], c["norm"])
        return {"y": _exact_rows(q, s["w"], s["w_scale"]) * scale[:, None]}
    if c["kind"] == "route":
        ids, weights = _exact_choice(s["logits"], c["top_k"], c["renormalize"])
        return dict(ids=ids.int(), weights=weights, offsets=None, slots=None, sources=None)
    if c["kind"] == "grouped":
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device=s["y"].device)
        for e, (a, b) in enumerate(zip(s["offsets_host"], s["offsets_host"][1:])):
            if a == b:
                continue
            z = _exact_rows(s["x"][a:b], s["w"][e], None if s["w_scale"] is None else s["w_scale"][e])
            if s["x_scale"] is not None:
                z = z * s["x_scale"][a:b, None].double()
            y[a:b] = z[:, :c["n"]] * torch.sigmoid(z[:, :c["n"]]) * z[:, c["n"]:] if c["gated"] else z
        return {"y": y}
    ids, weights = _exact_choice(s["logits"], c["top_k"], c["renormalize"])
    y = s["residual"].double()
    eight = c["weights"] == "8"
    x, x_scale = _exact_quantize(s["x"], False) if eight else (s["x"], None)
    for e in range(c["experts"]):
        token, place = torch.nonzero(ids == e, as_tuple=True)
        if not token.numel():
            continue
        z = _exact_rows(x[token], s["up"][0][e], s["up"][1][e] if eight else None)
        z = z * x_scale[token, None] if eight else z
        h = z[:, :c["n"]] * torch.sigmoid(z[:, :c["n"]]) * z[:, c["n"]:]
        if eight:
            h, h_scale = _exact_quantize(h.to(s["x"].dtype), False)
        z = _exact_rows(h, s["down"][0][e], s["down"][1][e] if eight else None)
        y.index_add_(0, token, (z * h_scale[:, None] if eight else z) * weights[token, place, None])
    return {"y": y}
