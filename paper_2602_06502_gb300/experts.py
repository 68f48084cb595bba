"""An instance's projections and expert layers over torch tensors: products with
16-bit weights or with 8-bit ones, of one set of weights or grouped by expert,
the quantising of rows, the choice of experts, and the layer made of them
(dm_quantize, dm_choose_experts, dm_product and dm_experts of include/dualmap.h).

Only marshalling: it checks shapes and types, allocates outputs and work
buffers on the device, and enqueues the C calls on torch's current stream of
the inputs' device.  A call's work buffer is its own, so calls on one set of
weights may overlap.  While an error stands (last_error) products do nothing, and
a new output is whatever memory held.  The calls serve: they give no gradients,
so with grad mode on they refuse tensors that want one.

A matrix's last dimension is contiguous and its rows begin on 16 bytes: a width
that is no multiple of 16 bytes lies in wider rows (x = buffer[:, :k]).
"""

import ctypes as C

import torch

from . import dualmap as D

TYPES = {torch.bfloat16: D.DM_BF16, torch.float16: D.DM_F16}
SCORES = {torch.bfloat16: D.DM_BF16, torch.float16: D.DM_F16, torch.float32: D.DM_F32}
_MOST = (1 << 31) - 1   # of rows and of a row's elements; ctypes would cut larger numbers off
_sizes = {}   # of work buffers, by device and shape


def _size(name, device, key, *args):
    """What the C call `name` answers for a work buffer on `device`; key: what it depends on."""
    at = (name, device, key)
    size = _sizes.get(at)
    if size is None:
        with torch.cuda.device(device):   # it depends on the device's SMs
            size = getattr(D.lib(), name)(*args)
        if not size:
            raise D.DualMapError(D.DM_ERR_INVALID_ARG, name)
        if len(_sizes) > 4096:
            _sizes.clear()
        _sizes[at] = size
    return size


def _call(name, device, *args):
    """Enqueues a C call on torch's current stream of the device."""
    if torch._C._cuda_getDevice() != device.index:
        with torch.cuda.device(device):
            return _call(name, device, *args)
    rc = getattr(D.lib(), name)(*args, torch._C._cuda_getCurrentRawStream(device.index))
    if rc:
        raise D.DualMapError(rc, name)


# These run once per call of a decode step, so they ask each tensor for little.

def _refuse_grad(name, x):
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires grad, and this call gives no gradients: use torch.no_grad() or detach it")


def _matrix(name, x, dtypes, device, n=None, k=None):
    """(address, distance of rows) of a matrix [n, k] (None: of any number)."""
    if x.dim() != 2 or x.dtype not in dtypes or x.device != device or device.type != "cuda":
        raise ValueError(f"{name}: a matrix on a CUDA device, with the other tensors, of one of the types {list(dtypes)}")
    rows, width = x.shape
    if (n is not None and rows != n) or (k is not None and width != k):
        raise ValueError(f"{name}: shape {(rows, width)}, wanted {(n, k)}")
    if rows > _MOST or width > _MOST:
        raise ValueError(f"{name}: at most 2^31 - 1 rows and as many columns")
    row, one = x.stride()
    if one != 1 and width > 1:
        raise ValueError(f"{name}: its last dimension is contiguous")
    if x.requires_grad:
        _refuse_grad(name, x)
    if rows <= 1:   # the stride of a dimension of one element says nothing
        row = 0
    elif row < width:
        raise ValueError(f"{name}: its rows lie one after another")
    return x.data_ptr(), row


def _vector(name, x, dtype, device, n):
    if x.dtype is not dtype or x.dim() != 1 or x.shape[0] != n or x.device != device or not x.is_contiguous():
        raise ValueError(f"{name}: contiguous {dtype} of length {n} on {device}")
    if x.requires_grad:
        _refuse_grad(name, x)
    return x.data_ptr()


def _work(size, device):
    """(tensor, address) of a work buffer; a size of 1 says that none is needed."""
    if size == 1:
        return None, None
    work = torch.empty(size, dtype=torch.uint8, device=device)
    return work, work.data_ptr()


def _eps(eps):
    if eps is None:
        return -1.0
    if not eps >= 0:
        raise ValueError("eps is not negative")
    return eps


def last_error(status):
    """The status of the first product that failed on the device among those of
    weights that share `status`, which it clears (synchronises)."""
    with torch.cuda.device(status.device):
        return D.dm_products_last_error(status, torch._C._cuda_getCurrentRawStream(status.device.index))


def quantize(x, *, eps=None, count=None):
    """(q, scale): the rows of x [rows, k], bfloat16 or float16, in 8 bits: q
    int8 [rows, k] = 127 x / max |x| rounded, scale float32 [rows].  eps: rows
    are first divided by the root of their mean square plus eps.  count: an
    int32 tensor of one element, the number of rows that there are."""
    device = x.device
    xp, row = _matrix("x", x, TYPES, device)
    rows, k = x.shape
    q_row = -(-k // 16) * 16
    q = torch.empty(rows, q_row, dtype=torch.int8, device=device)
    scale = torch.empty(rows, dtype=torch.float32, device=device)
    a = D.dm_quantize_args(xp, q.data_ptr(), scale.data_ptr(), None if count is None else _vector("count", count, torch.int32, device, 1),
                           row, q_row, TYPES[x.dtype], rows, k, _eps(eps))
    _call("dm_quantize", device, C.byref(a))
    return q if q_row == k else q[:, :k], scale


class Weights:
    """Weights of a product, w [n, k], or of many experts', [experts, n, k]:
    bfloat16 or float16, or int8 with scale float32 [(experts,) n].  Keeps the
    tensors; calls that fail on the device say so in last_error().  status: an
    int32 tensor of one element, 0, that several share, to be asked once."""

    def __init__(self, w, scale=None, *, status=None):
        if w.dim() not in (2, 3) or w.numel() == 0 or w.shape[-1] > 1 and w.stride(-1) != 1:
            raise ValueError("weights are [n, k] or [experts, n, k], not empty, the last dimension contiguous")
        if max(w.shape) > _MOST:
            raise ValueError("weights have at most 2^31 - 1 of each dimension")
        if (w.dtype is torch.int8) != (scale is not None) or (scale is None and w.dtype not in TYPES):
            raise ValueError("weights are bfloat16 or float16, or int8 with a scale")
        if w.device.type != "cuda":
            raise ValueError("weights live on a CUDA device")
        self.device = w.device
        for name, x in (("w", w), ("scale", scale)):
            if x is not None and x.requires_grad:
                raise ValueError(f"{name} requires grad, and products give no gradients: detach it")
        if scale is not None and (scale.dtype is not torch.float32 or scale.shape != w.shape[:-1] or not scale.is_contiguous() or
                                  scale.device != w.device):
            raise ValueError(f"scale: contiguous float32 of shape {tuple(w.shape[:-1])} on {w.device}")
        self.w, self.scale, self.dtype, self.grouped = w, scale, w.dtype, w.dim() == 3
        self.experts = w.shape[0] if self.grouped else 1
        self.n, self.k = w.shape[-2:]
        step = 16 // w.element_size()
        row = w.stride(-2) if self.n > 1 else -(-self.k // step) * step
        self.struct = D.dm_weights(w.data_ptr(), None if scale is None else scale.data_ptr(),
                                   D.DM_I8 if scale is not None else TYPES[w.dtype], self.experts, self.n, self.k, row,
                                   w.stride(0) if self.experts > 1 else 0)
        self.ref, self.key = C.byref(self.struct), (w.dtype, self.experts, self.n, self.k)
        if status is None:
            status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.status = status
        self.status_at = _vector("status", status, torch.int32, self.device, 1)
        self._streams = set()   # whose work may still use the weights
        if not D.dm_product_bytes(self.struct, 0):   # no set of weights: rows or experts that begin off 16 bytes, too many
            raise D.DualMapError(D.DM_ERR_INVALID_ARG, "dm_product_bytes")

    @classmethod
    def quantized(cls, w, *, status=None):
        """8-bit weights, a scale a channel, of bfloat16 or float16 ones."""
        q, scale = quantize(w.detach().flatten(0, -2))
        if w.dim() == 3:
            q, scale = q.unflatten(0, w.shape[:2]), scale.unflatten(0, w.shape[:2])
        return cls(q, scale, status=status)

    def last_error(self):
        """The status of the first product that failed on the device, which it clears (synchronises)."""
        return last_error(self.status)

    def _hold(self):
        """Keeps the memory, once it is dropped, from being given out before the
        current stream is done with it (once per stream)."""
        raw = torch._C._cuda_getCurrentRawStream(self.device.index)
        if raw not in self._streams:
            stream = torch.cuda.current_stream(self.device)
            for x in (self.w, self.scale, self.status):
                if x is not None:
                    x.record_stream(stream)
            self._streams.add(raw)


def product(x, weights, offsets=None, *, x_scale=None, sources=None, per_source=1, gated=False, out=None, dtype=None):
    """Rows times their expert's weights: y [rows, n], or [rows, n / 2] where
    gated: silu of the first half of the channels times the second.

    x [x_rows, k] of the weights' type; int8 with x_scale float32 [x_rows].
    offsets: int32 [experts + 1], expert e has rows offsets[e] .. offsets[e +
    1]; without it one expert has them all.  sources: int32 [rows], row r reads
    row sources[r] // per_source of x.  out: where y goes, [rows, n] of bfloat16,
    float16 or float32, which overlaps none of the inputs; rows outside the offsets
    stay as they were (in a new output: whatever memory held).  dtype: of a new
    output (default: x's, for int8 bfloat16)."""
    w, device = weights, weights.device
    xp, x_row = _matrix("x", x, (w.dtype,), device, None, w.k)
    if (x_scale is None) != (w.scale is None):
        raise ValueError("x_scale comes with int8 weights")
    sp = None if x_scale is None else _vector("x_scale", x_scale, torch.float32, device, x.shape[0])
    if offsets is None and w.experts > 1:
        raise ValueError("products of many experts want offsets")
    op = None if offsets is None else _vector("offsets", offsets, torch.int32, device, w.experts + 1)
    n = x.shape[0] if sources is None else sources.shape[0]
    if gated and w.n % 2:
        raise ValueError("a gated product has an even number of channels")
    if not 1 <= per_source < 1 << 32:
        raise ValueError("per_source is 1 to 2^32 - 1")
    width = w.n // 2 if gated else w.n
    if out is None:
        out = torch.empty(n, width, dtype=dtype or (torch.bfloat16 if w.scale is not None else w.dtype), device=device)
    yp, y_row = _matrix("out", out, SCORES, device, n, width)
    gathered = sources is not None
    size = _size("dm_product_bytes", device, (w.key, n, gated, gathered), w.ref, n, int(gated), int(gathered))
    w._hold()
    work, at = _work(size, device)
    a = D.dm_product_args(xp, sp, yp, op, None if sources is None else _vector("sources", sources, torch.int32, device, n),
                          w.status_at, at, size, x_row, y_row, n, x.shape[0], per_source, SCORES[out.dtype], gated, 0)
    _call("dm_product", device, w.ref, C.byref(a))
    return out


class Choice:
    """The experts of a batch's tokens (choose)."""

    def __init__(self, ids, weights, offsets, slots, sources):
        self.ids, self.weights, self.offsets, self.slots, self.sources = ids, weights, offsets, slots, sources


def choose(logits, top_k, *, renormalize=True):
    """The top_k experts of each row of logits [tokens, experts], bfloat16,
    float16 or float32, ties to the lowest id; a Choice of ids int32 [tokens,
    top_k], weights float32 [tokens, top_k] (softmax over the chosen, or over
    all where not renormalize), and the pairs sorted by expert: offsets int32
    [experts + 1], slots int32 [tokens, top_k] (pair -> slot) and sources int32
    [tokens * top_k] (slot -> pair, token * top_k + place).  An expert with a
    score of minus infinity is not chosen: id and slot -1, weight 0."""
    device = logits.device
    xp, row = _matrix("logits", logits, SCORES, device)
    tokens, experts = logits.shape
    if top_k > _MOST:
        raise D.DualMapError(D.DM_ERR_INVALID_ARG, "dm_choose_bytes")
    size = _size("dm_choose_bytes", device, (tokens, experts, top_k), tokens, experts, top_k)
    ids = torch.empty(tokens, top_k, dtype=torch.int32, device=device)
    weights = torch.empty(tokens, top_k, dtype=torch.float32, device=device)
    slots = torch.empty(tokens, top_k, dtype=torch.int32, device=device)
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=device)
    sources = torch.empty(tokens * top_k, dtype=torch.int32, device=device)
    work, at = _work(size, device)
    a = D.dm_choose_args(xp, row, SCORES[logits.dtype], tokens, experts, top_k, bool(renormalize), 0, ids.data_ptr(),
                         weights.data_ptr(), offsets.data_ptr(), slots.data_ptr(), sources.data_ptr(), at, size)
    _call("dm_choose_experts", device, C.byref(a))
    return Choice(ids, weights, offsets, slots, sources)


class Linear:
    """y = x w^T for one set of weights; with 8-bit weights the rows are
    quantised first."""

    def __init__(self, weights):
        if weights.grouped:
            raise ValueError("a projection has one set of weights [n, k]")
        self.weights = weights

    def __call__(self, x, *, eps=None, out=None):
        """x [rows, k], bfloat16 or float16; y of x's type, or out, which does not
        overlap x.  eps (8-bit weights): rows are first divided by the root of their
        mean square plus eps, which costs nothing here."""
        w = self.weights
        if w.scale is None:
            if eps is not None:
                raise ValueError("a norm comes with int8 weights")
            return product(x, w, out=out)
        device, rows = w.device, x.shape[0]
        xp, x_row = _matrix("x", x, TYPES, device, None, w.k)
        if out is None:
            out = torch.empty(rows, w.n, dtype=x.dtype, device=device)
        yp, y_row = _matrix("out", out, SCORES, device, rows, w.n)
        size = _size("dm_linear_bytes", device, (w.key, rows), w.ref, rows)
        w._hold()
        work, at = _work(size, device)
        a = D.dm_linear_args(xp, yp, w.status_at, at, size, x_row, y_row, TYPES[x.dtype], SCORES[out.dtype], rows, _eps(eps))
        _call("dm_linear", device, w.ref, C.byref(a))
        return out

    def last_error(self):
        return self.weights.last_error()


class Experts:
    """A layer of experts, each down(silu(g) u) with (g, u) = up(x): up [experts,
    2 m, k] and down [experts, k, m], both 16-bit or both int8.  Errors are those
    of up's status."""

    def __init__(self, up, down, top_k, *, renormalize=True):
        if not up.grouped or not down.grouped or up.device != down.device or up.dtype is not down.dtype:
            raise ValueError("up and down are experts' weights of one type on one device")
        if up.experts != down.experts or up.n != 2 * down.k or down.n != up.k:
            raise ValueError("up is [experts, 2 m, k] and down [experts, k, m]")
        if not 1 <= top_k <= min(up.experts, 32):
            raise ValueError("top_k is 1 to the number of experts, and at most 32")
        self.up, self.down, self.top_k, self.renormalize = up, down, top_k, bool(renormalize)
        self.key = up.key, down.key, top_k

    def __call__(self, x, logits, *, residual=None, out=None):
        """y [tokens, k] = residual + the sum over each token's top_k experts by
        logits [tokens, experts] of weight times expert(x [tokens, k]).  out may
        be residual, and overlaps nothing else."""
        up, device, tokens = self.up, self.up.device, x.shape[0]
        types = TYPES if up.scale is not None else (up.dtype,)
        xp, x_row = _matrix("x", x, types, device, None, up.k)
        lp, l_row = _matrix("logits", logits, SCORES, device, tokens, up.experts)
        if out is None:
            out = torch.empty(tokens, up.k, dtype=x.dtype, device=device)
        yp, y_row = _matrix("out", out, (x.dtype,), device, tokens, up.k)
        rp, r_row = (None, 0) if residual is None else _matrix("residual", residual, (x.dtype,), device, tokens, up.k)
        size = _size("dm_experts_bytes", device, (self.key, tokens), up.ref, self.down.ref, tokens, self.top_k)
        up._hold()
        self.down._hold()
        work = torch.empty(size, dtype=torch.uint8, device=device)
        a = D.dm_experts_args(xp, lp, rp, yp, up.status_at, work.data_ptr(), size, x_row, l_row, r_row, y_row,
                              TYPES[x.dtype], SCORES[logits.dtype], tokens, self.top_k, self.renormalize, 0)
        _call("dm_experts", device, up.ref, self.down.ref, C.byref(a))
        return out

    def last_error(self):
        """The status of the first call that failed on the device, which it clears (synchronises)."""
        return self.up.last_error()
