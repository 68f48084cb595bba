"""An instance's prefix cache over torch tensors: pages of keys and values,
sequences that share the pages of a common prefix, and the attention that
reads them (dm_cache_* of include/dualmap.h).

Only marshalling: it checks shapes and types, allocates outputs and work
buffers on the device, and enqueues the C calls on torch's current stream.
Calls on one cache, and the attention of one plan, have to be ordered by the
caller, as work that shares a tensor is.  The calls serve: they give no
gradients, so with grad mode on they refuse tensors that want one.
"""

import ctypes as C

import torch

from . import dualmap as D

TYPES = {torch.bfloat16: D.DM_BF16, torch.float16: D.DM_F16}
LAYOUTS = {"heads": D.DM_PAGES_HEADS, "tokens": D.DM_PAGES_TOKENS}


class Plan:
    """One step's division over the GPU (PagedCache.plan), for all its layers."""

    def __init__(self, struct, keep, tokens, q_heads, errors, stream):
        self.struct, self.ref, self.keep, self.tokens, self.q_heads = struct, C.byref(struct), keep, tokens, q_heads
        self.errors = errors   # that the cache had reported by then
        self.streams = {stream}   # whose work may still use the plan's buffer, first the one it was allocated on


class PagedCache:
    """k, v: [layers, pages, kv_heads, page_tokens, head_dim] (layout "heads")
    or [layers, pages, page_tokens, kv_heads, head_dim] ("tokens"), bfloat16 or
    float16, each page contiguous; tables int32 [max_seqs, max_blocks], lengths
    int32 [max_seqs], refs int32 [pages] (all zero in a cache without
    sequences).  The cache keeps these tensors and changes them."""

    def __init__(self, k, v, tables, lengths, refs, layout="heads"):
        if layout not in LAYOUTS:
            raise ValueError(f"layout {layout!r} is not one of {sorted(LAYOUTS)}")
        if k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype:
            raise ValueError("k and v are 5-dimensional, of one shape, layout and type")
        if k.dtype not in TYPES:
            raise ValueError(f"keys of type {k.dtype}: bfloat16 or float16 wanted")
        layers, pages, a, b, dim = k.shape
        if k.stride()[2:] != (b * dim, dim, 1):
            raise ValueError("a page of k or v is not contiguous")
        for name, x, shape in (("tables", tables, (lengths.shape[0], tables.shape[-1])), ("lengths", lengths, lengths.shape[:1]),
                               ("refs", refs, (pages,))):
            if x.dtype != torch.int32 or tuple(x.shape) != tuple(shape) or not x.is_contiguous():
                raise ValueError(f"{name}: contiguous int32 of shape {tuple(shape)} wanted")
        if len({x.device for x in (k, v, tables, lengths, refs)}) != 1 or k.device.type != "cuda":
            raise ValueError("k, v, tables, lengths and refs live on one CUDA device")
        self.k, self.v, self.tables, self.lengths, self.refs, self.layout = k, v, tables, lengths, refs, layout
        self.device, self.dtype, self.layers, self.head_dim = k.device, k.dtype, layers, dim
        self.kv_heads, self.page_tokens = (a, b) if layout == "heads" else (b, a)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.struct = D.dm_cache(
            k.data_ptr(), v.data_ptr(), TYPES[k.dtype], LAYOUTS[layout], layers, pages, self.page_tokens, self.kv_heads, dim,
            lengths.shape[0], tables.shape[1], 0, k.stride(0) if layers > 1 else 0, k.stride(1) if pages > 1 else a * b * dim,
            tables.data_ptr(), lengths.data_ptr(), refs.data_ptr(), self.status.data_ptr(), None, 0)
        size = D.dm_cache_work_bytes(self.struct)
        if not size:
            raise D.DualMapError(D.DM_ERR_INVALID_ARG, "dm_cache_work_bytes")
        self.work = torch.empty(size, dtype=torch.uint8, device=self.device)
        self.struct.work, self.struct.work_bytes = self.work.data_ptr(), size
        self._lib, self._ref, self._plan_bytes, self._errors = D.lib(), C.byref(self.struct), {}, 0
        self._streams = set()   # whose work may still use the cache

    @classmethod
    def empty(cls, *, pages, kv_heads, head_dim, max_seqs, max_tokens, page_tokens=16, layers=1, dtype=torch.bfloat16,
              layout="heads", device="cuda"):
        """A cache without sequences, each of up to max_tokens tokens."""
        if layout not in LAYOUTS:
            raise ValueError(f"layout {layout!r} is not one of {sorted(LAYOUTS)}")
        inner = (kv_heads, page_tokens) if layout == "heads" else (page_tokens, kv_heads)
        k = torch.empty((layers, pages) + inner + (head_dim,), dtype=dtype, device=device)
        ints = dict(dtype=torch.int32, device=device)
        return cls(k, torch.empty_like(k), torch.zeros(max_seqs, -(-max_tokens // page_tokens), **ints),
                   torch.zeros(max_seqs, **ints), torch.zeros(pages, **ints), layout)

    # These run once per call of a decode step, so they ask each tensor for
    # little: a call costs a few microseconds of Python.

    def _ints(self, name, x, n=None):
        """The address of a contiguous int32 vector (of n elements)."""
        if x.dtype is not torch.int32 or x.dim() != 1 or x.device != self.device or not x.is_contiguous() or \
                (n is not None and x.shape[0] != n):
            raise ValueError(f"{name}: contiguous int32 on {self.device}" + (f" of length {n}" if n is not None else ""))
        return x.data_ptr()

    @staticmethod
    def _no_grad(name, x):
        if x.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} requires grad, and this call gives no gradients: use torch.no_grad() or detach it")

    def _rows(self, name, x, tokens, heads):
        """Address and strides (token, head) of [tokens, heads, head_dim]."""
        shape, stride = (tokens, heads, self.head_dim), x.stride()
        if x.dtype is not self.dtype or x.device != self.device or x.shape != shape or stride[2] != 1:
            raise ValueError(f"{name}: {self.dtype} on {self.device} of shape {shape}, head_dim contiguous")
        self._no_grad(name, x)
        # the stride of a dimension of one element says nothing
        return x.data_ptr(), (stride[0] if tokens > 1 else 0), (stride[1] if heads > 1 else 0)

    def _vector(self, name, x):
        if x is None:
            return None
        if x.dtype is not self.dtype or x.shape != (self.head_dim,) or x.device != self.device or not x.is_contiguous():
            raise ValueError(f"{name}: contiguous {self.dtype} of shape {(self.head_dim,)} on {self.device}")
        self._no_grad(name, x)
        return x.data_ptr()

    def _call(self, name, *args):
        """Enqueues a dm_cache_* call on torch's current stream of the cache's device."""
        if torch.cuda.current_device() != self.device.index:
            with torch.cuda.device(self.device):
                return self._call(name, *args)
        stream = torch._C._cuda_getCurrentRawStream(self.device.index)
        if stream not in self._streams:
            self._hold(stream, self._streams, self.k, self.v, self.tables, self.lengths, self.refs, self.status, self.work)
        rc = getattr(self._lib, name)(self._ref, *args, stream)
        if rc:
            raise D.DualMapError(rc, name)

    def _hold(self, stream, seen, *tensors):
        """Keeps the memory of `tensors`, once they are dropped, from being given
        out before the current stream is done with them (once per stream)."""
        for x in tensors:
            x.record_stream(torch.cuda.current_stream(self.device))
        seen.add(stream)

    def last_error(self):
        """The status of the first call that was refused on the device, which it clears (synchronises)."""
        with torch.cuda.device(self.device):
            e = D.dm_cache_last_error(self.struct, torch._C._cuda_getCurrentRawStream(self.device.index))
        self._errors += e != 0
        return e

    def extend(self, seqs, add):
        """Sequence seqs[i] grows by add[i] tokens; the pages it lacks are taken."""
        n = seqs.shape[0]
        self._call("dm_cache_extend", self._ints("seqs", seqs), self._ints("add", add, n), n)

    def fork(self, parents, children, lengths):
        """The empty sequence children[i] becomes the first lengths[i] tokens of parents[i]."""
        n = parents.shape[0]
        self._call("dm_cache_fork", self._ints("parents", parents), self._ints("children", children, n),
                   self._ints("lengths", lengths, n), n)

    def free(self, seqs):
        """The sequences give up their pages."""
        self._call("dm_cache_free", self._ints("seqs", seqs), seqs.shape[0])

    def compact(self, tables_out=None, refs_out=None, moved=None):
        """Moves the pages in use to the lowest ids.  tables_out, refs_out: where
        the new bookkeeping goes (default: in place); moved: an int32 tensor of
        one element for the number of pages moved."""
        for name, x, like in (("tables_out", tables_out, self.tables), ("refs_out", refs_out, self.refs)):
            if x is not None and (x.dtype is not torch.int32 or x.shape != like.shape or not x.is_contiguous() or
                                  x.device != self.device):
                raise ValueError(f"{name}: contiguous int32 of shape {tuple(like.shape)} on {self.device}")
        self._call("dm_cache_compact", None if tables_out is None else tables_out.data_ptr(),
                   None if refs_out is None else refs_out.data_ptr(), None if moved is None else self._ints("moved", moved, 1))

    def append(self, seqs, offsets, q, k, v, cos=None, sin=None, *, layer=0, q_weight=None, k_weight=None, eps=1e-6,
               interleaved=False, out=None):
        """Norms and rotates one layer's new queries and keys and stores keys and
        values; returns the queries.

        Sequence seqs[i]'s new tokens are rows offsets[i] .. offsets[i + 1] of q
        [tokens, q_heads, head_dim], k and v [tokens, kv_heads, head_dim], and
        the last ones of the sequence, which has been extended by them; each is
        named once.  cos, sin: float32 [positions, rotated dims / 2]; without
        them nothing turns.
        q_weight, k_weight [head_dim]: without one there is no norm.  out:
        where the queries go; may be q."""
        n, tokens, heads = seqs.shape[0], k.shape[0], q.shape[1]
        if out is None:
            out = torch.empty(q.shape, dtype=self.dtype, device=self.device)
        qp, qt, qh = self._rows("q", q, tokens, heads)
        kp, kt, kh = self._rows("k", k, tokens, self.kv_heads)
        vp, vt, vh = self._rows("v", v, tokens, self.kv_heads)
        op, ot, oh = self._rows("out", out, tokens, heads)
        if (cos is None) != (sin is None):
            raise ValueError("cos and sin come together")
        cp = sp = None
        rows = dims = 0
        if cos is not None:
            for name, x in (("cos", cos), ("sin", sin)):
                if x.dtype is not torch.float32 or x.dim() != 2 or x.shape != cos.shape or not x.is_contiguous() or \
                        x.device != self.device:
                    raise ValueError(f"{name}: contiguous float32 [positions, rotated dims / 2] on {self.device}")
                self._no_grad(name, x)
            cp, sp, (rows, dims) = cos.data_ptr(), sin.data_ptr(), cos.shape
        a = D.dm_append_args(self._ints("seqs", seqs), self._ints("offsets", offsets, n + 1), n, tokens, layer, heads,
                             qp, kp, vp, op, qt, qh, kt, kh, vt, vh, ot, oh, self._vector("q_weight", q_weight),
                             self._vector("k_weight", k_weight), cp, sp, rows, 2 * dims, bool(interleaved), eps)
        self._call("dm_cache_append", C.byref(a))
        return out

    def plan(self, seqs, offsets, tokens, q_heads, group_offsets=None, group_prefix=None):
        """Divides the attention of a step of `tokens` query rows over the GPU.
        Group g: sequences group_offsets[g] .. group_offsets[g + 1] of the step,
        which start with the same group_prefix[g] tokens in the same pages."""
        n, groups, go, gp = seqs.shape[0], 0, None, None
        if (group_offsets is None) != (group_prefix is None):
            raise ValueError("group_offsets and group_prefix come together")
        if group_prefix is not None:
            groups = group_prefix.shape[0]
            gp, go = self._ints("group_prefix", group_prefix), self._ints("group_offsets", group_offsets, groups + 1)
        shape = (n, groups, tokens, q_heads)
        size = self._plan_bytes.get(shape)
        if size is None:
            with torch.cuda.device(self.device):   # it depends on the device's SMs
                size = D.dm_plan_bytes(self.struct, *shape)
            if not size:
                raise D.DualMapError(D.DM_ERR_INVALID_ARG, "dm_plan_bytes")
            if len(self._plan_bytes) > 4096:
                self._plan_bytes.clear()
            self._plan_bytes[shape] = size
        work = torch.empty(size, dtype=torch.uint8, device=self.device)
        s = D.dm_plan(self._ints("seqs", seqs), self._ints("offsets", offsets, n + 1), n, tokens, q_heads, groups, go, gp,
                      work.data_ptr(), size)
        self._call("dm_cache_plan", C.byref(s))
        return Plan(s, (seqs, offsets, group_offsets, group_prefix, work), tokens, q_heads, self._errors,
                    torch._C._cuda_getCurrentRawStream(self.device.index))

    def attend(self, plan, q, *, layer=0, scale=None, out=None, lse=None):
        """One layer's attention of the planned step: q [tokens, q_heads,
        head_dim], scale (default head_dim ** -0.5).  lse: float32 [tokens,
        q_heads] for the logarithms of the sums.  A plan that was refused writes
        nothing: a new output then is NaN once that error has been read."""
        if out is None:
            out = torch.empty(q.shape, dtype=self.dtype, device=self.device)
            if plan.errors != self._errors:   # the error may have been the plan's
                out.fill_(float("nan"))
        qp, qt, qh = self._rows("q", q, plan.tokens, plan.q_heads)
        op, ot, oh = self._rows("out", out, plan.tokens, plan.q_heads)
        if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (plan.tokens, plan.q_heads) or
                                not lse.is_contiguous() or lse.device != self.device):
            raise ValueError(f"lse: contiguous float32 of shape {(plan.tokens, plan.q_heads)} on {self.device}")
        stream = torch._C._cuda_getCurrentRawStream(self.device.index)
        if stream not in plan.streams:
            self._hold(stream, plan.streams, plan.keep[-1])
        a = D.dm_attend_args(layer, self.head_dim ** -0.5 if scale is None else scale, qp, op,
                             None if lse is None else lse.data_ptr(), qt, qh, ot, oh)
        self._call("dm_cache_attend", plan.ref, C.byref(a))
        return out
