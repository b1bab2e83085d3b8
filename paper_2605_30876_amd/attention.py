"""The attention half of a decode step's layers: rotary positions, a paged
key/value cache, and attention of a step's new tokens over it.

:class:`PagedCache` owns the pages and page tables of a number of sequences
(slots), :class:`Rope` the rotation's frequencies, :class:`BlockAttention` the
plan and workspace of one batch shape.  A step is

    cache.resize(slots, lens + new)           # pages for the new tokens
    att.begin(q_offsets, slots); att.plan()   # once, for all layers
    per layer: att.append(l, k, v, q); att.attend(l, q) -> out

:class:`AttentionLayer` adds a layer's projections and is what
:func:`.layer.decode_step` calls between its MoE layers.

Everything is enqueued on the current stream (or ``stream``); nothing is read
back, and calls whose outputs are given allocate nothing (but for a cache's
workspace beyond 64 MB), so a step can be captured in a HIP graph.  An object's calls share its workspace: calls
on one object must not overlap in time.
"""
from __future__ import annotations

import contextlib
import math

import torch

from . import lib


def _i32(t: torch.Tensor, name: str, device, n: int = 0) -> torch.Tensor:
    if t.dtype != torch.int32 or not t.is_contiguous() or t.numel() < n or t.device != device:
        raise ValueError(f"{name} must be a contiguous int32 tensor on {device} of at least {n} values, "
                         f"not {t.dtype} {list(t.shape)} on {t.device}")
    return t


def _stream(stream):
    """The current stream set to a call's: what the call allocates and fills for itself is then ordered with its kernels."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


class _On:
    """The device of an object's tensors as the current one."""

    def __init__(self, device: torch.device):
        self.device = device

    def __enter__(self):
        if self.device.type != "cuda":
            raise ValueError(f"the tensors are on {self.device}: the kernels need a GPU's")
        self.back = torch._C._cuda_getDevice()
        if self.device.index is not None and self.device.index != self.back:
            torch.cuda.set_device(self.device)

    def __exit__(self, *a):
        if self.device.index is not None and self.device.index != self.back:
            torch.cuda.set_device(self.back)


def _no_gradient(t: torch.Tensor, name: str):
    """These calls record nothing: a tensor whose gradient is asked for would lose it without a word."""
    if t.requires_grad and torch.is_grad_enabled():
        raise RuntimeError(f"{name} requires a gradient, which these calls do not record: call under torch.no_grad() or detach it "
                           f"(a rotation's gradient is its inverse)")


def _heads(t: torch.Tensor, name: str, rows: int | None, heads: int, dim: int, like: torch.dtype, device) -> torch.Tensor:
    """Checks a step's tensor [rows, heads, dim]: heads and their elements dense, rows any stride.  Returns it, a single row with
    the stride of dense ones (it may have any, which says nothing)."""
    shape = t.shape  # a new object each time: small calls are as long as these checks
    if len(shape) != 3 or shape[2] != dim or shape[1] != heads or (rows is not None and shape[0] < rows):
        raise ValueError(f"{name} must be [{'T' if rows is None else rows}, {heads}, {dim}], not {list(t.shape)}")
    if t.dtype != like or t.device != device:
        raise ValueError(f"{name} must be {like} on {device}, not {t.dtype} on {t.device}")
    if t.requires_grad:
        _no_gradient(t, name)
    by_row, by_head, by_element = t.stride()
    if by_element != 1 or (heads > 1 and by_head != dim):
        raise ValueError(f"{name}: heads and their elements must be dense (strides {t.stride()})")
    if (by_row < heads * dim or by_row % 8) and shape[0] == 1:
        return t.as_strided(shape, (heads * dim, dim, 1))
    return t


class Rope:
    """Rotary positions of the first ``rot_dim`` elements of a head.

    interleaved: pairs (2i, 2i+1) instead of (i, i + rot_dim/2).  scaling for
    contexts beyond the trained ``original`` length: "none", "linear", "ntk"
    or "yarn", by ``factor`` (see dmoe_rope_scaling)."""

    def __init__(self, rot_dim: int, base: float = 10000.0, interleaved: bool = False, scaling: str = "none",
                 factor: float = 1.0, original: int = 4096, device="cuda"):
        if scaling not in lib.ROPE_SCALING:
            raise ValueError(f"scaling must be one of {sorted(lib.ROPE_SCALING)}, not {scaling!r}")
        turns, self.scale = lib.dmoe_rope_turns(rot_dim, base, scaling, factor, original)
        self.rot_dim, self.interleaved = rot_dim, interleaved
        self.turns = torch.tensor(turns, dtype=torch.float64, device=device)
        self.c = lib.dmoe_rotary(lib.ptr(self.turns), rot_dim, int(interleaved), self.scale)

    def apply(self, x: torch.Tensor, positions: torch.Tensor, out: torch.Tensor | None = None, inverse: bool = False,
              stream=None) -> torch.Tensor:
        """x [T, heads, dim] rotated at positions [T] (int32) into out (default: x itself).  inverse: the gradient
        of a forward call with respect to x, given the gradient of its output."""
        T, heads, dim = x.shape
        row = _heads(x, "x", T, heads, dim, x.dtype, self.turns.device)
        to = row if out is None else _heads(out, "out", T, heads, dim, x.dtype, x.device)
        out = x if out is None else out
        if T == 0:
            return out
        _i32(positions, "positions", x.device, T)
        with _On(x.device):
            lib.dmoe_rope(row, to, T, heads, dim, positions, self.c, inverse, stream)
        return out


class PagedCache:
    """Keys and values of ``n_layers`` layers in ``n_pages`` pages of
    ``page_tokens`` tokens, held by ``n_slots`` sequences of up to
    ``max_pages`` pages.  k, v, table, lens, refs: existing arrays to use
    (layouts: dmoe_cache in include/dmoe.h) instead of new, empty ones (keys
    and values 0); the others are then made on their device.

    ``format``: what the pages hold: "plain", elements of ``dtype``; "fp8" or "fp4", codes of 8 or 4 bits with a scale per 32
    elements of a token's head; "fp8_fp4", keys in 8 bits and values in 4 (dmoe_kv_format).  The rows
    that are appended, read and attended with are of ``dtype`` all the same.  k and v of a cache of few bits are uint8.

    ``status`` holds the outcome of the last update that was given no tensor
    of its own for it; ``refused`` [n_slots] of every slot's last update, 0 if it was done.  A
    slot that is marked there has no new tokens: :meth:`BlockAttention.append`
    and ``attend`` leave its rows alone until an update of it succeeds (one to its present length does)."""

    def __init__(self, n_layers: int, n_pages: int, page_tokens: int, n_kv_heads: int, head_dim: int, n_slots: int,
                 max_pages: int, dtype: torch.dtype = torch.bfloat16, device="cuda", k=None, v=None, table=None, lens=None,
                 refs=None, format: str = "plain"):
        dt = {torch.float32: lib.DMOE_F32, torch.bfloat16: lib.DMOE_BF16}.get(dtype)
        if dt is None:
            raise TypeError(f"unsupported element type {dtype}")
        if format not in lib.KV_FORMAT:
            raise ValueError(f"format must be one of {sorted(lib.KV_FORMAT)}, not {format!r}")
        fmt = lib.KV_FORMAT[format]
        page_bytes = [size(dt, fmt, page_tokens, n_kv_heads, head_dim) for size in (lib.dmoe_cache_key_page_bytes, lib.dmoe_cache_value_page_bytes)]
        if page_bytes[0] == 0:
            raise ValueError(f"no such page: page_tokens={page_tokens}, n_kv_heads={n_kv_heads}, head_dim={head_dim}")
        self.n_layers, self.n_pages, self.page_tokens, self.n_kv_heads = n_layers, n_pages, page_tokens, n_kv_heads
        self.head_dim, self.n_slots, self.max_pages, self.dtype = head_dim, n_slots, max_pages, dtype
        self.format = format
        held = dtype if format == "plain" else torch.uint8
        elems = [n // torch.empty((), dtype=held).element_size() for n in page_bytes]
        # new arrays lie where the given ones do: a kernel follows the addresses of all of them
        device = next((t.device for t in (k, v, table, lens, refs) if t is not None), device)

        def pool(t, name, elems):
            if t is None:
                return torch.zeros((n_layers, n_pages, elems), dtype=held, device=device)
            if tuple(t.shape) != (n_layers, n_pages, elems) or t.dtype != held or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous {held} [{n_layers}, {n_pages}, {elems}]")
            return t

        def ints(t, name, shape, fill):
            if t is None:
                return torch.full(shape, fill, dtype=torch.int32, device=device)
            if tuple(t.shape) != shape:
                raise ValueError(f"{name} must be int32 {list(shape)}")
            return _i32(t, name, self.k.device)

        self.k, self.v = pool(k, "k", elems[0]), pool(v, "v", elems[1])
        if self.v.device != self.k.device:
            raise ValueError(f"k is on {self.k.device}, v on {self.v.device}")
        self.table = ints(table, "table", (n_slots, max_pages), -1)
        self.lens = ints(lens, "lens", (n_slots,), 0)
        self.refs = ints(refs, "refs", (n_pages,), 0)
        self.device = self.k.device
        self.status = torch.zeros((1,), dtype=torch.int32, device=device)
        self.refused = torch.zeros((n_slots,), dtype=torch.int32, device=device)
        self.c = lib.dmoe_cache(lib.ptr(self.k), lib.ptr(self.v), lib.ptr(self.table), lib.ptr(self.lens), lib.ptr(self.refs),
                                dt, n_layers, n_pages, page_tokens, n_kv_heads, head_dim, n_slots, max_pages,
                                lib.ptr(self.refused), fmt)
        # for calls on every slot, where that is not much; larger calls add one of their own
        nbytes = max(lib.dmoe_cache_update_workspace_size(min(n_slots, 4096), max_pages, n_pages),
                     lib.dmoe_cache_compact_workspace_size(n_pages))
        self._ws = [torch.empty((min(nbytes, 64 << 20),), dtype=torch.uint8, device=device)]

    def _workspace(self, nbytes: int, stream) -> torch.Tensor:
        """The last workspace, or a larger one of the call's stream outside graph capture (a captured call keeps the one
        it was captured with)."""
        if self._ws[-1].numel() < nbytes:
            capturing = torch.cuda.is_current_stream_capturing()
            with _stream(stream):
                if capturing or torch.cuda.is_current_stream_capturing():
                    raise RuntimeError("the cache's workspace is too small for this call: run it once before capturing it")
                self._ws.append(torch.empty((nbytes,), dtype=torch.uint8, device=self.device))
        return self._ws[-1]

    def update(self, dst: torch.Tensor, new_lens: torch.Tensor, src: torch.Tensor | None = None,
               keep: torch.Tensor | None = None, status: torch.Tensor | None = None, stream=None):
        """Entry i: slot dst[i] holds the first keep[i] tokens of slot src[i] (default: its own) and room for
        new_lens[i] (dmoe_cache_update).  int32 device tensors.  The outcome is left in ``status`` (default
        ``self.status``): 0 done, n > 0 pages lacking, -1 refused; unless 0 nothing was changed but ``self.refused``
        of the slots."""
        n = dst.numel()
        if n == 0:
            return
        d = self.device
        _i32(dst, "dst", d), _i32(new_lens, "new_lens", d, n)
        for t, name in ((src, "src"), (keep, "keep")):
            if t is not None:
                _i32(t, name, d, n)
        status = self.status if status is None else _i32(status, "status", d, 1)
        with _On(self.device):
            ws = self._workspace(lib.dmoe_cache_update_workspace_size(n, self.max_pages, self.n_pages), stream)
            lib.dmoe_cache_update(self.c, dst, src, keep, new_lens, n, status, ws, stream)

    def resize(self, slots: torch.Tensor, new_lens: torch.Tensor, stream=None, status: torch.Tensor | None = None):
        """Grows or truncates sequences to new_lens tokens."""
        self.update(slots, new_lens, status=status, stream=stream)

    def free(self, slots: torch.Tensor, stream=None, status: torch.Tensor | None = None):
        """Releases every page of the sequences."""
        with _stream(stream):
            self.update(slots, torch.zeros_like(slots), status=status, stream=stream)

    def fork(self, dst: torch.Tensor, src: torch.Tensor, keep: torch.Tensor, new_lens: torch.Tensor | None = None, stream=None,
             status: torch.Tensor | None = None):
        """Slot dst[i] becomes the first keep[i] tokens of slot src[i], sharing its full pages; with room for
        new_lens[i] tokens (default keep[i])."""
        self.update(dst, keep if new_lens is None else new_lens, src, keep, status, stream)

    def compact(self, table_out: torch.Tensor | None = None, refs_out: torch.Tensor | None = None,
                counts: torch.Tensor | None = None, stream=None):
        """Moves the live pages together at the pool's start.  table_out, refs_out: where the new table and counts
        go (default: in place); counts [2]: live pages, pages moved."""
        table_out = self.table if table_out is None else _i32(table_out, "table_out", self.device, self.table.numel())
        refs_out = self.refs if refs_out is None else _i32(refs_out, "refs_out", self.device, self.refs.numel())
        if counts is not None:
            _i32(counts, "counts", self.device, 2)
        with _On(self.device):
            ws = self._workspace(lib.dmoe_cache_compact_workspace_size(self.n_pages), stream)
            lib.dmoe_cache_compact(self.c, table_out, refs_out, counts, ws, stream)

    def read(self, layer: int, q_offsets: torch.Tensor, k: torch.Tensor | None = None, v: torch.Tensor | None = None,
             slots: torch.Tensor | None = None, starts: torch.Tensor | None = None, max_tokens: int | None = None, stream=None):
        """Keys and values of tokens as the cache holds them, into k and v [T, n_kv_heads, head_dim] (either may be None): rows
        q_offsets[i] .. q_offsets[i+1] receive the tokens from starts[i] on of slot slots[i] (default i), by default its
        last ones (dmoe_cache_read).  Tokens that the sequence does not have are 0, rows of no sequence stay as they
        are.  int32 device tensors; max_tokens: an upper bound of every sequence's tokens (default: every row)."""
        if k is None and v is None:
            raise ValueError("read() needs k or v")
        d, T, n = self.device, (v if k is None else k).shape[0], q_offsets.numel() - 1
        _i32(q_offsets, "q_offsets", d)
        if n < 1:
            raise ValueError("q_offsets must hold a value more than there are sequences")
        if slots is not None:
            _i32(slots, "slots", d, n)
        if starts is not None:
            _i32(starts, "starts", d, n)
        if k is not None:
            k = _heads(k, "k", T, self.n_kv_heads, self.head_dim, self.dtype, d)
        if v is not None:
            v = _heads(v, "v", T, self.n_kv_heads, self.head_dim, self.dtype, d)
            if v.shape[0] != T:
                raise ValueError(f"k and v must have the same rows, not {T} and {v.shape[0]}")
        if T == 0:
            return
        with _On(d):
            batch = lib.dmoe_batch(lib.ptr(q_offsets), lib.ptr(slots), n, T, T if max_tokens is None else min(max_tokens, T))
            lib.dmoe_cache_read(self.c, layer, batch, starts, k, v, stream)

    def copy_pages(self, pairs: torch.Tensor, stream=None):
        """Copies page pairs[i, 0] to page pairs[i, 1], all layers."""
        if pairs.numel() == 0:
            return
        if pairs.dim() != 2 or pairs.shape[1] != 2:
            raise ValueError(f"pairs must be [n, 2], not {list(pairs.shape)}")
        _i32(pairs, "pairs", self.device)
        with _On(self.device):
            lib.dmoe_cache_copy_pages(self.c, pairs, pairs.shape[0], stream)


class BlockAttention:
    """Attention of batches of up to ``n_seqs`` sequences, ``max_new`` new
    tokens each and ``T`` rows over a :class:`PagedCache`.

    mask_block: 0 every key of the sequence, 1 causal, n blocks of n tokens
    that see each other and everything before (a block-diffusion decoder's
    mask).  scale: default 1/sqrt(head_dim).  rope: rotates queries and keys
    as they are appended."""

    def __init__(self, cache: PagedCache, n_heads: int, n_seqs: int, max_new: int, T: int, mask_block: int = 0,
                 scale: float | None = None, rope: Rope | None = None):
        self.cache, self.n_heads, self.n_seqs, self.max_new, self.T = cache, n_heads, n_seqs, max_new, T
        self.mask_block, self.rope = mask_block, rope
        self.scale = 1.0 / math.sqrt(cache.head_dim) if scale is None else scale
        ints = lib.dmoe_attention_plan_ints(n_seqs, T, max_new, n_heads, cache.n_kv_heads)
        if ints == 0:
            raise ValueError(f"no such batch: n_seqs={n_seqs}, T={T}, max_new={max_new}, n_heads={n_heads}, "
                             f"n_kv_heads={cache.n_kv_heads}")
        if rope is not None and (rope.rot_dim > cache.head_dim or rope.turns.device != cache.device):
            raise ValueError(f"a rotation of {rope.rot_dim} elements on {rope.turns.device} does not fit head_dim={cache.head_dim} on "
                             f"{cache.device}")
        self._plan = torch.zeros((ints,), dtype=torch.int32, device=cache.device)
        nbytes = lib.dmoe_attention_workspace_size(cache.c.dt, n_seqs, T, max_new, n_heads, cache.n_kv_heads, cache.head_dim)
        self.workspace = torch.empty((nbytes,), dtype=torch.uint8, device=cache.device)
        self.batch, self._planned = None, False

    def begin(self, q_offsets: torch.Tensor, slots: torch.Tensor | None = None):
        """The step's batch: sequence i is rows q_offsets[i] .. q_offsets[i+1] of its tensors and slot slots[i]
        (default i) of the cache.  int32 device tensors, read by the calls that follow (kept here until the next
        begin(); a graph that captured such calls needs them as long as it lives); :meth:`attend` needs a :meth:`plan`
        of it first."""
        _i32(q_offsets, "q_offsets", self.cache.device, self.n_seqs + 1)
        if slots is not None:
            _i32(slots, "slots", self.cache.device, self.n_seqs)
        self._kept, self._planned = (q_offsets, slots), False
        self.batch = lib.dmoe_batch(lib.ptr(q_offsets), lib.ptr(slots), self.n_seqs, self.T, self.max_new)

    def _started(self):
        if self.batch is None:
            raise RuntimeError("begin() has not been called")
        return self.batch

    def plan(self, stream=None):
        """The step's work items, for :meth:`attend` of every layer: after the lengths are set, before the first attend;
        until offsets, slots or lengths change (pages may move)."""
        with _On(self.cache.device):
            lib.dmoe_attention_plan(self.cache.c, self._started(), self.n_heads, self.mask_block, self._plan, stream)
        self._planned = True

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, q: torch.Tensor | None = None,
               q_out: torch.Tensor | None = None, stream=None):
        """Stores the new keys (rotated) and values [T, n_kv_heads, head_dim] and rotates q [T, n_heads, head_dim]
        into q_out (default: q itself)."""
        c = self.cache
        k = _heads(k, "k", self.T, c.n_kv_heads, c.head_dim, c.dtype, c.device)
        v = _heads(v, "v", self.T, c.n_kv_heads, c.head_dim, c.dtype, c.device)
        if q is not None:
            q = _heads(q, "q", self.T, self.n_heads, c.head_dim, c.dtype, c.device)
            q_out = q if q_out is None else _heads(q_out, "q_out", self.T, self.n_heads, c.head_dim, c.dtype, c.device)
        elif q_out is not None:
            raise ValueError("q_out needs q")
        with _On(c.device):
            lib.dmoe_cache_append(c.c, layer, self._started(), k, v, q, q_out, self.n_heads,
                                  None if self.rope is None else self.rope.c, stream)

    def attend(self, layer: int, q: torch.Tensor, out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
               stream=None) -> torch.Tensor:
        """Attention of the (rotated) queries over the cache, into out [T, n_heads, head_dim] (default: a new tensor,
        allocated on the call's stream); lse [T, n_heads] (float32) receives the log-sum-exp of every row."""
        c = self.cache
        q = _heads(q, "q", self.T, self.n_heads, c.head_dim, c.dtype, c.device)
        if out is None:
            with _stream(stream):
                out = to = torch.empty_like(q)
        else:
            to = _heads(out, "out", self.T, self.n_heads, c.head_dim, c.dtype, c.device)
        if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous() or lse.numel() < self.T * self.n_heads
                                or lse.device != c.device):
            raise ValueError(f"lse must be contiguous float32 [{self.T}, {self.n_heads}] on {c.device}")
        if not self._planned:
            raise RuntimeError("plan() has not been called since begin()")
        with _On(c.device):
            lib.dmoe_attention(c.c, layer, self._started(), self.n_heads, self.mask_block, q, self.scale, self._plan, to, lse,
                               self.workspace, stream)
        return out


class AttentionLayer:
    """A layer's attention with its projections, for :func:`.layer.decode_step`:

        out = x + Wo attend(rotate(Wq x), append(rotate(Wk x), Wv x))

    ``w``: wq [n_heads*head_dim, H], wk and wv [n_kv_heads*head_dim, H], wo [H, n_heads*head_dim], of the cache's type.
    The projections are plain matrix products by the library torch calls;
    buffers are allocated here, so a call can be captured.  Layers of one
    step may share ``att`` (its batch and plan)."""

    def __init__(self, att: BlockAttention, layer: int, w: dict):
        c = att.cache
        q, kv = att.n_heads * c.head_dim, c.n_kv_heads * c.head_dim
        H = w["wo"].shape[0]
        for name, shape in (("wq", (q, H)), ("wk", (kv, H)), ("wv", (kv, H)), ("wo", (H, q))):
            if tuple(w[name].shape) != shape or w[name].dtype != c.dtype:
                raise ValueError(f"{name} must be {c.dtype} {list(shape)}, not {w[name].dtype} {list(w[name].shape)}")
        self.att, self.layer, self.w, self.H = att, layer, w, H
        new = lambda n: torch.empty((att.T, n), dtype=c.dtype, device=c.device)  # noqa: E731
        self.q, self.k, self.v = new(q), new(kv), new(kv)
        self.o, self.out = new(q), new(H)

    def __call__(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        """x [T, H] plus its attention (a buffer of this object); rows of no sequence are x's."""
        a, c, w = self.att, self.att.cache, self.w
        if tuple(x.shape) != (a.T, self.H) or x.dtype != c.dtype or x.device != c.device:
            raise ValueError(f"x must be {c.dtype} [{a.T}, {self.H}] on {c.device}, not {x.dtype} {list(x.shape)} on {x.device}")
        _no_gradient(x, "x")
        for name in ("wq", "wk", "wv", "wo"):
            _no_gradient(w[name], name)
        with torch.no_grad(), torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(c.device)):
            torch.mm(x, w["wq"].t(), out=self.q)
            torch.mm(x, w["wk"].t(), out=self.k)
            torch.mm(x, w["wv"].t(), out=self.v)
            q = self.q.view(a.T, a.n_heads, c.head_dim)
            a.append(self.layer, self.k.view(a.T, c.n_kv_heads, c.head_dim), self.v.view(a.T, c.n_kv_heads, c.head_dim), q)
            # rows of no sequence are 0 whichever they are: offsets change from step to step, also under a captured call
            self.o.zero_()
            a.attend(self.layer, q, self.o.view(a.T, a.n_heads, c.head_dim))
            torch.addmm(x, self.o, w["wo"].t(), out=self.out)
        return self.out
