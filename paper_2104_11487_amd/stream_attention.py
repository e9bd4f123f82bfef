"""Attention of a stream's new tokens over its earlier ones: rotary positions with several axes, a paged cache of keys and values (in the
tokens' type or in 4 bits), attention over it, and eviction by the attention that tokens received (include/skipconv.h, the C names; here
also torch-facing classes).

A 1 x 1 ``SkipConv`` layer's activation output, N x H x W x (heads * head_dim), viewed as
N*H*W x heads x head_dim, is a tensor of tokens that these calls take as it lies. Work is enqueued on the current torch
stream of the tensors' device; nothing is copied to the host. An object's calls are not thread-safe. ``Rotary.__call__`` runs under
autograd; the other calls record no graph and refuse tensors that require a gradient while gradients are recorded, or that carry a tangent.

    rotary = Rotary(axis_frequencies((11, 11, 10)), head_dim=64)
    cache = PagedCache.empty(pages=256, page_size=64, kv_heads=2, head_dim=64)
    batch = CacheBatch(page_table, row_start, kv_len, max_new=64 * 64)
    q = cache.append(k, v, batch, rotary=rotary, pos=pos, q=q)
    out = cache.attend(q, batch, causal=False)

A long stream's cache is a PackedCache, in 4 bits, and is kept short by eviction. A batch's kv_len counts its new tokens, so they are added to
the lengths that an eviction leaves, and the pages that it moves tokens to need room for them too:

    new = 64 * 64  # tokens of a frame; 4096 earlier ones are kept
    cache = PackedCache.empty(pages=256, page_size=64, kv_heads=2, head_dim=64)
    here, there = torch.arange(256, dtype=torch.int32, device="cuda").view(2, 1, 128)  # one sequence's pages, in turn: 128 hold 4096 + new tokens
    row_start = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    lengths = torch.zeros(1, dtype=torch.int32, device="cuda")
    weights = torch.empty(256, 2, 64, device="cuda")  # float32, pages x kv_heads x page_size
    for q, k, v, pos in frames:
        batch = CacheBatch(here, row_start, lengths + new, max_new=new)
        q = cache.append(k, v, batch, rotary=rotary, pos=pos, q=q)
        out, lse = cache.attend(q, batch, causal=False, return_lse=True)
        cache.weigh(q, lse, batch, weights, causal=False)
        lengths, kept = cache.evict(weights, batch, there, keep=4096, recent=256)
        here, there = there, here
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch
import torch.autograd.forward_ad as _forward

from . import skipconv as _S

SKIPCONV_PAIR_HALVES, SKIPCONV_PAIR_ADJACENT = 0, 1
_PAIRING = {"halves": SKIPCONV_PAIR_HALVES, "adjacent": SKIPCONV_PAIR_ADJACENT}
_DTYPE = {torch.float32: _S.SKIPCONV_F32, torch.bfloat16: _S.SKIPCONV_BF16}
_MOST = 0x7fffffff  # of a description's 32-bit fields, which keep the low bits of what is larger

skipconv_rotary, skipconv_cache = _S.skipconv_rotary, _S.skipconv_cache
skipconv_append, skipconv_attend = _S.skipconv_append, _S.skipconv_attend
skipconv_packing, skipconv_weigh, skipconv_evict = _S.skipconv_packing, _S.skipconv_weigh, _S.skipconv_evict


# ------------------------------------------------------------------ C names --

def skipconv_rotate(r: skipconv_rotary, tokens: int, heads: int, head_dim: int, dtype: int, x_ptr: int, x_token: int, x_head: int,
                    y_ptr: int, y_token: int, y_head: int, stream: int) -> None:
    _S._check(_S.lib().skipconv_rotate(ctypes.byref(r), tokens, heads, head_dim, dtype, x_ptr, x_token, x_head, y_ptr, y_token,
                                       y_head, stream))


def skipconv_cache_append(c: skipconv_cache, a: skipconv_append, stream: int) -> None:
    _S._check(_S.lib().skipconv_cache_append(ctypes.byref(c), ctypes.byref(a), stream))


def skipconv_attend_workspace(c: skipconv_cache, a: skipconv_attend) -> int:
    n = ctypes.c_size_t()
    _S._check(_S.lib().skipconv_attend_workspace(ctypes.byref(c), ctypes.byref(a), ctypes.byref(n)))
    return n.value


def skipconv_cache_attend(c: skipconv_cache, a: skipconv_attend, workspace_ptr: Optional[int], workspace_bytes: int, stream: int) -> None:
    _S._check(_S.lib().skipconv_cache_attend(ctypes.byref(c), ctypes.byref(a), workspace_ptr, workspace_bytes, stream))


def skipconv_packed_append(c: skipconv_cache, s: skipconv_packing, a: skipconv_append, stream: int) -> None:
    _S._check(_S.lib().skipconv_packed_append(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a), stream))


def skipconv_packed_attend_workspace(c: skipconv_cache, a: skipconv_attend) -> int:
    n = ctypes.c_size_t()
    _S._check(_S.lib().skipconv_packed_attend_workspace(ctypes.byref(c), ctypes.byref(a), ctypes.byref(n)))
    return n.value


def skipconv_packed_attend(c: skipconv_cache, s: skipconv_packing, a: skipconv_attend, workspace_ptr: Optional[int], workspace_bytes: int,
                           stream: int) -> None:
    _S._check(_S.lib().skipconv_packed_attend(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a), workspace_ptr, workspace_bytes, stream))


def skipconv_packed_unpack(c: skipconv_cache, s: skipconv_packing, list_ptr: int, count: int, k_ptr: int, v_ptr: int, stream: int) -> None:
    _S._check(_S.lib().skipconv_packed_unpack(ctypes.byref(c), ctypes.byref(s), list_ptr, count, k_ptr, v_ptr, stream))


def skipconv_cache_weigh(c: skipconv_cache, s: Optional[skipconv_packing], w: skipconv_weigh, stream: int) -> None:
    _S._check(_S.lib().skipconv_cache_weigh(ctypes.byref(c), None if s is None else ctypes.byref(s), ctypes.byref(w), stream))


def skipconv_cache_evict(c: skipconv_cache, s: Optional[skipconv_packing], e: skipconv_evict, stream: int) -> None:
    _S._check(_S.lib().skipconv_cache_evict(ctypes.byref(c), None if s is None else ctypes.byref(s), ctypes.byref(e), stream))


# ------------------------------------------------------------ torch classes --

def axis_frequencies(pairs: Sequence[int], base: float = 10000.0, device="cuda") -> torch.Tensor:
    """A table axes x sum(pairs) for ``Rotary``: axis a turns the next pairs[a] pairs, with
    frequencies base ** (-i / pairs[a])."""
    table = torch.zeros(len(pairs), sum(pairs), dtype=torch.float64)
    at = 0
    for a, n in enumerate(pairs):
        table[a, at:at + n] = base ** (-torch.arange(n, dtype=torch.float64) / max(n, 1))
        at += n
    return table.float().to(device)


def _need(ok: bool, message: str) -> None:
    if not ok:
        raise ValueError(message)


# The current stream's handle of a device (by index), without a Stream object around it; the current device's index.
_stream = torch._C._cuda_getCurrentRawStream
_current = torch._C._cuda_getDevice


def _enqueue(call, index: int, *args) -> None:
    """The call with the device's current stream as its last argument. That device is the current one meanwhile: a handle does not
    say which device it belongs to (a default stream's is 0 on each)."""
    if _current() == index:
        rc = call(*args, _stream(index))
    else:
        with torch.cuda.device(index):
            rc = call(*args, _stream(index))
    if rc:
        _S._check(rc)


def _refuse(x, name: str, tokens, heads, dim, dtype, index: int):
    want = ["tokens" if tokens is None else tokens, "heads" if heads is None else heads, dim]
    raise ValueError(f"{name} must be a {dtype} tensor {want} on GPU {index} with a packed last dimension; "
                     f"got {x.dtype} {list(x.shape)} with strides {x.stride()} on {x.device}")


def _heads_of(x: torch.Tensor, name: str, tokens: Optional[int], heads: Optional[int], dim: int, dtype, index: int):
    """Checks a tensor of heads; returns its tokens, heads and their strides."""
    shape = x.shape
    if len(shape) != 3:
        _refuse(x, name, tokens, heads, dim, dtype, index)
    t, h, d = shape
    st, sh, sd = x.stride()
    if d != dim or (tokens is not None and t != tokens) or (heads is not None and h != heads) or x.dtype is not dtype \
            or x.get_device() != index or (sd != 1 and x.numel() > 0):
        _refuse(x, name, tokens, heads, dim, dtype, index)
    return t, h, st, sh


# Whether gradients are recorded; what a kernel wrote, for autograd's check of the tensors that it saved.
_recording = torch.is_grad_enabled
_written = torch._C._increment_version


def _refuse_graph():
    raise ValueError("this call records no gradient, and a tensor of it requires one: call it under torch.no_grad(), or rotate by "
                     "calling the Rotary itself")


def _refuse_tangents(*tensors) -> None:
    """Forward-mode tangents, which torch.no_grad() leaves on: no call computes one. To be asked where a level of them is open."""
    for t in tensors:
        if t is not None and _forward.unpack_dual(t).tangent is not None:
            raise ValueError("this call computes no forward-mode gradient, and a tensor of it carries a tangent")


def _fixed(name: str) -> property:
    """What a description took at construction: to be read, not replaced (the description would keep the address of a tensor that is gone)."""
    return property(lambda self: getattr(self, name))


def _like(x: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(x, memory_format=torch.contiguous_format)


class Rotary:
    """Rotary positions with several axes.

    freq: float32 GPU tensor, axes x pairs: token t's pair j turns by the sum over the axes a of pos[t, a] * freq[a, j].
    pairing: "halves" (elements j and j + pairs of a head) or "adjacent" (2 j and 2 j + 1); elements past 2 * pairs stay.
    pos is an int32 GPU tensor, tokens x axes; x is tokens x heads x head_dim, float32 or bfloat16, of any strides with a packed
    last dimension. The table's values may change between calls, the tensor may not.
    """
    freq, axes, pairs, head_dim, pairing, device = map(_fixed, ("_freq", "_axes", "_pairs", "_head_dim", "_pairing", "_device"))

    def __init__(self, freq: torch.Tensor, head_dim: int, pairing: str = "halves"):
        _need(freq.is_cuda and freq.dtype == torch.float32 and freq.dim() == 2, "freq must be a float32 GPU tensor, axes x pairs")
        _need(pairing in _PAIRING, "pairing must be 'halves' or 'adjacent'")
        self._freq = freq.contiguous()
        self._axes, self._pairs = self._freq.shape
        _need(1 <= self._axes <= 8 and 1 <= self._pairs <= head_dim // 2, "freq must have 1..8 axes and 1..head_dim / 2 pairs")
        self._head_dim, self._pairing, self._device = head_dim, pairing, freq.device
        self._index = freq.get_device()
        self._desc = [skipconv_rotary(None, self._freq.data_ptr(), self._axes, self._pairs, _PAIRING[pairing], i) for i in (0, 1)]
        self._ref = [ctypes.byref(d) for d in self._desc]
        self._pointer = ctypes.pointer(self._desc[0])
        self._call = _S.lib().skipconv_rotate

    def desc(self, pos: torch.Tensor, tokens: int, inverse: bool = False) -> skipconv_rotary:
        """The C description for these positions (the object's own, valid until the next call of it)."""
        if pos.dtype is not torch.int32 or pos.get_device() != self._index or pos.shape != (tokens, self._axes) or not pos.is_contiguous():
            raise ValueError(f"pos must be a contiguous int32 tensor {[tokens, self._axes]} on {self._device}")
        d = self._desc[inverse]
        d.pos = pos.data_ptr()
        return d

    def rotate(self, x: torch.Tensor, pos: torch.Tensor, out: Optional[torch.Tensor] = None, inverse: bool = False) -> torch.Tensor:
        """x turned by its tokens' positions, into `out` (which may be x itself) or a new tensor."""
        dtype = x.dtype
        code = _DTYPE.get(dtype)
        if code is None:
            raise ValueError("x must be float32 or bfloat16")
        dim, index = self._head_dim, self._index
        tokens, heads, xt, xh = _heads_of(x, "x", None, None, dim, dtype, index)
        if _recording() and (x.requires_grad or self._freq.requires_grad or (out is not None and out.requires_grad)):
            _refuse_graph()
        if _forward._current_level >= 0:
            _refuse_tangents(x, self._freq, out)
        inverse = 1 if inverse else 0
        self.desc(pos, tokens, inverse)
        if out is None:
            out = _like(x)
            yt, yh = heads * dim, dim
        else:
            _, _, yt, yh = _heads_of(out, "out", tokens, heads, dim, dtype, index)
            _written((out,))
        _enqueue(self._call, index, self._ref[inverse], tokens, heads, dim, code, x.data_ptr(), xt, xh, out.data_ptr(), yt, yh)
        return out

    def backward(self, grad: torch.Tensor, pos: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The gradient of x from that of rotate(x, pos): the rotation is orthogonal, so it turns back."""
        return self.rotate(grad, pos, out, inverse=True)

    def __call__(self, x: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
        """rotate() under autograd: the gradient of x. The table has none."""
        if _recording() and self._freq.requires_grad:
            _refuse_graph()
        return _RotaryFunction.apply(x, pos, self._freq, self)


class _RotaryFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, freq, rotary):
        ctx.rotary = rotary
        # the table too, so that one that changed in the meantime is refused (one made under inference mode cannot be saved)
        ctx.save_for_backward(pos, None if freq.is_inference() else freq)
        return rotary.rotate(x, pos)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        if grad.stride(2) != 1:  # a broadcast gradient, such as a sum's
            grad = grad.contiguous()
        pos, _ = ctx.saved_tensors
        return ctx.rotary.backward(grad, pos), None, None, None


class CacheBatch:
    """Where the new tokens of a batch of sequences lie in a cache (int32 GPU tensors, read on the device by every call).

    page_table: sequences x width page numbers; row_start: sequences + 1, the first row of each sequence in the new
    tokens' tensors; kv_len: tokens of each sequence in the cache, the new ones included. max_new: the most new tokens that
    a sequence has, where the program knows it (it selects the kernel; the results are right whatever it is, though kernels differ in
    rounding). The tensors' values may change between calls, the tensors may not: others take another batch.
    """
    page_table, row_start, kv_len, sequences, device = map(_fixed, ("_page_table", "_row_start", "_kv_len", "_sequences", "_device"))

    def __init__(self, page_table: torch.Tensor, row_start: torch.Tensor, kv_len: torch.Tensor, max_new: int = 0):
        n, device = kv_len.shape[0], kv_len.device
        for t, name, shape in ((page_table, "page_table", (n, page_table.shape[-1])), (row_start, "row_start", (n + 1,)), (kv_len, "kv_len", (n,))):
            if t.dtype != torch.int32 or not t.is_cuda or t.device != device or tuple(t.shape) != shape or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on one GPU")
        _need(max_new >= 0, "max_new must be >= 0")
        self._page_table, self._row_start, self._kv_len, self.max_new = page_table, row_start, kv_len, min(int(max_new), _MOST)
        self._sequences, self._device = n, device
        self._index = kv_len.get_device()
        # what a description of the cache takes from here
        self._fields = (page_table.data_ptr(), row_start.data_ptr(), kv_len.data_ptr())
        self._width = page_table.shape[1]


class _Cache:
    """What the caches share: descriptions, and the calls on them. A subclass sets the pages' tensors and the library's functions."""
    pages, kv_heads, page_size, head_dim = map(_fixed, ("_pages", "_kv_heads", "_page_size", "_head_dim"))
    dtype, device = map(_fixed, ("_dtype", "_device"))

    def _describe(self, k: torch.Tensor, v: torch.Tensor, tensors, packing, append, attend, workspace):
        """k, v: what the C description's pages are; tensors: all that a call may write; packing: a reference to the C packing, or None."""
        self._tensors = tensors
        self._first, self._second, self._more = tensors[0], tensors[1], tensors[2:]
        c = skipconv_cache()
        c.k_pages, c.v_pages = k.data_ptr(), v.data_ptr()
        c.k_page, c.k_head, c.k_slot = k.stride()[:3]
        c.v_page, c.v_head, c.v_slot = v.stride()[:3]
        c.pages, c.page_size, c.kv_heads, c.head_dim, c.dtype = self._pages, self._page_size, self._kv_heads, self._head_dim, _DTYPE[self._dtype]
        self._c, self._ref, self._packing = c, ctypes.byref(c), packing
        self._refs = (self._ref,) if packing is None else (self._ref, packing)
        lib = _S.lib()
        self._append, self._attend, self._weigh, self._evict = append, attend, lib.skipconv_cache_weigh, lib.skipconv_cache_evict
        self._workspace = workspace
        self._need = {}  # workspace bytes of attend(), by the shapes that decide them

    def desc(self, batch: CacheBatch, tokens: int) -> skipconv_cache:
        """The C description for a batch (the object's own, valid until the next call of it)."""
        if batch._index != self._index:
            raise ValueError("the batch is on another device than the cache")
        c = self._c
        c.page_table, c.row_start, c.kv_len = batch._fields
        c.tokens, c.batch, c.table_width = tokens, batch._sequences, batch._width
        return c

    def _graph(self, *tensors) -> bool:
        """Whether gradients are recorded and one of these tensors, or of the pages, requires one. Tangents are refused at once."""
        if _forward._current_level >= 0:
            _refuse_tangents(*tensors, *self._tensors)
        if not _recording():
            return False
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
        for t in self._tensors:
            if t.requires_grad:
                return True
        return False

    def append(self, k: torch.Tensor, v: torch.Tensor, batch: CacheBatch, rotary: Optional[Rotary] = None,
               pos: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None):
        """Write the new tokens' keys and values (tokens x kv_heads x head_dim) into the cache, the keys turned by `rotary` at
        `pos` (int32, tokens x axes). With `q` (tokens x heads x head_dim): also returns it turned, in `q_out` (may be q) or a new tensor."""
        dim, dtype, index = self._head_dim, self._dtype, self._index
        tokens, _, kt, kh = _heads_of(k, "k", None, self._kv_heads, dim, dtype, index)
        _, _, vt, vh = _heads_of(v, "v", tokens, self._kv_heads, dim, dtype, index)
        # (in line, as attend()'s: these are the calls whose time on the host a stream's step is made of)
        if _recording() and (k.requires_grad or v.requires_grad or self._first.requires_grad or self._second.requires_grad
                             or (q is not None and q.requires_grad) or (q_out is not None and q_out.requires_grad)
                             or (rotary is not None and rotary._freq.requires_grad) or (self._more and self._graph())):
            _refuse_graph()
        if _forward._current_level >= 0:
            _refuse_tangents(k, v, q, q_out, None if rotary is None else rotary._freq, *self._tensors)
        a = skipconv_append(k.data_ptr(), v.data_ptr(), None, None, kt, kh, vt, vh)
        if rotary is not None:
            if pos is None or rotary._head_dim != dim:
                raise ValueError("a rotation needs pos and the cache's head_dim")
            if rotary._index != index:
                raise ValueError("the rotation is on another device than the cache")
            rotary.desc(pos, tokens, 0)
            a.rotary = rotary._pointer
        if q is not None:
            if rotary is None:
                raise ValueError("queries are only turned: pass rotary and pos")
            _, heads, a.q_token, a.q_head = _heads_of(q, "q", tokens, None, dim, dtype, index)
            if q_out is None:
                q_out = _like(q)
                a.q_out_token, a.q_out_head = heads * dim, dim
            else:
                _, _, a.q_out_token, a.q_out_head = _heads_of(q_out, "q_out", tokens, heads, dim, dtype, index)
                _written((q_out,))
            a.q, a.q_out, a.q_heads = q.data_ptr(), q_out.data_ptr(), heads
        elif q_out is not None:
            raise ValueError("q_out without q")
        self.desc(batch, tokens)
        _written(self._tensors)
        _enqueue(self._append, index, *self._refs, ctypes.byref(a))
        return q_out

    def attend(self, q: torch.Tensor, batch: CacheBatch, causal: bool = True, window: int = -1, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None, return_lse: bool = False):
        """Attention of the new tokens' queries (tokens x heads x head_dim, heads a multiple of kv_heads) over the cache.

        causal: a token sees those up to itself, and `window` of those before it (-1: all); otherwise it sees its whole
        sequence and `window` of the tokens before the new ones. scale: head_dim ** -0.5 by default. Returns
        tokens x heads x head_dim (zeros for a row that sees nothing), with return_lse also the float32 log of the
        sum of exponentials, tokens x heads (-inf there). Rows of no sequence are not written.
        """
        dim, dtype, index = self._head_dim, self._dtype, self._index
        tokens, heads, qt, qh = _heads_of(q, "q", None, None, dim, dtype, index)
        if _recording() and (q.requires_grad or self._first.requires_grad or self._second.requires_grad or (out is not None and out.requires_grad)
                             or (self._more and self._graph())):
            _refuse_graph()
        if _forward._current_level >= 0:
            _refuse_tangents(q, out, *self._tensors)
        if out is None:
            out = _like(q)
            ot, oh = heads * dim, dim
        else:
            _, _, ot, oh = _heads_of(out, "out", tokens, heads, dim, dtype, index)
            _written((out,))
        window = -1 if window < 0 else min(window, _MOST)  # no sequence is as long as that
        lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device) if return_lse else None
        a = skipconv_attend(q.data_ptr(), out.data_ptr(), lse.data_ptr() if return_lse else None, qt, qh, ot, oh, heads, 1 if causal else 0,
                            window, dim ** -0.5 if scale is None else scale, batch.max_new)
        c = self.desc(batch, tokens)
        shapes = (tokens, heads, batch._sequences, batch._width, window, batch.max_new)
        need = self._need.get(shapes)
        if need is None:
            need = self._workspace(c, a)
            if len(self._need) < 4096:
                self._need[shapes] = need
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        _enqueue(self._attend, index, *self._refs, ctypes.byref(a), ws.data_ptr() if need else None, need)
        return (out, lse) if return_lse else out

    def _weights(self, weights: torch.Tensor) -> None:
        shape = (self._pages, self._kv_heads, self._page_size)
        if weights.dtype is not torch.float32 or weights.get_device() != self._index or weights.shape != shape or not weights.is_contiguous():
            raise ValueError(f"weights must be a contiguous float32 tensor {list(shape)} on {self._device}")

    def weigh(self, q: torch.Tensor, lse: torch.Tensor, batch: CacheBatch, weights: torch.Tensor, causal: bool = True, window: int = -1,
              scale: Optional[float] = None, decay: float = 1.0) -> torch.Tensor:
        """Adds the attention weight that each cached token received from the new tokens' queries to `weights` (float32, pages x kv_heads x
        page_size), and returns it: decay times what it held, plus the sum over the query heads and the new tokens that see it of exp(score - lse);
        a new token's own is set, so its slot needs no clearing. q, lse: what attend() took, and returned with return_lse; the mask and the
        scale as there. A row whose lse is -inf gives nothing. Tokens of sequences without new ones stay as they are; sequences with new ones must not share slots.
        """
        dim, dtype, index = self._head_dim, self._dtype, self._index
        tokens, heads, qt, qh = _heads_of(q, "q", None, None, dim, dtype, index)
        if lse.dtype is not torch.float32 or lse.get_device() != index or lse.shape != (tokens, heads) or not lse.is_contiguous():
            raise ValueError(f"lse must be a contiguous float32 tensor {[tokens, heads]} on {self._device}")
        self._weights(weights)
        if self._graph(q, lse, weights):
            _refuse_graph()
        w = skipconv_weigh(q.data_ptr(), lse.data_ptr(), weights.data_ptr(), qt, qh, heads, 1 if causal else 0,
                           -1 if window < 0 else min(window, _MOST), dim ** -0.5 if scale is None else scale, decay, batch.max_new)
        self.desc(batch, tokens)
        _written((weights,))
        _enqueue(self._weigh, index, self._ref, self._packing, ctypes.byref(w))
        return weights

    def evict(self, weights: torch.Tensor, batch: CacheBatch, into: torch.Tensor, keep: int, recent: int = 0):
        """Keeps min(kv_len, keep) tokens of each sequence, for each key head its own: the last `recent` ones, and of the others those of
        the largest weights (of equal ones the earlier). In their order they become the tokens of the sequence in the pages of `into`
        (int32, sequences x width): keys, values and weights. These pages must be different ones, and hold no token of the batch.
        Returns (lengths, kept): int32, the tokens of each sequence now, and their earlier positions, sequences x kv_heads x keep, -1 past
        the last. The next tokens come behind them: CacheBatch(into, row_start, lengths + new), where new counts each sequence's new tokens (a batch's
        kv_len holds them), for which `into` needs room too; with kv_len = lengths they would take the places of the last ones kept.
        """
        index = self._index
        self._weights(weights)
        _need(1 <= keep <= _MOST and 0 <= recent <= keep, "keep must be >= 1, and recent 0..keep")
        n = batch._sequences
        if into.dtype is not torch.int32 or into.get_device() != index or into.dim() != 2 or into.shape[0] != n or not into.is_contiguous():
            raise ValueError(f"into must be a contiguous int32 tensor [{n}, width] on {self._device}")
        if self._graph(weights):
            _refuse_graph()
        lengths = torch.empty(n, dtype=torch.int32, device=into.device)
        kept = torch.empty((n, self._kv_heads, keep), dtype=torch.int32, device=into.device)
        e = skipconv_evict(weights.data_ptr(), into.data_ptr(), lengths.data_ptr(), kept.data_ptr(), into.shape[1], keep, recent)
        self.desc(batch, 0)
        _written((*self._tensors, weights))
        _enqueue(self._evict, index, self._ref, self._packing, ctypes.byref(e))
        return lengths, kept


class PagedCache(_Cache):
    """Keys and values of earlier tokens in pages.

    k_pages, v_pages: GPU tensors, pages x kv_heads x page_size x head_dim (views of another order are taken as they lie), float32 or
    bfloat16, 16-byte aligned rows; the caller owns them and the page numbers. Other pages take another cache.
    """
    k_pages, v_pages = map(_fixed, ("_k_pages", "_v_pages"))

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor):
        _need(k_pages.dim() == 4 and k_pages.is_cuda and k_pages.dtype in _DTYPE, "k_pages must be a 4-d float32 or bfloat16 GPU tensor")
        _need(v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype and v_pages.device == k_pages.device,
              "v_pages must match k_pages in shape, dtype and device")
        _need(k_pages.stride(3) == 1 and v_pages.stride(3) == 1, "the pages' last dimension must be packed")
        self._k_pages, self._v_pages = k_pages, v_pages
        self._pages, self._kv_heads, self._page_size, self._head_dim = k_pages.shape
        self._dtype, self._device, self._index = k_pages.dtype, k_pages.device, k_pages.get_device()
        lib = _S.lib()
        self._describe(k_pages, v_pages, (k_pages, v_pages), None, lib.skipconv_cache_append, lib.skipconv_cache_attend, skipconv_attend_workspace)

    @classmethod
    def empty(cls, pages: int, page_size: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, device="cuda") -> "PagedCache":
        """A cache of its own pages (not cleared: no token is read before it is appended)."""
        shape = (pages, kv_heads, page_size, head_dim)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device))


class PackedCache(_Cache):
    """A PagedCache in 4 bits: a third of the bytes, the same calls.

    k_codes, v_codes: uint8 GPU tensors, pages x kv_heads x page_size x 16 * groups, where groups = ceil(head_dim / 32); k_scales, v_scales:
    float16, pages x kv_heads x page_size x groups x 2 (views of another order are taken as they lie). Element e of a row is in the lower
    (e even) or upper half of byte e // 2; with (scale, minimum) of its group of 32 elements, a code stands for minimum + code * scale,
    rounded to float16. dtype: of the new tokens and queries. Elements are held between -32768 and 32768; one that is
    not finite makes its group NaN.
    """
    k_codes, v_codes, k_scales, v_scales = map(_fixed, ("_k_codes", "_v_codes", "_k_scales", "_v_scales"))

    def __init__(self, k_codes: torch.Tensor, v_codes: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor, head_dim: int,
                 dtype=torch.bfloat16):
        _need(dtype in _DTYPE, "dtype must be float32 or bfloat16")
        _need(head_dim >= 1, "head_dim must be >= 1")
        groups = -(-head_dim // 32)
        for x, name in ((k_codes, "k_codes"), (v_codes, "v_codes")):
            _need(x.dim() == 4 and x.is_cuda and x.dtype == torch.uint8 and x.shape[3] == 16 * groups and x.stride(3) == 1,
                  f"{name} must be a uint8 GPU tensor, pages x kv_heads x page_size x {16 * groups}, with a packed last dimension")
        _need(v_codes.shape == k_codes.shape and v_codes.device == k_codes.device, "v_codes must match k_codes in shape and device")
        for x, name in ((k_scales, "k_scales"), (v_scales, "v_scales")):
            _need(x.dtype == torch.float16 and x.device == k_codes.device and tuple(x.shape) == (*k_codes.shape[:3], groups, 2)
                  and x.stride(4) == 1 and (groups == 1 or x.stride(3) == 2),
                  f"{name} must be a float16 tensor {[*k_codes.shape[:3], groups, 2]} on the codes' device, its last two dimensions packed")
        self._k_codes, self._v_codes, self._k_scales, self._v_scales = k_codes, v_codes, k_scales, v_scales
        self._pages, self._kv_heads, self._page_size = k_codes.shape[:3]
        self._head_dim, self._dtype = head_dim, dtype
        self._device, self._index = k_codes.device, k_codes.get_device()
        self._scales = skipconv_packing(k_scales.data_ptr(), v_scales.data_ptr(), *k_scales.stride()[:3], *v_scales.stride()[:3])
        lib = _S.lib()
        self._describe(k_codes, v_codes, (k_codes, v_codes, k_scales, v_scales), ctypes.byref(self._scales), lib.skipconv_packed_append,
                       lib.skipconv_packed_attend, skipconv_packed_attend_workspace)

    @classmethod
    def empty(cls, pages: int, page_size: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, device="cuda") -> "PackedCache":
        """A cache of its own pages (not cleared: no token is read before it is appended)."""
        shape, groups = (pages, kv_heads, page_size), -(-head_dim // 32)
        codes = [torch.empty((*shape, 16 * groups), dtype=torch.uint8, device=device) for _ in range(2)]
        scales = [torch.empty((*shape, groups, 2), dtype=torch.float16, device=device) for _ in range(2)]
        return cls(*codes, *scales, head_dim, dtype)

    def unpack(self, pages: torch.Tensor):
        """The values of the pages whose numbers an int32 GPU tensor of any shape holds (a page table, say), exactly: (k, v), float16, the
        shape x kv_heads x page_size x head_dim. Zeros for a number outside the cache."""
        index = self._index
        if pages.dtype is not torch.int32 or pages.get_device() != index or not pages.is_contiguous():
            raise ValueError(f"pages must be a contiguous int32 tensor on {self._device}")
        if self._graph():
            _refuse_graph()
        k, v = (torch.empty((*pages.shape, self._kv_heads, self._page_size, self._head_dim), dtype=torch.float16, device=pages.device) for _ in range(2))
        _enqueue(_S.lib().skipconv_packed_unpack, index, *self._refs, pages.data_ptr(), pages.numel(), k.data_ptr(), v.data_ptr())
        return k, v
