"""Attention of a stream's new tokens over its earlier ones: rotary positions with several axes, a paged
cache of keys and values, and attention over it (include/skipconv.h, the C names; here also torch-facing classes).

A 1 x 1 ``SkipConv`` layer's activation output, N x H x W x (heads * head_dim), viewed as
N*H*W x heads x head_dim, is a tensor of tokens that these calls take as it lies. Work is enqueued on the current torch
stream of the tensors' device; nothing is copied to the host. An object's calls are not thread-safe. ``Rotary.__call__`` runs under
autograd; the other calls record no graph and refuse tensors that require a gradient while gradients are recorded.

    rotary = Rotary(axis_frequencies((11, 11, 10)), head_dim=64)
    cache = PagedCache.empty(pages=256, page_size=64, kv_heads=2, head_dim=64)
    batch = CacheBatch(page_table, row_start, kv_len, max_new=64 * 64)
    q = cache.append(k, v, batch, rotary=rotary, pos=pos, q=q)
    out = cache.attend(q, batch, causal=False)
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import skipconv as _S

SKIPCONV_PAIR_HALVES, SKIPCONV_PAIR_ADJACENT = 0, 1
_PAIRING = {"halves": SKIPCONV_PAIR_HALVES, "adjacent": SKIPCONV_PAIR_ADJACENT}
_DTYPE = {torch.float32: _S.SKIPCONV_F32, torch.bfloat16: _S.SKIPCONV_BF16}
_MOST = 0x7fffffff  # of a description's 32-bit fields, which keep the low bits of what is larger

skipconv_rotary, skipconv_cache = _S.skipconv_rotary, _S.skipconv_cache
skipconv_append, skipconv_attend = _S.skipconv_append, _S.skipconv_attend


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


class PagedCache:
    """Keys and values of earlier tokens in pages.

    k_pages, v_pages: GPU tensors, pages x kv_heads x page_size x head_dim (views of another order are taken as they lie), float32 or
    bfloat16, 16-byte aligned rows; the caller owns them and the page numbers. Other pages take another cache.
    """
    k_pages, v_pages, pages, kv_heads = map(_fixed, ("_k_pages", "_v_pages", "_pages", "_kv_heads"))
    page_size, head_dim, dtype, device = map(_fixed, ("_page_size", "_head_dim", "_dtype", "_device"))

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor):
        _need(k_pages.dim() == 4 and k_pages.is_cuda and k_pages.dtype in _DTYPE, "k_pages must be a 4-d float32 or bfloat16 GPU tensor")
        _need(v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype and v_pages.device == k_pages.device,
              "v_pages must match k_pages in shape, dtype and device")
        _need(k_pages.stride(3) == 1 and v_pages.stride(3) == 1, "the pages' last dimension must be packed")
        self._k_pages, self._v_pages = self._both = k_pages, v_pages
        self._pages, self._kv_heads, self._page_size, self._head_dim = k_pages.shape
        self._dtype, self._device, self._index = k_pages.dtype, k_pages.device, k_pages.get_device()
        c = skipconv_cache()
        c.k_pages, c.v_pages = k_pages.data_ptr(), v_pages.data_ptr()
        c.k_page, c.k_head, c.k_slot = k_pages.stride()[:3]
        c.v_page, c.v_head, c.v_slot = v_pages.stride()[:3]
        c.pages, c.page_size, c.kv_heads, c.head_dim, c.dtype = self._pages, self._page_size, self._kv_heads, self._head_dim, _DTYPE[self._dtype]
        self._c, self._ref = c, ctypes.byref(c)
        lib = _S.lib()
        self._append, self._attend = lib.skipconv_cache_append, lib.skipconv_cache_attend
        self._need = {}  # workspace bytes of attend(), by the shapes that decide them

    @classmethod
    def empty(cls, pages: int, page_size: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, device="cuda") -> "PagedCache":
        """A cache of its own pages (not cleared: no token is read before it is appended)."""
        shape = (pages, kv_heads, page_size, head_dim)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device))

    def desc(self, batch: CacheBatch, tokens: int) -> skipconv_cache:
        """The C description for a batch (the object's own, valid until the next call of it)."""
        if batch._index != self._index:
            raise ValueError("the batch is on another device than the cache")
        c = self._c
        c.page_table, c.row_start, c.kv_len = batch._fields
        c.tokens, c.batch, c.table_width = tokens, batch._sequences, batch._width
        return c

    def append(self, k: torch.Tensor, v: torch.Tensor, batch: CacheBatch, rotary: Optional[Rotary] = None,
               pos: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None):
        """Write the new tokens' keys and values (tokens x kv_heads x head_dim) into the cache, the keys turned by `rotary` at
        `pos` (int32, tokens x axes). With `q` (tokens x heads x head_dim): also returns it turned, in `q_out` (may be q) or a new tensor."""
        dim, dtype, index = self._head_dim, self._dtype, self._index
        tokens, _, kt, kh = _heads_of(k, "k", None, self._kv_heads, dim, dtype, index)
        _, _, vt, vh = _heads_of(v, "v", tokens, self._kv_heads, dim, dtype, index)
        if _recording() and (k.requires_grad or v.requires_grad or self._k_pages.requires_grad or self._v_pages.requires_grad
                             or (q is not None and q.requires_grad) or (q_out is not None and q_out.requires_grad)
                             or (rotary is not None and rotary._freq.requires_grad)):
            _refuse_graph()
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
        _written(self._both)
        _enqueue(self._append, index, self._ref, ctypes.byref(a))
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
        if _recording() and (q.requires_grad or self._k_pages.requires_grad or self._v_pages.requires_grad
                             or (out is not None and out.requires_grad)):
            _refuse_graph()
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
            need = skipconv_attend_workspace(c, a)
            if len(self._need) < 4096:
                self._need[shapes] = need
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        _enqueue(self._attend, index, self._ref, ctypes.byref(a), ws.data_ptr() if need else None, need)
        return (out, lse) if return_lse else out
