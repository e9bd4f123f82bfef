"""Attention of a stream's new tokens over its earlier ones: rotary positions with several axes, a paged
cache of keys and values, and attention over it (include/skipconv.h, the C names; here also torch-facing classes).

A 1 x 1 ``SkipConv`` layer's activation output, N x H x W x (heads * head_dim), viewed as
N*H*W x heads x head_dim, is a tensor of tokens that these calls take as it lies. Work is enqueued on the current torch
stream of the tensors' device; nothing is copied to the host.

    rotary = Rotary(axis_frequencies((11, 11, 10)), head_dim=64)
    cache = PagedCache.empty(pages=256, page_size=64, kv_heads=2, head_dim=64)
    batch = CacheBatch(page_table, row_start, kv_len, max_new=64 * 64)
    q = cache.append(k, v, batch, rotary=rotary, pos=pos, q=q)
    out = cache.attend(q, batch, causal=False)
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence

import torch

from . import skipconv as _S

SKIPCONV_PAIR_HALVES, SKIPCONV_PAIR_ADJACENT = 0, 1
_PAIRING = {"halves": SKIPCONV_PAIR_HALVES, "adjacent": SKIPCONV_PAIR_ADJACENT}
_DTYPE = {torch.float32: _S.SKIPCONV_F32, torch.bfloat16: _S.SKIPCONV_BF16}

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


def _stream(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _heads_of(x: torch.Tensor, name: str, tokens: Optional[int], heads: Optional[int], dim: int, dtype, device) -> None:
    s = x.shape
    if len(s) != 3 or s[2] != dim or (tokens is not None and s[0] != tokens) or (heads is not None and s[1] != heads) \
            or x.dtype != dtype or x.device != device or (x.stride(2) != 1 and x.numel() > 0):
        want = ["tokens" if tokens is None else tokens, "heads" if heads is None else heads, dim]
        raise ValueError(f"{name} must be a {dtype} tensor {want} on {device} with a packed last dimension")


class Rotary:
    """Rotary positions with several axes.

    freq: float32 GPU tensor, axes x pairs: token t's pair j turns by the sum over the axes a of pos[t, a] * freq[a, j].
    pairing: "halves" (elements j and j + pairs of a head) or "adjacent" (2 j and 2 j + 1); elements past 2 * pairs stay.
    pos is an int32 GPU tensor, tokens x axes; x is tokens x heads x head_dim, float32 or bfloat16, of any strides with a packed
    last dimension.
    """

    def __init__(self, freq: torch.Tensor, head_dim: int, pairing: str = "halves"):
        _need(freq.is_cuda and freq.dtype == torch.float32 and freq.dim() == 2, "freq must be a float32 GPU tensor, axes x pairs")
        _need(pairing in _PAIRING, "pairing must be 'halves' or 'adjacent'")
        self.freq = freq.contiguous()
        self.axes, self.pairs = self.freq.shape
        _need(1 <= self.axes <= 8 and 1 <= self.pairs <= head_dim // 2, "freq must have 1..8 axes and 1..head_dim / 2 pairs")
        self.head_dim, self.pairing, self.device = head_dim, pairing, freq.device
        self._desc = [skipconv_rotary(None, self.freq.data_ptr(), self.axes, self.pairs, _PAIRING[pairing], i) for i in (0, 1)]

    def desc(self, pos: torch.Tensor, tokens: int, inverse: bool = False) -> skipconv_rotary:
        """The C description for these positions."""
        if pos.dtype != torch.int32 or pos.device != self.device or tuple(pos.shape) != (tokens, self.axes) or not pos.is_contiguous():
            raise ValueError(f"pos must be a contiguous int32 tensor {[tokens, self.axes]} on {self.device}")
        d = self._desc[bool(inverse)]
        d.pos = pos.data_ptr()
        return d

    def rotate(self, x: torch.Tensor, pos: torch.Tensor, out: Optional[torch.Tensor] = None, inverse: bool = False) -> torch.Tensor:
        """x turned by its tokens' positions, into `out` (which may be x itself) or a new tensor."""
        _need(x.dtype in _DTYPE, "x must be float32 or bfloat16")
        _heads_of(x, "x", None, None, self.head_dim, x.dtype, self.device)
        tokens, heads, dim = x.shape
        if out is None:
            out = torch.empty((tokens, heads, dim), dtype=x.dtype, device=x.device)
        elif out is not x:
            _heads_of(out, "out", tokens, heads, dim, x.dtype, x.device)
        skipconv_rotate(self.desc(pos, tokens, inverse), tokens, heads, dim, _DTYPE[x.dtype], x.data_ptr(), x.stride(0), x.stride(1),
                        out.data_ptr(), out.stride(0), out.stride(1), _stream(x.device))
        return out

    def backward(self, grad: torch.Tensor, pos: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The gradient of x from that of rotate(x, pos): the rotation is orthogonal, so it turns back."""
        return self.rotate(grad, pos, out, inverse=True)

    def __call__(self, x: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
        """rotate() under autograd."""
        return _RotaryFunction.apply(x, pos, self)


class _RotaryFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, rotary):
        ctx.rotary = rotary
        ctx.save_for_backward(pos)
        return rotary.rotate(x, pos)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        if grad.stride(2) != 1:  # a broadcast gradient, such as a sum's
            grad = grad.contiguous()
        return ctx.rotary.backward(grad, ctx.saved_tensors[0]), None, None


class CacheBatch:
    """Where the new tokens of a batch of sequences lie in a cache (int32 GPU tensors, read on the device by every call).

    page_table: sequences x width page numbers; row_start: sequences + 1, the first row of each sequence in the new
    tokens' tensors; kv_len: tokens of each sequence in the cache, the new ones included. max_new: the most new tokens that
    a sequence has, where the program knows it (it selects the kernel; the results do not depend on it).
    """

    def __init__(self, page_table: torch.Tensor, row_start: torch.Tensor, kv_len: torch.Tensor, max_new: int = 0):
        n, device = kv_len.shape[0], kv_len.device
        for t, name, shape in ((page_table, "page_table", (n, page_table.shape[-1])), (row_start, "row_start", (n + 1,)), (kv_len, "kv_len", (n,))):
            if t.dtype != torch.int32 or not t.is_cuda or t.device != device or tuple(t.shape) != shape or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on one GPU")
        _need(max_new >= 0, "max_new must be >= 0")
        self.page_table, self.row_start, self.kv_len, self.max_new = page_table, row_start, kv_len, int(max_new)
        self.sequences, self.device = n, device


class PagedCache:
    """Keys and values of earlier tokens in pages.

    k_pages, v_pages: GPU tensors, pages x kv_heads x page_size x head_dim (views of another order are taken as they lie), float32 or
    bfloat16, 16-byte aligned rows; the caller owns them and the page numbers.
    """

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor):
        _need(k_pages.dim() == 4 and k_pages.is_cuda and k_pages.dtype in _DTYPE, "k_pages must be a 4-d float32 or bfloat16 GPU tensor")
        _need(v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype and v_pages.device == k_pages.device,
              "v_pages must match k_pages in shape, dtype and device")
        _need(k_pages.stride(3) == 1 and v_pages.stride(3) == 1, "the pages' last dimension must be packed")
        self.k_pages, self.v_pages = k_pages, v_pages
        self.pages, self.kv_heads, self.page_size, self.head_dim = k_pages.shape
        self.dtype, self.device = k_pages.dtype, k_pages.device
        c = skipconv_cache()
        c.k_pages, c.v_pages = k_pages.data_ptr(), v_pages.data_ptr()
        c.k_page, c.k_head, c.k_slot = k_pages.stride()[:3]
        c.v_page, c.v_head, c.v_slot = v_pages.stride()[:3]
        c.pages, c.page_size, c.kv_heads, c.head_dim, c.dtype = self.pages, self.page_size, self.kv_heads, self.head_dim, _DTYPE[self.dtype]
        self._c = c

    @classmethod
    def empty(cls, pages: int, page_size: int, kv_heads: int, head_dim: int, dtype=torch.bfloat16, device="cuda") -> "PagedCache":
        """A cache of its own pages (not cleared: no token is read before it is appended)."""
        shape = (pages, kv_heads, page_size, head_dim)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device))

    def desc(self, batch: CacheBatch, tokens: int) -> skipconv_cache:
        """The C description for a batch."""
        _need(batch.device == self.device, "the batch is on another device than the cache")
        c = self._c
        c.page_table, c.row_start, c.kv_len = batch.page_table.data_ptr(), batch.row_start.data_ptr(), batch.kv_len.data_ptr()
        c.tokens, c.batch, c.table_width = tokens, batch.sequences, batch.page_table.shape[1]
        return c

    def append(self, k: torch.Tensor, v: torch.Tensor, batch: CacheBatch, rotary: Optional[Rotary] = None,
               pos: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None):
        """Write the new tokens' keys and values (tokens x kv_heads x head_dim) into the cache, the keys turned by `rotary` at
        `pos` (int32, tokens x axes). With `q` (tokens x heads x head_dim): also returns it turned, in `q_out` (may be q) or a new tensor."""
        tokens = k.shape[0]
        _heads_of(k, "k", None, self.kv_heads, self.head_dim, self.dtype, self.device)
        _heads_of(v, "v", tokens, self.kv_heads, self.head_dim, self.dtype, self.device)
        a = skipconv_append()
        a.k, a.k_token, a.k_head = k.data_ptr(), k.stride(0), k.stride(1)
        a.v, a.v_token, a.v_head = v.data_ptr(), v.stride(0), v.stride(1)
        if rotary is not None:
            _need(pos is not None and rotary.head_dim == self.head_dim, "a rotation needs pos and the cache's head_dim")
            r = rotary.desc(pos, tokens)
            a.rotary = ctypes.pointer(r)
        if q is not None:
            _need(rotary is not None, "queries are only turned: pass rotary and pos")
            _heads_of(q, "q", tokens, None, self.head_dim, self.dtype, self.device)
            if q_out is None:
                q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            elif q_out is not q:
                _heads_of(q_out, "q_out", tokens, q.shape[1], self.head_dim, self.dtype, self.device)
            a.q, a.q_token, a.q_head, a.q_heads = q.data_ptr(), q.stride(0), q.stride(1), q.shape[1]
            a.q_out, a.q_out_token, a.q_out_head = q_out.data_ptr(), q_out.stride(0), q_out.stride(1)
        skipconv_cache_append(self.desc(batch, tokens), a, _stream(self.device))
        return q_out

    def attend(self, q: torch.Tensor, batch: CacheBatch, causal: bool = True, window: int = -1, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None, return_lse: bool = False):
        """Attention of the new tokens' queries (tokens x heads x head_dim, heads a multiple of kv_heads) over the cache.

        causal: a token sees those up to itself, and `window` of those before it (-1: all); otherwise it sees its whole
        sequence and `window` of the tokens before the new ones. scale: head_dim ** -0.5 by default. Returns
        tokens x heads x head_dim (zeros for a row that sees nothing), with return_lse also the float32 log of the
        sum of exponentials, tokens x heads (-inf there). Rows of no sequence are not written.
        """
        _heads_of(q, "q", None, None, self.head_dim, self.dtype, self.device)
        tokens, heads, dim = q.shape
        if out is None:
            out = torch.empty((tokens, heads, dim), dtype=q.dtype, device=q.device)
        else:
            _heads_of(out, "out", tokens, heads, dim, self.dtype, self.device)
        lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device) if return_lse else None
        a = skipconv_attend(q.data_ptr(), out.data_ptr(), lse.data_ptr() if return_lse else None, q.stride(0), q.stride(1), out.stride(0),
                            out.stride(1), heads, 1 if causal else 0, window, 1.0 / math.sqrt(dim) if scale is None else scale, batch.max_new)
        c = self.desc(batch, tokens)
        need = skipconv_attend_workspace(c, a)
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        skipconv_cache_attend(c, a, ws.data_ptr() if need else None, need, _stream(self.device))
        return (out, lse) if return_lse else out
