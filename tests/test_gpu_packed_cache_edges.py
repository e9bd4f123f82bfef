"""What the calls on the cache in 4 bits, on accumulated weight and on eviction promise at their edges, on the GPU against the oracle in 64 bits.

Bounds, and the caches that the tests are made of, are those of test_gpu_packed_cache.py.
"""
import ctypes
import textwrap

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import packed_cache_oracle as P  # noqa: E402
from oracle import stream_attention_oracle as O  # noqa: E402
from paper_2104_11487_amd import skipconv as S  # noqa: E402
from paper_2104_11487_amd import stream_attention as A  # noqa: E402
from parity_util import say  # noqa: E402
from test_gpu_packed_cache import (DT, U, _attend_both, _batch, _certain, _compare, _compare_weights, _device, _filled, _garbage, _gpu, _held, _laid,  # noqa: E402
                                   _largest, _packed, _rng, _same, _small, _stored)
pytestmark = pytest.mark.gpu


# dim, pairs, adjacent, dtype, layout: whole chunks of halves, of neighbours, and any pairs
INVERSES = [(64, 32, False, "bf16", "packed"), (128, 64, True, "bf16", "view"), (80, 31, False, "bf16", "packed"), (96, 45, True, "bf16", "packed"),
            (40, 20, False, "bf16", "odd"), (64, 32, False, "f32", "heads"), (32, 16, True, "f32", "packed"), (72, 35, False, "f32", "odd"), (8, 3, True, "f32", "packed")]


@pytest.mark.parametrize("inverse", [0, 1], ids=["forward", "backward"])
@pytest.mark.parametrize("dim,pairs,adjacent,dtype,layout", INVERSES)
def test_append_turns_the_way_that_its_rotation_says(dim, pairs, adjacent, dtype, layout, inverse):
    """A rotation's description may turn back: keys and queries, as skipconv_cache_append's. The class never asks for it, the C call may."""
    say(f"[packed append, inverse {inverse}] {dim} {pairs} {adjacent} {dtype} {layout}")
    rng = _rng(191 + dim)
    lens, heads, kv_heads, page, groups = [(9, 30), (1, 1), (20, 20)], 4, 2, 16, -(-dim // 32)
    table, starts, length, pages = _batch(rng, lens, page)
    tokens = int(starts[-1])
    (k, k64), (v, v64), (q, q64) = (_stored(rng.standard_normal((tokens, h, dim)) + 0.3, dtype) for h in (kv_heads, kv_heads, heads))
    pos, freq = rng.integers(0, 5000, (tokens, 3)).astype(np.int32), rng.random((3, pairs)).astype(np.float32)
    rotary, at, batch = A.Rotary(_gpu(freq), dim, "adjacent" if adjacent else "halves"), _gpu(pos), _device(table, starts, length)
    old = [_garbage((pages, kv_heads, page), groups) for _ in range(2)]
    packed, paged = _packed([c for c, _ in old], [s for _, s in old], dim, dtype), A.PagedCache.empty(pages, page, kv_heads, dim, dtype=DT[dtype])
    outs = []
    for cache in (packed, paged):
        x = [_laid(t, layout) for t in (k, v, q)]
        out = torch.empty((tokens, heads, dim), dtype=DT[dtype], device="cuda")
        turn = rotary.desc(at, tokens, bool(inverse))
        a = S.skipconv_append(x[0].data_ptr(), x[1].data_ptr(), x[2].data_ptr(), out.data_ptr(), *x[0].stride()[:2], *x[1].stride()[:2], *x[2].stride()[:2],
                              *out.stride()[:2], heads, ctypes.pointer(turn))
        stream = torch.cuda.current_stream().cuda_stream
        if cache is packed:
            A.skipconv_packed_append(cache.desc(batch, tokens), cache._scales, a, stream)
        else:
            A.skipconv_cache_append(cache.desc(batch, tokens), a, stream)
        torch.cuda.synchronize()
        outs.append(out)
    first, second = O.partners(pairs, adjacent)
    want = O.rotate(q64, pos, freq.astype(np.float64), adjacent, bool(inverse))
    bound = np.zeros_like(want)
    bound[..., first] = bound[..., second] = 8 * U * (np.abs(q64[..., first]) + np.abs(q64[..., second]))
    if dtype == "bf16":
        bound[..., :2 * pairs] += (2.0 ** -8 * np.abs(want) + 2.0 ** -8 * bound)[..., :2 * pairs]
    for out in outs:
        assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
    turned = O.rotate(k64, pos, freq.astype(np.float64), adjacent, bool(inverse))
    sure = _certain(turned)
    sure[..., 2 * pairs:] = True
    codes, scales = _held(packed)
    compared = 0
    for which, x, certain in ((0, turned, sure), (1, v64, np.ones(v64.shape, bool))):
        want_c, want_s = P.pack(x.astype(np.float32))
        for row, p, slot in O.places(table, starts, length, page, pages):
            for g in range(groups):
                fine = certain[row, :, 32 * g:32 * g + 32].all(-1)
                compared += fine.sum()
                assert np.array_equal(codes[which][p, fine, slot, 16 * g:16 * g + 16], want_c[row, fine, 16 * g:16 * g + 16])
                assert _same(scales[which][p, fine, slot, g], want_s[row, fine, g])
    assert compared > 0.7 * 2 * tokens * kv_heads * groups  # an element in doubt makes its group so


# what the rows' elements are, and the scale: the largest comes into fp16's range by a power of two, which the scale gives back
SIZES = {"zero": (0.0, 1e-3), "zero, tiny scale": (0.0, 1e-30), "subnormal": (1e-40, 1e-4), "tiny": (2.0 ** -120, 2.0 ** -20), "least scale": (1.0, 1e-45), "zero, scale 1": (0.0, 1.0)}


@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 256)])
@pytest.mark.parametrize("new", [1, 40, 300])
def test_rows_of_vanishing_queries_take_the_mean(new, dtype, dim, size):
    """Scores of next to nothing: every seen key counts alike, and the masked ones not at all. One of the rows is an ordinary one."""
    gain, scale = SIZES[size]
    rng = _rng(192 + new)
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, [(new, 2 * new + 61), (1, 9)], 4, 2, dim, 16, dtype)
    ordinary = q[0, 1].clone()
    q *= gain
    if gain == 0.0:
        q[0, 1] = ordinary  # beside rows of zeros
    q64 = q.double().cpu().numpy()
    for mask in ((True, -1), (True, 20), (False, 7), (False, -1)):
        want = O.attend(q64, k64, v64, table, starts, length, *mask, scale=scale)
        for hint, out, lse in _attend_both(cache, q, table, starts, length, causal=mask[0], window=mask[1], scale=scale):
            say(f"[packed attention, {size}] {new} {dtype} {dim} mask={mask} max_new={hint}")
            _compare(out, lse, want, dtype, dim, _largest(v64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 40, 300])
def test_scores_of_huge_queries_and_zero_keys_are_zero(new, dtype):
    """The scale and the largest element's power of two pass fp32 together: no score is 0 times infinity."""
    def spoil(codes, scales, table):
        codes[0][...] = 0
        scales[0][...] = 0.0
    rng = _rng(193 + new)
    cache, k64, v64, q, _, table, starts, length = _filled(rng, [(new, 2 * new + 61)], 4, 2, 64, 16, dtype, spoil=spoil)
    q = torch.full_like(q, 3e38)
    q64 = q.double().cpu().numpy()
    want = O.attend(q64, k64, v64, table, starts, length, scale=1e5)
    for hint, out, lse in _attend_both(cache, q, table, starts, length, scale=1e5):
        _compare(out, lse, want, dtype, 64, _largest(v64))
    batch = _device(table, starts, length)
    w = cache.weigh(q, lse, batch, torch.zeros(k64.shape[:3], device="cuda"), scale=1e5)
    want, size = P.weigh(np.zeros(k64.shape[:3]), q64, lse.double().cpu().numpy(), k64, table, starts, length, scale=1e5)
    _compare_weights(w.double().cpu().numpy(), want, size, 64, 1.0, 0.0, 2 * new)


@pytest.mark.parametrize("packed", [True, False], ids=["packed", "paged"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,new", [(64, 8), (128, 8), (64, 48), (128, 160), (256, 160)])
def test_rows_that_are_left_out_by_their_lse_give_nothing(dtype, packed, dim, new):
    """lse = -inf takes a row out, whatever it sees: a key that is NaN, in a block that all rows see or in one that some do not, gets nothing of it. An lse of
    infinity is what the formula makes of it: no weight for finite scores."""
    say(f"[weigh, left out] {dtype} packed={packed} {dim} {new}")
    lens, heads, kv_heads, page = [(new, 400)], 4, 2, 16
    bad = (20, 150, 400 - new + 1)  # seen by all rows, whole blocks around them; by some rows
    rng = _rng(194 + dim)

    def spoil(codes, scales, table):
        for at in bad:
            scales[0][table[0, at // page], 0, at % page] = np.nan
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, lens, heads, kv_heads, dim, page, dtype, spoil=spoil)
    if not packed:
        kp, k64 = _stored(k64, dtype)
        cache = A.PagedCache(kp, kp)
    with np.errstate(invalid="ignore"):
        _, lse, _ = O.attend(q64, k64, np.zeros_like(k64), table, starts, length)
    lse = lse.astype(np.float32)
    lse[:, :2] = -np.inf       # the rows of the key head with NaN
    lse[::3, 2] = -np.inf      # some of the other's
    given = lse.copy()
    given[1, 3] = np.inf       # the oracle's formula with its bound has no number for it
    lse[1, 3] = -np.inf
    before = rng.random(k64.shape[:3]).astype(np.float32)
    for hint in sorted({0, new, 1}):
        weights = cache.weigh(q, _gpu(given), _device(table, starts, length, max_new=hint), _gpu(before), decay=0.5)
        want, size = P.weigh(before, q64, lse.astype(np.float64), k64, table, starts, length, decay=0.5)
        assert np.isfinite(want).all()
        _compare_weights(weights.double().cpu().numpy(), want, size, dim, 0.5, before, 2 * new)


@pytest.mark.parametrize("packed", [True, False], ids=["packed", "paged"])
def test_evict_takes_arrays_side_by_side(packed):
    """Lengths and positions next to what the call reads, in one tensor: the C call's results are the class's."""
    rng = _rng(197)
    lens, heads, page, keep, recent = [(0, 90), (0, 33), (0, 64)], 2, 16, 40, 7
    cache, _, _, _, _, table, starts, length = _filled(rng, lens, heads, heads, 64, page, "bf16")
    if not packed:
        cache = A.PagedCache(*(torch.randn((cache.pages, heads, page, 64), device="cuda").bfloat16() for _ in range(2)))
    into = np.setdiff1d(np.arange(cache.pages), table)[:3, None].repeat(3, 1).astype(np.int32)  # the spare pages: not enough for all, so tokens go nowhere
    into[:, 1:] = -1
    weights = _gpu(rng.random((cache.pages, heads, page)).astype(np.float32))
    start, held = weights.clone(), [x.clone() for x in cache._tensors]
    want_lengths, want = cache.evict(weights, _device(table, starts, length), _gpu(into), keep=keep, recent=recent)
    want_weights, want_held = weights.clone(), [x.clone() for x in cache._tensors]
    sizes = [len(lens) * heads * keep, table.size, len(lens), len(lens), into.size]  # kept, table, kv_len, lengths, into
    whole = torch.full((sum(sizes),), -5, dtype=torch.int32, device="cuda")
    kept, tables, kv_len, lengths, to = whole.split(sizes)
    tables.copy_(_gpu(table).flatten()), kv_len.copy_(_gpu(length)), to.copy_(_gpu(into).flatten())
    weights.copy_(start)
    for x, y in zip(cache._tensors, held):
        x.copy_(y)
    c = cache.desc(A.CacheBatch(tables.view(table.shape), _gpu(starts), kv_len), 0)
    e = S.skipconv_evict(weights.data_ptr(), to.data_ptr(), lengths.data_ptr(), kept.data_ptr(), into.shape[1], keep, recent)
    A.skipconv_cache_evict(c, cache._scales if packed else None, e, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(lengths, want_lengths) and torch.equal(kept.view(want.shape), want) and torch.equal(weights, want_weights)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(cache._tensors, want_held))
    assert np.array_equal(tables.cpu().numpy().reshape(table.shape), table) and np.array_equal(kv_len.cpu().numpy(), length)


def test_the_modules_example_keeps_what_it_kept():
    """The loop of the module's documentation, as it stands there: what an eviction keeps, the next frame's tokens find."""
    text = A.__doc__.split("kept short by eviction")[1].split("\n\n", 1)[1]
    example = textwrap.dedent("\n".join(line for line in text.split("\n") if line.startswith("    ") or not line.strip()))
    assert "evict(" in example and "for " in example
    g = torch.Generator(device="cuda")
    g.manual_seed(195)
    new, kept_ones, appended = 64 * 64, [], []

    def held(cache, pages, length):
        return [x.transpose(0, 1).reshape(cache.kv_heads, -1, cache.head_dim)[:, :length].clone() for x in cache.unpack(pages)]

    def frames():
        for t in range(4):
            if t:
                kept_ones.append((names["kept"].clone(), held(names["cache"], names["here"][0], int(names["lengths"][0]))))
            k, v, q = (torch.randn(new, h, 64, device="cuda", generator=g).bfloat16() for h in (2, 2, 8))
            i = torch.arange(new, device="cuda")
            yield q, k, v, torch.stack([torch.full_like(i, t), i // 64, i % 64], 1).int()
        kept_ones.append((names["kept"].clone(), held(names["cache"], names["here"][0], int(names["lengths"][0]))))

    class Watched(A.PackedCache):  # looks at what a frame's append leaves
        def append(self, k, v, batch, **kw):
            got = super().append(k, v, batch, **kw)
            appended.append(held(self, batch.page_table[0], int(batch.kv_len[0])))
            return got
    names = dict(vars(A), torch=torch, frames=frames(), rotary=A.Rotary(A.axis_frequencies((11, 11, 10)), 64), PackedCache=Watched)
    exec(compile(example, "example", "exec"), names)
    assert len(kept_ones) == len(appended) == 4
    for t, ((kept, values), all_of) in enumerate(zip(kept_ones, appended)):
        before, total = (0 if t == 0 else 4096), all_of[0].shape[1]
        assert total == before + new and (kept >= 0).all() and kept.shape == (1, 2, 4096)
        for which in (0, 1):
            if t:  # the tokens that were kept are there yet when the new ones have come
                assert torch.equal(all_of[which][:, :before], kept_ones[t - 1][1][which])
            for h in range(2):  # and the next ones to stay are taken from them all
                assert torch.equal(values[which][h], all_of[which][h][kept[0, h].long()])
        assert (kept[0, :, -256:] == torch.arange(total - 256, total, device="cuda")).all()


@pytest.mark.parametrize("new", [1, 40, 300])
def test_small_elements_beside_large_ones(new):
    """bf16 elements of at least 2^-31 of their row's largest are taken exactly, smaller ones to 2^-39 of it. The large one meets a key's zero, so that the
    score is the small one's alone, and of size one by the scale."""
    kv, dim, page = 64, 64, 16
    half = np.arange(kv).reshape(4, 1, page) >= kv // 2  # of these keys element 33 is one; all else is zero
    codes, scales = np.zeros((4, 1, page, 32), np.uint8), np.zeros((4, 1, page, 2, 2), np.float16)
    codes[..., 16] = np.where(half, 1 << 4, 0)
    scales[..., 1, 0] = 1.0
    cache = _packed([codes] * 2, [scales] * 2, dim, "bf16")
    batch = _device(np.arange(4, dtype=np.int32)[None], np.array([0, new], np.int32), np.array([kv], np.int32))
    large = 255 / 128  # all bits of the mantissa
    slack = 4 * (2 * dim + 6) * U * large + 16 * U * (large + 1) + 2 * kv * U + 32 * U + 8 * U * np.log(kv * np.exp(large))
    total = lambda s: np.log(kv // 2 * (1 + np.exp(s)))  # noqa: E731
    for small in (-8, -25, -31, -33, -36, -39, -45):
        say(f"[packed attention, 2^{small} beside 1] {new}")
        q = torch.zeros((new, 2, dim), dtype=torch.bfloat16, device="cuda")
        q[..., 2], q[:, 0, 33] = large, large * 2.0 ** small
        _, lse = cache.attend(q, batch, causal=False, scale=2.0 ** -small, return_lse=True)
        lse = lse.double().cpu().numpy()
        off = 0.0 if small >= -31 else min(2.0 ** (-39 - small), 1.0) * large  # an element that vanishes is off by itself
        assert (lse[:, 0] >= total(large - off) - slack).all() and (lse[:, 0] <= total(large + off) + slack).all(), small
        assert np.abs(lse[:, 1] - np.log(kv)).max() <= slack


def test_no_tangent_is_lost():
    """Forward-mode tangents: the calls compute none, so tensors that carry one are refused, in every cache and in a rotation into a tensor."""
    import torch.autograd.forward_ad as forward
    cache, batch, q, weights = _small()
    lse, into = torch.zeros(2, 4, device="cuda"), torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    pages = [torch.zeros((cache.pages, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rotary, pos = A.Rotary(A.axis_frequencies((11, 11, 10)), 64), torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    before = [x.clone() for x in cache._tensors]
    with forward.dual_level():
        dual = lambda x: forward.make_dual(x.clone(), torch.ones_like(x))  # noqa: E731
        x = dual(q)
        learned = A.PackedCache(*cache._tensors[:2], *(dual(t) for t in cache._tensors[2:]), cache.head_dim)
        for c in (cache, A.PagedCache(*pages)):
            for call in (lambda: c.append(x[:, :2], q[:, 2:], batch), lambda: c.append(q[:, :2], x[:, 2:], batch), lambda: c.append(q[:, :2], q[:, 2:], batch, rotary=rotary, pos=pos, q=x),
                         lambda: c.attend(x, batch), lambda: c.attend(q, batch, out=dual(q)), lambda: c.weigh(x, lse, batch, weights), lambda: c.weigh(q, dual(lse), batch, weights),
                         lambda: c.weigh(q, lse, batch, dual(weights)), lambda: c.evict(dual(weights), batch, into, keep=8)):
                with pytest.raises(ValueError, match="gradient"):
                    call()
        for call in (lambda: learned.attend(q, batch), lambda: learned.unpack(into), lambda: learned.weigh(q, lse, batch, weights), lambda: rotary.rotate(x, pos),
                     lambda: rotary.rotate(q, pos, out=dual(q)), lambda: A.PagedCache(dual(pages[0]), pages[1]).attend(q, batch)):
            with pytest.raises(ValueError, match="gradient"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="gradient"):  # which leaves tangents on
                call()
        with pytest.raises((ValueError, RuntimeError)):
            rotary(x, pos)
        with torch.inference_mode():  # and that turns them off
            cache.attend(x, batch)
        plain = cache.attend(q, batch)  # tensors without one are as anywhere else
        cache.weigh(q, lse, batch, weights.clone())
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, cache._tensors))
    assert torch.equal(plain, cache.attend(q, batch))


def test_unpack_of_a_page_of_more_than_2_to_31_rows():
    """One page of 2049 heads of 2^20 slots: rows are counted past 32 bits. Codes of a slot are the same in every head, and the pairs of a head in every slot,
    so that the cache itself is small; what it stands for is 69 GB."""
    heads, page, dim = 2049, 1 << 20, 8
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 90 GB of free GPU memory")
    rng = _rng(196)
    codes = [_gpu(rng.integers(0, 256, (1, 1, page, 16)).astype(np.uint8)).expand(1, heads, page, 16) for _ in range(2)]
    scales = [_gpu(rng.random((1, heads, 1, 1, 2)).astype(np.float16)).expand(1, heads, page, 1, 2) for _ in range(2)]
    cache = A.PackedCache(*codes, *scales, dim)
    got = cache.unpack(torch.zeros(1, dtype=torch.int32, device="cuda"))
    for which in (0, 1):
        for h in (0, 1, 1023, 2046, 2047, 2048):
            c, s = (x[which][0, h if x is scales else 0].cpu().numpy() for x in (codes, scales))
            assert np.array_equal(got[which][0, h].double().cpu().numpy(), P.values(c, s, dim)), (which, h)
    del got
    torch.cuda.empty_cache()
