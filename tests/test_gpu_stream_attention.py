"""Rotary positions, the paged cache and attention over it on the GPU, against the oracle in 64 bits.

Bounds, per element, from the arithmetic (u = 2^-24):
  rotation   8 u (|a| + |b|) of the pair's elements (two products, a sum, the cosine and sine of an angle reduced to 2^-25 turns),
             and half a unit in the last place of bf16 (eight significant bits: 2^-8);
  attention  with A the weighted mean of |v|, Q the largest sum of |q k| * scale, S the largest |score|, n keys:
             scores (dim + 2) u Q, exponents 4 u (S + 1), sums n u, once in the numerator and once in the denominator:
             A * (4 (dim + 2) u Q + 16 u (S + 1) + 2 n u + 8 u); bf16 caches: the exponentials' rounding 2^-8 A, and that
             of the output 2^-8 |out|, a quarter more for their products.
Slots of the cache that hold no token are NaN, entries of the page table that hold no page are wild.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import stream_attention_oracle as O  # noqa: E402
from paper_2104_11487_amd import skipconv as S  # noqa: E402
from paper_2104_11487_amd import stream_attention as A  # noqa: E402
from parity_util import say  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def _stored(x, dtype):
    """A GPU tensor of x in the dtype, and its values in 64 bits."""
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DT[dtype])
    return t.cuda(), t.double().numpy()


def _laid(x, layout):
    """The GPU tensor tokens x heads x dim in another memory layout."""
    t, h, d = x.shape
    if layout == "view":  # the middle of a wider projection
        w = torch.full((t, h + 3, d), float("nan"), dtype=x.dtype, device="cuda")
        w[:, 1:1 + h] = x
        return w[:, 1:1 + h]
    if layout == "heads":  # heads outermost
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "odd":  # rows that begin anywhere
        w = torch.full((t * (h * d + 1) + 1,), float("nan"), dtype=x.dtype, device="cuda")
        v = w[1:].as_strided((t, h, d), (h * d + 1, d, 1))
        v.copy_(x)
        return v
    return x.contiguous()


# ---------------------------------------------------------------- rotation --

# tokens, heads, dim, pairs, axes, adjacent, dtype, layout
TURNS = [
    (1, 1, 2, 1, 1, False, "f32", "packed"), (1, 1, 64, 32, 3, False, "bf16", "packed"), (17, 5, 64, 32, 3, False, "bf16", "view"),
    (257, 3, 128, 64, 2, False, "bf16", "packed"), (33, 4, 80, 36, 3, True, "f32", "packed"), (33, 4, 80, 31, 3, False, "bf16", "packed"),
    (9, 2, 80, 31, 3, True, "bf16", "heads"), (9, 3, 96, 40, 3, False, "bf16", "heads"), (65, 2, 256, 78, 3, False, "bf16", "view"),
    (12, 2, 256, 128, 8, False, "f32", "view"), (7, 3, 36, 17, 2, False, "bf16", "odd"), (7, 3, 37, 18, 2, True, "f32", "odd"),
    (300, 40, 128, 64, 3, True, "bf16", "packed"), (5, 3, 1024, 512, 2, False, "bf16", "packed"), (5, 2, 1023, 511, 1, False, "bf16", "odd"),
    (3000, 2, 64, 24, 3, False, "f32", "packed"), (4, 70, 96, 48, 3, False, "f32", "packed"), (2, 200, 64, 32, 3, False, "bf16", "view"),
]


@pytest.mark.parametrize("inverse", [False, True], ids=["forward", "backward"])
@pytest.mark.parametrize("case", TURNS, ids=["x".join(map(str, c)) for c in TURNS])
def test_rotation(case, inverse):
    tokens, heads, dim, pairs, axes, adjacent, dtype, layout = case
    say(f"[rotation] {case} inverse={inverse}")
    rng = _rng(11 + tokens + dim)
    x, x64 = _stored(rng.standard_normal((tokens, heads, dim)), dtype)
    pos = rng.integers(-50, 100000, (tokens, axes)).astype(np.int32)
    freq = torch.from_numpy((rng.random((axes, pairs)) * 10.0 ** -rng.integers(0, 5, (axes, pairs))).astype(np.float32)).cuda()
    rotary = A.Rotary(freq, dim, "adjacent" if adjacent else "halves")
    at = torch.from_numpy(pos).cuda()
    src = _laid(x, layout)
    want = O.rotate(x64, pos, freq.cpu().double().numpy(), adjacent, inverse)
    first, second = O.partners(pairs, adjacent)
    bound = np.zeros_like(want)
    size = 8 * U * (np.abs(x64[..., first]) + np.abs(x64[..., second]))
    bound[..., first] = bound[..., second] = size
    if dtype == "bf16":
        bound[..., np.concatenate([first, second])] += (2.0 ** -8 * np.abs(want) + 2.0 ** -8 * bound)[..., np.concatenate([first, second])]
    got = (rotary.backward if inverse else rotary.rotate)(src, at)
    assert got.is_contiguous()
    assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()
    rest = got[..., 2 * pairs:]
    assert torch.equal(rest.view(torch.int32 if dtype == "f32" else torch.int16), x[..., 2 * pairs:].view(torch.int32 if dtype == "f32" else torch.int16))
    # into a tensor of another layout, and in place: the same bits
    into = _laid(torch.zeros_like(x), "heads")
    assert torch.equal(rotary.rotate(x, at, out=into, inverse=inverse), got)
    assert torch.equal(rotary.rotate(src, at, out=src, inverse=inverse), got)


def test_rotation_gradient():
    """Under autograd: against the formula's gradient, and against differences."""
    rng = _rng(12)
    x, _ = _stored(rng.standard_normal((6, 3, 20)), "f32")
    pos, freq = rng.integers(0, 40, (6, 2)).astype(np.int32), rng.random((2, 9)).astype(np.float32)
    rotary, at = A.Rotary(torch.from_numpy(freq).cuda(), 20), torch.from_numpy(pos).cuda()
    w, w64 = _stored(rng.standard_normal((6, 3, 20)), "f32")
    x.requires_grad_(True)
    (rotary(x, at) * w).sum().backward()
    want = O.rotate(w64, pos, freq.astype(np.float64), inverse=True)
    assert np.abs(x.grad.double().cpu().numpy() - want).max() <= 16 * U * np.abs(w64).max()
    # the loss is linear in x: a difference of any step is the gradient, up to the rounding of the loss's terms
    e, _ = _stored(rng.standard_normal((6, 3, 20)), "f32")
    with torch.no_grad():
        up, down = ((rotary(x + s * e, at).double() * w.double()).sum() for s in (1.0, -1.0))
    exact = (x.grad.double() * e.double()).sum()
    terms = float((w.double().abs().sum(-1) * (x.double().abs() + e.double().abs()).amax(-1)).sum())
    assert abs(float((up - down) / 2 - exact)) <= 32 * U * terms
    x.grad = None
    rotary(x, at).sum().backward()  # a broadcast gradient
    ones = O.rotate(np.ones((6, 3, 20)), pos, freq.astype(np.float64), inverse=True)
    assert np.abs(x.grad.double().cpu().numpy() - ones).max() <= 32 * U


def _small_call():
    """A cache, a batch, a rotation and what their calls take."""
    rng = _rng(54)
    cache, _, _, q, _, table, starts, length = _filled(rng, [(2, 40)], 4, 2, 64, 16, "bf16")
    return cache, _device(table, starts, length), A.Rotary(A.axis_frequencies((16, 16)), 64), torch.ones(2, 2, dtype=torch.int32, device="cuda"), q


def test_a_batch_of_no_sequence():
    cache, _, rotary, pos, q = _small_call()
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    none = A.CacheBatch(ints(0, 4), ints(1), ints(0))
    for tokens in (0, 2):  # rows of no sequence are not written
        x, at, out = q[:tokens], pos[:tokens], torch.full_like(q[:tokens], 3.0)
        pages = cache.k_pages.clone(), cache.v_pages.clone()
        cache.append(x[:, :2], x[:, 2:], none, rotary=rotary, pos=at, q=x, q_out=out)
        assert cache.attend(x, none, out=out) is out and (out == 3.0).all()
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(pages, (cache.k_pages, cache.v_pages)))


def test_no_gradient_is_lost():
    """Calls without a graph refuse tensors that require a gradient, unless none are recorded."""
    cache, batch, rotary, pos, q = _small_call()
    k, v = (x.contiguous().clone() for x in (q[:, :2], q[:, 2:]))
    out = torch.empty_like(q)
    calls = ((lambda: rotary.rotate(q, pos), (q, rotary.freq)), (lambda: rotary.rotate(q, pos, out=out), (q, out)), (lambda: rotary.backward(q, pos), (q,)),
             (lambda: rotary(q, pos), (rotary.freq,)), (lambda: cache.append(k, v, batch), (k, v, cache.k_pages, cache.v_pages)),
             (lambda: cache.append(k, v, batch, rotary=rotary, pos=pos, q=q, q_out=out), (k, v, q, out, rotary.freq)),
             (lambda: cache.attend(q, batch), (q, cache.k_pages, cache.v_pages)), (lambda: cache.attend(q, batch, out=out), (q, out)))
    for call, tensors in calls:
        call()
        for x in tensors:
            x.requires_grad_(True)
            with pytest.raises(ValueError, match="gradient"):
                call()
            with torch.no_grad():
                call()
            x.requires_grad_(False)


def test_what_a_call_writes_is_known_to_autograd():
    """A tensor that autograd saved and a call wrote over afterwards is refused by the backward pass, as after any operation in place."""
    cache, batch, rotary, pos, q = _small_call()
    k, v = (x.contiguous().clone() for x in (q[:, :2], q[:, 2:]))
    weight = torch.ones(1, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    out = torch.zeros_like(q)
    calls = ((lambda: rotary.rotate(q, pos, out=q), q), (lambda: cache.append(k, v, batch), cache.k_pages), (lambda: cache.append(k, v, batch), cache.v_pages),
             (lambda: cache.append(k, v, batch, rotary=rotary, pos=pos, q=q, q_out=q), q), (lambda: cache.attend(q, batch, out=out), out))
    for call, written in calls:
        loss = (weight * written).sum()  # saves `written` for the gradient of weight
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    x = torch.randn(2, 4, 64, device="cuda", requires_grad=True)
    with torch.inference_mode():
        other = A.Rotary(A.axis_frequencies((16, 16)), 64)
    other(x, pos).sum().backward()
    loss = rotary(x, pos).sum()
    rotary.freq.mul_(2.0)  # the gradient would turn back by other angles
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_axis_frequencies():
    f = A.axis_frequencies((3, 2, 4), base=100.0).cpu().numpy()
    assert f.shape == (3, 9) and (np.count_nonzero(f, axis=0) == 1).all()
    assert np.allclose(f[2, 5:], 100.0 ** (-np.arange(4) / 4), rtol=1e-7)


# ------------------------------------------------------------------- cache --

def _batch(rng, lens, page, spare=3, pages_first=0, width=None):
    """Page table (wild where it holds no page), starts and lengths of sequences with (new, kv) tokens."""
    held = [-(-kv // page) for _, kv in lens]
    width = width or max(held + [1]) + 2
    order = pages_first + rng.permutation(sum(held) + spare)
    table = rng.choice(np.array([-1, -12345, 1 << 30, 2 ** 31 - 1]), (len(lens), width)).astype(np.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    starts = np.concatenate([[0], np.cumsum([n for n, _ in lens])]).astype(np.int32)
    return table, starts, np.array([kv for _, kv in lens], np.int32), pages_first + sum(held) + spare


def _device(table, starts, lens, max_new=0):
    c = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    return A.CacheBatch(c(table), c(starts), c(lens), max_new=max_new)


def _pages(k, v, order):
    """The pages as tensors that a cache takes, slots outermost for order "slots"."""
    if order == "slots":
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    return k, v


# lens, q heads, kv heads, dim, pairs, adjacent, page, dtype, layout, order
APPENDS = [
    ([(1, 1)], 4, 2, 64, 32, False, 16, "bf16", "packed", "heads"),
    ([(1, 40), (1, 17), (1, 16), (1, 1)], 8, 2, 128, 64, False, 16, "bf16", "packed", "heads"),
    ([(5, 5), (0, 9), (17, 40), (0, 0), (1, 300)], 2, 1, 64, 31, False, 7, "bf16", "view", "slots"),
    ([(196, 500), (3, 3)], 3, 3, 80, 32, True, 196, "f32", "packed", "heads"),
    ([(30, 30), (2, 64)], 4, 4, 96, 48, True, 1, "bf16", "heads", "slots"),
    ([(9, 33)], 6, 2, 40, 20, False, 5, "bf16", "odd", "heads"),
    ([(1, 2)] * 130, 2, 1, 32, 16, False, 4, "f32", "packed", "heads"),
    ([(700, 900), (400, 400)], 4, 2, 64, 32, False, 64, "bf16", "view", "heads"),
    ([(4, 8)], 70, 20, 256, 100, False, 32, "bf16", "packed", "heads"),
]


@pytest.mark.parametrize("mode", ["queries", "keys", "copy"])
@pytest.mark.parametrize("case", APPENDS, ids=[f"{i}" for i in range(len(APPENDS))])
def test_append(case, mode):
    lens, heads, kv_heads, dim, pairs, adjacent, page, dtype, layout, order = case
    say(f"[append] {case[1:]} {mode}")
    rng = _rng(21 + dim + page)
    table, starts, length, pages = _batch(rng, lens, page)
    extra = 3  # rows of no sequence
    tokens = int(starts[-1]) + extra
    k, k64 = _stored(rng.standard_normal((tokens, kv_heads, dim)), dtype)
    v, v64 = _stored(rng.standard_normal((tokens, kv_heads, dim)), dtype)
    q, q64 = _stored(rng.standard_normal((tokens, heads, dim)), dtype)
    pos = rng.integers(0, 5000, (tokens, 3)).astype(np.int32)
    freq = rng.random((3, pairs)).astype(np.float32)
    rotary = A.Rotary(torch.from_numpy(freq).cuda(), dim, "adjacent" if adjacent else "halves")
    kp, kp64 = _stored(rng.standard_normal((pages, kv_heads, page, dim)), dtype)
    vp, vp64 = _stored(rng.standard_normal((pages, kv_heads, page, dim)), dtype)
    cache = A.PagedCache(*_pages(kp, vp, order))
    batch = _device(table, starts, length)
    at = torch.from_numpy(pos).cuda()
    turn = dict(rotary=rotary, pos=at) if mode != "copy" else {}
    q_out = torch.full((tokens, heads, dim), 7.0, dtype=DT[dtype], device="cuda")
    got_q = cache.append(_laid(k, layout), _laid(v, layout), batch, **turn, **(dict(q=_laid(q, layout), q_out=q_out) if mode == "queries" else {}))
    turned = rotary.rotate(k, at) if mode != "copy" else k
    # the rotation's values are test_rotation's matter: bit for bit the same here
    want_k, want_v = O.append(kp64, vp64, turned.double().cpu().numpy(), v64, table, starts, length)
    assert np.array_equal(cache.k_pages.double().cpu().numpy(), want_k) and np.array_equal(cache.v_pages.double().cpu().numpy(), want_v)
    if mode == "queries":
        assert got_q is q_out
        assert torch.equal(q_out[:-extra], rotary.rotate(q, at)[:-extra]) and (q_out[-extra:] == 7.0).all()
        inplace = q.clone()
        assert cache.append(k, v, batch, **turn, q=inplace, q_out=inplace) is inplace
        assert torch.equal(inplace[:-extra], q_out[:-extra]) and torch.equal(inplace[-extra:], q[-extra:])
    else:
        assert got_q is None


def test_append_leaves_out_what_has_no_place():
    rng = _rng(22)
    table = np.array([[1, 5, 0, 2]], np.int32)  # page 5 of 4 does not exist
    kp, vp = (_stored(rng.standard_normal((4, 2, 4, 64)), "bf16") for _ in range(2))
    k, v = (_stored(rng.standard_normal((10, 2, 64)), "bf16") for _ in range(2))
    for new, kv in ((10, 12), (10, 7), (10, 40)):  # over the missing page; from before the begin; past the table
        starts, length = np.array([0, new], np.int32), np.array([kv], np.int32)
        cache = A.PagedCache(kp[0].clone(), vp[0].clone())
        cache.append(k[0], v[0], _device(table, starts, length))
        want = O.append(kp[1], vp[1], k[1], v[1], table, starts, length)
        assert np.array_equal(cache.k_pages.double().cpu().numpy(), want[0]) and np.array_equal(cache.v_pages.double().cpu().numpy(), want[1])


# --------------------------------------------------------------- attention --

def _filled(rng, lens, heads, kv_heads, dim, page, dtype, order="heads", gain=1.0, spoil=None, width=None):
    table, starts, length, pages = _batch(rng, lens, page, width=width)
    kp, vp = (np.full((pages, kv_heads, page, dim), np.nan, np.float32) for _ in range(2))
    for b, (_, kv) in enumerate(lens):
        for i in range(0, kv, page):
            n = min(page, kv - i)
            kp[table[b, i // page], :, :n] = rng.standard_normal((kv_heads, n, dim))
            vp[table[b, i // page], :, :n] = 0.5 + rng.standard_normal((kv_heads, n, dim))
    if spoil:
        spoil(kp, vp, table)
    (kd, k64), (vd, v64) = _stored(kp, dtype), _stored(vp, dtype)
    q, q64 = _stored(gain * rng.standard_normal((int(starts[-1]), heads, dim)), dtype)
    return A.PagedCache(*_pages(kd, vd, order)), k64, v64, q, q64, table, starts, length


def _compare(out, lse, want, dtype, dim):
    o, l, b = want  # noqa: E741
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(o)) and np.array_equal(np.isinf(got), np.isinf(o))
    assert np.array_equal(got[np.isinf(o)], o[np.isinf(o)])
    with np.errstate(invalid="ignore"):
        q, s, n = (b[x][..., None] for x in ("size", "most", "count"))
        bound = b["weight"] * (4 * (dim + 2) * U * q + 16 * U * (s + 1) + 2 * n * U + 8 * U)
        if dtype == "bf16":
            bound = 1.25 * (bound + 2.0 ** -8 * b["weight"] + 2.0 ** -8 * np.abs(o))
        fine = np.isfinite(o)
        off = np.abs(got - o)
        ok = off[fine] <= bound[fine]
        assert ok.all(), f"{(~ok).sum()} of {ok.size} off, worst {np.max(off[fine] / np.maximum(bound[fine], 1e-30)):.3g} of the bound"
    none = np.isneginf(l)
    assert np.array_equal(np.isneginf(gl), none) and not got[none].any()
    size = (dim + 2) * U * b["size"] + (b["count"] + 16) * U + 8 * U * (b["most"] + np.abs(np.where(none, 0, l)))
    assert (np.abs(gl - l)[~none] <= size[~none]).all()


def _attend_both(cache, q, table, starts, length, **kw):
    """The call with every hint about the new tokens; all must hold, and equal calls give equal bits."""
    most = int(np.max(np.diff(starts), initial=0))
    for hint in sorted({0, most, 1}):
        batch = _device(table, starts, length, max_new=hint)
        out, lse = cache.attend(q, batch, return_lse=True, **kw)
        again = cache.attend(q, batch, **kw)
        assert torch.equal(out.view(torch.int16 if out.dtype == torch.bfloat16 else torch.int32),
                           again.view(torch.int16 if out.dtype == torch.bfloat16 else torch.int32))
        yield hint, out, lse


MASKS = [(True, -1), (False, -1), (True, 0), (True, 37), (False, 37), (True, 1000)]
# lens, heads, kv heads, dim, page, dtype, order
ATTENDS = [
    ([(1, 1)], 1, 1, 8, 1, "bf16", "heads"),
    ([(1, 77)], 4, 1, 64, 16, "bf16", "heads"),
    ([(1, 64), (1, 65), (1, 1), (1, 200), (1, 31)], 8, 2, 128, 16, "bf16", "slots"),
    ([(1, 3000)], 16, 2, 128, 64, "bf16", "heads"),
    ([(5, 5), (0, 40), (17, 90), (0, 0), (40, 333)], 6, 3, 80, 7, "bf16", "heads"),
    ([(3, 900), (2, 2)], 10, 2, 32, 3, "bf16", "slots"),
    ([(130, 300)], 4, 1, 64, 64, "bf16", "heads"),
    ([(70, 150), (33, 33)], 2, 2, 128, 16, "bf16", "slots"),
    ([(20, 196), (5, 700)], 6, 2, 96, 196, "bf16", "heads"),
    ([(25, 130)], 4, 2, 256, 32, "bf16", "heads"),
    ([(40, 41)], 3, 1, 160, 5, "bf16", "heads"),
    ([(1, 500), (2, 70)], 4, 2, 256, 16, "bf16", "heads"),
    ([(1, 300), (1, 20)], 4, 2, 192, 16, "bf16", "heads"),
    ([(1, 1), (1, 50)], 1, 1, 8, 1, "f32", "heads"),
    ([(1, 900), (2, 64), (3, 17)], 8, 2, 80, 196, "f32", "slots"),
    ([(100, 240), (0, 3), (9, 9)], 6, 3, 64, 16, "f32", "heads"),
    ([(60, 90)], 2, 1, 128, 9, "f32", "heads"),
    ([(30, 70), (1, 300)], 4, 2, 256, 32, "f32", "heads"),
    ([(1, 333), (4, 4)], 8, 4, 256, 16, "f32", "heads"),
    ([(33, 200)], 3, 3, 32, 64, "f32", "slots"),
    ([(40, 100)], 2, 1, 192, 4, "f32", "heads"),
    ([(5, 400)], 4, 1, 96, 8, "f32", "heads"),
    ([(1, 9)] * 70 + [(3, 60)] * 70, 2, 1, 64, 16, "bf16", "heads"),
]


@pytest.mark.parametrize("mask", MASKS, ids=[f"{'causal' if c else 'frame'}{w}" for c, w in MASKS])
@pytest.mark.parametrize("case", ATTENDS, ids=[f"{i}" for i in range(len(ATTENDS))])
def test_attention(case, mask):
    lens, heads, kv_heads, dim, page, dtype, order = case
    rng = _rng(31 + dim + page + len(lens))
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, lens, heads, kv_heads, dim, page, dtype, order)
    want = O.attend(q64, k64, v64, table, starts, length, *mask)
    for hint, out, lse in _attend_both(cache, q, table, starts, length, causal=mask[0], window=mask[1]):
        say(f"[attention] lens={lens[:5]} {case[1:]} mask={mask} max_new={hint}")
        _compare(out, lse, want, dtype, dim)


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 50), ("f32", 1), ("f32", 50)])
def test_more_rows_than_tokens(dtype, new):
    """Rows at positions before the sequence's begin see nothing."""
    rng = _rng(41)
    lens = [(new + 9, 9 if new == 1 else 30), (4, 0), (2, 2)]
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, lens, 4, 2, 64, 16, dtype)
    for mask in ((True, -1), (False, -1), (False, 5), (True, 2)):
        want = O.attend(q64, k64, v64, table, starts, length, *mask)
        for _, out, lse in _attend_both(cache, q, table, starts, length, causal=mask[0], window=mask[1]):
            _compare(out, lse, want, dtype, 64)


@pytest.mark.parametrize("window", [(1 << 30) - 1, (1 << 31) - 4, (1 << 31) - 1])
@pytest.mark.parametrize("dtype,new,kv", [("bf16", 6, 4), ("bf16", 50, 30), ("bf16", 300, 200), ("f32", 6, 4), ("f32", 50, 30)])
def test_windows_past_every_length(dtype, new, kv, window):
    """A window that no sequence is as long as hides nothing, also where rows lie before the sequence's begin."""
    rng = _rng(50)
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, [(new, kv), (2, 9), (4, 1)], 4, 2, 64, 16, dtype)
    for causal in (True, False):
        want = O.attend(q64, k64, v64, table, starts, length, causal, window)
        for hint, out, lse in _attend_both(cache, q, table, starts, length, causal=causal, window=window):
            say(f"[window] {dtype} new={new} kv={kv} window={window} causal={causal} max_new={hint}")
            _compare(out, lse, want, dtype, 64)


def test_numbers_past_32_bits():
    """Windows and hints that a description's 32-bit field does not hold mean what they say."""
    rng = _rng(51)
    cache, _, _, q, _, table, starts, length = _filled(rng, [(6, 90), (2, 9)], 4, 2, 64, 16, "bf16")
    batch = _device(table, starts, length)
    for causal in (True, False):
        whole = cache.attend(q, batch, causal=causal)
        for window in (1 << 31, 1 << 32, (1 << 33) + 5, -(1 << 31) - 1, -(1 << 40)):
            assert torch.equal(cache.attend(q, batch, causal=causal, window=window), whole), window
        for most in (1 << 31, (1 << 32) + 1, 1 << 40):
            assert torch.equal(cache.attend(q, _device(table, starts, length, max_new=most), causal=causal), whole), most


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,lens,heads", [("bf16", [(3, 100), (1, 70)], 4), ("bf16", [(90, 150)], 4), ("f32", [(3, 100), (1, 70)], 4), ("f32", [(90, 150)], 4)])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, lens, heads, value):
    """Keys and values of later tokens, and of tokens outside the window, that are not finite; a value that is seen arrives."""
    rng = _rng(42)

    def spoil(kp, vp, table):
        kv = lens[0][1]
        for at in (kv - 1, kv - 2, 0, 40):  # the newest tokens, and two that a window hides
            vp[table[0, at // 16], :, at % 16, 3:9] = value
        kp[table[0, (kv - 1) // 16], :, (kv - 1) % 16, 5] = value
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, lens, heads, 2, 64, 16, dtype, spoil=spoil)
    for mask in ((True, 20), (True, -1), (False, 20)):
        with np.errstate(all="ignore"):
            o, l, b = O.attend(q64, k64, v64, table, starts, length, *mask)  # noqa: E741
        for _, out, lse in _attend_both(cache, q, table, starts, length, causal=mask[0], window=mask[1]):
            got = out.double().cpu().numpy()
            # rows whose seen keys and values are finite: as ever
            clean = np.isfinite(o).all((1, 2)) & np.isfinite(l).all(1)
            assert clean.sum() >= (len(o) - 3 if mask == (True, 20) else 1 if len(lens) > 1 else 0)
            _compare(out[torch.from_numpy(clean).cuda()], lse[torch.from_numpy(clean).cuda()],
                     (o[clean], l[clean], {k: x[clean] for k, x in b.items()}), dtype, 64)
            # rows that see such a value but no such key: not finite there, finite elsewhere
            seen = ~np.isfinite(o).all((1, 2)) & np.isfinite(l).all(1)
            assert not np.isfinite(got[seen][..., 3:9]).any() and np.isfinite(got[seen][..., 9:]).all()


@pytest.mark.parametrize("dtype,new,kv", [("bf16", 1, 40), ("bf16", 1, 6000), ("bf16", 9, 6000), ("bf16", 50, 300), ("bf16", 200, 900),
                                          ("f32", 1, 6000), ("f32", 40, 3000)])
def test_scores_that_are_nan_stay_nan(dtype, new, kv):
    """A query that is NaN, or a key that a row sees, makes the whole row NaN (its sum of exponentials is), and no other row."""
    rng = _rng(48)

    def spoil(kp, vp, table):
        kp[table[1, 0], 1, 2, 7] = np.nan  # token 2 of the second sequence, key head 1
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, [(new, kv), (new, kv)], 4, 2, 64, 16, dtype, spoil=spoil)
    q[new - 1, 3] = float("nan")  # the first sequence's last row, one head
    q64[new - 1, 3] = np.nan
    with np.errstate(all="ignore"):
        o, l, b = O.attend(q64, k64, v64, table, starts, length)  # noqa: E741
    bad = np.isnan(l)
    assert bad[new - 1, 3] and bad[new:, 2:].all() and bad.sum() == 1 + 2 * new
    for _, out, lse in _attend_both(cache, q, table, starts, length):
        got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.repeat(bad[..., None], 64, 2)) and np.array_equal(np.isnan(gl), bad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 40])
def test_scores_of_great_range(dtype, new):
    """Scores from -1000 to 1000: the running reference moves, small exponentials vanish."""
    rng = _rng(43)
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, [(new, 700), (new, 200)], 2, 1, 64, 16, dtype, gain=100.0)
    want = O.attend(q64, k64, v64, table, starts, length)
    for _, out, lse in _attend_both(cache, q, table, starts, length):
        _compare(out, lse, want, dtype, 64)


@pytest.mark.parametrize("dtype,new,kv", [("bf16", 1, 9001), ("bf16", 3, 20000), ("bf16", 100, 3333), ("f32", 1, 9001), ("f32", 33, 2500)])
def test_keys_split_over_workgroups(dtype, new, kv):
    """One long sequence beside short ones: its keys are split, theirs are not."""
    rng = _rng(44)
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, [(new, 60), (new, kv), (1, 1)], 4, 2, 64, 32, dtype)
    for mask in ((True, -1), (False, 5000)):
        want = O.attend(q64, k64, v64, table, starts, length, *mask)
        for hint, out, lse in _attend_both(cache, q, table, starts, length, causal=mask[0], window=mask[1]):
            say(f"[split] {dtype} new={new} kv={kv} max_new={hint}")
            _compare(out, lse, want, dtype, 64)


@pytest.mark.parametrize("case", [(90, 1, 1500, 4, 2, 128, "bf16"), (70, 9, 1200, 6, 3, 80, "bf16"), (70, 2, 900, 8, 2, 256, "bf16"), (100, 1, 1300, 2, 1, 32, "bf16"),
                                  (20, 5, 2500, 4, 4, 96, "bf16"), (66, 17, 500, 4, 2, 64, "f32"), (70, 12, 400, 3, 1, 256, "f32"), (70, 2, 700, 4, 2, 128, "f32"),
                                  (2, 1000, 1000, 64, 8, 32, "bf16")], ids=lambda c: "-".join(map(str, c)))
def test_keys_shared_by_workgroups(case):
    """Sequences of all lengths, some empty, none of which has a whole number of shares: a workgroup's keys begin and end inside them."""
    count, new, kv, heads, kv_heads, dim, dtype = case
    rng = _rng(46 + count + dim)
    lens = [(new, kv), (0, 5), (min(new, 3), 3)]
    while len(lens) < count + 1:
        n = int(rng.integers(0, new + 1))
        lens.append((n, int(rng.integers(n, kv + 1))))
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, lens, heads, kv_heads, dim, 16, dtype)
    for mask in ((True, -1), (False, kv // 2)):
        want = O.attend(q64, k64, v64, table, starts, length, *mask)
        for hint, out, lse in _attend_both(cache, q, table, starts, length, causal=mask[0], window=mask[1]):
            say(f"[shares] {case} mask={mask} max_new={hint}")
            _compare(out, lse, want, dtype, dim)


def _dense(q64, k64, v64, table, starts, length, causal, window):
    """The oracle's attend() as dense products in 64 bits, sequence by sequence and head by head, for calls of many rows. The fourth result
    says which outputs see a value that is not finite (they count as zero in the others)."""
    tokens, heads, dim = q64.shape
    kv_heads, page = k64.shape[1], k64.shape[2]
    group = heads // kv_heads
    f64 = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out, weight, odd = f64(tokens, heads, dim), f64(tokens, heads, dim), f64(tokens, heads, dim)
    lse, size, most, count = f64(tokens, heads) - math.inf, f64(tokens, heads), f64(tokens, heads), f64(tokens, heads)
    for b, kv in enumerate(int(x) for x in length):
        t0, n = int(starts[b]), int(starts[b + 1] - starts[b])
        if n == 0 or kv == 0:
            continue
        held = table[b, :-(-kv // page)]
        at, col = kv - n + torch.arange(n, device="cuda")[:, None], torch.arange(kv, device="cuda")
        sees = col <= at if causal else (col >= 0).expand(n, kv)
        if window >= 0:
            sees = sees & (col >= (at if causal else kv - n) - window)
        for g in range(kv_heads):
            keys, values = (torch.from_numpy(x[held, g].reshape(-1, dim)[:kv]).cuda() for x in (k64, v64))
            fine = torch.isfinite(values)
            values = torch.where(fine, values, torch.zeros_like(values))
            for h in range(g * group, (g + 1) * group):
                q, rows = torch.from_numpy(q64[t0:t0 + n, h]).cuda(), slice(t0, t0 + n)
                score = dim ** -0.5 * (q @ keys.T)
                hidden = score.masked_fill(~sees, -math.inf)
                top = hidden.amax(1, keepdim=True).nan_to_num(neginf=0.0)
                e = (hidden - top).exp()
                total = e.sum(1, keepdim=True)
                scale = 1 / total.clamp(min=1e-300)
                out[rows, h], weight[rows, h] = e @ values * scale, e @ values.abs() * scale
                odd[rows, h] = sees.double() @ (~fine).double()
                lse[rows, h] = (top + total.log())[:, 0]
                size[rows, h] = (dim ** -0.5 * (q.abs() @ keys.abs().T)).masked_fill(~sees, 0.0).amax(1)
                most[rows, h] = score.abs().masked_fill(~sees, 0.0).amax(1)
                count[rows, h] = sees.sum(1).double()
    np_of = lambda x: x.cpu().numpy()  # noqa: E731
    return np_of(out), np_of(lse), {"weight": np_of(weight), "size": np_of(size), "most": np_of(most), "count": np_of(count)}, np_of(odd) > 0


@pytest.mark.parametrize("mask", MASKS, ids=[f"{'causal' if c else 'frame'}{w}" for c, w in MASKS])
def test_the_dense_oracle(mask):
    rng = _rng(56)
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, [(9, 5), (17, 60), (0, 8), (30, 30)], 6, 3, 24, 7, "f32")
    want, got = O.attend(q64, k64, v64, table, starts, length, *mask), _dense(q64, k64, v64, table, starts, length, *mask)
    for a, b in zip((want[0], want[1], *want[2].values()), (got[0], got[1], *got[2].values())):
        assert np.allclose(a, b, rtol=1e-11, atol=1e-11)
    assert not got[3].any()


# Calls of which a workgroup takes 256 rows of a key head: bf16 heads of up to 64, and as many such units as half of what fits the GPU.
# lens, heads, kv heads, dim, page, order, the form that the lengths give
DOUBLE = [
    ([(530, 700), (530, 640)], 64, 8, 64, 16, "heads", "short"),
    ([(530, 690), (530, 531)], 64, 8, 40, 7, "slots", "short"),
    ([(1040, 600), (3, 80)], 64, 8, 64, 16, "heads", "short"),
    ([(1100, 1500), (1, 900)], 64, 8, 64, 16, "slots", "shared"),
    ([(1024, 1537)], 64, 8, 32, 16, "heads", "shared"),
    ([(600, 1201), (0, 40), (530, 531)], 64, 8, 40, 7, "heads", "shared"),
    ([(1060, 2000)], 64, 8, 64, 9, "heads", "shared"),
    ([(2100, 2111)], 64, 8, 64, 16, "heads", "many"),
    ([(1050, 1900), (1060, 1063)], 64, 8, 32, 5, "slots", "many"),
]


def _double_case(rng, case, spoil=None):
    """The case's tensors; checked that it is what it says."""
    lens, heads, kv_heads, dim, page, order, form = case
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, lens, heads, kv_heads, dim, page, "bf16", order, spoil=spoil)
    rows = q.shape[0] * heads // kv_heads
    assert (rows >> 8) * kv_heads >= 256 and dim <= 64
    batch = _device(table, starts, length)
    a = S.skipconv_attend(None, None, None, *(heads * dim, dim) * 2, heads, 1, -1, 0.1, 0)
    room = {"short": table.shape[1] * page <= 768, "shared": table.shape[1] * page > 768, "many": True}
    few_units = ((rows >> 8) + min(len(lens), q.shape[0])) * kv_heads < 512
    assert room[form] and few_units == (form != "many")
    c = cache.desc(batch, q.shape[0])
    assert (A.skipconv_attend_workspace(c, a) > 0) == (form == "shared")
    if form != "many":  # the parts that a longer table takes show the rows of a unit
        c.table_width = 1 << 20
        assert A.skipconv_attend_workspace(c, a) == 2 * 512 * 256 * (dim + 2) * 4
    return cache, k64, v64, q, q64, table, starts, length


@pytest.mark.parametrize("mask", [(True, -1), (False, -1), (True, 200), (False, 333), (True, 0)], ids=lambda m: f"{'causal' if m[0] else 'frame'}{m[1]}")
@pytest.mark.parametrize("case", DOUBLE, ids=[f"{i}-{c[-1]}" for i, c in enumerate(DOUBLE)])
def test_two_row_blocks_a_wave(case, mask):
    cache, k64, v64, q, q64, table, starts, length = _double_case(_rng(57 + case[3] + case[4]), case)
    want = _dense(q64, k64, v64, table, starts, length, *mask)[:3]
    for hint, out, lse in _attend_both(cache, q, table, starts, length, causal=mask[0], window=mask[1]):
        say(f"[two blocks] {case} mask={mask} max_new={hint}")
        _compare(out, lse, want, "bf16", case[3])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("case", [DOUBLE[0], DOUBLE[1], DOUBLE[3], DOUBLE[7]], ids=lambda c: f"{c[-1]}-{c[3]}")
def test_two_row_blocks_a_wave_and_values_that_are_not_finite(case, value):
    """The newest tokens', which a causal mask hides from earlier rows, and ones that a window hides."""
    lens, dim = case[0], case[3]

    def spoil(kp, vp, table):
        kv, page = lens[0][1], case[4]
        for at in (kv - 1, kv - 2, kv - 300, 40, 0):
            vp[table[0, at // page], :, at % page, 3:9] = value
    cache, k64, v64, q, q64, table, starts, length = _double_case(_rng(58 + dim), case, spoil)
    for mask in ((True, -1), (True, 150), (False, 100)):
        o, l, b, odd = _dense(q64, k64, v64, table, starts, length, *mask)  # noqa: E741
        assert odd.any() and not odd.all() and not odd[..., 9:].any()
        for hint, out, lse in _attend_both(cache, q, table, starts, length, causal=mask[0], window=mask[1]):
            say(f"[two blocks, {value}] {case} mask={mask} max_new={hint}")
            got = torch.from_numpy(odd).cuda()
            assert not torch.isfinite(out[got]).any()
            _compare(out.masked_fill(got, 0.0), lse, (np.where(odd, 0.0, o), l, b), "bf16", dim)


def test_scale_strides_and_out():
    rng = _rng(45)
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, [(20, 90), (3, 64)], 4, 2, 64, 16, "bf16")
    want = O.attend(q64, k64, v64, table, starts, length, True, -1, 0.31)
    batch = _device(table, starts, length)
    wide = torch.full((23 + 2, 9, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    queries = _laid(torch.cat([q, q[:2]]), "heads")  # two rows of no sequence
    got, lse = cache.attend(queries, batch, scale=0.31, out=wide[:, 2:6], return_lse=True)
    assert got.data_ptr() == wide[:, 2:6].data_ptr()
    _compare(got[:23], lse[:23], want, "bf16", 64)
    assert (wide[:, :2] == 5.0).all() and (wide[:, 6:] == 5.0).all() and (wide[23:] == 5.0).all()


@pytest.mark.parametrize("dtype,group", [("bf16", 4), ("bf16", 40), ("f32", 4), ("f32", 40)])
def test_strides_of_dimensions_of_one_place(dtype, group):
    """One token, one key head, one page, or pages of one slot: the stride there may be any number, as a slice of a projection leaves it."""
    rng = _rng(55)

    def any_stride(x):
        """The tensor with each stride of a dimension of one place no multiple of 16 bytes."""
        return x.as_strided(x.shape, [s if n > 1 else 1001 + i for i, (n, s) in enumerate(zip(x.shape, x.stride()))])
    for lens, page in (([(1, 40)], 64), ([(1, 9)], 1), ([(1, 40)], 16)):
        cache, k64, v64, q, q64, table, starts, length = _filled(rng, lens, group, 1, 64, page, dtype)
        want = O.attend(q64, k64, v64, table, starts, length)
        keep = cache.k_pages[table[0, 0]:][:1], cache.v_pages[table[0, 0]:][:1]
        if page == 64:  # a cache of one page
            cache, table = A.PagedCache(*(any_stride(x.contiguous()) for x in keep)), np.zeros_like(table)
        else:
            cache = A.PagedCache(any_stride(cache.k_pages), any_stride(cache.v_pages))
        batch, out = _device(table, starts, length), torch.empty_like(q)
        for src in (any_stride(q), any_stride(q.repeat(2, 1, 1)[:1])):
            got, lse = cache.attend(src, batch, out=any_stride(out), return_lse=True)
            _compare(got, lse, want, dtype, 64)
        # appending the token again, and the rotation: as with packed strides
        rotary, pos = A.Rotary(A.axis_frequencies((16, 16)), 64), torch.ones(1, 2, dtype=torch.int32, device="cuda")
        k, v = q[:, :1], q[:, 1:2]
        turned = rotary.rotate(q, pos)
        assert torch.equal(rotary.rotate(any_stride(q), pos, out=any_stride(out)), turned)
        assert torch.equal(cache.append(any_stride(k), any_stride(v), batch, rotary=rotary, pos=pos, q=any_stride(q)), turned)
        at = int(length[0]) - 1
        assert torch.equal(cache.k_pages[table[0, at // page], 0, at % page], turned[0, 0]) and torch.equal(cache.v_pages[table[0, at // page], 0, at % page], v[0, 0])


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 40), ("f32", 1), ("f32", 40)])
def test_offsets_past_32_bits(dtype, new):
    """Pages whose element offsets pass 2^32."""
    rng = _rng(46)
    pages, kv_heads, page, dim = (1 << 32) // (2 * 16 * 64) + 64, 2, 16, 64
    kp, vp = (torch.empty((pages, kv_heads, page, dim), dtype=DT[dtype], device="cuda") for _ in range(2))
    cache = A.PagedCache(kp, vp)
    table, starts, length, _ = _batch(rng, [(new, 100)], page, pages_first=pages - 16)
    k, k64 = _stored(rng.standard_normal((100, kv_heads, dim)), dtype)
    v, v64 = _stored(rng.standard_normal((100, kv_heads, dim)), dtype)
    cache.append(k, v, _device(table, np.array([0, 100], np.int32), length))
    q, q64 = _stored(rng.standard_normal((new, 4, dim)), dtype)
    k_pages, v_pages = (np.full((16, kv_heads, page, dim), np.nan) for _ in range(2))
    k_pages, v_pages = O.append(k_pages, v_pages, k64, v64, table - (pages - 16), [0, 100], length)
    want = O.attend(q64, k_pages, v_pages, table - (pages - 16), starts, length)
    for _, out, lse in _attend_both(cache, q, table, starts, length):
        _compare(out, lse, want, dtype, dim)


def test_another_stream_and_graph_replays():
    """A step (append, attend) on a stream of its own, then captured and replayed with new inputs in between."""
    rng = _rng(47)
    lens = [(1, 400), (1, 33)]
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, lens, 8, 2, 64, 16, "bf16")
    batch = _device(table, starts, length, max_new=1)
    freq, pos = A.axis_frequencies((11, 11, 10)), torch.tensor([[3, 2, 1], [1, 1, 9]], dtype=torch.int32, device="cuda")
    rotary = A.Rotary(freq, 64)
    k, v = (torch.randn(2, 2, 64, device="cuda").bfloat16() for _ in range(2))

    def step():
        return cache.attend(cache.append(k, v, batch, rotary=rotary, pos=pos, q=q), batch, return_lse=True)
    eager = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = step()
    side.synchronize()
    assert torch.equal(eager[0], other[0]) and torch.equal(eager[1], other[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in held]
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), f"replay {i}"


def test_the_tensors_device_is_current_in_every_call(monkeypatch):
    """With another device current, a call makes the tensors' device the current one around its launch, and leaves it afterwards."""
    rng = _rng(52)
    cache, _, _, q, _, table, starts, length = _filled(rng, [(2, 40)], 4, 2, 64, 16, "bf16")
    batch, rotary = _device(table, starts, length), A.Rotary(A.axis_frequencies((16, 16)), 64)
    pos = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    entered = []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            entered.append(self.index)

        def __exit__(self, *_):
            entered.append("left")
    calls = (lambda: rotary.rotate(q, pos), lambda: cache.append(q[:, :2], q[:, 2:], batch, rotary=rotary, pos=pos, q=q), lambda: cache.attend(q, batch))
    for call in calls:  # as it is: nothing to do
        call()
    monkeypatch.setattr(torch.cuda, "device", Device)
    for call in calls:
        call()
    assert entered == []
    monkeypatch.setattr(A, "_current", lambda: 1, raising=False)
    for call in calls:
        call()
        assert entered == [0, "left"]
        entered.clear()
    with pytest.raises(S.SkipConvError):
        cache.attend(q, batch, scale=0.0)
    assert entered == [0, "left"]


def test_what_a_description_holds_is_not_replaced():
    """Tensors and sizes whose addresses and values were taken once; their values are written in place, and the next call reads those."""
    rng = _rng(53)
    cache, k64, v64, q, q64, table, starts, length = _filled(rng, [(1, 40)], 4, 2, 64, 16, "bf16")
    batch, rotary = _device(table, starts, length), A.Rotary(A.axis_frequencies((16, 16)), 64)
    for held, names in ((batch, ("page_table", "row_start", "kv_len", "sequences")), (rotary, ("freq", "axes", "pairs", "head_dim", "pairing")),
                        (cache, ("k_pages", "v_pages", "pages", "kv_heads", "page_size", "head_dim", "dtype"))):
        for name in names:
            value = getattr(held, name)
            with pytest.raises(AttributeError):
                setattr(held, name, value.clone() if torch.is_tensor(value) else value)
            assert getattr(held, name) is value
    batch.kv_len.fill_(17)
    out, lse = cache.attend(q, batch, return_lse=True)
    _compare(out, lse, O.attend(q64, k64, v64, table, starts, np.array([17], np.int32)), "bf16", 64)


def test_an_output_without_queries_is_refused():
    """Nothing would be written to it, and it would be returned as if."""
    cache, batch, rotary, pos, q = _small_call()
    for turn in ({}, dict(rotary=rotary, pos=pos)):
        with pytest.raises(ValueError, match="q_out"):
            cache.append(q[:, :2], q[:, 2:], batch, q_out=torch.empty_like(q), **turn)


def test_a_rotation_on_another_device_is_refused():
    """Its table would be read from a device that the cache is not on. (One device stands for two: the rotation is told another index.)"""
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    cache = A.PagedCache(k, k.clone())
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    batch, rotary, pos = A.CacheBatch(ints(0, 1)[None], ints(0, 1), ints(5)), A.Rotary(A.axis_frequencies((16, 16)), 64), ints(1, 2)[None]

    class Elsewhere:
        dtype, shape = pos.dtype, pos.shape
        is_contiguous, data_ptr = pos.is_contiguous, pos.data_ptr

        def get_device(self):
            return 1
    rotary._index = 1
    kv = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="another device"):
        cache.append(kv, kv, batch, rotary=rotary, pos=Elsewhere())


def test_refusals():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    cache = A.PagedCache(k, k.clone())
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = A.CacheBatch(ints(0, 1)[None], ints(0, 1), ints(5))
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    kv = q[:, :2]
    rotary = A.Rotary(A.axis_frequencies((16, 16)), 64)
    pos = ints(1, 2)[None]
    for bad in (lambda: A.PagedCache(k, k.float()), lambda: A.PagedCache(k[0], k[0]), lambda: A.PagedCache(k.half(), k.half()),
                lambda: A.PagedCache(k.cpu(), k.cpu()), lambda: A.PagedCache(k.transpose(2, 3), k.transpose(2, 3)),
                lambda: A.CacheBatch(ints(0, 1), ints(0, 1), ints(5)), lambda: A.CacheBatch(ints(0, 1)[None], ints(0), ints(5)),
                lambda: A.CacheBatch(ints(0, 1)[None].long(), ints(0, 1), ints(5)), lambda: A.CacheBatch(ints(0, 1)[None], ints(0, 1), ints(5), max_new=-1),
                lambda: A.Rotary(A.axis_frequencies((33,)), 64), lambda: A.Rotary(A.axis_frequencies((8,)), 64, "pairs"),
                lambda: A.Rotary(A.axis_frequencies((8,)).double(), 64), lambda: A.Rotary(A.axis_frequencies((8,)).cpu(), 64),
                lambda: rotary.rotate(q, pos[:, :1]), lambda: rotary.rotate(q, pos.long()), lambda: rotary.rotate(q[..., :32], pos),
                lambda: rotary.rotate(q.half(), pos), lambda: rotary.rotate(q, pos, out=q.float()), lambda: rotary.rotate(q.transpose(1, 2), pos),
                lambda: cache.append(kv, kv[:, :1], batch), lambda: cache.append(kv, kv, batch, rotary=rotary), lambda: cache.append(kv, kv, batch, q=q),
                lambda: cache.append(kv.float(), kv.float(), batch), lambda: cache.append(kv, kv, batch, rotary=A.Rotary(A.axis_frequencies((8,)), 32), pos=pos[:, :1]),
                lambda: cache.attend(q.float(), batch), lambda: cache.attend(q[..., :32], batch), lambda: cache.attend(q[0], batch),
                lambda: cache.attend(q, batch, out=q.float())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: cache.attend(q[:, :3], batch), lambda: cache.attend(q, batch, scale=0.0),
                lambda: cache.attend(torch.zeros(1 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")[4:-4].view(1, 4, 64), batch)):
        with pytest.raises(S.SkipConvError) as e:
            bad()
        assert e.value.code == S.SKIPCONV_E_INVALID_ARG
    out, lse = cache.attend(q, A.CacheBatch(ints(0, 1)[None], ints(0, 1), ints(0)), return_lse=True)
    assert not out.any() and torch.isneginf(lse).all()


def test_frames_of_skip_conv_layers():
    """The example's path: Skip-Conv projections, append and attention frame by frame with a window of frames that rolls, against the
    oracle on the layers' own activation outputs."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "frame_attention.py")
    spec = importlib.util.spec_from_file_location("frame_attention", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    rng = _rng(49)
    n, h, w, c, dim, heads, kv_heads, history = 2, 8, 12, 32, 32, 4, 2, 2
    weights = [_stored(rng.standard_normal((k * dim, c, 1, 1)) * (2 / c) ** 0.5, "bf16")[0] for k in (heads, kv_heads, kv_heads)]
    model = example.FrameAttention(weights, n=n, h=h, w=w, head_dim=dim, history=history, eps=0.5, block=4, page_size=32)
    base = rng.random((n, h, w, c))
    past = []
    for t in range(5):
        frame = base.copy()
        frame[:, t:t + 3, 2 * t:2 * t + 4] = rng.random((n, min(3, h - t), 4, c))
        out = model.step(_stored(frame, "bf16")[0])
        q, k, v = (layer.activation().double().cpu().numpy().reshape(n * h * w, -1, dim) for layer in model.layers)
        pos, freq = model.pos.cpu().numpy(), model.rotary.freq.cpu().double().numpy()
        assert (pos[:, 0] == t).all()
        turn = lambda x: torch.from_numpy(O.rotate(x, pos, freq)).bfloat16().double().numpy()  # noqa: E731
        past.append((turn(k), v))
        past = past[-(history + 1):]
        keys, values = (np.concatenate([p[i].reshape(n, h * w, kv_heads, dim) for p in past], 1) for i in (0, 1))
        length = np.full(n, keys.shape[1])
        pages = lambda x: x.transpose(0, 2, 1, 3)  # noqa: E731  (one page a stream)
        want = O.attend(turn(q), pages(keys), pages(values), np.arange(n)[:, None], np.arange(n + 1) * h * w, length, False, -1)
        # keys and queries that a rounding of the turned value takes to its neighbour move a score by up to 2^-8 of each term
        o, _, b = want
        got = out.double().cpu().numpy().reshape(n * h * w, heads, dim)
        bound = 2.0 ** -8 * np.abs(o) + b["weight"] * (2.0 ** -8 + np.expm1(2 * 2.0 ** -8 * b["size"])[..., None] * 2)
        assert (np.abs(got - o) <= 1.25 * bound).all()
