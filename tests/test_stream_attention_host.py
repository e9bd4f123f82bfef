"""Streaming attention on the CPU: the oracle against independent forms (complex products, a dense softmax, differences), and the
refusals of the entry points, which come before any GPU work."""
import ctypes
import math

import numpy as np
import pytest

from oracle import stream_attention_oracle as O
from paper_2104_11487_amd import skipconv as S


def _rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


# ------------------------------------------------------------------ oracle --

@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_is_a_complex_product(adjacent):
    rng = _rng(1)
    x, pos, freq = rng.standard_normal((5, 3, 22)), rng.integers(-9, 200, (5, 3)), rng.random((3, 9))
    y = O.rotate(x, pos, freq, adjacent)
    first, second = O.partners(9, adjacent)
    z = (x[..., first] + 1j * x[..., second]) * np.exp(1j * (pos @ freq))[:, None]
    assert np.allclose(y[..., first], z.real, atol=1e-12) and np.allclose(y[..., second], z.imag, atol=1e-12)
    assert np.array_equal(y[..., 18:], x[..., 18:])


def test_rotation_depends_on_distance_only_and_turns_back():
    rng = _rng(2)
    q, k, freq = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16)), rng.random((3, 8))
    pos, other, shift = (rng.integers(0, 50, (1, 3)) for _ in range(3))
    dot = lambda a, b: float((a * b).sum())  # noqa: E731
    one = dot(O.rotate(q, pos, freq), O.rotate(k, other, freq))
    two = dot(O.rotate(q, pos + shift, freq), O.rotate(k, other + shift, freq))
    assert abs(one - two) < 1e-10
    assert np.allclose(O.rotate(O.rotate(q, pos, freq), pos, freq, inverse=True), q, atol=1e-12)


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_gradient_against_differences(adjacent):
    rng = _rng(3)
    x, pos, freq, dy = rng.standard_normal((2, 2, 10)), rng.integers(0, 30, (2, 2)), rng.random((2, 4)), rng.standard_normal((2, 2, 10))
    dx = O.rotate(dy, pos, freq, adjacent, inverse=True)
    step = 1e-5
    for at in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[at] = step
        d = ((O.rotate(x + e, pos, freq, adjacent) - O.rotate(x - e, pos, freq, adjacent)) * dy).sum() / (2 * step)
        assert abs(d - dx[at]) < 1e-8


@pytest.mark.parametrize("causal,window", [(True, -1), (True, 3), (True, 0), (False, -1), (False, 2)])
def test_attention_is_a_masked_softmax(causal, window):
    rng = _rng(4)
    n, length, dim, page, heads, kv_heads = 5, 13, 8, 4, 4, 2
    table = rng.permutation(8)[None, :4]
    kp, vp = rng.standard_normal((8, kv_heads, page, dim)), rng.standard_normal((8, kv_heads, page, dim))
    q = rng.standard_normal((n, heads, dim))
    out, lse, _ = O.attend(q, kp, vp, table, [0, n], [length], causal, window)
    keys = np.concatenate([kp[p] for p in table[0]], 1)[:, :length].repeat(2, 0)  # heads x length x dim
    values = np.concatenate([vp[p] for p in table[0]], 1)[:, :length].repeat(2, 0)
    s = np.einsum("ihd,hld->hil", q, keys) / math.sqrt(dim)
    row, col = np.arange(n)[:, None] + length - n, np.arange(length)[None]
    ok = (col <= row) if causal else np.ones((n, length), bool)
    if window >= 0:
        ok &= col >= (row if causal else length - n) - window
    s = np.where(ok, s, -np.inf)
    p = np.exp(s) / np.exp(s).sum(-1, keepdims=True)
    assert np.allclose(out, np.einsum("hil,hld->ihd", p, values), atol=1e-12)
    assert np.allclose(lse, np.log(np.exp(s).sum(-1)).T, atol=1e-12)


def test_a_row_that_sees_nothing_and_unseen_values():
    rng = _rng(5)
    kp, vp = rng.standard_normal((2, 1, 4, 8)), rng.standard_normal((2, 1, 4, 8))
    vp[0, 0, 3] = np.nan  # token 3: seen by the last row only
    kp[1] = np.inf        # past the sequence
    q = rng.standard_normal((6, 1, 8))
    out, lse, _ = O.attend(q, kp, vp, np.array([[0, 1]]), [0, 6], [4])  # six rows for four tokens: two see nothing
    assert not out[:2].any() and np.isneginf(lse[:2]).all()
    assert np.isfinite(out[2:5]).all() and np.isnan(out[5]).all()


def test_append_places():
    table = np.array([[3, 1, 9], [-1, 2, 0]])
    got = O.places(table, [0, 3, 7], [5, 10], 4, 4)
    # sequence 0: tokens 2, 3 | 4; sequence 1: tokens 6, 7 | 8, 9
    assert got == [(0, 3, 2), (1, 3, 3), (2, 1, 0), (3, 2, 2), (4, 2, 3), (5, 0, 0), (6, 0, 1)]
    assert O.places(table, [0, 2, 2], [1, 0], 4, 4) == [(1, 3, 0)]  # a token before the sequence's begin has no place
    assert O.places(table, [0, 2, 2], [13, 0], 4, 4) == []          # pages 9 and past the table


# ---------------------------------------------------------------- refusals --

A = 1 << 20  # an aligned address that no call may reach


def _rotary(**kw):
    r = S.skipconv_rotary(A, A, 3, 16, 0, 0)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _rotate(r, tokens=4, heads=2, dim=32, dtype=1, x=A, xs=(64, 32), y=2 * A, ys=(64, 32)):
    return S.lib().skipconv_rotate(ctypes.byref(r), tokens, heads, dim, dtype, x, *xs, y, *ys, None)


def _cache(**kw):
    c = S.skipconv_cache(A, A, 4 * 16 * 64, 16 * 64, 64, 4 * 16 * 64, 16 * 64, 64, A, A, A, 8, 2, 4, 32, 16, 4, 64, 1)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _attend(**kw):
    a = S.skipconv_attend(A, 2 * A, None, 512, 64, 512, 64, 8, 1, -1, 0.125, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _append(**kw):
    a = S.skipconv_append(A, A, None, None, 256, 64, 256, 64, 512, 64, 512, 64, 8, None)
    r = _rotary(pairs=32)
    a._keep = r
    a.rotary = ctypes.pointer(r)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


INVALID, UNSUPPORTED, SMALL = S.SKIPCONV_E_INVALID_ARG, S.SKIPCONV_E_UNSUPPORTED, S.SKIPCONV_E_SMALL_BUFFER


@pytest.mark.parametrize("rotary,call,code", [
    (dict(axes=0), {}, INVALID), (dict(axes=9), {}, INVALID), (dict(pairs=0), {}, INVALID), (dict(pairs=17), {}, INVALID),
    (dict(pairing=2), {}, INVALID), (dict(inverse=2), {}, INVALID), (dict(freq=None), {}, INVALID), (dict(pos=None), {}, INVALID),
    ({}, dict(dtype=2), INVALID), ({}, dict(tokens=-1), INVALID), ({}, dict(heads=-1), INVALID), ({}, dict(dim=1025), UNSUPPORTED),
    ({}, dict(dim=1), UNSUPPORTED), ({}, dict(tokens=1 << 31), UNSUPPORTED), ({}, dict(x=None), INVALID), ({}, dict(y=None), INVALID),
    ({}, dict(x=A, y=A, ys=(128, 32)), INVALID), ({}, dict(ys=(0, 32)), INVALID), ({}, dict(ys=(64, 0)), INVALID), ({}, dict(x=A + 1), INVALID),
])
def test_rotate_refusals(rotary, call, code):
    assert _rotate(_rotary(**rotary), **call) == code
    assert "rot" in S.skipconv_last_error()


def test_nothing_to_do():
    assert _rotate(_rotary(pos=None), tokens=0, x=None, y=None) == S.SKIPCONV_OK
    assert _rotate(_rotary(), heads=0) == S.SKIPCONV_OK
    lib = S.lib()
    for kw in (dict(tokens=0), dict(batch=0)):
        c = _cache(**kw)
        assert lib.skipconv_cache_append(ctypes.byref(c), ctypes.byref(_append()), None) == S.SKIPCONV_OK
        assert lib.skipconv_cache_attend(ctypes.byref(c), ctypes.byref(_attend()), None, 0, None) == S.SKIPCONV_OK
        n = ctypes.c_size_t(7)
        assert lib.skipconv_attend_workspace(ctypes.byref(c), ctypes.byref(_attend()), ctypes.byref(n)) == S.SKIPCONV_OK and n.value == 0


def test_a_batch_of_no_sequence_has_no_arrays():
    lib = S.lib()
    for tokens in (0, 8):
        c = _cache(batch=0, tokens=tokens, page_table=None, row_start=None, kv_len=None)
        assert lib.skipconv_cache_append(ctypes.byref(c), ctypes.byref(_append()), None) == S.SKIPCONV_OK
        assert lib.skipconv_cache_attend(ctypes.byref(c), ctypes.byref(_attend()), None, 0, None) == S.SKIPCONV_OK


CACHE = [
    (dict(dtype=2), INVALID), (dict(tokens=-1), INVALID), (dict(batch=-1), INVALID), (dict(kv_heads=0), INVALID), (dict(pages=0), INVALID),
    (dict(page_size=0), INVALID), (dict(table_width=0), INVALID), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED),
    (dict(head_dim=0), UNSUPPORTED), (dict(tokens=1 << 31), UNSUPPORTED), (dict(table_width=1 << 20, page_size=2048), UNSUPPORTED),
    (dict(k_slot=68), INVALID), (dict(v_page=-64), INVALID), (dict(k_head=4), INVALID),
    (dict(k_pages=None), INVALID), (dict(row_start=None), INVALID), (dict(kv_len=None), INVALID), (dict(page_table=None), INVALID),
    (dict(v_pages=A + 8), INVALID),
]


@pytest.mark.parametrize("kw,code", CACHE)
def test_cache_refusals(kw, code):
    lib, c = S.lib(), _cache(**kw)
    assert lib.skipconv_cache_append(ctypes.byref(c), ctypes.byref(_append()), None) == code
    assert "cache" in S.skipconv_last_error()
    assert lib.skipconv_cache_attend(ctypes.byref(c), ctypes.byref(_attend()), A, 1 << 40, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(q=A), INVALID), (dict(q=A, q_out=A, q_heads=0), INVALID),
    (dict(q=A, q_out=A, rotary=None), INVALID), (dict(q=A, q_out=A, q_out_token=1024), INVALID), (dict(q=A, q_out=2 * A, q_out_head=0), INVALID),
    (dict(k=A + 1), INVALID), (dict(rotary=ctypes.pointer(_rotary(pairs=33))), INVALID),
])
def test_append_refusals(kw, code):
    assert S.lib().skipconv_cache_append(ctypes.byref(_cache()), ctypes.byref(_append(**kw)), None) == code
    assert S.lib().skipconv_cache_append(None, ctypes.byref(_append()), None) == INVALID
    assert S.lib().skipconv_cache_append(ctypes.byref(_cache()), None, None) == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(q_heads=6), INVALID), (dict(q_heads=0), INVALID), (dict(causal=2), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(max_new=-1), INVALID), (dict(q=None), INVALID),
    (dict(out=None), INVALID), (dict(q=A + 8), INVALID), (dict(out=A + 2), INVALID), (dict(q_head=68), INVALID), (dict(out_token=12), INVALID),
    (dict(out_token=0), INVALID), (dict(out_head=0), INVALID), (dict(lse=A + 2), INVALID),
])
def test_attend_refusals(kw, code):
    assert S.lib().skipconv_cache_attend(ctypes.byref(_cache()), ctypes.byref(_attend(**kw)), A, 1 << 40, None) == code
    assert "attend" in S.skipconv_last_error()


def test_attend_workspace():
    lib, c, a, n = S.lib(), _cache(table_width=1024), _attend(), ctypes.c_size_t()  # 16384 keys a sequence: split
    assert lib.skipconv_attend_workspace(ctypes.byref(c), ctypes.byref(a), ctypes.byref(n)) == S.SKIPCONV_OK
    assert n.value > 0
    assert lib.skipconv_cache_attend(ctypes.byref(c), ctypes.byref(a), A, n.value - 1, None) == SMALL
    assert lib.skipconv_cache_attend(ctypes.byref(c), ctypes.byref(a), A + 4, n.value, None) == INVALID
    assert lib.skipconv_cache_attend(ctypes.byref(c), ctypes.byref(a), None, n.value, None) == INVALID
    assert lib.skipconv_attend_workspace(ctypes.byref(c), ctypes.byref(a), None) == INVALID
    assert lib.skipconv_attend_workspace(None, ctypes.byref(a), ctypes.byref(n)) == INVALID
    short = _cache()  # 512 keys a sequence at most: one workgroup an item
    assert lib.skipconv_attend_workspace(ctypes.byref(short), ctypes.byref(a), ctypes.byref(n)) == S.SKIPCONV_OK and n.value == 0
    c = _cache(tokens=1 << 20, batch=4)  # rows enough to fill the GPU: nothing is split
    assert lib.skipconv_attend_workspace(ctypes.byref(c), ctypes.byref(a), ctypes.byref(n)) == S.SKIPCONV_OK and n.value == 0
