"""The cache in 4 bits, accumulated weight and eviction on the CPU: the oracle against independent forms, and the refusals of the entry points,
which come before any GPU work."""
import ctypes
import math

import numpy as np
import pytest

from oracle import packed_cache_oracle as P
from oracle import stream_attention_oracle as O
from paper_2104_11487_amd import skipconv as S


def _rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


# ------------------------------------------------------------------ oracle --

@pytest.mark.parametrize("dim", [8, 32, 40, 96])
def test_a_held_element_is_within_half_a_step(dim):
    """By the format: half a step of (max - min) / 15, and the roundings of minimum, scale (15 of them) and value to fp16."""
    x = (_rng(1).standard_normal((50, dim)) * 3 + 1).astype(np.float32)
    codes, scales = P.pack(x)
    assert codes.shape == (50, 16 * -(-dim // 32)) and scales.shape == (50, -(-dim // 32), 2)
    back = P.values(codes, scales, dim)
    for g in range(0, dim, 32):
        part = x[:, g:g + 32].astype(np.float64)
        step = (part.max(1) - part.min(1)) / 15
        bound = 0.5 * step + 2.0 ** -11 * (2 * np.abs(part).max(1) + 16 * step)
        assert (np.abs(back[:, g:g + 32] - part) <= bound[:, None]).all()
    used = np.zeros((50, 32 * scales.shape[1]), bool)
    used[:, :dim] = True
    nibbles = np.stack([codes & 15, codes >> 4], -1).reshape(50, -1)
    assert not nibbles[~used].any() and (nibbles.max(1) == 15).all()


def test_what_is_on_the_grid_is_held_exactly():
    """Integers from -7 to 8: minimum -7, scale 1."""
    x = (np.arange(32) % 16 - 7).astype(np.float32)[None]
    codes, scales = P.pack(x)
    assert np.array_equal(P.values(codes, scales, 32), x) and scales.tolist() == [[[1.0, -7.0]]]
    assert codes[0].tolist() == [(2 * i % 16) | (2 * i + 1) % 16 << 4 for i in range(16)]


def test_elements_past_the_range_and_not_finite():
    x = np.zeros((3, 64), np.float32)
    x[0, 3], x[1, 40], x[2, 40] = 1e9, np.nan, -np.inf
    back = P.values(*P.pack(x), 64)
    assert abs(back[0, 3] - 32768) <= 32 and not back[0, 4:].any()
    assert np.isnan(back[1:, 32:]).all() and not back[1:, :32].any()


def test_ties_round_to_the_even_code():
    x = np.concatenate([[0.0, 15.0], np.arange(30) % 14 + 0.5]).astype(np.float32)[None]  # step 1: every .5 is a tie
    codes, _ = P.pack(x)
    nibbles = np.stack([codes & 15, codes >> 4], -1).reshape(-1)
    assert nibbles[2:].tolist() == [2 * round((i % 14 + 0.5) / 2 + (0.25 if (i % 14) % 2 else -0.25)) for i in range(30)]


@pytest.mark.parametrize("causal,window", [(True, -1), (True, 3), (False, 2)])
def test_weight_is_the_column_sum_of_the_softmax(causal, window):
    rng = _rng(2)
    n, length, dim, page, heads, kv_heads = 5, 13, 8, 4, 4, 2
    table = rng.permutation(8)[None, :4]
    kp, q = rng.standard_normal((8, kv_heads, page, dim)), rng.standard_normal((n, heads, dim))
    _, lse, _ = O.attend(q, kp, kp, table, [0, n], [length], causal, window)
    before = rng.random((8, kv_heads, page))
    got, size = P.weigh(before, q, lse, kp, table, [0, n], [length], causal, window, decay=0.5)
    keys = np.concatenate([kp[p] for p in table[0]], 1)[:, :length].repeat(2, 0)
    s = np.einsum("ihd,hld->hil", q, keys) / math.sqrt(dim)
    row, col = np.arange(n)[:, None] + length - n, np.arange(length)[None]
    ok = (col <= row) if causal else np.ones((n, length), bool)
    if window >= 0:
        ok &= col >= (row if causal else length - n) - window
    s = np.where(ok, s, -np.inf)
    p = np.exp(s) / np.exp(s).sum(-1, keepdims=True)
    want = p.sum(1).reshape(2, 2, length).sum(1)
    for j in range(length):
        old = 0.5 * before[table[0, j // page], :, j % page] if j < length - n else 0.0
        assert np.allclose(got[table[0, j // page], :, j % page], old + want[:, j], atol=1e-12)
    rest = np.ones((8, page), bool)
    for j in range(length):
        rest[table[0, j // page], j % page] = False
    assert np.array_equal(got.transpose(0, 2, 1)[rest], before.transpose(0, 2, 1)[rest])
    assert np.allclose(size[..., 0].sum(), n * heads)


def test_eviction_keeps_the_heaviest_and_the_newest():
    rng = _rng(3)
    weights = rng.integers(0, 4, (6, 2, 4)).astype(np.float32)  # many ties
    table = np.array([[4, 0, 2], [5, 1, 3]])
    lengths, kept = P.evict(weights, table, [11, 3], 5, 2)
    assert lengths.tolist() == [5, 3] and kept[1, :, :3].tolist() == [[0, 1, 2]] * 2 and (kept[1, :, 3:] == -1).all()
    for h in range(2):
        w = weights[table[0], h].reshape(-1)[:11]
        assert kept[0, h, 3:].tolist() == [9, 10]
        stay = kept[0, h, :3]
        order = np.argsort(-w[:9], kind="stable")[:3]
        assert sorted(order.tolist()) == stay.tolist()
    into = np.array([[1, 3], [0, 2]])  # of other pages: moved as they were
    rows = rng.random((6, 2, 4, 3))
    moved = P.move(rows, table, into, kept, 4, 6)
    assert np.array_equal(moved[1, 0, 0], rows[table[0, kept[0, 0, 0] // 4], 0, kept[0, 0, 0] % 4])
    assert np.array_equal(moved[3, 1, 0], rows[table[0, kept[0, 1, 4] // 4], 1, kept[0, 1, 4] % 4]) and np.array_equal(moved[4], rows[4])


def test_eviction_of_weights_that_are_no_numbers():
    w = np.array([[[1.0, np.nan, 0.0, -0.0, np.inf, -np.inf, np.nan, 5.0]]], np.float32)
    kept = lambda keep: P.evict(w, np.array([[0]]), [8], keep, 0)[1][0, 0].tolist()  # noqa: E731
    assert kept(1) == [1] and kept(2) == [1, 6] and kept(3) == [1, 4, 6] and kept(5) == [0, 1, 4, 6, 7] and kept(6) == [0, 1, 2, 4, 6, 7]


# ---------------------------------------------------------------- refusals --

A = 1 << 20  # an aligned address that no call may reach
INVALID, UNSUPPORTED, SMALL = S.SKIPCONV_E_INVALID_ARG, S.SKIPCONV_E_UNSUPPORTED, S.SKIPCONV_E_SMALL_BUFFER


def _with(x, **kw):
    for k, v in kw.items():
        setattr(x, k, v)
    return x


def _cache(**kw):  # 32 pages of 4 heads x 16 slots, heads of 64: rows of 32 bytes
    return _with(S.skipconv_cache(A, A, 4 * 16 * 32, 16 * 32, 32, 4 * 16 * 32, 16 * 32, 32, A, A, A, 8, 2, 4, 32, 16, 4, 64, 1), **kw)


def _packing(**kw):
    return _with(S.skipconv_packing(A, A, 4 * 16 * 4, 16 * 4, 4, 4 * 16 * 4, 16 * 4, 4), **kw)


def _attend(**kw):
    return _with(S.skipconv_attend(A, 2 * A, None, 512, 64, 512, 64, 8, 1, -1, 0.125, 0), **kw)


def _append(**kw):
    r = S.skipconv_rotary(A, A, 3, 32, 0, 0)
    a = S.skipconv_append(A, A, None, None, 256, 64, 256, 64, 512, 64, 512, 64, 8, ctypes.pointer(r))
    a._keep = r
    return _with(a, **kw)


def _weigh(**kw):
    return _with(S.skipconv_weigh(A, A, A, 512, 64, 8, 1, -1, 0.125, 1.0, 0), **kw)


def _evict(**kw):
    return _with(S.skipconv_evict(A, A, A, A, 4, 60, 8), **kw)


R = ctypes.byref


def _calls(c, s):
    """Every call on a cache in 4 bits."""
    lib = S.lib()
    return (lib.skipconv_packed_append(R(c), R(s), R(_append()), None), lib.skipconv_packed_attend(R(c), R(s), R(_attend()), A, 1 << 40, None),
            lib.skipconv_cache_weigh(R(c), R(s), R(_weigh()), None))


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), INVALID), (dict(tokens=-1), INVALID), (dict(batch=-1), INVALID), (dict(kv_heads=0), INVALID), (dict(pages=0), INVALID),
    (dict(page_size=0), INVALID), (dict(table_width=0), INVALID), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED),
    (dict(tokens=1 << 31), UNSUPPORTED), (dict(table_width=1 << 20, page_size=2048), UNSUPPORTED), (dict(k_slot=40), INVALID), (dict(v_page=-64), INVALID),
    (dict(k_pages=None), INVALID), (dict(row_start=None), INVALID), (dict(kv_len=None), INVALID), (dict(page_table=None), INVALID), (dict(v_pages=A + 8), INVALID),
])
def test_cache_refusals(kw, code):
    assert _calls(_cache(**kw), _packing()) == (code,) * 3
    assert "cache" in S.skipconv_last_error()
    lib = S.lib()
    if not {"tokens", "row_start"} & set(kw):
        assert lib.skipconv_cache_evict(R(_cache(**kw)), R(_packing()), R(_evict()), None) == code
    if not {"tokens", "row_start", "batch", "kv_len", "page_table", "table_width"} & set(kw):
        assert lib.skipconv_packed_unpack(R(_cache(**kw)), R(_packing()), A, 4, A, A, None) == code


@pytest.mark.parametrize("kw", [dict(k_scales=None), dict(v_scales=None), dict(k_scales=A + 2), dict(v_scales=A + 1), dict(ks_page=255), dict(vs_head=-2), dict(ks_slot=3)])
def test_packing_refusals(kw):
    lib, c, s = S.lib(), _cache(), _packing(**kw)
    assert _calls(c, s) == (INVALID,) * 3 and "packing" in S.skipconv_last_error()
    assert lib.skipconv_cache_evict(R(c), R(s), R(_evict()), None) == INVALID
    assert lib.skipconv_packed_unpack(R(c), R(s), A, 4, A, A, None) == INVALID


def test_no_description():
    lib, c, s = S.lib(), _cache(), _packing()
    for rc in (lib.skipconv_packed_append(None, R(s), R(_append()), None), lib.skipconv_packed_append(R(c), None, R(_append()), None),
               lib.skipconv_packed_append(R(c), R(s), None, None), lib.skipconv_packed_attend(None, R(s), R(_attend()), None, 0, None),
               lib.skipconv_packed_attend(R(c), None, R(_attend()), None, 0, None), lib.skipconv_packed_attend(R(c), R(s), None, None, 0, None),
               lib.skipconv_packed_attend_workspace(None, R(_attend()), R(ctypes.c_size_t())), lib.skipconv_packed_attend_workspace(R(c), R(_attend()), None),
               lib.skipconv_packed_unpack(None, R(s), A, 1, A, A, None), lib.skipconv_packed_unpack(R(c), None, A, 1, A, A, None),
               lib.skipconv_cache_weigh(None, R(s), R(_weigh()), None), lib.skipconv_cache_weigh(R(c), R(s), None, None),
               lib.skipconv_cache_evict(None, R(s), R(_evict()), None), lib.skipconv_cache_evict(R(c), R(s), None, None)):
        assert rc == INVALID and "NULL" in S.skipconv_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(q=A), INVALID), (dict(q=A, q_out=A, q_heads=0), INVALID), (dict(q=A, q_out=A, rotary=None), INVALID),
    (dict(q=A, q_out=A, q_out_token=1024), INVALID), (dict(q=A, q_out=2 * A, q_out_head=0), INVALID), (dict(k=A + 1), INVALID),
])
def test_append_refusals(kw, code):
    assert S.lib().skipconv_packed_append(R(_cache()), R(_packing()), R(_append(**kw)), None) == code


@pytest.mark.parametrize("kw", [
    dict(q_heads=6), dict(q_heads=0), dict(causal=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(max_new=-1),
    dict(q=None), dict(out=None), dict(q=A + 8), dict(out=A + 2), dict(q_head=68), dict(out_token=12), dict(out_token=0), dict(out_head=0), dict(lse=A + 2),
])
def test_attend_refusals(kw):
    assert S.lib().skipconv_packed_attend(R(_cache()), R(_packing()), R(_attend(**kw)), A, 1 << 40, None) == INVALID
    assert "attend" in S.skipconv_last_error()


def test_attend_workspace():
    lib, c, s, a, n = S.lib(), _cache(table_width=1024), _packing(), _attend(), ctypes.c_size_t()  # 16384 keys a sequence: split
    assert lib.skipconv_packed_attend_workspace(R(c), R(a), R(n)) == S.SKIPCONV_OK and n.value > 0
    assert lib.skipconv_packed_attend(R(c), R(s), R(a), A, n.value - 1, None) == SMALL
    assert lib.skipconv_packed_attend(R(c), R(s), R(a), A + 4, n.value, None) == INVALID
    assert lib.skipconv_packed_attend(R(c), R(s), R(a), None, n.value, None) == INVALID
    c = _cache(tokens=1 << 20, batch=4)  # rows enough to fill the GPU: nothing is split
    assert lib.skipconv_packed_attend_workspace(R(c), R(a), R(n)) == S.SKIPCONV_OK and n.value == 0


@pytest.mark.parametrize("kw,code", [
    (dict(list=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(list=A + 2), INVALID), (dict(k=A + 8), INVALID), (dict(v=A + 2), INVALID),
    (dict(count=-1), INVALID), (dict(count=1 << 40), UNSUPPORTED),
])
def test_unpack_refusals(kw, code):
    x = dict(dict(list=A, count=4, k=A, v=A), **kw)
    assert S.lib().skipconv_packed_unpack(R(_cache()), R(_packing()), x["list"], x["count"], x["k"], x["v"], None) == code
    assert "unpack" in S.skipconv_last_error()


@pytest.mark.parametrize("kw", [
    dict(q_heads=6), dict(q_heads=0), dict(causal=2), dict(scale=0.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(decay=float("nan")), dict(decay=float("inf")),
    dict(max_new=-1), dict(q=None), dict(lse=None), dict(weights=None), dict(q=A + 8), dict(q_head=68), dict(lse=A + 2), dict(weights=A + 1),
])
def test_weigh_refusals(kw):
    lib = S.lib()
    for c, s in ((_cache(), R(_packing())), (_cache(), None)):
        assert lib.skipconv_cache_weigh(R(c), s, R(_weigh(**kw)), None) == INVALID
        assert "weigh" in S.skipconv_last_error()


def test_weigh_refuses_rows_near_2_to_31():
    """Blocks of rows are counted up to 192 rows ahead: the count stays a 32-bit integer."""
    lib = S.lib()
    for s in (R(_packing()), None):
        for tokens in (((1 << 31) - 1025) // 16 + 1, ((1 << 31) - 1) // 16):
            assert lib.skipconv_cache_weigh(R(_cache(tokens=tokens, kv_heads=2)), s, R(_weigh(q_heads=16)), None) == UNSUPPORTED
            assert "weigh" in S.skipconv_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(keep=0), INVALID), (dict(keep=-1), INVALID), (dict(recent=-1), INVALID), (dict(recent=61), INVALID), (dict(into_width=0), INVALID), (dict(into_width=3), INVALID),
    (dict(weights=None), INVALID), (dict(into=None), INVALID), (dict(lengths=None), INVALID), (dict(kept=None), INVALID), (dict(weights=A + 2), INVALID), (dict(into=A + 1), INVALID),
    (dict(kept=A + 2), INVALID), (dict(lengths=A + 2), INVALID),
])
def test_evict_refusals(kw, code):
    lib = S.lib()
    for s in (R(_packing()), None):
        assert lib.skipconv_cache_evict(R(_cache()), s, R(_evict(**kw)), None) == code
        assert "evict" in S.skipconv_last_error()
    many = _cache(batch=1 << 28)
    assert lib.skipconv_cache_evict(R(many), None, R(_evict()), None) == UNSUPPORTED


def test_nothing_to_do():
    lib = S.lib()
    for kw in (dict(tokens=0), dict(batch=0, page_table=None, row_start=None, kv_len=None), dict(batch=0, tokens=0)):
        c, n = _cache(**kw), ctypes.c_size_t(7)
        assert _calls(c, _packing()) == (S.SKIPCONV_OK,) * 3
        assert lib.skipconv_cache_weigh(R(c), None, R(_weigh()), None) == S.SKIPCONV_OK
        assert lib.skipconv_packed_attend_workspace(R(c), R(_attend()), R(n)) == S.SKIPCONV_OK and n.value == 0
        if c.batch == 0:
            assert lib.skipconv_cache_evict(R(c), R(_packing()), R(_evict()), None) == S.SKIPCONV_OK
    assert lib.skipconv_packed_unpack(R(_cache()), R(_packing()), None, 0, None, None, None) == S.SKIPCONV_OK
