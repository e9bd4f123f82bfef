"""Refusals of the calls on the cache in 4 bits, on accumulated weight and on eviction, on the CPU: they come before any GPU work."""
import ctypes

import pytest

from paper_2104_11487_amd import skipconv as S
from test_packed_cache_host import A, INVALID, R, _attend, _cache, _evict, _packing, _weigh

TABLE, INTO, LENGTHS, KEPT, WEIGHTS, KV_LEN = (i * A for i in range(1, 7))
SIZE = dict(kv_len=4 * 2, table=4 * 2 * 4, into=4 * 2 * 4, lengths=4 * 2, kept=4 * 2 * 4 * 60)  # bytes: 2 sequences of 4 pages, 4 key heads, 60 kept tokens


@pytest.mark.parametrize("which,at", [
    ("lengths", KV_LEN), ("lengths", KV_LEN + SIZE["kv_len"] - 4), ("lengths", KV_LEN - SIZE["lengths"] + 4), ("lengths", TABLE), ("lengths", TABLE + SIZE["table"] - 4),
    ("lengths", INTO), ("lengths", INTO + SIZE["into"] - 4), ("lengths", KEPT + SIZE["kept"] - 4), ("kept", KV_LEN), ("kept", KV_LEN - SIZE["kept"] + 4), ("kept", TABLE),
    ("kept", INTO - SIZE["kept"] + 4), ("kept", INTO + SIZE["into"] - 4), ("kept", LENGTHS), ("kept", LENGTHS + SIZE["lengths"] - 4), ("kept", LENGTHS - SIZE["kept"] + 4),
])
def test_evict_refuses_to_write_what_it_reads(which, at):
    """Lengths written over kv_len (in a graph whose batch stays, say) would be read as kv_len by the workgroups of the other key heads."""
    e = _evict(**dict(dict(into=INTO, lengths=LENGTHS, kept=KEPT, weights=WEIGHTS), **{which: at}))
    for s in (R(_packing()), None):
        assert S.lib().skipconv_cache_evict(R(_cache(page_table=TABLE, kv_len=KV_LEN)), s, R(e), None) == INVALID
        assert "evict" in S.skipconv_last_error() and "overlap" in S.skipconv_last_error()


@pytest.mark.parametrize("scale,code", [(3e38, INVALID), (2.37e38, INVALID), (2.3e38, S.SKIPCONV_OK), (1e-45, S.SKIPCONV_OK)])
def test_scales_whose_power_of_two_is_infinite(scale, code):
    """scale * log2 e past fp32 would make a score of zero NaN. (No token: calls that are accepted launch nothing.)"""
    lib, c, s = S.lib(), _cache(tokens=0), _packing()
    calls = (lib.skipconv_cache_attend(R(c), R(_attend(scale=scale)), A, 1 << 40, None), lib.skipconv_packed_attend(R(c), R(s), R(_attend(scale=scale)), A, 1 << 40, None),
             lib.skipconv_packed_attend_workspace(R(c), R(_attend(scale=scale)), R(ctypes.c_size_t())), lib.skipconv_cache_weigh(R(c), None, R(_weigh(scale=scale)), None),
             lib.skipconv_cache_weigh(R(c), R(s), R(_weigh(scale=scale)), None))
    assert calls == (code,) * 5 and (code == S.SKIPCONV_OK or "scale" in S.skipconv_last_error())
