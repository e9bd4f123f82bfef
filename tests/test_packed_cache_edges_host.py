"""Refusals of the calls on the cache in 4 bits, on accumulated weight and on eviction, on the CPU: they come before any GPU work."""
import pytest

from paper_2104_11487_amd import skipconv as S
from test_packed_cache_host import A, INVALID, R, _cache, _evict, _packing

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
