"""What the calls on the cache in 4 bits, on accumulated weight and on eviction promise at their edges, on the GPU against the oracle in 64 bits.

Bounds, and the caches that the tests are made of, are those of test_gpu_packed_cache.py.
"""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import packed_cache_oracle as P  # noqa: E402
from oracle import stream_attention_oracle as O  # noqa: E402
from paper_2104_11487_amd import skipconv as S  # noqa: E402
from paper_2104_11487_amd import stream_attention as A  # noqa: E402
from parity_util import say  # noqa: E402
from test_gpu_packed_cache import DT, U, _batch, _certain, _device, _garbage, _gpu, _held, _laid, _packed, _rng, _same, _stored  # noqa: E402
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
