"""The cache of a long stream, held in 4 bits and kept short, operator by operator.

Attention of a stream's new tokens over the tokens before reads the whole cache for every token, and the cache only grows.
The operators here make it a third of its size and bound its length:

* ``append``: the new tokens' keys (rotated on the way) and values into a paged cache of 4-bit codes; then the values that the
  sequences' pages hold (``unpack``);
* ``attend``: attention of the new tokens over such a cache;
* ``weigh``: the attention weight that each cached token received from the new tokens, added to what it had before;
* ``evict``: of each sequence and key head the heaviest tokens and the newest ones are kept, and moved to other pages.

A group of 32 elements of a head (the last one may be shorter) has a scale and a minimum in fp16, and an element a code of 4 bits: it
stands for minimum + code * scale, rounded to fp16. ``weigh`` and ``evict`` also take the float cache (``bits`` 16 and 32).

A case's sequences have ``new`` new tokens at most and ``kv`` tokens at most in the cache with them; ``mix`` seeds the lengths of
ragged batches, so that they belong to the case and not to the inputs. Pages of a sequence lie anywhere in the cache. Positions are
(frame, row, column) on a grid of ``gh`` x ``gw`` tokens a frame.
"""
import math
import random

import torch

own = False  # False: the plain forms below; True: the framework's operators

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE = 10000.0   # lowest frequency of an axis: 1 / BASE
SPARE = 3        # pages of the cache that no sequence holds
GROUP = 32       # elements with a scale and a minimum
MOST = 32768.0   # what elements are held up to


def _case(name, op, dtype, batch, new, kv, heads, kv_heads, dim, page, ragged=False, mix=1, bits=4, **more):
    c = {"name": name, "op": op, "dtype": dtype, "batch": batch, "new": new, "kv": kv, "heads": heads, "kv_heads": kv_heads, "dim": dim,
         "page": page, "ragged": ragged, "mix": mix, "bits": bits}
    c.update(more)
    return c


def _append(name, dtype, batch, new, kv, heads, kv_heads, dim, pairs, page, ragged=False, mix=1, axes=3, adjacent=False, packed=False,
            gh=64, gw=64):
    return _case(name, "append", dtype, batch, new, kv, heads, kv_heads, dim, page, ragged, mix, pairs=pairs, axes=axes,
                 adjacent=adjacent, packed=packed, gh=gh, gw=gw)


def _attend(name, dtype, batch, new, kv, heads, kv_heads, dim, page, causal=True, window=-1, ragged=False, mix=1, lse=False):
    return _case(name, "attend", dtype, batch, new, kv, heads, kv_heads, dim, page, ragged, mix, causal=causal, window=window, lse=lse)


def _weigh(name, dtype, batch, new, kv, heads, kv_heads, dim, page, causal=True, window=-1, ragged=False, mix=1, bits=4, decay=1.0):
    return _case(name, "weigh", dtype, batch, new, kv, heads, kv_heads, dim, page, ragged, mix, bits, causal=causal, window=window, decay=decay)


def _evict(name, dtype, batch, kv, kv_heads, dim, page, keep, recent, ragged=False, mix=1, bits=4):
    return _case(name, "evict", dtype, batch, 0, kv, kv_heads, kv_heads, dim, page, ragged, mix, bits, keep=keep, recent=recent)


def listed():
    return [
        # the next token of 32 streams into pages of 16
        _append("append_step", "bf16", 32, 1, 512, 16, 4, 128, 64, 16, ragged=True, gh=16, gw=16),
        # a 64 x 64 frame of each of four streams behind the frame before, out of a packed projection
        _append("append_frame", "bf16", 4, 64 * 64, 2 * 64 * 64, 8, 4, 64, 32, 64, packed=True),
        # one token of one short stream: the smallest call, latency only
        _attend("token_short", "bf16", 1, 1, 777, 16, 4, 64, 16),
        # the next token of 64 sequences of all lengths: bound by the cache's bytes
        _attend("tokens_ragged", "bf16", 64, 1, 16384, 32, 4, 128, 16, ragged=True),
        # the next token of one very long stream: few rows, a long axis
        _attend("token_long", "bf16", 1, 1, 262141, 8, 2, 128, 64),
        # a 64 x 64 frame of each of four streams, over itself and the two frames before it
        _attend("frame_window", "bf16", 4, 64 * 64, 5 * 64 * 64, 8, 4, 64, 64, causal=False, window=2 * 64 * 64, lse=True),
        # a long prompt in two sequences of unequal length, causal over the chunks before: the largest call
        _attend("prompt", "bf16", 2, 8192, 24576, 16, 4, 128, 64, ragged=True, mix=3),
        # fp32 streams of unequal progress, a frame of 14 x 14 sites a page, a window that begins and ends inside pages
        _attend("ragged_f32", "f32", 9, 300, 2500, 6, 3, 80, 196, ragged=True, window=700, mix=5, lse=True),
        # what the next token of 32 sequences of all lengths looked at, added up step by step
        _weigh("weigh_step", "bf16", 32, 1, 16384, 32, 4, 128, 16, ragged=True, decay=0.96875),
        # what the last 512 tokens of four prompts look at, over a cache of bf16
        _weigh("weigh_prompt", "bf16", 4, 512, 12000, 8, 2, 64, 64, bits=16),
        # a stream that has passed its budget by a few pages
        _evict("evict_step", "bf16", 1, 1100, 4, 64, 16, 1024, 64),
        # streams of all lengths brought down to a budget at once
        _evict("evict_ragged", "bf16", 16, 32768, 4, 128, 64, 8192, 256, ragged=True, mix=2),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


DIMS = (32, 64, 80, 96, 128, 256)
PAGES = (16, 32, 64, 196, 256)


def draw(rng):
    costly, padded = max(_cost(c) for c in listed()), max(_padded(c) for c in listed())
    while True:
        kind = rng.choice(["append_step", "append", "token", "tokens", "chunk", "chunk", "f32", "weigh", "weigh_chunk", "evict", "evict"])
        dtype = "f32" if kind == "f32" or rng.random() < 0.15 else "bf16"
        dim, axes = rng.choice(DIMS), rng.choice((1, 2, 3, 3))
        pairs = dim // 2 if rng.random() < 0.6 else max(axes, dim // 2 - rng.randint(1, dim // 4))
        gh, gw = _log_int(rng, 7, 128), _log_int(rng, 7, 128)
        kv_heads, group, page = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 2, 4, 6, 8)), rng.choice(PAGES)
        mix, ragged = rng.randint(1, 1 << 20), rng.random() < 0.6
        bits = 4 if rng.random() < 0.6 else 32 if dtype == "f32" else 16
        mask = {"causal": rng.random() < 0.6, "window": -1}
        if kind in ("append_step", "append"):
            batch, new = (_log_int(rng, 1, 128), 1) if kind == "append_step" else (_log_int(rng, 1, 16), _log_int(rng, 2, 4096))
            kv = max(new, _log_int(rng, 1, 8192))
            c = _append("", dtype, batch, new, kv, kv_heads * group, kv_heads, dim, pairs, page, ragged, mix, adjacent=rng.random() < 0.4,
                        packed=rng.random() < 0.4, gh=gh, gw=gw, axes=axes)
        elif kind == "evict":
            batch, kv = _log_int(rng, 1, 32), _log_int(rng, 16, 32768)
            keep = _log_int(rng, 1, kv)
            c = _evict("", dtype, batch, kv, kv_heads, dim, page, keep, rng.choice((0, 1, keep // 8, keep // 2, keep)), ragged, mix, bits)
        else:
            if kind == "token":
                batch, new, kv = rng.choice((1, 1, 2, 3)), rng.choice((1, 1, 1, 2, 5)), _log_int(rng, 1, 262144)
            elif kind in ("tokens", "weigh"):
                batch, new, kv = _log_int(rng, 4, 128), 1, _log_int(rng, 16, 16384)
            elif kind == "chunk":
                batch, new, kv = _log_int(rng, 1, 8), _log_int(rng, 8, 8192), _log_int(rng, 64, 32768)
            else:
                batch, new, kv = _log_int(rng, 1, 16), _log_int(rng, 1, 1024), _log_int(rng, 16, 4096)
            kv = max(kv, new)
            if rng.random() < 0.4:
                mask["window"] = _log_int(rng, 1, kv)
            if kind.startswith("weigh"):
                c = _weigh("", dtype, batch, new, kv, kv_heads * group, kv_heads, dim, page, ragged=ragged, mix=mix, bits=bits,
                           decay=rng.choice((1.0, 0.0, 0.5, 0.96875)), **mask)
            else:
                c = _attend("", dtype, batch, new, kv, kv_heads * group, kv_heads, dim, page, ragged=ragged, mix=mix, lse=rng.random() < 0.3, **mask)
        del c["name"]
        if _cost(c) <= costly and _padded(c) <= padded:
            return c


# ------------------------------------------------------------- the inputs --

def _lengths(case):
    """(new tokens, tokens in the cache with them) of each sequence."""
    if not case["ragged"]:
        return [(case["new"], case["kv"])] * case["batch"]
    rng = random.Random(case["mix"])
    out = [(case["new"], case["kv"])]
    for _ in range(case["batch"] - 1):
        kv = rng.randint(0 if case["new"] != 1 else 1, case["kv"])
        out.append((case["new"] if case["new"] < 2 else min(kv, rng.choice((0, 1, rng.randint(0, case["new"]), rng.randint(0, case["new"])))), kv))
    rng.shuffle(out)
    return out


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _frequencies(case):
    """A table of axes x pairs: the pairs are dealt to the axes in turn-sized sections, each with a ladder of its own."""
    axes, pairs = case["axes"], case["pairs"]
    f = torch.zeros(axes, pairs)
    at = 0
    for a in range(axes):
        n = pairs // axes + (a < pairs % axes)
        f[a, at:at + n] = BASE ** (-torch.arange(n, dtype=torch.float32) / n)
        at += n
    return f.cuda()


def _grid(p, case):
    """Positions (frame, row, column) of the tokens `p` of a stream, or the last axes of them."""
    area = case["gh"] * case["gw"]
    if case["axes"] == 1:
        return p[:, None].to(torch.int32).contiguous()
    full = torch.stack([p // area, p // case["gw"] % case["gh"], p % case["gw"]], 1)
    return full[:, 3 - case["axes"]:].to(torch.int32).contiguous()


def _features(shape, dtype, g, mean=0.0, gain=1.0):
    """Projections of feature maps: channels with a mean of their own around a spread of one."""
    x = torch.randn(shape, device="cuda", generator=g, dtype=DTYPES[dtype])
    if mean:
        x += mean * torch.randn(shape[-1], device="cuda", generator=g, dtype=torch.float32).to(x.dtype)
    return x.mul_(gain) if gain != 1.0 else x


def _rows(case, g, heads):
    """Tensors tokens x heads[i] x dim, views of one projection's rows where the case is packed."""
    tokens = sum(n for n, _ in _lengths(case))
    if case["packed"]:
        whole = _features((tokens, sum(heads), case["dim"]), case["dtype"], g, 0.5)
        return list(whole.split(heads, 1))
    return [_features((tokens, h, case["dim"]), case["dtype"], g, 0.5) for h in heads]


def _groups(dim):
    return -(-dim // GROUP)


def _held(shape, case, g, mean):
    """Pages in 4 bits, as features of a spread of one around `mean` have them: codes (two a byte, the lower half first) and (scale, minimum)."""
    n = _groups(case["dim"])
    codes = torch.empty(shape + (16 * n,), dtype=torch.uint8, device="cuda")
    for page in range(0, shape[0], 4096):  # the normal numbers of a few pages at a time
        part = codes[page:page + 4096]
        low, high = (torch.randn(part.shape, device="cuda", generator=g, dtype=torch.float16).mul_(3.7).add_(7.5).round_().clamp_(0, 15).to(torch.uint8)
                     for _ in range(2))
        part.copy_(low + 16 * high)
    scale = 0.27 * (1 + 0.15 * torch.randn(shape + (n,), device="cuda", generator=g).clamp_(-3, 3))
    low = mean - 7.5 * scale + 0.2 * torch.randn(shape + (n,), device="cuda", generator=g)
    return codes, torch.stack([scale, low], -1).to(torch.float16)


def _cache(case, g):
    """The cache's pages and what says where a batch's tokens lie in it; for an eviction also the pages that the kept ones go to."""
    lens, page = _lengths(case), case["page"]
    held = [-(-kv // page) for _, kv in lens]
    more = -(-min(case["keep"], case["kv"]) // page) * len(lens) if case["op"] == "evict" else 0
    count = sum(held) + more + SPARE
    order = torch.randperm(count, device="cuda", generator=g).to(torch.int32)
    table = torch.zeros(len(lens), max(held + [1]), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n, _ in lens:
        starts.append(starts[-1] + n)
    shape = (count, case["kv_heads"], page)
    s = {}
    if case["bits"] == 4:
        s["k_codes"], s["k_scales"] = _held(shape, case, g, 0.0)
        s["v_codes"], s["v_scales"] = _held(shape, case, g, 0.5)
    else:
        s["k_pages"] = _features(shape + (case["dim"],), case["dtype"], g, 0.0)
        s["v_pages"] = _features(shape + (case["dim"],), case["dtype"], g, 0.5)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    s.update(table=table, starts=ints(starts), lengths=ints([kv for _, kv in lens]), most_new=max(n for n, _ in lens),
             most_kv=max(max(kv for _, kv in lens), 1))
    if more:
        s["into"] = order[at:at + more].view(len(lens), -1)
    return s


def prepare(case, seed):
    g = _generator(seed * 1013 + 11)
    s = {"case": dict(case)}
    s.update(_cache(case, g))
    op = case["op"]
    if op == "append":
        s["q"], s["k"], s["v"] = _rows(case, g, [case["heads"], case["kv_heads"], case["kv_heads"]])
        p = torch.cat([torch.arange(kv - n, kv) for n, kv in _lengths(case)]).cuda()
        s.update(pos=_grid(p, case), freq=_frequencies(case))
    elif op in ("attend", "weigh"):  # queries that favour some keys
        tokens = sum(n for n, _ in _lengths(case))
        s["q"] = _features((tokens, case["heads"], case["dim"]), case["dtype"], g, 0.0, 1.5)
    if op in ("weigh", "evict"):
        shape = (s["k_codes"] if case["bits"] == 4 else s["k_pages"]).shape[:3]
        # weights as attention leaves them: many small ones, a few large ones, the untouched ones alike
        w = torch.randn(shape, device="cuda", generator=g).mul_(2.0).exp_().mul_(1e-3)
        s["weights"] = torch.where(w < 2e-5, torch.zeros_like(w), w)
    if op == "weigh":
        s["before"] = s["weights"].clone()
        s["lse"] = _lse(s)
    return s


# -------------------------------------------------- the framework's operators --

def _handles(s):
    """What a program makes once and keeps beside its tensors."""
    if "handles" not in s:
        from paper_2104_11487_amd import stream_attention as A

        c, h = s["case"], {}
        if "freq" in s:
            h["rotary"] = A.Rotary(s["freq"], c["dim"], pairing="adjacent" if c["adjacent"] else "halves")
        if c["bits"] == 4:
            h["cache"] = A.PackedCache(s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"], c["dim"], dtype=DTYPES[c["dtype"]])
        else:
            h["cache"] = A.PagedCache(s["k_pages"], s["v_pages"])
        h["batch"] = A.CacheBatch(s["table"], s["starts"], s["lengths"], max_new=s["most_new"])
        s["handles"] = h
    return s["handles"]


def _run_own(s):
    c, h = s["case"], _handles(s)
    cache, batch = h["cache"], h["batch"]
    if c["op"] == "append":
        q = cache.append(s["k"], s["v"], batch, rotary=h["rotary"], pos=s["pos"], q=s["q"])
        k, v = cache.unpack(s["table"])
        return {"q": q, "k": k, "v": v}
    if c["op"] == "attend":
        return cache.attend(s["q"], batch, causal=c["causal"], window=c["window"], return_lse=c["lse"])
    if c["op"] == "weigh":
        s["weights"].copy_(s["before"])  # so that a pass can be made again
        return cache.weigh(s["q"], s["lse"], batch, s["weights"], causal=c["causal"], window=c["window"], decay=c["decay"])
    lengths, kept = cache.evict(s["weights"], batch, s["into"], keep=c["keep"], recent=c["recent"])
    held = cache.unpack(s["into"]) if c["bits"] == 4 else (s["k_pages"], s["v_pages"])
    return {"lengths": lengths, "kept": kept, "weights": s["weights"], "k": held[0], "v": held[1]}


# ------------------------------------------------------------ the plain forms --

def _values(codes, scales, dim):
    """The fp16 values that codes stand for, ... x dim, as fp32."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float().view(*scales.shape[:-1], GROUP)
    pair = scales.float()
    return (pair[..., 1:] + c * pair[..., :1]).half().float().flatten(-2)[..., :dim]


def _pack(x):
    """(codes, scales) of fp32 elements, ... x dim."""
    dim, n = x.shape[-1], _groups(x.shape[-1])
    y = x.clamp(-MOST, MOST)
    fill = torch.nn.functional.pad
    low = fill(y, (0, n * GROUP - dim), value=math.inf).unflatten(-1, (n, GROUP)).amin(-1).half()
    high = fill(y, (0, n * GROUP - dim), value=-math.inf).unflatten(-1, (n, GROUP)).amax(-1)
    scale = ((high - low.float()) / 15).clamp(min=0).half()
    each = fill(y, (0, n * GROUP - dim)).unflatten(-1, (n, GROUP))
    c = ((each - low.float()[..., None]) / scale.float()[..., None]).round().clamp(0, 15)
    c = torch.where(scale[..., None] > 0, c, torch.zeros_like(c)).flatten(-2)
    c[..., dim:] = 0
    c = c.to(torch.uint8)
    return c[..., 0::2] + 16 * c[..., 1::2], torch.stack((scale, low), -1)


def _turn(x, pos, freq, adjacent):
    """x (tokens x heads x dim) rotated in 64 bits (what follows rounds at borders), as fp32."""
    angle = (pos.double()[:, :, None] * freq.double()).sum(1)[:, None]
    cos, sin = angle.cos(), angle.sin()
    n = freq.shape[1]
    x = x.double()
    y = x.clone()
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if adjacent else (slice(0, n), slice(n, 2 * n))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y.float()


def _owners(s, tokens):
    """The sequence of each token, its place among that sequence's new tokens, and its position there."""
    starts = s["starts"].long()
    t = torch.arange(tokens, device="cuda")
    b = torch.searchsorted(starts[1:], t, right=True)
    i = t - starts[b]
    return b, i, s["lengths"].long()[b] - (starts[b + 1] - starts[b]) + i


def _plain_append(s):
    c = s["case"]
    b, _, p = _owners(s, s["k"].shape[0])
    page, slot = s["table"][b, p // c["page"]].long(), p % c["page"]
    for name, x in (("k", _turn(s["k"], s["pos"], s["freq"], c["adjacent"])), ("v", s["v"].float())):
        s[name + "_codes"][page, :, slot], s[name + "_scales"][page, :, slot] = _pack(x)
    q = _turn(s["q"], s["pos"], s["freq"], c["adjacent"]).to(DTYPES[c["dtype"]])
    at = s["table"].long()
    return {"q": q, "k": _values(s["k_codes"][at], s["k_scales"][at], c["dim"]).half(), "v": _values(s["v_codes"][at], s["v_scales"][at], c["dim"]).half()}


def _gathered(s, name, where, slot):
    """Keys (values) of the tokens at pages `where`, slots `slot` (batch x longest): batch x longest x kv_heads x dim in fp32."""
    if s["case"]["bits"] == 4:
        return _values(s[name + "_codes"][where, :, slot], s[name + "_scales"][where, :, slot], s["case"]["dim"])
    return s[name + "_pages"][where, :, slot].float()


def _places(s):
    """Page and slot of the sequences' tokens, batch x longest (past an end: of the last token)."""
    page, lengths = s["case"]["page"], s["lengths"].long()
    at = torch.minimum(torch.arange(s["most_kv"], device="cuda"), (lengths[:, None] - 1).clamp(min=0))
    return s["table"].gather(1, at // page).long(), at % page


def _scores(s):
    """All sequences side by side, padded to the longest: scores batch x kv_heads x new x group x longest, -inf where nothing is seen."""
    c = s["case"]
    batch, heads, kv_heads, dim = c["batch"], c["heads"], c["kv_heads"], c["dim"]
    group, most, longest = heads // kv_heads, s["most_new"], s["most_kv"]
    starts, lengths = s["starts"].long(), s["lengths"].long()
    new = starts[1:] - starts[:-1]
    j, col = torch.arange(most, device="cuda"), torch.arange(longest, device="cuda")
    row = (starts[:-1, None] + j).clamp(max=max(s["q"].shape[0] - 1, 0))
    q = s["q"][row].float().view(batch, most, kv_heads, group, dim).permute(0, 2, 1, 3, 4).reshape(batch, kv_heads, most * group, dim)
    where, slot = _places(s)
    k = _gathered(s, "k", where, slot).permute(0, 2, 3, 1).contiguous()  # batch, kv_heads, dim, longest
    score = torch.matmul(q, k).mul_(1.0 / math.sqrt(dim)).view(batch, kv_heads, most, group, longest)
    first = lengths - new
    p = first[:, None] + j
    seen = (col <= p[..., None]) if c["causal"] else (col < lengths[:, None, None])
    if c["window"] >= 0:
        low = (p if c["causal"] else first[:, None].expand(batch, most)) - c["window"]
        seen = seen & (col >= low[..., None])
    seen = seen & (j < new[:, None])[..., None]
    return score.masked_fill_(~seen[:, None, :, None], -math.inf)


def _softmax_parts(score):
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    score = score.sub_(top).exp_()
    return top, score, score.sum(-1, keepdim=True)


def _by_token(s, x):
    """batch x kv_heads x new x group (x dim) as tokens x heads (x dim)."""
    b, i, _ = _owners(s, s["q"].shape[0])
    x = x.permute(0, 2, 1, 3, *range(4, x.dim()))[b, i]
    return x.reshape(x.shape[0], -1, *x.shape[3:])


def _lse(s):
    top, _, total = _softmax_parts(_scores(s))
    return _by_token(s, (top + total.log())[..., 0]).contiguous()


def _plain_attend(s):
    c = s["case"]
    batch, kv_heads, dim = c["batch"], c["kv_heads"], c["dim"]
    top, score, total = _softmax_parts(_scores(s))
    v = _gathered(s, "v", *_places(s)).permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(score.flatten(2, 3), v).view(batch, kv_heads, s["most_new"], -1, dim)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    out = _by_token(s, o).to(DTYPES[c["dtype"]])
    return (out, _by_token(s, (top + total.log())[..., 0])) if c["lse"] else out


def _plain_weigh(s):
    c = s["case"]
    s["weights"].copy_(s["before"])
    lengths, starts = s["lengths"].long(), s["starts"].long()
    new = starts[1:] - starts[:-1]
    j = torch.arange(s["most_new"], device="cuda")
    row = (starts[:-1, None] + j).clamp(max=max(s["q"].shape[0] - 1, 0))
    lse = s["lse"][row].view(c["batch"], s["most_new"], c["kv_heads"], -1).permute(0, 2, 1, 3)[..., None]
    lse = torch.where(lse == -math.inf, torch.zeros_like(lse), lse)
    got = _scores(s).sub_(lse).exp_().sum((2, 3)).permute(0, 2, 1)  # batch, longest, kv_heads
    where, slot = _places(s)
    col = torch.arange(s["most_kv"], device="cuda")
    held = torch.where((col < (lengths - new)[:, None])[..., None], s["weights"][where, :, slot] * c["decay"], torch.zeros_like(got))
    there = (col < lengths[:, None]) & (new > 0)[:, None]  # a sequence without new tokens stays as it is
    s["weights"][where[there], :, slot[there]] = (held + got)[there]
    return s["weights"]


def _plain_evict(s):
    c = s["case"]
    lengths, page, keep = s["lengths"].long(), c["page"], min(c["keep"], s["most_kv"])
    where, slot = _places(s)
    col = torch.arange(s["most_kv"], device="cuda")
    w = s["weights"][where, :, slot].permute(0, 2, 1)  # batch, kv_heads, longest
    w = torch.where((col >= (lengths - c["recent"])[:, None])[:, None], math.inf, w).masked_fill((col >= lengths[:, None])[:, None], -math.inf)
    first = w.sort(dim=-1, descending=True, stable=True).indices[..., :keep]  # of equal weights the earlier one
    count = lengths.clamp(max=keep)
    kept = torch.where(torch.arange(keep, device="cuda") < count[:, None, None], first, s["most_kv"]).sort(-1).values
    kept = torch.where(kept < s["most_kv"], kept, -1)
    b, h, i = (kept >= 0).nonzero(as_tuple=True)
    source = kept[b, h, i]
    to, at, to_slot, at_slot = s["into"][b, i // page].long(), s["table"][b, source // page].long(), i % page, source % page
    for name in ("k_codes", "k_scales", "v_codes", "v_scales") if c["bits"] == 4 else ("k_pages", "v_pages"):
        s[name][to, h, to_slot] = s[name][at, h, at_slot]
    s["weights"][to, h, to_slot] = s["weights"][at, h, at_slot]
    held = s["into"].long()
    kv = [_values(s[n + "_codes"][held], s[n + "_scales"][held], c["dim"]).half() if c["bits"] == 4 else s[n + "_pages"] for n in "kv"]
    if keep < c["keep"]:
        kept = torch.nn.functional.pad(kept, (0, c["keep"] - keep), value=-1)
    return {"lengths": count.int(), "kept": kept.int(), "weights": s["weights"], "k": kv[0], "v": kv[1]}


def run(state):
    if own:
        return _run_own(state)
    return {"append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[state["case"]["op"]](state)


# ----------------------------------------------------------- what it takes --

def _span(case, n, kv, i):
    """Tokens that new token i of n sees: [lo, hi)."""
    p = kv - n + i
    hi = p + 1 if case["causal"] else kv
    lo = 0 if case["window"] < 0 else max(0, (p if case["causal"] else kv - n) - case["window"])
    return lo, hi


def work(case):
    e, dim, page = (4 if case["dtype"] == "f32" else 2), case["dim"], case["page"]
    row = 20 * _groups(dim) if case["bits"] == 4 else dim * e  # bytes of a token's key, or value, of one head
    lens, heads, kv_heads = _lengths(case), case["heads"], case["kv_heads"]
    tokens = sum(n for n, _ in lens)
    if case["op"] == "append":
        pages = len(lens) * max(1, max(-(-kv // page) for _, kv in lens)) * page
        return {"bytes": float(tokens * ((2 * heads + 2 * kv_heads) * dim * e + 2 * kv_heads * row + 4 * case["axes"])
                               + pages * kv_heads * 2 * (row + 2 * dim)),
                "flops": 6.0 * tokens * (heads + kv_heads) * case["pairs"] + 4.0 * (tokens + pages) * kv_heads * dim}
    if case["op"] == "evict":
        kept = sum(min(kv, case["keep"]) for _, kv in lens) * kv_heads
        pages = len(lens) * -(-min(case["keep"], case["kv"]) // page) * page * kv_heads if case["bits"] == 4 else 0
        return {"bytes": float(4 * sum(kv for _, kv in lens) * kv_heads + kept * (4 * row + 12) + pages * 2 * (row + 2 * dim)),
                "flops": float(sum(kv for _, kv in lens) * kv_heads)}
    pairs, rows = 0, 0
    for n, kv in lens:
        if n:
            spans = [_span(case, n, kv, i) for i in range(n)]
            pairs += sum(hi - lo for lo, hi in spans)
            rows += spans[-1][1] - spans[0][0]
    if case["op"] == "weigh":
        every = sum(kv for _, kv in lens) * kv_heads  # weights: also copied once for the pass
        return {"bytes": float(tokens * heads * (dim * e + 4) + rows * kv_heads * row + 8 * every), "flops": 2.0 * pairs * heads * dim}
    return {"bytes": float(2 * tokens * heads * dim * e + 2 * rows * kv_heads * row + (4 * tokens * heads if case["lse"] else 0)),
            "flops": 4.0 * pairs * heads * dim}


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 8e12, w["flops"] / (0.16e15 if case["dtype"] == "f32" else 2.5e15))


def _padded(case):
    """Values of the plain form's padded scores, keys and values."""
    lens = _lengths(case)
    most, longest = max(n for n, _ in lens), max(kv for _, kv in lens)
    return case["batch"] * (most * case["heads"] * longest + 2 * longest * case["kv_heads"] * case["dim"])


# -------------------------------------------------------------- in 64 bits --

def _exact_turn(x, pos, freq, adjacent):
    """Each pair as a complex number times exp(i angle)."""
    angle = pos.double() @ freq.double()
    w = torch.polar(torch.ones_like(angle), angle)[:, None]
    n = freq.shape[1]
    x = x.double()
    part, rest = x[..., :2 * n], x[..., 2 * n:]
    z = torch.complex(part[..., 0::2], part[..., 1::2]) if adjacent else torch.complex(part[..., :n], part[..., n:])
    z = z * w
    both = torch.stack((z.real, z.imag), -1).flatten(-2) if adjacent else torch.cat((z.real, z.imag), -1)
    return torch.cat((both, rest), -1)


def _exact_held(x):
    """What the elements, in 64 bits, are held as: group by group, with the roundings that the format has."""
    out = torch.empty_like(x)
    for i in range(0, x.shape[-1], GROUP):
        y = x[..., i:i + GROUP].float().double().clamp(-MOST, MOST)
        low, high = torch.aminmax(y, dim=-1, keepdim=True)
        low = low.half().double()
        scale = ((high - low).float().double() / 15).clamp(min=0).float().half().double()
        steps = torch.where(scale > 0, (y - low).float().double() / scale, 0.0).float().double()
        out[..., i:i + GROUP] = (low + steps.round().clamp(0, 15) * scale).half().double()
    return out


def _exact_pages(s, name, at):
    """The values of pages `at`, ... x kv_heads x page x dim."""
    c = s["case"]
    if c["bits"] != 4:
        return s[name + "_pages"][at].double()
    out = torch.empty(*at.shape, c["kv_heads"], c["page"], 2 * s[name + "_codes"].shape[-1], dtype=torch.float64, device="cuda")
    codes, scales = s[name + "_codes"][at], s[name + "_scales"][at].double()
    for half in (0, 1):
        code = (codes // 16 if half else codes % 16).double()
        which = torch.arange(code.shape[-1], device="cuda") // (GROUP // 2)
        out[..., half::2] = (scales[..., which, 1] + code * scales[..., which, 0]).half().double()
    return out[..., :c["dim"]]


def _exact_append(s, lens):
    c = s["case"]
    kv = {}
    at = s["table"].long()
    for name in "kv":
        x = _exact_held(_exact_turn(s["k"], s["pos"], s["freq"], c["adjacent"]) if name == "k" else s["v"].double())
        whole = _exact_pages(s, name, torch.arange(s["k_codes"].shape[0], device="cuda"))
        t = 0
        for b, (n, kv_len) in enumerate(lens):
            p = kv_len - n
            while p < kv_len:  # page by page
                m = min(kv_len, (p // c["page"] + 1) * c["page"]) - p
                whole[at[b, p // c["page"]], :, p % c["page"]:p % c["page"] + m] = x[t:t + m].transpose(0, 1)
                p, t = p + m, t + m
        kv[name] = whole[at]
    return {"q": _exact_turn(s["q"], s["pos"], s["freq"], c["adjacent"]), "k": kv["k"], "v": kv["v"]}


def _exact_evict(s, lens):
    c = s["case"]
    page, keep = c["page"], c["keep"]
    weights = s["weights"].double()
    lengths, kept = [], torch.full((len(lens), c["kv_heads"], keep), -1, dtype=torch.int32, device="cuda")
    pages = {n: s[n] for n in s if n.endswith(("_pages", "_codes", "_scales"))}
    for b, (_, kv) in enumerate(lens):
        lengths.append(min(kv, keep))
        if not kv:
            continue
        held = s["table"][b, :-(-kv // page)].long()
        for h in range(c["kv_heads"]):
            w = weights[held, h].reshape(-1)[:kv].cpu().tolist()
            late = max(0, kv - c["recent"])
            order = list(range(late, kv)) + sorted(range(late), key=lambda i: (-w[i], i))
            chosen = torch.tensor(sorted(order[:keep]), device="cuda")
            kept[b, h, :chosen.numel()] = chosen.int()
            at, slot = held[chosen // page], chosen % page
            place = torch.arange(chosen.numel(), device="cuda")
            to, to_slot = s["into"][b].long()[place // page], place % page
            for x in pages.values():
                x[to, h, to_slot] = x[at, h, slot]
            weights[to, h, to_slot] = weights[at, h, slot]
    where = s["into"].long() if c["bits"] == 4 else torch.arange(s["weights"].shape[0], device="cuda")
    return {"lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "kept": kept, "weights": weights,
            "k": _exact_pages(s, "k", where), "v": _exact_pages(s, "v", where)}


def exact(case, seed):
    s = prepare(case, seed)
    page, lens = case["page"], _lengths(case)
    if case["op"] == "append":
        return _exact_append(s, lens)
    if case["op"] == "evict":
        return _exact_evict(s, lens)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    group, table = heads // kv_heads, s["table"].long()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    weights = s["before"].double() if case["op"] == "weigh" else None
    t = 0
    for b, (n, kv) in enumerate(lens):
        held = table[b, :-(-kv // page)]
        for h in range(kv_heads if n and kv else 0):
            keys = _exact_pages(s, "k", held)[:, h].reshape(-1, dim)[:kv]
            values = _exact_pages(s, "v", held)[:, h].reshape(-1, dim)[:kv] if weights is None else None
            got = torch.zeros(kv, dtype=torch.float64, device="cuda")
            for i in range(0, n, 1024):
                m = min(n, i + 1024) - i
                lo, hi = _span(case, n, kv, i)[0], _span(case, n, kv, i + m - 1)[1]
                rows = slice(t + i, t + i + m), slice(h * group, (h + 1) * group)
                q = s["q"][rows].double().reshape(m * group, dim)
                score = (q @ keys[lo:hi].t().contiguous()).view(m, group, hi - lo) / math.sqrt(dim)
                col, p = torch.arange(lo, hi, device="cuda"), kv - n + i + torch.arange(m, device="cuda")[:, None]
                ok = torch.ones(m, hi - lo, dtype=torch.bool, device="cuda")
                if case["causal"]:
                    ok &= col <= p
                    if case["window"] >= 0:
                        ok &= col >= p - case["window"]
                score = score.masked_fill(~ok[:, None], -math.inf)
                if weights is None:
                    out[rows] = (torch.softmax(score, -1).view(m * group, -1) @ values[lo:hi]).view(m, group, dim)
                    lse[rows] = torch.logsumexp(score, -1)
                else:
                    got[lo:hi] += (score - s["lse"][rows].double()[..., None]).exp().sum((0, 1))
            if weights is not None:
                at, slot = held[torch.arange(kv, device="cuda") // page], torch.arange(kv, device="cuda") % page
                old = weights[at, h, slot] * case["decay"]
                old[kv - n:] = 0
                weights[at, h, slot] = old + got
        t += n
    if weights is not None:
        return weights
    return (out, lse) if case["lse"] else out
