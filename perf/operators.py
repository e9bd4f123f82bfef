"""Attention of a video stream's new tokens over the tokens of earlier frames, operator by operator.

Three operators that a program calls on every frame (or every token) of a stream:

* ``rotary``: rotary positions with several axes (time, height, width) applied to the heads of a feature map's
  tokens, and the gradient of that;
* ``append``: the new tokens' keys and values written into a paged cache, rotated on the way, and their queries
  rotated in the same call;
* ``attend``: attention of the new tokens over the cache.

A case's sequences have ``new`` new tokens at most and ``kv`` tokens at most in the cache with them; ``mix`` seeds the
lengths of ragged batches, so that they belong to the case and not to the inputs. Pages of a sequence lie anywhere in
the cache. Positions are (frame, row, column) on a grid of ``gh`` x ``gw`` tokens a frame.
"""
import math
import random

import torch

own = False  # False: the plain forms below; True: the framework's operators

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE = 10000.0  # lowest frequency of an axis: 1 / BASE
SPARE = 3       # pages of the cache that no sequence holds


def _case(name, op, dtype, **more):
    c = {"name": name, "op": op, "dtype": dtype}
    c.update(more)
    return c


def _rotary(name, dtype, tokens, heads, dim, pairs, axes=3, adjacent=False, packed=False, grad=False, gh=64, gw=64):
    return _case(name, "rotary", dtype, tokens=tokens, heads=heads, dim=dim, pairs=pairs, axes=axes, adjacent=adjacent, packed=packed,
                 grad=grad, gh=gh, gw=gw)


def _append(name, dtype, batch, new, kv, heads, kv_heads, dim, pairs, page, ragged=False, mix=1, axes=3, adjacent=False, packed=False,
            gh=64, gw=64):
    return _case(name, "append", dtype, batch=batch, new=new, kv=kv, heads=heads, kv_heads=kv_heads, dim=dim, pairs=pairs, page=page,
                 ragged=ragged, mix=mix, axes=axes, adjacent=adjacent, packed=packed, gh=gh, gw=gw)


def _attend(name, dtype, batch, new, kv, heads, kv_heads, dim, page, causal=True, window=-1, ragged=False, mix=1, lse=False):
    return _case(name, "attend", dtype, batch=batch, new=new, kv=kv, heads=heads, kv_heads=kv_heads, dim=dim, page=page, causal=causal,
                 window=window, ragged=ragged, mix=mix, lse=lse)


def listed():
    return [
        # one token of each of 16 streams: the smallest call, latency only
        _rotary("rotary_step", "bf16", 16, 8, 64, 32),
        # a clip of 8 frames of 64 x 64 sites, the queries inside a packed projection of queries, keys and values
        _rotary("rotary_clip", "bf16", 8 * 64 * 64, 16, 128, 64, packed=True),
        # training in fp32: the gradient through the rotation of a 128 x 96 frame, heads only partly rotated, neighbours as pairs
        _rotary("rotary_grad", "f32", 128 * 96, 6, 80, 36, adjacent=True, grad=True, gh=128, gw=96),
        # the next token of 32 sequences into pages of 16
        _append("append_step", "bf16", 32, 1, 2048, 16, 4, 128, 64, 16, ragged=True, gh=16, gw=16),
        # a 64 x 64 frame of each of four streams, read from the packed projection
        _append("append_frame", "bf16", 4, 64 * 64, 4 * 64 * 64, 8, 4, 64, 32, 64, packed=True),
        # fp32 streams of unequal progress, one frame of 14 x 14 sites a page, some with nothing new
        _append("append_ragged", "f32", 7, 420, 1500, 4, 4, 80, 32, 196, ragged=True, adjacent=True, gh=14, gw=14),
        # one token of one short stream: the smallest call, latency only
        _attend("token_short", "bf16", 1, 1, 777, 16, 4, 64, 16),
        # the next token of 64 sequences of all lengths: bound by the cache's bytes
        _attend("tokens_ragged", "bf16", 64, 1, 16384, 32, 4, 128, 16, ragged=True),
        # the next token of one very long stream: few rows, a long axis
        _attend("token_long", "bf16", 1, 1, 262141, 8, 2, 128, 64, lse=True),
        # a 64 x 64 frame of each of four streams, over itself and the two frames before it
        _attend("frame_window", "bf16", 4, 64 * 64, 5 * 64 * 64, 8, 4, 64, 64, causal=False, window=2 * 64 * 64),
        # a long prompt in two sequences of unequal length, causal over the chunks before: the largest call
        _attend("prompt", "bf16", 2, 8192, 24576, 16, 4, 128, 64, ragged=True, mix=3),
        # fp32 streams of unequal progress, a frame of 14 x 14 sites a page, a window that begins and ends inside pages
        _attend("ragged_f32", "f32", 9, 300, 2500, 6, 3, 80, 196, ragged=True, window=700, mix=5, lse=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


DIMS = (32, 64, 80, 96, 128, 256)
PAGES = (16, 32, 64, 196, 256)


def draw(rng):
    costly, padded = max(_cost(c) for c in listed()), max(_padded(c) for c in listed())
    while True:
        kind = rng.choice(["rotary", "grad", "append_step", "append", "token", "tokens", "chunk", "chunk", "f32"])
        dtype = "f32" if kind in ("grad", "f32") or rng.random() < 0.15 else "bf16"
        dim, axes = rng.choice(DIMS), rng.choice((1, 2, 3, 3))
        pairs = dim // 2 if rng.random() < 0.6 else max(axes, dim // 2 - rng.randint(1, dim // 4))
        gh, gw = _log_int(rng, 7, 128), _log_int(rng, 7, 128)
        kv_heads, group, page = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 2, 4, 6, 8)), rng.choice(PAGES)
        more = {"adjacent": rng.random() < 0.4, "packed": rng.random() < 0.4, "gh": gh, "gw": gw, "axes": axes}
        mix, ragged = rng.randint(1, 1 << 20), rng.random() < 0.6
        if kind in ("rotary", "grad"):
            c = _rotary("", dtype, _log_int(rng, 1, 32768), rng.choice((1, 3, 4, 8, 16)), dim, pairs, grad=kind == "grad", **more)
            if _frames(c) * (c["axes"] > 1) > 256 or c["axes"] == 1 and c["tokens"] > 1024:
                continue  # 32-bit angles of the plain form stay good
        elif kind in ("append_step", "append"):
            batch, new = (_log_int(rng, 1, 128), 1) if kind == "append_step" else (_log_int(rng, 1, 16), _log_int(rng, 2, 4096))
            kv = max(new, _log_int(rng, 1, 16384))
            c = _append("", dtype, batch, new, kv, kv_heads * group, kv_heads, dim, pairs, page, ragged, mix, **more)
            if _frames(c) * (c["axes"] > 1) > 256 or c["axes"] == 1 and kv > 1024:
                continue
        else:
            if kind == "token":
                batch, new, kv = rng.choice((1, 1, 2, 3)), rng.choice((1, 1, 1, 2, 5)), _log_int(rng, 1, 262144)
            elif kind == "tokens":
                batch, new, kv = _log_int(rng, 4, 128), 1, _log_int(rng, 16, 16384)
            elif kind == "chunk":
                batch, new, kv = _log_int(rng, 1, 8), _log_int(rng, 8, 8192), _log_int(rng, 64, 32768)
            else:
                batch, new, kv = _log_int(rng, 1, 16), _log_int(rng, 1, 1024), _log_int(rng, 16, 4096)
            c = _attend("", dtype, batch, new, max(kv, new), kv_heads * group, kv_heads, dim, page, rng.random() < 0.6,
                        _log_int(rng, 1, kv) if rng.random() < 0.4 else -1, ragged, mix, rng.random() < 0.3)
        del c["name"]
        if _cost(c) <= costly and _padded(c) <= padded:
            return c


# ------------------------------------------------------------- the inputs --

def _frames(case):
    return -(-(case["tokens"] if case["op"] == "rotary" else case["kv"]) // (case["gh"] * case["gw"]))


def _lengths(case):
    """(new tokens, tokens in the cache with them) of each sequence."""
    if not case["ragged"]:
        return [(case["new"], case["kv"])] * case["batch"]
    rng = random.Random(case["mix"])
    out = [(case["new"], case["kv"])]
    for _ in range(case["batch"] - 1):
        kv = rng.randint(0 if case["new"] > 1 else 1, case["kv"])
        out.append((1 if case["new"] == 1 else min(kv, rng.choice((0, 1, rng.randint(0, case["new"]), rng.randint(0, case["new"])))), kv))
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
    x = torch.randn(shape, device="cuda", generator=g, dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    if mean:
        x += mean * torch.randn(shape[-1], device="cuda", generator=g, dtype=torch.float32).to(x.dtype)
    return x.mul_(gain) if gain != 1.0 else x


def _rows(case, g, heads):
    """Tensors tokens x heads[i] x dim, views of one projection's rows where the case is packed."""
    tokens = case["tokens"] if case["op"] == "rotary" else sum(n for n, _ in _lengths(case))
    if case.get("packed"):
        whole = _features((tokens, sum(heads), case["dim"]), case["dtype"], g, 0.5)
        return list(whole.split(heads, 1))
    return [_features((tokens, h, case["dim"]), case["dtype"], g, 0.5) for h in heads]


def _cache(case, g):
    """The cache's pages and what says where a batch's tokens lie in it."""
    lens, page = _lengths(case), case["page"]
    held = [-(-kv // page) for _, kv in lens]
    count = sum(held) + SPARE
    order = torch.randperm(count, device="cuda", generator=g).to(torch.int32)
    table = torch.zeros(len(lens), max(held + [1]), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n, _ in lens:
        starts.append(starts[-1] + n)
    shape = (count, case["kv_heads"], page, case["dim"])
    k = _features(shape, case["dtype"], g, 0.0)
    v = _features(shape, case["dtype"], g, 0.5)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"k_pages": k, "v_pages": v, "table": table, "starts": ints(starts), "lengths": ints([kv for _, kv in lens]),
            "most_new": max(n for n, _ in lens), "most_kv": max(max(kv for _, kv in lens), 1)}


def prepare(case, seed):
    g = _generator(seed * 1009 + 7)
    s = {"case": dict(case)}
    if case["op"] == "rotary":
        p = torch.arange(case["tokens"], device="cuda")
        s.update(x=_rows(case, g, [case["heads"]] * (3 if case["packed"] else 1))[0], pos=_grid(p, case), freq=_frequencies(case))
        return s
    s.update(_cache(case, g))
    if case["op"] == "append":
        s["q"], s["k"], s["v"] = _rows(case, g, [case["heads"], case["kv_heads"], case["kv_heads"]])
        p = torch.cat([torch.arange(kv - n, kv) for n, kv in _lengths(case)]).cuda()
        s.update(pos=_grid(p, case), freq=_frequencies(case))
    else:  # queries that favour some keys
        tokens = sum(n for n, _ in _lengths(case))
        s["q"] = _features((tokens, case["heads"], case["dim"]), case["dtype"], g, 0.0, 1.5)
    return s


# -------------------------------------------------- the framework's operators --

def _handles(s):
    """What a program makes once and keeps beside its tensors."""
    if "handles" not in s:
        from paper_2104_11487_amd import stream_attention as A

        c, h = s["case"], {}
        if "freq" in s:
            h["rotary"] = A.Rotary(s["freq"], c["dim"], pairing="adjacent" if c["adjacent"] else "halves")
        if "k_pages" in s:
            h["cache"] = A.PagedCache(s["k_pages"], s["v_pages"])
            h["batch"] = A.CacheBatch(s["table"], s["starts"], s["lengths"], max_new=s["most_new"])
        s["handles"] = h
    return s["handles"]


def _run_own(s):
    c, h = s["case"], _handles(s)
    if c["op"] == "rotary":
        return (h["rotary"].backward if c["grad"] else h["rotary"].rotate)(s["x"], s["pos"])
    if c["op"] == "append":
        q = h["cache"].append(s["k"], s["v"], h["batch"], rotary=h["rotary"], pos=s["pos"], q=s["q"])
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if c["lse"]:
        return h["cache"].attend(s["q"], h["batch"], causal=c["causal"], window=c["window"], return_lse=True)
    return h["cache"].attend(s["q"], h["batch"], causal=c["causal"], window=c["window"])


# ------------------------------------------------------------ the plain forms --

def _turn(x, pos, freq, adjacent, sign=1.0):
    """x (tokens x heads x dim) rotated, in 32 bits."""
    angle = (pos.float()[:, :, None] * freq).sum(1)[:, None]
    cos, sin = angle.cos(), sign * angle.sin()
    n = freq.shape[1]
    x = x.float()
    y = x.clone()
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if adjacent else (slice(0, n), slice(n, 2 * n))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _owners(s, tokens):
    """The sequence of each token, its place among that sequence's new tokens, and its position there."""
    starts = s["starts"].long()
    t = torch.arange(tokens, device="cuda")
    b = torch.searchsorted(starts[1:], t, right=True)
    i = t - starts[b]
    return b, i, s["lengths"].long()[b] - (starts[b + 1] - starts[b]) + i


def _plain_append(s):
    c = s["case"]
    dtype = DTYPES[c["dtype"]]
    b, _, p = _owners(s, s["k"].shape[0])
    page, slot = s["table"][b, p // c["page"]].long(), p % c["page"]
    s["k_pages"][page, :, slot] = _turn(s["k"], s["pos"], s["freq"], c["adjacent"]).to(dtype)
    s["v_pages"][page, :, slot] = s["v"]
    return {"q": _turn(s["q"], s["pos"], s["freq"], c["adjacent"]).to(dtype), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attend(s):
    """All sequences side by side, padded to the longest: scores, softmax and the sum of values, in 32 bits."""
    c = s["case"]
    batch, heads, kv_heads, dim, page = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    group, most, longest = heads // kv_heads, s["most_new"], s["most_kv"]
    starts, lengths = s["starts"].long(), s["lengths"].long()
    new = starts[1:] - starts[:-1]
    tokens = s["q"].shape[0]
    j, col = torch.arange(most, device="cuda"), torch.arange(longest, device="cuda")
    row = (starts[:-1, None] + j).clamp(max=max(tokens - 1, 0))
    q = s["q"][row].float().view(batch, most, kv_heads, group, dim).permute(0, 2, 1, 3, 4).reshape(batch, kv_heads, most * group, dim)
    at = torch.minimum(col, (lengths[:, None] - 1).clamp(min=0))
    where, slot = s["table"].gather(1, at // page).long(), at % page
    k = s["k_pages"][where, :, slot].float().permute(0, 2, 3, 1).contiguous()  # batch, kv_heads, dim, longest
    score = torch.matmul(q, k).mul_(1.0 / math.sqrt(dim)).view(batch, kv_heads, most, group, longest)
    del k
    first = lengths - new
    p = first[:, None] + j
    seen = (col <= p[..., None]) if c["causal"] else (col < lengths[:, None, None])
    if c["window"] >= 0:
        low = (p if c["causal"] else first[:, None].expand(batch, most)) - c["window"]
        seen = seen & (col >= low[..., None])
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    score = score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    v = s["v_pages"][where, :, slot].float().permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(score.view(batch, kv_heads, most * group, longest), v).view(batch, kv_heads, most, group, dim)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    b, i, _ = _owners(s, tokens)
    out = o.permute(0, 2, 1, 3, 4)[b, i].reshape(tokens, heads, dim).to(DTYPES[c["dtype"]])
    if not c["lse"]:
        return out
    lse = (top + total.log())[..., 0].permute(0, 2, 1, 3)[b, i].reshape(tokens, heads)
    return out, lse


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["op"] == "rotary":
        return _turn(state["x"], state["pos"], state["freq"], c["adjacent"], -1.0 if c["grad"] else 1.0).to(DTYPES[c["dtype"]])
    return _plain_append(state) if c["op"] == "append" else _plain_attend(state)


# ----------------------------------------------------------- what it takes --

def _span(case, n, kv, i):
    """Tokens that new token i of n sees: [lo, hi)."""
    p = kv - n + i
    hi = p + 1 if case["causal"] else kv
    lo = 0 if case["window"] < 0 else max(0, (p if case["causal"] else kv - n) - case["window"])
    return lo, hi


def work(case):
    e, dim = (4 if case["dtype"] == "f32" else 2), case["dim"]
    if case["op"] == "rotary":
        t, h = case["tokens"], case["heads"]
        return {"bytes": 2.0 * t * h * dim * e + 4 * t * case["axes"], "flops": 6.0 * t * h * case["pairs"]}
    lens, heads, kv_heads = _lengths(case), case["heads"], case["kv_heads"]
    tokens = sum(n for n, _ in lens)
    if case["op"] == "append":
        return {"bytes": 2.0 * tokens * (heads + 2 * kv_heads) * dim * e + 4 * tokens * case["axes"],
                "flops": 6.0 * tokens * (heads + kv_heads) * case["pairs"]}
    pairs, rows = 0, 0
    for n, kv in lens:
        if n:
            spans = [_span(case, n, kv, i) for i in range(n)]
            pairs += sum(hi - lo for lo, hi in spans)
            rows += spans[-1][1] - spans[0][0]
    total = 2.0 * tokens * heads * dim * e + 2.0 * rows * kv_heads * dim * e + (4.0 * tokens * heads if case["lse"] else 0.0)
    return {"bytes": total, "flops": 4.0 * pairs * heads * dim}


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 8e12, w["flops"] / (0.16e15 if case["dtype"] == "f32" else 2.5e15))


def _padded(case):
    """Values of the plain form's padded scores, keys and values."""
    if case["op"] != "attend":
        return 0
    lens = _lengths(case)
    most, longest = max(n for n, _ in lens), max(kv for _, kv in lens)
    return case["batch"] * (most * case["heads"] * longest + 2 * longest * case["kv_heads"] * case["dim"])


# -------------------------------------------------------------- in 64 bits --

def _exact_turn(x, pos, freq, adjacent, back=False):
    """Each pair as a complex number times exp(i angle)."""
    angle = pos.double() @ freq.double()
    w = torch.polar(torch.ones_like(angle), -angle if back else angle)[:, None]
    n = freq.shape[1]
    x = x.double()
    part, rest = x[..., :2 * n], x[..., 2 * n:]
    z = torch.complex(part[..., 0::2], part[..., 1::2]) if adjacent else torch.complex(part[..., :n], part[..., n:])
    z = z * w
    both = torch.stack((z.real, z.imag), -1).flatten(-2) if adjacent else torch.cat((z.real, z.imag), -1)
    return torch.cat((both, rest), -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_turn(s["x"], s["pos"], s["freq"], case["adjacent"], case["grad"])
    table = s["table"].tolist() if case["op"] == "append" else s["table"].long()
    page, lens = case["page"], _lengths(case)
    if case["op"] == "append":
        k, v = _exact_turn(s["k"], s["pos"], s["freq"], case["adjacent"]), s["v"].double()
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        t = 0
        for b, (n, kv) in enumerate(lens):
            p = kv - n
            while p < kv:  # page by page
                m = min(kv, (p // page + 1) * page) - p
                at, o = table[b][p // page], p % page
                kp[at, :, o:o + m] = k[t:t + m].transpose(0, 1)
                vp[at, :, o:o + m] = v[t:t + m].transpose(0, 1)
                p, t = p + m, t + m
        return {"q": _exact_turn(s["q"], s["pos"], s["freq"], case["adjacent"]), "k_pages": kp, "v_pages": vp}
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    group = heads // kv_heads
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    t = 0
    for b, (n, kv) in enumerate(lens):
        if n and kv:
            held = table[b, :-(-kv // page)]
            for h in range(kv_heads):
                keys = s["k_pages"][held, h].reshape(-1, dim)[:kv].double()
                values = s["v_pages"][held, h].reshape(-1, dim)[:kv].double()
                for i in range(0, n, 1024):
                    m = min(n, i + 1024) - i
                    lo, hi = _span(case, n, kv, i)[0], _span(case, n, kv, i + m - 1)[1]
                    q = s["q"][t + i:t + i + m, h * group:(h + 1) * group].double().reshape(m * group, dim)
                    score = (q @ keys[lo:hi].t().contiguous()).view(m, group, hi - lo) / math.sqrt(dim)
                    col, p = torch.arange(lo, hi, device="cuda"), kv - n + i + torch.arange(m, device="cuda")[:, None]
                    ok = torch.ones(m, hi - lo, dtype=torch.bool, device="cuda")
                    if case["causal"]:
                        ok &= col <= p
                        if case["window"] >= 0:
                            ok &= col >= p - case["window"]
                    score = score.masked_fill(~ok[:, None], -math.inf)
                    prob = torch.softmax(score, -1)
                    out[t + i:t + i + m, h * group:(h + 1) * group] = (prob.view(m * group, -1) @ values[lo:hi]).view(m, group, dim)
                    lse[t + i:t + i + m, h * group:(h + 1) * group] = torch.logsumexp(score, -1)
        t += n
    return (out, lse) if case["lse"] else out
