"""What serving a model on the paged cache needs beside single-token attention, as cases that can be timed and compared.

The cache is that of perf/operators.py: a pool of pages of `page` tokens for all H key/value heads of a layer,

    codes      [P, H, page, m]        uint8: the product-quantised keys
    values     [P, H, page/8, d_k, 8] int8 or float8_e4m3fn: token t of a page at [t // 8, :, t % 8]
    exponents  [P, H]                 int8: a stored q stands for q * 2^exponent

with sequences as rows of `table`, `lengths` tokens long.

    chunk    the last counts[b] tokens of every sequence attend over its pages: row n stands at position p = lengths[b] - counts[b] + n and
             sees the tokens l <= p:  o = softmax(scale * s) V, s_l = q . (C_0[code_l0], C_1[code_l1], ...)
    weigh    every token's weight takes up the attention that the newest query pays it:  w_l = decay * w_l + sum_g softmax(scale * s_g)_l,
             s_gl = sum_i lut[g, i, code_li]
    evict    the k = min(length, keep) tokens of each head that are kept - the last `recent`, the first `first`, of the others the
             heaviest - enter other pages in their order; a page's exponent is the least e with |v| <= (127 or 448) 2^e over its tokens
    select   the n best continuations of each request over its beams and the vocabulary by  scores[r] + logits[r] - logsumexp(logits[r])

Among equal weights or scores the lowest position, beam and token go first.
"""
import math

import torch

own = False

K = 256
LOW_E, HIGH_E = -40, 40     # exponents of an all-zero page, and of the largest that is kept


def listed():
    return [
        # Eight drafted tokens of each of 16 users are verified at once: latency.
        {"name": "chunk_drafts", "kind": "chunk", "B": 16, "H": 12, "group": 1, "N": 8, "before": 1000, "ragged": 0.5, "empty": 0, "d_k": 64,
         "m": 4, "page": 64, "type": "int8", "dtype": "float16", "order": "heads", "sharp": 1.0},
        # The first pieces of eight prompts of unequal lengths, nothing in the cache before them.
        {"name": "chunk_prompts", "kind": "chunk", "B": 8, "H": 12, "group": 1, "N": 1000, "before": 0, "ragged": 0.6, "empty": 1, "d_k": 64,
         "m": 8, "page": 16, "type": "int8", "dtype": "float32", "order": "tokens", "sharp": 0.5},
        # A batch of pieces with four query heads on each key/value head, behind thousands of tokens.
        {"name": "chunk_grouped", "kind": "chunk", "B": 4, "H": 8, "group": 4, "N": 512, "before": 5000, "ragged": 0.3, "empty": 0,
         "d_k": 128, "m": 8, "page": 64, "type": "float8", "dtype": "float16", "order": "tokens", "sharp": 1.0},
        # One long prompt's last piece.
        {"name": "chunk_long", "kind": "chunk", "B": 1, "H": 32, "group": 1, "N": 2048, "before": 30001, "ragged": 0.0, "empty": 0,
         "d_k": 128, "m": 16, "page": 128, "type": "int8", "dtype": "float16", "order": "heads", "sharp": 0.125},
        # One user's step on a short context: latency.
        {"name": "weigh_one_user", "kind": "weigh", "B": 1, "H": 12, "group": 1, "L": 1024, "ragged": 0.0, "empty": 0, "d_k": 64, "m": 2,
         "page": 16, "decay": 1.0, "sharp": 1.0},
        # A batch of unequal lengths, four query heads on each key/value head.
        {"name": "weigh_grouped", "kind": "weigh", "B": 24, "H": 8, "group": 4, "L": 8191, "ragged": 0.9, "empty": 1, "d_k": 128, "m": 8,
         "page": 32, "decay": 0.99, "sharp": 1.0},
        # Long contexts in a batch.
        {"name": "weigh_long", "kind": "weigh", "B": 8, "H": 32, "group": 1, "L": 32768, "ragged": 0.0, "empty": 0, "d_k": 128, "m": 8,
         "page": 64, "decay": 1.0, "sharp": 0.125},
        # A few caches are brought down to half.
        {"name": "evict_few", "kind": "evict", "B": 4, "H": 12, "L": 1024, "ragged": 0.2, "share": 0.5, "first": 4, "recent": 64, "d_k": 64,
         "m": 4, "page": 16, "type": "int8"},
        # A batch of long caches, a little over half kept: 0.4 GB are read.
        {"name": "evict_long", "kind": "evict", "B": 8, "H": 16, "L": 20000, "ragged": 0.1, "share": 0.55, "first": 16, "recent": 1024,
         "d_k": 128, "m": 8, "page": 64, "type": "float8"},
        # One request, four beams: latency.
        {"name": "select_one", "kind": "select", "Q": 1, "beams": 4, "V": 50257, "n": 8, "dead": 0, "dtype": "float32"},
        # A batch of requests, half-precision logits with many equal ones, some beams ended.
        {"name": "select_batch", "kind": "select", "Q": 32, "beams": 4, "V": 32001, "n": 8, "dead": 1, "dtype": "float16"},
        # Many requests with eight beams and a large vocabulary: 0.27 GB of logits.
        {"name": "select_many", "kind": "select", "Q": 64, "beams": 8, "V": 131072, "n": 16, "dead": 0, "dtype": "float32"},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["chunk", "chunk", "chunk", "weigh", "weigh", "evict", "select", "select"])
    while True:
        c = {"kind": kind}
        if kind == "select":
            c.update(Q=_log_int(rng, 1, 128), beams=_log_int(rng, 1, 16), V=_log_int(rng, 100, 262144), n=_log_int(rng, 1, 64), dead=rng.choice([0, 1]),
                     dtype=rng.choice(["float16", "float32"]))
            c["dead"] = min(c["dead"], c["beams"] - 1)
            c["n"] = min(c["n"], c["V"])
            if work(c)["bytes"] <= 2.7e8:
                return c
            continue
        c.update(H=rng.choice([1, 4, 8, 12, 25, 32]), d_k=rng.choice([64, 128]), m=rng.choice([2, 4, 8, 16]), page=rng.choice([16, 32, 64, 128]))
        ragged = rng.choice([0.0, 0.3, 0.9])
        if kind == "evict":
            c.update(B=_log_int(rng, 1, 32), L=_log_int(rng, 8, 32768), ragged=ragged, share=rng.choice([0.1, 0.5, 0.9, 1.0]),
                     first=rng.choice([0, 4, 16]), recent=rng.choice([0, 1, 64, 500]), type=rng.choice(["int8", "float8"]))
            if work(c)["bytes"] <= 4.5e8:
                return c
            continue
        c.update(B=_log_int(rng, 1, 64), ragged=ragged, empty=rng.choice([0, 0, 1]), sharp=rng.choice([0.125, 1.0]),
                 group=rng.choice([g for g in (1, 2, 4, 8) if g * c["m"] <= 64]))
        c["empty"] = min(c["empty"], c["B"] - 1)
        if kind == "weigh":
            c.update(L=_log_int(rng, 1, 32768), decay=rng.choice([1.0, 0.9]))
            if work(c)["bytes"] <= 1.35e8:
                return c
            continue
        c.update(N=_log_int(rng, 1, 4096), before=rng.choice([0, _log_int(rng, 1, 32768)]), type=rng.choice(["int8", "float8"]),
                 dtype=rng.choice(["float16", "float32"]), order=rng.choice(["heads", "tokens"]))
        if c["B"] * c["H"] * c["group"] * c["N"] * (c["before"] + c["N"]) <= 2.1e9 and work(c)["flops"] <= 1.0e12:
            return c


# ---- sizes ------------------------------------------------------------------------------------------------------
def _spread(n, most, ragged):
    """n lengths from `most` down to (1 - ragged) most, at least 1."""
    return [max(1, int(round(most * (1.0 - ragged * (i / (n - 1) if n > 1 else 0.0))))) for i in range(n)]


def _ceil(a, b):
    return -(-a // b)


def _counts(c):
    """New tokens of every sequence of a chunk; none for the empty ones."""
    return _spread(c["B"] - c["empty"], c["N"], c["ragged"]) + [0] * c["empty"]


def _lengths(c):
    """The sequences' lengths, in no particular order yet."""
    if c["kind"] == "chunk":
        live = c["B"] - c["empty"]
        before = _spread(live, c["before"], c["ragged"]) if c["before"] else [0] * live
        return [n + x for n, x in zip(_counts(c), before)] + [0] * c["empty"]
    if c["kind"] == "weigh":
        return _spread(c["B"] - c["empty"], c["L"], c["ragged"]) + [0] * c["empty"]
    return _spread(c["B"], c["L"], c["ragged"])


def _kept(c):
    return [max(1, int(n * c["share"])) for n in _lengths(c)]


def _pages(c):
    used = sum(_ceil(n, c["page"]) for n in _lengths(c))
    if c["kind"] == "evict":
        used += sum(_ceil(n, c["page"]) for n in _kept(c))
    return used + _ceil(used, 8) + 1


def work(case):
    """Each input read once, each output written once."""
    c = case
    if c["kind"] == "select":
        rows = c["Q"] * c["beams"]
        return {"bytes": rows * (c["V"] * (2 if c["dtype"] == "float16" else 4) + 4) + c["Q"] * c["n"] * 12, "flops": rows * c["V"] * 3}
    H, d_k, m, page = c["H"], c["d_k"], c["m"], c["page"]
    lengths = _lengths(c)
    total, pages = sum(lengths), sum(_ceil(n, page) for n in lengths)
    if c["kind"] == "chunk":
        # row n of a sequence sees before + n + 1 tokens
        pairs = sum(k * (n - k) + k * (k + 1) // 2 for n, k in zip(lengths, _counts(c)))
        rows = sum(_counts(c)) * H * c["group"]
        e = 2 if c["dtype"] == "float16" else 4
        return {"bytes": total * H * (m + d_k) + pages * (4 + H) + rows * d_k * (e + 4) + H * K * d_k * 4 + 8 * c["B"],
                "flops": pairs * H * c["group"] * 4 * d_k}
    if c["kind"] == "weigh":
        heads = (c["B"] - c["empty"]) * H * c["group"]
        return {"bytes": total * H * (m + 8) + pages * 4 + heads * m * K * 4 + 4 * c["B"], "flops": total * H * c["group"] * (m + 4)}
    kept = sum(_kept(c))
    # the weights of all tokens; kept tokens read and written, their weights written too
    return {"bytes": total * H * 4 + kept * H * (2 * (m + d_k) + 4) + pages * 4, "flops": kept * H * d_k}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + salt) % (1 << 62))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _skewed(g, *shape):
    """Codes: a few centroids are met much more often than the others."""
    return (torch.rand(shape, generator=g, device="cuda").pow_(1.8) * K).clamp_(0, K - 1).to(torch.uint8)


def _pool(g, c):
    P, H, d_k, m, page = _pages(c), c["H"], c["d_k"], c["m"], c["page"]
    s = {"codes": _skewed(g, P, H, page, m), "exponents": torch.randint(-7, -3, (P, H), generator=g, device="cuda").to(torch.int8)}
    if c["kind"] == "weigh":
        # (it does not look at the values, whatever their type)
        s["values"] = torch.zeros((P, H, page // 8, d_k, 8), dtype=torch.int8, device="cuda")
        return s
    v = _randn(g, P, H, page // 8, d_k, 8)
    s["values"] = (v * 30).round_().clamp_(-127, 127).to(torch.int8) if c["type"] == "int8" else (v * 100).clamp_(-448, 448).to(torch.float8_e4m3fn)
    return s


def _rows(ids, page, lengths, width):
    """A table whose rows hold the pages `ids` one after another, and -1 behind them."""
    n = _ints([_ceil(x, page) for x in lengths])
    at = torch.arange(width, device="cuda")[None]
    first = (n.cumsum(0) - n)[:, None]
    return torch.where(at < n[:, None], ids[(first + at).clamp(max=ids.shape[0] - 1)], -1).to(torch.int32)


def _centroids(g, c):
    """Sub-vectors of keys of low rank, as real keys nearly are: [H, m, K, d_sub]."""
    rank = 8 if c["d_k"] <= 64 else 16
    key = _randn(g, c["H"], K, rank) @ _randn(g, c["H"], rank, c["d_k"]) + 0.1 * _randn(g, c["H"], K, c["d_k"])
    return key.view(c["H"], K, c["m"], c["d_k"] // c["m"]).transpose(1, 2).contiguous()


def prepare(case, seed):
    c = case
    g = _gen(seed, 0)
    if c["kind"] == "select":
        R, V = c["Q"] * c["beams"], c["V"]
        # logits as models give them: near their mean with a few far above; fp16 makes many equal
        x = _randn(g, R, V)
        x = (2.0 * x + x.clamp(min=2.0).sub_(2.0).mul_(3.0)).to(getattr(torch, c["dtype"]))
        scores = -8.0 * torch.rand((R,), generator=g, device="cuda")
        if c["dead"]:
            scores.view(c["Q"], c["beams"])[:, -c["dead"]:] = -math.inf
        return {"case": c, "logits": x, "scores": scores}
    B, H, d_k, m, page = c["B"], c["H"], c["d_k"], c["m"], c["page"]
    s = {"case": c, "pool": _pool(g, c)}
    P, lengths = _pages(c), _lengths(c)
    order = torch.randperm(B, generator=torch.Generator().manual_seed(int(seed))).tolist()
    lengths = [lengths[i] for i in order]
    ids = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    s["lengths"] = _ints(lengths)
    s["table"] = _rows(ids, page, lengths, max(1, _ceil(max(lengths), page)))
    if c["kind"] == "chunk":
        counts, hq, N = _counts(c), H * c["group"], c["N"]
        s["counts"] = _ints([counts[i] for i in order])
        s["codebooks"] = _centroids(g, c)
        q = (_randn(g, B, N, hq, d_k) if c["order"] == "tokens" else _randn(g, B, hq, N, d_k)).mul_(c["sharp"]).to(getattr(torch, c["dtype"]))
        s["q"] = q.transpose(1, 2) if c["order"] == "tokens" else q
        s["scale"] = 1.0 / math.sqrt(d_k)
        s["out"] = torch.zeros((B, hq, N, d_k), device="cuda")
    elif c["kind"] == "weigh":
        q = _randn(g, B, H, c["group"], m, 1, d_k // m) * c["sharp"]
        s["lut"] = (q * _centroids(g, c).view(H, 1, m, K, d_k // m)).sum(-1).view(B, H * c["group"], m, K).contiguous()
        s["scale"] = 1.0 / math.sqrt(d_k)
        # what some tens of earlier queries left
        s["weights"] = torch.rand((B, H, s["table"].shape[1] * page), generator=g, device="cuda").pow_(4.0).mul_(64.0 / c["L"])
    else:
        kept = _kept(c)
        kept = [kept[i] for i in order]
        used = sum(_ceil(n, page) for n in lengths)
        s["keep"] = _ints(kept)
        s["table_out"] = _rows(ids[used:], page, kept, _ceil(max(kept), page))
        # attention sums: a few tokens hold most of it, and many have got none
        w = _randn(g, B, H, s["table"].shape[1] * page).mul_(2.0).exp_()
        s["weights"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.2, 0.0, w)
        s["weights_out"] = torch.zeros((B, H, s["table_out"].shape[1] * page), device="cuda")
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------
def _two_to(e):
    """2^e as fp32, e in [-126, 127]: exact."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _codes(s):
    """[B, H, L, m] int64, L = entries of a row times the page's tokens."""
    B, W = s["table"].shape
    return s["pool"]["codes"][s["table"].clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(B, s["case"]["H"], W * s["case"]["page"], -1).long()


def _softmax(x):
    """Over the last axis; rows of -inf alone give zeros."""
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    z = w.sum(-1, keepdim=True)
    return w, torch.where(z > 0, z, 1.0)


def _chunk(s):
    c, pool, lengths, counts, table = s["case"], s["pool"], s["lengths"], s["counts"], s["table"]
    B, H, g, N, d_k, m, page = c["B"], c["H"], c["group"], c["N"], c["d_k"], c["m"], c["page"]
    L = table.shape[1] * page
    ids = table.clamp(min=0).long()
    code = _codes(s)
    head, sub = torch.arange(H, device=table.device)[:, None, None], torch.arange(m, device=table.device)
    key = s["codebooks"][head, sub, code].reshape(B, H, L, d_k)
    v = pool["values"][ids].float() * _two_to(pool["exponents"][ids])[..., None, None, None]
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(B, H, L, d_k)
    v = torch.where(torch.arange(L, device=v.device)[:, None] < lengths[:, None, None, None], v, 0.0)
    x = torch.matmul(s["q"].float().reshape(B, H, g * N, d_k), key.transpose(2, 3).contiguous()).view(B, H, g, N, L)
    n = torch.arange(N, device=table.device)
    seen = torch.arange(L, device=table.device) <= (lengths - counts)[:, None, None] + n[:, None]
    w, z = _softmax(torch.where(seen[:, None, None], x.mul_(s["scale"]), -math.inf))
    o = torch.matmul(w.view(B, H, g * N, L), v).view(B, H, g, N, d_k) / z
    live = (n < counts[:, None])[:, None, :, None]
    s["out"].copy_(torch.where(live, o.view(B, H * g, N, d_k), s["out"]))
    return s["out"]


def _weigh(s):
    c = s["case"]
    B, H, g, m = c["B"], c["H"], c["group"], c["m"]
    L = s["table"].shape[1] * c["page"]
    code = _codes(s).transpose(2, 3)[:, :, None]
    x = s["lut"].view(B, H, g, m, K).gather(4, code.expand(B, H, g, m, L)).sum(3) * s["scale"]
    seen = torch.arange(L, device=x.device) < s["lengths"][:, None]
    w, z = _softmax(torch.where(seen[:, None, None], x, -math.inf))
    new = s["weights"] * c["decay"] + (w / z).sum(2)
    s["weights"].copy_(torch.where(seen[:, None], new, s["weights"]))
    return s["weights"]


def _quantise(v, e, kind):
    x = v * _two_to(-e.to(torch.int32))
    return x.round().clamp(-127, 127).to(torch.int8) if kind == "int8" else x.clamp(-448, 448).to(torch.float8_e4m3fn)


def _exponent(top, kind):
    f, k = torch.frexp(top)
    e = k - 7 + (f > 127 / 128).int() if kind == "int8" else k - 9 + (f > 448 / 512).int()
    return torch.where(top > 0, e, LOW_E).clamp(LOW_E, HIGH_E)


def _evict(s):
    c, pool, weights, table, table_out = s["case"], s["pool"], s["weights"], s["table"], s["table_out"]
    B, H, d_k, m, page = c["B"], c["H"], c["d_k"], c["m"], c["page"]
    L, W = weights.shape[2], table_out.shape[1]
    M = W * page
    n = s["lengths"].long()[:, None, None]
    k = torch.minimum(n, s["keep"].long()[:, None, None])
    recent = k.clamp(max=c["recent"])
    first = (k - recent).clamp(max=c["first"])
    at = torch.arange(L, device=table.device).view(1, 1, L)
    rank = torch.where((at < first) | (at >= n - recent), math.inf, weights)
    rank = torch.where(at < n, rank, -math.inf)
    best = rank.sort(dim=-1, descending=True, stable=True).indices
    chosen = torch.zeros((B, H, L), dtype=torch.bool, device=table.device).scatter_(2, best, (at < k).expand(B, H, L))
    # the kept tokens' positions in their order
    place = torch.where(chosen, chosen.int().cumsum(-1) - 1, M).long()
    from_ = torch.zeros((B, H, max(M, L) + 1), dtype=torch.int64, device=table.device).scatter_(2, place, at.expand(B, H, L))[:, :, :M]
    inside = (torch.arange(M, device=table.device) < k).expand(B, H, M)
    head = torch.arange(H, device=table.device)[:, None]
    src = table.clamp(min=0).long()[torch.arange(B, device=table.device)[:, None, None], from_ // page]
    t = from_ % page
    codes = pool["codes"][src, head, t]
    v = pool["values"].view(torch.uint8)[src, head, t // 8, :, t % 8].view(pool["values"].dtype).float()
    v = v * _two_to(pool["exponents"][src, head])[..., None]
    top = torch.where(inside[..., None], v, 0.0).view(B, H, W, page * d_k).abs().amax(-1)
    e = _exponent(top, c["type"])
    q = _quantise(v.view(B, H, W, page, d_k), e[..., None, None], c["type"]).view(torch.uint8).view(B, H, M, d_k)
    b, h, i = inside.nonzero(as_tuple=True)
    dst, t = table_out[b, i // page].long(), i % page
    pool["codes"][dst, h, t] = codes[b, h, i]
    pool["values"].view(torch.uint8)[dst, h, t // 8, :, t % 8] = q[b, h, i]
    pool["exponents"][dst, h] = e[b, h, i // page].to(torch.int8)
    s["weights_out"].copy_(torch.where(inside, weights.gather(2, from_), s["weights_out"]))
    return {"pool": pool, "weights": s["weights_out"]}


def _select(s):
    c, x = s["case"], s["logits"].double()
    Q, beams, V, n = c["Q"], c["beams"], c["V"], c["n"]
    # (64 bits: two continuations' scores may lie closer than fp32 tells apart)
    top = x.amax(-1, keepdim=True)
    x = x - (top + torch.exp((x - top).float()).double().sum(-1, keepdim=True).log()) + s["scores"].double()[:, None]
    x, at = x.view(Q, beams * V).sort(dim=-1, descending=True, stable=True)
    x, at = x[:, :n], at[:, :n]
    parent = torch.arange(Q, device=x.device)[:, None] * beams + at // V
    found = x > -math.inf
    return {"scores": x.float(), "parents": torch.where(found, parent, -1).to(torch.int32), "tokens": torch.where(found, at % V, -1).to(torch.int32)}


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"chunk": _chunk, "weigh": _weigh, "evict": _evict, "select": _select}[c["kind"]](s)
    import paper_2601_10155_amd as lk
    if c["kind"] == "select":
        scores, parents, tokens = lk.lookat_beam_select(s["logits"], s["scores"], c["beams"], c["n"])
        return {"scores": scores, "parents": parents, "tokens": tokens}
    pool = lk.PagePool(s["pool"]["codes"], s["pool"]["values"], s["pool"]["exponents"])
    if c["kind"] == "chunk":
        return lk.lookat_attend_pages_chunk(s["q"], s["codebooks"], pool, s["table"], s["lengths"], s["scale"], counts=s["counts"], out=s["out"])
    if c["kind"] == "weigh":
        return lk.lookat_pages_weigh(s["lut"], pool, s["table"], s["lengths"], s["scale"], s["weights"], decay=c["decay"])
    lk.lookat_pages_evict(pool, s["table"], s["lengths"], s["weights"], s["keep"], s["table_out"], first=c["first"], recent=c["recent"],
                          weights_out=s["weights_out"])
    return {"pool": s["pool"], "weights": s["weights_out"]}


# ---- the same in 64 bits, head by head ------------------------------------------------------------------------------
def _tokens(x, b, h, s, n):
    """One head's rows of a sequence: codes [n, m] int64 or values [n, d_k] fp64."""
    ids = s["table"][b, : _ceil(n, s["case"]["page"])].long()
    if x == "codes":
        return s["pool"]["codes"][ids, h].reshape(-1, s["case"]["m"])[:n].long()
    size = torch.exp2(s["pool"]["exponents"][ids, h].double())
    v = s["pool"]["values"][ids, h].double() * size[:, None, None, None]
    return v.transpose(-1, -2).reshape(-1, s["case"]["d_k"])[:n]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "select":
        out = {"scores": [], "parents": [], "tokens": []}
        for q in range(c["Q"]):
            rows = slice(q * c["beams"], (q + 1) * c["beams"])
            x = (torch.log_softmax(s["logits"][rows].double(), -1) + s["scores"][rows].double()[:, None]).reshape(-1)
            v, at = torch.sort(x, descending=True, stable=True)
            v, at = v[: c["n"]], at[: c["n"]]
            none = torch.isneginf(v)
            out["scores"].append(v)
            out["parents"].append(torch.where(none, -1, q * c["beams"] + torch.div(at, c["V"], rounding_mode="floor")))
            out["tokens"].append(torch.where(none, -1, torch.remainder(at, c["V"])))
        return {k: torch.stack(v) if k == "scores" else torch.stack(v).int() for k, v in out.items()}
    B, H, m, page = c["B"], c["H"], c["m"], c["page"]
    lengths = s["lengths"].tolist()
    sub = torch.arange(m, device="cuda")
    if c["kind"] == "chunk":
        g, N = c["group"], c["N"]
        out = s["out"].double()
        for b, (n, k) in enumerate(zip(lengths, s["counts"].tolist())):
            if k == 0:
                continue
            later = torch.arange(n, device="cuda") > torch.arange(n - k, n, device="cuda")[:, None]
            for h in range(H):
                key = s["codebooks"][h].double()[sub, _tokens("codes", b, h, s, n)].reshape(n, -1)
                v = _tokens("values", b, h, s, n)
                for i in range(h * g, (h + 1) * g):
                    x = (s["q"][b, i, :k].double() @ key.T * s["scale"]).masked_fill_(later, -math.inf)
                    out[b, i, :k] = torch.softmax(x, -1) @ v
        return out
    if c["kind"] == "weigh":
        g = c["group"]
        out = s["weights"].double()
        for b, n in enumerate(lengths):
            for h in range(H if n else 0):
                x = s["lut"][b, h * g:(h + 1) * g].double()[:, sub, _tokens("codes", b, h, s, n)].sum(-1)
                out[b, h, :n] = c["decay"] * out[b, h, :n] + torch.softmax(x * s["scale"], -1).sum(0)
        return out
    pool, most = s["pool"], 127.0 if c["type"] == "int8" else 448.0
    moved = []
    for b, (n, k) in enumerate(zip(lengths, s["keep"].tolist())):
        for h in range(H):
            w = s["weights"][b, h, :n]
            recent = min(c["recent"], k)
            first = min(c["first"], k - recent)
            middle = w[first: n - recent]
            heavy = torch.sort(-middle, stable=True).indices[: k - first - recent] + first
            at = torch.cat([torch.arange(first, device="cuda"), heavy.sort().values, torch.arange(n - recent, n, device="cuda")])
            moved.append((b, h, k, at, _tokens("codes", b, h, s, n)[at], _tokens("values", b, h, s, n)[at]))
    for b, h, k, at, codes, v in moved:
        P = _ceil(k, page)
        ids = s["table_out"][b, :P].long()
        v = torch.cat([v, torch.zeros((P * page - k, c["d_k"]), dtype=torch.float64, device="cuda")]).view(P, page, -1)
        e = torch.ceil(torch.log2(v.abs().amax((1, 2)) / most))
        q = v / torch.exp2(e)[:, None, None]
        q = (q.round().to(torch.int8) if c["type"] == "int8" else q.float().to(torch.float8_e4m3fn)).view(torch.uint8)
        i = torch.arange(k, device="cuda")
        to, t = ids[i // page], i % page
        pool["codes"][to, h, t] = codes.to(torch.uint8)
        pool["values"].view(torch.uint8)[to, h, t // 8, :, t % 8] = q.reshape(P * page, -1)[:k]
        pool["exponents"][ids, h] = e.to(torch.int8)
        s["weights_out"][b, h, :k] = s["weights"][b, h, at]
    return {"pool": pool, "weights": s["weights_out"].double()}
