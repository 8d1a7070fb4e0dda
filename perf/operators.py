"""The operators on a paged key/value cache held in 8 bits, as cases that can be timed and compared.

The cache is a pool of pages of `page` tokens for all H key/value heads of a layer:

    codes      [P, H, page, m]        uint8: the product-quantised keys
    values     [P, H, page/8, d_k, 8] int8 or float8_e4m3fn: token t of a page at [t // 8, :, t % 8]
    exponents  [P, H]                 int8: a stored q stands for q * 2^exponent

and a sequence is a row of `table` (page ids), its tokens counted by `lengths`.  `refs` counts the rows that hold a page.

    attend   o = softmax(scale * s) V over a row's first `length` tokens, s_l = sum_i lut[i, code_l[i]]
    write    tokens enter pages: exponent = least e with |v| <= (127 or 448) 2^e over the page's tokens, q = round(v 2^-e)
    turn     one step of a search over several continuations: the last children are freed, new ones forked from their parents
             (pages shared), room for one token reserved (the shared last page copied first)
    copy     whole pages onto others
    compact  live pages move into the lowest places, the tables follow

A stored int8 is returned as the whole number it is, beside its exponent: the scales are powers of two, so that the
rounding is exact in every form and the numbers have to be equal.
"""
import math

import torch

own = False

K = 256
LOW_E, HIGH_E = -40, 40     # exponents of an all-zero page, and of the largest that is kept


def listed():
    return [
        # One user, short context, small heads: the latency of a call is what counts.
        {"name": "attend_one_user", "kind": "attend", "B": 1, "H": 12, "group": 1, "L": 1024, "ragged": 0.0, "empty": 0, "d_k": 64,
         "m": 2, "page": 16, "type": "int8", "sharp": 0.125},
        # The benchmark's batch, 32 sequences of up to 1024 tokens, one of them just ended.
        {"name": "attend_batch", "kind": "attend", "B": 32, "H": 12, "group": 1, "L": 1024, "ragged": 0.5, "empty": 1, "d_k": 64,
         "m": 4, "page": 64, "type": "int8", "sharp": 1.0},
        # Long contexts in a batch: 1.1 GB of cache in one call.
        {"name": "attend_long_batch", "kind": "attend", "B": 8, "H": 32, "group": 1, "L": 32768, "ragged": 0.0, "empty": 0, "d_k": 128,
         "m": 8, "page": 64, "type": "int8", "sharp": 0.125},
        # Eight query heads on each of eight key/value heads, lengths of every size, floating 8-bit values.
        {"name": "attend_grouped", "kind": "attend", "B": 12, "H": 8, "group": 8, "L": 8191, "ragged": 0.95, "empty": 2, "d_k": 128,
         "m": 8, "page": 32, "type": "float8", "sharp": 1.0},
        # A decode step's new token enters 32 caches: latency.
        {"name": "write_token", "kind": "write", "B": 32, "H": 12, "N": 1, "before": 777, "ragged": 0.0, "d_k": 64, "m": 4, "page": 64,
         "type": "int8", "dtype": "float16"},
        # The next pieces of four long prompts, of unequal lengths, from the middle of a page on.
        {"name": "write_prompt", "kind": "write", "B": 4, "H": 32, "N": 2048, "before": 1000, "ragged": 0.3, "d_k": 128, "m": 16, "page": 64,
         "type": "float8", "dtype": "float32"},
        # Four continuations of each of four requests.
        {"name": "turn_few", "kind": "turn", "S": 16, "fan": 4, "L": 1000, "ragged": 0.2, "spare": 1.5, "H": 12, "d_k": 64, "m": 4,
         "page": 16, "type": "int8"},
        # Many requests with long shared beginnings.
        {"name": "turn_many", "kind": "turn", "S": 192, "fan": 2, "L": 4100, "ragged": 0.9, "spare": 1.5, "H": 8, "d_k": 128, "m": 8,
         "page": 64, "type": "float8"},
        # A few pages: a beginning taken over for another request.
        {"name": "copy_few", "kind": "copy", "n": 16, "P": 512, "H": 12, "d_k": 64, "m": 4, "page": 16, "type": "int8"},
        # A quarter of a large pool.
        {"name": "copy_many", "kind": "copy", "n": 1024, "P": 4096, "H": 8, "d_k": 128, "m": 8, "page": 64, "type": "int8"},
        # A small pool after some requests ended.
        {"name": "compact_few", "kind": "compact", "P": 1024, "live": 0.6, "S": 24, "W": 64, "H": 12, "d_k": 64, "m": 4, "page": 16,
         "type": "int8"},
        # A large pool, half of it in use and in pieces.
        {"name": "compact_many", "kind": "compact", "P": 16000, "live": 0.5, "S": 160, "W": 512, "H": 8, "d_k": 64, "m": 8, "page": 32,
         "type": "float8"},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "write", "write", "turn", "copy", "compact"])
    while True:
        d_k = rng.choice([64, 128])
        m = rng.choice([2, 4, 8, 16])
        H = rng.choice([1, 4, 8, 12, 25, 32])
        page = rng.choice([16, 32, 64, 128])
        c = {"kind": kind, "H": H, "d_k": d_k, "m": m, "page": page, "type": rng.choice(["int8", "float8"])}
        ragged = rng.choice([0.0, 0.3, 0.95])
        if kind == "attend":
            # (the tables of a key/value head's queries have to fit the on-chip memory: 64 with the reduction buffer)
            c.update(B=_log_int(rng, 1, 64), L=_log_int(rng, 1, 32768), ragged=ragged, empty=rng.choice([0, 0, 1]),
                     group=rng.choice([g for g in (1, 2, 4, 8) if g * m <= 64]), sharp=rng.choice([0.125, 1.0]))
            c["empty"] = min(c["empty"], c["B"] - 1)
        elif kind == "write":
            c.update(B=_log_int(rng, 1, 64), N=rng.choice([1, _log_int(rng, 2, 4096)]), before=rng.choice([0, _log_int(rng, 1, 4096)]),
                     ragged=ragged, dtype=rng.choice(["float16", "float32"]))
        elif kind == "turn":
            c.update(S=_log_int(rng, 2, 256), fan=rng.choice([1, 2, 4]), L=_log_int(rng, 1, 8192), ragged=ragged, spare=1.5)
        elif kind == "copy":
            n = _log_int(rng, 1, 1024)
            c.update(n=n, P=max(2 * n + 1, _log_int(rng, 16, 4096)))
        else:
            S = _log_int(rng, 1, 256)
            W = _log_int(rng, 1, 256)
            c.update(S=S, W=W, P=max(8, int(S * W * rng.choice([0.7, 1.1]))), live=rng.choice([0.3, 0.6, 0.9]))
        pool = _pages(c) * c["H"] * c["page"] * (c["d_k"] + c["m"])
        if work(c)["bytes"] <= 1.1e9 and pool <= 1.3e9:
            return c


# ---- sizes ------------------------------------------------------------------------------------------------------
def _spread(n, most, ragged):
    """n lengths from `most` down to (1 - ragged) most, at least 1."""
    return [max(1, int(round(most * (1.0 - ragged * (i / (n - 1) if n > 1 else 0.0))))) for i in range(n)]


def _lengths(c):
    """The sequences' lengths, in no particular order yet (attend: as they are; write: after the write; turn: the parents')."""
    if c["kind"] == "attend":
        n = _spread(c["B"] - c["empty"], c["L"], c["ragged"])
        return n + [0] * c["empty"]
    if c["kind"] == "write":
        return [c["before"] + n for n in _spread(c["B"], c["N"], c["ragged"])]
    return _spread(c["S"], c["L"], c["ragged"])


def _ceil(a, b):
    return -(-a // b)


def _pages(c):
    if c["kind"] in ("copy", "compact"):
        return c["P"]
    used = sum(_ceil(n, c["page"]) for n in _lengths(c))
    if c["kind"] == "turn":
        return int(used * c["spare"]) + 2 * c["S"] + 4
    return used + _ceil(used, 8) + 1


def _live(c):
    """Pages of a compaction's pool that are in use."""
    return max(1, min(int(c["P"] * c["live"]), c["S"] * c["W"]))


def work(case):
    """Each input read once, each output written once.  Scores and weighted values count their additions and
    multiplications; what moves pages computes nothing."""
    c = case
    H, d_k, m, page = c["H"], c["d_k"], c["m"], c["page"]
    row = H * (m + d_k)                      # a token's bytes
    if c["kind"] == "attend":
        n, g = sum(_lengths(c)), c["group"]
        heads = (c["B"] - c["empty"]) * H * g
        pages = sum(_ceil(x, page) for x in _lengths(c))
        return {"bytes": n * row + pages * (4 + H) + heads * m * K * 4 + c["B"] * H * g * d_k * 4 + 4 * c["B"],
                "flops": n * H * g * (m + 2 * d_k)}
    if c["kind"] == "write":
        n = sum(_spread(c["B"], c["N"], c["ragged"]))
        e = 2 if c["dtype"] == "float16" else 4
        pages = sum(_ceil(c["before"] + x, page) - c["before"] // page for x in _spread(c["B"], c["N"], c["ragged"]))
        return {"bytes": n * H * (2 * m + d_k * (e + 1)) + pages * (4 + H) + 8 * c["B"], "flops": n * H * d_k * 2}
    if c["kind"] == "turn":
        # the children's rows twice (given up, made again), their pages' counts, the shared last pages
        rows = sum(_ceil(n, page) for n in _lengths(c))
        shared = sum(1 for n in _lengths(c) if n % page)
        return {"bytes": 2 * shared * page * row + rows * 4 * 6 + _pages(c) * 4 + c["S"] * 48, "flops": 0}
    if c["kind"] == "copy":
        return {"bytes": 2 * c["n"] * (page * row + H) + 8 * c["n"], "flops": 0}
    # the live pages over the border are spread as all pages are
    n = _live(c)
    moved = n * (1 - n / c["P"])
    return {"bytes": 2 * moved * (page * row + H) + 8 * c["P"] + 8 * n + 8 * c["S"], "flops": 0}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + salt) % (1 << 62))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _perm(g, n):
    return torch.randperm(n, generator=g, device="cuda").to(torch.int32)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _skewed(g, *shape):
    """Codes: a few centroids are met much more often than the others."""
    return (torch.rand(shape, generator=g, device="cuda").pow_(1.8) * K).clamp_(0, K - 1).to(torch.uint8)


def _pool(g, c):
    P, H, d_k, m, page = _pages(c), c["H"], c["d_k"], c["m"], c["page"]
    v = _randn(g, P, H, page // 8, d_k, 8)
    v = (v * 30).round_().clamp_(-127, 127).to(torch.int8) if c["type"] == "int8" else (v * 100).clamp_(-448, 448).to(torch.float8_e4m3fn)
    e = torch.randint(-7, -3, (P, H), generator=g, device="cuda").to(torch.int8)
    return {"codes": _skewed(g, P, H, page, m), "values": v, "exponents": e}


def _rows(g, c, lengths, width, pages):
    """A table whose rows hold pages of their own, in no order, and -1 behind them."""
    n = _ints([_ceil(x, c["page"]) for x in lengths])
    at = torch.arange(width, device="cuda")[None]
    first = (n.cumsum(0) - n)[:, None]
    ids = _perm(g, pages)
    return torch.where(at < n[:, None], ids[(first + at).clamp(max=pages - 1)], -1).to(torch.int32)


def prepare(case, seed):
    c = case
    g = _gen(seed, 0)
    H, d_k, m, page = c["H"], c["d_k"], c["m"], c["page"]
    s = {"case": c, "pool": _pool(g, c)}
    if c["kind"] in ("attend", "write"):
        B, lengths = c["B"], _lengths(c)
        order = torch.randperm(B, generator=torch.Generator().manual_seed(int(seed))).tolist()
        lengths = [lengths[i] for i in order]
        s["lengths"] = _ints(lengths)
        s["table"] = _rows(g, c, lengths, max(1, _ceil(max(lengths), page)), _pages(c))
    if c["kind"] == "attend":
        # tables of queries against centroids that are sub-vectors of keys of low rank, as real keys nearly are
        rank = 8 if d_k <= 64 else 16
        key = _randn(g, H, K, rank) @ _randn(g, H, rank, d_k) + 0.1 * _randn(g, H, K, d_k)
        q = _randn(g, B, H, c["group"], m, 1, d_k // m) * c["sharp"]
        book = key.view(H, 1, K, m, d_k // m).transpose(2, 3)
        s["lut"] = (q * book).sum(-1).view(B, H * c["group"], m, K).contiguous()
        s["scale"] = 1.0 / math.sqrt(d_k)
        s["out"] = torch.empty((B, H * c["group"], d_k), device="cuda")
    elif c["kind"] == "write":
        N = c["N"]
        s["counts"] = s["lengths"] - c["before"]
        s["new_codes"] = _skewed(g, B, H, N, m)
        # tokens and heads of unequal size: a page's largest value comes anywhere in it
        size = (0.5 * _randn(g, B, H, N, 1)).exp_()
        s["new_values"] = (_randn(g, B, H, N, d_k) * size).to(getattr(torch, c["dtype"]))
    elif c["kind"] == "turn":
        S, P, lengths = c["S"], _pages(c), _lengths(c)
        width = _ceil(max(lengths) + 1, page)
        s["table"] = torch.cat([_rows(g, c, lengths, width, P), torch.full((S, width), -1, dtype=torch.int32, device="cuda")])
        s["lengths"] = torch.cat([_ints(lengths), torch.zeros(S, dtype=torch.int32, device="cuda")])
        s["refs"] = torch.zeros(P + 1, dtype=torch.int32, device="cuda")
        s["refs"][s["table"][:S].long()] = 1          # (the last place takes the rows' -1)
        s["refs"] = s["refs"][:P].clone()
        s["children"] = _ints(range(S, 2 * S))
        parents = torch.randint(0, _ceil(S, c["fan"]), (S,), generator=g, device="cuda") * c["fan"]
        s["parents"] = parents.clamp_(max=S - 1).to(torch.int32)
        s["wanted"] = torch.zeros(2 * S, dtype=torch.int32, device="cuda")
        s["wanted"][S:] = s["lengths"][s["parents"].long()] + 1
    elif c["kind"] == "copy":
        ids = _perm(g, c["P"])
        s["src"], s["dst"] = ids[: c["n"]].clone(), ids[c["n"]: 2 * c["n"]].clone()
    else:
        P, S, W, n = c["P"], c["S"], c["W"], _live(c)
        # n pages dealt to the rows one after another; the last token of each row somewhere in its last page
        held = torch.full((S,), n // S, dtype=torch.int64, device="cuda") + (torch.arange(S, device="cuda") < n % S)
        s["lengths"] = (held * page - torch.randint(0, page, (S,), generator=g, device="cuda")).clamp_(min=0).to(torch.int32)
        held = (s["lengths"] + page - 1) // page
        at = torch.arange(W, device="cuda")[None]
        ids = _perm(g, P)[: max(n, 1)]
        place = (held.cumsum(0) - held)[:, None] + at
        s["table"] = torch.where(at < held[:, None], ids[place.clamp(max=n - 1).long()], -1).to(torch.int32)
        refs = torch.zeros(P + 1, dtype=torch.int32, device="cuda")
        refs[s["table"].long()] = 1
        s["refs"] = refs[:P].clone()
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------
def _two_to(e):
    """2^e as fp32, e in [-126, 127]: exact."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _attend(s):
    c, pool, lut, lengths, table = s["case"], s["pool"], s["lut"], s["lengths"], s["table"]
    B, H, g, d_k, m, page = c["B"], c["H"], c["group"], c["d_k"], c["m"], c["page"]
    W = table.shape[1]
    ids = table.clamp(min=0).long()
    codes = pool["codes"][ids].permute(0, 2, 4, 1, 3).reshape(B, H, 1, m, W * page).long()
    v = pool["values"][ids].float() * _two_to(pool["exponents"][ids])[..., None, None, None]
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(B, H, W * page, d_k)
    x = lut.view(B, H, g, m, K).gather(4, codes.expand(B, H, g, m, W * page)).sum(3) * s["scale"]
    seen = torch.arange(W * page, device=x.device) < lengths[:, None]
    x = torch.where(seen[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    v = torch.where(seen[:, None, :, None], v, 0.0)
    z = w.sum(-1, keepdim=True)
    s["out"].copy_((torch.matmul(w, v) / torch.where(z > 0, z, 1.0)).view(B, H * g, d_k))
    return s["out"]


def _quantise(v, e, kind):
    x = v * _two_to(-e.to(torch.int32))
    return x.round().clamp(-127, 127).to(torch.int8) if kind == "int8" else x.clamp(-448, 448).to(torch.float8_e4m3fn)


def _exponent(top, kind):
    f, k = torch.frexp(top)
    e = k - 7 + (f > 127 / 128).int() if kind == "int8" else k - 9 + (f > 448 / 512).int()
    return torch.where(top > 0, e, LOW_E).clamp(LOW_E, HIGH_E)


def _write(s):
    c, pool, table, lengths, counts = s["case"], s["pool"], s["table"], s["lengths"].long(), s["counts"].long()
    B, H, N, d_k, page, W = c["B"], c["H"], c["N"], c["d_k"], c["page"], s["table"].shape[1]
    dev = table.device
    v = s["new_values"].float()
    start = lengths - counts
    n = torch.arange(N, device=dev)
    pos = start[:, None] + n
    inside = n < counts[:, None]
    at = torch.where(inside, pos, 0)
    # the largest value of each touched page's new tokens, over (sequence, page of the sequence), per head
    cell = torch.where(inside, torch.arange(B, device=dev)[:, None] * W + at // page, B * W)
    top = torch.zeros((B * W + 1, H), device=dev)
    top.scatter_reduce_(0, cell.view(-1, 1).expand(-1, H), v.abs().amax(-1).transpose(1, 2).reshape(-1, H), "amax")
    e = _exponent(top[:-1].view(B, W, H), c["type"])
    w = torch.arange(W, device=dev)
    touched = (w >= (start // page)[:, None]) & (w * page < lengths[:, None]) & (counts > 0)[:, None]
    kept = touched & (w * page < start[:, None])
    ids = table.clamp(min=0).long()
    old = pool["exponents"][ids].int()
    e = torch.where(kept[..., None], torch.maximum(old, e), e)
    # the tokens that a page keeps, in its new exponent
    b, p = kept.nonzero(as_tuple=True)
    page_ids = ids[b, p]
    q = pool["values"][page_ids]
    back = _quantise(q.float(), (e - old)[b, p][..., None, None, None], c["type"])
    token = torch.arange(page, device=dev).view(page // 8, 8)
    keeps = (p * page)[:, None, None] + token < start[b][:, None, None]
    pool["values"][page_ids] = torch.where(keeps[:, None, :, None, :], back.view(torch.uint8), q.view(torch.uint8)).view(q.dtype)
    b, p = touched.nonzero(as_tuple=True)
    pool["exponents"][ids[b, p]] = e[b, p].to(torch.int8)
    # the new tokens
    b, i = inside.nonzero(as_tuple=True)
    t = pos[b, i]
    page_ids, t_in = ids[b, t // page], t % page
    q = _quantise(v[b, :, i], e[b, t // page][..., None], c["type"])
    pool["values"].view(torch.uint8)[page_ids, :, t_in // 8, :, t_in % 8] = q.view(torch.uint8)
    pool["codes"][page_ids, :, t_in] = s["new_codes"][b, :, i]
    return pool


def _move(pool, src, dst):
    """Pages src onto pages dst, as bytes."""
    codes, values, exponents = pool["codes"], pool["values"].view(torch.uint8), pool["exponents"]
    codes[dst], values[dst], exponents[dst] = codes[src], values[src], exponents[src]


def _held(table, lengths, page):
    """Which places of the rows hold pages."""
    return torch.arange(table.shape[1], device=table.device) * page < lengths[:, None]


def _turn(s):
    c, pool, table, lengths, refs = s["case"], s["pool"], s["table"], s["lengths"], s["refs"]
    page, (S, W), P = c["page"], s["table"].shape, s["refs"].shape[0]
    src, dst = s["parents"].long(), s["children"].long()
    # the last children are given up
    rows = table[dst]
    held = _held(rows, lengths[dst], page)
    refs.index_add_(0, rows.clamp(min=0).view(-1).long(), -held.int().view(-1))
    table[dst] = torch.where(held, -1, rows)
    lengths[dst] = 0
    # forks share the parents' pages
    rows, n = table[src], lengths[src]
    held = _held(rows, n, page)
    refs.index_add_(0, rows.clamp(min=0).view(-1).long(), held.int().view(-1))
    table[dst] = torch.where(held, rows, table[dst])
    lengths[dst] = n
    # room for what is wanted: a page of its own for a shared last page that grows, then new pages
    wanted = s["wanted"]
    grows = wanted > lengths
    w = torch.arange(W, device=table.device)
    last = (lengths // page).long().clamp(max=W - 1)
    tail = table.gather(1, last[:, None])[:, 0]
    shared = grows & (lengths % page != 0) & (refs[tail.clamp(min=0).long()] > 1)
    new = grows[:, None] & (w * page >= lengths[:, None]) & (w * page < wanted[:, None])
    new = new | (shared[:, None] & (w == last[:, None]))
    place = (new.view(-1).cumsum(0) - 1).clamp(min=0)
    free = refs == 0
    rank = torch.where(free, free.cumsum(0) - 1, P)
    listed_free = torch.zeros(P + 1, dtype=torch.int32, device=table.device).scatter_(
        0, rank, torch.arange(P, dtype=torch.int32, device=table.device))
    missing = (new.sum() - free.sum()).clamp(min=0).to(torch.int32).view(1)
    got = listed_free[place.clamp(max=P - 1)].view(S, W)
    enough = (missing == 0)
    new, shared = new & enough, shared & enough
    refs.index_add_(0, tail.clamp(min=0).long(), -shared.int())
    table.copy_(torch.where(new, got, table))
    refs.index_add_(0, got.view(-1).long(), new.int().view(-1))
    i = shared.nonzero(as_tuple=True)[0]
    _move(pool, tail[i].long(), table[i, last[i]].long())
    lengths.copy_(torch.where(grows & enough, wanted, lengths))
    return {"pool": pool, "table": table, "lengths": lengths, "refs": refs, "missing": missing}


def _copy(s):
    _move(s["pool"], s["src"].long(), s["dst"].long())
    return s["pool"]


def _compact(s):
    c, pool, table, lengths, refs = s["case"], s["pool"], s["table"], s["lengths"], s["refs"]
    P = refs.shape[0]
    live = refs > 0
    n = live.sum()
    at = torch.arange(P, device=refs.device)
    moves, hole = live & (at >= n), ~live & (at < n)
    src, dst = moves.nonzero(as_tuple=True)[0], hole.nonzero(as_tuple=True)[0]
    to = at.clone()
    to[src] = dst
    new_refs = torch.where(live & (at < n), refs, 0)
    new_refs[dst] = refs[src]
    held = _held(table, lengths, c["page"])
    new_table = torch.where(held, to[table.clamp(min=0).long()].to(torch.int32), -1)
    _move(pool, src, dst)
    return {"pool": pool, "table": new_table, "refs": new_refs, "live": n.to(torch.int32).view(1)}


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        return {"attend": _attend, "write": _write, "turn": _turn, "copy": _copy, "compact": _compact}[kind](s)
    import paper_2601_10155_amd as lk
    pool = lk.PagePool(s["pool"]["codes"], s["pool"]["values"], s["pool"]["exponents"])
    if kind == "attend":
        return lk.lookat_attend_pages(s["lut"], pool, s["table"], s["lengths"], s["scale"], out=s["out"])
    if kind == "write":
        lk.lookat_pages_write(pool, s["new_codes"], s["new_values"], s["table"], s["lengths"], s["counts"])
        return s["pool"]
    if kind == "turn":
        table, lengths, refs = s["table"], s["lengths"], s["refs"]
        lk.lookat_pages_free(pool, table, lengths, refs, s["children"])
        lk.lookat_pages_fork(pool, table, lengths, refs, s["parents"], s["children"])
        missing = lk.lookat_pages_reserve(pool, table, lengths, refs, s["wanted"])
        return {"pool": s["pool"], "table": table, "lengths": lengths, "refs": refs, "missing": missing}
    if kind == "copy":
        lk.lookat_pages_copy(pool, s["src"], s["dst"])
        return s["pool"]
    table, refs, live = lk.lookat_pages_compact(pool, s["table"], s["lengths"], s["refs"])
    return {"pool": s["pool"], "table": table, "refs": refs, "live": live}


# ---- the same in 64 bits, sequence by sequence ----------------------------------------------------------------------
def _token_rows(q, tokens):
    """One head's page part [page/8, d_k, 8] -> the rows [tokens, d_k] that it holds, fp64."""
    return q.double().transpose(-1, -2).reshape(-1, q.shape[-2])[:tokens]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    pool, page = s["pool"], c["page"]
    if c["kind"] == "attend":
        H, g, m = c["H"], c["group"], c["m"]
        out = torch.zeros((c["B"], H * g, c["d_k"]), dtype=torch.float64, device="cuda")
        sub = torch.arange(m, device="cuda")
        for b, n in enumerate(s["lengths"].tolist()):
            if n == 0:
                continue
            ids = s["table"][b, : _ceil(n, page)].long()
            for h in range(H):
                codes = pool["codes"][ids, h].view(-1, m)[:n].long()
                size = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), pool["exponents"][ids, h].long())
                v = (pool["values"][ids, h].double() * size[:, None, None, None]).transpose(-1, -2).reshape(-1, c["d_k"])[:n]
                score = s["lut"][b, h * g:(h + 1) * g].double()[:, sub, codes].sum(-1)
                out[b, h * g:(h + 1) * g] = torch.softmax(score * s["scale"], -1) @ v
        return out
    if c["kind"] == "write":
        most = 127.0 if c["type"] == "int8" else 448.0
        as_stored = (lambda x: x.round().to(torch.int8)) if c["type"] == "int8" else (lambda x: x.float().to(torch.float8_e4m3fn))
        for b, (n, count) in enumerate(zip(s["lengths"].tolist(), s["counts"].tolist())):
            start = n - count
            for p in range(start // page, _ceil(n, page)):
                a, z, i = max(start, p * page), min(n, (p + 1) * page), int(s["table"][b, p])
                new = s["new_values"][b, :, a - start: z - start].double()
                e = torch.ceil(torch.log2(new.abs().amax((1, 2)) / most)).long()
                keep = a - p * page
                rows = pool["values"][i].double().transpose(-1, -2).reshape(c["H"], page, -1)
                was = pool["exponents"][i].long()
                if keep:
                    e = torch.maximum(e, was)
                size = torch.exp2(e.double())[:, None, None]
                held = pool["values"][i].view(torch.uint8).transpose(-1, -2).reshape(c["H"], page, -1).clone()
                held[:, :keep] = as_stored(rows[:, :keep] * torch.exp2(was.double())[:, None, None] / size).view(torch.uint8)
                held[:, keep: keep + z - a] = as_stored(new / size).view(torch.uint8)
                pool["values"].view(torch.uint8)[i] = held.view(c["H"], page // 8, 8, -1).transpose(-1, -2)
                pool["exponents"][i] = e.to(torch.int8)
                pool["codes"][i][:, keep: keep + z - a] = s["new_codes"][b, :, a - start: z - start]
        return pool
    if c["kind"] == "copy":
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            for x in pool.values():
                x.view(torch.uint8)[b] = x.view(torch.uint8)[a]
        return pool
    table, lengths, refs = (s[k].tolist() for k in ("table", "lengths", "refs"))

    def move(a, b):
        for x in pool.values():
            x.view(torch.uint8)[b] = x.view(torch.uint8)[a]

    if c["kind"] == "turn":
        for src, dst, want in zip(s["parents"].tolist(), s["children"].tolist(), s["wanted"].tolist()[c["S"]:]):
            n = _ceil(lengths[src], page)
            table[dst][:n] = table[src][:n]
            lengths[dst] = lengths[src]
            for i in table[src][:n]:
                refs[i] += 1
        free = [i for i, r in enumerate(refs) if r == 0][::-1]
        was = list(refs)
        for row, want in enumerate(s["wanted"].tolist()):
            n = lengths[row]
            if want <= n:
                continue
            if n % page and was[table[row][n // page]] > 1:
                to = free.pop()
                move(table[row][n // page], to)
                refs[table[row][n // page]] -= 1
                refs[to] = 1
                table[row][n // page] = to
            for p in range(_ceil(n, page), _ceil(want, page)):
                table[row][p] = free.pop()
                refs[table[row][p]] = 1
            lengths[row] = want
        return {"pool": pool, "table": _ints(table), "lengths": _ints(lengths), "refs": _ints(refs), "missing": _ints([0])}
    n = sum(r > 0 for r in refs)
    holes = [i for i in range(n) if refs[i] == 0]
    to = {}
    for i in range(n, len(refs)):
        if refs[i]:
            to[i] = holes[len(to)]
            refs[to[i]], refs[i] = refs[i], 0
            move(i, to[i])
    for row, length in zip(table, lengths):
        k = _ceil(length, page)
        row[:] = [to.get(i, i) for i in row[:k]] + [-1] * (len(row) - k)
    return {"pool": pool, "table": _ints(table), "refs": _ints(refs), "live": _ints([n])}
