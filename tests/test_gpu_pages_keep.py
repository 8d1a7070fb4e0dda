"""Attention sums and eviction over the paged cache: sums against 64 bits at a derived bound, kept tokens bit for bit (whole pools)."""
import math

import numpy as np
import pytest
import torch

import pages_ref as pr
from bars import record
from test_gpu_pages import TORCH, assert_pool, dev, i32, lk, on_gpu, random_cache, random_table  # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def weigh_reference(c, lut, table, lengths, scale, decay, weights):
    """(weights, bound).  A logit (log2 units): m scaled entries and the maximum's subtraction, off by d = (m + 3) u (sum |entries| + |maximum|); a weight by
    d ln 2 + 2 u (exponential unit) of itself, the sum of n of them by as much and sqrt(n + 64) u * 4, the quotient and the addition by 2 u of theirs."""
    B, Hq = lut.shape[:2]
    g = Hq // c.H
    out, bound = weights.astype(np.float64).copy(), np.zeros(weights.shape)
    for b in range(B):
        reach = min(max(0, int(lengths[b])), table.shape[1] * c.page)
        at = np.array([t for t in range(reach) if 0 <= table[b, t // c.page] < c.P], dtype=np.int64)
        codes, _ = c.tokens(table[b], reach)
        columns = min(reach, out.shape[2])
        out[b, :, :columns] = decay * out[b, :, :columns] if decay else 0.0
        bound[b, :, :columns] += 2 * U * np.abs(out[b, :, :columns])
        for hq in range(Hq if len(at) else 0):
            h = hq // g
            entries = np.stack([lut[b, hq, i].astype(np.float64)[codes[h, :, i]] for i in range(c.m)])
            x = entries.sum(0) * scale
            p = np.exp(x - x.max())
            p /= p.sum()
            size = np.abs(entries).sum(0).max() * abs(scale) * 1.4427
            rel = 2 * ((c.m + 3) * U * 2 * size * 0.6932 + 2 * U) + (4 * math.sqrt(len(at) + 64) + 4 + g) * U
            inside = at < out.shape[2]
            out[b, h, at[inside]] += p[inside]
            bound[b, h, at[inside]] += rel * p[inside] + 2.0 ** -126
    return out, bound


def random_lut(rng, B, Hq, m, size=1.0):
    return (rng.standard_normal((B, Hq, m, 256)) * size).astype(np.float32)


@pytest.mark.parametrize("m", [2, 4, 8, 16])
@pytest.mark.parametrize("g", [1, 2, 4, 8])
def test_weigh(lk, m, g):  # noqa: F811
    rng = np.random.default_rng(m * g)
    H, page, W, P = 3, 32, 40, 130
    lengths = [1, 0, 1023, 1025, 31, 1280, -4]
    c = random_cache(rng, P, H, 64, m, page, "int8")
    table = random_table(rng, [max(0, n) for n in lengths], page, W, P)
    table[2, 3], table[2, 9], table[4, 0] = -1, P, 1 << 30
    lut = random_lut(rng, len(lengths), H * g, m, 4.0)
    start = rng.random((len(lengths), H, 1280)).astype(np.float32) / 500
    for decay, max_length in ((1.0, 0), (0.5, 1280), (0.0, 100)):
        weights = dev(np.full_like(start, np.nan) if decay == 0 else start)
        kept = weights.clone()
        got = lk.lookat_pages_weigh(dev(lut), on_gpu(lk, c), dev(table), i32(*lengths), 0.3, weights, decay=decay, max_length=max_length)
        assert got is weights
        want, bound = weigh_reference(c, lut, table, lengths, 0.3, decay, start)
        for b, n in enumerate(lengths):
            n = max(n, 0)
            assert torch.equal(weights[b, :, n:].isnan(), kept[b, :, n:].isnan()) and torch.equal(weights[b, :, n:].nan_to_num(), kept[b, :, n:].nan_to_num())
            x = got[b, :, :n].cpu().numpy()
            record("attention sums", float(np.max(np.abs(x - want[b, :, :n]), initial=0)))
            assert np.all(np.abs(x - want[b, :, :n]) <= bound[b, :, :n])


@pytest.mark.parametrize("B,H,L,g", [(1, 2, 70000, 1), (1, 1, 40000, 8), (40, 4, 700, 2), (2, 70, 9000, 4)])
def test_weigh_long_and_many(lk, B, H, L, g):  # noqa: F811
    """Sequences that several workgroups share, in ranges by launch size and by what a workgroup holds; columns for the first tokens only."""
    rng = np.random.default_rng(L)
    m, page = 4, 128
    lengths = [max(1, L - 97 * b) for b in range(B)]
    held = [-(-n // page) for n in lengths]
    c = pr.Cache(rng.integers(0, 256, (sum(held), H, page, m), dtype=np.uint8), np.zeros((sum(held), H, page // 8, 64, 8), np.uint8),
                 np.zeros((sum(held), H), np.int8), "int8")
    table = random_table(rng, lengths, page, max(held) + 1, sum(held))
    lut = random_lut(rng, B, H * g, m, 2.0)
    pool, d_lut, d_table, d_len = on_gpu(lk, c), dev(lut), dev(table), i32(*lengths)
    code = torch.from_numpy(c.codes).cuda()[d_table.clamp(min=0).long()].permute(0, 2, 4, 1, 3).reshape(B, H, 1, m, -1).long()
    x = d_lut.double().view(B, H, g, m, 256).gather(4, code.expand(B, H, g, m, code.shape[-1])).sum(3) * 0.5
    size = float(d_lut.abs().amax(-1).sum(-1).max()) * 0.5 * 1.4427
    x = x.masked_fill(torch.arange(x.shape[-1], device="cuda") >= d_len[:, None, None, None], -math.inf)
    p = torch.softmax(x, -1).sum(2)
    rel = 2 * ((m + 3) * U * 2 * size * 0.6932 + 2 * U) + (4 * math.sqrt(L + 64) + 4 + g) * U
    for columns, max_length in ((x.shape[-1], 0), (L // 2, L)):
        weights = torch.full((B, H, columns), 0.25 / L, device="cuda")
        lk.lookat_pages_weigh(d_lut, pool, d_table, d_len, 0.5, weights, max_length=max_length)
        want = 0.25 / L + p[..., :columns]
        assert bool(((weights.double() - want).abs() <= rel * p[..., :columns] + 4 * U * want).all())
        again = torch.full((B, H, columns), 0.25 / L, device="cuda")
        lk.lookat_pages_weigh(d_lut, pool, d_table, d_len, 0.5, again, max_length=max_length)
        assert torch.equal(weights, again)


@pytest.mark.parametrize("m,g,B,H,L", [(2, 1, 33, 3, 1000), (16, 2, 33, 3, 500), (8, 4, 33, 3, 250), (4, 8, 33, 3, 250), (4, 1, 35, 16, 8190),
                                       (16, 2, 35, 16, 4090), (8, 4, 35, 16, 2040), (4, 8, 35, 16, 1020), (16, 1, 1, 600, 31),
                                       (2, 8, 35, 16, 4500), (4, 4, 35, 16, 8300)])
def test_weigh_many_heads(lk, m, g, B, H, L):  # noqa: F811
    """Small workgroups, short code and long: lengths from none to the row's room, pages outside the pool, tables that are not finite."""
    rng = np.random.default_rng(L + m)
    page = 16
    lengths = [L - b * L // max(1, B - 1) for b in range(B)]
    W = -(-L // page)
    P = 50
    table = rng.integers(0, P, (B, W)).astype(np.int32)           # (values are not read, so sequences may hold the same page)
    table[0, W // 2], table[B // 3, 0] = -1, P
    codes = torch.from_numpy(rng.integers(0, 256, (P, H, page, m), dtype=np.uint8)).cuda()
    pool = lk.PagePool(codes, torch.zeros((P, H, page // 8, 64, 8), dtype=torch.int8, device="cuda"), torch.zeros((P, H), dtype=torch.int8, device="cuda"))
    lut = random_lut(rng, B, H * g, m, 2.0)
    if B > 1:
        lut[0, g] = -np.inf                                       # (a query head without weight; one of NaN where there is another key/value head)
        lut[B // 2, 2 * g, 0] = np.nan
    d_lut, d_table, d_len = dev(lut), dev(table), i32(*lengths)
    start = torch.from_numpy(rng.random((B, H, W * page)).astype(np.float32) / L).cuda()
    weights = start.clone()
    lk.lookat_pages_weigh(d_lut, pool, d_table, d_len, 0.5, weights, decay=0.75)
    there = ((d_table >= 0) & (d_table < P)).repeat_interleave(page, 1) & (torch.arange(W * page, device="cuda") < d_len[:, None])
    size = float(d_lut.abs().nan_to_num(0, 0, 0).amax(-1).sum(-1).max()) * 0.5 * 1.4427
    rel = 2 * ((m + 3) * U * 2 * size * 0.6932 + 2 * U) + (4 * math.sqrt(L + 64) + 4 + g) * U
    for b in range(B):
        n = lengths[b]
        assert torch.equal(weights[b, :, n:], start[b, :, n:])
        if not n:
            continue
        code = codes[d_table[b].clamp(0, P - 1).long()].permute(1, 3, 0, 2).reshape(H, 1, m, -1)[..., :n].long()
        x = d_lut[b].double().view(H, g, m, 256).gather(3, code.expand(H, g, m, n)).sum(2) * 0.5
        x = x.masked_fill(~there[b, :n], -math.inf)
        top = x.amax(-1, keepdim=True)
        w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
        p = (w / torch.where(w.sum(-1, keepdim=True) == 0, 1.0, w.sum(-1, keepdim=True))).sum(1)
        want = 0.75 * start[b, :, :n].double() + p
        nan = p.isnan()
        assert torch.equal(weights[b, :, :n].isnan(), nan)
        assert bool(((weights[b, :, :n].double() - want).abs() <= rel * p + 4 * U * want)[~nan].all())


@pytest.mark.parametrize("W", [3, 200])
def test_weigh_scores_that_are_not_finite(lk, W):  # noqa: F811
    """A head of -inf alone adds nothing, far negative scores keep their weight (also where other ranges hold -inf alone), NaN and +inf show."""
    rng = np.random.default_rng(5)
    H, m, page = 5, 2, 128
    n = W * page
    c = random_cache(rng, W, H, 64, m, page, "int8")
    table = rng.permutation(W).astype(np.int32)[None]
    lut = random_lut(rng, 1, H, m)
    lut[0, 0] = -np.inf
    lut[0, 1, 0, 7] = np.nan
    lut[0, 2, 1, 9] = np.inf
    lut[0, 3] -= 3000.0
    lut[0, 4] = -np.inf
    lut[0, 4, :, 3] = -900.0
    for i in range(W):
        c.codes[i, 4] = 5
    c.codes[table[0, W // 2], 4, 17] = 3
    weights = torch.zeros((1, H, n), device="cuda")
    lk.lookat_pages_weigh(dev(lut), on_gpu(lk, c), dev(table), i32(n), 1.0, weights)
    w = weights.cpu().numpy()[0]
    assert not w[0].any()
    assert np.isnan(w[1]).all() and np.isnan(w[2]).all()
    assert abs(w[3].sum(dtype=np.float64) - 1) < 1e-4 * 3 and w[3].min() >= 0
    assert w[4, W // 2 * page + 17] == 1 and np.count_nonzero(w[4]) == 1


def evict_reference(c, table, lengths, weights, keep, first, recent, table_out, weights_out):
    """The cache after the call, places per (b, h), weights_out."""
    after = pr.Cache(c.codes, c.values, c.exponents, c.kind)
    out = None if weights_out is None else weights_out.copy()
    places = {}
    for b in range(len(lengths)):
        n = min(max(0, int(lengths[b])), table.shape[1] * c.page)
        k = max(0, min(n, int(keep[b]), table_out.shape[1] * c.page))
        last = min(recent, k)
        head = min(first, k - last)
        for h in range(c.H):
            w = np.zeros(n, np.float32)
            w[:min(n, weights.shape[2])] = weights[b, h, :n]
            rank = [(-np.inf if np.isnan(x) else float(x)) for x in w]
            order = sorted(range(head, n - last), key=lambda t: (np.isnan(w[t]), -rank[t], t))
            at = sorted(list(range(head)) + order[:k - head - last] + list(range(n - last, n)))
            places[b, h] = at
            for slot in range(-(-k // c.page)):
                to = int(table_out[b, slot])
                if not 0 <= to < c.P:
                    continue
                mine = [(j, t) for j, t in enumerate(at[slot * c.page:(slot + 1) * c.page]) if 0 <= table[b, t // c.page] < c.P]
                if not mine:
                    continue
                v = []
                for j, t in mine:
                    i = int(table[b, t // c.page])
                    e = min(max(int(c.exponents[i, h]), pr.LOW), pr.HIGH)
                    v.append(pr.from_bytes(c.row(i, h, t % c.page), c.kind) * 2.0 ** e)
                    after.codes[to, h, j] = c.codes[i, h, t % c.page]
                x = np.stack(v)
                e = pr.exponent(float(np.max(np.abs(np.where(np.isnan(x), 0, x)))), c.kind)
                after.exponents[to, h] = e
                for (j, _), y in zip(mine, x):
                    after.row(to, h, j)[:] = pr.to_bytes(y * 2.0 ** -e, c.kind)
            if out is not None:
                m = min(k, out.shape[2])
                out[b, h, :m] = w[at][:m]
    return after, places, out


def spread_weights(rng, *shape):
    w = np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    w[rng.random(shape) < 0.3] = 0.0
    w[rng.random(shape) < 0.1] = 1.0
    return w


@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("d_k,m,page", [(64, 4, 16), (64, 2, 64), (128, 8, 32), (128, 16, 128), (64, 16, 128)])
@pytest.mark.parametrize("first,recent,room", [(0, 0, 0), (4, 30, 0), (1000, 7, 0), (3, 1000, 0), (4, 30, 1 << 14)])
def test_evict(lk, d_k, m, page, kind, first, recent, room):  # noqa: F811
    """Lengths of zero and one, all kept, none, one, pages that end inside the kept tokens, ties, places for fewer than asked, rows with room for many
    more tokens (which the launch goes by)."""
    rng = np.random.default_rng(page + first)
    H, B = 2, 9
    lengths = [200, 1, 0, page, 129, 200, 64, 200, 77]
    keep = [100, 1, 5, page, 1, 0, 64, 5000, -3]
    W = -(-200 // page)
    W_out = max(1, W - 1) if page < 128 else W
    P = B * (W + W_out) + 2
    c = random_cache(rng, P, H, d_k, m, page, kind, -9, 5)
    ids = rng.permutation(P).astype(np.int32)
    table = ids[:B * W].reshape(B, W)
    table_out = ids[B * W: B * (W + W_out)].reshape(B, W_out)
    if room:
        W_out = room // page
        table_out = np.concatenate([table_out, np.full((B, W_out - table_out.shape[1]), -1, np.int32)], 1)
    weights = spread_weights(rng, B, H, 200)
    weights[0, 0, 20:40] = -weights[0, 0, 20:40]
    out = np.full((B, H, 90), -5.0, np.float32)
    pool, ws = on_gpu(lk, c), None
    d_out = dev(out)
    ws = torch.empty(lk.pages_evict_workspace_bytes(pool, B, W_out), dtype=torch.uint8, device="cuda")
    lk.lookat_pages_evict(pool, dev(table), i32(*lengths), dev(weights), i32(*keep), dev(table_out), first=first, recent=recent, weights_out=d_out,
                          workspace=ws)
    after, places, want = evict_reference(c, table, lengths, weights, keep, first, recent, table_out, out)
    got = ws.view(torch.int32).view(B, H, W_out * page).cpu().numpy()
    for (b, h), at in places.items():
        assert got[b, h, :len(at)].tolist() == at, (b, h)
    assert np.array_equal(d_out.cpu().numpy(), want)
    assert_pool(pool, after)


@pytest.mark.parametrize("longest", [100, 2047, 3000])
def test_evict_many_heads(lk, longest):  # noqa: F811
    """Small workgroups for the choice: a long sequence among short ones, equal weights and NaN, kept tokens from as many octets as there are."""
    rng = np.random.default_rng(longest)
    B, H, page, keep = 33, 16, 16, 40
    lengths = [longest] + [int(n) for n in rng.integers(0, 60, B - 1)]
    W, W_out = -(-longest // page), 3
    P = sum(-(-n // page) for n in lengths) + B * W_out
    c = random_cache(rng, P, H, 64, 4, page, "int8", -6, -3)
    ids = rng.permutation(P).astype(np.int32)
    table, used = np.full((B, W), -1, np.int32), 0
    for b, n in enumerate(lengths):
        held = -(-n // page)
        table[b, :held], used = ids[used:used + held], used + held
    table_out = ids[used:].reshape(B, W_out)
    weights = spread_weights(rng, B, H, W * page)
    weights[:, 1] = np.round(weights[:, 1])
    weights[:, 2, ::3] = np.nan
    weights[0, 3] = 0.5
    pool, out = on_gpu(lk, c), torch.full((B, H, W_out * page), -2.0, device="cuda")
    lk.lookat_pages_evict(pool, dev(table), i32(*lengths), dev(weights), i32(*[keep] * B), dev(table_out), first=2, recent=3, weights_out=out)
    after, _, want = evict_reference(c, table, lengths, weights, [keep] * B, 2, 3, table_out, np.full((B, H, W_out * page), -2.0, np.float32))
    assert np.array_equal(out.cpu().numpy(), want, equal_nan=True)
    assert_pool(pool, after)


def test_evict_weights_of_all_kinds(lk):  # noqa: F811
    """Equal weights, zeros of both signs, infinities, NaN, subnormals, fewer columns than tokens, strided weights, ids outside the pool."""
    rng = np.random.default_rng(3)
    H, page, n, B, W, W_out = 2, 32, 300, 8, 10, 6
    P = B * (W + W_out)
    c = random_cache(rng, P, H, 64, 4, page, "float8")
    c.values[rng.random(c.values.shape) < 0.01] = 0x7f         # (stored by something else: counts as zero)
    c.exponents[3] = 100
    c.exponents[4] = -128
    ids = rng.permutation(P).astype(np.int32)
    table, table_out = ids[:B * W].reshape(B, W), ids[B * W:].reshape(B, W_out)
    table[6, 2], table[6, 7], table_out[7, 1] = -1, P, -1
    w = np.zeros((B, H, 250), np.float32)
    w[1] = 1.0
    w[2] = rng.choice(np.array([0.0, -0.0], np.float32), (H, 250))
    w[3] = rng.choice(np.array([np.inf, -np.inf, np.nan, 1.0, -1.0], np.float32), (H, 250))
    w[4] = rng.integers(0, 50, (H, 250)) * np.float32(1e-45)
    w[5] = rng.integers(0, 3, (H, 250))
    w[6:] = spread_weights(rng, 2, H, 250)
    wide = np.full((B, H, 400), 9e9, np.float32)
    wide[:, :, :250] = w
    keep = [170, 100, 100, 140, 55, 131, 150, 192]
    for first, recent in ((0, 0), (5, 17)):
        pool = on_gpu(lk, c)
        lk.lookat_pages_evict(pool, dev(table), i32(*[n] * B), dev(wide)[:, :, :250], i32(*keep), dev(table_out), first=first, recent=recent)
        after, _, _ = evict_reference(c, table, [n] * B, w, keep, first, recent, table_out, None)
        assert_pool(pool, after)


def test_evict_long(lk):  # noqa: F811
    """More tokens than a workgroup has threads in several rounds, and positions of which many are equal."""
    rng = np.random.default_rng(4)
    page, n, H = 128, 70001, 1
    W = -(-n // page)
    keep = 30000
    W_out = -(-keep // page)
    c = random_cache(rng, W + W_out, H, 64, 2, page, "int8", -4, -1)
    ids = rng.permutation(W + W_out).astype(np.int32)
    table, table_out = ids[None, :W], ids[None, W:]
    weights = rng.integers(0, 40, (1, H, n)).astype(np.float32) / 7
    pool = on_gpu(lk, c)
    lk.lookat_pages_evict(pool, dev(table), i32(n), dev(weights), i32(keep), dev(table_out), first=10, recent=100)
    after, _, _ = evict_reference(c, table, [n], weights, [keep], 10, 100, table_out, None)
    assert_pool(pool, after)


def test_weigh_and_evict_in_a_graph(lk):  # noqa: F811
    """A decode step that weighs and evicts, captured once: replays on other inputs give what eager calls give."""
    rng = np.random.default_rng(6)
    H, g, m, page, B, W, W_out = 2, 4, 8, 64, 3, 40, 10
    P = B * (W + W_out)
    c = random_cache(rng, P, H, 128, m, page, "int8")
    ids = rng.permutation(P).astype(np.int32)
    table, table_out = dev(ids[:B * W].reshape(B, W)), dev(ids[B * W:].reshape(B, W_out))
    lengths, keep = i32(2500, 700, 64), i32(600, 600, 600)
    lut = dev(random_lut(rng, B, H * g, m))
    pool = on_gpu(lk, c)
    weights, weights_out = torch.zeros((B, H, W * page), device="cuda"), torch.zeros((B, H, W_out * page), device="cuda")
    ws1 = torch.empty(max(1, lk.pages_weigh_workspace_bytes(pool, B, g, W)), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(lk.pages_evict_workspace_bytes(pool, B, W_out), dtype=torch.uint8, device="cuda")

    def step():
        lk.lookat_pages_weigh(lut, pool, table, lengths, 0.2, weights, decay=0.9, workspace=ws1)
        lk.lookat_pages_evict(pool, table, lengths, weights, keep, table_out, first=4, recent=32, weights_out=weights_out, workspace=ws2)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        lut.mul_(-0.7)
        lengths.copy_(i32(2500 - 100 * k, 700, 64 + k))
        start = weights.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (weights, weights_out, *(y.view(torch.uint8) for y in pool))]
        weights.copy_(start)
        pool.values.view(torch.uint8)[table_out.long().view(-1)] = 0
        weights_out.zero_()
        step()
        k = lengths.clamp(max=600).tolist()
        for b in range(B):
            assert torch.equal(got[1][b, :, :k[b]], weights_out[b, :, :k[b]])
            pages = table_out[b, :k[b] // page].long()
            assert torch.equal(got[3][pages], pool.values.view(torch.uint8)[pages])
            assert torch.equal(got[4][pages], pool.exponents.view(torch.uint8)[pages])
        assert torch.equal(got[0], weights)
