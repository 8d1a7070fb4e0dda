"""Attention of a chunk over the paged cache against a plain form in 64 bits, at a bound derived in `reference`."""
import math

import numpy as np
import pytest
import torch

import pages_ref as pr
from bars import record
from test_gpu_pages import TORCH, dev, i32, lk, on_gpu, random_cache, random_table  # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def reference(c, q, books, table, lengths, counts, scale, out):
    """(out, bound) with `out` [B, Hq, N, d_k] kept where no row counts.

    The bound: a product with a centroid is off by 2^-22 of itself, with an fp32 query twice that and the product of the small terms, 2^-22, again
    (3 * 2^-22; 2^-39 of the largest entries' products besides, for entries below 2^-17 of those), its sum over d_k coordinates in fp32 by d_k u of
    sum |q||k^|; scaling and the exponent's addition by 3 u of what they give and of the reference.  That is d for a logit in log2 units; the
    weight is off by d ln 2 + 2^-21 (exponential unit, two fp16 terms) of itself, numerator and denominator both.  Sums of n terms: 4 sqrt(n + 64) u.
    Last, where fp16 ends, as in pages_ref.Cache.attend: 2^(e - 32) sum |q|, e the exponent of the token of the largest logit with exponent."""
    B, Hq, N, d_k = q.shape
    H, m = books.shape[:2]
    g = Hq // H
    out = out.astype(np.float64).copy()
    bound = np.zeros_like(out)
    books = books.astype(np.float64)
    for b in range(B):
        count = max(0, N if counts is None else int(counts[b]))
        given = max(0, int(lengths[b]))
        reach = min(given, table.shape[1] * c.page)
        pos = [t for t in range(reach) if 0 <= table[b, t // c.page] < c.P]
        codes, v, e = c.tokens(table[b], reach, True)
        for h in range(H):
            key = books[h][np.arange(m), codes[h]].reshape(-1, d_k) if len(pos) else np.zeros((0, d_k))
            biggest = np.abs(books[h][np.isfinite(books[h])]).max()
            for n in range(min(count, N)):
                seen = sum(1 for t in pos if t <= given - count + n)
                for hq in range(h * g, (h + 1) * g):
                    out[b, hq, n] = 0
                    if not seen:
                        continue
                    x = q[b, hq, n].astype(np.float64)
                    y = key[:seen] @ x * scale
                    p = np.exp(y - y.max())
                    p /= p.sum()
                    out[b, hq, n] = p @ v[h, :seen]
                    size = (np.abs(key[:seen]) @ np.abs(x)).max() * abs(scale) * 1.4427
                    tail = d_k * np.abs(x).max() * biggest * abs(scale) * 1.4427 * 2.0 ** -38
                    d = (3 * 2.0 ** -22 + (d_k + 3) * U) * size + tail + 6 * U * (size + 64)
                    rel = 2 * (d * 0.6932 + 2.0 ** -21) + 4 * math.sqrt(seen + 64) * U
                    top = float(e[h, np.argmax(y / math.log(2) + e[h, :seen])])
                    floor = 1.01 * 2.0 ** (top - 32) * np.abs(v[h, :seen] * 2.0 ** -e[h, :seen, None]).sum(0)
                    bound[b, hq, n] = rel * (p @ np.abs(v[h, :seen])) + floor
    return out, bound


def check(lk, c, q, books, table, lengths, counts, scale=None, order="heads", label="chunk attention", **kw):  # noqa: F811
    scale = 1 / math.sqrt(c.d_k) if scale is None else scale
    start = np.full(q.shape, -7.5, np.float32)
    out = dev(start)
    x = dev(q.transpose(0, 2, 1, 3)).transpose(1, 2) if order == "tokens" else dev(q)
    got = lk.lookat_attend_pages_chunk(x, dev(books), on_gpu(lk, c), dev(table), i32(*lengths), scale, counts=None if counts is None else i32(*counts),
                                       out=out, **kw)
    assert got is out
    want, bound = reference(c, q, books, table, lengths, counts, scale, start)
    got = got.cpu().numpy().astype(np.float64)
    record(label, float(np.max(np.abs(got - want))))
    worst = np.max(np.abs(got - want) - bound)
    assert worst <= 0, (worst, np.argwhere(np.abs(got - want) > bound)[:5].tolist())
    return got


def books_of(rng, H, m, d_k, size=1.0):
    return (rng.standard_normal((H, m, 256, d_k // m)) * size).astype(np.float32)


SHAPES = [(64, 4, 16), (64, 16, 64), (128, 8, 32), (128, 16, 128), (64, 2, 128), (128, 2, 64), (64, 8, 32), (128, 4, 16)]


@pytest.mark.parametrize("dtype", ["float16", "float32"])
@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("d_k,m,page", SHAPES)
def test_chunks(lk, d_k, m, page, kind, dtype):  # noqa: F811
    """Rows at the start, behind other tokens, fewer than given, none, more than the sequence has tokens; pages that end inside a tile of keys."""
    rng = np.random.default_rng(d_k + m + page)
    N, H, g = 37, 2, 2
    lengths = [37, 100, 1, 0, 64, 129, 20, 36]
    counts = [37, 37, 1, 0, 5, 40, 30, 37]
    W = max(-(-n // page) for n in lengths)
    c = random_cache(rng, 40, H, d_k, m, page, kind)
    table = random_table(rng, lengths, page, W, 40)
    q = rng.standard_normal((8, H * g, N, d_k)).astype(dtype)
    for order, splits in (("heads", 0), ("tokens", 1), ("heads", 3)):
        check(lk, c, q, books_of(rng, H, m, d_k), table, lengths, counts, order=order, num_splits=splits)


@pytest.mark.parametrize("g", [1, 3, 8, 64])
@pytest.mark.parametrize("N", [1, 2, 33, 130, 300])
def test_rows_and_groups(lk, N, g):  # noqa: F811
    """Tiles of rows filled in part, rows of a token on both sides of a tile's end, both sizes of workgroups."""
    rng = np.random.default_rng(N * g)
    if N * g > 2600:
        N = 2600 // g
    H, d_k, m, page = 1, 64, 8, 32
    lengths = [N + 70, N]
    c = random_cache(rng, 40, H, d_k, m, page, "int8")
    table = random_table(rng, lengths, page, 12, 40)
    q = rng.standard_normal((2, H * g, N, d_k)).astype(np.float16)
    check(lk, c, q, books_of(rng, H, m, d_k), table, lengths, None)


@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_sharp_logits_and_exponents(lk, kind):  # noqa: F811
    """Logits of hundreds, and pages whose exponents lie 80 apart."""
    rng = np.random.default_rng(8)
    c = random_cache(rng, 24, 2, 128, 8, 16, kind, -40, 41)
    lengths = [200, 150]
    table = random_table(rng, lengths, 16, 13, 24)
    q = (rng.standard_normal((2, 4, 50, 128)) * 8).astype(np.float32)
    check(lk, c, q, books_of(rng, 2, 8, 128, 3.0), table, lengths, [50, 20], label="chunk attention, sharp (relative to 2^40)")


def test_pages_outside_the_pool_and_bytes_behind_the_end(lk):  # noqa: F811
    """Ids outside the pool hold no tokens; what pages have behind a sequence's end, NaN among it, and centroids that no token has do not matter."""
    rng = np.random.default_rng(9)
    c = random_cache(rng, 24, 2, 64, 4, 16, "float8")
    lengths, counts = [90, 75, 60, 40], [20, 20, 20, 20]
    table = random_table(rng, lengths, 16, 6, 24)
    table[0, 2], table[1, 0], table[1, 4], table[2, :] = -1, 24, 1 << 30, -5
    held = {}
    for b in range(4):
        for t in range(lengths[b]):
            held.setdefault(int(table[b, t // 16]), set()).add(t % 16)
    used = np.zeros((2, 4, 256), bool)
    for i in range(24):
        for t in range(16):
            if t in held.get(i, ()):
                for h in range(2):
                    used[h, np.arange(4), c.codes[i, h, t]] = True
            else:
                c.row(i, 0, t)[:] = 0x7f
                c.row(i, 1, t)[:] = 0xff
    books = books_of(rng, 2, 4, 64)
    clean = books.copy()
    books[~used] = np.nan
    books[0][~used[0]] = np.inf
    q = rng.standard_normal((4, 2, 20, 64)).astype(np.float16)
    want, bound = reference(c, q, clean, table, lengths, counts, 0.125, np.zeros(q.shape))
    for splits in (1, 2):
        got = lk.lookat_attend_pages_chunk(dev(q), dev(books), on_gpu(lk, c), dev(table), i32(*lengths), 0.125, counts=i32(*counts), num_splits=splits)
        got = got.cpu().numpy()
        assert np.all(np.abs(got - want) <= bound)
        assert not got[2].any()


def test_scores_that_are_not_finite(lk):  # noqa: F811
    """A query row with a NaN, one that makes scores infinite: their rows alone."""
    rng = np.random.default_rng(10)
    c = random_cache(rng, 8, 1, 64, 4, 32, "int8")
    table = random_table(rng, [100], 32, 4, 8)
    books = books_of(rng, 1, 4, 64)
    q = rng.standard_normal((1, 2, 40, 64)).astype(np.float32)
    want, bound = reference(c, q, books, table, [100], None, 0.125, np.zeros(q.shape))
    q[0, 0, 3, 5] = np.nan
    q[0, 1, 7, 9] = np.inf
    got = lk.lookat_attend_pages_chunk(dev(q), dev(books), on_gpu(lk, c), dev(table), i32(100), 0.125).cpu().numpy()
    assert np.isnan(got[0, 0, 3]).all() and np.isnan(got[0, 1, 7]).all()
    got[0, 0, 3], got[0, 1, 7] = want[0, 0, 3], want[0, 1, 7]
    assert np.all(np.abs(got - want) <= bound)


@pytest.mark.parametrize("q_size,book_size,scale", [(1e-6, 1.0, 1e5), (1.0, 1e-30, 1e29), (1e30, 1e-28, 0.01), (1e37, 1e-37, 0.3), (1e-37, 1e36, 1.0), (2.0, 1.0, -0.2),
                                                    (1.0, 1.0, 0.0)])
def test_sizes_and_scales(lk, q_size, book_size, scale):  # noqa: F811
    """Queries and centroids near both ends of their types, a scale below zero and one of zero."""
    rng = np.random.default_rng(13)
    for dtype in ("float16", "float32"):
        if dtype == "float16" and not 1e-7 < q_size < 1e4:
            continue
        for N, before in ((6, 90), (140, 0)):
            c = random_cache(rng, 20, 2, 64, 4, 16, "int8")
            table = random_table(rng, [N + before, N], 16, 10, 20)
            q = (rng.standard_normal((2, 2, N, 64)) * q_size).astype(dtype)
            check(lk, c, q, books_of(rng, 2, 4, 64, book_size), table, [N + before, N], None, scale)


def test_strides_offsets_and_graphs(lk):  # noqa: F811
    """Queries inside a larger projection, tables with room behind the rows, another stream, a captured call replayed on new inputs."""
    rng = np.random.default_rng(11)
    H, g, d_k, m, page, N, B = 2, 4, 128, 8, 64, 24, 3
    lengths, counts = [300, 90, 24], [24, 24, 20]
    c = random_cache(rng, 12, H, d_k, m, page, "int8")
    wide = np.full((B, 9), -1, np.int32)
    wide[:, :5] = random_table(rng, lengths, page, 5, 12)
    books = books_of(rng, H, m, d_k)
    qkv = rng.standard_normal((B, N, H * g + 2 * H, d_k)).astype(np.float16)
    q = qkv[:, :, :H * g].transpose(0, 2, 1, 3)
    want, bound = reference(c, q, books, wide[:, :5], lengths, counts, 0.09, np.zeros(q.shape))
    pool, d_books, d_wide, d_qkv = on_gpu(lk, c), dev(books), dev(wide), dev(qkv)
    d_q, d_len, d_cnt = d_qkv[:, :, :H * g].transpose(1, 2), i32(*lengths), i32(*counts)
    need = lk.attend_pages_chunk_workspace_bytes(pool, B, N, g, 5, 0, 2)
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros((B, H * g, N, d_k), device="cuda")
    call = lambda: lk.lookat_attend_pages_chunk(d_q, d_books, pool, d_wide[:, :5], d_len, 0.09, counts=d_cnt, num_splits=2, workspace=ws, out=out)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    assert np.all(np.abs(out.cpu().numpy() - want) <= bound)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        d_qkv.mul_(-0.5)
        d_len.copy_(i32(300 - k, 90, 24))
        out.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone()
        out.fill_(-1.0)
        call()
        assert torch.equal(first, out)
    # any alignment: copied by the binding
    odd = torch.empty(d_q.numel() + 1, dtype=torch.float16, device="cuda")[1:].view(d_q.shape).copy_(d_q)
    assert torch.equal(lk.lookat_attend_pages_chunk(odd, d_books, pool, d_wide[:, :5], d_len, 0.09, counts=d_cnt, num_splits=2),
                       lk.lookat_attend_pages_chunk(d_q, d_books, pool, d_wide[:, :5], d_len, 0.09, counts=d_cnt, num_splits=2))


def test_one_row_is_attention_of_one_token(lk):  # noqa: F811
    """A chunk of one row and lookat_attend_pages on its tables agree to both bounds."""
    rng = np.random.default_rng(12)
    c = random_cache(rng, 40, 4, 64, 4, 64, "float8")
    lengths = [700, 65, 1]
    table = random_table(rng, lengths, 64, 11, 40)
    books = books_of(rng, 4, 4, 64)
    q = rng.standard_normal((3, 8, 1, 64)).astype(np.float32)
    got = check(lk, c, q, books, table, lengths, None)
    lut = lk.lookat_build_lut(dev(q.reshape(3, 4, 2, 64)), dev(books)).view(3, 8, 4, 256)
    one = lk.lookat_attend_pages(lut, on_gpu(lk, c), dev(table), i32(*lengths), 0.125).cpu().numpy()
    _, bound = reference(c, q, books, table, lengths, None, 0.125, np.zeros(q.shape))
    assert np.all(np.abs(got[:, :, 0] - one) <= 2 * bound[:, :, 0])


@pytest.mark.parametrize("dtype", ["float16", "float32"])
@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("B,H,g,N,before,d_k,m,page", [
    (2, 43, 1, 770, 1400, 128, 8, 32),    # 256 rows to a workgroup
    (2, 43, 2, 385, 1800, 128, 16, 128),
    (8, 32, 1, 260, 150, 128, 8, 32),     # 128 rows
    (3, 90, 2, 140, 0, 128, 16, 128),     # ... with two rows to a token, prompts
    (6, 2, 4, 100, 900, 128, 2, 64),      # few heads
    (5, 20, 3, 70, 333, 64, 16, 16),
    (40, 16, 4, 4, 60, 64, 4, 64),        # few rows of many heads that see little: two wavefronts
    (40, 16, 5, 6, 100, 128, 4, 128),
    (2, 3, 8, 16, 5000, 64, 8, 64),       # few rows in ranges: 128 of few heads
    (1, 1, 4, 8, 9000, 128, 8, 128),
    (10, 10, 2, 128, 100, 128, 2, 64),    # 128 rows to a workgroup
    (6, 20, 2, 150, 100, 64, 8, 32),
    (40, 16, 1, 50, 20, 64, 16, 16),      # two wavefronts, two tiles of rows
    (2, 3, 1, 700, 0, 64, 8, 16),         # many rows of few heads
    (1, 2, 2, 300, 1500, 128, 2, 64),
    (2, 2, 1, 400, 77, 64, 16, 128)])
def test_every_kernel(lk, B, H, g, N, before, d_k, m, page, dtype, kind):  # noqa: F811
    """The kernels that large and small launches take, against torch in 64 bits."""
    against_torch(lk, B, H, g, N, before, d_k, m, page, dtype, kind)


@pytest.mark.parametrize("B,H,g,N,before,d_k,m,page", [(2, 43, 1, 770, 1400, 128, 4, 64), (8, 32, 1, 260, 400, 128, 8, 32), (10, 10, 2, 128, 300, 128, 4, 64), (6, 20, 2, 150, 200, 64, 8, 32),
                                                       (40, 16, 2, 8, 200, 64, 8, 16), (3, 5, 1, 100, 900, 128, 16, 16)])
def test_every_kernel_in_ranges(lk, B, H, g, N, before, d_k, m, page):  # noqa: F811
    for splits, dtype in ((2, "float16"), (5, "float32")):
        against_torch(lk, B, H, g, N, before, d_k, m, page, dtype, "float8", splits)


def against_torch(lk, B, H, g, N, before, d_k, m, page, dtype, kind, splits=0):  # noqa: F811
    """The bound is that of `reference`, with the row's own sizes."""
    gen = torch.Generator(device="cuda").manual_seed(B + N)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    lengths = [max(1, N + before - 3 * b) for b in range(B)]
    counts = [max(1, N - 2 * b) for b in range(B)]
    W = -(-max(lengths) // page)
    P = B * W
    v = rnd(P, H, page // 8, d_k, 8) * 30
    v = v.round().clamp(-127, 127).to(torch.int8) if kind == "int8" else v.to(torch.float8_e4m3fn)
    pool = lk.PagePool(torch.randint(0, 256, (P, H, page, m), generator=gen, device="cuda", dtype=torch.uint8), v,
                       torch.randint(-8, -2, (P, H), generator=gen, device="cuda").to(torch.int8))
    table = torch.randperm(P, generator=gen, device="cuda").to(torch.int32).view(B, W)
    books = rnd(H, m, 256, d_k // m)
    q = rnd(B, N, H * g, d_k).to(getattr(torch, dtype)).transpose(1, 2)
    scale = 1 / math.sqrt(d_k)
    got = lk.lookat_attend_pages_chunk(q, books, pool, table, i32(*lengths), scale, counts=i32(*counts), num_splits=splits)
    head, sub = torch.arange(H, device="cuda")[:, None, None], torch.arange(m, device="cuda")
    for b in range(B):
        n, k, ids = lengths[b], counts[b], table[b].long()
        code = pool.codes[ids].permute(1, 0, 2, 3).reshape(H, -1, m)[:, :n].long()
        key = books.double()[head, sub, code].reshape(H, n, d_k)
        val = pool.values[ids].double() * torch.exp2(pool.exponents[ids].double())[..., None, None, None]
        val = val.permute(1, 0, 2, 4, 3).reshape(H, -1, d_k)[:, :n]
        x = q[b, :, :k].double().reshape(H, g * k, d_k)
        y = torch.matmul(x, key.transpose(1, 2).contiguous()).view(H, g, k, n) * scale
        size = torch.matmul(x.abs(), key.abs().transpose(1, 2).contiguous()).amax(-1).view(H, g, k, 1) * scale * 1.4427
        seen = torch.arange(n, device="cuda") <= n - k + torch.arange(k, device="cuda")[:, None]
        p = torch.softmax(y.masked_fill(~seen, -math.inf), -1)
        p = torch.where(seen.any(-1, keepdim=True), p, 0.0)       # (rows ahead of the first token: zeros)
        want = torch.matmul(p.view(H, g * k, n), val).view(H * g, k, d_k)
        d = (3 * 2.0 ** -22 + (d_k + 3) * U) * size + 6 * U * (size + 64) \
            + d_k * 2.0 ** -38 * x.abs().amax(-1).view(H, g, k, 1) * books.abs().amax().double() * scale * 1.4427
        rel = 2 * (d * 0.6932 + 2.0 ** -21) + 4 * math.sqrt(n + 64) * U
        # (the last term of `reference`, with every exponent at its largest)
        floor = 1.01 * 2.0 ** (-3 - 32) * pool.values[ids].double().abs().amax() * n
        bound = (rel * torch.matmul(p.view(H, g * k, n), val.abs()).view(H, g, k, d_k)).reshape(H * g, k, d_k) + floor
        off = (got[b, :, :k].double() - want).abs()
        record("chunk attention, every kernel", float(off.max()))
        assert bool((off <= bound).all()), (b, float((off - bound).max()))
        assert not got[b, :, k:].any()
