"""Chunks, eviction and beam selection at the ends of what their documentation allows."""
import math

import numpy as np
import pytest
import torch

from bars import record
from test_gpu_pages import assert_pool, dev, i32, lk, on_gpu, random_cache  # noqa: F401
from test_gpu_pages_chunk import U
from test_gpu_pages_keep import evict_reference, spread_weights

pytestmark = pytest.mark.gpu

# sizes of chunks that take every kernel: B, H, g, N, before, d_k, m, page, num_splits
CHUNKS = [
    (2, 43, 1, 770, 1400, 128, 8, 32, 0),     # 256 rows to a workgroup
    (8, 32, 1, 260, 150, 128, 8, 32, 0),      # 128 rows
    (10, 10, 2, 128, 100, 128, 2, 64, 0),
    (6, 20, 2, 150, 100, 64, 8, 32, 0),
    (8, 32, 1, 260, 0, 64, 16, 16, 0),        # ... with centroids of four coordinates
    (6, 2, 4, 100, 900, 128, 2, 64, 0),       # few rows or heads: eight wavefronts, two blocks of rows
    (5, 20, 3, 7, 333, 64, 16, 16, 0),
    (8, 3, 2, 8, 200, 64, 8, 64, 0),          # ... one
    (40, 16, 4, 4, 60, 64, 4, 64, 0),         # two wavefronts, one block
    (40, 16, 5, 6, 100, 128, 4, 128, 0),      # ... two
    (40, 16, 1, 50, 20, 64, 16, 16, 0),
    (6, 20, 2, 150, 200, 64, 8, 32, 3),       # in ranges
    (8, 32, 1, 260, 400, 128, 8, 32, 2),
    (2, 3, 8, 16, 1000, 64, 8, 64, 4),
    (8, 3, 2, 8, 200, 128, 8, 64, 0),         # one block of rows at d_k = 128, eight wavefronts and two
    (40, 16, 4, 4, 60, 128, 16, 64, 0),
    (40, 16, 1, 50, 20, 64, 8, 32, 0),        # two wavefronts, two blocks, centroids of eight coordinates
    (8, 3, 2, 8, 200, 64, 16, 64, 0),         # one block, centroids of four, eight wavefronts and two
    (40, 16, 4, 4, 60, 64, 16, 64, 0),
    (40, 16, 5, 6, 100, 128, 4, 128, 3)]      # two wavefronts in ranges, the last of them short


@pytest.mark.parametrize("dtype", ["float16", "float32"])
@pytest.mark.parametrize("B,H,g,N,before,d_k,m,page,splits", CHUNKS)
def test_a_stored_nan_reaches_the_rows_that_see_its_token(lk, B, H, g, N, before, d_k, m, page, splits, dtype):  # noqa: F811
    """e4m3 has a NaN.  The coordinate that holds one is NaN in the rows from its token's position on, and no other output is touched: the
    bound is that of test_gpu_pages_chunk's `against_torch`, with zeros in the NaNs' places."""
    gen = torch.Generator(device="cuda").manual_seed(B + N + d_k)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    lengths = [max(1, N + before - 3 * b) for b in range(B)]
    counts = [max(1, N - 2 * b) for b in range(B)]
    W = -(-max(lengths) // page)
    P = B * W
    stored = (rnd(P, H, page // 8, d_k, 8) * 30).to(torch.float8_e4m3fn).view(torch.uint8)
    table = torch.randperm(P, generator=gen, device="cuda").to(torch.int32).view(B, W)
    for b in range(B):
        n, k = lengths[b], counts[b]
        # (the last token, the first of the chunk, some between, and one that all rows see)
        for x, t in enumerate(sorted({max(0, n - x) for x in (1, k, 1 + k // 3, 1 + k // 2, k + 40)})):
            stored[table[b, t // page].long(), (3 * b + x) % H, t % page // 8, (17 * b + 5 * x) % d_k, t % 8] = 0x7f if x % 2 else 0xff
        if n < W * page:                              # (and bytes that no row sees)
            stored[table[b, n // page].long(), :, n % page // 8, :, n % 8] = 0x7f
    pool = lk.PagePool(torch.randint(0, 256, (P, H, page, m), generator=gen, device="cuda", dtype=torch.uint8), stored.view(torch.float8_e4m3fn),
                       torch.randint(-8, -2, (P, H), generator=gen, device="cuda").to(torch.int8))
    books = rnd(H, m, 256, d_k // m)
    q = rnd(B, H * g, N, d_k).to(getattr(torch, dtype))
    scale = 1 / math.sqrt(d_k)
    got = lk.lookat_attend_pages_chunk(q, books, pool, table, i32(*lengths), scale, counts=i32(*counts), num_splits=splits)
    head, sub = torch.arange(H, device="cuda")[:, None, None], torch.arange(m, device="cuda")
    reached = 0
    for b in range(B):
        n, k, ids = lengths[b], counts[b], table[b].long()
        code = pool.codes[ids].permute(1, 0, 2, 3).reshape(H, -1, m)[:, :n].long()
        key = books.double()[head, sub, code].reshape(H, n, d_k)
        val = pool.values[ids].double() * torch.exp2(pool.exponents[ids].double())[..., None, None, None]
        val = val.permute(1, 0, 2, 4, 3).reshape(H, -1, d_k)[:, :n]
        nan, val = val.isnan(), val.nan_to_num(0.0)
        x = q[b, :, :k].double().reshape(H, g * k, d_k)
        y = torch.matmul(x, key.transpose(1, 2).contiguous()).view(H, g, k, n) * scale
        size = torch.matmul(x.abs(), key.abs().transpose(1, 2).contiguous()).amax(-1).view(H, g, k, 1) * scale * 1.4427
        seen = torch.arange(n, device="cuda") <= n - k + torch.arange(k, device="cuda")[:, None]
        p = torch.softmax(y.masked_fill(~seen, -math.inf), -1)
        p = torch.where(seen.any(-1, keepdim=True), p, 0.0)
        want = torch.matmul(p.view(H, g * k, n), val).view(H, g, k, d_k)
        want = want.masked_fill((torch.matmul(seen.double(), nan.double()) > 0).view(H, 1, k, d_k), math.nan).view(H * g, k, d_k)
        d = (3 * 2.0 ** -22 + (d_k + 3) * U) * size + 6 * U * (size + 64) \
            + d_k * 2.0 ** -38 * x.abs().amax(-1).view(H, g, k, 1) * books.abs().amax().double() * scale * 1.4427
        rel = 2 * (d * 0.6932 + 2.0 ** -21) + 4 * math.sqrt(n + 64) * U
        floor = 1.01 * 2.0 ** (-3 - 32) * 448 * n
        bound = (rel * torch.matmul(p.view(H, g * k, n), val.abs()).view(H, g, k, d_k)).reshape(H * g, k, d_k) + floor
        mine = got[b, :, :k].double()
        assert torch.equal(mine.isnan(), want.isnan()), (b, int((mine.isnan() != want.isnan()).sum()))
        assert bool(((mine - want).abs() <= bound)[~want.isnan()].all()), b
        assert not got[b, :, k:].any()
        reached += int(want.isnan().sum())
    assert reached


@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("dtype", ["float16", "float32"])
@pytest.mark.parametrize("B,H,g,N,before,d_k,m,page,splits", [CHUNKS[i] for i in (1, 3, 5, 7, 8, 11)])
def test_a_scale_of_nan(lk, B, H, g, N, before, d_k, m, page, splits, dtype, kind):  # noqa: F811
    """Every row that sees a token is NaN, as attention of one token is; a row that sees none gives zeros."""
    rng = np.random.default_rng(N)
    lengths = [N + before - b for b in range(B)]
    lengths[0] = 3                                    # (its first rows stand before its first token)
    W = -(-max(lengths) // page)
    c = random_cache(rng, W, H, d_k, m, page, kind)
    pool, table = on_gpu(lk, c), dev(np.tile(rng.permutation(W).astype(np.int32), (B, 1)))
    books = dev(rng.standard_normal((H, m, 256, d_k // m)).astype(np.float32))
    q = dev(rng.standard_normal((B, H * g, N, d_k)).astype(dtype))
    got = lk.lookat_attend_pages_chunk(q, books, pool, table, i32(*lengths), math.nan, num_splits=splits)
    sees = i32(*lengths)[:, None] - N + torch.arange(N, device="cuda") >= 0
    assert torch.equal(got.isnan(), sees[:, None, :, None].expand(got.shape))
    assert not got.nan_to_num(0.0).any()
    if g in (1, 2, 4, 8):
        lut = dev(rng.standard_normal((B, H * g, m, 256)).astype(np.float32))
        one = lk.lookat_attend_pages(lut, pool, table, i32(*[0, *lengths[1:]]), math.nan)
        assert bool(one[1:].isnan().all()) and not one[0].any()


@pytest.mark.parametrize("N,H,splits", [(4, 2, 1), (4, 2, 3), (200, 60, 1), (200, 60, 2)])
@pytest.mark.parametrize("d_k,m", [(64, 8), (128, 16)])
def test_a_stored_nan_among_scores_of_minus_infinity(lk, N, H, splits, d_k, m):  # noqa: F811
    """A row whose scores are all -inf gives zeros, but NaN at the coordinates at which it sees one, whether its tokens are cut into ranges or not."""
    gen = torch.Generator(device="cuda").manual_seed(N)
    n, page = N + 100, 32
    W = -(-n // page)
    stored = (torch.randn((W, H, page // 8, d_k, 8), generator=gen, device="cuda") * 30).to(torch.float8_e4m3fn).view(torch.uint8)
    at = n - 1 - N // 2
    stored[at // page, :, at % page // 8, 3, at % 8] = 0x7f
    stored[1, 0, 0, 7, 5] = 0xff                      # (one that all rows see)
    pool = lk.PagePool(torch.randint(0, 256, (W, H, page, m), generator=gen, device="cuda", dtype=torch.uint8), stored.view(torch.float8_e4m3fn),
                       torch.zeros((W, H), dtype=torch.int8, device="cuda"))
    books = torch.rand((H, m, 256, d_k // m), generator=gen, device="cuda") + 0.5
    q = -torch.rand((1, H, N, d_k), generator=gen, device="cuda") - 0.5
    got = lk.lookat_attend_pages_chunk(q, books, pool, torch.arange(W, dtype=torch.int32, device="cuda")[None], i32(n), 3e38, num_splits=splits)
    want = torch.zeros_like(got)
    want[0, :, at - (n - N):, 3] = math.nan
    want[0, 0, :, 7] = math.nan
    assert torch.equal(got.isnan(), want.isnan())
    assert not got.nan_to_num(0.0).any()


SUM = 2.0 ** -18       # of a row's sum of exponentials (include/lookat_search.h); a score is off by as much, and by its own rounding


@pytest.mark.parametrize("dtype", ["float16", "float32"])
@pytest.mark.parametrize("V", [20000, 131072])
def test_peaks_above_many_equal_logits(lk, V, dtype):  # noqa: F811
    """Every term's rounding goes the same way.  Terms e^d beside peaks of 1: with u = 2^-24 a term is off by |d| u for the difference, |d| (u + u / 4) for its product
    with log2(e), 2 u for the exponential, and the sum of a lane's terms by 16 u; for d > -14 that is 50 u < 2^-18."""
    top = 0.0
    for base in np.arange(-9, 12, 0.37):
        d = -torch.linspace(0.05, 14, 160, device="cuda", dtype=torch.float64)
        x = (base + d[:, None]).expand(160, V).to(getattr(torch, dtype)).contiguous()
        x[:, ::2048] = float(base)
        want = x[:, 0].double() - torch.logsumexp(x.double(), -1)
        s = lk.lookat_beam_select(x, torch.zeros(160, device="cuda"), 1, 1)[0][:, 0].double()
        off = (s - want).abs() - 2.0 ** -24 * want.abs()
        top = max(top, float(off.max()))
    record(f"log-sum of a peaked row, {V} {dtype}", top)
    assert top <= SUM


@pytest.mark.parametrize("room,n", [(5000, 4900), (8192, 8192), (8193, 8193), (20000, 20000), (32768, 32768), (32768, 700), (32769, 30000)])
@pytest.mark.parametrize("page,kind", [(16, "int8"), (128, "float8")])
def test_the_choice_of_long_evictions(lk, room, n, page, kind):  # noqa: F811
    """Weights of 8 and of 32 tokens a thread in registers, and read again: many equal weights on both sides of the border, NaN, lengths far below a row's room."""
    rng = np.random.default_rng(room + n)
    H, B = 3, 2
    W = -(-room // page)
    lengths, keep = [n, n // 3], [n // 4 + 1, n // 10]
    W_out = -(-max(keep) // page)
    held = [-(-x // page) for x in lengths]
    P = sum(held) + B * W_out
    c = random_cache(rng, P, H, 64, 4, page, kind, -5, -2)
    ids = rng.permutation(P).astype(np.int32)
    table = np.full((B, W), -1, np.int32)
    table[0, :held[0]], table[1, :held[1]] = ids[:held[0]], ids[held[0]: sum(held)]
    table_out = ids[sum(held):].reshape(B, W_out)
    weights = spread_weights(rng, B, H, W * page)
    weights[:, 1] = rng.integers(0, 4, weights[:, 1].shape) / 7      # (the border lies among equal ones)
    weights[0, 2] = 0.25                                             # (all equal)
    weights[1, 2, ::5] = np.nan
    start = np.full((B, H, W_out * page), -2.0, np.float32)
    pool, out = on_gpu(lk, c), dev(start)
    ws = torch.empty(lk.pages_evict_workspace_bytes(pool, B, W_out), dtype=torch.uint8, device="cuda")
    lk.lookat_pages_evict(pool, dev(table), i32(*lengths), dev(weights), i32(*keep), dev(table_out), first=4, recent=64, weights_out=out, workspace=ws)
    after, places, want = evict_reference(c, table, lengths, weights, keep, 4, 64, table_out, start)
    got = ws.view(torch.int32).view(B, H, W_out * page).cpu().numpy()
    for (b, h), at in places.items():
        assert got[b, h, :len(at)].tolist() == at, (b, h)
    assert np.array_equal(out.cpu().numpy(), want, equal_nan=True)
    assert_pool(pool, after)


def select_reference(x, scores, beams, n):
    """In 64 bits by a stable sort: scores, parents, tokens, and the least distance between neighbours of different beams that are not equal."""
    R, V = x.shape
    s = (x.double() - torch.logsumexp(x.double(), -1, keepdim=True) + scores.double()[:, None]).view(R // beams, beams * V)
    s, at = torch.where(s.isnan(), -math.inf, s).sort(dim=-1, descending=True, stable=True)
    s, at = s[:, :n + 1], at[:, :n + 1]
    row = torch.arange(R // beams, device=x.device)[:, None] * beams + at // V
    gap = (s[:, :-1] - s[:, 1:])[(row[:, :-1] != row[:, 1:]) & (s[:, :-1] != s[:, 1:]) & s[:, 1:].isfinite()]
    none = s[:, :n] == -math.inf
    return s[:, :n], row[:, :n].masked_fill(none, -1), (at % V)[:, :n].masked_fill(none, -1), float(gap.min()) if gap.numel() else math.inf


def check_select(lk, x, scores, beams, n):  # noqa: F811
    want = select_reference(x, scores, beams, n)
    assert want[3] > 2 * SUM, "the inputs have a near tie"
    s, parents, tokens = lk.lookat_beam_select(x, scores, beams, n)
    assert torch.equal(parents.long(), want[1]) and torch.equal(tokens.long(), want[2])
    ok = want[0].isfinite()
    assert torch.equal(s.isneginf(), ~ok)
    assert bool(((s.double() - want[0]).abs() <= SUM + 2.0 ** -24 * want[0].abs())[ok].all())


@pytest.mark.parametrize("dtype", ["float16", "float32"])
@pytest.mark.parametrize("Q,beams,V,n", [(1, 5, 300000, 9), (1, 3, 400001, 64), (2, 17, 70000, 30), (1, 600, 1025, 12), (300, 2, 30001, 5)])
def test_selection_by_32_logits_a_lane(lk, Q, beams, V, n, dtype):  # noqa: F811
    """Large launches and many lists.  Beams far apart, so that half-precision logits make no near ties between them."""
    gen = torch.Generator(device="cuda").manual_seed(V + n)
    x = torch.randn((Q * beams, V), generator=gen, device="cuda")
    x = (2 * x + 4 * (x - 2).clamp(min=0)).to(getattr(torch, dtype))
    if beams > 2:
        x[1] = -math.inf
        x[2, : V - 3] = -math.inf
    # (scores with a near tie between beams are passed over)
    for seed in range(40):
        scores = -torch.rand(Q * beams, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * 30
        if select_reference(x, scores, beams, n)[3] > 2 * SUM:
            break
    check_select(lk, x, scores, beams, n)


@pytest.mark.parametrize("dtype", ["float16", "float32"])
@pytest.mark.parametrize("n", [1, 40, 64])
@pytest.mark.parametrize("beams,V", [(1, 40000), (5, 300000)])       # (16 and 32 logits a lane)
def test_equal_logits(lk, beams, V, n, dtype):  # noqa: F811
    """More equal logits than a list holds, the n-th of them in either half of its part or between its halves, at the ends of parts and of the row."""
    at = torch.arange(V, device="cuda")
    rows = [torch.zeros(V, device="cuda"), (at % 2).float(), (at % 2048 >= 1004).float(), (at % 2048 >= 1084).float() * 2, (at % 2048 >= 2000).float(),
            (at >= V - 700).float(), torch.where(at % 2 == 0, 0.0, -0.0), torch.where(at == V - 1, 1.0, 0.0), torch.where(at < 30, -math.inf, 3.0)]
    for row in rows:
        x = row.to(getattr(torch, dtype)).expand(beams, V).contiguous()
        scores = torch.zeros(beams, device="cuda")
        check_select(lk, x, scores, beams, n)
        check_select(lk, x, scores - 5 * torch.arange(beams, device="cuda"), beams, n)


def test_scores_in_place(lk):  # noqa: F811
    """A search step whose scores take the place of the last ones (as many beams as before), eager and replayed."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    Q, beams, V = 40, 5, 3001
    x = torch.randn((Q * beams, V), generator=gen, device="cuda")
    start = -torch.rand(Q * beams, generator=gen, device="cuda")
    want = lk.lookat_beam_select(x, start, beams, beams)
    scores = start.clone()
    parents, tokens = torch.empty((Q, beams), dtype=torch.int32, device="cuda"), torch.empty((Q, beams), dtype=torch.int32, device="cuda")
    ws = torch.empty(lk.beam_select_workspace_bytes(Q, beams, V, beams), dtype=torch.uint8, device="cuda")
    step = lambda: lk.lookat_beam_select(x, scores, beams, beams, scores_out=scores.view(Q, beams), parents=parents, tokens=tokens, workspace=ws)  # noqa: E731
    step()
    assert torch.equal(scores.view(Q, beams), want[0]) and torch.equal(parents, want[1]) and torch.equal(tokens, want[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        want = lk.lookat_beam_select(x, scores.clone(), beams, beams)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(scores.view(Q, beams), want[0]) and torch.equal(parents, want[1]) and torch.equal(tokens, want[2])
