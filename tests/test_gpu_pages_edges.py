"""The paged cache on the GPU at the edges: tables that are not finite, the ends of fp32, many sequences, what a weight has to be worth."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import pages_ref as pr
from bars import record
from test_gpu_pages import Watch, assert_pool, dev, i32, lk, on_gpu, random_cache, random_table, same_books  # noqa: F401
from test_pages_weights import FORMS, LENGTHS, weights_case, weights_reference

pytestmark = pytest.mark.gpu

CUTS = [{"num_splits": 1}, {"num_splits": 3}, {}, {"max_length": 64}]


# ---- tables that are not finite -----------------------------------------------------------------------------------
def not_finite_case(kind, group, d_k, m):
    """One short and one long sequence (cut by length where the call chooses), a cache of two heads, finite tables."""
    rng = np.random.default_rng(group + d_k + m)
    lengths, H = [70, 2500], 2
    c = random_cache(rng, 50, H, d_k, m, 64, kind)
    table = random_table(rng, lengths, 64, 40, 50)
    lut = (rng.standard_normal((2, H * group, m, 256)) * 2).astype(np.float32)
    return c, table, lengths, lut


def a_code(c, table, length, b, h, i):
    """The code of subspace i that the token in the middle of sequence b has in head h."""
    t = length // 2
    return int(c.codes[table[b, t // c.page], h, t % c.page, i])


@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("group,d_k,m", [(1, 64, 4), (2, 128, 8), (4, 64, 2), (8, 128, 8)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_attend_shows_scores_that_are_no_numbers(lk, kind, group, d_k, m, value):  # noqa: F811
    """A NaN or +inf score: its row is NaN, cut or not, and no other one."""
    c, table, lengths, lut = not_finite_case(kind, group, d_k, m)
    hit = [(0, 0), (1, 2 * group - 1)]                    # (sequence, query head)
    broken = lut.copy()
    for b, hq in hit:
        broken[b, hq, m - 1, a_code(c, table, lengths[b], b, hq // group, m - 1)] = value
    ref, bound = c.attend(lut, table, lengths, 0.1)
    for kw in CUTS:
        out = lk.lookat_attend_pages(dev(broken), on_gpu(lk, c), dev(table), i32(*lengths), 0.1, **kw).cpu().numpy()
        for b in range(2):
            for hq in range(2 * group):
                if (b, hq) in hit:
                    assert np.isnan(out[b, hq]).all(), (b, hq, kw)
                else:
                    assert np.all(np.abs(out[b, hq] - ref[b, hq]) <= bound[b, hq]), (b, hq, kw)


class WithoutTokens(pr.Cache):
    """One head of a cache, without the tokens whose code of subspace i is even."""

    def __init__(self, c, h, i):
        super().__init__(c.codes[:, h: h + 1], c.values[:, h: h + 1], c.exponents[:, h: h + 1], c.kind)
        self.i = i

    def tokens(self, table_row, length, exponents=False):
        every = super().tokens(table_row, length, True)
        return tuple(x[:, every[0][0, :, self.i] % 2 == 1] for x in every)


@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("group,d_k,m", [(1, 64, 4), (2, 128, 8), (8, 128, 8)])
def test_attend_minus_infinity_is_a_token_without_weight(lk, kind, group, d_k, m):  # noqa: F811
    """Half of the codes of one subspace at -inf: the tokens that have them count for nothing.  All of them: zeros."""
    c, table, lengths, lut = not_finite_case(kind, group, d_k, m)
    lut[0, 0, 1, ::2] = lut[1, 1, 0, ::2] = -math.inf
    nothing = group * 2 - 1
    lut[1, nothing, 0, :] = -math.inf
    scale = 0.1
    for kw in CUTS:
        out = lk.lookat_attend_pages(dev(lut), on_gpu(lk, c), dev(table), i32(*lengths), scale, **kw).cpu().numpy()
        assert np.isfinite(out).all() and np.all(out[1, nothing] == 0)
        for b, hq, i in ((0, 0, 1), (1, 1, 0)):
            if (b, hq) == (1, nothing):
                continue
            few = WithoutTokens(c, hq // group, i)
            ref, bound = few.attend(lut[b: b + 1, hq: hq + 1], table[b: b + 1], [lengths[b]], scale)
            assert np.all(np.abs(out[b, hq] - ref[0, 0]) <= bound[0, 0]), (b, hq, kw)


@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("group,d_k,m", [(1, 64, 4), (2, 128, 8), (4, 64, 2), (8, 128, 8)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_attend_table_entries_that_no_token_has(lk, kind, group, d_k, m, value):  # noqa: F811
    """Every entry that no token of the sequence looks up is not finite; what lies behind the last token and in the pool's first page (which lanes
    without a token read) has such codes."""
    rng = np.random.default_rng(group + d_k + m)
    lengths, H, page = [70, 1, 33, 0, 130, 64], 2, 32
    c = random_cache(rng, 20, H, d_k, m, page, kind)
    table = random_table(rng, lengths, page, 6, 19) + 1   # (page 0 is nobody's)
    table[table == 0] = -1
    table[4, 2] = 20                                      # a hole: tokens 64 to 95
    c.codes[:] |= 1
    c.codes[0] = 0
    for b, n in enumerate(lengths):
        if n % page:
            c.codes[table[b, n // page], :, n % page:] &= 0xfe
    lut = (rng.standard_normal((len(lengths), H * group, m, 256)) * 2).astype(np.float32)
    ref, bound = c.attend(lut, table, lengths, 0.1)
    lut[..., ::2] = value                                 # the tokens' codes are odd
    for kw in CUTS:
        out = lk.lookat_attend_pages(dev(lut), on_gpu(lk, c), dev(table), i32(*lengths), 0.1, **kw).cpu().numpy()
        assert np.all(np.abs(out - ref) <= bound), kw


@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("group,d_k,m", [(1, 64, 4), (2, 128, 8), (4, 64, 2), (8, 128, 8)])
@pytest.mark.parametrize("level", [-2.0e38, -2.1e38, -2.358e38, 2.358e38])
def test_attend_equal_scores_at_the_ends_of_fp32(lk, kind, group, d_k, m, level):  # noqa: F811
    """Scores that are the same to the last bit are equal weights, down to the lowest number: the mean of the values.  All exponents are
    equal, every weight is a power of two, the same for all tokens, and the sums are of whole numbers (int8) or of multiples of 2^-9 below
    448 * 2500: 24 bits hold int8's sums exactly and e4m3's to 2500 roundings of half a step.  The quotient, its product and the merge's weights:
    four roundings.  2^-20 (int8) or 2500 * 2^-24 of the mean size, doubled for the hardware's reciprocal and exponential."""
    c, table, lengths, lut = not_finite_case(kind, group, d_k, m)
    c.exponents[:] = -3
    lut[:] = 0
    lut[:, :, 1] = level
    for kw in CUTS:
        out = lk.lookat_attend_pages(dev(lut), on_gpu(lk, c), dev(table), i32(*lengths), 1.0, **kw).cpu().numpy()
        for b in range(2):
            _, v = c.tokens(table[b], lengths[b])
            ref = np.repeat(v.mean(1), group, 0)
            bound = np.repeat(np.abs(v).mean(1), group, 0) * (2 ** -19 if kind == "int8" else 2 * 2500 * 2.0 ** -24)
            assert np.all(np.abs(out[b] - ref) <= bound), (b, kw)


# ---- the books at their limits --------------------------------------------------------------------------------------
def test_lists_as_long_as_there_can_be_sequences(lk):  # noqa: F811
    """65535 sequences and lists of as many entries, every pair and slot named twice: the first one counts."""
    S, n, P = 65535, 32767, 40000
    pool = lk.page_pool(P, 1, 64, 2, 16)
    table = torch.full((S, 1), -1, dtype=torch.int32, device="cuda")
    lengths, refs = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.zeros(P, dtype=torch.int32, device="cuda")
    held = torch.arange(n, device="cuda")
    table[:n, 0], lengths[:n], refs[:n] = held.flip(0).int() + 100, (held % 16 + 1).int(), 0
    refs[100: 100 + n] = 1
    src = torch.cat([held, held.roll(1), held[:1]]).int()                 # the second half names other parents for the same children
    dst = torch.cat([held + n, held + n, held[:1] + n]).int()
    lk.lookat_pages_fork(pool, table, lengths, refs, src, dst)
    torch.cuda.synchronize()
    assert torch.equal(table[n: 2 * n], table[:n]) and torch.equal(lengths[n: 2 * n], lengths[:n])
    assert int(refs.sum()) == 2 * n and torch.all(refs[100: 100 + n] == 2) and int(lengths[-1]) == 0 and int(table[-1]) == -1
    slots = torch.cat([held.flip(0), held, held[:1]]).int()
    lk.lookat_pages_free(pool, table, lengths, refs, slots)
    torch.cuda.synchronize()
    assert torch.all(lengths[:n] == 0) and torch.all(table[:n] == -1) and torch.all(refs[100: 100 + n] == 1) and int(refs.sum()) == n
    assert torch.all(lengths[n: 2 * n] > 0)


@pytest.mark.parametrize("S", [1023, 1025, 5000, 65535])
def test_reserve_for_many_sequences(lk, S):  # noqa: F811
    """Needs that are summed up over several workgroups: pages in order over all sequences, shared last pages copied, rows that are too short and
    pages that are too few reported."""
    rng = np.random.default_rng(S)
    W, page, half = 3, 16, S // 2
    lengths = np.zeros(S, np.int32)
    lengths[:half] = rng.integers(0, 2 * page + 1, half)
    used = int((-(-lengths // page)).sum())
    P = used + 2 * S
    table = random_table(rng, lengths.tolist(), page, W, P)
    shared = rng.random(half) < 0.5                       # the second half begins as some of the first
    table[half: 2 * half][shared], lengths[half: 2 * half][shared] = table[:half][shared], lengths[:half][shared]
    refs = np.bincount(table[table >= 0], minlength=P).astype(np.int32)
    c = random_cache(rng, P, 1, 64, 2, page, "int8")
    b, pool = pr.Books(table, lengths, refs, page), on_gpu(lk, c)
    books = dev(table), dev(lengths), dev(refs)

    def reserve(wanted, label):
        copies = torch.full((2, S), -5, dtype=torch.int32, device="cuda")
        was = b.table.copy()
        missing = int(lk.lookat_pages_reserve(pool, *books, dev(wanted.astype(np.int32)), copies=copies))
        assert missing == b.reserve(wanted, c), label
        same_books(books, b)
        assert_pool(pool, c)
        moved = (was != b.table) & (was >= 0)
        s, w = np.nonzero(moved)
        pairs = np.full((2, S), -1)
        pairs[0, s], pairs[1, s] = was[s, w], b.table[s, w]
        assert np.array_equal(copies.cpu().numpy(), pairs), label
        return missing

    grow = lengths + rng.integers(-2, page + 2, S) * (rng.random(S) < 0.8)
    short = grow.copy()
    short[[0, S // 3, S - 1]] = [W * page + 1, 2 ** 31 - 1, W * page + page + 1]
    assert reserve(short, "short rows") > 2 ** 26
    assert reserve(grow, "a token too many in the fullest rows") == int((grow > W * page).sum())
    assert reserve(np.minimum(grow, W * page), "room") == 0
    # all but a few of the pages taken by others: nothing is changed
    need = int((-(-W * page // page) - -(-b.lengths // page)).sum())
    free = np.flatnonzero(b.refs == 0)
    b.refs[free[: len(free) - need + 5]] += 1
    books[2].copy_(dev(b.refs))
    assert reserve(np.full(S, W * page), "few pages") >= 5


def test_the_books_work_grows_with_the_number_of_sequences(lk):  # noqa: F811
    """Four times the sequences, all growing into a new page: four times the workgroups, each with the same work (if each looked at all of the
    sequences, sixteen times: it took twelve)."""
    best = []
    for S in (16384, 65535):
        pool = lk.page_pool(S, 1, 64, 2, 16)
        table, zeros = torch.full((S, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
        ones, missing = torch.ones_like(zeros), torch.empty(1, dtype=torch.int32, device="cuda")
        times = []
        for _ in range(8):
            lengths, refs = zeros.clone(), zeros.clone()
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            lk.lookat_pages_reserve(pool, table, lengths, refs, ones, missing)
            end.record()
            torch.cuda.synchronize()
            assert int(missing) == 0 and int(refs.sum()) == S and torch.equal(table[:, 0], torch.arange(S, device="cuda", dtype=torch.int32))
            times.append(begin.elapsed_time(end))
        best.append(min(times))
    assert best[1] < 7 * best[0], best


# ---- pools without anything in them -----------------------------------------------------------------------------------
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("pages,H,d_k,m,page", [(0, 2, 64, 4, 16), (10, 0, 64, 4, 16), (10, 2, 0, 4, 16), (10, 2, 64, 0, 16), (10, 2, 64, 4, 0)])
def test_empty_pools_are_refused(lk, monkeypatch, native, pages, H, d_k, m, page):  # noqa: F811
    from paper_2601_10155_amd import binding
    if not native:
        monkeypatch.setattr(binding, "_marshal", Watch(None))
    pool = lk.page_pool(pages, H, d_k, m, page)
    table, n, refs = torch.full((3, 4), -1, dtype=torch.int32, device="cuda"), i32(0, 0, 0), torch.zeros(pages, dtype=torch.int32, device="cuda")
    lut = torch.zeros((3, 2, m, 256), device="cuda")
    codes, values = torch.zeros((3, H, 1, m), dtype=torch.uint8, device="cuda"), torch.zeros((3, H, 1, d_k), device="cuda")
    for call in (lambda: lk.lookat_attend_pages(lut, pool, table, n, 1.0), lambda: lk.lookat_attend_pages(lut[:, :H].contiguous(), pool, table, n, 1.0),
                 lambda: lk.lookat_pages_write(pool, codes, values, table, n), lambda: lk.lookat_pages_copy(pool, n, n),
                 lambda: lk.lookat_pages_fork(pool, table, n, refs, n, n), lambda: lk.lookat_pages_free(pool, table, n, refs, n),
                 lambda: lk.lookat_pages_reserve(pool, table, n, refs, i32(1, 1, 1)), lambda: lk.lookat_pages_compact(pool, table, n, refs)):
        with pytest.raises((ValueError, lk.LookatError)):
            call()
    torch.cuda.synchronize()
    assert torch.all(table == -1) and torch.all(n == 0)


# ---- what a weight is worth -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("group,d_k,m", FORMS)
def test_attend_weights_have_two_terms(lk, group, d_k, m, kind):  # noqa: F811
    c, table, lut = weights_case(group, d_k, m, kind)
    ref, bound = weights_reference(c, table, lut)
    for kw in ({}, {"max_length": 5000, "W": 100}, {"num_splits": 2}):
        wide = np.full((len(LENGTHS), kw.pop("W", 1)), -1, np.int32)
        wide[:, :1] = table
        out = lk.lookat_attend_pages(dev(lut), on_gpu(lk, c), dev(wide), i32(*LENGTHS), 1.0, **kw).cpu().numpy()
        off = np.abs(out - ref)
        record("attend_pages, weights (of the close bound)", float(np.max(off / np.maximum(bound, 1e-30))))
        assert np.all(off <= bound), f"{np.max(off / np.maximum(bound, 1e-30))} times the bound"


# ---- the timed cases' search step, over several passes ------------------------------------------------------------------
@pytest.mark.parametrize("case", [
    {"S": 16, "fan": 4, "L": 1000, "ragged": 0.2, "H": 3, "d_k": 64, "m": 4, "page": 16, "type": "int8"},
    {"S": 75, "fan": 2, "L": 333, "ragged": 0.9, "H": 2, "d_k": 128, "m": 8, "page": 64, "type": "float8"},
    {"S": 9, "fan": 1, "L": 32, "ragged": 0.0, "H": 1, "d_k": 64, "m": 2, "page": 32, "type": "int8"}])
def test_search_steps_that_give_up_real_children(lk, case):  # noqa: F811
    """perf/operators.py's search step three times over: from the second pass on the children that are given up hold pages.  Its plain form
    beside it, books and pools equal after each."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("operators_of_the_paged_cache", path)
    operators = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(operators)
    case = {"kind": "turn", "spare": 1.5, **case}
    here, plain = operators.prepare(case, 1), operators.prepare(case, 1)
    for n in range(3):
        held = here["lengths"][case["S"]:] > 0
        assert torch.all(held) if n else not torch.any(held)
        results = []
        for operators.own, state in ((True, here), (False, plain)):
            out = operators.run(state)
            results.append([out["table"], out["lengths"], out["refs"], out["missing"], *(out["pool"][k].view(torch.uint8) for k in ("codes", "values", "exponents"))])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(*results)), f"pass {n}"
        assert int(results[0][3]) == 0
        # other parents: a child may take over a longer or a shorter beginning than the one it had
        for state in (here, plain):
            state["parents"] = state["parents"].roll(1).contiguous()
            state["wanted"][case["S"]:] = state["lengths"][state["parents"].long()] + 1
