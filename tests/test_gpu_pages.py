"""The paged 8-bit cache on the GPU against tests/pages_ref.py: stored bytes, exponents, codes and books bit for bit (whole pools, so that
what a call must leave alone is checked too), attention at a bound derived in pages_ref.Cache.attend."""
import math

import numpy as np
import pytest
import torch

import pages_ref as pr
from bars import record

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lk():
    import paper_2601_10155_amd as pkg
    pkg.load_library()
    return pkg


TORCH = {"int8": torch.int8, "float8": torch.float8_e4m3fn}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def random_cache(rng, P, H, d_k, m, page, kind, low=-7, high=-3):
    """Pages full of numbers of the type, none of them NaN."""
    v = rng.standard_normal((P, H, page // 8, d_k, 8)) * (30 if kind == "int8" else 100)
    return pr.Cache(rng.integers(0, 256, (P, H, page, m), dtype=np.uint8), pr.to_bytes(v, kind), rng.integers(low, high, (P, H)).astype(np.int8), kind)


def on_gpu(lk, c):
    return lk.PagePool(dev(c.codes), dev(c.values).view(TORCH[c.kind]), dev(c.exponents))


def assert_pool(pool, c):
    torch.cuda.synchronize()
    assert np.array_equal(pool.exponents.cpu().numpy(), c.exponents), "exponents"
    assert np.array_equal(pool.codes.cpu().numpy(), c.codes), "codes"
    got = pool.values.view(torch.uint8).cpu().numpy()
    assert np.array_equal(got, c.values), f"values: {np.argwhere(got != c.values)[:5].tolist()}"


def random_table(rng, lengths, page, W, P):
    """Rows of pages of their own, in no order; -1 behind them."""
    ids = rng.permutation(P)
    table = np.full((len(lengths), W), -1, np.int32)
    at = 0
    for s, n in enumerate(lengths):
        k = -(-n // page)
        table[s, :k] = ids[at: at + k]
        at += k
    return table


# ---- writing -----------------------------------------------------------------------------------------------------
SHAPES = [(64, 4, 16), (64, 2, 64), (128, 8, 32), (128, 16, 128), (64, 16, 128), (128, 4, 64)]


@pytest.mark.parametrize("dtype", ["float16", "float32"])
@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("d_k,m,page", SHAPES)
def test_write(lk, d_k, m, page, kind, dtype):
    rng = np.random.default_rng(d_k + m + page)
    # lengths after the write and rows given: from the start, inside a page, over several, one token, none, more rows than tokens
    N = 2 * page + 5
    lengths = [N, page + 3, 3 * page, 1, 0, 2 * page + 1, page, 7, 4 * page]
    counts = [N, 3, 2 * page + 5, 1, 4, 1, 0, 12, page]
    B, H = len(lengths), 3
    W, P = 4, 40
    c = random_cache(rng, P, H, d_k, m, page, kind)
    table = random_table(rng, lengths, page, W, P)
    codes = rng.integers(0, 256, (B, H, N, m), dtype=np.uint8)
    size = np.exp(rng.standard_normal((B, H, N, 1)))
    values = (rng.standard_normal((B, H, N, d_k)) * size).astype(dtype)
    pool = on_gpu(lk, c)
    lk.lookat_pages_write(pool, dev(codes), dev(values), dev(table), i32(*lengths), i32(*counts))
    c.write(codes, values, table, lengths, counts)
    assert_pool(pool, c)
    # once more: the same bytes
    lk.lookat_pages_write(pool, dev(codes), dev(values), dev(table), i32(*lengths), i32(*counts))
    assert_pool(pool, c)


@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_write_token_by_token(lk, kind):
    """A decode loop's appends: the exponent of a page grows with its tokens, those it holds follow; head sizes and pages of all kinds."""
    for d_k, m, page, seed in ((64, 4, 16, 0), (128, 8, 64, 1)):
        rng = np.random.default_rng(seed)
        B, H, steps = 3, 5, 2 * page + 3
        c = random_cache(rng, 12, H, d_k, m, page, kind)
        table = np.array([[3, 7, 1], [0, 2, 9], [11, 4, 5]], np.int32)
        pool = on_gpu(lk, c)
        start = [0, 5, page - 1]
        for n in range(steps):
            lengths = [min(s + n + 1, 3 * page) for s in start]
            codes = rng.integers(0, 256, (B, H, 1, m), dtype=np.uint8)
            values = (rng.standard_normal((B, H, 1, d_k)) * 1.4 ** (n % 25) * 10.0 ** -(n % 7)).astype(np.float16)
            lk.lookat_pages_write(pool, dev(codes), dev(values), dev(table), i32(*lengths))
            c.write(codes, values, table, lengths)
        assert_pool(pool, c)


@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_write_extremes(lk, kind):
    """Zeros, subnormals, the largest fp32, infinities, NaN, exact borders of an exponent, ties."""
    rng = np.random.default_rng(3)
    d_k, m, page, H = 64, 2, 16, 2
    q = pr.most(kind)
    rows = [np.zeros(d_k), np.full(d_k, 1e-42), np.full(d_k, 3e38), np.full(d_k, math.inf), np.full(d_k, math.nan), np.full(d_k, q * 2.0 ** -3),
            np.full(d_k, np.nextafter(np.float32(q * 2.0 ** -3), np.float32(9e9))), np.full(d_k, -q), np.arange(d_k) + 0.5, -(np.arange(d_k) + 0.5),
            np.concatenate([[q], rng.standard_normal(d_k - 1) * q / 3]), np.concatenate([[math.nan, -math.inf], np.arange(d_k - 2)]),
            np.full(d_k, 2.0 ** -41), np.full(d_k, 2.0 ** 60)]
    B = len(rows)
    values = np.repeat(np.stack(rows).astype(np.float32)[:, None, None], H, 1)
    codes = np.zeros((B, H, 1, m), np.uint8)
    for before in (0, 4):                                # alone in the page, and behind four tokens
        c = random_cache(rng, B, H, d_k, m, page, kind)
        c.exponents[:] = -2
        pool = on_gpu(lk, c)
        table = np.arange(B, dtype=np.int32)[:, None]
        lengths = [before + 1] * B
        lk.lookat_pages_write(pool, dev(codes), dev(values), dev(table), i32(*lengths))
        c.write(codes, values, table, lengths)
        assert_pool(pool, c)


def test_write_views_short_rows_and_bad_pages(lk):
    rng = np.random.default_rng(4)
    d_k, m, page, H, N = 64, 4, 16, 2, 40
    lengths = [40, 40, 33, 100]                          # the last one is longer than its row
    counts = [40, 20, 33, 40]
    B, W, P = 4, 3, 16
    c = random_cache(rng, P, H, d_k, m, page, "int8")
    wide = np.full((B, 7), 5, np.int32)                  # (page 5 stands behind the rows: nothing may reach it)
    wide[:, 2: 2 + W] = [[0, -1, 1], [2, 3, P], [4, -2147483648, 2147483647], [6, 7, 8]]
    wide = dev(wide)
    table = wide[:, 2: 2 + W]
    codes = dev(rng.integers(0, 256, (B, H, N + 11, m), dtype=np.uint8))[:, :, 3: 3 + N]
    values = dev(rng.standard_normal((B, H, N + 9, d_k)).astype(np.float16))[:, :, 6: 6 + N]
    pool = on_gpu(lk, c)
    lk.lookat_pages_write(pool, codes, values, table, i32(*lengths), i32(*counts))
    c.write(codes.cpu().numpy(), values.cpu().numpy(), table.cpu().numpy(), lengths, counts)
    assert_pool(pool, c)
    # nothing to write
    lk.lookat_pages_write(pool, codes[:, :, :0], values[:, :, :0], table, i32(*lengths))
    lk.lookat_pages_write(pool, codes, values, table, i32(0, -5, 0, -2147483648), i32(3, 3, 2147483647, 9))
    lk.lookat_pages_write(pool, codes, values, table, i32(*lengths), i32(0, -1, 0, -2147483648))
    assert_pool(pool, c)


# ---- attention ------------------------------------------------------------------------------------------------------
def attend_case(lk, rng, c, lengths, group, sharp=1.0, W=None, **kw):
    """(device out, reference out, bound); the table has spare entries with ids outside the pool behind each row."""
    page = c.page
    W = W or max(1, -(-max(lengths) // page)) + 1
    table = random_table(rng, lengths, page, W, c.P)
    table[table < 0] = rng.integers(c.P, 2 ** 31, int((table < 0).sum()))
    lut = (rng.standard_normal((len(lengths), c.H * group, c.m, 256)) * sharp).astype(np.float32)
    scale = 1.0 / math.sqrt(c.d_k)
    pool = on_gpu(lk, c)
    out = torch.full((len(lengths), c.H * group, c.d_k), math.nan, device="cuda")
    lk.lookat_attend_pages(dev(lut), pool, dev(table), i32(*lengths), scale, out=out, **kw)
    torch.cuda.synchronize()
    assert_pool(pool, c)
    return out.cpu().numpy(), *c.attend(lut, table, lengths, scale)


def assert_attend(got, label):
    out, ref, bound = got
    assert np.isfinite(out).all()
    assert np.all(out[np.all(ref == 0, -1)] == 0)
    err = np.abs(out - ref)
    record(f"attend_pages, {label} (of the derived bound)", float(np.max(err / np.maximum(bound, 1e-30))))
    assert np.all(err <= bound), f"{label}: {np.max(err / np.maximum(bound, 1e-30))} times the bound"


LENGTHS = [1, 0, 63, 64, 65, 17, 300, 128, 257, 511, 16, 1000]


@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("d_k,m,page", [(64, 2, 16), (64, 4, 64), (64, 8, 32), (64, 16, 128), (128, 2, 128), (128, 4, 16), (128, 8, 64), (128, 16, 32)])
def test_attend(lk, d_k, m, page, group, kind):
    rng = np.random.default_rng(d_k * m + page + group)
    H = 2
    c = random_cache(rng, sum(-(-n // page) for n in LENGTHS) + 2, H, d_k, m, page, kind)
    for splits in (0, 1, 3):
        assert_attend(attend_case(lk, rng, c, LENGTHS, group, 3.0, num_splits=splits), f"group {group}, {kind}")


@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("d_k,m,page", [(64, 2, 16), (64, 16, 64), (128, 4, 128), (128, 16, 32)])
def test_attend_short(lk, d_k, m, page, group, kind):
    """Rows of four tiles at most (workgroups of four wavefronts), and a host that takes longer ones for such."""
    rng = np.random.default_rng(d_k + m + page + group)
    lengths = [1, 0, 64, 65, 128, 127, 3, 100]
    c = random_cache(rng, 64, 3, d_k, m, page, kind)
    for kw in ({"W": 128 // page}, {"W": 128 // page, "num_splits": 1}, {"W": 128 // page, "num_splits": 2}):
        assert_attend(attend_case(lk, rng, c, lengths, group, 3.0, **kw), f"short rows, {kind}")
    assert_attend(attend_case(lk, rng, c, [256, 255, 193, 1], group, 3.0, W=256 // page), f"short rows, {kind}")
    assert_attend(attend_case(lk, rng, c, [333, 5, 190], group, 3.0, max_length=256), f"short rows, {kind}")


@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_attend_long(lk, kind):
    """Long rows in many ranges, short ones beside them, a table wider than any sequence and a host that knows less than is there."""
    rng = np.random.default_rng(11)
    c = random_cache(rng, 700, 1, 128, 8, 16, kind)
    lengths = [5003, 3, 0, 2048, 2049]
    for kw in ({}, {"num_splits": 16}, {"num_splits": 700}, {"max_length": 100}, {"max_length": 1}, {"max_length": 100, "num_splits": 4},
               {"max_length": 1 << 40, "W": 5000}):
        assert_attend(attend_case(lk, rng, c, lengths, 4, **kw), f"long rows, {kind}")
    lengths = [20001]
    c = random_cache(rng, 320, 2, 64, 4, 64, kind)
    for splits in (0, 1, 13):
        assert_attend(attend_case(lk, rng, c, lengths, 1, 0.2, num_splits=splits), f"one long row, {kind}")


@pytest.mark.parametrize("B", [63, 64, 65, 300, 1024, 1025, 1500])
def test_attend_many_sequences(lk, B):
    """Ranges by length over few and many sequences (a lane, a thread or several sequences a thread look at them), and equal ranges beyond."""
    rng = np.random.default_rng(B)
    lengths = (np.exp(rng.uniform(0, np.log(5000 if B < 200 else 300), B))).astype(int)
    lengths[rng.integers(0, B, B // 5)] = 0
    lengths[[0, B // 2, B - 1]] = [4500, 2049, 6001]      # cut into ranges, whatever the others are
    lengths = lengths.tolist()
    c = random_cache(rng, sum(-(-n // 128) for n in lengths), 1, 64, 2, 128, "int8")
    assert_attend(attend_case(lk, rng, c, lengths, 1), "many sequences")


@pytest.mark.parametrize("H,group,d_k,m,lengths", [
    (128, 8, 64, 4, [3500, 2500]),                        # 4 ranges a head wanted, 5 at first: longer ones, 4
    (128, 8, 64, 4, [3500, 2500, 0, 1, 700]),             # 8 at first: left so
    (520, 8, 64, 4, [2100, 40]),                          # more heads than ranges wanted
    (32, 8, 128, 16, [8000, 5200, 5200]),                 # 128 KB of tables: 8 wanted, 10 at first, 7
    (7, 4, 128, 8, [30001, 2049, 15000])])
def test_attend_large_tables(lk, H, group, d_k, m, lengths):
    """Ranges that the chip holds at once: fewer and longer ones where the sequences' last ranges would make too many."""
    rng = np.random.default_rng(H + m)
    c = random_cache(rng, sum(-(-n // 128) for n in lengths) + 2, H, d_k, m, 128, "int8")
    assert_attend(attend_case(lk, rng, c, lengths, group), "large tables")


@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_attend_peaked_and_flat(lk, kind):
    """Logits from nothing to hundreds, rising and falling along the row (the reference has to follow)."""
    rng = np.random.default_rng(12)
    for sharp in (0.0, 1e-3, 40.0, 400.0):
        c = random_cache(rng, 30, 2, 64, 4, 64, kind)
        assert_attend(attend_case(lk, rng, c, [700, 900], 2, sharp), f"peaked, {kind}")
    # equal logits, low or high, up to the ends of fp32 (where no weights are left to tell apart, but numbers)
    c = random_cache(rng, 40, 1, 64, 4, 16, kind)
    table = np.arange(40, dtype=np.int32)[None]
    for level in (-1e3, 1e3, -1e31, 1e31, -3e37, 3e37):
        lut = np.full((1, 1, 4, 256), level, np.float32)
        for splits in (1, 3):
            out = lk.lookat_attend_pages(dev(lut), on_gpu(lk, c), dev(table), i32(600), 0.125, num_splits=splits).cpu().numpy()
            if abs(level) < 1e4:
                assert_attend((out, *c.attend(lut, table, [600], 0.125)), f"equal logits, {kind}")
            assert np.isfinite(out).all() and np.abs(out).max() > 0
    # a table whose entries grow with the code, and codes that grow along the row
    c = random_cache(rng, 16, 1, 64, 2, 64, kind)
    table = np.arange(16, dtype=np.int32)[None]
    for codes in (np.arange(1024) // 4, 255 - np.arange(1024) // 4):
        c.codes[:] = codes.reshape(16, 1, 64, 1)
        lut = np.broadcast_to(np.arange(256, dtype=np.float32) * 3, (1, 1, 2, 256)).copy()
        out = lk.lookat_attend_pages(dev(lut), on_gpu(lk, c), dev(table), i32(1000), 0.125)
        assert_attend((out.cpu().numpy(), *c.attend(lut, table, [1000], 0.125)), f"a slope, {kind}")


@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_attend_exponents_far_apart(lk, kind):
    """Pages of all-zero values (lowest exponent), of tiny and of huge ones in one sequence, whichever of them has the weight."""
    rng = np.random.default_rng(13)
    for _ in range(6):
        c = random_cache(rng, 20, 2, 64, 4, 16, kind)
        c.exponents[:] = rng.choice([-40, -30, -20, -5, 0, 12, 25, 40], c.exponents.shape)
        zero = c.exponents == -40
        c.values[zero] = 0
        assert_attend(attend_case(lk, rng, c, [300], 2, rng.choice([1.0, 20.0, 100.0])), f"exponents far apart, {kind}")
    c = random_cache(rng, 20, 2, 64, 4, 16, kind)
    c.exponents[:] = -40
    c.values[:] = 0
    out, ref, _ = attend_case(lk, rng, c, [300, 5], 2)
    assert np.all(out == 0)


@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_attend_what_is_not_there_does_not_matter(lk, kind):
    """Behind a sequence's last token, and in pages outside the pool: NaN bytes, wild exponents, any code; and no page at all."""
    rng = np.random.default_rng(14)
    d_k, m, page, H, group = 128, 8, 32, 2, 2
    lengths = [1, 31, 33, 70, 64, 100, 96, 50]
    c = random_cache(rng, 40, H, d_k, m, page, kind)
    W = 4
    table = random_table(rng, lengths, page, W, 40)
    for b, n in enumerate(lengths):
        if n % page:
            last = table[b, n // page]
            for t in range(n % page, page):
                c.values[last, :, t // 8, :, t % 8] = rng.choice([0x7f, 0xff, 0x80, 0x7e], (H, d_k))
    used = table[table >= 0]
    for i in set(range(40)) - set(used.tolist()):
        c.values[i], c.exponents[i] = 0x7f, 127
    table[table < 0] = 39 if 39 not in used else -1
    table[5, 1], table[6, 0], table[7] = -1, 40, [2 ** 31 - 1, -2 ** 31, 0, 0]     # a hole, a hole at the start, nothing at all
    lut = (rng.standard_normal((len(lengths), H * group, m, 256)) * 2).astype(np.float32)
    for splits in (1, 2, 4):
        out = lk.lookat_attend_pages(dev(lut), on_gpu(lk, c), dev(table), i32(*lengths), 0.1, num_splits=splits).cpu().numpy()
        assert np.all(out[7] == 0)
        assert_attend((out, *c.attend(lut, table, lengths, 0.1)), f"what is not there, {kind}")
    # longer than the row: the row's tokens; negative: none
    out = lk.lookat_attend_pages(dev(lut), on_gpu(lk, c), dev(table), i32(*[-3, 2 ** 31 - 1, 33, 70, 64, 100, 96, 0]), 0.1)
    assert torch.all(out[0] == 0) and torch.all(out[7] == 0)
    wild = np.where(np.isnan(pr.from_bytes(c.values, kind)), 0, c.values).astype(np.uint8)
    c.values[:] = wild
    out = lk.lookat_attend_pages(dev(lut), on_gpu(lk, c), dev(table), i32(*[-3, 2 ** 31 - 1, 33, 70, 64, 100, 96, 0]), 0.1).cpu().numpy()
    assert np.isfinite(out[2:]).all()


def test_attend_views_streams_and_a_given_workspace(lk):
    rng = np.random.default_rng(15)
    c = random_cache(rng, 60, 3, 64, 4, 16, "int8")
    lengths = [100, 333, 257]
    table = np.full((3, 40), -7, np.int32)
    table[:, 5:26] = random_table(rng, lengths, 16, 21, 60)
    table, pool = dev(table)[:, 5:26], on_gpu(lk, c)
    lut = (rng.standard_normal((3, 3, 4, 256)) * 2).astype(np.float32)
    lut_d, n = dev(lut), i32(*lengths)
    first = lk.lookat_attend_pages(lut_d, pool, table, n, 0.125, num_splits=3)
    assert_attend((first.cpu().numpy(), *c.attend(lut, table.cpu().numpy(), lengths, 0.125)), "views")
    ws = torch.full((lk.attend_pages_workspace_bytes(pool, 3, 1, 21, 0, 3),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(first, lk.lookat_attend_pages(lut_d, pool, table, n, 0.125, num_splits=3, workspace=ws))
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for s in side:                                       # two calls in flight, each with a workspace of its own
        with torch.cuda.stream(s):
            outs.append(lk.lookat_attend_pages(lut_d, pool, table, n, 0.125, num_splits=3))
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)
    with pytest.raises(lk.LookatError):
        lk.lookat_attend_pages(lut_d[:, :3].repeat(1, 3, 1, 1), pool, table, n, 0.125)      # three query heads on each


# ---- upkeep -----------------------------------------------------------------------------------------------------
def same_books(got, b):
    torch.cuda.synchronize()
    table, lengths, refs = (x.cpu().numpy() for x in got)
    assert np.array_equal(lengths, b.lengths) and np.array_equal(refs, b.refs) and np.array_equal(table, b.table)


def test_copy(lk):
    rng = np.random.default_rng(20)
    for H, d_k, m, page, P, n in ((1, 64, 2, 16, 9, 3), (12, 64, 4, 16, 64, 30), (8, 128, 8, 64, 40, 20), (3, 128, 16, 128, 12, 6)):
        c = random_cache(rng, P, H, d_k, m, page, "int8")
        pool = on_gpu(lk, c)
        ids = rng.permutation(P).astype(np.int32)
        src, dst = ids[:n].copy(), ids[n: 2 * n].copy()
        src[0] = src[-1]                                 # a source may be named twice
        lk.lookat_pages_copy(pool, dev(src), dev(dst))
        for x in (c.codes, c.values, c.exponents):
            x[dst] = x[src]
        assert_pool(pool, c)
        # pairs that are passed over, and none
        lk.lookat_pages_copy(pool, i32(0, -1, P, 2 ** 31 - 1, -2 ** 31), i32(0, 1, 1, 1, 1))
        lk.lookat_pages_copy(pool, i32(0, 0, 0), i32(-1, P, 2 ** 31 - 1))
        lk.lookat_pages_copy(pool, i32(), i32())
        assert_pool(pool, c)


def books_of(rng, S, W, P, page, fill=0.5):
    lengths = np.array([int(rng.integers(0, int(W * page * fill) + 1)) for _ in range(S)], np.int32)
    lengths[rng.random(S) < 0.3] = 0
    table = random_table(rng, lengths, page, W, P)
    refs = np.zeros(P, np.int32)
    refs[table[table >= 0]] = 1
    return pr.Books(table, lengths, refs, page)


@pytest.mark.parametrize("S,W,P,page", [(1, 1, 1, 16), (7, 5, 40, 16), (40, 12, 700, 32), (300, 9, 5000, 64), (1500, 3, 3000, 128)])
def test_books(lk, S, W, P, page):
    """Random turns of freeing, forking, reserving and compacting, the books equal after each, the pages' contents too."""
    rng = np.random.default_rng(S + P)
    H, d_k, m = 1, 64, 2
    c = random_cache(rng, P, H, d_k, m, page, "int8")
    b = books_of(rng, S, W, P, page)
    pool = on_gpu(lk, c)
    wide = torch.full((S, W + 3), -9, dtype=torch.int32, device="cuda")
    wide[:, 1: 1 + W] = dev(b.table)
    table, lengths, refs = wide[:, 1: 1 + W], dev(b.lengths), dev(b.refs)
    other = on_gpu(lk, c)
    for turn in range(8):
        n = int(rng.integers(1, S + 1))
        slots = rng.integers(-1, S + 1, n).astype(np.int32)               # repeated ones and ones that do not exist among them
        lk.lookat_pages_free(pool, table, lengths, refs, dev(slots))
        b.free(slots.tolist())
        same_books((table, lengths, refs), b)
        src, dst = rng.integers(-1, S + 1, n).astype(np.int32), rng.integers(-1, S + 1, n).astype(np.int32)
        lk.lookat_pages_fork(pool, table, lengths, refs, dev(src), dev(dst))
        b.fork(src.tolist(), dst.tolist())
        same_books((table, lengths, refs), b)
        more = rng.integers(-3, page + 2, S) if turn % 3 else rng.integers(0, W * page, S) * (rng.random(S) < 0.2)
        wanted = np.minimum(b.lengths + more, W * page + (turn == 5)).astype(np.int32)
        copies = torch.full((2, S), -5, dtype=torch.int32, device="cuda")
        missing = lk.lookat_pages_reserve(pool, table, lengths, refs, dev(wanted), copies=copies)
        lk.lookat_pages_copy(other, *copies)                              # a second layer's pool with the same books
        before = b.table.copy()
        expected = b.reserve(wanted, c)
        moved = [(s, before[s, w], b.table[s, w]) for s, w in np.argwhere((before != b.table) & (before >= 0)).tolist() if b.lengths[s] > 0]
        pairs = np.full((2, S), -1)
        for s, old, new in moved:
            pairs[:, s] = old, new
        assert np.array_equal(copies.cpu().numpy(), pairs)
        assert int(missing) == expected
        same_books((table, lengths, refs), b)
        assert_pool(pool, c)
        if turn % 2:
            new_table, new_refs, live = lk.lookat_pages_compact(pool, table, lengths, refs)
            t, r, n = b.compact(c)
            same_books((table, lengths, refs), b)                         # the old ones stay
            assert int(live) == n and np.array_equal(new_refs.cpu().numpy(), r) and np.array_equal(new_table.cpu().numpy(), t)
            assert_pool(pool, c)
            again = lk.lookat_pages_compact(other, table, lengths, refs)
            assert all(torch.equal(x, y) for x, y in zip(again, (new_table, new_refs, live)))
            assert_pool(other, c)
            b.table, b.refs = t, r
            table.copy_(new_table), refs.copy_(new_refs)
    assert torch.all(wide[:, 0] == -9) and torch.all(wide[:, 1 + W:] == -9)


def test_reserve_changes_nothing_when_pages_or_room_are_missing(lk):
    rng = np.random.default_rng(22)
    c = random_cache(rng, 10, 2, 64, 4, 16, "float8")
    pool = on_gpu(lk, c)
    b = pr.Books(np.array([[3, 4, -1], [3, 4, -1], [5, -1, -1]], np.int32), np.array([20, 20, 16], np.int32),
                 np.array([0, 0, 0, 2, 2, 1, 0, 1, 1, 1], np.int32), 16)
    table, lengths, refs = dev(b.table), dev(b.lengths), dev(b.refs)
    for wanted in ([48, 48, 48], [21, 21, 49], [2 ** 31 - 1, 0, 0], [2 ** 31 - 1] * 3, [33, 33, 17]):
        missing = int(lk.lookat_pages_reserve(pool, table, lengths, refs, i32(*wanted)))
        assert missing == b.reserve(wanted, c) > 0
        same_books((table, lengths, refs), b)
        assert_pool(pool, c)
    # exactly enough: two copies of the shared last page and two new ones
    assert int(lk.lookat_pages_reserve(pool, table, lengths, refs, i32(33, 21, 17))) == b.reserve([33, 21, 17], c) == 0
    same_books((table, lengths, refs), b)
    assert_pool(pool, c)
    assert refs[4].item() == 0 and refs[3].item() == 2


def test_compact_large_pools(lk):
    """Counts over many segments of the ranking, full, empty and single pools."""
    rng = np.random.default_rng(23)
    for P, live in ((1, 0), (1, 1), (1024, 1024), (1025, 1), (70001, 35000), (200000, 199999)):
        refs = np.zeros(P, np.int32)
        refs[rng.permutation(P)[:live]] = rng.integers(1, 5, live)
        codes, values = torch.zeros((P, 1, 16, 2), dtype=torch.uint8, device="cuda"), torch.zeros((P, 1, 2, 64, 8), dtype=torch.int8, device="cuda")
        mark = torch.arange(P, device="cuda")
        for k in range(3):
            codes[:, 0, k, 0] = (mark >> (8 * k)).to(torch.uint8)
            values.view(torch.uint8)[:, 0, 1, 63, k] = (mark >> (8 * k)).to(torch.uint8)
        pool = lk.PagePool(codes, values, (mark % 100).to(torch.int8).view(P, 1).contiguous())
        used = np.flatnonzero(refs)[: 4 * 300]
        table = np.full((4, 300), -1, np.int32)
        lengths = np.zeros(4, np.int32)
        for s in range(4):
            mine = used[s::4]
            table[s, : len(mine)] = mine
            lengths[s] = len(mine) * 16
        new_table, new_refs, n = lk.lookat_pages_compact(pool, dev(table), dev(lengths), dev(refs))
        b = pr.Books(table, lengths, refs, 16)
        t, r, count = b.compact()
        assert int(n) == count == live
        assert np.array_equal(new_refs.cpu().numpy(), r) and np.array_equal(new_table.cpu().numpy(), t)
        # the page that lies at each place now
        expected = np.arange(P)
        holes, movers = np.flatnonzero(refs[:live] == 0), live + np.flatnonzero(refs[live:])
        expected[holes] = movers
        got = sum(codes[:, 0, k, 0].long() << (8 * k) for k in range(3)).cpu().numpy()
        also = sum(values.view(torch.uint8)[:, 0, 1, 63, k].long() << (8 * k) for k in range(3)).cpu().numpy()
        assert np.array_equal(got, expected) and np.array_equal(also, expected)
        assert np.array_equal(pool.exponents.cpu().numpy()[:, 0], expected % 100)


# ---- sizes that pass 32 bits ----------------------------------------------------------------------------------------
def test_pools_beyond_four_gib(lk):
    """Pages whose values lie 2^32 bytes and more behind the pool's start: written, attended to, copied, reserved and compacted."""
    rng = np.random.default_rng(50)
    P, H, d_k, m, page = 40000, 8, 128, 16, 128                          # 131 KB of values a page: 5.2 GB
    pool = lk.PagePool(torch.empty((P, H, page, m), dtype=torch.uint8, device="cuda"),
                       torch.empty((P, H, page // 8, d_k, 8), dtype=torch.int8, device="cuda"), torch.empty((P, H), dtype=torch.int8, device="cuda"))
    ids = np.array([P - 1, 0, 33001, 17, 32768, 39000, 5, 36000])        # (2^32 bytes are 32768 pages)
    c = random_cache(rng, len(ids), H, d_k, m, page, "int8")
    at = torch.from_numpy(ids).cuda()
    for x, y in zip(pool, (c.codes, c.values.view(np.int8), c.exponents)):
        x[at] = dev(y)

    def assert_pages():
        torch.cuda.synchronize()
        for x, y in zip(pool, (c.codes, c.values.view(np.int8), c.exponents)):
            assert np.array_equal(x[at].cpu().numpy(), y)

    small = np.array([[0, 1, 2], [4, 3, 5]], np.int32)                    # the reference's page numbers
    table, lengths, counts = dev(ids[small].astype(np.int32)), [300, 290], [200, 33]
    codes = rng.integers(0, 256, (2, H, 200, m), dtype=np.uint8)
    values = rng.standard_normal((2, H, 200, d_k)).astype(np.float16)
    lk.lookat_pages_write(pool, dev(codes), dev(values), table, i32(*lengths), i32(*counts))
    c.write(codes, values, small, lengths, counts)
    lk.lookat_pages_write(pool, dev(codes[:, :, :1]), dev(values[:, :, :1]), table, i32(301, 291))
    c.write(codes[:, :, :1], values[:, :, :1], small, [301, 291])
    assert_pages()
    lut = (rng.standard_normal((2, H * 2, m, 256)) * 2).astype(np.float32)
    for splits in (0, 1, 2):
        out = lk.lookat_attend_pages(dev(lut), pool, table, i32(301, 291), 0.1, num_splits=splits)
        assert_attend((out.cpu().numpy(), *c.attend(lut, small, [301, 291], 0.1)), "a large pool")
    lk.lookat_pages_copy(pool, i32(P - 1, 5), i32(36000, 39000))
    for x in (c.codes, c.values, c.exponents):
        x[[7, 5]] = x[[0, 6]]
    assert_pages()
    # both sequences forked and grown by one token: the shared last pages (33001, 39000) go to the two lowest free ones
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    refs[:32000] = 1
    refs[table.long()] = 1
    books = torch.cat([table, torch.full_like(table, -1)])
    n = i32(301, 291, 0, 0)
    lk.lookat_pages_fork(pool, books, n, refs, i32(0, 1), i32(2, 3))
    assert int(lk.lookat_pages_reserve(pool, books, n, refs, i32(0, 0, 302, 292))) == 0
    assert books[2:, 2].tolist() == [32000, 32001] and refs[[33001, 39000]].tolist() == [1, 1]
    for x in pool:
        assert torch.equal(x[books[2:, 2].long()], x[books[:2, 2].long()])
    # 32007 pages in use: those above move down
    before = [x[books.clamp(min=0).long()].clone() for x in pool]
    moved, _, live = lk.lookat_pages_compact(pool, books, n, refs)
    assert int(live) == 32006 and int(moved.max()) < 32006
    for x, y in zip(pool, before):
        assert torch.equal(x[moved.long()], y)


# ---- together -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_a_search_over_continuations(lk, kind):
    """As a program uses the set: prompts are reserved, encoded and written, continuations forked, tokens reserved, written and attended to, some
    continuations given up, the pool compacted; every step's output against the reference cache, and the compaction does not
    change an output by a bit."""
    rng = np.random.default_rng(30)
    H, group, d_k, m, page, S, W, P = 2, 2, 64, 4, 16, 8, 10, 64
    c = random_cache(rng, P, H, d_k, m, page, kind)
    pool = on_gpu(lk, c)
    b = pr.Books(np.full((S, W), -1, np.int32), np.zeros(S, np.int32), np.zeros(P, np.int32), page)
    table, lengths, refs = dev(b.table), dev(b.lengths), dev(b.refs)
    books = dev((rng.standard_normal((H, m, 256, d_k // m)) * 2).astype(np.float32))
    scale = 1 / math.sqrt(d_k)

    def grow(counts):
        """Reserve, encode, write counts[s] tokens of every sequence; then one query each."""
        nonlocal table, refs
        counts = np.array(counts, np.int32)
        wanted = (b.lengths + counts).astype(np.int32)
        assert int(lk.lookat_pages_reserve(pool, table, lengths, refs, dev(wanted))) == b.reserve(wanted, c) == 0
        N = int(counts.max())
        keys = dev(rng.standard_normal((S, H, N, d_k)).astype(np.float32) * 2)
        values = rng.standard_normal((S, H, N, d_k)).astype(np.float16)
        codes = lk.lookat_encode_keys(keys, books)
        lk.lookat_pages_write(pool, codes, dev(values), table, lengths, dev(counts))
        c.write(codes.cpu().numpy(), values, b.table, b.lengths, counts)
        assert_pool(pool, c)
        same_books((table, lengths, refs), b)
        q = dev(rng.standard_normal((S, H, group, d_k)).astype(np.float16))
        lut = lk.lookat_build_lut(q, books).view(S, H * group, m, 256)
        out = lk.lookat_attend_pages(lut, pool, table, lengths, scale, max_length=int(b.lengths.max()))
        assert_attend((out.cpu().numpy(), *c.attend(lut.cpu().numpy(), b.table, b.lengths, scale)), f"a search, {kind}")
        return lut, out

    grow([37, 50, 0, 0, 0, 0, 0, 0])                      # two prompts
    for _ in range(3):
        parents = [0, 0, 1, 1, 0, 1]
        lk.lookat_pages_fork(pool, table, lengths, refs, i32(*parents), i32(2, 3, 4, 5, 6, 7))
        b.fork(parents, [2, 3, 4, 5, 6, 7])
        for step in range(page + 2):
            lut, out = grow([0, 0, 1, 1, 1, 1, step % 2, 1])
        new_table, new_refs, live = lk.lookat_pages_compact(pool, table, lengths, refs)
        b.table, b.refs, n = b.compact(c)
        assert int(live) == n
        table, refs = new_table, new_refs
        again = lk.lookat_attend_pages(lut, pool, table, lengths, scale, max_length=int(b.lengths.max()))
        assert torch.equal(out, again)
        lk.lookat_pages_free(pool, table, lengths, refs, i32(0, 1, 4, 5, 6, 7))
        b.free([0, 1, 4, 5, 6, 7])
        # the two that are left take the first places
        lk.lookat_pages_fork(pool, table, lengths, refs, i32(2, 3), i32(0, 1))
        b.fork([2, 3], [0, 1])
        lk.lookat_pages_free(pool, table, lengths, refs, i32(2, 3))
        b.free([2, 3])
        same_books((table, lengths, refs), b)


@pytest.mark.parametrize("group,d_k,m,splits", [(4, 128, 8, 2), (8, 128, 8, 0), (1, 64, 4, 0)])
def test_a_captured_decode_step(lk, group, d_k, m, splits):
    """Reserve, encode, write, tables, attention and compaction's ranking of books captured once, replayed for many tokens, each
    replay against the same calls made eagerly on a second cache; eager work between the replays."""
    rng = np.random.default_rng(31)
    B, H, page, W = 3, 2, 16, 6 if splits else 140          # (140 pages: 2240 tokens, cut by length)
    P = B * W
    books = dev((rng.standard_normal((H, m, 256, d_k // m)) * 2).astype(np.float32))
    scale = 1 / math.sqrt(d_k)
    one = i32(*[1] * B)

    class Side:
        def __init__(self):
            self.pool = lk.page_pool(P, H, d_k, m, page)
            self.table = torch.full((B, W), -1, dtype=torch.int32, device="cuda")
            self.lengths, self.refs = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(P, dtype=torch.int32, device="cuda")
            self.k, self.v = torch.zeros((B, H, 1, d_k), device="cuda"), torch.zeros((B, H, 1, d_k), device="cuda", dtype=torch.float16)
            self.q = torch.zeros((B, H, group, d_k), device="cuda", dtype=torch.float16)
            self.out = torch.zeros((B, H * group, d_k), device="cuda")

        def step(self):
            self.missing = lk.lookat_pages_reserve(self.pool, self.table, self.lengths, self.refs, self.lengths + one)
            codes = lk.lookat_encode_keys(self.k, books)
            lk.lookat_pages_write(self.pool, codes, self.v, self.table, self.lengths, one)
            lut = lk.lookat_build_lut(self.q, books).view(B, H * group, m, 256)
            lk.lookat_attend_pages(lut, self.pool, self.table, self.lengths, scale, num_splits=splits, out=self.out)
            self.compacted = lk.lookat_pages_compact(self.pool, self.table, self.lengths, self.refs)

        def state(self):
            return [self.pool.codes, self.pool.values, self.pool.exponents, self.table, self.lengths, self.refs, self.out, self.missing, *self.compacted]

    captured, eager = Side(), Side()
    # (a first eager step on a third cache, so that nothing is looked up for the first time under capture)
    warm = Side()
    warm.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    for n in range(40):
        for name, shape in (("k", (B, H, 1, d_k)), ("v", (B, H, 1, d_k)), ("q", (B, H, group, d_k))):
            x = dev(rng.standard_normal(shape).astype(np.float32))
            getattr(captured, name).copy_(x)
            getattr(eager, name).copy_(x)
        graph.replay()
        eager.step()
        warm.step()
        if n % 3 == 0:
            torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured.state(), eager.state())), f"replay {n}"
    assert int(captured.lengths[0]) == 40 and int(captured.missing) == 0


# ---- the binding -------------------------------------------------------------------------------------------------
class Watch:
    """Stands in for the native marshalling: passes calls on and notes which were taken, or takes none."""

    def __init__(self, native):
        self.native, self.taken = native, {}

    def __getattr__(self, name):
        def f(*a):
            rc = getattr(self.native, name)(*a) if self.native else None
            self.taken[name] = rc is not None
            return rc
        return f


def test_native_and_python_marshalling_agree(lk, monkeypatch):
    """A turn of every call through either: the same state, and the native one takes the calls that need no work."""
    from paper_2601_10155_amd import binding
    native = binding._marshal
    states = []
    for watch in (Watch(native), Watch(None)):
        monkeypatch.setattr(binding, "_marshal", watch)
        rng = np.random.default_rng(40)
        c = random_cache(rng, 40, 3, 64, 4, 16, "float8")
        pool = on_gpu(lk, c)
        lengths = [100, 17, 64, 0, 0]
        wide = torch.full((5, 11), -1, dtype=torch.int32, device="cuda")
        wide[:, 2:10] = dev(random_table(rng, lengths, 16, 8, 40))
        table, n = wide[:, 2:10], i32(*lengths)
        refs = torch.zeros(40, dtype=torch.int32, device="cuda")
        refs[table[table >= 0].long()] = 1
        lut = dev(rng.standard_normal((5, 6, 4, 256)).astype(np.float32))
        out = torch.zeros((5, 6, 64), device="cuda")
        lk.lookat_pages_fork(pool, table, n, refs, i32(0, 1), i32(3, 4))
        missing = lk.lookat_pages_reserve(pool, table, n, refs, n + 9)
        given = torch.full((1,), 7, dtype=torch.int32, device="cuda")
        ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
        assert lk.lookat_pages_reserve(pool, table, n, refs, n.clone(), given, workspace=ws) is given
        codes = dev(rng.integers(0, 256, (5, 3, 12, 4), dtype=np.uint8))[:, :, 2:11]
        for dtype in (np.float16, np.float32):
            values = dev(rng.standard_normal((5, 3, 9, 64)).astype(dtype))
            lk.lookat_pages_write(pool, codes, values, table, n, i32(9, 3, 0, 1, 9))
        lk.lookat_pages_write(pool, codes, values, table, n)
        made = lk.lookat_attend_pages(lut, pool, table, n, 0.125, 200)
        assert lk.lookat_attend_pages(lut, pool, table, n, 0.125, num_splits=2, out=out) is out
        free = torch.nonzero(refs == 0)[:, 0].to(torch.int32)
        lk.lookat_pages_copy(pool, table[0, :2].contiguous(), free[:2].contiguous())
        lk.lookat_pages_free(pool, table, n, refs, i32(1, 2))
        compacted = lk.lookat_pages_compact(pool, table, n, refs)
        outs = torch.empty((5, 8), dtype=torch.int32, device="cuda"), torch.empty_like(refs), torch.empty_like(given)
        again = lk.lookat_pages_compact(pool, table, n, refs, *outs)
        assert all(x is y for x, y in zip(again, outs)) and all(torch.equal(x, y) for x, y in zip(again, compacted))
        torch.cuda.synchronize()
        states.append([wide, n, refs, missing, given, made, out, *compacted, pool.codes, pool.values.view(torch.uint8), pool.exponents])
        if watch.native:
            assert watch.taken == {name: True for name in ("pages_fork", "pages_reserve", "pages_write", "attend_pages", "pages_copy", "pages_free", "pages_compact")}
    assert all(torch.equal(x, y) for x, y in zip(*states))


@pytest.mark.parametrize("native", [True, False])
def test_what_the_binding_refuses(lk, monkeypatch, native):
    from paper_2601_10155_amd import binding
    if not native:
        monkeypatch.setattr(binding, "_marshal", Watch(None))
    pool = lk.page_pool(10, 2, 64, 4, 16)
    table, n, refs = torch.full((3, 4), -1, dtype=torch.int32, device="cuda"), i32(0, 0, 0), i32(*[0] * 10)
    lut = torch.zeros((3, 2, 4, 256), device="cuda")
    codes, values = torch.zeros((3, 2, 1, 4), dtype=torch.uint8, device="cuda"), torch.zeros((3, 2, 1, 64), device="cuda")
    for bad in (lambda: lk.lookat_attend_pages(lut, pool, table.long(), n, 1.0), lambda: lk.lookat_attend_pages(lut, pool, table.t(), n, 1.0),
                lambda: lk.lookat_attend_pages(lut, pool, table, n[:2], 1.0), lambda: lk.lookat_attend_pages(lut.half(), pool, table, n, 1.0),
                lambda: lk.lookat_attend_pages(lut[:, :, :3], pool, table, n, 1.0), lambda: lk.lookat_attend_pages(lut[:2], pool, table, n, 1.0),
                lambda: lk.lookat_attend_pages(lut[:, :1].contiguous(), pool, table, n, 1.0), lambda: lk.lookat_attend_pages(lut, pool, table.cpu(), n, 1.0),
                lambda: lk.lookat_attend_pages(lut, pool, table, n, 1.0, out=lut), lambda: lk.lookat_attend_pages(lut.cpu(), pool, table, n, 1.0),
                lambda: lk.lookat_pages_write(pool, codes, values[:2], table, n), lambda: lk.lookat_pages_write(pool, codes, values[..., :32], table, n),
                lambda: lk.lookat_pages_write(pool, codes, values, table[:2], n), lambda: lk.lookat_pages_write(pool, codes.int(), values, table, n),
                lambda: lk.lookat_pages_write(pool, codes, values.permute(0, 1, 3, 2).contiguous().permute(0, 1, 3, 2).expand(3, 2, 2, 64), table, n),
                lambda: lk.lookat_pages_write(pool, codes, values, table, n, n.long()), lambda: lk.lookat_pages_copy(pool, n, n[:1]),
                lambda: lk.lookat_pages_copy(pool, n.float(), n), lambda: lk.lookat_pages_fork(pool, table, n, refs[:9], n, n),
                lambda: lk.lookat_pages_free(pool, table, n, refs, n.view(1, 3)), lambda: lk.lookat_pages_reserve(pool, table, n, refs, n[:1]),
                lambda: lk.lookat_pages_compact(pool, table, n, refs, table_out=table[:2].clone())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        lk.lookat_pages_write(pool, codes, values.double(), table, n)
    for bad in (lambda: lk.lookat_pages_reserve(pool, table, n, refs, n), lambda: lk.lookat_pages_compact(pool, table, n, refs, table_out=table),
                lambda: lk.lookat_attend_pages(lut, pool, table, n, 1.0, max_length=-1), lambda: lk.lookat_attend_pages(lut, pool, table, n, 1.0, num_splits=70000),
                lambda: lk.lookat_pages_copy(lk.page_pool(4, 1, 64, 32, 16), n, n)):
        with pytest.raises(lk.LookatError):
            bad()
    torch.cuda.synchronize()
    assert torch.all(table == -1) and torch.all(n == 0)


@pytest.mark.parametrize("native", [True, False])
def test_the_binding_refuses_a_workspace_with_less_memory_than_elements(lk, monkeypatch, native):
    from paper_2601_10155_amd import binding
    if not native:
        monkeypatch.setattr(binding, "_marshal", Watch(None))
    pool = lk.page_pool(10, 2, 64, 4, 16)
    table, n, refs = torch.full((3, 4), -1, dtype=torch.int32, device="cuda"), i32(0, 0, 0), i32(*[0] * 10)
    lut, few = torch.zeros((3, 2, 4, 256), device="cuda"), torch.empty(1, dtype=torch.uint8, device="cuda").expand(1 << 20)
    for bad in (lambda: lk.lookat_attend_pages(lut, pool, table, n, 1.0, num_splits=2, workspace=few),
                lambda: lk.lookat_pages_reserve(pool, table, n, refs, i32(1, 1, 1), workspace=few),
                lambda: lk.lookat_pages_compact(pool, table, n, refs, workspace=few)):
        with pytest.raises(ValueError):
            bad()
