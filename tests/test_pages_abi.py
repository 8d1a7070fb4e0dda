"""The paged cache's entry points: what they refuse, before anything reaches the GPU, and the reference's own pins.  CPU only."""
import ctypes
import math

import numpy as np
import pytest
import torch

import pages_ref as pr
from paper_2601_10155_amd import binding
from paper_2601_10155_amd.binding import _Pool as Pool
from test_abi import E_ALIGN, E_DTYPE, E_NULL, E_SHAPE, E_UNSUP, E_WS, FAKE, OK, lib  # noqa: F401

PAGES, H, D, M, PAGE = 100, 3, 64, 4, 32


def pool(**kw):
    f = dict(pages=PAGES, H=H, d_k=D, m=M, page=PAGE, value_type=1, codes=FAKE, values=FAKE, exponents=FAKE)
    f.update(kw)
    return Pool(**f)


BAD_POOLS = [({"pages": 0}, E_SHAPE), ({"H": -1}, E_SHAPE), ({"page": 0}, E_SHAPE), ({"value_type": 0}, E_DTYPE), ({"value_type": 3}, E_DTYPE),
             ({"d_k": 96}, E_UNSUP), ({"m": 1}, E_UNSUP), ({"m": 32}, E_UNSUP), ({"page": 8}, E_UNSUP), ({"page": 48}, E_UNSUP),
             ({"page": 256}, E_UNSUP), ({"pages": (1 << 30) + 1}, E_UNSUP), ({"H": 4097}, E_UNSUP), ({"codes": None}, E_NULL), ({"values": None}, E_NULL),
             ({"exponents": None}, E_NULL), ({"codes": FAKE + 8}, E_ALIGN), ({"values": FAKE + 4}, E_ALIGN)]


def calls(lib):
    """Every entry point as f(pool, **changes), with arguments that would be valid."""
    def entry(f, names, good):
        def call(p, **kw):
            a = dict(zip(names, good))
            a.update(kw)
            return f(None if p is None else ctypes.byref(p), *a.values())
        return call
    big = 1 << 20
    books = ("S", "table", "W", "stride", "lengths", "refs")
    good = (5, FAKE, 7, 7, FAKE, FAKE)
    return {
        "write": entry(lib.lookat_pages_write, ("B", "N", "codes", "cs", "values", "dtype", "vs", "table", "W", "stride", "lengths", "counts", "stream"),
                       (5, 10, FAKE, 10 * M, FAKE, 1, 10 * D, FAKE, 7, 7, FAKE, None, None)),
        "attend": entry(lib.lookat_attend_pages, ("B", "group", "lut", "table", "W", "stride", "lengths", "max_length", "scale", "splits", "ws", "wsb", "out", "stream"),
                        (5, 2, FAKE, FAKE, 7, 7, FAKE, 0, ctypes.c_float(0.1), 3, FAKE, big, FAKE, None)),
        "copy": entry(lib.lookat_pages_copy, ("n", "src", "dst", "stream"), (4, FAKE, FAKE, None)),
        "fork": entry(lib.lookat_pages_fork, books + ("n", "src", "dst", "stream"), good + (2, FAKE, FAKE, None)),
        "free": entry(lib.lookat_pages_free, books + ("n", "slots", "stream"), good + (2, FAKE, None)),
        "reserve": entry(lib.lookat_pages_reserve, books + ("new", "missing", "copies", "ws", "wsb", "stream"), good + (FAKE + 64, FAKE, None, FAKE, big, None)),
        "compact": entry(lib.lookat_pages_compact, ("S", "table", "W", "stride", "lengths", "refs", "table_out", "out_stride", "refs_out", "live", "ws", "wsb", "stream"),
                         good + (FAKE + 4096, 7, FAKE + 4096, FAKE, FAKE, big, None)),
    }


@pytest.mark.parametrize("name", ["write", "attend", "copy", "fork", "free", "reserve", "compact"])
def test_every_call_refuses_bad_pools(lib, name):  # noqa: F811
    call = calls(lib)[name]
    assert call(None) == E_NULL
    for change, status in BAD_POOLS:
        assert call(pool(**change)) == status, change
        assert lib.lookat_last_error()


@pytest.mark.parametrize("name", ["write", "attend", "fork", "free", "reserve", "compact"])
def test_every_call_refuses_bad_tables(lib, name):  # noqa: F811
    call = calls(lib)[name]
    rows = "B" if name in ("write", "attend") else "S"
    assert call(pool(), **{rows: 0}) == E_SHAPE
    assert call(pool(), **{rows: 65536}) == E_UNSUP
    assert call(pool(), W=0) == E_SHAPE
    assert call(pool(), stride=6) == E_SHAPE
    assert call(pool(), table=None) == E_NULL
    assert call(pool(), table=FAKE + 2) == E_ALIGN
    assert call(pool(), W=1 << 26, stride=1 << 26) == E_UNSUP       # 2^26 pages of 32 tokens
    assert call(pool(), lengths=None) == E_NULL
    assert call(pool(), lengths=FAKE + 2) == E_ALIGN
    if name not in ("write", "attend"):
        assert call(pool(), refs=None) == E_NULL


def test_write_refusals(lib):  # noqa: F811
    call = calls(lib)["write"]
    assert call(pool(), N=0) == OK
    assert call(pool(), N=-1) == E_SHAPE
    assert call(pool(), N=(1 << 30) + 1) == E_UNSUP
    assert call(pool(), dtype=3) == E_DTYPE
    assert call(pool(), codes=None) == E_NULL and call(pool(), values=None) == E_NULL
    assert call(pool(), cs=10 * M - 4) == E_SHAPE and call(pool(), vs=10 * D - 8) == E_SHAPE
    assert call(pool(), cs=10 * M + 2) == E_ALIGN and call(pool(), vs=10 * D + 4) == E_ALIGN
    assert call(pool(), codes=FAKE + 2) == E_ALIGN and call(pool(), values=FAKE + 8) == E_ALIGN
    assert call(pool(), counts=FAKE + 1) == E_ALIGN


def test_attend_refusals_and_workspace(lib):  # noqa: F811
    call = calls(lib)["attend"]
    p = pool()
    assert call(p, group=3) == E_UNSUP and call(p, group=0) == E_UNSUP and call(p, group=16) == E_UNSUP
    assert call(p, max_length=-1) == E_SHAPE
    assert call(p, splits=-1) == E_SHAPE and call(p, splits=65536) == E_SHAPE
    assert call(p, lut=None) == E_NULL and call(p, out=None) == E_NULL
    assert call(p, lut=FAKE + 4) == E_ALIGN and call(p, out=FAKE + 8) == E_ALIGN
    need = lib.lookat_attend_pages_workspace_bytes
    assert need(ctypes.byref(p), 5, 2, 7, 0, 1) == 0
    assert need(ctypes.byref(p), 5, 2, 7, 0, 3) == 5 * H * 2 * 3 * (D + 2) * 4
    assert call(p, ws=None) == E_WS and call(p, wsb=need(ctypes.byref(p), 5, 2, 7, 0, 3) - 1) == E_WS
    assert call(p, ws=FAKE + 4) == E_ALIGN
    assert need(ctypes.byref(p), 5, 3, 7, 0, 0) == 0 and need(None, 5, 1, 7, 0, 3) == 0           # (refused by the call)
    # long caches are cut into ranges, unless the caller knows that they are short
    assert need(ctypes.byref(p), 1, 1, 1024, 0, 0) > 0 and need(ctypes.byref(p), 1, 1, 1024, 64, 0) == 0
    assert call(p, W=1024, stride=1024, splits=0, wsb=need(ctypes.byref(p), 5, 2, 1024, 0, 0) - 1) == E_WS


def test_upkeep_refusals(lib):  # noqa: F811
    c = calls(lib)
    for name in ("copy", "fork", "free"):
        assert c[name](pool(), n=0) == OK
        assert c[name](pool(), n=-1) == E_SHAPE
        key = "slots" if name == "free" else "src"
        assert c[name](pool(), **{key: None}) == E_NULL
        assert c[name](pool(), **{key: FAKE + 1}) == E_ALIGN
    assert c["copy"](pool(H=4096, page=128, d_k=128, m=16), n=1 << 30) == E_UNSUP
    r = c["reserve"]
    assert r(pool(), new=None) == E_NULL and r(pool(), missing=None) == E_NULL and r(pool(), copies=FAKE + 2) == E_ALIGN
    assert r(pool(), new=FAKE) == E_SHAPE and r(pool(), new=FAKE + 16) == E_SHAPE and r(pool(), new=FAKE - 4) == E_SHAPE      # over lengths
    need = lib.lookat_pages_reserve_workspace_bytes(ctypes.byref(pool()), 5)
    assert need > 0 and r(pool(), wsb=need - 1) == E_WS and r(pool(), ws=None) == E_WS and r(pool(), ws=FAKE + 4) == E_ALIGN
    k = c["compact"]
    assert k(pool(), table_out=None) == E_NULL and k(pool(), refs_out=None) == E_NULL and k(pool(), live=None) == E_NULL
    assert k(pool(), table_out=FAKE) == E_SHAPE and k(pool(), refs_out=FAKE + 8) == E_SHAPE      # over the old ones
    assert k(pool(), out_stride=6) == E_SHAPE
    need = lib.lookat_pages_compact_workspace_bytes(ctypes.byref(pool()))
    assert need > 0 and k(pool(), wsb=need - 1) == E_WS


def test_more_threads_than_one_launch_counts(lib):  # noqa: F811
    """2^32 threads along x: refused by name, not by whatever a launch of them would do."""
    c, many = calls(lib), 1 << 24                                         # workgroups of 256
    for name in ("copy", "fork", "free"):
        assert c[name](pool(), n=many) == E_UNSUP and b"launch" in lib.lookat_last_error()
    assert c["write"](pool(page=16), N=1 << 28, cs=M << 28, vs=D << 28, W=1 << 26, stride=1 << 26) == E_UNSUP
    assert b"launch" in lib.lookat_last_error()
    for splits in (0, 1):                                                 # (65535 * 129 and not more than 4096 heads: 2^23 workgroups of 512)
        assert c["attend"](pool(H=129), B=65535, W=4, stride=4, splits=splits) == E_UNSUP
        assert b"launch" in lib.lookat_last_error()


def test_binding_refuses_what_is_not_a_pool():
    p = binding.PagePool(torch.zeros((4, 2, 16, 4), dtype=torch.uint8), torch.zeros((4, 2, 2, 64, 8), dtype=torch.int8),
                         torch.zeros((4, 2), dtype=torch.int8))
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="device memory"):
        binding.lookat_pages_copy(p, ints(0), ints(1))
    for bad in (p._replace(codes=p.codes.int()), p._replace(values=p.values[:, :, :1]), p._replace(exponents=p.exponents[:3]),
                p._replace(values=p.values.permute(0, 1, 2, 4, 3)), p._replace(exponents=p.exponents.float())):
        with pytest.raises(ValueError):
            binding.lookat_pages_copy(bad, ints(0), ints(1))
    with pytest.raises(TypeError):
        binding.lookat_pages_copy(p._replace(values=p.values.float()), ints(0), ints(1))
    with pytest.raises(TypeError):
        binding.page_pool(4, 2, 64, 4, value_dtype=torch.float16, device="cpu")
    made = binding.page_pool(4, 2, 64, 4, 16, torch.float8_e4m3fn, device="cpu")
    assert made.codes.shape == (4, 2, 16, 4) and made.values.shape == (4, 2, 2, 64, 8) and made.exponents.shape == (4, 2)


# ---- the reference's own pins ---------------------------------------------------------------------------------------
def test_binding_refuses_a_workspace_with_less_memory_than_elements():
    p = binding.page_pool(4, 2, 64, 4, 16, device="cpu")
    with pytest.raises(ValueError, match="contiguous"):
        binding._scratch(torch.empty(1, dtype=torch.uint8).expand(4096), 1024, p)
    given = torch.empty(4096, dtype=torch.uint8)
    assert binding._scratch(given, 1024, p) is given and binding._scratch(given, 8192, p).numel() == 8192


def test_reference_e4m3_against_torch():
    every = torch.arange(256, dtype=torch.uint8)
    values = every.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(pr.E4M3, values, equal_nan=True)
    rng = np.random.default_rng(5)
    grid = pr.E4M3[:127]
    mid = (grid[1:] + grid[:-1]) / 2                                         # ties, exact in fp32
    x = np.concatenate([rng.standard_normal(4000) * 100, rng.standard_normal(1000) * 0.01, grid, mid, -mid, [0.0, 1e-9, 448.0]])
    x = x.clip(-448, 448).astype(np.float32)
    assert np.array_equal(pr.to_bytes(x, "float8"), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert pr.to_bytes(np.array([math.nan, 1e9, -math.inf]), "float8").tolist() == [0, 126, 254]


@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_reference_exponents(kind):
    rng = np.random.default_rng(6)
    for top in np.concatenate([np.exp(rng.uniform(-20, 30, 500)), pr.most(kind) * 2.0 ** np.arange(-20, 20), np.nextafter(pr.most(kind) * 2.0 ** np.arange(-20, 20), 1e30)]):
        e = pr.exponent(float(top), kind)
        assert top <= pr.most(kind) * 2.0 ** e and top > pr.most(kind) * 2.0 ** (e - 1)
    assert pr.exponent(0.0, kind) == -40 and pr.exponent(math.inf, kind) == 40 and pr.exponent(1e-300, kind) == -40


@pytest.mark.parametrize("kind", ["int8", "float8"])
def test_reference_rounding_stays_within_a_step(kind):
    """Tokens written one at a time, growing: however often a page's exponent grew, what is stored is less than a step (int8) off the value; in
    the floating type, whose steps grow with the numbers, half a step of the value (2^-4 of it) and the rounding steps of its
    subnormals (2^-9, at most one each time the exponent grows: halved every time, below one together)."""
    rng = np.random.default_rng(7)
    H, d, page = 1, 64, 16
    c = pr.Cache(np.zeros((1, H, page, 2), np.uint8), np.zeros((1, H, page // 8, d, 8), np.uint8), np.zeros((1, H), np.int8), kind)
    v = rng.standard_normal((1, H, page, d)) * 1.7 ** np.arange(page)[None, None, :, None]
    table = np.zeros((1, 1), np.int32)
    for n in range(page):
        c.write(np.zeros((1, H, 1, 2), np.uint8), v[:, :, n: n + 1], table, [n + 1])
    step = 2.0 ** float(c.exponents[0, 0])
    off = np.abs(c.tokens(table[0], page)[1] - v[0])
    assert np.all(off < (step if kind == "int8" else np.maximum(np.abs(v[0]) * 2.0 ** -4 * 1.0001, step * 2.0 ** -9)))
