"""Chunk attention, attention sums, eviction and beam selection: what their entry points refuse, before anything reaches the GPU, and what they ask
for.  CPU only."""
import ctypes

import pytest
import torch

from paper_2601_10155_amd import binding
from test_abi import E_ALIGN, E_DTYPE, E_NULL, E_SHAPE, E_UNSUP, E_WS, FAKE, OK, lib  # noqa: F401
from test_pages_abi import BAD_POOLS, D, H, M, PAGE, pool

BIG = 1 << 26


def entry(f, names, good, by_pool=True):
    def call(p=None, **kw):
        a = dict(zip(names, good))
        a.update(kw)
        return f(*([None if p is None else ctypes.byref(p)] if by_pool else []), *a.values())
    return call


def calls(lib):  # noqa: F811
    f32 = ctypes.c_float
    return {
        "chunk": entry(lib.lookat_attend_pages_chunk, ("B", "N", "group", "q", "dtype", "qb", "qh", "qn", "books", "table", "W", "stride", "lengths", "counts",
                                                       "max_length", "scale", "splits", "ws", "wsb", "out", "stream"),
                       (5, 9, 2, FAKE, 1, 9 * 2 * H * D, 9 * D, D, FAKE, FAKE, 7, 7, FAKE, None, 0, f32(0.1), 3, FAKE, BIG, FAKE, None)),
        "weigh": entry(lib.lookat_pages_weigh, ("B", "group", "lut", "table", "W", "stride", "lengths", "max_length", "scale", "decay", "weights", "columns",
                                                "ws_bh", "ws", "wsb", "stream"),
                       (5, 2, FAKE, FAKE, 7, 7, FAKE, 0, f32(0.1), f32(1.0), FAKE, 200, 224, FAKE, BIG, None)),
        "evict": entry(lib.lookat_pages_evict, ("B", "table", "W", "stride", "lengths", "weights", "columns", "w_bh", "keep", "first", "recent", "table_out",
                                                "W_out", "out_stride", "weights_out", "columns_out", "o_bh", "ws", "wsb", "stream"),
                       (5, FAKE, 7, 7, FAKE, FAKE, 200, 224, FAKE, 4, 16, FAKE, 3, 3, FAKE, 96, 96, FAKE, BIG, None)),
    }


@pytest.mark.parametrize("name", ["chunk", "weigh", "evict"])
def test_pools_and_tables(lib, name):  # noqa: F811
    call = calls(lib)[name]
    assert call(None) == E_NULL
    for change, status in BAD_POOLS:
        assert call(pool(**change)) == status, change
        assert lib.lookat_last_error()
    assert call(pool(), B=0) == E_SHAPE and call(pool(), B=65536) == E_UNSUP
    assert call(pool(), W=0) == E_SHAPE and call(pool(), stride=6) == E_SHAPE
    assert call(pool(), table=None) == E_NULL and call(pool(), table=FAKE + 2) == E_ALIGN
    assert call(pool(), W=1 << 26, stride=1 << 26) == E_UNSUP
    assert call(pool(), lengths=None) == E_NULL and call(pool(), lengths=FAKE + 2) == E_ALIGN
    assert call(pool(), ws=FAKE + 4) == E_ALIGN or name == "weigh"


def test_chunk(lib):  # noqa: F811
    call, p = calls(lib)["chunk"], pool()
    assert call(p, N=0) == OK and call(p, N=-1) == E_SHAPE
    assert call(p, group=0) == E_SHAPE and call(p, group=65) == E_UNSUP
    assert call(p, N=1 << 24, group=2) == E_UNSUP
    assert call(pool(H=4096), group=16) == E_UNSUP
    assert call(p, dtype=3) == E_DTYPE and call(p, dtype=0) == E_DTYPE
    for x in ("q", "books", "out"):
        assert call(p, **{x: None}) == E_NULL and call(p, **{x: FAKE + 8}) == E_ALIGN
    for x in ("qb", "qh", "qn"):
        assert call(p, **{x: 4}) == E_ALIGN and call(p, **{x: 2, "dtype": 2}) == E_ALIGN
    assert call(p, counts=FAKE + 1) == E_ALIGN
    assert call(p, max_length=-1) == E_SHAPE and call(p, splits=-1) == E_SHAPE and call(p, splits=65536) == E_SHAPE
    need = lib.lookat_attend_pages_chunk_workspace_bytes
    bytes_ = need(ctypes.byref(p), 5, 9, 2, 7, 0, 3)
    books = H * 256 * D * 4 + 16
    assert need(ctypes.byref(p), 5, 9, 2, 7, 0, 1) == books
    assert bytes_ == books + 5 * H * 3 * 32 * (D + 4) * 4        # (18 rows: tiles of 32)
    assert call(p, ws=None) == E_WS and call(p, wsb=bytes_ - 1) == E_WS
    assert need(ctypes.byref(p), 5, 0, 2, 7, 0, 0) == 0 and need(None, 5, 9, 2, 7, 0, 0) == 0 and need(ctypes.byref(p), 5, 9, 65, 7, 0, 0) == 0
    # a launch counts its threads in 32 bits
    assert call(pool(H=4096), B=65535, group=1, N=1 << 20, splits=1, wsb=1 << 62) == E_UNSUP
    assert call(pool(H=4096), B=65535, group=1, N=64, splits=65535, wsb=1 << 62) == E_UNSUP


def test_weigh(lib):  # noqa: F811
    call, p = calls(lib)["weigh"], pool()
    assert call(p, group=3) == E_UNSUP and call(p, group=0) == E_UNSUP and call(p, group=16) == E_UNSUP
    assert call(p, max_length=-1) == E_SHAPE
    assert call(p, columns=0) == E_SHAPE and call(p, ws_bh=199) == E_SHAPE
    assert call(p, lut=None) == E_NULL and call(p, weights=None) == E_NULL
    assert call(p, lut=FAKE + 4) == E_ALIGN and call(p, weights=FAKE + 2) == E_ALIGN
    need = lib.lookat_pages_weigh_workspace_bytes
    assert need(ctypes.byref(p), 5, 2, 7, 0) == 0                # (short rows are not cut)
    long = need(ctypes.byref(p), 5, 2, 4096, 0)
    assert long > 0 and need(None, 5, 2, 4096, 0) == 0 and need(ctypes.byref(p), 5, 3, 4096, 0) == 0
    assert call(p, W=4096, stride=4096, ws=None) == E_WS and call(p, W=4096, stride=4096, wsb=long - 1) == E_WS
    assert call(p, W=4096, stride=4096, ws=FAKE + 8) == E_ALIGN
    assert call(pool(H=4096), B=65535, wsb=1 << 62) == E_UNSUP


def test_evict(lib):  # noqa: F811
    call, p = calls(lib)["evict"], pool()
    assert call(p, W_out=0) == E_SHAPE and call(p, W_out=1 << 26, out_stride=1 << 26) == E_UNSUP and call(p, out_stride=2) == E_SHAPE
    assert call(p, table_out=None) == E_NULL and call(p, table_out=FAKE + 2) == E_ALIGN
    assert call(p, columns=0) == E_SHAPE and call(p, w_bh=199) == E_SHAPE
    assert call(p, columns_out=0) == E_SHAPE and call(p, o_bh=95) == E_SHAPE
    assert call(p, first=-1) == E_SHAPE and call(p, recent=-1) == E_SHAPE
    assert call(p, weights=None) == E_NULL and call(p, keep=None) == E_NULL
    for x in ("weights", "keep", "weights_out"):
        assert call(p, **{x: FAKE + 2}) == E_ALIGN
    need = lib.lookat_pages_evict_workspace_bytes
    assert need(ctypes.byref(p), 5, 3) == 5 * H * 3 * PAGE * 4 and need(None, 5, 3) == 0 and need(ctypes.byref(p), 0, 3) == 0
    assert call(p, ws=None) == E_WS and call(p, wsb=5 * H * 3 * PAGE * 4 - 1) == E_WS
    assert call(pool(H=4096), B=65535, wsb=1 << 62) == E_UNSUP


def test_select(lib):  # noqa: F811
    names = ("Q", "beams", "V", "n", "logits", "dtype", "stride", "scores", "first", "scores_out", "parents", "tokens", "ws", "wsb", "stream")
    f = entry(lib.lookat_beam_select, names, (3, 4, 1000, 8, FAKE, 1, 1000, FAKE, 0, FAKE, FAKE, FAKE, FAKE, BIG, None), by_pool=False)
    call = lambda **kw: f(**kw)  # noqa: E731
    for x in ("Q", "beams", "V", "n"):
        assert call(**{x: 0}) == E_SHAPE and call(**{x: -1}) == E_SHAPE
    assert call(n=65) == E_UNSUP and call(beams=1025) == E_UNSUP and call(Q=20000) == E_UNSUP and call(V=(1 << 24) + 1, stride=1 << 25) == E_UNSUP
    assert call(dtype=3) == E_DTYPE
    assert call(stride=999) == E_SHAPE
    assert call(first=-1) == E_SHAPE and call(first=0x7fffffff) == E_SHAPE
    for x in ("logits", "scores", "scores_out", "parents", "tokens"):
        assert call(**{x: None}) == E_NULL and call(**{x: FAKE + 1}) == E_ALIGN
    assert call(logits=FAKE + 2, dtype=2) == E_ALIGN and call(scores=FAKE + 2) == E_ALIGN
    need = lib.lookat_beam_select_workspace_bytes
    bytes_ = need(3, 4, 1000, 8)
    assert bytes_ > 0 and need(3, 4, 1000, 65) == 0 and need(0, 4, 1000, 8) == 0
    assert call(ws=None) == E_WS and call(wsb=bytes_ - 1) == E_WS and call(ws=FAKE + 8) == E_ALIGN
    assert call(Q=64, beams=1023, V=1 << 24, stride=1 << 24, n=64, wsb=1 << 62) == E_UNSUP


def test_the_binding_refuses_tensors_on_the_host(lib):  # noqa: F811
    x = binding.PagePool(torch.zeros((2, 1, 16, 4), dtype=torch.uint8), torch.zeros((2, 1, 2, 64, 8), dtype=torch.int8), torch.zeros((2, 1), dtype=torch.int8))
    i, w = torch.zeros(1, dtype=torch.int32), torch.zeros((1, 1, 16))
    with pytest.raises(ValueError):
        binding.lookat_attend_pages_chunk(torch.zeros((1, 1, 1, 64)), torch.zeros((1, 4, 256, 16)), x, i[None], i, 0.1)
    with pytest.raises(ValueError):
        binding.lookat_pages_weigh(torch.zeros((1, 1, 4, 256)), x, i[None], i, 0.1, w)
    with pytest.raises(ValueError):
        binding.lookat_pages_evict(x, i[None], i, w, i, i[None])
    with pytest.raises(ValueError):
        binding.lookat_beam_select(torch.zeros((2, 10)), torch.zeros(2), 2, 3)
