"""Prompts in chunks, a search over continuations and a budget for the cache, as a user runs them together, against the same steps in plain numpy; and
the native marshalling of these calls against the Python one."""
import math

import numpy as np
import pytest
import torch

import pages_ref as pr
from test_gpu_beam_select import reference as select_reference
from test_gpu_marshal import both  # noqa: F401
from test_gpu_pages import TORCH, assert_pool, dev, i32, lk, on_gpu, random_cache, random_table  # noqa: F401
from test_gpu_pages_chunk import books_of, reference as chunk_reference
from test_gpu_pages_keep import evict_reference, weigh_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,d_k,m,page,g", [("int8", 64, 4, 16, 2), ("float8", 128, 8, 32, 1)])
def test_prompts_search_and_budget(lk, kind, d_k, m, page, g):  # noqa: F811
    """Two requests of three beams.  Slots 0-5 and 6-11 hold the beams in turn, 12-17 what is kept of them."""
    rng = np.random.default_rng(21)
    Q, beams, H, V, W, P = 2, 3, 2, 500, 8, 120
    R, S, scale = Q * beams, 3 * Q * beams, 1 / math.sqrt(d_k)
    books = books_of(rng, H, m, d_k)
    d_books = dev(books)
    c = random_cache(rng, P, H, d_k, m, page, kind)
    ref = pr.Books(np.full((S, W), -1, np.int32), np.zeros(S, np.int32), np.zeros(P, np.int32), page)
    pool, table, lengths, refs = on_gpu(lk, c), dev(ref.table), dev(ref.lengths), dev(ref.refs)

    def same_books():
        for a, b in ((table, ref.table), (lengths, ref.lengths), (refs, ref.refs)):
            assert np.array_equal(a.cpu().numpy(), b)

    def reserve(new):
        assert int(lk.lookat_pages_reserve(pool, table, lengths, refs, dev(np.array(new, np.int32)))) == 0
        assert ref.reserve(new, c) == 0

    def write(rows, keys, values, counts):
        codes = lk.lookat_encode_keys(dev(keys), d_books)
        lk.lookat_pages_write(pool, codes, dev(values), table[rows], lengths[rows], i32(*counts))
        c.write(codes.cpu().numpy(), values, ref.table[rows], ref.lengths[rows], counts)

    # the prompts, in two pieces
    firsts = [q * beams for q in range(Q)]
    for counts in ([24, 30], [13, 0]):
        new = np.zeros(S, np.int32)
        for slot, n in zip(firsts, counts):
            new[slot] = ref.lengths[slot] + n
        reserve(new)
        n = max(counts)
        k, v = rng.standard_normal((Q, H, n, d_k)).astype(np.float16), rng.standard_normal((Q, H, n, d_k)).astype(np.float16)
        q = rng.standard_normal((Q, H * g, n, d_k)).astype(np.float16)
        write(firsts, k, v, counts)
        out = lk.lookat_attend_pages_chunk(dev(q), d_books, pool, table[firsts], lengths[firsts], scale, counts=i32(*counts))
        want, bound = chunk_reference(c, q, books, ref.table[firsts], ref.lengths[firsts], counts, scale, np.zeros(q.shape))
        assert np.all(np.abs(out.cpu().numpy() - want) <= bound)
    same_books()
    src, dst = [q * beams for q in range(Q) for _ in range(1, beams)], [q * beams + i for q in range(Q) for i in range(1, beams)]
    lk.lookat_pages_fork(pool, table, lengths, refs, i32(*src), i32(*dst))
    ref.fork(src, dst)
    same_books()

    weights = torch.zeros((S, H, W * page), device="cuda")
    ref_weights = np.zeros((S, H, W * page), np.float32)
    scores = np.where(np.arange(R) % beams == 0, 0.0, -np.inf).astype(np.float32)      # (the beams of a request that begins are one)
    for step in range(4):
        old, new_slots = (step % 2) * R, ((step + 1) % 2) * R
        logits = (3 * rng.standard_normal((R, V))).astype(np.float16)
        s, parents, tokens = lk.lookat_beam_select(dev(logits), dev(scores), beams, beams, first_parent=old)
        want = select_reference(logits, scores, beams, beams, old)
        assert want[3] > 2.0 ** -20
        assert np.array_equal(parents.cpu().numpy(), want[1]) and np.array_equal(tokens.cpu().numpy(), want[2])
        parents, scores = parents.view(-1), s.view(-1).cpu().numpy()
        children = torch.arange(new_slots, new_slots + R, dtype=torch.int32, device="cuda")
        lk.lookat_pages_free(pool, table, lengths, refs, children)
        lk.lookat_pages_fork(pool, table, lengths, refs, parents, children)
        ref.free(list(range(new_slots, new_slots + R)))
        ref.fork(parents.cpu().tolist(), list(range(new_slots, new_slots + R)))
        weights[new_slots:new_slots + R] = weights[parents.long()]
        ref_weights[new_slots:new_slots + R] = ref_weights[parents.cpu().numpy()]
        new = np.zeros(S, np.int32)
        new[new_slots:new_slots + R] = ref.lengths[new_slots:new_slots + R] + 1
        reserve(new)
        rows = list(range(new_slots, new_slots + R))
        k, v = rng.standard_normal((R, H, 1, d_k)).astype(np.float16), rng.standard_normal((R, H, 1, d_k)).astype(np.float16)
        write(rows, k, v, [1] * R)
        q = rng.standard_normal((R, H, g, d_k)).astype(np.float16)
        lut = lk.lookat_build_lut(dev(q), d_books).view(R, H * g, m, 256)
        out = lk.lookat_attend_pages(lut, pool, table[rows], lengths[rows], scale)
        want, bound = c.attend(lut.cpu().numpy(), ref.table[rows], ref.lengths[rows], scale)
        assert np.all(np.abs(out.cpu().numpy() - want) <= bound)
        mine = weights[new_slots:new_slots + R]
        lk.lookat_pages_weigh(lut, pool, table[rows], lengths[rows], scale, mine, decay=0.9)
        want, bound = weigh_reference(c, lut.cpu().numpy(), ref.table[rows], ref.lengths[rows], scale, 0.9, ref_weights[rows])
        assert np.all(np.abs(mine.cpu().numpy() - want) <= bound)
        ref_weights[rows] = mine.cpu().numpy()            # (what is chosen below goes by the device's weights)
        same_books()
        assert_pool(pool, c)
    # down to 20 tokens: room, the tokens, the old sequences given up
    rows, kept = list(range(R)) if 4 % 2 == 0 else list(range(R, 2 * R)), list(range(2 * R, 3 * R))
    keep = [20, 18, 20, 1, 20, 33]
    new = np.zeros(S, np.int32)
    new[kept] = np.minimum(keep, ref.lengths[rows])
    reserve(new)
    moved = torch.zeros((R, H, W * page), device="cuda")
    lk.lookat_pages_evict(pool, table[rows], lengths[rows], weights[rows], i32(*keep), table[kept], first=2, recent=5, weights_out=moved)
    after, places, want = evict_reference(c, ref.table[rows], ref.lengths[rows], ref_weights[rows], keep, 2, 5, ref.table[kept], np.zeros((R, H, W * page), np.float32))
    assert np.array_equal(moved.cpu().numpy(), want)
    assert_pool(pool, after)
    c.codes, c.values, c.exponents = after.codes, after.values, after.exponents
    lk.lookat_pages_free(pool, table, lengths, refs, torch.arange(2 * R, dtype=torch.int32, device="cuda"))
    ref.free(list(range(2 * R)))
    same_books()
    assert int((refs > 0).sum()) == sum(-(-int(n) // page) for n in np.minimum(keep, new[kept]))
    out = lk.lookat_attend_pages(lut, pool, table[kept], lengths[kept], scale)
    want, bound = c.attend(lut.cpu().numpy(), ref.table[kept], ref.lengths[kept], scale)
    assert np.all(np.abs(out.cpu().numpy() - want) <= bound)


def serving_case(lk, dtype):  # noqa: F811
    rng = np.random.default_rng(7)
    c = random_cache(rng, 40, 4, 64, 4, 16, "int8")
    table = random_table(rng, [60, 33, 17], 16, 4, 40)
    free = np.setdiff1d(np.arange(40), table)[:9].reshape(3, 3).astype(np.int32)
    return {"pool": on_gpu(lk, c), "table": dev(table), "lengths": i32(60, 33, 17), "counts": i32(9, 2, 9), "books": dev(books_of(rng, 4, 4, 64)),
            "q": dev(rng.standard_normal((3, 9, 8, 64))).to(dtype).transpose(1, 2), "lut": dev(rng.standard_normal((3, 8, 4, 256)).astype(np.float32)),
            "weights": dev(rng.random((3, 4, 70)).astype(np.float32))[:, :, :64], "keep": i32(30, 20, 5), "out": dev(free),
            "logits": dev(rng.standard_normal((6, 900))).to(dtype), "scores": dev(-rng.random(6).astype(np.float32))}


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_calls_that_are_taken(lk, both, dtype):  # noqa: F811
    s = serving_case(lk, dtype)
    chunk = lambda **kw: lk.lookat_attend_pages_chunk(s["q"], s["books"], s["pool"], s["table"], s["lengths"], 0.1, **kw)  # noqa: E731
    for kw in ({}, {"counts": s["counts"]}, {"num_splits": 2}, {"counts": s["counts"], "out": torch.ones((3, 8, 9, 64), device="cuda")}):
        a, b, taken = both(lambda: chunk(**kw).clone())
        assert taken and torch.equal(a, b)

    def weigh():
        w = s["weights"].clone()
        assert lk.lookat_pages_weigh(s["lut"], s["pool"], s["table"], s["lengths"], 0.1, w, decay=0.5) is w
        return w
    a, b, taken = both(weigh)
    assert taken and torch.equal(a, b)

    def evict():
        w, pool = torch.zeros((3, 4, 40), device="cuda"), lk.PagePool(*(x.clone() for x in s["pool"]))
        lk.lookat_pages_evict(pool, s["table"], s["lengths"], s["weights"], s["keep"], s["out"], first=1, recent=3, weights_out=w)
        return [w, *(x.view(torch.uint8) for x in pool)]
    a, b, taken = both(evict)
    assert taken and all(torch.equal(x, y) for x, y in zip(a, b))
    a, b, taken = both(lambda: lk.lookat_beam_select(s["logits"], s["scores"], 3, 5, first_parent=6))
    assert taken and all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_that_are_left_or_refused(lk, both):  # noqa: F811
    s = serving_case(lk, torch.float16)
    # odd alignment: copied by the Python function; given outputs: looked at there
    odd = torch.empty(s["q"].numel() + 1, dtype=torch.float16, device="cuda")[1:].view(s["q"].shape).copy_(s["q"])
    a, b, taken = both(lambda: lk.lookat_attend_pages_chunk(odd, s["books"], s["pool"], s["table"], s["lengths"], 0.1))
    assert not taken and torch.equal(a, b)
    scores_out = torch.empty((2, 5), device="cuda")
    assert lk.lookat_beam_select(s["logits"], s["scores"], 3, 5, scores_out=scores_out)[0] is scores_out
    none = lk.lookat_attend_pages_chunk(s["q"][:, :, :0], s["books"], s["pool"], s["table"], s["lengths"], 0.1)
    assert none.shape == (3, 8, 0, 64)
    chunk = lambda **kw: lk.lookat_attend_pages_chunk(**{"q": s["q"], "codebooks": s["books"], "pool": s["pool"], "table": s["table"], "lengths": s["lengths"],  # noqa: E731
                                                         "scale": 0.1, **kw})
    for kw, error in (({"q": s["q"].double()}, TypeError), ({"q": s["q"][:, :7]}, ValueError), ({"q": s["q"][:2]}, ValueError), ({"q": s["q"].cpu()}, ValueError),
                      ({"codebooks": s["books"][:3]}, ValueError), ({"codebooks": s["books"].half()}, ValueError), ({"table": s["table"].long()}, ValueError),
                      ({"lengths": s["lengths"][:2]}, ValueError), ({"counts": s["counts"].long()}, ValueError),
                      ({"out": torch.zeros((3, 8, 9, 32), device="cuda")}, ValueError), ({"num_splits": -1}, lk.LookatError)):
        with pytest.raises(error):
            chunk(**kw)
    weigh = lambda **kw: lk.lookat_pages_weigh(**{"lut": s["lut"], "pool": s["pool"], "table": s["table"], "lengths": s["lengths"], "scale": 0.1,  # noqa: E731
                                                  "weights": s["weights"], **kw})
    for kw, error in (({"lut": s["lut"][:, :7]}, ValueError), ({"lut": s["lut"][:, :4].repeat(1, 3, 1, 1)}, lk.LookatError), ({"weights": s["weights"][:, :3]}, ValueError),
                      ({"weights": s["weights"].double()}, ValueError), ({"weights": s["weights"].transpose(0, 1)}, ValueError),
                      ({"weights": s["weights"][:, :, ::2]}, ValueError), ({"weights": s["weights"][:, :, :0]}, ValueError)):
        with pytest.raises(error):
            weigh(**kw)
    evict = lambda **kw: lk.lookat_pages_evict(**{"pool": s["pool"], "table": s["table"], "lengths": s["lengths"], "weights": s["weights"], "keep": s["keep"],  # noqa: E731
                                                  "table_out": s["out"], **kw})
    for kw, error in (({"table_out": s["out"][:2]}, ValueError), ({"keep": s["keep"].long()}, ValueError), ({"first": -1}, lk.LookatError),
                      ({"weights_out": torch.zeros((3, 3, 40), device="cuda")}, ValueError)):
        with pytest.raises(error):
            evict(**kw)
    select = lambda **kw: lk.lookat_beam_select(**{"logits": s["logits"], "scores": s["scores"], "beams": 3, "n": 5, **kw})  # noqa: E731
    for kw, error in (({"beams": 4}, ValueError), ({"beams": 0}, ValueError), ({"n": 0}, ValueError), ({"n": 65}, lk.LookatError), ({"logits": s["logits"].double()}, TypeError),
                      ({"logits": s["logits"].t()}, ValueError), ({"logits": s["logits"][:1].expand(6, -1)}, ValueError), ({"scores": s["scores"].half()}, ValueError),
                      ({"scores": s["scores"].cpu()}, ValueError), ({"first_parent": -1}, lk.LookatError)):
        with pytest.raises(error):
            select(**kw)


def test_numbers_beyond_32_bits_are_refused(lk):  # noqa: F811
    s = serving_case(lk, torch.float16)
    for big in (2 ** 32, 2 ** 32 + 1, -2 ** 32):
        with pytest.raises(ValueError, match="num_splits"):
            lk.lookat_attend_pages_chunk(s["q"], s["books"], s["pool"], s["table"], s["lengths"], 0.1, num_splits=big)
        for name in ("first", "recent"):
            with pytest.raises(ValueError, match=name):
                lk.lookat_pages_evict(s["pool"], s["table"], s["lengths"], s["weights"], s["keep"], s["out"], **{name: big})
        for name in ("n", "beams", "first_parent"):
            with pytest.raises(ValueError, match=name):
                lk.lookat_beam_select(s["logits"], s["scores"], **{"beams": 3, "n": 5, name: big})
