"""Beam search's selection against 64 bits: parents and tokens exactly (cases without near ties between beams), scores to fp32's rounding."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lk():
    import paper_2601_10155_amd as pkg
    pkg.load_library()
    return pkg


def reference(logits, scores, beams, n, first_parent=0):
    """(scores fp64, parents, tokens, the least distance between candidates of different beams that the choice depends on)."""
    R, V = logits.shape
    Q = R // beams
    x = logits.astype(np.float64)
    s = np.full((Q, n), -np.inf)
    parents, tokens, near = np.full((Q, n), -1), np.full((Q, n), -1), np.inf
    for q in range(Q):
        found = []
        for r in range(q * beams, (q + 1) * beams):
            row, base = x[r], float(scores[r])
            if not np.isfinite(base) or np.isnan(row).any() or np.isposinf(row).any() or not np.isfinite(row).any():
                continue
            top = row.max()
            lse = top + math.log(np.exp(row - top).sum())
            order = np.lexsort((np.arange(V), -row))[:n + 1]
            found += [(base + row[t] - lse, r, int(t)) for t in order if np.isfinite(row[t])]
        # (within a row the scores differ as the logits do, also where 64 bits do not hold the difference: 1 beside 3.4e38)
        found.sort(key=lambda c: (-c[0], c[1], -x[c[1], c[2]], c[2]))
        for a, b in zip(found[:n], found[1:n + 1]):
            if a[1] != b[1] and a[0] != b[0]:
                near = min(near, a[0] - b[0])
        for i, (v, r, t) in enumerate(found[:n]):
            s[q, i], parents[q, i], tokens[q, i] = v, first_parent + r, t
    return s, parents, tokens, near


def check(lk, logits, scores, beams, n, device_logits=None, **kw):
    want = reference(logits, scores, beams, n, kw.get("first_parent", 0))
    # (a row's sum is good to 2^-22 of itself: closer candidates of different beams would not be decided)
    assert want[3] > 2.0 ** -20, "the inputs have a near tie"
    x = torch.from_numpy(logits).cuda() if device_logits is None else device_logits
    got = lk.lookat_beam_select(x, torch.from_numpy(scores).cuda(), beams, n, **kw)
    s, parents, tokens = (t.cpu().numpy() for t in got)
    assert np.array_equal(parents, want[1]), np.argwhere(parents != want[1])[:4]
    assert np.array_equal(tokens, want[2]), np.argwhere(tokens != want[2])[:4]
    assert np.array_equal(np.isneginf(s), np.isneginf(want[0]))
    ok = np.isfinite(want[0])
    # the sum's relative error and the rounding of the score
    assert np.all(np.abs(s[ok] - want[0][ok]) <= 2.0 ** -22 + 2.0 ** -24 * np.abs(want[0][ok]))


@pytest.mark.parametrize("dtype", ["float16", "float32"])
@pytest.mark.parametrize("Q,beams,V,n", [(1, 1, 1, 1), (1, 4, 50257, 8), (3, 2, 100, 64), (2, 5, 511, 7), (2, 3, 513, 16), (5, 1, 2049, 64), (2, 8, 20000, 33),
                                         (1, 16, 4096, 64), (40, 4, 1000, 3), (1, 300, 37, 10), (16, 8, 32001, 16)])
def test_select(lk, Q, beams, V, n, dtype):
    rng = np.random.default_rng(Q + beams + V + n)
    logits = (3 * rng.standard_normal((Q * beams, V))).astype(dtype)
    scores = (-10 * rng.random(Q * beams)).astype(np.float32)
    check(lk, logits, scores, beams, n, first_parent=Q * beams)


@pytest.mark.parametrize("dtype", ["float16", "float32"])
def test_ties(lk, dtype):
    """Constant rows, rows of a few values, equal beams: the lowest row and token; more equal logits than a list holds."""
    rng = np.random.default_rng(1)
    V, n = 9001, 64
    rows = [np.zeros(V), rng.integers(0, 2, V) * 2.0, np.where(rng.random(V) < 0.002, 5.0, 1.0), np.where(np.arange(V) > 8000, 1.0, 0.9990234375),
            rng.choice([0.0, -0.0], V), np.arange(V) % 100]
    for row in rows:
        x = np.stack([row, row, row + 1]).astype(dtype)
        for scores in ([0, 0, 0], [-1, -1, -1], [-math.inf, -2, -2]):
            check(lk, x, np.array(scores, np.float32), 3, n)
            check(lk, x, np.array(scores, np.float32), 1, 5)


def test_masks_and_values_that_are_not_finite(lk):
    rng = np.random.default_rng(2)
    V, n = 5000, 20
    x = (2 * rng.standard_normal((12, V))).astype(np.float32)
    scores = (-5 * rng.random(12)).astype(np.float32)
    x[0] = -math.inf                                   # nothing can be chosen
    x[1, 10:] = -math.inf                              # ten tokens
    x[2, 4321] = math.nan
    x[3, 77] = math.inf
    x[4, : V // 2] = -math.inf
    scores[5] = -math.inf
    scores[6] = math.nan
    scores[7] = math.inf
    x[8] = -3.4e38                                     # the type's lowest value
    x[9] *= 1e30
    x[10] = math.nan
    x[11, 0] = 3.4e38
    check(lk, x, scores, 12, n)
    for beams in (1, 2, 3, 4):
        check(lk, x, scores, beams, n)
    half = np.clip(x, -65504, 65504).astype(np.float16)
    half[1, 10:] = -math.inf
    check(lk, half, scores, 2, n)


@pytest.mark.parametrize("Q,beams,V,n", [(1, 2, 200001, 5), (1, 5, 300000, 9), (2, 17, 3000, 30), (1, 1024, 1025, 12), (3, 6, 1024, 63)])
def test_many_parts_and_many_beams(lk, Q, beams, V, n):
    """More parts of a row than its lanes hold, rows that do not fill the last wavefront; a row without tokens and one of NaN among them."""
    rng = np.random.default_rng(V)
    logits = (3 * rng.standard_normal((Q * beams, V))).astype(np.float32)
    scores = (-4 * rng.random(Q * beams)).astype(np.float32)
    if beams > 2:
        logits[1] = -math.inf
        logits[Q * beams - 1, V - 1] = math.nan
        logits[2, : V - 3] = -math.inf
    check(lk, logits, scores, beams, n)


def test_peaked_and_flat_rows(lk):
    """Sums that one logit makes, sums that all make, logits and scores of large size."""
    rng = np.random.default_rng(3)
    V = 131072
    x = np.stack([rng.standard_normal(V) * 0.01, np.where(np.arange(V) == 999, 30.0, rng.standard_normal(V)), rng.standard_normal(V) * 50 + 1000,
                  rng.standard_normal(V) - 500]).astype(np.float32)
    check(lk, x, np.array([-1, -2.5, -0.25, -3], np.float32), 4, 16)
    check(lk, x, np.array([-1e6, -1, -1, -1], np.float32), 1, 16)


def test_strides_alignment_and_outputs(lk):
    """Rows inside a wider tensor at every alignment of the type, outputs and workspace given, another stream."""
    rng = np.random.default_rng(4)
    for dtype in ("float16", "float32"):
        wide = (3 * rng.standard_normal((6, 7013))).astype(dtype)
        d = torch.from_numpy(wide).cuda()
        scores = (-3 * rng.random(6)).astype(np.float32)
        for a in range(4):
            check(lk, wide[:, a:a + 7001], scores, 3, 9, device_logits=d[:, a:a + 7001])
        ws = torch.empty(lk.beam_select_workspace_bytes(2, 3, 7001, 9), dtype=torch.uint8, device="cuda")
        s, p, t = torch.empty((2, 9), device="cuda"), torch.empty((2, 9), dtype=torch.int32, device="cuda"), torch.empty((2, 9), dtype=torch.int32, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = lk.lookat_beam_select(d[:, :7001], torch.from_numpy(scores).cuda(), 3, 9, scores_out=s, parents=p, tokens=t, workspace=ws)
        side.synchronize()
        assert got[0] is s and got[1] is p and got[2] is t
        want = reference(wide[:, :7001], scores, 3, 9)
        assert np.array_equal(p.cpu().numpy(), want[1]) and np.array_equal(t.cpu().numpy(), want[2])


def test_graph(lk):
    x, scores = torch.randn((8, 30000), device="cuda"), -torch.rand(8, device="cuda")
    ws = torch.empty(lk.beam_select_workspace_bytes(2, 4, 30000, 8), dtype=torch.uint8, device="cuda")
    out = lk.lookat_beam_select(x, scores, 4, 8, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lk.lookat_beam_select(x, scores, 4, 8, scores_out=out[0], parents=out[1], tokens=out[2], workspace=ws)
    for _ in range(3):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        eager = lk.lookat_beam_select(x, scores, 4, 8)
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
