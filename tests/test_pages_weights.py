"""What a softmax weight of the paged attention has to be worth: a bound close enough to tell two fp16 terms from one.  The part that needs
no GPU: inputs, the result in 64 bits, the bound, and that weights of one term would miss it (by 30 to 100 times)."""
import math

import numpy as np
import pytest

import pages_ref as pr

U = 2.0 ** -24
LENGTHS = [1, 2, 3, 5, 9, 17, 33, 64]                    # (one tile each)
FORMS = [(1, 64, 2), (2, 64, 8), (1, 128, 16), (4, 64, 4), (2, 128, 16), (8, 128, 8), (4, 128, 2), (8, 64, 16)]


def weights_case(group, d_k, m, kind):
    """A cache with every exponent 0, tables whose scores (base 2) span less than ten: no weight is near the end of fp16."""
    rng = np.random.default_rng(100 * group + d_k + m)
    H, page = 2, 64
    v = rng.standard_normal((len(LENGTHS), H, page // 8, d_k, 8)) * (40 if kind == "int8" else 120)
    c = pr.Cache(rng.integers(0, 256, (len(LENGTHS), H, page, m), dtype=np.uint8), pr.to_bytes(v, kind), np.zeros((len(LENGTHS), H), np.int8), kind)
    lut = (rng.standard_normal((len(LENGTHS), H * group, m, 256)) * 0.8 / math.sqrt(m)).clip(-3 / m, 3 / m).astype(np.float32)
    return c, np.arange(len(LENGTHS), dtype=np.int32)[:, None], lut


def weights_reference(c, table, lut, terms=None):
    """(result [B, H*g, d_k], bound); with `terms` the result if the numerator's weights were sums of so many fp16 numbers.

    At scale 1 a score in base 2 is a sum of m products lut * log2(e).  The constant and the product are rounded (2 u of the product), the sum m
    times (u of S, the sum of the products' sizes), the reference's offset of 7 and the difference to it twice (u of 2 S + 7 each): off by
    d = u ((m + 6) S + 14) at most.  The weight: d ln 2 and the exponential's last bit (2 u), in numerator and denominator; its two fp16 terms: the first
    leaves 2^-11 of the weight, the second 2^-11 of that.  n tokens are added up in fp32 in the numerator (both terms) and in the denominator,
    then eight wavefronts' sums, a quotient and a product: 3 n + 16 roundings."""
    B, Hq = lut.shape[:2]
    out, bound = np.zeros((B, Hq, c.d_k)), np.zeros((B, Hq, c.d_k))
    for b in range(B):
        codes, v = c.tokens(table[b], LENGTHS[b])
        n = LENGTHS[b]
        for hq in range(Hq):
            h = hq // (Hq // c.H)
            entries = np.stack([lut[b, hq, i].astype(np.float64)[codes[h, :, i]] for i in range(c.m)]) / math.log(2)
            y = entries.sum(0)
            assert y.max() - y.min() < 10
            w = 2.0 ** (y - y.max() + 7)
            used, left = np.zeros_like(w), w.copy()
            for _ in range(terms or 0):
                used += left.astype(np.float16)
                left = w - used
            out[b, hq] = (w if terms is None else used) @ v[h] / w.sum()
            size = np.abs(entries).sum(0).max()
            d = U * ((c.m + 6) * size + 14)
            rel = 2 * (d * math.log(2) + 2 * U) + 2.0 ** -22 + (3 * n + 16) * U
            bound[b, hq] = rel * (w @ np.abs(v[h])) / w.sum()
    return out, bound


@pytest.mark.parametrize("kind", ["int8", "float8"])
@pytest.mark.parametrize("group,d_k,m", FORMS)
def test_the_bound_tells_one_term_from_two(group, d_k, m, kind):
    c, table, lut = weights_case(group, d_k, m, kind)
    ref, bound = weights_reference(c, table, lut)
    for terms, low, high in ((1, 8, math.inf), (2, 0, 0.1)):
        off = np.abs(weights_reference(c, table, lut, terms)[0] - ref)
        assert low <= np.max(off / np.maximum(bound, 1e-30)) <= high, (terms, np.max(off / np.maximum(bound, 1e-30)))
