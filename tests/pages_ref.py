"""The paged 8-bit cache in plain numpy, 64 bits: what the GPU tests compare with.  Shares nothing with the library."""
import math

import numpy as np

LOW, HIGH = -40, 40


def _e4m3_table():
    """The 256 numbers of the 8-bit floating type (sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7f and 0xff are NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.ldexp(m / 8, -6) if e == 0 else math.ldexp(1 + m / 8, e - 7)
        x = math.nan if (c & 127) == 127 else x
        out[c] = -x if c & 128 else x
    return out


E4M3 = _e4m3_table()


def most(kind):
    return 127.0 if kind == "int8" else 448.0


def to_bytes(x, kind):
    """Numbers -> stored bytes (uint8): to nearest, ties to even, larger ones to the largest, NaN to 0."""
    x = np.where(np.isnan(x), 0.0, np.asarray(x, dtype=np.float64))
    x = np.clip(x, -most(kind), most(kind))
    if kind == "int8":
        return np.rint(x).astype(np.int8).view(np.uint8)
    grid = E4M3[:127]                                   # ascending, codes 0..126
    a = np.abs(x)
    hi = np.searchsorted(grid, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    up, down = grid[hi] - a, a - grid[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def from_bytes(b, kind):
    return b.view(np.int8).astype(np.float64) if kind == "int8" else E4M3[b]


def exponent(top, kind):
    """Least e in [LOW, HIGH] with top <= most * 2^e."""
    if not top > 0:
        return LOW
    if math.isinf(top):
        return HIGH
    e = math.frexp(top / most(kind))[1] - 1             # 2^e <= top / most, but for rounding of the quotient
    while top > math.ldexp(most(kind), e):
        e += 1
    while top <= math.ldexp(most(kind), e - 1):
        e -= 1
    return min(max(e, LOW), HIGH)


class Cache:
    """A pool (arrays as on the device, values as bytes) with the operations on it."""

    def __init__(self, codes, values, exponents, kind):
        self.codes, self.values, self.exponents, self.kind = codes.copy(), values.copy(), exponents.copy(), kind
        self.P, self.H, self.page, self.m = codes.shape
        self.d_k = values.shape[3]

    def row(self, i, h, t):
        """A token's stored bytes [d_k] (a view)."""
        return self.values[i, h, t // 8, :, t % 8]

    def write(self, codes, values, table, lengths, counts=None):
        B, H, N, _ = codes.shape
        W = table.shape[1]
        for b in range(B):
            length = max(0, int(lengths[b]))
            count = max(0, N if counts is None else int(counts[b]))
            first = length - count
            new = {}                                    # page slot -> [(token in page, row)]
            for n in range(min(count, N)):
                pos = first + n
                if 0 <= pos < W * self.page:
                    new.setdefault(pos // self.page, []).append((pos % self.page, n))
            begin = max(first, 0)
            for slot, tokens in new.items():
                i = int(table[b, slot])
                if not 0 <= i < self.P:
                    continue
                kept = range(max(0, begin - slot * self.page))
                for h in range(H):
                    v = np.stack([values[b, h, n].astype(np.float64) for _, n in tokens])
                    e = exponent(float(np.nanmax(np.abs(np.where(np.isnan(v), 0, v)))), self.kind)
                    was = int(self.exponents[i, h])
                    if kept:
                        e = max(e, was)
                        for t in kept:
                            if e != was:
                                self.row(i, h, t)[:] = to_bytes(from_bytes(self.row(i, h, t), self.kind) * 2.0 ** (was - e), self.kind)
                    self.exponents[i, h] = e
                    for t, n in tokens:
                        self.row(i, h, t)[:] = to_bytes(values[b, h, n].astype(np.float64) * 2.0 ** -e, self.kind)
                        self.codes[i, h, t] = codes[b, h, n]

    def tokens(self, table_row, length, exponents=False):
        """Codes [H, n, m] and values [H, n, d_k] of the tokens that can be reached (and their exponents [H, n])."""
        c, v, e = [], [], []
        for t in range(min(max(0, length), len(table_row) * self.page)):
            i = int(table_row[t // self.page])
            if 0 <= i < self.P:
                c.append(self.codes[i, :, t % self.page])
                e.append(self.exponents[i].astype(np.float64))
                v.append(from_bytes(self.values[i, :, t % self.page // 8, :, t % 8], self.kind) * 2.0 ** e[-1][:, None])
        if not c:
            c, v, e = np.zeros((0, self.H, self.m), np.uint8), np.zeros((0, self.H, self.d_k)), np.zeros((0, self.H))
        got = np.stack(c, 1) if len(c) else c.transpose(1, 0, 2), np.stack(v, 1) if len(v) else v.transpose(1, 0, 2)
        return (*got, np.stack(e, 1) if len(e) else e.T) if exponents else got

    def attend(self, lut, table, lengths, scale):
        """(out [B, H*g, d_k], bound [B, H*g, d_k] on what fp32 arithmetic may be off by).

        The bound, with u = 2^-24: a logit (log2 units) is a sum of m scaled table entries and an exponent, off by at most
        d = (m + 3) u (sum |entries| + |e| + |reference|); its weight by d ln 2 + 2^-21 of itself (exponential unit, two fp16 terms), numerator
        and denominator both: twice that of sum p |v|.  Sums of n terms in fp32, in pieces of 32: 4 sqrt(n + 64) u of the same sum.
        Last, the two fp16 terms end where fp16 does: a weight's second term is rounded to a multiple of 2^-24, off by 2^-25 at most, however
        small the weight is.  Weights are w = 2^(y - R + 7), y = logit + e, and R is never above max y: the token of the largest y has w >= 2^7, so
        the denominator sum w 2^-e is 2^(7 - e) of that token or more, and the numerator sum w q is off by 2^-25 sum |q| at most:
        2^-32 2^e sum |q| together, e being that token's exponent (and 1.01 times that for the logits' own roundings in max y)."""
        B, Hq = lut.shape[:2]
        g = Hq // self.H
        out, bound = np.zeros((B, Hq, self.d_k)), np.zeros((B, Hq, self.d_k))
        for b in range(B):
            codes, v, e = self.tokens(table[b], int(lengths[b]), True)
            n = codes.shape[1]
            if n == 0:
                continue
            for hq in range(Hq):
                h = hq // g
                entries = np.stack([lut[b, hq, i].astype(np.float64)[codes[h, :, i]] for i in range(self.m)])
                x = entries.sum(0) * scale
                p = np.exp(x - x.max())
                p /= p.sum()
                out[b, hq] = p @ v[h]
                size = np.abs(entries).sum(0).max() * abs(scale) * 1.4427 + 64
                u = 2.0 ** -24
                rel = 2 * ((self.m + 3) * u * 2 * size * 0.6932 + 2.0 ** -21) + 4 * math.sqrt(n + 64) * u
                top = float(e[h, np.argmax(x / math.log(2) + e[h])])
                floor = 1.01 * 2.0 ** (top - 32) * np.abs(v[h] * 2.0 ** -e[h][:, None]).sum(0)
                bound[b, hq] = rel * (p @ np.abs(v[h])) + floor
        return out, bound


class Books:
    """Tables, lengths and counts."""

    def __init__(self, table, lengths, refs, page):
        self.table, self.lengths, self.refs, self.page = table.copy(), lengths.copy(), refs.copy(), page
        self.S, self.W = table.shape

    def held(self, s):
        return -(-min(max(0, int(self.lengths[s])), self.W * self.page) // self.page)

    def free(self, slots):
        for s in slots:
            if not 0 <= s < self.S:
                continue
            for w in range(self.held(s)):
                i = self.table[s, w]
                if 0 <= i < len(self.refs):
                    self.refs[i] -= 1
                self.table[s, w] = -1
            self.lengths[s] = 0

    def fork(self, src, dst):
        was = self.lengths.copy()
        for i, (a, b) in enumerate(zip(src, dst)):
            if not (0 <= a < self.S and 0 <= b < self.S) or a in dst or b in list(dst[:i]) or was[b] > 0 or was[a] <= 0:
                continue
            n = self.held(a)
            self.table[b, :n] = self.table[a, :n]
            self.lengths[b] = self.lengths[a]
            for x in self.table[a, :n]:
                if 0 <= x < len(self.refs):
                    self.refs[x] += 1

    def reserve(self, new_lengths, cache=None):
        need = []                                       # (slot, entry, page to copy or None)
        count = over = 0
        for s in range(self.S):
            has, want = max(0, int(self.lengths[s])), int(new_lengths[s])
            if want <= has:
                continue
            mine = []
            if has % self.page and has // self.page < self.W:
                i = self.table[s, has // self.page]
                if 0 <= i < len(self.refs) and self.refs[i] > 1:
                    mine.append((s, has // self.page, int(i)))
            first, last = -(-has // self.page), -(-want // self.page)
            count += len(mine) + last - first
            if mine or last > first:
                over += max(0, last - self.W)
            need += mine + [(s, w, None) for w in range(first, min(last, self.W))]
        free = [i for i in range(len(self.refs)) if self.refs[i] <= 0]
        missing = max(0, count - len(free)) + over
        if missing:
            return missing
        for (s, w, old), i in zip(need, free):
            if old is not None:
                self.refs[old] -= 1
                if cache is not None:
                    for x in (cache.codes, cache.values, cache.exponents):
                        x[i] = x[old]
            self.table[s, w] = i
            self.refs[i] = 1
        for s in range(self.S):
            if int(new_lengths[s]) > max(0, int(self.lengths[s])):
                self.lengths[s] = new_lengths[s]
        return 0

    def compact(self, cache=None):
        """New (table, refs, live); the cache's pages move in place."""
        n = int((self.refs > 0).sum())
        holes = [i for i in range(n) if self.refs[i] <= 0]
        movers = [i for i in range(n, len(self.refs)) if self.refs[i] > 0]
        to = dict(zip(movers, holes))
        refs = np.zeros_like(self.refs)
        for i in range(len(self.refs)):
            if self.refs[i] > 0:
                refs[to.get(i, i)] = self.refs[i]
        table = np.full_like(self.table, -1)
        for s in range(self.S):
            for w in range(self.held(s)):
                i = int(self.table[s, w])
                table[s, w] = to.get(i, i) if 0 <= i < len(self.refs) and self.refs[i] > 0 else -1
        if cache is not None:
            for a, b in to.items():
                for x in (cache.codes, cache.values, cache.exponents):
                    x[b] = x[a]
        return table, refs, n
