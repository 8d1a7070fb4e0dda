// Attention of a chunk of new tokens over the paged cache: every row sees the tokens up to its own position.
//
//   s = q . k^,  k^ = (C_0[code_0], C_1[code_1], ...),   out = sum_{l <= p} softmax_l(scale s) q_l 2^e(l)
//
// With many rows per cached token the sum over table entries is a dense product with the keys' centroids, and belongs on the matrix cores
// (v_mfma_f32_32x32x16_f16), as does the weighted sum:
//   * S^T = K^ Q^T: a wavefront owns 32 rows (columns of S^T).  Centroids enter as two fp16 terms of 2^s w (22 bits; s one power of two per
//     head, which brings the head's largest centroid entry to 2^14), fp16 queries exactly, fp32 queries as two terms of their own power of
//     two (the product of the two small terms, 2^-22, is dropped).
//   * a lane then holds 16 or 32 scores of ONE row: running reference and sum need no exchange but with the lane that holds the row's other keys.
//     Reference and page exponents as in attention of one token: y = scale log2(e) s + e, w = 2^(y - R).
//   * O^T = V^T P^T: keys are dealt to the rows of K^ (bits 2 and 3 of a row's number exchanged) such that the eight weights that a lane holds
//     of an operand belong to eight consecutive tokens: the weights, as two fp16 terms, are the operand where they are, and the values' operand
//     is eight consecutive stored bytes, as the page holds them.
// The centroids are split once per call by a small kernel, into the workspace (or by every workgroup, see below).  A workgroup of NW wavefronts (32 NW
// rows of one key/value head, query heads of a group side by side) fetches the centroids of KEYS keys by code into LDS, two buffers of as many keys in
// turn; their ids, codes, centroids and values are requested four, three, two and one tiles ahead.
#include "pages_values.h"

namespace lookat {

typedef float v16f __attribute__((ext_vector_type(16)));

struct ChunkArgs {
    const void *q;
    const float *codebooks;
    const char *books;                    // [H, m, 256, 2, d_sub] fp16: both terms of a centroid
    const float *unscale;                 // [H] 2^-s
    const int32_t *table, *lengths, *counts;
    float *part, *out;
    int64_t q_b, q_h, q_n, table_stride;  // strides in elements
    int32_t W, N, group, dsub_log2;
    int32_t tiles, splits, units;         // row tiles of a (sequence, head), ranges, (sequence, head) pairs
    int32_t whole, left, per_die;         // workgroups of a die for whole rounds of units, of all dies for the others, of one die for the others
    float scale_log2e;
};

constexpr int kBookTop = 14;              // the largest centroid entry comes between 2^14 and 2^15
constexpr int kPartPad = 4;               // a partial row: d_k sums, reference, sum, two unused

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// The power of two that brings x (its magnitude's bits) between 2^kBookTop and twice that, as far as fp32 goes.
__device__ __forceinline__ int lift_of(uint32_t bits)
{
    const int s = bits ? kBookTop + 127 - (int)(bits >> 23) : 0;
    return s > 126 ? 126 : s < -126 ? -126 : s;
}

// The largest magnitude of four coordinates and those before, as bits.  (Entries that are not finite do not count: no token may have them.)
__device__ __forceinline__ uint32_t finite_top(const v4u &x, uint32_t top)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t a = x[k] & 0x7fffffffu;
        top = a < 0x7f800000u && a > top ? a : top;
    }
    return top;
}
// Coordinates 4 u .. 4 u + 3 of a head's [m, 256, d_sub], times f, as two fp16 terms to their places in its [m, 256, 2, d_sub].
__device__ __forceinline__ void split_book(const v4u &x, float f, int u, int dsub_log2, char *book)
{
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float a = __uint_as_float(x[2 * k]) * f, b = __uint_as_float(x[2 * k + 1]) * f;
        const v2h hh = {(_Float16)a, (_Float16)b};
        const v2h ll = {(_Float16)(a - (float)hh.x), (_Float16)(b - (float)hh.y)};
        hi[k] = __builtin_bit_cast(uint32_t, hh);
        lo[k] = __builtin_bit_cast(uint32_t, ll);
    }
    const int first = 4 * u, centroid = first >> dsub_log2, j = first & ((1 << dsub_log2) - 1);
    char *to = book + ((((centroid << dsub_log2) * 2) + j) << 1);
    *reinterpret_cast<v2u *>(to) = (v2u){hi[0], hi[1]};
    *reinterpret_cast<v2u *>(to + (2 << dsub_log2)) = (v2u){lo[0], lo[1]};
}

constexpr int kBookThreads = 512, kBookParts = 8;
// grid: (part, head)
__global__ __launch_bounds__(kBookThreads) void chunk_books_kernel(const float *codebooks, char *books, float *unscale, int d_k, int dsub_log2)
{
    __shared__ uint32_t tops[kBookThreads / kWave];
    const int h = blockIdx.y, tid = threadIdx.x, units = kCentroids * d_k / 4;        // 4 coordinates each
    const v4u *src = reinterpret_cast<const v4u *>(codebooks) + (int64_t)h * units;
    uint32_t top = 0;
    for (int u = tid; u < units; u += kBookThreads) {
        const v4u x = src[u];
        top = finite_top(x, top);
    }
    top = __float_as_uint(wave_max(__uint_as_float(top)));
    if ((tid & (kWave - 1)) == 0)
        tops[tid / kWave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBookThreads / kWave; ++w)
        top = tops[w] > top ? tops[w] : top;
    const int s = lift_of(top);
    if (blockIdx.x == 0 && tid == 0)
        unscale[h] = power_of_two(-s);
    const float f = power_of_two(s);
    const int per = units / kBookParts;
    for (int u = blockIdx.x * per + tid; u < (int)(blockIdx.x + 1) * per; u += kBookThreads)
        split_book(src[u], f, u, dsub_log2, books + (int64_t)h * kCentroids * d_k * 4);
}

// What a tile of rows of one sequence sees.
struct ChunkSpan {
    int64_t first;        // position of row 0
    int length, count;    // tokens in reach, rows that count
};
__device__ __forceinline__ ChunkSpan chunk_span(const ChunkArgs &a, int b, int page_log2)
{
    ChunkSpan s;
    const int64_t given = a.lengths[b] < 0 ? 0 : a.lengths[b];
    int count = a.counts ? a.counts[b] : a.N;
    count = count < 0 ? 0 : count;
    s.first = given - count;
    s.count = count < a.N ? count : a.N;
    s.length = clamp_length((int)given, a.W, page_log2);
    return s;
}
__device__ __forceinline__ int seen_of(const ChunkSpan &s, int n)
{
    const int64_t x = s.first + n + 1;
    return x < 0 ? 0 : x < s.length ? (int)x : s.length;
}
// Key tiles of a row tile's range: [t0, t1), and how many ranges have any.
struct KeyRange {
    int end, t0, t1, ranges;
};
template <int KEYS>
__device__ __forceinline__ KeyRange key_range(const ChunkSpan &s, int last_row, int splits, int split)
{
    KeyRange r;
    r.end = seen_of(s, last_row);
    const int tiles = (r.end + KEYS - 1) / KEYS, per = (tiles + splits - 1) / splits;
    r.ranges = per ? (tiles + per - 1) / per : 1;
    r.t0 = split * per;
    r.t1 = tiles - r.t0 < per ? tiles : r.t0 + per;
    return r;
}

// Which work a workgroup has.  Units (sequence, head) are dealt to the dies in turn, all workgroups of a unit on one die (they read the same keys,
// values and centroids); the units that eight dies do not divide are dealt by workgroups.  The last rows come first: they see most.  A die's
// workgroups go round its 32 compute units, and every second round turns back, so that no compute unit gets the longest of each (us a call, without the turn /
// so: prompts of 96 heads x 400 to 1000 fp32 rows 48.0 / 47.0, 64 x 1000 fp16 rows 41.6 / 40.6, but 96 x 400 to 1000 fp16 40.8 / 41.3).
struct Place {
    int unit, tile, split;
    bool any;
};
__device__ __forceinline__ Place place_of(const ChunkArgs &a)
{
    constexpr int kRound = 32;
    const int die = (int)(blockIdx.x % kXcds), per_unit = a.tiles * a.splits;
    int nth = (int)(blockIdx.x / kXcds);
    const bool whole = nth < a.whole;
    const int most = whole ? a.whole : a.whole + a.per_die, start = nth - (nth - (whole ? 0 : a.whole)) % kRound;
    const int size = most - start < kRound ? most - start : kRound;
    if ((start / kRound) & 1)
        nth = start + size - 1 - (nth - start);
    Place x;
    int level;
    if (whole) {
        const int units = a.whole / per_unit;
        level = nth / units;
        x.unit = (nth - level * units) * kXcds + die;
        x.any = true;
    } else {
        const int index = (nth - a.whole) * kXcds + die, units = a.left / per_unit;
        x.any = index < a.left;
        level = units ? index / units : 0;
        x.unit = a.units - units + index - level * units;
    }
    x.tile = a.tiles - 1 - level / a.splits;
    x.split = level % a.splits;
    return x;
}

// What the first fp16 term of each of a pair of weights left, as a pair: (w0 - h.x, w1 - h.y), each rounded once.
__device__ __forceinline__ uint32_t left_of(float w0, float w1, uint32_t h)
{
    uint32_t r;
    asm("v_fma_mixlo_f16 %0, %1, 1.0, -%2 op_sel_hi:[0,0,1]" : "=v"(r) : "v"(w0), "v"(h));
    asm("v_fma_mixhi_f16 %0, %1, 1.0, -%2 op_sel:[0,0,1] op_sel_hi:[0,0,1]" : "+v"(r) : "v"(w1), "v"(h));
    return r;
}

// A stored NaN (e4m3 alone has one) belongs to the rows that see its token; for the others it would be multiplied by a weight of zero.  So in the
// tiles whose tokens not all rows see zeros take the NaNs' places, and where there was one, what the rows that see it have is made NaN behind the
// results' stores: without a NaN those tiles alone have a few instructions more.
// Zeros in the places of NaNs (0x7f, 0xff); `any` is not zero if there was one.
__device__ __forceinline__ void drop_nans(v4u &x, uint32_t &any)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t n = ((x[k] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
        x[k] &= ~((n << 1) - (n >> 7));
        any |= n;
    }
}
// Whether one of the tokens [first, last) has a NaN at coordinate d.
template <int DK>
__device__ __forceinline__ bool sees_nan(const uint8_t *head_values, uint32_t value_step, const int32_t *row, int pages, int page_log2, int first, int last, int d)
{
#pragma unroll 1
    for (int l = first; l < last; ++l) {
        const int id = row[l >> page_log2], t = l & ((1 << page_log2) - 1);
        if ((uint32_t)id < (uint32_t)pages && (head_values[(uint64_t)(uint32_t)id * value_step + (uint32_t)((t & ~7) * DK + d * 8 + (t & 7))] & 0x7f) == 0x7f)
            return true;
    }
    return false;
}

// Wavefronts to a SIMD that the registers have to allow.
constexpr int kChunkWaves = 2;

template <int DK, bool SMALL, bool Q32, bool FP8, int NW, int KEYS>
__global__ __launch_bounds__(NW *kWave, kChunkWaves) void chunk_kernel(PoolArgs p, ChunkArgs a)
{
    constexpr int threads = NW * kWave, CH = DK / 8, STEPS = DK / 16, CB = DK / 32, TQ = 32 * NW;
    constexpr int TPK = threads / KEYS, CPT = CH / TPK;          // threads of a key, 8-coordinate pieces that each of them fetches
    constexpr int KB = KEYS / 32, GROUPS = KEYS / 16;            // blocks of a product, groups of tokens that lie in one page
    constexpr int kPlane = KEYS * DK * 2, kBuffer = 2 * kPlane, kValues = KEYS * DK * 2;
    constexpr int kItems = KEYS / 8 * DK / 2, VPT = (kItems + threads - 1) / threads;    // two coordinates of eight tokens: 16 stored bytes
    static_assert(CH % TPK == 0, "whole pieces for every thread");
    __shared__ __align__(16) char keys_s[2 * kBuffer];           // [buffer][term][key][coordinate]
    __shared__ __align__(16) char values_s[2 * kValues];         // [buffer][octet][coordinate][token]
    __shared__ int ids_s[4][GROUPS], exps_s[4][GROUPS];          // of 16 tokens, by tile modulo 4
    __shared__ int nan_s;                                        // whether drop_nans found one
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, half = lane >> 5, col = lane & 31;
    const Place at_work = place_of(a);
    if (!at_work.any)
        return;
    const int unit = at_work.unit, tile = at_work.tile, split = at_work.split;
    const int b = unit / p.H, h = unit - b * p.H;
    const ChunkSpan span = chunk_span(a, b, p.page_log2);
    const int r0 = tile * TQ, n_first = r0 / a.group;
    if (n_first >= span.count)
        return;
    int n_last = (r0 + TQ - 1) / a.group;
    n_last = n_last < span.count ? n_last : span.count - 1;
    const KeyRange range = key_range<KEYS>(span, n_last, a.splits, split);
    if (split >= range.ranges)
        return;
    const int32_t *row = a.table + b * a.table_stride;
    const int page_mask = (1 << p.page_log2) - 1;
    // bytes from page to page (below 2^27), and this head's part of page 0
    const uint32_t code_step = (uint32_t)(p.H * p.m) << p.page_log2, value_step = (uint32_t)(p.H * DK) << p.page_log2;
    const uint8_t *head_codes = p.codes + ((uint32_t)(h * p.m) << p.page_log2), *head_values = p.values + ((uint32_t)(h * DK) << p.page_log2);
    const int8_t *head_exponents = p.exponents + h;

    // this lane's row
    const int r = r0 + wave * 32 + col, n = r / a.group, hq = h * a.group + r - n * a.group;
    const bool mine = n < span.count;
    const int seen = mine ? seen_of(span, n) : range.end;
    const int seen_by_all = seen_of(span, n_first);
    const int n_at = n < a.N ? n : a.N - 1;

    // ---- the keys of a tile ----
    const int kk = tid / TPK, sub = tid % TPK, last_key = range.end > 0 ? range.end - 1 : 0;
    const int krow = (kk & ~12) | (kk & 4) << 1 | (kk & 8) >> 1;
    // (What is loaded for a later tile is looked at only there: nothing waits for it in this one.)
    auto load_id = [&](int t) -> int {
        const int key = t * KEYS + kk;
        return row[(key < range.end ? key : last_key) >> p.page_log2];
    };
    // the page of this thread's 16 tokens, which lie in one, or -1: none of them is there
    auto page_of = [&](int t, int id) -> int { return t * KEYS + (kk & ~15) < range.end && (uint32_t)id < (uint32_t)p.pages ? id : -1; };
    constexpr int CODES = SMALL ? 2 * CPT : CPT;
    uint32_t codes[CODES];
    int exponent;
    auto load_codes = [&](int t, int raw_id, uint32_t (&codes)[CODES], int &exponent) {
        const int id = page_of(t, raw_id);
        const uint32_t page = id < 0 ? 0 : id;
        const uint8_t *c = head_codes + (uint64_t)page * code_step + (uint32_t)(((t * KEYS + kk) & page_mask) * p.m);
#pragma unroll
        for (int j = 0; j < CPT; ++j) {
            const int chunk = sub + j * TPK;
            if constexpr (SMALL) {
                codes[2 * j] = c[2 * chunk];
                codes[2 * j + 1] = c[2 * chunk + 1];
            } else {
                codes[j] = c[(chunk * 8) >> a.dsub_log2];
            }
        }
        exponent = head_exponents[(uint64_t)page * (uint32_t)p.H];
    };
    v4u piece[CPT][2];
    const char *books = a.books + (int64_t)h * kCentroids * DK * 4;
    auto load_centroids = [&](const uint32_t (&codes)[CODES], v4u (&piece)[CPT][2]) {
#pragma unroll
        for (int j = 0; j < CPT; ++j) {
            const int chunk = sub + j * TPK;
            if constexpr (SMALL) {
                // four coordinates to a centroid: its terms are 16 bytes
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    piece[j][k] = *reinterpret_cast<const v4u *>(books + (((2 * chunk + k) * kCentroids + (int)codes[2 * j + k]) << 4));
            } else {
                const int i = (chunk * 8) >> a.dsub_log2, within = (chunk * 8) & ((1 << a.dsub_log2) - 1);
                const char *at = books + (((i * kCentroids + (int)codes[j]) << a.dsub_log2) * 2 + within) * 2;
                piece[j][0] = *reinterpret_cast<const v4u *>(at);
                piece[j][1] = *reinterpret_cast<const v4u *>(at + (2 << a.dsub_log2));
            }
        }
    };
    auto put_page = [&](int t, int id, int e) {
        if ((kk & 15) == 0 && sub == 0) {
            ids_s[t & 3][kk >> 4] = id;
            exps_s[t & 3][kk >> 4] = id < 0 ? 0 : e;
        }
    };
    auto put_keys = [&](int t, int raw_id, int e, const v4u (&piece)[CPT][2]) {
        const int id = page_of(t, raw_id);
        char *to = keys_s + (t & 1) * kBuffer + krow * (DK * 2);
#pragma unroll
        for (int j = 0; j < CPT; ++j) {
            const int chunk = sub + j * TPK, at = (chunk ^ (krow & (CH - 1))) << 4;
            v4u hi = piece[j][0], lo = piece[j][1];
            if constexpr (SMALL) {
                hi = (v4u){piece[j][0].x, piece[j][0].y, piece[j][1].x, piece[j][1].y};
                lo = (v4u){piece[j][0].z, piece[j][0].w, piece[j][1].z, piece[j][1].w};
            }
            if (id < 0 || t * KEYS + kk >= range.end)     // no token: zeros, whatever the centroids hold
                hi = lo = (v4u){0, 0, 0, 0};
            *reinterpret_cast<v4u *>(to + at) = hi;
            *reinterpret_cast<v4u *>(to + kPlane + at) = lo;
        }
        put_page(t, id, e);
    };
    // ---- the values of a tile ----
    v4u stored[VPT];
    auto load_values = [&](int t) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int item = tid + j * threads;
            if (kItems % threads == 0 || item < kItems) {
                const int octet = item / (DK / 2), pair = item % (DK / 2), id = ids_s[t & 3][octet >> 1];
                stored[j] = *reinterpret_cast<const v4u *>(head_values + (uint64_t)(uint32_t)(id < 0 ? 0 : id) * value_step +
                                                           (uint32_t)(((t * KEYS + 8 * octet) & page_mask) * DK + pair * 16));
            }
        }
    };
    auto put_values = [&](int t) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int item = tid + j * threads;
            if (kItems % threads == 0 || item < kItems) {
                if constexpr (FP8) {
                    // bytes without a token behind them, which may be NaN, and NaNs that not all rows see: zeros in their place
                    if ((t + 1) * KEYS > seen_by_all) {
                        const int m = range.end - t * KEYS - 8 * (item / (DK / 2));
                        const uint32_t lo = m >= 4 ? ~0u : m <= 0 ? 0u : (1u << (8 * m)) - 1;
                        const uint32_t hi = m >= 8 ? ~0u : m <= 4 ? 0u : (1u << (8 * (m - 4))) - 1;
                        stored[j].x &= lo, stored[j].y &= hi;
                        stored[j].z &= lo, stored[j].w &= hi;
                        uint32_t any = 0;
                        drop_nans(stored[j], any);
                        if (any)
                            nan_s = 1;
                    }
                    if (ids_s[t & 3][item / (DK / 2) >> 1] < 0)
                        stored[j] = (v4u){0, 0, 0, 0};
                }
                v8h *to = reinterpret_cast<v8h *>(values_s + (t & 1) * kValues) + 2 * item;
                to[0] = widen<FP8>(stored[j].x, stored[j].y);
                to[1] = widen<FP8>(stored[j].z, stored[j].w);
            }
        }
    };
    int id0 = load_id(range.t0), id1 = load_id(range.t0 + 1), id2 = load_id(range.t0 + 2), id3 = load_id(range.t0 + 3);

    // ---- the rows as operand: coordinates 16 s + 8 half .. + 7 of row `col` ----
    v8h qh[STEPS], ql[Q32 ? STEPS : 1];
    float unscale = a.unscale[h];
    const int64_t q_at = b * a.q_b + hq * a.q_h + n_at * a.q_n + 8 * half;
    if constexpr (!Q32) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            qh[s] = *reinterpret_cast<const v8h *>(static_cast<const _Float16 *>(a.q) + q_at + 16 * s);
    } else {
        const float *src = static_cast<const float *>(a.q) + q_at;
        v4f x[STEPS][2];
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                x[s][k] = *reinterpret_cast<const v4f *>(src + 16 * s + 4 * k);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    top = fmaxf(top, fabsf(x[s][k][e]));
            }
        float u, v;
        lanes_xor32(top, u, v);
        const int lift = lift_of(__float_as_uint(fmaxf(u, v)));
        const float f = power_of_two(lift);
        unscale *= power_of_two(-lift);
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = x[s][e / 4][e % 4] * f;
                qh[s][e] = (_Float16)w;
                ql[s][e] = (_Float16)(w - (float)qh[s][e]);
            }
    }
    // A negative scale turns the rows around, one of NaN makes their scores NaN (fmaxf would pass over it), and a scale of zero becomes fp32's
    // least, so that a score of -inf stays one.
    if (!(a.scale_log2e >= 0.f)) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            qh[s] = a.scale_log2e < 0.f ? -qh[s] : qh[s] * (_Float16)NAN;
            if constexpr (Q32)
                ql[s] = -ql[s];
        }
    }
    const float to_log2 = fmaxf(fabsf(a.scale_log2e * unscale), 1.17549435e-38f);

    v16f acc[CB], s[KB], s_next[KB];
    auto score = [&](int t, v16f (&to)[KB]) {
        const char *from = keys_s + (t & 1) * kBuffer;
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                to[k][i] = 0.f;
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                const char *at = from + (32 * k + col) * (DK * 2) + (((2 * st + half) ^ (col & (CH - 1))) << 4);
                const v8h hi = *reinterpret_cast<const v8h *>(at), lo = *reinterpret_cast<const v8h *>(at + kPlane);
                to[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi, qh[st], to[k], 0, 0, 0);
                to[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lo, qh[st], to[k], 0, 0, 0);
                if constexpr (Q32)
                    to[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi, ql[st], to[k], 0, 0, 0);
            }
    };

    // Two tiles of keys and one of values are staged, the scores of the first are there before the loop.  (What can be requested together is: page
    // ids, then the codes of three tiles and the values, then the centroids of two.)
    put_page(range.t0, page_of(range.t0, id0), 0);
    if (FP8 && tid == 0)
        nan_s = 0;
    __syncthreads();
    load_values(range.t0);
    {
        uint32_t codes0[CODES], codes1[CODES];
        int exponent0, exponent1;
        v4u piece1[CPT][2];
        load_codes(range.t0, id0, codes0, exponent0);
        load_codes(range.t0 + 1, id1, codes1, exponent1);
        load_codes(range.t0 + 2, id2, codes, exponent);
        load_centroids(codes0, piece);
        load_centroids(codes1, piece1);
        put_keys(range.t0, id0, exponent0, piece);
        put_keys(range.t0 + 1, id1, exponent1, piece1);
    }
    put_values(range.t0);
    __syncthreads();
    score(range.t0, s);
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            acc[c][i] = 0.f;
    float ref = kNoReference, z = 0.f;    // the reference less kRefLift
    __syncthreads();

    for (int t = range.t0; t < range.t1; ++t) {
        const int slot = t & 3;
        int ids[GROUPS], exps[GROUPS], all = 0;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            ids[g] = __builtin_amdgcn_readfirstlane(ids_s[slot][g]);
            exps[g] = __builtin_amdgcn_readfirstlane(exps_s[slot][g]);
            all |= ids[g];
        }
        // values of the next tile, centroids of the one behind it, codes of the third, page ids of the fourth
        load_values(t + 1);
        int e2 = exponent;
        asm volatile("" : "+v"(e2));      // (else its load is moved into the branch that stores it, and waited for there)
        load_centroids(codes, piece);
        load_codes(t + 3, id3, codes, exponent);
        const int id4 = load_id(t + 4);

        // score i of block k belongs to token 32 k + 16 (i / 8) + 8 half + i % 8
        if (all < 0 || (t + 1) * KEYS > seen_by_all) {
            const int limit = seen - t * KEYS - 8 * half;
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[k][i] = 32 * k + 16 * (i / 8) + i % 8 < (ids[2 * k + i / 8] < 0 ? -64 : limit) ? s[k][i] : -INFINITY;
        }
        // the largest logit (log2 units, exponent added; to_log2 is above zero)
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            float m = s[g / 2][8 * (g % 2)];
#pragma unroll
            for (int i = 1; i < 8; ++i)
                m = fmaxf(m, s[g / 2][8 * (g % 2) + i]);
            top = fmaxf(top, fmaf(m, to_log2, (float)exps[g]));
        }
        if (__builtin_amdgcn_ballot_w64(top - ref > kRefLift + kRefLag)) {
            float u, w;
            lanes_xor32(top, u, w);
            const float to = fmaxf(ref, fmaxf(u, w) - kRefLift), fix = fast_exp2(ref - to);
            ref = to;
            z *= fix;
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    acc[c][i] *= fix;
        }
        // the next tile's scores, this one's weights and its weighted sum, 16 tokens at a time
        score(t + 1, s_next);
        const v8h *from = reinterpret_cast<const v8h *>(values_s + (t & 1) * kValues) + half * DK + col;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            float sum = 0.f;
            v4u hi, lo;
            const float shift = (float)exps[g] - ref;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w0 = fast_exp2(fmaf(s[g / 2][8 * (g % 2) + 2 * i], to_log2, shift));
                const float w1 = fast_exp2(fmaf(s[g / 2][8 * (g % 2) + 2 * i + 1], to_log2, shift));
                sum += w0;
                sum += w1;
                // (cut, not rounded: the second term takes up what is left all the same)
                hi[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(w0, w1));
                lo[i] = left_of(w0, w1, hi[i]);
            }
            z = fmaf(sum, power_of_two(-exps[g]), z);
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                const v8h x = from[2 * g * DK + 32 * c];
                acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, __builtin_bit_cast(v8h, hi), acc[c], 0, 0, 0);
                acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, __builtin_bit_cast(v8h, lo), acc[c], 0, 0, 0);
            }
        }
        // (these buffers were last read before the barrier that ended the tile before)
        put_keys(t + 2, id2, e2, piece);
        put_values(t + 1);
#pragma unroll
        for (int k = 0; k < KB; ++k)
            s[k] = s_next[k];
        id2 = id3;
        id3 = id4;
        __syncthreads();
    }

    float u, w;
    lanes_xor32(z, u, w);
    z = u + w;
    if (mine) {
        float f = 1.f;
        float *to;
        if (range.ranges == 1) {
            f = z == 0.f ? 0.f : 1.f / z;     // (nothing to sum: zeros; a sum that is NaN stays one)
            to = a.out + ((int64_t)(b * p.H * a.group + hq) * a.N + n) * DK;
        } else {
            to = a.part + (((int64_t)unit * a.tiles + tile) * a.splits + split) * TQ * (DK + kPartPad) + (wave * 32 + col) * (DK + kPartPad);
            if (half == 0)
                *reinterpret_cast<float2 *>(to + DK) = make_float2(ref, z);
        }
        // register i of acc[c] is coordinate 32 c + i % 4 + 8 (i / 4) + 4 half
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const v4f o = {acc[c][i] * f, acc[c][i + 1] * f, acc[c][i + 2] * f, acc[c][i + 3] * f};
                *reinterpret_cast<v4f *>(to + 32 * c + 2 * i + 4 * half) = o;
            }
        if constexpr (FP8)
            if (nan_s) {
                const int first = (seen_by_all / KEYS > range.t0 ? seen_by_all / KEYS : range.t0) * KEYS, last = seen < range.t1 * KEYS ? seen : range.t1 * KEYS;
#pragma unroll 1
                for (int i = 0; i < DK / 2; ++i) {
                    const int d = 8 * (i / 4) + 4 * half + i % 4;
                    if (sees_nan<DK>(head_values, value_step, row, p.pages, p.page_log2, first, last, d))
                        to[d] = NAN;
                }
            }
    }
}

// Few rows (drafted tokens, the ends of prompts), and few heads: 16 RB rows of a (sequence, head) to a workgroup, whose wavefronts take tiles of 32 tokens in
// turn, each for itself, values as in attention of one token, and the wavefronts' results are merged in LDS.  v_mfma_f32_16x16x32_f16: keys are dealt to
// the two blocks of 16 such that a lane's eight scores belong to one octet.
// A workgroup of eight wavefronts splits its head's codebook itself, into LDS (64 or 128 KB), and looks its operands up there; one of two takes them from the
// books in memory.  Looked up in memory by eight wavefronts a tile's operands were 4 KB to 16 KB of scattered 64-byte pieces: us a call, so / from LDS, 16 x 12
// x 8 rows behind 1000 tokens 15.9 / 9.7, 32 x 2 behind 20000, d_k = 128 56.0 / 27.8, 1280 x 2 behind 200 to 2000, d_k = 128 118 / 76.
constexpr int kFewWaves = 8, kBriefWaves = 2, kFewKeys = 32;
__host__ __device__ constexpr bool few_staged(int waves) { return waves == kFewWaves; }
__host__ __device__ constexpr size_t few_lds_bytes(int d_k, int waves) { return (size_t)waves * 16 * (d_k + 4) * 4 + waves * 16 * 8; }

template <int DK, bool SMALL, bool Q32, bool FP8, int RB, int WAVES>
__global__ __launch_bounds__(WAVES *kWave, 2) void chunk_few_kernel(PoolArgs p, ChunkArgs a)
{
    constexpr bool STAGED = few_staged(WAVES);
    constexpr int STEPS = DK / 32, CB = DK / 32, TQ = 16 * RB, ROW = DK + 4;
    __shared__ float tops_s[STAGED ? WAVES : 1];
    __shared__ int nans_s[WAVES];         // whether drop_nans found one
    extern __shared__ __align__(16) char few_s[];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, quad = lane >> 4, col = lane & 15;
    const Place at = place_of(a);
    if (!at.any)
        return;
    const int b = at.unit / p.H, h = at.unit - b * p.H, tile = at.tile, split = at.split;
    const ChunkSpan span = chunk_span(a, b, p.page_log2);
    const int r0 = tile * TQ, n_first = r0 / a.group;
    if (n_first >= span.count)
        return;
    int n_last = (r0 + TQ - 1) / a.group;
    n_last = n_last < span.count ? n_last : span.count - 1;
    const KeyRange range = key_range<kFewKeys>(span, n_last, a.splits, split);
    if (split >= range.ranges)
        return;
    const int32_t *row = a.table + b * a.table_stride;
    const int page_mask = (1 << p.page_log2) - 1;
    // bytes from page to page (below 2^27), and this head's part of page 0
    const uint32_t code_step = (uint32_t)(p.H * p.m) << p.page_log2, value_step = (uint32_t)(p.H * DK) << p.page_log2;
    const uint8_t *head_codes = p.codes + ((uint32_t)(h * p.m) << p.page_log2), *head_values = p.values + ((uint32_t)(h * DK) << p.page_log2);
    const int8_t *head_exponents = p.exponents + h;
    const int seen_by_all = seen_of(span, n_first);

    // a page id of the octet `o` of tile t
    // (as it stands in the table: looked at by page_of, where it is used)
    const int last_key = range.end > 0 ? range.end - 1 : 0;
    auto load_id = [&](int t, int o) -> int {
        const int key = t * kFewKeys + 8 * o;
        return row[(key < range.end ? key : last_key) >> p.page_log2];
    };
    auto page_of = [&](int t, int o, int id) -> int { return t * kFewKeys + 8 * o < range.end && (uint32_t)id < (uint32_t)p.pages ? id : -1; };
    // keys: row `col` of block k is token 8 (col / 4) + 4 k + col % 4
    const int my_octet = col >> 2, my_key = 8 * my_octet + (col & 3);
    constexpr int CODES = SMALL ? 2 : 1;
    uint32_t codes[2][STEPS][CODES];
    auto load_codes = [&](int t, int raw_id) {
        const int id = page_of(t, my_octet, raw_id);
        const uint8_t *c = head_codes + (uint64_t)(uint32_t)(id < 0 ? 0 : id) * code_step + (uint32_t)(((t * kFewKeys + my_key) & page_mask) * p.m);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
                if constexpr (SMALL) {
                    codes[k][s][0] = c[4 * k * p.m + 2 * (4 * s + quad)];
                    codes[k][s][1] = c[4 * k * p.m + 2 * (4 * s + quad) + 1];
                } else {
                    codes[k][s][0] = c[4 * k * p.m + ((8 * (4 * s + quad)) >> a.dsub_log2)];
                }
    };
    v4u piece[2][STEPS][2];
    const char *books = STAGED ? few_s : a.books + (int64_t)h * kCentroids * DK * 4;
    auto load_centroids = [&]() {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int chunk = 4 * s + quad;
                if constexpr (SMALL) {
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        piece[k][s][e] = *reinterpret_cast<const v4u *>(books + (((2 * chunk + e) * kCentroids + (int)codes[k][s][e]) << 4));
                } else {
                    const int i = (chunk * 8) >> a.dsub_log2, within = (chunk * 8) & ((1 << a.dsub_log2) - 1);
                    const char *from = books + (((i * kCentroids + (int)codes[k][s][0]) << a.dsub_log2) * 2 + within) * 2;
                    piece[k][s][0] = *reinterpret_cast<const v4u *>(from);
                    piece[k][s][1] = *reinterpret_cast<const v4u *>(from + (2 << a.dsub_log2));
                }
            }
    };

    int t = range.t0 + wave;
    int id_k0 = load_id(t, my_octet), id_k1 = load_id(t + WAVES, my_octet), id_k2 = load_id(t + 2 * WAVES, my_octet);
    int id_v0 = load_id(t, quad), id_v1 = load_id(t + WAVES, quad);

    // the rows as operand: coordinates 32 s + 8 quad .. + 7 of row `col` of every block
    v8h qh[RB][STEPS], ql[Q32 ? RB : 1][STEPS];
    float to_log2[RB];
    int seen[RB];
    float unscale;
    if constexpr (STAGED) {
        // the head's centroids into LDS, scaled and split as in chunk_books_kernel
        constexpr int EACH = kCentroids * DK / 4 / (WAVES * kWave);
        const v4u *src = reinterpret_cast<const v4u *>(a.codebooks) + (int64_t)h * (kCentroids * DK / 4);
        v4u x[EACH];
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < EACH; ++u)
            x[u] = src[u * (WAVES * kWave) + tid];
#pragma unroll
        for (int u = 0; u < EACH; ++u)
            top = finite_top(x[u], top);
        const float wave_top = wave_max(__uint_as_float(top));
        if (lane == 0)
            tops_s[wave] = wave_top;
        __syncthreads();
        float head_top = tops_s[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
            head_top = fmaxf(head_top, tops_s[w]);
        const int lift = lift_of(__float_as_uint(head_top));
        unscale = power_of_two(-lift);
        const float f = power_of_two(lift);
#pragma unroll
        for (int u = 0; u < EACH; ++u)
            split_book(x[u], f, u * (WAVES * kWave) + tid, a.dsub_log2, few_s);
        __syncthreads();
    } else {
        unscale = a.unscale[h];
    }
#pragma unroll
    for (int j = 0; j < RB; ++j) {
        const int r = r0 + 16 * j + col, n = r / a.group, hq = h * a.group + r - n * a.group;
        const int n_at = n < a.N ? n : a.N - 1;
        seen[j] = n < span.count ? seen_of(span, n) : range.end;
        const int64_t q_at = b * a.q_b + hq * a.q_h + n_at * a.q_n + 8 * quad;
        to_log2[j] = a.scale_log2e * unscale;
        if constexpr (!Q32) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
                qh[j][s] = *reinterpret_cast<const v8h *>(static_cast<const _Float16 *>(a.q) + q_at + 32 * s);
        } else {
            v4f x[STEPS][2];
            float top = 0.f;
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    x[s][k] = *reinterpret_cast<const v4f *>(static_cast<const float *>(a.q) + q_at + 32 * s + 4 * k);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        top = fmaxf(top, fabsf(x[s][k][e]));
                }
            float u, v;
            lanes_xor16(top, u, v);
            lanes_xor32(fmaxf(u, v), u, v);
            const int lift = lift_of(__float_as_uint(fmaxf(u, v)));
            const float f = power_of_two(lift);
            to_log2[j] = a.scale_log2e * (unscale * power_of_two(-lift));
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float w = x[s][e / 4][e % 4] * f;
                    qh[j][s][e] = (_Float16)w;
                    ql[j][s][e] = (_Float16)(w - (float)qh[j][s][e]);
                }
        }
        // A negative scale turns the rows around, one of NaN makes their scores NaN (fmaxf would pass over it), and a scale of zero becomes fp32's
        // least, so that a score of -inf stays one.
        if (!(a.scale_log2e >= 0.f)) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                qh[j][s] = a.scale_log2e < 0.f ? -qh[j][s] : qh[j][s] * (_Float16)NAN;
                if constexpr (Q32)
                    ql[j][s] = -ql[j][s];
            }
        }
        to_log2[j] = fmaxf(fabsf(to_log2[j]), 1.17549435e-38f);
    }

    v4f acc[RB][CB][2];
    float ref[RB], z[RB];                 // the reference less kRefLift
#pragma unroll
    for (int j = 0; j < RB; ++j) {
        ref[j] = kNoReference;
        z[j] = 0.f;
#pragma unroll
        for (int c = 0; c < CB; ++c)
            acc[j][c][0] = acc[j][c][1] = (v4f){0.f, 0.f, 0.f, 0.f};
    }
    int nans = 0;                         // whether drop_nans found one in a tile of this wavefront
    if (t < range.t1) {
        load_codes(t, id_k0);
        if constexpr (!STAGED) {
            load_centroids();
            load_codes(t + WAVES, id_k1);
        }
    }
    while (t < range.t1) {
        // values of this tile
        const int id_v = page_of(t, quad, id_v0), id_k = page_of(t, my_octet, id_k0);
        const uint32_t page = id_v < 0 ? 0 : id_v;
        const uint8_t *src = head_values + (uint64_t)page * value_step + (uint32_t)(((t * kFewKeys + 8 * quad) & page_mask) * DK + col * 16);
        v4u v[CB];
#pragma unroll
        for (int c = 0; c < CB; ++c)
            v[c] = *reinterpret_cast<const v4u *>(src + c * 256);
        const int stored_e = head_exponents[(uint64_t)page * (uint32_t)p.H];
        const float e = id_v < 0 ? 0.f : (float)stored_e;
        if constexpr (STAGED) {
            load_centroids();
            load_codes(t + WAVES, id_k1);
        }
        // scores: element 4 k + i belongs to token 8 quad + 4 k + i
        const bool edge = (t + 1) * kFewKeys > seen_by_all || __builtin_amdgcn_ballot_w64(id_k < 0 || id_v < 0);
        if (edge) {
            // no token: zeros, whatever the centroids hold
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (id_k < 0 || t * kFewKeys + my_key + 4 * k >= range.end)
#pragma unroll
                    for (int s = 0; s < STEPS; ++s)
                        piece[k][s][0] = piece[k][s][1] = (v4u){0, 0, 0, 0};
        }
        v4f s[RB][2];
#pragma unroll
        for (int j = 0; j < RB; ++j)
            s[j][0] = s[j][1] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                v4u hi = piece[k][st][0], lo = piece[k][st][1];
                if constexpr (SMALL) {
                    hi = (v4u){piece[k][st][0].x, piece[k][st][0].y, piece[k][st][1].x, piece[k][st][1].y};
                    lo = (v4u){piece[k][st][0].z, piece[k][st][0].w, piece[k][st][1].z, piece[k][st][1].w};
                }
#pragma unroll
                for (int j = 0; j < RB; ++j) {
                    s[j][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, hi), qh[j][st], s[j][k], 0, 0, 0);
                    s[j][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, lo), qh[j][st], s[j][k], 0, 0, 0);
                    if constexpr (Q32)
                        s[j][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, hi), ql[j][st], s[j][k], 0, 0, 0);
                }
            }
        // centroids of the next tile, codes of the one behind it, page ids of the third
        const int id_kn = load_id(t + 3 * WAVES, my_octet), id_vn = load_id(t + 2 * WAVES, quad);
        if constexpr (!STAGED)
            if (t + WAVES < range.t1) {
                load_centroids();
                load_codes(t + 2 * WAVES, id_k2);
            }
        if (edge) {
            const int have = id_v < 0 ? 0 : range.end - t * kFewKeys - 8 * quad;
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                const int limit = id_v < 0 ? 0 : seen[j] - t * kFewKeys - 8 * quad;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    s[j][i / 4][i % 4] = i < limit ? s[j][i / 4][i % 4] : -INFINITY;
            }
            if constexpr (FP8) {
                // bytes without a token behind them may be NaN: zeros in their place
                const uint32_t lo = have >= 4 ? ~0u : have <= 0 ? 0u : (1u << (8 * have)) - 1;
                const uint32_t hi = have >= 8 ? ~0u : have <= 4 ? 0u : (1u << (8 * (have - 4))) - 1;
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    v[c].x &= lo, v[c].y &= hi;
                    v[c].z &= lo, v[c].w &= hi;
                }
                // and NaNs that not all rows see
                if ((t + 1) * kFewKeys > seen_by_all) {
                    uint32_t any = 0;
#pragma unroll
                    for (int c = 0; c < CB; ++c)
                        drop_nans(v[c], any);
                    nans |= __builtin_amdgcn_ballot_w64(any != 0) != 0;
                }
            }
        }
        const float unexp = power_of_two(-(int)e);
        v4u hi[RB], lo[RB];
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            float m = s[j][0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i)
                m = fmaxf(m, s[j][i / 4][i % 4]);
            const float top = fmaf(m, to_log2[j], e);
            if (__builtin_amdgcn_ballot_w64(top - ref[j] > kRefLift + kRefLag)) {
                float u, w;
                lanes_xor16(top, u, w);
                lanes_xor32(fmaxf(u, w), u, w);
                const float to = fmaxf(ref[j], fmaxf(u, w) - kRefLift), fix = fast_exp2(ref[j] - to);
                ref[j] = to;
                z[j] *= fix;
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    acc[j][c][0] *= fix;
                    acc[j][c][1] *= fix;
                }
            }
            const float shift = e - ref[j];
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w0 = fast_exp2(fmaf(s[j][i / 2][2 * (i % 2)], to_log2[j], shift));
                const float w1 = fast_exp2(fmaf(s[j][i / 2][2 * (i % 2) + 1], to_log2[j], shift));
                sum += w0;
                sum += w1;
                hi[j][i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(w0, w1));
                lo[j][i] = left_of(w0, w1, hi[j][i]);
            }
            z[j] = fmaf(sum, unexp, z[j]);
        }
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const v8h x0 = widen<FP8>(v[c].x, v[c].y), x1 = widen<FP8>(v[c].z, v[c].w);
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                acc[j][c][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x0, __builtin_bit_cast(v8h, hi[j]), acc[j][c][0], 0, 0, 0);
                acc[j][c][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x1, __builtin_bit_cast(v8h, hi[j]), acc[j][c][1], 0, 0, 0);
                acc[j][c][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x0, __builtin_bit_cast(v8h, lo[j]), acc[j][c][0], 0, 0, 0);
                acc[j][c][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x1, __builtin_bit_cast(v8h, lo[j]), acc[j][c][1], 0, 0, 0);
            }
        }
        t += WAVES;
        id_k0 = id_k1;
        id_k1 = id_k2;
        id_k2 = id_kn;
        id_v0 = id_v1;
        id_v1 = id_vn;
    }

    // The wavefronts' results, 16 rows at a time: references and sums first, so that every wavefront brings its own to the common reference.
    float *results = reinterpret_cast<float *>(few_s);
    float2 *stats = reinterpret_cast<float2 *>(few_s + (size_t)WAVES * 16 * ROW * 4);
    if constexpr (STAGED)
        __syncthreads();                  // (the centroids were read)
    int any = 0;
#pragma unroll
    for (int j = 0; j < RB; ++j) {
        float u, w;
        lanes_xor16(z[j], u, w);
        lanes_xor32(u + w, u, w);
        if (quad == 0)
            stats[wave * 16 + col] = make_float2(ref[j], u + w);
        if (FP8 && j == 0 && lane == 0)
            nans_s[wave] = nans;
        __syncthreads();
        if (FP8 && j == 0) {
#pragma unroll
            for (int k = 0; k < WAVES; ++k)
                any |= nans_s[k];
            any = __builtin_amdgcn_readfirstlane(any);
        }
        float top = kNoReference;
#pragma unroll
        for (int k = 0; k < WAVES; ++k)
            top = fmaxf(top, stats[k * 16 + col].x);
        const float f = fast_exp2(ref[j] - top);
        // register i of acc[c][x] is coordinate 32 c + 2 (4 quad + i) + x
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int i = 0; i < 4; i += 2)
                *reinterpret_cast<v4f *>(results + (wave * 16 + col) * ROW + 32 * c + 8 * quad + 2 * i) =
                    (v4f){acc[j][c][0][i] * f, acc[j][c][1][i] * f, acc[j][c][0][i + 1] * f, acc[j][c][1][i + 1] * f};
        __syncthreads();
        for (int x = tid; x < 16 * (DK / 4); x += WAVES * kWave) {
            const int k = x / (DK / 4), d = x % (DK / 4) * 4;
            const int r = r0 + 16 * j + k, n = r / a.group, hq = h * a.group + r - n * a.group;
            if (n >= span.count)
                continue;
            float best = kNoReference, sum = 0.f;
#pragma unroll
            for (int y = 0; y < WAVES; ++y)
                best = fmaxf(best, stats[y * 16 + k].x);
            v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < WAVES; ++y) {
                const float2 st = stats[y * 16 + k];
                sum = fmaf(fast_exp2(st.x - best), st.y, sum);
                o += *reinterpret_cast<const v4f *>(results + (y * 16 + k) * ROW + d);
            }
            if (range.ranges == 1) {
                const float g = sum == 0.f ? 0.f : 1.f / sum;        // (nothing to sum: zeros; a sum that is NaN stays one)
                *reinterpret_cast<v4f *>(a.out + ((int64_t)(b * p.H * a.group + hq) * a.N + n) * DK + d) = o * g;
            } else {
                float *to = a.part + ((((int64_t)at.unit * a.tiles + tile) * a.splits + split) * TQ + 16 * j + k) * (DK + kPartPad);
                *reinterpret_cast<v4f *>(to + d) = o;
                if (d == 0)
                    *reinterpret_cast<float2 *>(to + DK) = make_float2(best, sum);
            }
        }
        if (j + 1 < RB)
            __syncthreads();
    }
    if constexpr (FP8) {
        if (any) {
            __syncthreads();              // (the results were stored)
            const int first = (seen_by_all / kFewKeys > range.t0 ? seen_by_all / kFewKeys : range.t0) * kFewKeys, end = range.t1 * kFewKeys;
#pragma unroll 1
            for (int item = tid; item < TQ * DK; item += WAVES * kWave) {
                const int r = r0 + item / DK, n = r / a.group, hq = h * a.group + r - n * a.group, d = item % DK;
                if (n >= span.count)
                    continue;
                const int seen = seen_of(span, n);
                float *to = range.ranges == 1 ? a.out + ((int64_t)(b * p.H * a.group + hq) * a.N + n) * DK
                                              : a.part + ((((int64_t)at.unit * a.tiles + tile) * a.splits + split) * TQ + item / DK) * (DK + kPartPad);
                if (sees_nan<DK>(head_values, value_step, row, p.pages, p.page_log2, first, seen < end ? seen : end, d))
                    to[d] = NAN;
            }
        }
    }
}

// Merges the ranges of one row: a thread per coordinate.
__global__ void chunk_merge_kernel(ChunkArgs a, int H, int d_k, int page_log2, int TQ, int keys)
{
    const int n = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, d = threadIdx.x;
    const ChunkSpan span = chunk_span(a, b, page_log2);
    if (n >= span.count)
        return;
    const int h = hq / a.group, r = n * a.group + hq - h * a.group, tile = r / TQ;
    int n_last = (tile * TQ + TQ - 1) / a.group;
    n_last = n_last < span.count ? n_last : span.count - 1;
    const int ranges = (keys == 32 ? key_range<32>(span, n_last, a.splits, 0) : key_range<64>(span, n_last, a.splits, 0)).ranges;
    if (ranges == 1)
        return;
    const int stride = d_k + kPartPad;
    const float *x = a.part + (((int64_t)b * H + h) * a.tiles + tile) * a.splits * TQ * stride + (r - tile * TQ) * stride;
    float top = kNoReference, o = 0.f, z = 0.f;
    for (int s = 0; s < ranges; ++s, x += (int64_t)TQ * stride) {
        const float m = x[d_k], to = fmaxf(top, m), fix = fast_exp2(top - to), f = fast_exp2(m - to);
        o = fmaf(f, x[d], o * fix);
        z = fmaf(f, x[d_k + 1], z * fix);
        top = to;
    }
    a.out[((int64_t)(b * H * a.group + hq) * a.N + n) * d_k + d] = z == 0.f ? o * 0.f : o / z;     // (nothing to sum: zeros, but a stored NaN stays one)
}

// ---- host -------------------------------------------------------------------------------------------------------
struct ChunkCut {
    int few, waves, rows;                 // row blocks of the kernel for few rows or 0, wavefronts of a workgroup, rows of a tile
    int tiles, splits;
    int64_t work;
    size_t books, unscale, part;          // bytes, each a multiple of 16
};
static ChunkCut chunk_cut(const lookat_page_pool *p, int32_t B, int32_t N, int32_t group, int32_t W, int64_t max_length, int32_t num_splits)
{
    ChunkCut c;
    const int64_t units = (int64_t)B * p->H, rows = (int64_t)N * group;
    // The kernel for few rows, us a call with it / without.  One tile of its rows, or few workgroups: 240 (sequence, head) pairs x 32 rows x 632 tokens, d_k = 128
    // 17.8 / 46, 8 x 48 x 248, d_k = 64 8.9 / 15.7, 40 x 256 x 1256 26 / 33, 16 x 1024 x 9024, d_k = 128 155 / 181, 1 x 2048 x 10048 25 / 41.  Two tiles at d_k = 64:
    // 400 x 64 x 664 29 / 37, but at d_k = 128 61 / 57 and, fp32 rows, 79 / 67, though 1264 tokens 81 / 93.  Some more where there is more to see: 200 x 128 x
    // 1028, d_k = 128 73 / 86, but 200 x 128 x 228 31 / 30, 400 x 96 x 996 91 / 80, 96 x 600 x 600 98 / 47.
    const int64_t room = (int64_t)W * p->page, longest = max_length > 0 && max_length < room ? max_length : room, groups = units * ((rows + 31) / 32);
    const bool few = rows <= 32 || groups <= 512 || (rows <= 64 && p->d_k == 64) || ((rows <= 64 || groups <= 1024) && longest > 1000);
    c.few = !few ? 0 : rows <= 16 ? 1 : 2;
    // (Without it: 256 rows to a workgroup where they read long sequences and fill the chip, 128 otherwise: us a call at d_k = 128, 256 / 128, 32 x 2048 x 32049
    // 1917 / 2209, 128 x 1000 x 5000 575 / 634, 128 x 2000 x 2000 315 / 322, 96 x 600 x 2600 268 / 176, 320 x 380 x 880 167 / 125.)
    // Its workgroups have eight wavefronts, or two where there are many and a head has little to see, not worth its centroids in LDS: us a call, eight / two,
    // d_k = 64 768 x 8 rows x 8 tokens 13.1 / 9.4, 1280 x 8 x 308 23.3 / 23.5, 375 x 1 x 32 8.8 / 9.6, 400 x 20 x 320 16.8 / 16.6, 400 x 64 x 1264 51.3 / 47.2; d_k = 128
    // 768 x 12 x 128 26.1 / 20.9, 400 x 20 x 70 21.7 / 17.0 (fp32 rows 26.4 / 18.6), 400 x 20 x 320 25.1 / 27.0 (32.5 / 33.2), 1280 x 20 x 320 61.7 / 47.4
    // (79 / 71), 1280 x 32 x 632 77 / 76 (100 / 123).
    const int64_t brief = groups <= (rows <= 16 ? 512 : 256) ? 0 : rows <= 16 ? 256 : groups <= 512 ? 128 : rows <= 32 || p->d_k == 128 ? 448 : 1536;
    c.waves = c.few ? (longest > brief ? kFewWaves : kBriefWaves)
                    : p->d_k == 128 && rows >= 768 && longest > 2048 && units * ((rows + 255) / 256) >= 256 ? 8 : 4;
    c.rows = c.few ? 16 * c.few : 32 * c.waves;
    c.tiles = (int)((rows + c.rows - 1) / c.rows);
    c.splits = num_splits;
    if (!num_splits) {
        const int64_t target = 256 * 8 / c.waves, most = (longest + 511) / 512;
        int64_t s = (target + units * c.tiles / 2) / (units * c.tiles);
        s = s < most ? s : most;
        c.splits = (int)(s < 1 ? 1 : s);
    }
    c.work = units * c.tiles * c.splits;
    c.books = (size_t)p->H * kCentroids * p->d_k * 4;
    c.unscale = ((size_t)p->H * 4 + 15) / 16 * 16;
    c.part = c.splits > 1 ? (size_t)c.work * c.rows * (p->d_k + kPartPad) * 4 : 0;
    return c;
}

static int check_chunk(const lookat_page_pool *pool, int32_t B, int32_t N, int32_t group, int32_t W, int64_t max_length, int32_t num_splits)
{
    if (int rc = check_pool(pool))
        return rc;
    if (B <= 0 || W <= 0)
        return fail(LOOKAT_ERR_SHAPE, "B=%d and W=%d must be positive", B, W);
    if (N < 0 || group <= 0)
        return fail(LOOKAT_ERR_SHAPE, "N=%d must not be negative, group=%d must be positive", N, group);
    if (group > 64)
        return fail(LOOKAT_ERR_UNSUPPORTED, "group=%d: at most 64 query heads per key/value head", group);
    if (B > 65535 || (int64_t)W * pool->page > (1 << 30))
        return fail(LOOKAT_ERR_UNSUPPORTED, "B=%d, W=%d pages of %d tokens: at most 65535 sequences of 2^30 tokens", B, W, pool->page);
    if ((int64_t)N * group > (1 << 24) || (int64_t)pool->H * group > 65535)
        return fail(LOOKAT_ERR_UNSUPPORTED, "N=%d, H=%d, group=%d: at most 2^24 rows of a head (N * group) and 65535 query heads", N, pool->H, group);
    if (max_length < 0)
        return fail(LOOKAT_ERR_SHAPE, "max_length=%lld must not be negative", (long long)max_length);
    if (num_splits < 0 || num_splits > 65535)
        return fail(LOOKAT_ERR_SHAPE, "num_splits=%d out of range [0,65535]", num_splits);
    return LOOKAT_OK;
}

// Tokens of a tile: 64, or 32 at d_k = 128 where fp32 rows take the registers or the workgroup is small.  (d_k = 64, us a call, 32 / 64: 32 x 2048 rows 78 / 68,
// behind 2000 tokens 152 / 140, 64 x 1000 fp32 47.7 / 44.1, 96 heads x 400 to 1000 fp32 47.6 / 47.0.)
constexpr int chunk_keys(int d_k, int waves, bool q32) { return d_k == 64 || (waves == 8 && !q32) ? 64 : 32; }

template <int DK, bool SMALL, int NW>
static int launch_chunk(const PoolArgs &p, const ChunkArgs &a, bool q32, bool fp8, unsigned groups, hipStream_t st)
{
    constexpr int K32 = chunk_keys(DK, NW, true), K16 = chunk_keys(DK, NW, false);
    const auto f = q32 ? (fp8 ? &chunk_kernel<DK, SMALL, true, true, NW, K32> : &chunk_kernel<DK, SMALL, true, false, NW, K32>)
                       : (fp8 ? &chunk_kernel<DK, SMALL, false, true, NW, K16> : &chunk_kernel<DK, SMALL, false, false, NW, K16>);
    hipLaunchKernelGGL(f, dim3(groups), dim3(NW * kWave), 0, st, p, a);
    return check_launch("lookat_attend_pages_chunk");
}
// Whether two wavefronts take two blocks of rows.
constexpr bool two_brief_blocks(int d_k, bool q32) { return d_k == 64 || !q32; }

template <int DK, bool SMALL, int RB, int WAVES>
static int launch_few(const PoolArgs &p, const ChunkArgs &a, bool q32, bool fp8, unsigned groups, hipStream_t st)
{
    constexpr int R32 = RB == 2 && WAVES == kBriefWaves && !two_brief_blocks(DK, true) ? 1 : RB;
    const auto f = q32 ? (fp8 ? &chunk_few_kernel<DK, SMALL, true, true, R32, WAVES> : &chunk_few_kernel<DK, SMALL, true, false, R32, WAVES>)
                       : (fp8 ? &chunk_few_kernel<DK, SMALL, false, true, RB, WAVES> : &chunk_few_kernel<DK, SMALL, false, false, RB, WAVES>);
    constexpr size_t results = few_lds_bytes(DK, WAVES), book = few_staged(WAVES) ? (size_t)kCentroids * DK * 4 : 0, lds = results > book ? results : book;
    if (lds > 60 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(f), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess)
            return fail(LOOKAT_ERR_HIP, "lookat_attend_pages_chunk: %s", hipGetErrorString(e));
    }
    hipLaunchKernelGGL(f, dim3(groups), dim3(WAVES * kWave), lds, st, p, a);
    return check_launch("lookat_attend_pages_chunk");
}
template <int DK, bool SMALL>
static int launch_rows(const ChunkCut &c, const PoolArgs &p, const ChunkArgs &a, bool q32, bool fp8, unsigned groups, hipStream_t st)
{
    switch (c.few) {
    case 1: return c.waves == kFewWaves ? launch_few<DK, SMALL, 1, kFewWaves>(p, a, q32, fp8, groups, st)
                                        : launch_few<DK, SMALL, 1, kBriefWaves>(p, a, q32, fp8, groups, st);
    case 2: return c.waves == kFewWaves ? launch_few<DK, SMALL, 2, kFewWaves>(p, a, q32, fp8, groups, st)
                                        : launch_few<DK, SMALL, 2, kBriefWaves>(p, a, q32, fp8, groups, st);
    default:
        if constexpr (DK == 128)
            if (c.waves == 8)
                return launch_chunk<DK, SMALL, 8>(p, a, q32, fp8, groups, st);
        return launch_chunk<DK, SMALL, 4>(p, a, q32, fp8, groups, st);
    }
}

}  // namespace lookat

extern "C" size_t lookat_attend_pages_chunk_workspace_bytes(const lookat_page_pool *pool, int32_t B, int32_t N, int32_t group, int32_t W,
                                                            int64_t max_length, int32_t num_splits)
{
    using namespace lookat;
    clear_error();
    if (check_chunk(pool, B, N, group, W, max_length, num_splits) != LOOKAT_OK || N == 0)
        return 0;
    const ChunkCut c = chunk_cut(pool, B, N, group, W, max_length, num_splits);
    return c.books + c.unscale + c.part;
}

extern "C" int lookat_attend_pages_chunk(const lookat_page_pool *pool, int32_t B, int32_t N, int32_t group, const void *q, lookat_dtype q_dtype,
                                         int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_n, const float *codebooks,
                                         const int32_t *table, int32_t W, int64_t table_stride, const int32_t *lengths, const int32_t *counts,
                                         int64_t max_length, float scale, int32_t num_splits, void *workspace, size_t workspace_bytes,
                                         float *out, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_chunk(pool, B, N, group, W, max_length, num_splits))
        return rc;
    if (q_dtype != LOOKAT_F16 && q_dtype != LOOKAT_F32)
        return fail(LOOKAT_ERR_DTYPE, "q_dtype=%d is neither LOOKAT_F16 nor LOOKAT_F32", (int)q_dtype);
    if (int rc = check_table(pool, "B", B, table, W, table_stride))
        return rc;
    if (N == 0)
        return LOOKAT_OK;
    if (!q || !codebooks || !lengths || !out)
        return fail(LOOKAT_ERR_NULL, "q, codebooks, lengths and out must be non-NULL");
    const int64_t unit = q_dtype == LOOKAT_F16 ? 8 : 4;
    if (!aligned16(q) || !aligned16(codebooks) || !aligned16(out) || q_stride_b % unit || q_stride_h % unit || q_stride_n % unit)
        return fail(LOOKAT_ERR_ALIGN, "q, its strides, codebooks and out must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(lengths) | reinterpret_cast<uintptr_t>(counts)) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "lengths and counts must be 4-byte aligned");
    ChunkCut cut = chunk_cut(pool, B, N, group, W, max_length, num_splits);
    const size_t need = cut.books + cut.unscale + cut.part;
    if (!workspace || workspace_bytes < need)
        return fail(LOOKAT_ERR_WORKSPACE, "workspace of %zu bytes needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
    if (!aligned16(workspace))
        return fail(LOOKAT_ERR_ALIGN, "workspace must be 16-byte aligned");
    // fp32 rows at d_k = 128 in two wavefronts: one block of 16 rows, of two the registers do not hold both terms beside the accumulators and
    // operands (33 to 35 were spilled; us a call, two / one, 400 x 20 rows x 70 tokens 22.1 / 16.5, 1280 x 20 x 320 74 / 59, 1280 x 32 x 432
    // 94 / 85, 768 x 24 x 124 31.1 / 33.1).  Partial rows take no more room: as many ranges, and ceil(rows / 16) * 16 <= ceil(rows / 32) * 32.
    if (cut.few == 2 && cut.waves == kBriefWaves && !two_brief_blocks(pool->d_k, q_dtype == LOOKAT_F32)) {
        cut.few = 1;
        cut.rows = 16;
        cut.tiles = (int)(((int64_t)N * group + cut.rows - 1) / cut.rows);
        cut.work = (int64_t)B * pool->H * cut.tiles * cut.splits;
    }
    const int64_t all_units = (int64_t)B * pool->H, per_unit = (int64_t)cut.tiles * cut.splits, whole = all_units / kXcds * per_unit;
    const int64_t left = all_units % kXcds * per_unit, per_die = (left + kXcds - 1) / kXcds, groups = (whole + per_die) * kXcds;
    if (!fits_launch(groups, cut.waves * kWave))
        return fail(LOOKAT_ERR_UNSUPPORTED, "B*H*rows*num_splits: %lld workgroups exceed one launch", (long long)cut.work);
    if (cut.splits > 1 && !fits_launch((int64_t)N * pool->H * group * B, pool->d_k))
        return fail(LOOKAT_ERR_UNSUPPORTED, "N=%d rows of %d heads in %d sequences exceed one launch when cut into ranges", N, pool->H * group, B);
    const PoolArgs p = pool_args(pool);
    const int dsub = p.d_k / p.m, dsub_log2 = 31 - __builtin_clz((unsigned)dsub);
    ChunkArgs a;
    a.q = q;
    a.codebooks = codebooks;
    char *books = static_cast<char *>(workspace);
    float *unscale = reinterpret_cast<float *>(books + cut.books);
    a.books = books;
    a.unscale = unscale;
    a.table = table;
    a.lengths = lengths;
    a.counts = counts;
    a.part = reinterpret_cast<float *>(books + cut.books + cut.unscale);
    a.out = out;
    a.q_b = q_stride_b;
    a.q_h = q_stride_h;
    a.q_n = q_stride_n;
    a.table_stride = table_stride;
    a.W = W;
    a.N = N;
    a.group = group;
    a.dsub_log2 = dsub_log2;
    a.tiles = cut.tiles;
    a.splits = cut.splits;
    a.units = (int32_t)all_units;
    a.whole = (int32_t)whole;
    a.left = (int32_t)left;
    a.per_die = (int32_t)per_die;
    a.scale_log2e = scale * kLog2e;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (!(cut.few && few_staged(cut.waves))) {
        hipLaunchKernelGGL(chunk_books_kernel, dim3(kBookParts, p.H), dim3(kBookThreads), 0, st, codebooks, books, unscale, p.d_k, dsub_log2);
        if (int rc = check_launch("lookat_attend_pages_chunk (codebooks)"))
            return rc;
    }
    const bool q32 = q_dtype == LOOKAT_F32, fp8 = pool->value_type == LOOKAT_VALUES_E4M3;
    const int rc = p.d_k == 128 ? launch_rows<128, false>(cut, p, a, q32, fp8, (unsigned)groups, st)
                   : dsub == 4  ? launch_rows<64, true>(cut, p, a, q32, fp8, (unsigned)groups, st)
                                : launch_rows<64, false>(cut, p, a, q32, fp8, (unsigned)groups, st);
    if (rc != LOOKAT_OK)
        return rc;
    if (cut.splits == 1)
        return LOOKAT_OK;
    hipLaunchKernelGGL(chunk_merge_kernel, dim3((unsigned)N, (unsigned)(p.H * group), (unsigned)B), dim3(p.d_k), 0, st, a, p.H, p.d_k, p.page_log2,
                       cut.rows, cut.few ? kFewKeys : chunk_keys(p.d_k, cut.waves, q32));
    return check_launch("lookat_attend_pages_chunk (merge)");
}
