// Attention of a chunk of new tokens over the paged cache: every row sees the tokens up to its own position.
//
//   s = q . k^,  k^ = (C_0[code_0], C_1[code_1], ...),   out = sum_{l <= p} softmax_l(scale s) q_l 2^e(l)
//
// With many rows per cached token the sum over table entries is a dense product with the keys' centroids, and belongs on the matrix cores
// (v_mfma_f32_32x32x16_f16), as does the weighted sum:
//   * S^T = K^ Q^T: a wavefront owns 32 rows (columns of S^T).  Centroids enter as two fp16 terms of 2^s w (22 bits; s one power of two per
//     head, which brings the head's largest centroid entry to 2^14), fp16 queries exactly, fp32 queries as two terms of their own power of
//     two (the product of the two small terms, 2^-22, is dropped).
//   * a lane then holds 32 scores of ONE row: running reference and sum need no exchange but with the lane that holds the row's other keys.
//     Reference and page exponents as in attention of one token: y = scale log2(e) s + e, w = 2^(y - R).
//   * O^T = V^T P^T: keys are dealt to the rows of K^ (bits 2 and 3 of a row's number exchanged) such that the eight weights that a lane holds
//     of an operand belong to eight consecutive tokens: the weights, as two fp16 terms, are the operand where they are, and the values' operand
//     is eight consecutive stored bytes, as the page holds them.
// The centroids are split once per call by a small kernel, into the workspace.  A workgroup of NW wavefronts (32 NW rows of one key/value head,
// query heads of a group side by side) fetches the centroids of 64 keys by code into LDS, two buffers of 64 keys in turn; their ids, codes and
// centroids are requested three, two and one tiles ahead.
#include "pages_values.h"

namespace lookat {

typedef float v16f __attribute__((ext_vector_type(16)));

struct ChunkArgs {
    const void *q;
    const char *books;                    // [H, m, 256, 2, d_sub] fp16: both terms of a centroid
    const float *unscale;                 // [H] 2^-s
    const int32_t *table, *lengths, *counts;
    float *part, *out;
    int64_t q_b, q_h, q_n, table_stride;  // strides in elements
    int32_t W, N, group, dsub_log2;
    int32_t tiles, splits, work, per_die; // row tiles of a (sequence, head), ranges, workgroups with something to do, of them per die
    float scale_log2e;
};

constexpr int kChunkKeys = 64;
constexpr int kBookTop = 14;              // the largest centroid entry comes between 2^14 and 2^15
constexpr int kPartPad = 4;               // a partial row: d_k sums, reference, sum, two unused

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// The power of two that brings x (its magnitude's bits) between 2^kBookTop and twice that, as far as fp32 goes.
__device__ __forceinline__ int lift_of(uint32_t bits)
{
    const int s = bits ? kBookTop + 127 - (int)(bits >> 23) : 0;
    return s > 100 ? 100 : s < -100 ? -100 : s;
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
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t a = x[k] & 0x7fffffffu;
            top = a < 0x7f800000u && a > top ? a : top;       // (entries that are not finite do not count: no token may have them)
        }
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
    for (int u = blockIdx.x * per + tid; u < (int)(blockIdx.x + 1) * per; u += kBookThreads) {
        const v4u x = src[u];
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
        char *to = books + ((((int64_t)h * kCentroids * d_k + ((int64_t)centroid << dsub_log2)) * 2 + j) << 1);
        *reinterpret_cast<v2u *>(to) = (v2u){hi[0], hi[1]};
        *reinterpret_cast<v2u *>(to + (2 << dsub_log2)) = (v2u){lo[0], lo[1]};
    }
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
__device__ __forceinline__ KeyRange key_range(const ChunkSpan &s, int last_row, int splits, int split)
{
    KeyRange r;
    r.end = seen_of(s, last_row);
    const int tiles = (r.end + kChunkKeys - 1) / kChunkKeys, per = (tiles + splits - 1) / splits;
    r.ranges = per ? (tiles + per - 1) / per : 1;
    r.t0 = split * per;
    r.t1 = tiles - r.t0 < per ? tiles : r.t0 + per;
    return r;
}

template <int DK, bool SMALL, bool Q32, bool FP8, int NW>
__global__ __launch_bounds__(NW *kWave, 2) void chunk_kernel(PoolArgs p, ChunkArgs a)
{
    constexpr int CH = DK / 8, STEPS = DK / 16, CB = DK / 64, TQ = 32 * NW;
    constexpr int CPT = CH / NW > 0 ? CH / NW : 1;               // 8-coordinate pieces of a key that a thread fetches
    constexpr int kPlane = kChunkKeys * DK * 2, kBuffer = 2 * kPlane;
    static_assert(CH % NW == 0, "whole pieces for every thread");
    __shared__ __align__(16) char keys_s[2 * kBuffer];
    __shared__ int ids_s[2][4], exps_s[2][4];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, half = lane >> 5, col = lane & 31;
    const int index = (int)(blockIdx.x % kXcds) * a.per_die + (int)(blockIdx.x / kXcds);
    if ((int)(blockIdx.x / kXcds) >= a.per_die || index >= a.work)
        return;
    const int per_unit = a.tiles * a.splits, unit = index / per_unit, rest = index - unit * per_unit;
    const int tile = a.tiles - 1 - rest / a.splits, split = rest % a.splits;
    const int b = unit / p.H, h = unit - b * p.H;
    const ChunkSpan span = chunk_span(a, b, p.page_log2);
    const int r0 = tile * TQ, n_first = r0 / a.group;
    if (n_first >= span.count)
        return;
    int n_last = (r0 + TQ - 1) / a.group;
    n_last = n_last < span.count ? n_last : span.count - 1;
    const KeyRange range = key_range(span, n_last, a.splits, split);
    if (split >= range.ranges)
        return;
    const int32_t *row = a.table + b * a.table_stride;
    const int page_mask = (1 << p.page_log2) - 1;

    // this lane's row
    const int r = r0 + wave * 32 + col, n = r / a.group, hq = h * a.group + r - n * a.group;
    const bool mine = n < span.count;
    const int seen = mine ? seen_of(span, n) : range.end;
    const int seen_by_all = seen_of(span, n_first);
    const int n_at = n < a.N ? n : a.N - 1;

    // ---- the keys of a tile ----
    const int kk = tid / NW, sub = tid % NW;
    const int krow = (kk & ~12) | (kk & 4) << 1 | (kk & 8) >> 1;
    auto load_id = [&](int t) -> int {
        const int key = t * kChunkKeys + kk;
        int id = -1;
        if (key < range.end)
            id = row[key >> p.page_log2];
        return (uint32_t)id < (uint32_t)p.pages ? id : -1;
    };
    constexpr int CODES = SMALL ? 2 * CPT : CPT;
    uint32_t codes[CODES];
    int exponent;
    auto load_codes = [&](int t, int id) {
        const int key = t * kChunkKeys + kk;
        const int64_t place = (int64_t)(id < 0 ? 0 : id) * p.H + h;
        const uint8_t *c = p.codes + ((place << p.page_log2) + (key & page_mask)) * p.m;
#pragma unroll
        for (int j = 0; j < CPT; ++j) {
            const int chunk = sub + j * NW;
            if constexpr (SMALL) {
                codes[2 * j] = c[2 * chunk];
                codes[2 * j + 1] = c[2 * chunk + 1];
            } else {
                codes[j] = c[(chunk * 8) >> a.dsub_log2];
            }
        }
        exponent = p.exponents[place];
    };
    v4u piece[CPT][2];
    const char *books = a.books + (int64_t)h * kCentroids * DK * 4;
    auto load_centroids = [&]() {
#pragma unroll
        for (int j = 0; j < CPT; ++j) {
            const int chunk = sub + j * NW;
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
    auto put = [&](int t, int id, int e) {
        char *to = keys_s + (t & 1) * kBuffer + krow * (DK * 2);
#pragma unroll
        for (int j = 0; j < CPT; ++j) {
            const int chunk = sub + j * NW, at = (chunk ^ (krow & (CH - 1))) << 4;
            v4u hi = piece[j][0], lo = piece[j][1];
            if constexpr (SMALL) {
                hi = (v4u){piece[j][0].x, piece[j][0].y, piece[j][1].x, piece[j][1].y};
                lo = (v4u){piece[j][0].z, piece[j][0].w, piece[j][1].z, piece[j][1].w};
            }
            if (id < 0)                   // no token: zeros, whatever the centroids hold
                hi = lo = (v4u){0, 0, 0, 0};
            *reinterpret_cast<v4u *>(to + at) = hi;
            *reinterpret_cast<v4u *>(to + kPlane + at) = lo;
        }
        if ((kk & 15) == 0 && sub == 0) {
            ids_s[t & 1][kk >> 4] = id;
            exps_s[t & 1][kk >> 4] = id < 0 ? 0 : e;
        }
    };
    int id1 = load_id(range.t0), id2 = load_id(range.t0 + 1), id3 = load_id(range.t0 + 2);

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
    const float to_log2 = a.scale_log2e * unscale;

    load_codes(range.t0, id1);
    load_centroids();
    const int exponent0 = exponent;
    load_codes(range.t0 + 1, id2);
    put(range.t0, id1, exponent0);
    __syncthreads();

    v16f acc[CB][2];
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            acc[c][0][i] = acc[c][1][i] = 0.f;
    float ref = kNoReference, z = 0.f;    // the reference less kRefLift

    for (int t = range.t0; t < range.t1; ++t) {
        const int slot = t & 1;
        int ids[4], exps[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            ids[g] = __builtin_amdgcn_readfirstlane(ids_s[slot][g]);
            exps[g] = __builtin_amdgcn_readfirstlane(exps_s[slot][g]);
        }
        // values of this tile, centroids of the next, codes of the one behind it, page ids of the third
        v4u v[4][CB];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int64_t at = ((int64_t)(ids[g] < 0 ? 0 : ids[g]) * p.H + h) << p.page_log2;
            const uint8_t *src = p.values + (at + ((t * kChunkKeys + 16 * g) & page_mask)) * DK + half * (8 * DK) + col * 16;
#pragma unroll
            for (int c = 0; c < CB; ++c)
                v[g][c] = *reinterpret_cast<const v4u *>(src + c * 512);
        }
        const int e1 = exponent;
        load_centroids();
        load_codes(t + 2, id3);
        const int id4 = load_id(t + 3);

        // scores
        v16f s[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[k][i] = 0.f;
        const char *from = keys_s + slot * kBuffer;
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const char *at = from + (32 * k + col) * (DK * 2) + (((2 * st + half) ^ (col & (CH - 1))) << 4);
                const v8h hi = *reinterpret_cast<const v8h *>(at), lo = *reinterpret_cast<const v8h *>(at + kPlane);
                s[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi, qh[st], s[k], 0, 0, 0);
                s[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lo, qh[st], s[k], 0, 0, 0);
                if constexpr (Q32)
                    s[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hi, ql[st], s[k], 0, 0, 0);
            }
        // logits: score i of block k belongs to token 32 k + 16 (i / 8) + 8 half + i % 8
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[k][i] = fmaf(s[k][i], to_log2, (float)exps[2 * k + i / 8]);
        const bool absent = (ids[0] | ids[1] | ids[2] | ids[3]) < 0;
        if (absent || (t + 1) * kChunkKeys > seen_by_all) {
            const int limit = seen - t * kChunkKeys - 8 * half;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[k][i] = 32 * k + 16 * (i / 8) + i % 8 < (ids[2 * k + i / 8] < 0 ? -64 : limit) ? s[k][i] : -INFINITY;
            if constexpr (FP8) {
                // bytes without a token behind them may be NaN: zeros in their place
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int m = ids[g] < 0 ? 0 : range.end - t * kChunkKeys - 16 * g - 8 * half;
                    const uint32_t lo = m >= 4 ? ~0u : m <= 0 ? 0u : (1u << (8 * m)) - 1;
                    const uint32_t hi = m >= 8 ? ~0u : m <= 4 ? 0u : (1u << (8 * (m - 4))) - 1;
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        v[g][c].x &= lo, v[g][c].y &= hi;
                        v[g][c].z &= lo, v[g][c].w &= hi;
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                top = fmaxf(top, s[k][i]);
        if (__builtin_amdgcn_ballot_w64(top - ref > kRefLift + kRefLag)) {
            float u, w;
            lanes_xor32(top, u, w);
            const float to = fmaxf(ref, fmaxf(u, w) - kRefLift), fix = fast_exp2(ref - to);
            ref = to;
            z *= fix;
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    acc[c][0][i] *= fix;
                    acc[c][1][i] *= fix;
                }
        }
        // weights and the weighted sum, 16 tokens at a time
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float w[8], sum = 0.f;
            v8h hi, lo;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = fast_exp2(s[g / 2][8 * (g % 2) + i] - ref);
                sum += w[i];
                hi[i] = (_Float16)w[i];
                lo[i] = (_Float16)(w[i] - (float)hi[i]);
            }
            z = fmaf(sum, power_of_two(-exps[g]), z);
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                const v8h a0 = widen<FP8>(v[g][c].x, v[g][c].y), a1 = widen<FP8>(v[g][c].z, v[g][c].w);
                acc[c][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a0, hi, acc[c][0], 0, 0, 0);
                acc[c][1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a1, hi, acc[c][1], 0, 0, 0);
                acc[c][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a0, lo, acc[c][0], 0, 0, 0);
                acc[c][1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a1, lo, acc[c][1], 0, 0, 0);
            }
        }
        put(t + 1, id2, e1);
        id2 = id3;
        id3 = id4;
        __syncthreads();
    }

    float u, w;
    lanes_xor32(z, u, w);
    z = u + w;
    if (!mine)
        return;
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
    // register i of a result is coordinate 64 c + 2 ((i % 4) + 8 (i / 4) + 4 half) of acc[c][0], the next one of acc[c][1]
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const v4f o = {acc[c][0][i] * f, acc[c][1][i] * f, acc[c][0][i + 1] * f, acc[c][1][i + 1] * f};
            *reinterpret_cast<v4f *>(to + 64 * c + 16 * (i / 4) + 8 * half + 2 * (i % 4)) = o;
        }
}

// Merges the ranges of one row: a thread per coordinate.
__global__ void chunk_merge_kernel(ChunkArgs a, int H, int d_k, int page_log2, int TQ)
{
    const int n = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, d = threadIdx.x;
    const ChunkSpan span = chunk_span(a, b, page_log2);
    if (n >= span.count)
        return;
    const int h = hq / a.group, r = n * a.group + hq - h * a.group, tile = r / TQ;
    int n_last = (tile * TQ + TQ - 1) / a.group;
    n_last = n_last < span.count ? n_last : span.count - 1;
    const int ranges = key_range(span, n_last, a.splits, 0).ranges;
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
    a.out[((int64_t)(b * H * a.group + hq) * a.N + n) * d_k + d] = z == 0.f ? 0.f : o / z;
}

// ---- host -------------------------------------------------------------------------------------------------------
struct ChunkCut {
    int waves, tiles, splits;
    int64_t work;
    size_t books, unscale, part;          // bytes, each a multiple of 16
};
static ChunkCut chunk_cut(const lookat_page_pool *p, int32_t B, int32_t N, int32_t group, int32_t W, int64_t max_length, int32_t num_splits)
{
    ChunkCut c;
    const int64_t units = (int64_t)B * p->H, rows = (int64_t)N * group;
    c.waves = rows <= 128 || units * ((rows + 255) / 256) < 256 ? 4 : 8;
    const int TQ = 32 * c.waves;
    c.tiles = (int)((rows + TQ - 1) / TQ);
    const int64_t room = (int64_t)W * p->page, longest = max_length > 0 && max_length < room ? max_length : room;
    c.splits = num_splits;
    if (!num_splits) {
        const int64_t target = 256 * 8 / c.waves, most = (longest + 255) / 256;
        int64_t s = (target + units * c.tiles / 2) / (units * c.tiles);
        s = s < most ? s : most;
        c.splits = (int)(s < 1 ? 1 : s);
    }
    c.work = units * c.tiles * c.splits;
    c.books = (size_t)p->H * kCentroids * p->d_k * 4;
    c.unscale = ((size_t)p->H * 4 + 15) / 16 * 16;
    c.part = c.splits > 1 ? (size_t)c.work * TQ * (p->d_k + kPartPad) * 4 : 0;
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

template <int DK, bool SMALL, int NW>
static void launch_chunk(const PoolArgs &p, const ChunkArgs &a, bool q32, bool fp8, hipStream_t st)
{
    const auto f = q32 ? (fp8 ? &chunk_kernel<DK, SMALL, true, true, NW> : &chunk_kernel<DK, SMALL, true, false, NW>)
                       : (fp8 ? &chunk_kernel<DK, SMALL, false, true, NW> : &chunk_kernel<DK, SMALL, false, false, NW>);
    hipLaunchKernelGGL(f, dim3((unsigned)(a.per_die * kXcds)), dim3(NW * kWave), 0, st, p, a);
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
    const ChunkCut cut = chunk_cut(pool, B, N, group, W, max_length, num_splits);
    const size_t need = cut.books + cut.unscale + cut.part;
    if (!workspace || workspace_bytes < need)
        return fail(LOOKAT_ERR_WORKSPACE, "workspace of %zu bytes needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
    if (!aligned16(workspace))
        return fail(LOOKAT_ERR_ALIGN, "workspace must be 16-byte aligned");
    if (cut.work > 0x7fffffff || !fits_launch((cut.work + kXcds - 1) / kXcds * kXcds, cut.waves * kWave))
        return fail(LOOKAT_ERR_UNSUPPORTED, "B*H*rows*num_splits: %lld workgroups exceed one launch", (long long)cut.work);
    if (cut.splits > 1 && !fits_launch((int64_t)N * pool->H * group * B, pool->d_k))
        return fail(LOOKAT_ERR_UNSUPPORTED, "N=%d rows of %d heads in %d sequences exceed one launch when cut into ranges", N, pool->H * group, B);
    const PoolArgs p = pool_args(pool);
    const int dsub = p.d_k / p.m, dsub_log2 = 31 - __builtin_clz((unsigned)dsub);
    ChunkArgs a;
    a.q = q;
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
    a.work = (int32_t)cut.work;
    a.per_die = (int32_t)((cut.work + kXcds - 1) / kXcds);
    a.scale_log2e = scale * kLog2e;
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(chunk_books_kernel, dim3(kBookParts, p.H), dim3(kBookThreads), 0, st, codebooks, books, unscale, p.d_k, dsub_log2);
    if (int rc = check_launch("lookat_attend_pages_chunk (codebooks)"))
        return rc;
    const bool q32 = q_dtype == LOOKAT_F32, fp8 = pool->value_type == LOOKAT_VALUES_E4M3;
    if (p.d_k == 128)
        cut.waves == 8 ? launch_chunk<128, false, 8>(p, a, q32, fp8, st) : launch_chunk<128, false, 4>(p, a, q32, fp8, st);
    else if (dsub == 4)
        cut.waves == 8 ? launch_chunk<64, true, 8>(p, a, q32, fp8, st) : launch_chunk<64, true, 4>(p, a, q32, fp8, st);
    else
        cut.waves == 8 ? launch_chunk<64, false, 8>(p, a, q32, fp8, st) : launch_chunk<64, false, 4>(p, a, q32, fp8, st);
    if (int rc = check_launch("lookat_attend_pages_chunk"))
        return rc;
    if (cut.splits == 1)
        return LOOKAT_OK;
    hipLaunchKernelGGL(chunk_merge_kernel, dim3((unsigned)N, (unsigned)(p.H * group), (unsigned)B), dim3(p.d_k), 0, st, a, p.H, p.d_k, p.page_log2,
                       32 * cut.waves);
    return check_launch("lookat_attend_pages_chunk (merge)");
}
