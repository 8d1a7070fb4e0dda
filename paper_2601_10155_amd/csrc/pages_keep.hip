// Holding a cache to a budget: every token's sum of the attention it was paid, and moving the heaviest tokens into fewer pages.
#include "pages_quantise.h"
#include "decode_common.h"

namespace lookat {

// ---- attention sums ---------------------------------------------------------------------------------------------
//   w_l = decay w_l + sum_g 2^(y_gl - M_g) / Z_g,   y_gl = scale log2(e) sum_i lut_gi[code_li],   M_g = max_l y_gl,  Z_g = sum_l 2^(y_gl - M_g)
//
// A workgroup of 1024 threads takes a range of one (sequence, key/value head): its scores stay in registers (kWeighScores a thread, over the
// group's query heads) from the maximum to the weights, so that codes are read and looked up once.  Where one range does not hold a sequence or
// there are few of them, sequences are cut: a first launch brings the ranges' maxima and sums, a second one scores again and adds.
struct WeighArgs {
    const float *lut;
    const int32_t *table, *lengths;
    float *weights;
    float2 *stats;                        // [units, splits, G] maximum and sum of a range
    int64_t table_stride, weight_stride;
    int32_t W, columns, units, splits, chunk;
    float scale_log2e, decay;
};

constexpr int kWeighThreads = 1024, kWeighWaves = kWeighThreads / kWave, kWeighScores = 32;
__host__ __device__ constexpr int weigh_tokens(int G) { return kWeighThreads * (kWeighScores / G); }     // of a range, at most

enum WeighPhase { kWeighAll, kWeighStats, kWeighAdd };

template <int M, int G, int PHASE>
__global__ __launch_bounds__(kWeighThreads) void weigh_kernel(PoolArgs p, WeighArgs a)
{
    constexpr int GP = G < 4 ? G : 4, PLANES = G / GP, T = kWeighScores / G;
    typedef float vg __attribute__((ext_vector_type(GP)));
    extern __shared__ __align__(16) float tables[];       // [plane][i][c][head of the plane]
    __shared__ float red[2][G][kWeighWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int unit = (int)(blockIdx.x / kXcds) / a.splits * kXcds + (int)(blockIdx.x % kXcds), split = (int)(blockIdx.x / kXcds) % a.splits;
    if (unit >= a.units)
        return;
    const int b = unit / p.H, h = unit - b * p.H;
    const int length = clamp_length(a.lengths[b], a.W, p.page_log2);
    const int k0 = split * a.chunk, k1 = length - k0 < a.chunk ? length : k0 + a.chunk;
    if (k0 >= k1)
        return;
    const int32_t *row = a.table + b * a.table_stride;
    const int page_mask = (1 << p.page_log2) - 1;

    {
        const float *lut = a.lut + (int64_t)unit * G * M * kCentroids;
        for (int j = tid; j < G * M * kCentroids; j += kWeighThreads) {
            const int g = j / (M * kCentroids), entry = j % (M * kCentroids);
            tables[(g / GP * M * kCentroids + entry) * GP + g % GP] = lut[j] * a.scale_log2e;
        }
    }
    __syncthreads();

    float y[T][G], top[G];
#pragma unroll
    for (int g = 0; g < G; ++g)
        top[g] = -INFINITY;
#pragma unroll
    for (int t = 0; t < T; ++t) {
#pragma unroll
        for (int g = 0; g < G; ++g)
            y[t][g] = -INFINITY;
        const int key = k0 + t * kWeighThreads + tid;
        if (k0 + t * kWeighThreads < k1 && key < k1) {
            const int id = row[key >> p.page_log2];
            if ((uint32_t)id < (uint32_t)p.pages) {
                const uint8_t *c = p.codes + ((((int64_t)id * p.H + h) << p.page_log2) + (key & page_mask)) * M;
                uint32_t codes[(M + 3) / 4];
                if constexpr (M == 2) {
                    codes[0] = *reinterpret_cast<const uint16_t *>(c);
                } else if constexpr (M == 4) {
                    codes[0] = *reinterpret_cast<const uint32_t *>(c);
                } else if constexpr (M == 8) {
                    const v2u x = *reinterpret_cast<const v2u *>(c);
                    codes[0] = x.x, codes[1] = x.y;
                } else {
                    const v4u x = *reinterpret_cast<const v4u *>(c);
                    codes[0] = x.x, codes[1] = x.y, codes[2] = x.z, codes[3] = x.w;
                }
#pragma unroll
                for (int q = 0; q < PLANES; ++q) {
                    vg s = {};
#pragma unroll
                    for (int i = 0; i < M; ++i)
                        s += reinterpret_cast<const vg *>(tables)[(q * M + i) * kCentroids + ((codes[i / 4] >> (8 * (i % 4))) & 0xffu)];
#pragma unroll
                    for (int g = 0; g < GP; ++g)
                        y[t][q * GP + g] = s[g];
                }
            }
        }
#pragma unroll
        for (int g = 0; g < G; ++g)
            top[g] = fmaxf(top[g], y[t][g]);
    }

    // (a maximum of -inf counts as 0: differences are -inf then, and weights nothing)
    float sum[G];
    if constexpr (PHASE != kWeighAdd) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            top[g] = wave_max(top[g]);
            if (lane == 0)
                red[0][g][wave] = top[g];
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < G; ++g) {
            top[g] = wave_max(red[0][g][lane & (kWeighWaves - 1)]);
            top[g] = top[g] == -INFINITY ? 0.f : top[g];
            sum[g] = 0.f;
        }
#pragma unroll
        for (int t = 0; t < T; ++t)
            if (k0 + t * kWeighThreads < k1)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    y[t][g] = fast_exp2(y[t][g] - top[g]);
                    sum[g] += y[t][g];
                }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            sum[g] = wave_sum(sum[g]);
            if (lane == 0)
                red[1][g][wave] = sum[g];
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kWeighWaves; ++w)
                s += red[1][g][w];
            sum[g] = s;
        }
        if constexpr (PHASE == kWeighStats) {
            if (tid < G) {
                float m = top[0], s = sum[0];
#pragma unroll
                for (int g = 1; g < G; ++g) {
                    m = tid == g ? top[g] : m;
                    s = tid == g ? sum[g] : s;
                }
                // (a range without weight has no maximum)
                a.stats[((int64_t)unit * a.splits + split) * G + tid] = make_float2(s == 0.f ? -INFINITY : m, s);
            }
            return;
        }
    } else {
        const int ranges = (length + a.chunk - 1) / a.chunk;
        const float2 *stats = a.stats + (int64_t)unit * a.splits * G;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float m = -INFINITY, s = 0.f;
            for (int r = lane; r < ranges; r += kWave)
                m = fmaxf(m, stats[r * G + g].x);
            m = wave_max(m);
            m = m == -INFINITY ? 0.f : m;
            for (int r = lane; r < ranges; r += kWave)
                s = fmaf(stats[r * G + g].y, fast_exp2(stats[r * G + g].x - m), s);
            top[g] = m;
            sum[g] = wave_sum(s);
        }
#pragma unroll
        for (int t = 0; t < T; ++t)
            if (k0 + t * kWeighThreads < k1)
#pragma unroll
                for (int g = 0; g < G; ++g)
                    y[t][g] = fast_exp2(y[t][g] - top[g]);
    }
#pragma unroll
    for (int g = 0; g < G; ++g)
        sum[g] = sum[g] == 0.f ? 0.f : 1.f / sum[g];
    float *weights = a.weights + (int64_t)unit * a.weight_stride;
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int key = k0 + t * kWeighThreads + tid;
        if (k0 + t * kWeighThreads < k1 && key < k1 && key < a.columns) {
            float w = y[t][0] * sum[0];
#pragma unroll
            for (int g = 1; g < G; ++g)
                w = fmaf(y[t][g], sum[g], w);
            weights[key] = a.decay == 0.f ? w : fmaf(a.decay, weights[key], w);
        }
    }
}

// ---- keeping the heaviest ----------------------------------------------------------------------------------------
// A first kernel, a workgroup per (sequence, head), finds the weight of the last token that is kept by three passes over its digits (11, 11 and
// 10 bits of the weight as an ordered number, counted in LDS), then lists the kept positions in their order: a wavefront takes consecutive
// tokens, so that counts before its own are all it needs from the others.  A second kernel, a workgroup per (sequence, head, new page), moves
// the tokens: largest value, exponent, rounding.
struct EvictArgs {
    const float *weights;
    const int32_t *table, *lengths, *keep, *table_out;
    float *weights_out;
    int32_t *places;                      // [units, W_out * page] positions of the kept tokens
    int64_t table_stride, weight_stride, out_stride, weight_out_stride;
    int32_t W, W_out, columns, columns_out, first, recent;
};

// Kept tokens of a sequence of n.
__device__ __forceinline__ int kept_of(const EvictArgs &a, int b, int n, int page_log2)
{
    const int k = a.keep[b] < n ? a.keep[b] : n, room = a.W_out << page_log2;
    return k < 0 ? 0 : k < room ? k : room;
}
// A weight as a number that is ordered as weights are; NaN below all others, both zeros one.
__device__ __forceinline__ uint32_t order_of(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);
    return w != w ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / kWave, kPickBins = 2048;

__global__ __launch_bounds__(kPickThreads) void evict_pick_kernel(EvictArgs a, int H, int page_log2)
{
    __shared__ uint32_t bins[kPickBins];
    __shared__ uint32_t sums[kPickWaves];
    __shared__ uint32_t found[2];
    __shared__ int2 counts[kPickWaves];
    const int unit = blockIdx.x, b = unit / H, tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int n = clamp_length(a.lengths[b], a.W, page_log2), k = kept_of(a, b, n, page_log2);
    if (k == 0)
        return;
    const int recent = a.recent < k ? a.recent : k, first = a.first < k - recent ? a.first : k - recent;
    const int last = n - recent;          // tokens [first, last) compete for the places that are left
    int left = k - recent - first;
    const float *weights = a.weights + (int64_t)unit * a.weight_stride;
    auto order_at = [&](int at) -> uint32_t { return order_of(at < a.columns ? weights[at] : 0.f); };
    uint32_t border = 0;                  // digits found so far
    const bool all = left >= last - first;
    if (!all && left > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
            for (int j = tid; j < kPickBins; j += kPickThreads)
                bins[j] = 0;
            __syncthreads();
            for (int at = first + tid; at < last; at += kPickThreads) {
                const uint32_t u = order_at(at);
                if (pass == 0 || (u >> (shift + width)) == border)
                    atomicAdd(&bins[(u >> shift) & ((1u << width) - 1)], 1u);
            }
            __syncthreads();
            // the bin in which the tokens above make `left`: bins from the top, two to a thread
            const int j1 = kPickBins - 1 - 2 * tid, j0 = j1 - 1;
            const uint32_t c1 = bins[j1], c0 = bins[j0];
            uint32_t upto = c1 + c0;
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) {
                const uint32_t x = __shfl_up(upto, d);
                upto += lane >= d ? x : 0;
            }
            if (lane == kWave - 1)
                sums[wave] = upto;
            __syncthreads();
            for (int w = 0; w < wave; ++w)
                upto += sums[w];
            const uint32_t above1 = upto - c1 - c0, above0 = upto - c0, want = (uint32_t)left;
            if (above1 < want && above1 + c1 >= want) {
                found[0] = (uint32_t)j1;
                found[1] = above1;
            } else if (above0 < want && above0 + c0 >= want) {
                found[0] = (uint32_t)j0;
                found[1] = above0;
            }
            __syncthreads();
            border = border << width | found[0];
            left -= (int)found[1];
            __syncthreads();
        }
    }
    // now `left` of the tokens of weight `border` are kept, the lowest, and all above it
    const int each = ((n + kPickWaves - 1) / kPickWaves + kWave - 1) / kWave * kWave;
    const int from = wave * each < n ? wave * each : n, to = from + each < n ? from + each : n;
    // 2: kept, 1: kept if there is room, 0: not
    auto state_of = [&](int at) -> int {
        if (at >= to)
            return 0;
        if (at < first || at >= last || all)
            return 2;
        if (left <= 0 && border == 0)
            return 0;                     // (no place is left for the middle)
        const uint32_t u = order_at(at);
        return u > border ? 2 : u == border ? 1 : 0;
    };
    int above = 0, equal = 0;
    for (int t = from; t < to; t += kWave) {
        const int s = state_of(t + lane);
        above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(s == 2));
        equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(s == 1));
    }
    if (lane == 0)
        counts[wave] = make_int2(above, equal);
    __syncthreads();
    int before = 0, ties = 0;
    for (int w = 0; w < wave; ++w) {
        before += counts[w].x;
        ties += counts[w].y;
    }
    before += ties < left ? ties : left;
    int32_t *places = a.places + (int64_t)unit * ((int64_t)a.W_out << page_log2);
    float *weights_out = a.weights_out ? a.weights_out + (int64_t)unit * a.weight_out_stride : nullptr;
    const uint64_t below = (1ull << lane) - 1;
    for (int t = from; t < to; t += kWave) {
        const int at = t + lane, s = state_of(at);
        const uint64_t tie = __builtin_amdgcn_ballot_w64(s == 1);
        const bool kept = s == 2 || (s == 1 && ties + __builtin_popcountll(tie & below) < left);
        const uint64_t mask = __builtin_amdgcn_ballot_w64(kept);
        const int place = before + __builtin_popcountll(mask & below);
        if (kept) {
            places[place] = at;
            if (weights_out && place < a.columns_out)
                weights_out[place] = at < a.columns ? weights[at] : 0.f;
        }
        before += __builtin_popcountll(mask);
        ties += __builtin_popcountll(tie);
    }
}

constexpr int kMoveThreads = 256;
// grid: (new page of the sequence, head, sequence)
template <int DK, bool FP8>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(PoolArgs p, EvictArgs a)
{
    __shared__ int64_t source[128];       // a token's first byte in the values, or -1
    __shared__ int exps[128];
    __shared__ float tops[kMoveThreads / kWave];
    const int b = blockIdx.z, h = blockIdx.y, slot = blockIdx.x, tid = threadIdx.x;
    const int n = clamp_length(a.lengths[b], a.W, p.page_log2), k = kept_of(a, b, n, p.page_log2);
    const int page = 1 << p.page_log2, j0 = slot << p.page_log2;
    if (j0 >= k)
        return;
    const int to_id = a.table_out[b * a.out_stride + slot];
    if ((uint32_t)to_id >= (uint32_t)p.pages)
        return;
    const int tokens = k - j0 < page ? k - j0 : page;
    const int64_t to = (int64_t)to_id * p.H + h;
    const int32_t *places = a.places + ((int64_t)b * p.H + h) * ((int64_t)a.W_out << p.page_log2) + j0;
    if (tid < page) {
        int64_t at = -1;
        int e = 0;
        if (tid < tokens) {
            const int pos = places[tid], id = a.table[b * a.table_stride + (pos >> p.page_log2)], t = pos & (page - 1);
            if ((uint32_t)id < (uint32_t)p.pages) {
                const int64_t from = (int64_t)id * p.H + h;
                e = p.exponents[from];
                e = e < kLowExponent ? kLowExponent : e > kHighExponent ? kHighExponent : e;
                at = (from << p.page_log2) * DK + (int64_t)(t & ~7) * DK + (t & 7);
                copy_code(p.codes + (to << p.page_log2) * p.m + (int64_t)tid * p.m, p.codes + ((from << p.page_log2) + t) * p.m, p.m, 0);
            }
        }
        source[tid] = at;
        exps[tid] = e;
    }
    __syncthreads();
    const int items = (page / 8) * DK, rounds = (items + kMoveThreads - 1) / kMoveThreads;    // an item: eight tokens of a coordinate
    constexpr int most = 128 / 8 * DK / kMoveThreads;
    uint32_t lo[most], hi[most];
    float top = -1.f;                     // (below zero: no token at all)
#pragma unroll
    for (int r = 0; r < most; ++r) {
        lo[r] = hi[r] = 0;
        if (r >= rounds)
            continue;
        const int item = tid + r * kMoveThreads, octet = item / DK, d = item % DK;
        if (item >= items)
            continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t at = source[octet * 8 + i];
            if (at >= 0) {
                const uint32_t x = p.values[at + d * 8];
                if (i < 4)
                    lo[r] |= x << (8 * i);
                else
                    hi[r] |= x << (8 * (i - 4));
            }
        }
        float x[8];
        unpack4<FP8>(lo[r], *reinterpret_cast<float(*)[4]>(x));
        unpack4<FP8>(hi[r], *reinterpret_cast<float(*)[4]>(x + 4));
#pragma unroll
        for (int i = 0; i < 8; ++i)
            top = source[octet * 8 + i] >= 0 ? fmaxf(top, fabsf(x[i]) * two_to(exps[octet * 8 + i])) : top;
    }
    top = wave_max(top);
    if ((tid & (kWave - 1)) == 0)
        tops[tid / kWave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kMoveThreads / kWave; ++w)
        top = fmaxf(top, tops[w]);
    if (top < 0.f)
        return;
    const int e = exponent_of<FP8>(top);
    uint8_t *values = p.values + (to << p.page_log2) * DK;
#pragma unroll
    for (int r = 0; r < most; ++r) {
        const int item = tid + r * kMoveThreads, octet = item / DK;
        if (r >= rounds || item >= items)
            continue;
        float x[8];
        unpack4<FP8>(lo[r], *reinterpret_cast<float(*)[4]>(x));
        unpack4<FP8>(hi[r], *reinterpret_cast<float(*)[4]>(x + 4));
        uint64_t mask = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] *= two_to(exps[octet * 8 + i] - e);
            mask |= source[octet * 8 + i] >= 0 ? 0xffull << (8 * i) : 0;
        }
        if (!mask)
            continue;
        uint64_t w = (uint64_t)pack4<FP8>(x[4], x[5], x[6], x[7]) << 32 | pack4<FP8>(x[0], x[1], x[2], x[3]);
        uint64_t *dst = reinterpret_cast<uint64_t *>(values) + item;
        if (mask != ~0ull)                // (what lies behind the last token stays)
            w = (w & mask) | (*dst & ~mask);
        *dst = w;
    }
    if (tid == 0)
        p.exponents[to] = (int8_t)e;
}

// ---- host -------------------------------------------------------------------------------------------------------
struct WeighCut {
    int splits, chunk;
};
static WeighCut weigh_cut(const lookat_page_pool *p, int32_t B, int32_t G, int32_t W, int64_t max_length)
{
    const int64_t units = (int64_t)B * p->H, room = (int64_t)W * p->page, longest = max_length > 0 && max_length < room ? max_length : room;
    // Every token in reach has its range: the cut goes by the row's room where the caller's longest length does not hold.
    const int64_t most = weigh_tokens(G);
    int64_t want = units >= 128 ? 1 : (256 + units - 1) / units;
    const int64_t useful = (longest + 2047) / 2048;
    want = want < useful ? want : useful;
    int64_t chunk = (longest + want - 1) / want;
    chunk = (chunk + kWeighThreads - 1) / kWeighThreads * kWeighThreads;
    chunk = chunk < most ? chunk : most;
    WeighCut c;
    c.chunk = (int)chunk;
    c.splits = (int)((room + chunk - 1) / chunk);
    return c;
}
static size_t weigh_bytes(const lookat_page_pool *p, int32_t B, int32_t G, const WeighCut &c)
{
    return c.splits > 1 ? ((size_t)B * p->H * c.splits * G * sizeof(float2) + 15) / 16 * 16 : 0;
}
static int check_weigh(const lookat_page_pool *pool, int32_t B, int32_t group, int32_t W, int64_t max_length)
{
    if (int rc = check_pool(pool))
        return rc;
    if (B <= 0 || W <= 0)
        return fail(LOOKAT_ERR_SHAPE, "B=%d and W=%d must be positive", B, W);
    if (group != 1 && group != 2 && group != 4 && group != 8)
        return fail(LOOKAT_ERR_UNSUPPORTED, "group=%d: query heads per key/value head must be 1, 2, 4 or 8", group);
    if (B > 65535 || (int64_t)W * pool->page > (1 << 30))
        return fail(LOOKAT_ERR_UNSUPPORTED, "B=%d, W=%d pages of %d tokens: at most 65535 sequences of 2^30 tokens", B, W, pool->page);
    if (max_length < 0)
        return fail(LOOKAT_ERR_SHAPE, "max_length=%lld must not be negative", (long long)max_length);
    return LOOKAT_OK;
}

template <int M, int G, int PHASE>
static int launch_weigh_phase(const PoolArgs &p, const WeighArgs &a, int64_t groups, hipStream_t st)
{
    constexpr size_t lds = (size_t)G * M * kCentroids * 4;
    const auto f = &weigh_kernel<M, G, PHASE>;
    if (lds > 60 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(f), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess)
            return fail(LOOKAT_ERR_HIP, "lookat_pages_weigh: %s", hipGetErrorString(e));
    }
    hipLaunchKernelGGL(f, dim3((unsigned)groups), dim3(kWeighThreads), lds, st, p, a);
    return check_launch("lookat_pages_weigh");
}
template <int M, int G>
static int launch_weigh(const PoolArgs &p, const WeighArgs &a, int64_t groups, hipStream_t st)
{
    if (a.splits == 1)
        return launch_weigh_phase<M, G, kWeighAll>(p, a, groups, st);
    if (int rc = launch_weigh_phase<M, G, kWeighStats>(p, a, groups, st))
        return rc;
    return launch_weigh_phase<M, G, kWeighAdd>(p, a, groups, st);
}
template <int M>
static int launch_weigh_g(int G, const PoolArgs &p, const WeighArgs &a, int64_t groups, hipStream_t st)
{
    switch (G) {
    case 1: return launch_weigh<M, 1>(p, a, groups, st);
    case 2: return launch_weigh<M, 2>(p, a, groups, st);
    case 4: return launch_weigh<M, 4>(p, a, groups, st);
    default: return launch_weigh<M, 8>(p, a, groups, st);
    }
}

static int check_evict(const lookat_page_pool *pool, int32_t B, int32_t W, int32_t W_out)
{
    if (int rc = check_pool(pool))
        return rc;
    if (B <= 0 || W <= 0 || W_out <= 0)
        return fail(LOOKAT_ERR_SHAPE, "B=%d, W=%d and W_out=%d must be positive", B, W, W_out);
    if (B > 65535 || (int64_t)W * pool->page > (1 << 30) || (int64_t)W_out * pool->page > (1 << 30))
        return fail(LOOKAT_ERR_UNSUPPORTED, "B=%d, W=%d, W_out=%d pages of %d tokens: at most 65535 sequences of 2^30 tokens", B, W, W_out, pool->page);
    return LOOKAT_OK;
}
static size_t evict_bytes(const lookat_page_pool *p, int32_t B, int32_t W_out) { return (size_t)B * p->H * W_out * p->page * 4; }

}  // namespace lookat

extern "C" size_t lookat_pages_weigh_workspace_bytes(const lookat_page_pool *pool, int32_t B, int32_t group, int32_t W, int64_t max_length)
{
    using namespace lookat;
    clear_error();
    if (check_weigh(pool, B, group, W, max_length) != LOOKAT_OK)
        return 0;
    return weigh_bytes(pool, B, group, weigh_cut(pool, B, group, W, max_length));
}

extern "C" int lookat_pages_weigh(const lookat_page_pool *pool, int32_t B, int32_t group, const float *lut, const int32_t *table, int32_t W,
                                  int64_t table_stride, const int32_t *lengths, int64_t max_length, float scale, float decay, float *weights,
                                  int32_t columns, int64_t weight_stride_bh, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_weigh(pool, B, group, W, max_length))
        return rc;
    if (int rc = check_table(pool, "B", B, table, W, table_stride))
        return rc;
    if (columns <= 0 || weight_stride_bh < columns)
        return fail(LOOKAT_ERR_SHAPE, "columns=%d must be positive and weight_stride_bh=%lld no smaller", columns, (long long)weight_stride_bh);
    if (!lut || !lengths || !weights)
        return fail(LOOKAT_ERR_NULL, "lut, lengths and weights must be non-NULL");
    if (!aligned16(lut))
        return fail(LOOKAT_ERR_ALIGN, "lut must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(lengths) | reinterpret_cast<uintptr_t>(weights)) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "lengths and weights must be 4-byte aligned");
    const WeighCut cut = weigh_cut(pool, B, group, W, max_length);
    const size_t need = weigh_bytes(pool, B, group, cut);
    if (need) {
        if (!workspace || workspace_bytes < need)
            return fail(LOOKAT_ERR_WORKSPACE, "workspace of %zu bytes needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
        if (!aligned16(workspace))
            return fail(LOOKAT_ERR_ALIGN, "workspace must be 16-byte aligned");
    }
    const int64_t units = (int64_t)B * pool->H, groups = (units + kXcds - 1) / kXcds * kXcds * cut.splits;
    if (!fits_launch(groups, kWeighThreads))
        return fail(LOOKAT_ERR_UNSUPPORTED, "B*H*ranges: %lld workgroups exceed one launch", (long long)groups);
    const PoolArgs p = pool_args(pool);
    WeighArgs a;
    a.lut = lut;
    a.table = table;
    a.lengths = lengths;
    a.weights = weights;
    a.stats = static_cast<float2 *>(workspace);
    a.table_stride = table_stride;
    a.weight_stride = weight_stride_bh;
    a.W = W;
    a.columns = columns;
    a.units = (int32_t)units;
    a.splits = cut.splits;
    a.chunk = cut.chunk;
    a.scale_log2e = scale * kLog2e;
    a.decay = decay;
    hipStream_t st = static_cast<hipStream_t>(stream);
    switch (p.m) {
    case 2: return launch_weigh_g<2>(group, p, a, groups, st);
    case 4: return launch_weigh_g<4>(group, p, a, groups, st);
    case 8: return launch_weigh_g<8>(group, p, a, groups, st);
    default: return launch_weigh_g<16>(group, p, a, groups, st);
    }
}

extern "C" size_t lookat_pages_evict_workspace_bytes(const lookat_page_pool *pool, int32_t B, int32_t W_out)
{
    using namespace lookat;
    clear_error();
    if (check_evict(pool, B, 1, W_out) != LOOKAT_OK)
        return 0;
    return evict_bytes(pool, B, W_out);
}

extern "C" int lookat_pages_evict(const lookat_page_pool *pool, int32_t B, const int32_t *table, int32_t W, int64_t table_stride, const int32_t *lengths,
                                  const float *weights, int32_t columns, int64_t weight_stride_bh, const int32_t *keep, int32_t first, int32_t recent,
                                  const int32_t *table_out, int32_t W_out, int64_t table_out_stride, float *weights_out, int32_t columns_out,
                                  int64_t weight_out_stride_bh, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_evict(pool, B, W, W_out))
        return rc;
    if (int rc = check_table(pool, "B", B, table, W, table_stride))
        return rc;
    if (int rc = check_table(pool, "B", B, table_out, W_out, table_out_stride))
        return rc;
    if (columns <= 0 || weight_stride_bh < columns)
        return fail(LOOKAT_ERR_SHAPE, "columns=%d must be positive and weight_stride_bh=%lld no smaller", columns, (long long)weight_stride_bh);
    if (weights_out && (columns_out <= 0 || weight_out_stride_bh < columns_out))
        return fail(LOOKAT_ERR_SHAPE, "columns_out=%d must be positive and weight_out_stride_bh=%lld no smaller", columns_out,
                    (long long)weight_out_stride_bh);
    if (first < 0 || recent < 0)
        return fail(LOOKAT_ERR_SHAPE, "first=%d and recent=%d must not be negative", first, recent);
    if (!lengths || !weights || !keep)
        return fail(LOOKAT_ERR_NULL, "lengths, weights and keep must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(lengths) | reinterpret_cast<uintptr_t>(weights) | reinterpret_cast<uintptr_t>(keep) |
         reinterpret_cast<uintptr_t>(weights_out)) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "lengths, weights, keep and weights_out must be 4-byte aligned");
    const size_t need = evict_bytes(pool, B, W_out);
    if (!workspace || workspace_bytes < need)
        return fail(LOOKAT_ERR_WORKSPACE, "workspace of %zu bytes needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
    if (!aligned16(workspace))
        return fail(LOOKAT_ERR_ALIGN, "workspace must be 16-byte aligned");
    const int64_t units = (int64_t)B * pool->H;
    if (!fits_launch(units, kPickThreads) || !fits_launch(W_out, kMoveThreads))
        return fail(LOOKAT_ERR_UNSUPPORTED, "B*H=%lld heads or W_out=%d pages exceed one launch", (long long)units, W_out);
    const PoolArgs p = pool_args(pool);
    EvictArgs a;
    a.weights = weights;
    a.table = table;
    a.lengths = lengths;
    a.keep = keep;
    a.table_out = table_out;
    a.weights_out = weights_out;
    a.places = static_cast<int32_t *>(workspace);
    a.table_stride = table_stride;
    a.weight_stride = weight_stride_bh;
    a.out_stride = table_out_stride;
    a.weight_out_stride = weight_out_stride_bh;
    a.W = W;
    a.W_out = W_out;
    a.columns = columns;
    a.columns_out = columns_out;
    a.first = first;
    a.recent = recent;
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(evict_pick_kernel, dim3((unsigned)units), dim3(kPickThreads), 0, st, a, p.H, p.page_log2);
    if (int rc = check_launch("lookat_pages_evict (choice)"))
        return rc;
    const bool fp8 = pool->value_type == LOOKAT_VALUES_E4M3;
    const auto f = p.d_k == 64 ? (fp8 ? &evict_move_kernel<64, true> : &evict_move_kernel<64, false>)
                               : (fp8 ? &evict_move_kernel<128, true> : &evict_move_kernel<128, false>);
    hipLaunchKernelGGL(f, dim3((unsigned)W_out, (unsigned)p.H, (unsigned)B), dim3(kMoveThreads), 0, st, p, a);
    return check_launch("lookat_pages_evict");
}
