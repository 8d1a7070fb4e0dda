// Holding a cache to a budget: every token's sum of the attention it was paid, and moving the heaviest tokens into fewer pages.
#include <type_traits>

#include "pages_quantise.h"
#include "decode_common.h"

namespace lookat {

// ---- attention sums ---------------------------------------------------------------------------------------------
//   w_l = decay w_l + sum_g 2^(y_gl - M_g) / Z_g,   y_gl = scale log2(e) sum_i lut_gi[code_li],   M_g = max_l y_gl,  Z_g = sum_l 2^(y_gl - M_g)
//
// A workgroup of 1024 or 256 threads takes a range of one (sequence, key/value head): its scores stay in registers (kWeighScores a thread, over
// the group's query heads) from the maximum to the weights, so that codes are read and looked up once.  Where one range does not hold a sequence or
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

constexpr int kWeighThreads = 1024, kWeighSmall = 256, kWeighScores = 32, kWeighFew = 4;
__host__ __device__ constexpr int weigh_tokens(int G, int threads) { return threads * (kWeighScores / G); }     // of a range, at most
__host__ __device__ constexpr int weigh_few(int G) { return kWeighFew / G > 0 ? kWeighFew / G : 1; }                          // scores of a thread in the short code

enum WeighPhase { kWeighAll, kWeighStats, kWeighAdd };

template <int M, int G, int PHASE, int T, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void weigh_kernel(PoolArgs p, WeighArgs a)
{
    constexpr int WAVES = THREADS / kWave;
    constexpr int GP = G < 4 ? G : 4, PLANES = G / GP;
    typedef float vg __attribute__((ext_vector_type(GP)));
    extern __shared__ __align__(16) float tables[];       // [plane][i][c][head of the plane]
    __shared__ float red[2][G][WAVES];
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
    const uint32_t code_step = (uint32_t)(p.H * M) << p.page_log2;
    const uint8_t *head_codes = p.codes + ((uint32_t)(h * M) << p.page_log2);

    // The first tokens' pages and codes are requested ahead of the tables, the old weights behind them: they are needed last.  Then one group of
    // tokens is requested while the one before it is looked up.
    constexpr int WORDS = (M + 3) / 4, most = WORDS == 4 || G == 8 ? 2 : 4, U = T < most ? T : most;
    static_assert(T % U == 0, "whole groups");
    uint32_t codes[2][U][WORDS];
    bool there[2][U];
    auto request = [&](int t0) {
        int id[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int key = k0 + (t0 + u) * THREADS + tid;
            id[u] = row[(key < k1 ? key : k1 - 1) >> p.page_log2];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int key = k0 + (t0 + u) * THREADS + tid;
            there[t0 / U & 1][u] = key < k1 && (uint32_t)id[u] < (uint32_t)p.pages;
            const uint8_t *c = head_codes + (uint64_t)(uint32_t)(there[t0 / U & 1][u] ? id[u] : 0) * code_step + (uint32_t)(key & page_mask) * M;
            if constexpr (M == 2) {
                codes[t0 / U & 1][u][0] = *reinterpret_cast<const uint16_t *>(c);
            } else if constexpr (M == 4) {
                codes[t0 / U & 1][u][0] = *reinterpret_cast<const uint32_t *>(c);
            } else if constexpr (M == 8) {
                const v2u x = *reinterpret_cast<const v2u *>(c);
                codes[t0 / U & 1][u][0] = x.x, codes[t0 / U & 1][u][1] = x.y;
            } else {
                const v4u x = *reinterpret_cast<const v4u *>(c);
                codes[t0 / U & 1][u][0] = x.x, codes[t0 / U & 1][u][1] = x.y, codes[t0 / U & 1][u][2] = x.z, codes[t0 / U & 1][u][3] = x.w;
            }
        }
    };
    request(0);
    {
        const v4f *lut = reinterpret_cast<const v4f *>(a.lut + (int64_t)unit * G * M * kCentroids);
        for (int j = tid; j < PLANES * M * (kCentroids / 4); j += THREADS) {
            const int plane = j / (M * (kCentroids / 4)), entry = j % (M * (kCentroids / 4));
            v4f x[GP];
#pragma unroll
            for (int g = 0; g < GP; ++g)
                x[g] = lut[(plane * GP + g) * (M * (kCentroids / 4)) + entry];
#pragma unroll
            for (int k = 0; k < GP; ++k) {                // ordered entry, head
                v4f y;
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    y[w] = x[(4 * k + w) % GP][(4 * k + w) / GP] * a.scale_log2e;
                reinterpret_cast<v4f *>(tables)[j * GP + k] = y;
            }
        }
    }
    float *weights = a.weights + (int64_t)unit * a.weight_stride;
    float old[T];
    if constexpr (PHASE != kWeighStats) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int key = k0 + t * THREADS + tid;
            old[t] = a.decay != 0.f && key < k1 && key < a.columns ? weights[key] : 0.f;
        }
    }
    __syncthreads();

    float y[T][G], top[G];
#pragma unroll
    for (int g = 0; g < G; ++g)
        top[g] = -INFINITY;
#pragma unroll
    for (int t0 = 0; t0 < T; t0 += U) {
        if (k0 + t0 * THREADS >= k1) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int g = 0; g < G; ++g)
                    y[t0 + u][g] = -INFINITY;
            continue;
        }
        if (t0 + U < T && k0 + (t0 + U) * THREADS < k1)
            request(t0 + U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int q = 0; q < PLANES; ++q) {
                vg s = {};
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    if (G * M >= 16 && i % (16 / GP) == 0)
                        __builtin_amdgcn_sched_barrier(0);        // (look-ups in flight at once: 16 registers of them)
                    s += reinterpret_cast<const vg *>(tables)[(q * M + i) * kCentroids + ((codes[t0 / U & 1][u][i / 4] >> (8 * (i % 4))) & 0xffu)];
                }
#pragma unroll
                for (int g = 0; g < GP; ++g) {
                    const float x = GP == 1 ? (float)s[0] : (float)s[g];
                    y[t0 + u][q * GP + g] = there[t0 / U & 1][u] ? x : -INFINITY;
                    if constexpr (PHASE == kWeighAdd)
                        asm volatile("" : "+v"(y[t0 + u][q * GP + g]));   // (summed up here: not all terms kept until the maximum is known)
                    else
                        top[q * GP + g] = fmaxf(top[q * GP + g], y[t0 + u][q * GP + g]);
                }
            }
        }
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
            top[g] = wave_max(red[0][g][lane & (WAVES - 1)]);
            top[g] = top[g] == -INFINITY ? 0.f : top[g];
            sum[g] = 0.f;
        }
#pragma unroll
        for (int t = 0; t < T; ++t)
            if (k0 + t * THREADS < k1)
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
            sum[g] = wave_sum(lane < WAVES ? red[1][g][lane] : 0.f);
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
#pragma unroll 1
            for (int r = lane; r < ranges; r += kWave)
                m = fmaxf(m, stats[r * G + g].x);
            m = wave_max(m);
            m = m == -INFINITY ? 0.f : m;
#pragma unroll 1
            for (int r = lane; r < ranges; r += kWave)
                s = fmaf(stats[r * G + g].y, fast_exp2(stats[r * G + g].x - m), s);
            top[g] = m;
            sum[g] = wave_sum(s);
        }
#pragma unroll
        for (int t = 0; t < T; ++t)
            if (k0 + t * THREADS < k1)
#pragma unroll
                for (int g = 0; g < G; ++g)
                    y[t][g] = fast_exp2(y[t][g] - top[g]);
    }
#pragma unroll
    for (int g = 0; g < G; ++g)
        sum[g] = sum[g] == 0.f ? 0.f : 1.f / sum[g];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int key = k0 + t * THREADS + tid;
        if (k0 + t * THREADS < k1 && key < k1 && key < a.columns) {
            float w = y[t][0] * sum[0];
#pragma unroll
            for (int g = 1; g < G; ++g)
                w = fmaf(y[t][g], sum[g], w);
            weights[key] = a.decay == 0.f ? w : fmaf(a.decay, old[t], w);
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

__device__ __forceinline__ int ballot_count(bool b) { return __builtin_popcountll(__builtin_amdgcn_ballot_w64(b)); }

constexpr int kPickThreads = 1024, kPickSmall = 256, kPickBins = 2048;

// KEYS: the weights of up to so many tokens a thread stay in registers; 0: they are read again in every pass.  Token i * THREADS + tid is the thread's i-th.
template <int KEYS, int THREADS>
__global__ __launch_bounds__(THREADS) void evict_pick_kernel(EvictArgs a, int H, int page_log2)
{
    constexpr int kPickWaves = THREADS / kWave, kPickCopies = THREADS / 256, kBinsEach = kPickBins / THREADS;
    __shared__ __align__(16) uint32_t bins[kPickBins * kPickCopies];    // (a bin's copies side by side: many tokens have the same weight, zero among them)
    __shared__ uint32_t sums[kPickWaves];
    __shared__ uint32_t found[2];
    constexpr bool HELD = KEYS > 0;
    constexpr int kPickKeys = HELD ? KEYS : 1, kEach = (kPickKeys * kPickWaves + kWave - 1) / kWave;
    __shared__ uint32_t counts[2][kPickKeys * kPickWaves];
    const int unit = blockIdx.x, b = unit / H, tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int n = clamp_length(a.lengths[b], a.W, page_log2), k = kept_of(a, b, n, page_log2);
    if (k == 0)
        return;
    // The k greatest of n: tokens that are kept whatever they weigh count above all weights.  What is behind the last token counts as the least, and
    // is never reached: among equal ones the lowest positions go first, and k <= n.
    const int recent = a.recent < k ? a.recent : k, first = a.first < k - recent ? a.first : k - recent, last = n - recent;
    int left = k;
    const float *weights = a.weights + (int64_t)unit * a.weight_stride;
    auto weight_at = [&](int at) -> float { return at < n && at < a.columns ? weights[at] : 0.f; };
    auto order_at = [&](int at, float w) -> uint32_t { return at >= n ? 0 : at < first || at >= last ? 0xffffffffu : order_of(w); };
    float held_w[kPickKeys];
    uint32_t held[kPickKeys];
    if constexpr (HELD) {
#pragma unroll
        for (int i = 0; i < kPickKeys; ++i)
            held_w[i] = i * THREADS < n ? weight_at(i * THREADS + tid) : 0.f;
#pragma unroll
        for (int i = 0; i < kPickKeys; ++i)
            held[i] = order_at(i * THREADS + tid, held_w[i]);
    }
    // f(token, its order, its weight, index) for every token of this thread
    auto each = [&](auto f) {
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < kPickKeys; ++i)
                if (i * THREADS < n)
                    f(i * THREADS + tid, held[i], held_w[i], i);
        } else {
            for (int64_t at = tid, i = 0; at - tid < n; at += THREADS, ++i) {
                const float w = weight_at((int)at);
                f((int)at, order_at((int)at, w), w, (int)i);
            }
        }
    };
    uint32_t border = 0;                  // digits found so far
    for (int j = tid; j < kPickBins * kPickCopies; j += THREADS)
        bins[j] = 0;
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        constexpr int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
        const int shift = shifts[pass], width = widths[pass];
        each([&](int, uint32_t u, float, int) {
            if (pass == 0 || (u >> (shift + width)) == border)
                atomicAdd(&bins[((u >> shift) & ((1u << width) - 1)) * kPickCopies + (lane & (kPickCopies - 1))], 1u);
        });
        __syncthreads();
        // the bin in which the tokens above make `left`: bins from the top, kBinsEach to a thread, cleared for the next pass
        const int low = kPickBins - (tid + 1) * kBinsEach;
        static_assert(kBinsEach * kPickCopies == 8, "two loads");
        u32x4 *mine = reinterpret_cast<u32x4 *>(bins + low * kPickCopies);
        const u32x4 words[2] = {mine[0], mine[1]};
        mine[0] = mine[1] = (u32x4){0, 0, 0, 0};
        uint32_t c[kBinsEach], upto = 0;
#pragma unroll
        for (int j = 0; j < kBinsEach; ++j) {
            c[j] = 0;
#pragma unroll
            for (int x = j * kPickCopies; x < (j + 1) * kPickCopies; ++x)
                c[j] += words[x / 4][x % 4];
            upto += c[j];
        }
        const uint32_t total = upto;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const uint32_t x = __shfl_up(upto, d);
            upto += lane >= d ? x : 0;
        }
        if (lane == kWave - 1)
            sums[wave] = upto;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kPickWaves; ++w)
            upto += w < wave ? sums[w] : 0;
        uint32_t above = upto - total;
#pragma unroll
        for (int j = kBinsEach - 1; j >= 0; --j) {
            if (above < (uint32_t)left && above + c[j] >= (uint32_t)left) {
                found[0] = (uint32_t)(low + j);
                found[1] = above;
            }
            above += c[j];
        }
        __syncthreads();
        border = border << width | found[0];
        left -= (int)found[1];
    }
    // Now all tokens above `border` are kept (sure), and of those at it (ties) the `left` lowest.
    int32_t *places = a.places + (int64_t)unit * ((int64_t)a.W_out << page_log2);
    float *weights_out = a.weights_out ? a.weights_out + (int64_t)unit * a.weight_out_stride : nullptr;
    const uint64_t below = (1ull << lane) - 1;
    // A place is the number of kept tokens before one: `above` and `equal` of those before these 64.
    auto store = [&](int at, uint32_t u, float w, int above, int equal) {
        const bool sure = u > border, tie = u == border;
        const uint64_t sures = __builtin_amdgcn_ballot_w64(sure), tied = __builtin_amdgcn_ballot_w64(tie);
        const int ties = equal + __builtin_popcountll(tied & below);
        if (sure || (tie && ties < left)) {
            const int place = above + __builtin_popcountll(sures & below) + (ties < left ? ties : left);
            places[place] = at;
            if (weights_out && place < a.columns_out)
                weights_out[place] = w;
        }
    };
    if constexpr (HELD) {
        // counts of every 64 tokens, then their sums, then the places
        each([&](int, uint32_t u, float, int i) {
            const int sures = ballot_count(u > border), ties = ballot_count(u == border);
            if (lane == 0) {
                counts[0][i * kPickWaves + wave] = sures;
                counts[1][i * kPickWaves + wave] = ties;
            }
        });
        __syncthreads();
        // (two wavefronts, one for each kind, up to eight counts a lane; those of tokens that are not there are left out)
        if (wave < 2) {
            const int used = (n + THREADS - 1) / THREADS * kPickWaves;
            uint32_t c[kEach], total = 0;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                c[j] = lane * kEach + j < used ? counts[wave][lane * kEach + j] : 0;
                total += c[j];
            }
            uint32_t upto = total;
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) {
                const uint32_t x = __shfl_up(upto, d);
                upto += lane >= d ? x : 0;
            }
            upto -= total;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                if (lane * kEach + j < used)
                    counts[wave][lane * kEach + j] = upto;
                upto += c[j];
            }
        }
        __syncthreads();
        each([&](int at, uint32_t u, float w, int i) { store(at, u, w, (int)counts[0][i * kPickWaves + wave], (int)counts[1][i * kPickWaves + wave]); });
    } else {
        // 1024 tokens at a time
        int above_all = 0, equal_all = 0;
        each([&](int at, uint32_t u, float w, int) {
            const int sures = ballot_count(u > border), ties = ballot_count(u == border);
            __syncthreads();              // (the last counts were read)
            if (lane == 0) {
                counts[0][wave] = sures;
                counts[1][wave] = ties;
            }
            __syncthreads();
            int above = above_all, equal = equal_all;
#pragma unroll
            for (int x = 0; x < kPickWaves; ++x) {
                above += x < wave ? counts[0][x] : 0;
                equal += x < wave ? counts[1][x] : 0;
                above_all += counts[0][x];
                equal_all += counts[1][x];
            }
            store(at, u, w, above, equal);
        });
    }
}

// Moving.  A token is one byte in eight of what a page holds for its octet and coordinate, so octets are read whole, a lane per coordinate, 512
// consecutive bytes a wavefront, and a new octet is put together from the octets that its tokens come from (mostly two or three) by byte permutes
// whose selectors are the same for all lanes.  A wavefront takes 64 new tokens (128 where a page has as many), a lane each while it is found out where
// they are; no wavefront waits for another.  The bytes stay in registers until the largest value, and with it the exponent, is known; where all
// tokens of an octet had that exponent they are stored as they are.
constexpr int kMoveWaves = 4, kMoveThreads = kMoveWaves * kWave;
constexpr int kMoveAhead = 3;             // octets requested at once for a new one
constexpr int kMoveBatch = 2;             // new octets (64 coordinates of them) whose octets are requested together
constexpr int kMixed = 127;               // no exponent: the tokens of an octet have several

struct MoveSource {
    int64_t at;                           // an octet's first byte in the values
    uint32_t lo, hi;                      // where its bytes go in the new octet: selectors of v_perm_b32, 12 for none
};
typedef short v2s __attribute__((ext_vector_type(2)));

// The largest |stored| of eight bytes as a number of fp32; e4m3's NaN counts above all.
template <bool FP8>
__device__ __forceinline__ float largest(uint32_t lo, uint32_t hi)
{
    if constexpr (FP8) {
        // (without their signs the bytes are ordered as the numbers)
        const v2s a = __builtin_bit_cast(v2s, lo & 0x007f007fu), b = __builtin_bit_cast(v2s, lo >> 8 & 0x007f007fu);
        const v2s c = __builtin_bit_cast(v2s, hi & 0x007f007fu), d = __builtin_bit_cast(v2s, hi >> 8 & 0x007f007fu);
        const v2s m = __builtin_elementwise_max(__builtin_elementwise_max(a, b), __builtin_elementwise_max(c, d));
        const int top = m.x > m.y ? m.x : m.y;
        return top == 0x7f ? INFINITY : __builtin_amdgcn_cvt_f32_fp8(top, 0);
    } else {
        const v2s l = __builtin_bit_cast(v2s, lo), h = __builtin_bit_cast(v2s, hi);
        const v2s a = (l << 8) >> 8, b = l >> 8, c = (h << 8) >> 8, d = h >> 8;
        const v2s most = __builtin_elementwise_max(__builtin_elementwise_max(a, b), __builtin_elementwise_max(c, d));
        const v2s least = __builtin_elementwise_min(__builtin_elementwise_min(a, b), __builtin_elementwise_min(c, d));
        const int x = most.x > most.y ? most.x : most.y, y = least.x < least.y ? least.x : least.y;
        return (float)(x > -y ? x : -y);
    }
}

// Four stored numbers, none of them NaN, times a power of two after which none is above the largest.
template <bool FP8>
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f)
{
    if constexpr (FP8) {
        const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, f, true);
        const int r = __builtin_amdgcn_cvt_pk_fp8_f32(a.x, a.y, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b.x, b.y, r, true);
    } else {
        float x[4];
        unpack4<FP8>(w, x);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] *= f;
        return pack4<FP8>(x[0], x[1], x[2], x[3]);
    }
}

// grid: (new pages of the sequence in fours of wavefronts, head, sequence)
template <int DK, bool FP8, int PAGE>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(PoolArgs p, EvictArgs a)
{
    constexpr int TOKENS = PAGE > kWave ? PAGE : kWave;
    constexpr int EACH = TOKENS / kWave, PAGES = TOKENS / PAGE, OCTETS = TOKENS / 8, CB = DK / kWave;
    constexpr int PIECES = PAGE / 8 * CB, BATCHES = PIECES / kMoveBatch;     // of a page
    constexpr int page_log2 = PAGE == 16 ? 4 : PAGE == 32 ? 5 : PAGE == 64 ? 6 : 7;
    __shared__ MoveSource sources_s[kMoveWaves][TOKENS];
    __shared__ __align__(16) float scales_s[kMoveWaves][TOKENS];      // 2^exponent
    __shared__ int octet_e_s[kMoveWaves][OCTETS], octet_n_s[kMoveWaves][OCTETS];
    __shared__ uint32_t octet_has_s[kMoveWaves][OCTETS];  // a bit for every token
    const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    MoveSource *sources = sources_s[wave];
    float *scales = scales_s[wave];
    int *octet_e = octet_e_s[wave], *octet_n = octet_n_s[wave];
    uint32_t *octet_has = octet_has_s[wave];
    const int n = clamp_length(a.lengths[b], a.W, page_log2), k = kept_of(a, b, n, page_log2);
    const int slot0 = (int)(blockIdx.x * kMoveWaves + wave) * PAGES, j0 = slot0 * PAGE;
    if (j0 >= k)
        return;
    const int32_t *places = a.places + ((int64_t)b * p.H + h) * ((int64_t)a.W_out << page_log2);
    const int32_t *row = a.table + b * a.table_stride, *row_out = a.table_out + b * a.out_stride;
    int pos[EACH], id[EACH], to_id[EACH], exponent[EACH];
#pragma unroll
    for (int g = 0; g < EACH; ++g) {
        const int j = j0 + g * kWave + lane;
        pos[g] = j < k ? places[j] : -1;
        to_id[g] = j < k ? row_out[j >> page_log2] : -1;
    }
#pragma unroll
    for (int g = 0; g < EACH; ++g) {
        id[g] = pos[g] >= 0 ? row[pos[g] >> page_log2] : -1;
        if ((uint32_t)id[g] >= (uint32_t)p.pages || (uint32_t)to_id[g] >= (uint32_t)p.pages)
            id[g] = -1;
    }
    const int first = lane & ~7, me = lane & 7;
#pragma unroll
    for (int g = 0; g < EACH; ++g) {
        const int t = pos[g] & (PAGE - 1), token = g * kWave + lane;
        const int64_t from = (int64_t)(id[g] < 0 ? 0 : id[g]) * p.H + h;
        const int64_t at = id[g] < 0 ? -1 : ((from << page_log2) + (t & ~7)) * DK;
        exponent[g] = p.exponents[from];
        // the octets that this octet's eight tokens come from, one entry for each, written by its first token
        const uint32_t has = (uint32_t)(__builtin_amdgcn_ballot_w64(at >= 0) >> first) & 0xff;
        uint32_t sel[2] = {0, 0};
        bool leads = at >= 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t other = __shfl(at, first + i);
            const int other_t = __shfl(t, first + i);
            sel[i / 4] |= (uint32_t)(other == at ? other_t & 7 : 12) << (8 * (i % 4));
            leads = leads && !(i < me && other == at);
        }
        const uint32_t heads = (uint32_t)(__builtin_amdgcn_ballot_w64(leads) >> first) & 0xff;
        // (the entries behind them name bytes that are there and take none: every new octet requests as many, without a branch, so that what is
        // waited for is counted)
        const int used = __builtin_popcount(heads);
        MoveSource s = {0, 0x0c0c0c0cu, 0x0c0c0c0cu};
        if (me >= used)
            sources[token] = s;
        if (leads) {
            s.at = at;
            s.lo = sel[0];
            s.hi = sel[1];
            sources[(token & ~7) + __builtin_popcount(heads & ((1u << me) - 1))] = s;
        }
        if (me == 0) {
            octet_n[token / 8] = used;
            octet_has[token / 8] = has;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

    uint8_t *values = p.values;
    uint64_t ahead[2][kMoveBatch][kMoveAhead];
    auto request = [&](int octet0, int batch) {
#pragma unroll
        for (int r = 0; r < kMoveBatch; ++r) {
            const int piece = batch * kMoveBatch + r, octet = octet0 + piece / CB, d = piece % CB * kWave + lane;
#pragma unroll
            for (int i = 0; i < kMoveAhead; ++i)
                ahead[batch & 1][r][i] = *reinterpret_cast<const uint64_t *>(values + sources[octet * 8 + i].at + d * 8);
        }
    };
    request(0, 0);
    // (while the octets are on their way: the tokens' exponents and codes)
#pragma unroll
    for (int g = 0; g < EACH; ++g) {
        const int e = exponent[g] < kLowExponent ? kLowExponent : exponent[g] > kHighExponent ? kHighExponent : exponent[g], token = g * kWave + lane;
        const uint32_t has = (uint32_t)(__builtin_amdgcn_ballot_w64(id[g] >= 0) >> first) & 0xff;
        scales[token] = two_to(e);
        bool same = true;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int other_e = __shfl(e, first + i);     // (by all lanes)
            same = same && (!(has >> i & 1) || other_e == e);
        }
        if (has ? me == __builtin_ctz(has) : me == 0)
            octet_e[token / 8] = same ? e : kMixed;
        if (id[g] >= 0) {
            const int64_t from = ((int64_t)id[g] * p.H + h) << page_log2, to = ((int64_t)to_id[g] * p.H + h) << page_log2;
            copy_code(p.codes + (to + (token & (PAGE - 1))) * p.m, p.codes + (from + (pos[g] & (PAGE - 1))) * p.m, p.m, 0);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

#pragma unroll 1
    for (int x = 0; x < PAGES; ++x) {
        const int octet0 = x * (PAGE / 8);
        uint32_t lo[PIECES], hi[PIECES];
        float most = -1.f;                // (below zero: no token at all)
        uint32_t odd = 0;                 // pieces that have to be looked at token by token: several exponents, NaN
        if (x > 0)
            request(octet0, 0);
#pragma unroll
        for (int batch = 0; batch < BATCHES; ++batch) {
            if (batch + 1 < BATCHES)
                request(octet0, batch + 1);
#pragma unroll
            for (int r = 0; r < kMoveBatch; ++r) {
                const int piece = batch * kMoveBatch + r, octet = octet0 + piece / CB, d = piece % CB * kWave + lane;
                lo[piece] = hi[piece] = 0;
                const int count = __builtin_amdgcn_readfirstlane(octet_n[octet]);
                auto take = [&](const MoveSource &s, uint64_t y) {
                    lo[piece] |= __builtin_amdgcn_perm((uint32_t)(y >> 32), (uint32_t)y, s.lo);
                    hi[piece] |= __builtin_amdgcn_perm((uint32_t)(y >> 32), (uint32_t)y, s.hi);
                };
#pragma unroll
                for (int i = 0; i < kMoveAhead; ++i)
                    take(sources[octet * 8 + i], ahead[batch & 1][r][i]);
                auto take_more = [&](auto upto) {
                    constexpr int N = decltype(upto)::value;
                    uint64_t more[N - kMoveAhead];
#pragma unroll
                    for (int i = kMoveAhead; i < N; ++i)
                        more[i - kMoveAhead] = *reinterpret_cast<const uint64_t *>(values + sources[octet * 8 + i].at + d * 8);
#pragma unroll
                    for (int i = kMoveAhead; i < N; ++i)
                        take(sources[octet * 8 + i], more[i - kMoveAhead]);
                };
                // (the others at once: few kept tokens come from as many octets)
                if (count > kMoveAhead + 1)
                    take_more(std::integral_constant<int, 8>());
                else if (count > kMoveAhead)
                    take_more(std::integral_constant<int, kMoveAhead + 1>());
                if (!count)
                    continue;
                const int e = __builtin_amdgcn_readfirstlane(octet_e[octet]);
                const float y = largest<FP8>(lo[piece], hi[piece]);
                if (e != kMixed && !__builtin_amdgcn_ballot_w64(y == INFINITY)) {
                    most = fmaxf(most, y * two_to(e));
                    continue;
                }
                odd |= 1u << piece;
                float z[8];
                unpack4<FP8>(lo[piece], *reinterpret_cast<float(*)[4]>(z));
                unpack4<FP8>(hi[piece], *reinterpret_cast<float(*)[4]>(z + 4));
                most = fmaxf(most, 0.f);
#pragma unroll
                for (int i = 0; i < 8; ++i)       // (a token that is not there has zeros)
                    most = fmaxf(most, fabsf(z[i]) * scales[octet * 8 + i]);
            }
        }
        most = wave_max(most);
        if (most < 0.f)
            continue;
        const int e = exponent_of<FP8>(most);
        // (the page's first token has its new id if any has; behind the sequence's last page nothing is there)
        const int64_t to = (int64_t)row_out[slot0 + x] * p.H + h;
        uint64_t *out = reinterpret_cast<uint64_t *>(values + (to << page_log2) * DK);
#pragma unroll
        for (int piece = 0; piece < PIECES; ++piece) {
            const int octet = octet0 + piece / CB, d = piece % CB * kWave + lane;
            const uint32_t has = __builtin_amdgcn_readfirstlane(octet_has[octet]);
            if (!has)
                continue;
            uint64_t w = (uint64_t)hi[piece] << 32 | lo[piece];
            const int was = __builtin_amdgcn_readfirstlane(octet_e[octet]);
            if (odd >> piece & 1) {
                float y[8];
                unpack4<FP8>(lo[piece], *reinterpret_cast<float(*)[4]>(y));
                unpack4<FP8>(hi[piece], *reinterpret_cast<float(*)[4]>(y + 4));
                const float f = two_to(-e);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    y[i] *= scales[octet * 8 + i] * f;
                w = (uint64_t)pack4<FP8>(y[4], y[5], y[6], y[7]) << 32 | pack4<FP8>(y[0], y[1], y[2], y[3]);
            } else if (was != e) {
                w = (uint64_t)rescale4<FP8>(hi[piece], two_to(was - e)) << 32 | rescale4<FP8>(lo[piece], two_to(was - e));
            }
            uint64_t *dst = out + (piece / CB) * DK + d;
            if (has != 0xff) {            // (what lies behind the last token stays)
                uint64_t mask = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    mask |= has >> i & 1 ? 0xffull << (8 * i) : 0;
                w = (w & mask) | (*dst & ~mask);
            }
            __builtin_nontemporal_store(w, dst);
        }
        if (lane == 0)
            p.exponents[to] = (int8_t)e;
    }
}

// ---- host -------------------------------------------------------------------------------------------------------
struct WeighCut {
    int splits, chunk, threads;
};
static WeighCut weigh_cut(const lookat_page_pool *p, int32_t B, int32_t G, int32_t W, int64_t max_length)
{
    const int64_t units = (int64_t)B * p->H, room = (int64_t)W * p->page, longest = max_length > 0 && max_length < room ? max_length : room;
    WeighCut c;
    // Small workgroups where there are more heads than large ones run at once, or where their short code holds a row (us a call of large / small ones:
    // 40 x 32 heads x 90 to 900 tokens, m = 16, 16.2 / 11.0, 64 x 32 x 30 to 300 in groups of 2 21.1 / 10.4, 64 x 12 x 500 to 5000 32.0 / 15.3, 16 x 12 x 900
    // 4.7 / 3.8, but 16 x 32 x 2000 6.4 / 8.1), while their tables leave room for 16 wavefronts of them.  Rows that a large one does not hold are cut either
    // way: 24 x 32 x 8927 in groups of 8 122 / 93, 20 x 32 x 6300 to 9000 in groups of 4 60.7 / 40.5.
    const bool brief = units >= 96 && room <= weigh_few(G) * kWeighSmall;
    const int64_t small = weigh_tokens(G, kWeighSmall);
    if ((units > 512 || brief) && G * p->m <= 32 && (room <= small || (room > weigh_tokens(G, kWeighThreads) && room <= 1024 * small))) {
        c.threads = kWeighSmall;
        c.chunk = (int)(room <= small ? (room + kWeighSmall - 1) / kWeighSmall * kWeighSmall : small);
        c.splits = (int)((room + c.chunk - 1) / c.chunk);
        return c;
    }
    c.threads = kWeighThreads;
    // Every token in reach has its range: the cut goes by the row's room where the caller's longest length does not hold.
    const int64_t most = weigh_tokens(G, kWeighThreads);
    int64_t want = units >= 128 ? 1 : (256 + units - 1) / units;
    const int64_t useful = (longest + 2047) / 2048;
    want = want < useful ? want : useful;
    int64_t chunk = (longest + want - 1) / want;
    chunk = (chunk + kWeighThreads - 1) / kWeighThreads * kWeighThreads;
    chunk = chunk < most && room <= 1024 * chunk ? chunk : most;      // (rows with far more room than the caller knows of tokens: few workgroups)
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

template <int M, int G, int PHASE, int T, int THREADS>
static int launch_weigh_phase(const PoolArgs &p, const WeighArgs &a, int64_t groups, hipStream_t st)
{
    constexpr size_t lds = (size_t)G * M * kCentroids * 4;
    const auto f = &weigh_kernel<M, G, PHASE, T, THREADS>;
    if (lds > 60 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(f), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess)
            return fail(LOOKAT_ERR_HIP, "lookat_pages_weigh: %s", hipGetErrorString(e));
    }
    hipLaunchKernelGGL(f, dim3((unsigned)groups), dim3(THREADS), lds, st, p, a);
    return check_launch("lookat_pages_weigh");
}
template <int M, int G, int T, int THREADS>
static int launch_weigh_threads(const PoolArgs &p, const WeighArgs &a, int64_t groups, hipStream_t st)
{
    if (a.splits == 1)
        return launch_weigh_phase<M, G, kWeighAll, T, THREADS>(p, a, groups, st);
    if (int rc = launch_weigh_phase<M, G, kWeighStats, T, THREADS>(p, a, groups, st))
        return rc;
    return launch_weigh_phase<M, G, kWeighAdd, T, THREADS>(p, a, groups, st);
}
template <int M, int G, int T>
static int launch_weigh_phases(const PoolArgs &p, const WeighArgs &a, int threads, int64_t groups, hipStream_t st)
{
    if constexpr (G * M <= 32)
        if (threads == kWeighSmall)
            return launch_weigh_threads<M, G, T, kWeighSmall>(p, a, groups, st);
    return launch_weigh_threads<M, G, T, kWeighThreads>(p, a, groups, st);
}
// Few scores a thread where that is enough: short code (us a call with it / with the long code: 12 heads x 1024 tokens 4.2 / 8.1, 16 x 8 x 1000 in groups of
// 4 7.0 / 9.7).
template <int M, int G>
static int launch_weigh(const PoolArgs &p, const WeighArgs &a, int threads, int64_t groups, hipStream_t st)
{
    constexpr int few = weigh_few(G);
    return a.chunk <= few * threads ? launch_weigh_phases<M, G, few>(p, a, threads, groups, st)
                                    : launch_weigh_phases<M, G, kWeighScores / G>(p, a, threads, groups, st);
}
template <int M>
static int launch_weigh_g(int G, const PoolArgs &p, const WeighArgs &a, int threads, int64_t groups, hipStream_t st)
{
    switch (G) {
    case 1: return launch_weigh<M, 1>(p, a, threads, groups, st);
    case 2: return launch_weigh<M, 2>(p, a, threads, groups, st);
    case 4: return launch_weigh<M, 4>(p, a, threads, groups, st);
    default: return launch_weigh<M, 8>(p, a, threads, groups, st);
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
template <int PAGE>
static auto move_kernel(int d_k, bool fp8)
{
    return d_k == 64 ? (fp8 ? &evict_move_kernel<64, true, PAGE> : &evict_move_kernel<64, false, PAGE>)
                     : (fp8 ? &evict_move_kernel<128, true, PAGE> : &evict_move_kernel<128, false, PAGE>);
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
    if (!fits_launch(groups, cut.threads))
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
    case 2: return launch_weigh_g<2>(group, p, a, cut.threads, groups, st);
    case 4: return launch_weigh_g<4>(group, p, a, cut.threads, groups, st);
    case 8: return launch_weigh_g<8>(group, p, a, cut.threads, groups, st);
    default: return launch_weigh_g<16>(group, p, a, cut.threads, groups, st);
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
    const int per_group = (pool->page < kWave ? kWave / pool->page : 1) * kMoveWaves, groups = (W_out + per_group - 1) / per_group;
    if (!fits_launch(units, kPickThreads) || !fits_launch(groups, kMoveThreads))
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
    // By the room of a row: a variant for few tokens is short code, and weights that stay in registers are read once (us a call of 48 heads x 1024 tokens
    // to half, kept by 2 / by 32 / read again 15.6 / 23.9 / 16.5, x 8000 24.3 / 30.6 / 34.4 (by 8 first), 128 x 20000 - / 134 / 159).  Small workgroups
    // where there are more heads than large ones run at once: 1024 x 700 37.0, so 29.5, 1024 x 500 to 5000 69.0 / 63.6, 768 x 300 24.8 / 19.1.
    const int64_t each = ((int64_t)W * pool->page + kPickThreads - 1) / kPickThreads;
    const bool small = units > 512 && each <= 8;
    const auto pick = small        ? (each <= 2 ? &evict_pick_kernel<8, kPickSmall> : &evict_pick_kernel<32, kPickSmall>)
                      : each <= 2  ? &evict_pick_kernel<2, kPickThreads>
                      : each <= 8  ? &evict_pick_kernel<8, kPickThreads>
                      : each <= 32 ? &evict_pick_kernel<32, kPickThreads>
                                   : &evict_pick_kernel<0, kPickThreads>;
    hipLaunchKernelGGL(pick, dim3((unsigned)units), dim3(small ? kPickSmall : kPickThreads), 0, st, a, p.H, p.page_log2);
    if (int rc = check_launch("lookat_pages_evict (choice)"))
        return rc;
    const bool fp8 = pool->value_type == LOOKAT_VALUES_E4M3;
    const auto f = pool->page == 16   ? move_kernel<16>(p.d_k, fp8)
                   : pool->page == 32 ? move_kernel<32>(p.d_k, fp8)
                   : pool->page == 64 ? move_kernel<64>(p.d_k, fp8)
                                      : move_kernel<128>(p.d_k, fp8);
    hipLaunchKernelGGL(f, dim3((unsigned)groups, (unsigned)p.H, (unsigned)B), dim3(kMoveThreads), 0, st, p, a);
    return check_launch("lookat_pages_evict");
}
