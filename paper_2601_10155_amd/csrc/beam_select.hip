// Beam search's selection: the n best of  scores[r] + logit - log sum exp(logits[r])  over a request's beams and the vocabulary.
//
// Two launches.  In the first a wavefront takes 64 E consecutive logits of a row, E to a lane, in registers: their maximum m, their n best in order, and
// the sum of exp(x - m).  A lower bound on the n-th best is the n-th largest of the lanes' maxima (found bit by bit with ballots); few logits reach
// it, and one lane takes each and counts those ahead of it.  Where more than 64 reach it (large n) the n-th best itself is found bit by bit
// among them, first its value, then among equal ones its place; where more than kListed do (many equal logits), among all.  Listed logits near m
// enter the sum in 64 bits, so that the terms that dominate a peaked row's sum carry no fp32 rounding.  The others are off by |d| u for the
// difference d = x - m, 1.25 |d| u for its product with log2(e) and 2 u for the exponential, u = 2^-24, and their sum over a lane, by pairs, by 16 u at
// most.  In a row of many equal logits all of that may go one way: 50 u = 2^-18.4 at d = -14, and with up to 2^24 logits no d gives more; 5.4e-7 was
// the most in 250 thousand such rows.  (The sum one term after the other: 9.3e-7, and 64 x 8 x 131072 56.5 us a call, so 57.0; the product's rounding carried
// along: 64.8.)
// In the second launch a workgroup takes a request.  A lower bound on the n-th best score, found as above from a few entries of every sorted list,
// leaves few candidates, whose places are counted.  Where more than kMostFound reach the bound (many equal scores) each wavefront takes the n best of its
// share of the lists one by one, and those are merged by counting.
#include <type_traits>

#include "common.h"
#include "lookat_search.h"

namespace lookat {

struct PartSum {
    double sum;                           // of exp(x - top) over a part's logits
    float top, unused;
};
struct SelectArgs {
    const void *logits;
    const float *scores;
    PartSum *stats;                       // [rows, parts]
    float *best;                          // [rows, parts, n] logits, falling
    int32_t *best_tokens;                 // ... and their tokens
    float *scores_out;
    int32_t *parents, *tokens;
    int64_t stride;
    int32_t rows, V, n, beams, parts, first_parent;
};

constexpr int kSelectWaves = 4, kSelectThreads = kSelectWaves * kWave;
constexpr int kShare = 8, kListed = kShare * kWave;       // logits of a part that reach the first border, at most, before the search goes over all
constexpr int kPlaceBits = 11;                            // of a logit's number in its part
constexpr float kLog2eF = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kNear = 3.f;              // listed logits that are nearer to their part's maximum enter its sum in 64 bits

typedef uint32_t u4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);          // (both zeros one)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
// What this wavefront's lanes wrote to LDS before is there for its lanes' reads behind it.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ int ballot_count(bool b) { return __builtin_popcountll(__builtin_amdgcn_ballot_w64(b)); }

__device__ __forceinline__ double wave_sum_double(double x)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2)
        x += __shfl_xor(x, d);
    return x;
}

template <typename FT, int E>
__global__ __launch_bounds__(kSelectThreads) void select_rows_kernel(SelectArgs a)
{
    constexpr int PER = 16 / (int)sizeof(FT), LOADS = E / PER;     // a load's logits
    static_assert(kWave * E <= 1 << kPlaceBits, "a logit's number fits its bits");
    constexpr int kPairLevels = E == 16 ? 4 : 5;
    static_assert(E == 1 << kPairLevels, "whole pairs");
    __shared__ uint64_t lists[kSelectWaves][kListed];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t item = (int64_t)blockIdx.x * kSelectWaves + wave;
    const int row = (int)(item / a.parts), part = (int)(item - (int64_t)row * a.parts);
    if (row >= a.rows)
        return;
    const int first = part * (kWave * E);
    const int count = a.V - first < kWave * E ? a.V - first : kWave * E;
    const FT *src = static_cast<const FT *>(a.logits) + row * a.stride + first;
    // logit j of a lane is number (j / PER) * 64 PER + lane * PER + j % PER of the part
    float x[E];
    if (count == kWave * E) {
        u4_any raw[LOADS];
#pragma unroll
        for (int k = 0; k < LOADS; ++k)
            raw[k] = __builtin_nontemporal_load(reinterpret_cast<const u4_any *>(src + (k * kWave + lane) * PER));
#pragma unroll
        for (int k = 0; k < LOADS; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (PER == 4) {
                    x[k * 4 + i] = __uint_as_float(raw[k][i]);
                } else {
                    const uint32_t w = raw[k][i];
                    const float2 f = __half22float2(__builtin_bit_cast(__half2, w));
                    x[k * 8 + 2 * i] = f.x;
                    x[k * 8 + 2 * i + 1] = f.y;
                }
            }
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int at = (j / PER) * (kWave * PER) + lane * PER + j % PER;
            x[j] = at < count ? (float)src[at] : -INFINITY;
        }
    }
    auto number = [&](int j) -> int { return (j / PER) * (kWave * PER) + lane * PER + j % PER; };

    float top = x[0];
#pragma unroll
    for (int j = 1; j < E; ++j)
        top = fmaxf(top, x[j]);
    const uint32_t order = ordered(top);
    uint32_t bound = 0;
#pragma unroll
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t t = bound | 1u << bit;
        bound = ballot_count(order >= t) >= a.n ? t : bound;
    }
    float border = fmaxf(unordered(bound), kLowest);      // (-inf, and the NaN that no bound stands for, are below)
    const float m = wave_max(top), base = m == -INFINITY ? 0.f : m;
    // One sweep lists the logits that reach the border (up to number `most` of those at it) and adds up the others.  Few reach it: the list's part is
    // branched over.  (The difference first: rows that differ by a constant then have the same sum, and their ties stay ties.)
    const uint64_t below = (1ull << lane) - 1;
    int found = 0;
    float rest = 0.f;
    auto sweep = [&](auto all, float at_least, int most) {
        found = 0;
        float pairs[kPairLevels + 1];     // sums of 2^level terms
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const bool reaches = x[j] >= at_least;
            bool list = reaches;
            if constexpr (!decltype(all)::value)
                list = reaches && (x[j] > at_least || number(j) <= most);
            const uint64_t mask = __builtin_amdgcn_ballot_w64(list);
            if (mask) {
                const int place = found + __builtin_popcountll(mask & below);
                if (list && place < kListed)
                    lists[wave][place] = (uint64_t)ordered(x[j]) << 32 | (uint32_t)~number(j);
                found += __builtin_popcountll(mask);
            }
            const float e = fast_exp2((x[j] - base) * kLog2eF);
            float sum = reaches ? 0.f : e;
            int level = 0;
#pragma unroll
            for (; j >> level & 1; ++level)
                sum += pairs[level];
            pairs[level] = sum;
        }
        rest = pairs[kPairLevels];
    };
    sweep(std::true_type(), border, 0);
    float ties = 0.f;                     // logits at the border that are not listed
    if (found > kWave && found <= kListed) {
        // The n greatest of the list, every lane with its share of it: first the n-th logit, then, of equal ones, the n-th place.
        wave_fence();
        uint64_t keys[kShare];
#pragma unroll
        for (int j = 0; j < kShare; ++j)
            keys[j] = j * kWave + lane < found ? lists[wave][j * kWave + lane] : 0;
        uint64_t nth = 0;
#pragma unroll 1
        for (int bit = 63; bit >= 0; bit = bit == 32 ? kPlaceBits - 1 : bit - 1) {
            if (bit == kPlaceBits - 1)
                nth |= 0xffffffffu >> kPlaceBits << kPlaceBits;       // (a place is the complement of a number below 2^kPlaceBits)
            const uint64_t t = nth | 1ull << bit;
            int c = 0;
#pragma unroll
            for (int j = 0; j < kShare; ++j)
                if (j * kWave < found)
                    c += ballot_count(keys[j] >= t);
            nth = c >= a.n ? t : nth;
            if (c == a.n)                 // (these are the n greatest: us a call for 16 x 4 x 50257, n = 64, all digits 43, so 26)
                break;
        }
        wave_fence();
        int kept = 0;
#pragma unroll
        for (int j = 0; j < kShare; ++j)
            if (j * kWave < found) {
                const bool keep = keys[j] >= nth;
                const uint64_t mask = __builtin_amdgcn_ballot_w64(keep);
                if (keep)
                    lists[wave][kept + __builtin_popcountll(mask & below)] = keys[j];
                else if (keys[j])
                    rest += fast_exp2((unordered((uint32_t)(keys[j] >> 32)) - base) * kLog2eF);
                kept += __builtin_popcountll(mask);
            }
        found = kept;
    } else if (found > kWave) {
        uint32_t nth = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const float t = unordered(nth | 1u << bit);
            int c = 0;
#pragma unroll
            for (int j = 0; j < E; ++j)
                c += ballot_count(x[j] >= t);
            nth = c >= a.n ? nth | 1u << bit : nth;
        }
        border = fmaxf(unordered(nth), kLowest);
        int above = 0, equal = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            above += ballot_count(x[j] > border);
            equal += ballot_count(x[j] == border);
        }
        const int want = a.n - above;
        int most = 0x7fffffff;            // of the logits at the border those up to this number
        if (equal > want) {
            most = 0;
            for (int bit = 30; bit >= 0; --bit) {
                if (1 << bit >= kWave * E)
                    continue;
                const int t = most | 1 << bit;
                int c = 0;
#pragma unroll
                for (int j = 0; j < E; ++j)
                    c += ballot_count(x[j] == border && number(j) < t);
                most = c < want ? t : most;
            }
            ties = (float)(equal - want);
        }
        sweep(std::false_type(), border, most);
    }
    wave_fence();
    const uint64_t key = lane < found ? lists[wave][lane] : 0;
    int rank = 0;
    // (out of LDS, the same address for all lanes: read across lanes instead 62.5 us for 64 x 8 x 131072, n = 16, so 59.9)
    for (int j = 0; j < found; ++j)
        rank += lists[wave][j] > key;
    const float logit = unordered((uint32_t)(key >> 32));
    const bool listed = lane < found && rank < a.n;
    // listed logits near the maximum in 64 bits, the others of them as the rest
    double sum = 0;
    if (lane < found && !(listed && logit > m - kNear))
        rest += fast_exp2((logit - base) * kLog2eF);
    else if (lane < found)
        sum = exp((double)logit - (double)base);
    if (ties > 0.f && lane == 0)
        rest += ties * fast_exp2((border - base) * kLog2eF);
    sum = wave_sum_double(sum + (double)rest);
    float *best = a.best + item * a.n;
    int32_t *tokens = a.best_tokens + item * a.n;
    if (listed) {
        best[rank] = logit;
        tokens[rank] = first + (int)~(uint32_t)key;
    }
    for (int j = found + lane; j < a.n; j += kWave)
        best[j] = -INFINITY;
    if (lane == 0)
        a.stats[item] = PartSum{sum, m, 0.f};
}

// A candidate, and the order among them: score, then row, then logit, then token (within a row the score's rounding decides nothing).
struct Pick {
    double score;
    int row, token;
    float logit;
};
__device__ __forceinline__ bool ahead(const Pick &a, const Pick &b)
{
    if (a.score != b.score)
        return a.score > b.score;
    if (a.row != b.row)
        return a.row < b.row;
    return a.logit != b.logit ? a.logit > b.logit : a.token < b.token;
}
// A score as fp32; those below its range, which are candidates all the same, as its lowest number.
__device__ __forceinline__ float rounded(double score) { return score > -(double)INFINITY ? fmaxf((float)score, kLowest) : -INFINITY; }

// Four wavefronts: the bound is found by each of them from all threads' best (us for 4 beams of 50257, four / eight / sixteen 8.0 / 9.9 / 16.0).
constexpr int kMergeWaves = 4, kMergeThreads = kMergeWaves * kWave;
constexpr int kMostPicks = 64, kMostBeams = 1024, kMostFound = 1024, kBatch = 4, kAllAtOnce = 1024;

__global__ __launch_bounds__(kMergeThreads) void select_merge_kernel(SelectArgs a)
{
    __shared__ double bases[kMostBeams];
    __shared__ Pick picks[kMostFound];
    __shared__ uint32_t tops[kMergeThreads];
    __shared__ int found_s;
    const int q = blockIdx.x, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, n = a.n, parts = a.parts;
    const int64_t row0 = (int64_t)q * a.beams;
    // The rows' sums, 64 or 16 lanes a row, each with up to kHeld parts in registers (a wavefront a row whatever their number: us a call for 4 x 16 x 1000
    // 22.7, so 14.6).
    auto sum_up = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value, kHeld = 128 / L;
        const int within = lane & (L - 1);
        for (int r = (wave * kWave + lane) / L; r < a.beams; r += kMergeThreads / L) {
            const PartSum *stats = a.stats + (row0 + r) * parts;
            const float score = a.scores[row0 + r];
            const PartSum nothing = {0, -INFINITY, 0.f};
            PartSum held[kHeld];
#pragma unroll
            for (int k = 0; k < kHeld; ++k)
                held[k] = k * L + within < parts ? stats[k * L + within] : nothing;
            float m = held[0].top;
#pragma unroll
            for (int k = 1; k < kHeld; ++k)
                m = fmaxf(m, held[k].top);
            for (int j = kHeld * L + within; j < parts; j += L)
                m = fmaxf(m, stats[j].top);
#pragma unroll
            for (int d = 1; d < L; d *= 2)
                m = fmaxf(m, __shfl_xor(m, d));
            // (a part of -inf alone has a sum of zero, or NaN)
            auto scaled = [&](const PartSum &s) -> double { return s.sum * (s.top == -INFINITY ? 1.0 : exp((double)s.top - (double)m)); };
            double sum = scaled(held[0]);
#pragma unroll
            for (int k = 1; k < kHeld; ++k)
                if (k * L < parts)
                    sum += scaled(held[k]);
            for (int j = kHeld * L + within; j < parts; j += L)
                sum += scaled(stats[j]);
#pragma unroll
            for (int d = 1; d < L; d *= 2)
                sum += __shfl_xor(sum, d);
            // -inf: no candidates (a sum that is NaN or infinite, a score that is not finite)
            const bool none = !(fabsf(m) < INFINITY) || !(sum < (double)INFINITY) || !(fabsf(score) < INFINITY);
            if (within == 0)
                bases[r] = none ? -(double)INFINITY : (double)score - ((double)m + log(sum));
        }
    };
    if (a.beams <= kMergeWaves)
        sum_up(std::integral_constant<int, kWave>());
    else
        sum_up(std::integral_constant<int, 16>());
    __syncthreads();

    const int lists = a.beams * parts, step = kMergeThreads;
    const float *best = a.best + row0 * parts * n;        // the lists of a request follow each other
    const int32_t *best_tokens = a.best_tokens + row0 * parts * n;
    auto candidate = [&](int list, int j) -> Pick {
        Pick c;
        c.row = list / parts;
        c.logit = best[(int64_t)list * n + j];
        c.token = best_tokens[(int64_t)list * n + j];     // (not looked at where the logit is -inf)
        c.score = bases[c.row] + (double)c.logit;
        return c;
    };
    // the best of this lane's lists behind `last`
    auto next = [&](bool any, const Pick &last) -> Pick {
        Pick first;
        first.score = -(double)INFINITY;
        first.row = first.token = 0x7fffffff;
        first.logit = -INFINITY;
        for (int list = wave * kWave + lane; list < lists; list += step)
            for (int j = 0; j < n; ++j) {
                const Pick c = candidate(list, j);
                if (!(c.score > -(double)INFINITY))
                    break;
                if (any && !ahead(last, c))
                    continue;
                if (ahead(c, first))
                    first = c;
                break;
            }
        return first;
    };
    // the wavefronts' n best of their lists, into picks
    auto one_by_one = [&]() {
        Pick mine = next(false, Pick());
        for (int k = 0; k < n; ++k) {
            double top = mine.score;
#pragma unroll
            for (int d = 1; d < kWave; d *= 2)
                top = fmax(top, __shfl_xor(top, d));
            Pick pick;
            pick.score = top;
            pick.row = pick.token = -1;
            pick.logit = -INFINITY;
            int owner = -1;
            if (top > -(double)INFINITY) {
                uint64_t tied = __builtin_amdgcn_ballot_w64(mine.score == top);
                while (tied) {
                    const int l = __builtin_ctzll(tied);
                    tied &= tied - 1;
                    Pick c;
                    c.score = top;
                    c.row = __builtin_amdgcn_readlane(mine.row, l);
                    c.token = __builtin_amdgcn_readlane(mine.token, l);
                    c.logit = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine.logit), l));
                    if (owner < 0 || ahead(c, pick)) {
                        pick = c;
                        owner = l;
                    }
                }
            }
            if (lane == 0)
                picks[wave * n + k] = pick;
            if (lane == owner)
                mine = next(true, pick);
        }
    };
    // A bound that n candidates reach, from the first `deep` entries of every list (rounded to fp32, which keeps their order).
    const int deep = lists >= kMergeThreads ? 1 : (kMergeThreads + lists - 1) / lists < n ? (kMergeThreads + lists - 1) / lists : n;
    float top = -INFINITY;
    for (int item0 = threadIdx.x; item0 < lists * deep; item0 += kBatch * step) {
        float x[kBatch];
        int row[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int item = item0 + u * step < lists * deep ? item0 + u * step : item0, list = item / deep;
            row[u] = list / parts;
            x[u] = best[(int64_t)list * n + item - list * deep];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            top = fmaxf(top, rounded(bases[row[u]] + (double)x[u]));
    }
    tops[threadIdx.x] = ordered(top);
    if (threadIdx.x == 0)
        found_s = 0;
    __syncthreads();
    uint32_t order[kMergeWaves], bound = 0;
#pragma unroll
    for (int w = 0; w < kMergeWaves; ++w)
        order[w] = tops[w * kWave + lane];
    int reached = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 0 && reached != n; --bit) {
        const uint32_t t = bound | 1u << bit;
        int c = 0;
#pragma unroll
        for (int w = 0; w < kMergeWaves; ++w)
            c += ballot_count(order[w] >= t);
        bound = c >= n ? t : bound;
        reached = c >= n ? c : reached;
    }
    float border = unordered(bound);
    if (reached == n) {
        border = INFINITY;
#pragma unroll
        for (int w = 0; w < kMergeWaves; ++w)
            border = order[w] >= bound ? fminf(border, unordered(order[w])) : border;
        border = -wave_max(-border);
    }
    border = fmaxf(border, kLowest);
    // Few entries are looked at all at once, many list by list from the heads on (us a call, list by list / so,
    // 119 x 4 x 2092 logits, n = 49, 588 entries, 25.6 / 18.1, 6 x 12 x 803, n = 14, 168 13.7 / 12.5, but 65 x 14 x 18185, n = 13, 3276 27.2 / 29.5).
    if (lists * n <= kAllAtOnce) {
        for (int item0 = threadIdx.x; item0 < lists * n; item0 += kBatch * step) {
            float x[kBatch];
            int32_t token[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int item = item0 + u * step < lists * n ? item0 + u * step : item0;
                x[u] = best[item];
                token[u] = best_tokens[item];
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int item = item0 + u * step, row = (item < lists * n ? item : item0) / n / parts;
                const double score = bases[row] + (double)x[u];
                if (item < lists * n && rounded(score) >= border) {
                    const int at = atomicAdd(&found_s, 1);
                    if (at < kMostFound)
                        picks[at] = Pick{score, row, token[u], x[u]};
                }
            }
        }
    } else {
        for (int list0 = threadIdx.x; list0 < lists; list0 += kBatch * step) {
            float heads[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                heads[u] = best[(int64_t)(list0 + u * step < lists ? list0 + u * step : list0) * n];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int list = list0 + u * step;
                bool more = list < lists && rounded(bases[list / parts] + (double)heads[u]) >= border;
                for (int j0 = 0; j0 < n && more; j0 += kBatch) {
                    Pick c[kBatch];
#pragma unroll
                    for (int i = 0; i < kBatch; ++i)
                        c[i] = candidate(list, j0 + i < n ? j0 + i : n - 1);
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) {
                        more = more && j0 + i < n && rounded(c[i].score) >= border;
                        if (more) {
                            const int at = atomicAdd(&found_s, 1);
                            if (at < kMostFound)
                                picks[at] = c[i];
                        }
                    }
                }
            }
        }
    }
    __syncthreads();
    int found = found_s;
    const bool listed = found > kMostFound;
    if (listed) {
        __syncthreads();
        found = kMergeWaves * n;
        one_by_one();
        __syncthreads();
    }
    __syncthreads();
    // a thread per candidate: its place is the number of those ahead of it
    for (int i = threadIdx.x; i < found; i += kMergeThreads) {
        const Pick c = picks[i];
        if (!(c.score > -(double)INFINITY))
            continue;
        // (scores first: who is ahead of whom among equal ones is looked at only where there are any)
        int rank = 0, equal = 0;
#pragma unroll 4
        for (int j = 0; j < found; ++j) {
            const double other = picks[j].score;
            rank += other > c.score;
            equal += other == c.score;
        }
        if (equal > 1) {                  // (not with itself alone)
            rank = 0;
            for (int j = 0; j < found; ++j)
                rank += ahead(picks[j], c);
        }
        if (rank < n) {
            a.scores_out[(int64_t)q * n + rank] = rounded(c.score);
            a.parents[(int64_t)q * n + rank] = a.first_parent + (int)row0 + c.row;
            a.tokens[(int64_t)q * n + rank] = c.token;
        }
    }
    // and what has no candidate
    int real = found;
    if (listed)
        for (int j = 0; j < found; ++j)
            real -= !(picks[j].score > -(double)INFINITY);
    for (int j = real + threadIdx.x; j < n; j += kMergeThreads) {
        a.scores_out[(int64_t)q * n + j] = -INFINITY;
        a.parents[(int64_t)q * n + j] = a.tokens[(int64_t)q * n + j] = -1;
    }
}

// ---- host -------------------------------------------------------------------------------------------------------
struct SelectCut {
    int each, parts;
    size_t stats, best;                   // bytes, each a multiple of 16
};
static SelectCut select_cut(int32_t Q, int32_t beams, int32_t V, int32_t n)
{
    SelectCut c;
    const int64_t rows = (int64_t)Q * beams;
    // Logits of a lane: 32, or 16 where there would be few wavefronts.  us of the launch, 8 / 16 / 32 / 64: 4 x 50257 fp32 4.7 / 5.0 / 6.0 / - (and 10.0
    // / 8.3 / 7.9 / - of the merge), 128 x 32001 fp16 9.5 / 7.7 / 9.0 / -, 512 x 131072 fp32 (a call) 133 / 80.9 / 63.5 / 79.8.  And 32 where a request
    // would have more than 512 lists to merge: us a call, 16 / 32, 1 x 16 x 262144 (4096 lists) 30.7 / 22.2, 8 x 8 x 131072 (1024) 20.3 / 18.8,
    // but 16 x 4 x 50257, n = 64 (200) 25.9 / 34.8.
    c.each = rows * V < (16LL << 20) && beams * ((V + 1023) / 1024) <= 512 ? 16 : 32;
    const int64_t per = (int64_t)kWave * c.each;
    c.parts = (int)((V + per - 1) / per);
    c.stats = ((size_t)rows * c.parts * sizeof(PartSum) + 15) / 16 * 16;
    c.best = ((size_t)rows * c.parts * n * 4 + 15) / 16 * 16;
    return c;
}
static int check_select(int32_t Q, int32_t beams, int32_t V, int32_t n)
{
    if (Q <= 0 || beams <= 0 || V <= 0 || n <= 0)
        return fail(LOOKAT_ERR_SHAPE, "Q=%d, beams=%d, V=%d and n=%d must be positive", Q, beams, V, n);
    if (n > kMostPicks || beams > kMostBeams || (int64_t)Q * beams > 65535 || V > (1 << 24))
        return fail(LOOKAT_ERR_UNSUPPORTED, "Q=%d, beams=%d, V=%d, n=%d: at most 64 candidates, 1024 beams, 65535 rows and 2^24 tokens", Q, beams, V, n);
    return LOOKAT_OK;
}

}  // namespace lookat

extern "C" size_t lookat_beam_select_workspace_bytes(int32_t Q, int32_t beams, int32_t V, int32_t n)
{
    using namespace lookat;
    clear_error();
    if (check_select(Q, beams, V, n) != LOOKAT_OK)
        return 0;
    const SelectCut c = select_cut(Q, beams, V, n);
    return c.stats + 2 * c.best;
}

extern "C" int lookat_beam_select(int32_t Q, int32_t beams, int32_t V, int32_t n, const void *logits, lookat_dtype logit_dtype, int64_t logit_stride,
                                  const float *scores, int32_t first_parent, float *scores_out, int32_t *parents, int32_t *tokens, void *workspace,
                                  size_t workspace_bytes, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_select(Q, beams, V, n))
        return rc;
    if (logit_dtype != LOOKAT_F16 && logit_dtype != LOOKAT_F32)
        return fail(LOOKAT_ERR_DTYPE, "logit_dtype=%d is neither LOOKAT_F16 nor LOOKAT_F32", (int)logit_dtype);
    if (logit_stride < V)
        return fail(LOOKAT_ERR_SHAPE, "logit_stride=%lld smaller than a row of V=%d", (long long)logit_stride, V);
    if (first_parent < 0 || first_parent > 0x7fffffff - 65535)
        return fail(LOOKAT_ERR_SHAPE, "first_parent=%d out of range", first_parent);
    if (!logits || !scores || !scores_out || !parents || !tokens)
        return fail(LOOKAT_ERR_NULL, "logits, scores, scores_out, parents and tokens must be non-NULL");
    if (reinterpret_cast<uintptr_t>(logits) & (logit_dtype == LOOKAT_F16 ? 1u : 3u))
        return fail(LOOKAT_ERR_ALIGN, "logits must be aligned to their type");
    if ((reinterpret_cast<uintptr_t>(scores) | reinterpret_cast<uintptr_t>(scores_out) | reinterpret_cast<uintptr_t>(parents) |
         reinterpret_cast<uintptr_t>(tokens)) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "scores, scores_out, parents and tokens must be 4-byte aligned");
    const SelectCut cut = select_cut(Q, beams, V, n);
    const size_t need = cut.stats + 2 * cut.best;
    if (!workspace || workspace_bytes < need)
        return fail(LOOKAT_ERR_WORKSPACE, "workspace of %zu bytes needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
    if (!aligned16(workspace))
        return fail(LOOKAT_ERR_ALIGN, "workspace must be 16-byte aligned");
    const int64_t rows = (int64_t)Q * beams, groups = (rows * cut.parts + kSelectWaves - 1) / kSelectWaves;
    if (groups * kSelectThreads > 0xffffffffLL || rows * cut.parts * n > 0x7fffffffLL)
        return fail(LOOKAT_ERR_UNSUPPORTED, "Q*beams=%lld rows of V=%d tokens exceed one launch", (long long)rows, V);
    SelectArgs a;
    a.logits = logits;
    a.scores = scores;
    a.stats = static_cast<PartSum *>(workspace);
    a.best = reinterpret_cast<float *>(static_cast<char *>(workspace) + cut.stats);
    a.best_tokens = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + cut.stats + cut.best);
    a.scores_out = scores_out;
    a.parents = parents;
    a.tokens = tokens;
    a.stride = logit_stride;
    a.rows = (int32_t)rows;
    a.V = V;
    a.n = n;
    a.beams = beams;
    a.parts = cut.parts;
    a.first_parent = first_parent;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool half = logit_dtype == LOOKAT_F16;
    const auto f = cut.each == 16 ? (half ? &select_rows_kernel<_Float16, 16> : &select_rows_kernel<float, 16>)
                                  : (half ? &select_rows_kernel<_Float16, 32> : &select_rows_kernel<float, 32>);
    hipLaunchKernelGGL(f, dim3((unsigned)groups), dim3(kSelectThreads), 0, st, a);
    if (int rc = check_launch("lookat_beam_select (rows)"))
        return rc;
    hipLaunchKernelGGL(select_merge_kernel, dim3((unsigned)Q), dim3(kMergeThreads), 0, st, a);
    return check_launch("lookat_beam_select");
}
