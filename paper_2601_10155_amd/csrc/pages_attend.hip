// Attention decode over the paged cache: product-quantised keys, 8-bit values with a power-of-two scale per page and head.
//
//   s_l = sum_i lut_i[code_l,i],   out = sum_l softmax_l(scale s) q_l 2^e(l)
//
// computed in one pass with the page's exponent added to the logit: y_l = scale log2(e) s_l + e(l), R a running reference near max y,
//   w_l = 2^(y_l - R),   out = sum_l w_l q_l / sum_l w_l 2^-e(l).
// So the stored integers enter the product as they are (exact in fp16), the weights are as precise as the largest contribution to the result
// needs whatever the pages' exponents are, and no per-page rescaling is done.
//
// Bound: the stream of codes and values from HBM, m + d_k bytes per token and key/value head.
//
// One workgroup = one (sequence, key/value head, range); its wavefronts take the range's 64-token tiles in turn.  In a tile
//   * scoring: a lane per token: its page from the table, its codes (one load), m look-ups per query head in the head's table in LDS.  The
//     tables of 2 or 4 query heads lie interleaved, so that one LDS read serves them all;
//   * the weighted sum runs on the matrix cores (v_mfma_f32_16x16x32_f16), out^T[d, n] += V^T[d, l] P^T[l, n]: columns n < G are the weights
//     of query head n rounded to fp16, columns G..2G-1 what that left (22 bits together), the other columns repeat them.  Each lane's
//     operand is eight tokens of one coordinate: eight consecutive bytes of the page as it is stored, widened to fp16 in registers.  The weights
//     go from a lane per token to that layout through 2 KB of LDS per wavefront.
#include "pages.h"
#include "decode_common.h"

namespace lookat {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

struct AttendArgs {
    const float *lut;
    const int32_t *table, *lengths;
    float *part, *out;
    int64_t table_stride;
    int32_t W, units, splits, chunk;      // units = sequences * key/value heads; chunk tokens per range (a multiple of 64)
    float scale_log2e;
};

constexpr float kRefLag = 8.f;            // the reference moves when a logit exceeds it by more (log2 units)
constexpr float kRefLift = 7.f;           // weights are 2^7 at the reference, below 2^15: fp16's range, its subnormals far below
constexpr int kWeightRow = 72;            // halves between the staged weights of two columns: 64 tokens, 16 bytes of padding

// Eight stored bytes (two registers) to eight fp16 numbers, exactly.
template <bool FP8>
__device__ __forceinline__ v8h widen(uint32_t lo, uint32_t hi)
{
    uint32_t w[4];
    if constexpr (FP8) {
        const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
        const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
        w[0] = __builtin_bit_cast(uint32_t, a);
        w[1] = __builtin_bit_cast(uint32_t, b);
        w[2] = __builtin_bit_cast(uint32_t, c);
        w[3] = __builtin_bit_cast(uint32_t, d);
    } else {
        // q + 128 behind the exponent byte of 1024: 1024 + 128 + q, less 1152
        const v2h bias = {(_Float16)-1152.f, (_Float16)-1152.f};
        lo ^= 0x80808080u;
        hi ^= 0x80808080u;
        const uint32_t u[4] = {__builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u),
                               __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = __builtin_bit_cast(uint32_t, (v2h)(__builtin_bit_cast(v2h, u[i]) + bias));
    }
    const v4u r = {w[0], w[1], w[2], w[3]};
    return __builtin_bit_cast(v8h, r);
}

// LDS of a workgroup: tables and staged weights while it streams, the wavefronts' results afterwards.
__host__ __device__ constexpr size_t attend_lds_bytes(int G, int M, int d_k, int waves)
{
    const size_t stream = (size_t)G * M * kCentroids * 4 + (size_t)waves * 2 * G * kWeightRow * 2;
    const size_t merge = (size_t)waves * G * (d_k + 2) * 4;
    return stream > merge ? stream : merge;
}

template <int DK, int M, int G, bool FP8>
__global__ __launch_bounds__(1024) void attend_pages_kernel(PoolArgs p, AttendArgs a)
{
    extern __shared__ __align__(16) char lds[];
    constexpr int GP = G < 4 ? G : 4;                     // query heads whose tables are interleaved
    typedef float vg __attribute__((ext_vector_type(GP)));
    constexpr int CB = DK / 32;                           // 16-byte loads per lane and 32 tokens
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, waves = blockDim.x / kWave;
    // ranges of one (sequence, head) on one die: its tables are fetched into one L2
    const int unit = (int)(blockIdx.x / kXcds) / a.splits * kXcds + blockIdx.x % kXcds, split = (int)(blockIdx.x / kXcds) % a.splits;
    if (unit >= a.units)
        return;
    const int b = unit / p.H, h = unit - b * p.H;
    const int length = clamp_length(a.lengths[b], a.W, p.page_log2);
    const int k0 = split * a.chunk;
    const int k1 = split == a.splits - 1 || length - k0 < a.chunk ? length : k0 + a.chunk;
    if (k0 >= k1 && split > 0)
        return;                                           // (the merge knows the length)
    const int32_t *row = a.table + b * a.table_stride;
    const int page_mask = (1 << p.page_log2) - 1;
    const int col = lane & 15, quad = lane >> 4;

    // a token's page, or -1: behind the range's end, or an id outside the pool
    auto page_of = [&](int key) -> int {
        int id = -1;
        if (key < k1)
            id = row[key >> p.page_log2];
        return (uint32_t)id < (uint32_t)p.pages ? id : -1;
    };
    uint32_t codes[(M + 3) / 4];
    int exponent = 0;
    v4u v[2][CB];
    uint32_t keep[2][2];                                  // FP8: the bytes of an octet that hold tokens
    auto request = [&](int t, int id) {
        const int key = t + lane;
        const int64_t place = (int64_t)(id < 0 ? 0 : id) * p.H + h;
        const uint8_t *c = p.codes + ((place << p.page_log2) + (key & page_mask)) * M;
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
        exponent = p.exponents[place];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const int first = kk * 32 + quad * 8;         // the octet's first token in the tile
            const int oid = __shfl(id, first);
            const int64_t at = ((int64_t)(oid < 0 ? 0 : oid) * p.H + h) << p.page_log2;
            const uint8_t *src = p.values + (at + ((t + first) & page_mask)) * DK + col * 16;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                v[kk][cb] = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(src + cb * 256));
            if constexpr (FP8) {
                // (bytes behind the last token may be NaN)
                const int n = oid < 0 ? 0 : k1 - t - first;
                keep[kk][0] = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
                keep[kk][1] = n >= 8 ? ~0u : n <= 4 ? 0u : (1u << (8 * (n - 4))) - 1;
            }
        }
    };

    int t = k0 + wave * kWave;
    const int step = waves * kWave;
    int id = page_of(t + lane);
    float *tables = reinterpret_cast<float *>(lds);
    {
        // tables [query head][i][c] -> [plane of GP heads][i][c][head], scaled
        const float *src = a.lut + (int64_t)unit * G * M * kCentroids;
        for (int j = tid; j < M * kCentroids; j += blockDim.x) {
#pragma unroll
            for (int g0 = 0; g0 < G; g0 += GP) {
                vg x;
#pragma unroll
                for (int g = 0; g < GP; ++g)
                    x[g] = src[(g0 + g) * (M * kCentroids) + j] * a.scale_log2e;
                reinterpret_cast<vg *>(tables)[(g0 / GP) * (M * kCentroids) + j] = x;
            }
        }
    }
    if (t < k1)
        request(t, id);
    int id_next = page_of(t + step + lane);
    __syncthreads();

    _Float16 *weights = reinterpret_cast<_Float16 *>(lds + (size_t)G * M * kCentroids * 4) + (size_t)wave * 2 * G * kWeightRow;
    v4f acc[2 * CB];
#pragma unroll
    for (int c = 0; c < 2 * CB; ++c)
        acc[c] = (v4f){0.f, 0.f, 0.f, 0.f};
    float ref[G], z[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        ref[g] = -1e30f;
        z[g] = 0.f;
    }

    while (t < k1) {
        // logits
        float y[G];
#pragma unroll
        for (int g = 0; g < G; ++g)
            y[g] = 0.f;
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const uint32_t c = (codes[i / 4] >> (8 * (i % 4))) & 0xffu;
#pragma unroll
            for (int g0 = 0; g0 < G; g0 += GP) {
                const vg x = reinterpret_cast<const vg *>(tables)[((g0 / GP) * M + i) * kCentroids + c];
#pragma unroll
                for (int g = 0; g < GP; ++g)
                    y[g0 + g] += x[g];
            }
        }
        bool above = false;
        exponent = id < 0 ? 0 : exponent;                 // (a lane without a token has read some page's)
#pragma unroll
        for (int g = 0; g < G; ++g) {
            y[g] = id < 0 ? -INFINITY : y[g] + (float)exponent;
            above |= y[g] > ref[g] + kRefLag;
        }
        if (__builtin_amdgcn_ballot_w64(above)) {
            float fix_n = 1.f;                            // for the column that this lane accumulates
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float to = fmaxf(ref[g], wave_max(y[g]));
                const float fix = fast_exp2(ref[g] - to);
                ref[g] = to;
                z[g] *= fix;
                fix_n = (lane & (G - 1)) == g ? fix : fix_n;
            }
#pragma unroll
            for (int c = 0; c < 2 * CB; ++c)
                acc[c] *= fix_n;
        }
        const float unscale = __uint_as_float((uint32_t)(127 - exponent) << 23);      // 2^-e
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float w = fast_exp2(y[g] - (ref[g] - kRefLift));
            z[g] = fmaf(w, unscale, z[g]);
            const _Float16 hi = (_Float16)w;
            weights[g * kWeightRow + lane] = hi;
            weights[(G + g) * kWeightRow + lane] = (_Float16)(w - (float)hi);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const v8h wt = *reinterpret_cast<const v8h *>(weights + (col & (2 * G - 1)) * kWeightRow + kk * 32 + quad * 8);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                v4u x = v[kk][cb];
                if constexpr (FP8) {
                    x.x &= keep[kk][0], x.y &= keep[kk][1];
                    x.z &= keep[kk][0], x.w &= keep[kk][1];
                }
                acc[2 * cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen<FP8>(x.x, x.y), wt, acc[2 * cb], 0, 0, 0);
                acc[2 * cb + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen<FP8>(x.z, x.w), wt, acc[2 * cb + 1], 0, 0, 0);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        __builtin_amdgcn_wave_barrier();                  // (the next tile's weights overwrite these)
        t += step;
        id = id_next;
        if (t < k1) {
            request(t, id);
            id_next = page_of(t + step + lane);
        }
    }

    // the wavefronts' results
#pragma unroll
    for (int g = 0; g < G; ++g)
        z[g] = wave_sum(z[g]);
    __syncthreads();                                      // every wavefront is done with its tables
    float *red = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int c = 0; c < 2 * CB; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float both = acc[c][r] + __shfl_xor(acc[c][r], G);      // columns n and n + G: the two terms of a weight
            // row 4 quad + r of the instruction's result is coordinate 2 (4 quad + r) + (c & 1) of the 32 that a load covers
            if (col < G)
                red[(wave * G + col) * (DK + 2) + (c / 2) * 32 + 2 * (4 * quad + r) + (c & 1)] = both;
        }
    if (lane == 0) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            red[(wave * G + g) * (DK + 2) + DK] = ref[g];
            red[(wave * G + g) * (DK + 2) + DK + 1] = z[g];
        }
    }
    __syncthreads();
    for (int j = tid; j < G * DK; j += blockDim.x) {
        const int g = j / DK, d = j - g * DK;
        float top = -1e30f, o = 0.f, sum = 0.f;
        for (int w = 0; w < waves; ++w)
            top = fmaxf(top, red[(w * G + g) * (DK + 2) + DK]);
        for (int w = 0; w < waves; ++w) {
            const float *x = red + (w * G + g) * (DK + 2);
            const float f = fast_exp2(x[DK] - top);
            o = fmaf(f, x[d], o);
            sum = fmaf(f, x[DK + 1], sum);
        }
        if (a.splits == 1) {
            a.out[((int64_t)unit * G + g) * DK + d] = sum > 0.f ? o / sum : 0.f;
        } else {
            float *part = a.part + (((int64_t)unit * G + g) * a.splits + split) * (DK + 2);
            part[d] = o;
            if (d == 0) {
                part[DK] = top;
                part[DK + 1] = sum;
            }
        }
    }
}

// Merges the ranges of one (sequence, query head) that its length reaches.  Thread per coordinate; the ranges' loads are issued eight at a time.
__global__ __launch_bounds__(128) void attend_pages_merge_kernel(const float *__restrict__ part, float *__restrict__ out,
                                                                 const int32_t *__restrict__ lengths, int splits, int chunk, int d_k, int per_sequence,
                                                                 int W, int page_log2)
{
    constexpr int GR = 8;
    const int head = blockIdx.x, d = threadIdx.x;
    const int length = clamp_length(lengths[head / per_sequence], W, page_log2);
    int n = (length + chunk - 1) / chunk;
    n = n < 1 ? 1 : n > splits ? splits : n;
    const float *x = part + (int64_t)head * splits * (d_k + 2);
    float top = -1e30f, o = 0.f, z = 0.f;
    for (int s0 = 0; s0 < n; s0 += GR) {
        float m_[GR], z_[GR], o_[GR];
#pragma unroll
        for (int j = 0; j < GR; ++j) {
            const float *y = x + (int64_t)(s0 + j < n ? s0 + j : s0) * (d_k + 2);
            m_[j] = y[d_k];
            z_[j] = s0 + j < n ? y[d_k + 1] : 0.f;
            o_[j] = s0 + j < n ? y[d] : 0.f;
        }
        float to = top;
#pragma unroll
        for (int j = 0; j < GR; ++j)
            to = fmaxf(to, m_[j]);
        const float fix = fast_exp2(top - to);
        o *= fix;
        z *= fix;
#pragma unroll
        for (int j = 0; j < GR; ++j) {
            const float f = fast_exp2(m_[j] - to);
            o = fmaf(f, o_[j], o);
            z = fmaf(f, z_[j], z);
        }
        top = to;
    }
    out[(int64_t)head * d_k + d] = z > 0.f ? o / z : 0.f;
}

// ---- host -------------------------------------------------------------------------------------------------------
static int attend_waves(int G, int m)
{
    const int tables = G * m;       // KB
    return tables <= 16 ? 4 : tables <= 32 ? 8 : tables <= 64 ? 16 : 8;
}

// Ranges per (sequence, key/value head).
static int attend_auto_splits(const lookat_page_pool *p, int32_t B, int32_t G, int64_t longest)
{
    const int64_t units = (int64_t)B * p->H;
    int64_t want = (1024 + units - 1) / units;
    const int64_t cap = (longest + 1023) / 1024;
    want = want < cap ? want : cap;
    return (int)(want < 1 ? 1 : want);
}

static int check_attend(const lookat_page_pool *pool, int32_t B, int32_t group, int32_t W, int64_t max_length, int32_t num_splits)
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
    if (num_splits < 0 || num_splits > 65535)
        return fail(LOOKAT_ERR_SHAPE, "num_splits=%d out of range [0,65535]", num_splits);
    return LOOKAT_OK;
}

static int64_t longest_of(const lookat_page_pool *pool, int32_t W, int64_t max_length)
{
    const int64_t room = (int64_t)W * pool->page;
    return max_length > 0 && max_length < room ? max_length : room;
}

template <int DK, int M, int G>
static int launch_attend(const PoolArgs &p, const AttendArgs &a, bool fp8, dim3 grid, hipStream_t st)
{
    const int waves = attend_waves(G, M);
    const size_t lds = attend_lds_bytes(G, M, DK, waves);
    const void *f = fp8 ? reinterpret_cast<const void *>(&attend_pages_kernel<DK, M, G, true>)
                        : reinterpret_cast<const void *>(&attend_pages_kernel<DK, M, G, false>);
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess)
            return fail(LOOKAT_ERR_HIP, "lookat_attend_pages: %s", hipGetErrorString(e));
    }
    if (fp8)
        hipLaunchKernelGGL((attend_pages_kernel<DK, M, G, true>), grid, dim3(waves * kWave), lds, st, p, a);
    else
        hipLaunchKernelGGL((attend_pages_kernel<DK, M, G, false>), grid, dim3(waves * kWave), lds, st, p, a);
    return check_launch("lookat_attend_pages");
}
template <int DK, int M>
static int launch_attend_g(int G, const PoolArgs &p, const AttendArgs &a, bool fp8, dim3 grid, hipStream_t st)
{
    switch (G) {
    case 1: return launch_attend<DK, M, 1>(p, a, fp8, grid, st);
    case 2: return launch_attend<DK, M, 2>(p, a, fp8, grid, st);
    case 4: return launch_attend<DK, M, 4>(p, a, fp8, grid, st);
    default: return launch_attend<DK, M, 8>(p, a, fp8, grid, st);
    }
}
template <int DK>
static int launch_attend_m(int G, const PoolArgs &p, const AttendArgs &a, bool fp8, dim3 grid, hipStream_t st)
{
    switch (p.m) {
    case 2: return launch_attend_g<DK, 2>(G, p, a, fp8, grid, st);
    case 4: return launch_attend_g<DK, 4>(G, p, a, fp8, grid, st);
    case 8: return launch_attend_g<DK, 8>(G, p, a, fp8, grid, st);
    default: return launch_attend_g<DK, 16>(G, p, a, fp8, grid, st);
    }
}

}  // namespace lookat

extern "C" int32_t lookat_attend_pages_auto_splits(const lookat_page_pool *pool, int32_t B, int32_t group, int32_t W, int64_t max_length)
{
    using namespace lookat;
    clear_error();
    if (check_attend(pool, B, group, W, max_length, 0) != LOOKAT_OK)
        return 0;
    return attend_auto_splits(pool, B, group, longest_of(pool, W, max_length));
}

extern "C" size_t lookat_attend_pages_workspace_bytes(const lookat_page_pool *pool, int32_t B, int32_t group, int32_t W, int64_t max_length,
                                                      int32_t num_splits)
{
    using namespace lookat;
    clear_error();
    if (check_attend(pool, B, group, W, max_length, num_splits) != LOOKAT_OK)
        return 0;
    const int S = num_splits ? num_splits : attend_auto_splits(pool, B, group, longest_of(pool, W, max_length));
    return S == 1 ? 0 : (size_t)B * pool->H * group * S * (pool->d_k + 2) * sizeof(float);
}

extern "C" int lookat_attend_pages(const lookat_page_pool *pool, int32_t B, int32_t group, const float *lut, const int32_t *table, int32_t W,
                                   int64_t table_stride, const int32_t *lengths, int64_t max_length, float scale, int32_t num_splits,
                                   void *workspace, size_t workspace_bytes, float *out, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_attend(pool, B, group, W, max_length, num_splits))
        return rc;
    if (int rc = check_table(pool, "B", B, table, W, table_stride))
        return rc;
    if (!lut || !lengths || !out)
        return fail(LOOKAT_ERR_NULL, "lut, lengths and out must be non-NULL");
    if (!aligned16(lut) || !aligned16(out))
        return fail(LOOKAT_ERR_ALIGN, "lut and out must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(lengths) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "lengths must be 4-byte aligned");
    const int64_t longest = longest_of(pool, W, max_length);
    const int S = num_splits ? num_splits : attend_auto_splits(pool, B, group, longest);
    const size_t need = lookat_attend_pages_workspace_bytes(pool, B, group, W, max_length, S);
    if (need) {
        if (!workspace || workspace_bytes < need)
            return fail(LOOKAT_ERR_WORKSPACE, "workspace of %zu bytes needed for %d splits, got %zu", need, S, workspace ? workspace_bytes : (size_t)0);
        if (!aligned16(workspace))
            return fail(LOOKAT_ERR_ALIGN, "workspace must be 16-byte aligned");
    }
    const int64_t units = (int64_t)B * pool->H;
    const int64_t groups = (units + kXcds - 1) / kXcds * kXcds * S;
    if (groups > 0x7fffffffLL || units * group > 0x7fffffffLL)
        return fail(LOOKAT_ERR_UNSUPPORTED, "B*H*num_splits=%lld workgroups exceed one launch", (long long)groups);
    const PoolArgs p = pool_args(pool);
    AttendArgs a;
    a.lut = lut;
    a.table = table;
    a.lengths = lengths;
    a.part = static_cast<float *>(workspace);
    a.out = out;
    a.table_stride = table_stride;
    a.W = W;
    a.units = (int32_t)units;
    a.splits = S;
    a.chunk = (int32_t)(((longest + S - 1) / S + kTile - 1) / kTile * kTile);
    a.scale_log2e = scale * kLog2e;
    const bool fp8 = pool->value_type == LOOKAT_VALUES_E4M3;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)groups);
    const int rc = p.d_k == 64 ? launch_attend_m<64>(group, p, a, fp8, grid, st) : launch_attend_m<128>(group, p, a, fp8, grid, st);
    if (rc != LOOKAT_OK || S == 1)
        return rc;
    hipLaunchKernelGGL(attend_pages_merge_kernel, dim3((unsigned)(units * group)), dim3(p.d_k), 0, st, a.part, out, lengths, S, a.chunk, p.d_k,
                       pool->H * group, W, p.page_log2);
    return check_launch("lookat_attend_pages (merge)");
}
