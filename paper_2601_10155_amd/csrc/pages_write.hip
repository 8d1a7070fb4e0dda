// Tokens into the pages of an 8-bit cache: codes copied, values quantised with one power-of-two exponent per page and head.
//
//   e = min { e : max |v| <= Q 2^e } (Q = 127 or 448),   q = round(v 2^-e)      (kept tokens: q' = round(q 2^(e_old - e)))
//
// v 2^-e is exact in fp32, so every stored number is one rounding (to nearest, ties to even) away from its value, whatever computes it.
// Memory-bound: each value is read once (2 or 4 bytes) and written once (1 byte).  A thread owns 8 tokens x 16 bytes of coordinates (8 in
// fp16, 4 in fp32): it loads 8 rows of 16 bytes, all requested before the first is used, keeps them in registers while the page's threads
// agree on the exponent, and writes what those numbers occupy in the page ([octet][coordinate][token]: 64 or 32 consecutive bytes) as 16-byte
// stores: the transposition costs no shared memory.  A single token (a decode step's) has a kernel of its own, a wavefront per head.
// Measured: 4 x 32 x 2048 fp32 tokens, d_k = 128, m = 16 (150 MB) 28.0 us, 5.3 TB/s (a copy of 1 GiB: 5.1); 8 x 32 x 8192 fp16 (0.83 GB) 172 us,
// 4.8 TB/s; one token of 32 x 12 3.1 us (launch and three dependent loads).  Loads past the cache: 28.3 us against 33.5 without (fp32, more than
// the cache holds; fp16 prompts that fit it 21.2 / 18.7); stores past it cost (the 0.83 GB: 287 us, 64 bytes at a time reach HBM).
#include "pages_quantise.h"

namespace lookat {

struct WriteArgs {
    const uint8_t *codes;
    const void *values;
    const int32_t *table, *lengths, *counts;
    int64_t code_stride, value_stride, table_stride;
    int64_t N;
    int32_t W;
};

// Where the tokens of a sequence go: row 0 at position `first`, positions [start, end) are written (all in 64 bits: lengths and counts may be
// any 32-bit numbers).
struct Span {
    int64_t first;
    int start, end;
};
__device__ __forceinline__ Span span_of(const WriteArgs &a, int b, int page_log2)
{
    const int64_t given = a.lengths[b] < 0 ? 0 : a.lengths[b], most = (int64_t)a.W << page_log2;
    int64_t count = a.counts ? a.counts[b] : a.N;
    count = count < 0 ? 0 : count;
    Span s;
    s.first = given - count;
    int64_t end = s.first + (count < a.N ? count : a.N);
    end = end < most ? end : most;
    const int64_t start = s.first > 0 ? s.first : 0;
    s.end = (int)(end > 0 ? end : 0);
    s.start = (int)(start < s.end ? start : s.end);
    return s;
}

template <typename FT>
__device__ __forceinline__ void to_f32(const u32x4 &raw, float (&x)[16 / sizeof(FT)])
{
    if constexpr (sizeof(FT) == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t w = raw[k];                            // (a bit cast of the element itself takes element 0 for every k)
            const float2 f = __half22float2(__builtin_bit_cast(__half2, w));
            x[2 * k] = f.x;
            x[2 * k + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            x[k] = __uint_as_float(raw[k]);
    }
}

// The largest value of the caller's aligned group of 2^n lanes, n in 4 to 6.
__device__ __forceinline__ float group_top(float x, int n)
{
    float a, b;
    x = fmaxf(x, dpp_mov<0xB1>(x, x));
    x = fmaxf(x, dpp_mov<0x4E>(x, x));
    x = fmaxf(x, dpp_mov<0x141>(x, x));
    x = fmaxf(x, dpp_mov<0x140>(x, x));
    if (n > 4) {
        lanes_xor16(x, a, b);
        x = fmaxf(a, b);
    }
    if (n > 5) {
        lanes_xor32(x, a, b);
        x = fmaxf(a, b);
    }
    return x;
}

constexpr int kWriteThreads = 512;

// grid: (touched page of the sequence, group of heads, sequence)
template <int DK, typename FT, bool FP8>
__global__ __launch_bounds__(kWriteThreads) void pages_write_kernel(PoolArgs p, WriteArgs a)
{
    constexpr int CW = 16 / sizeof(FT);                           // coordinates of a thread
    constexpr int groups = DK / CW, groups_log2 = groups == 8 ? 3 : groups == 16 ? 4 : 5;
    const int b = blockIdx.z, tid = threadIdx.x;
    const int page = 1 << p.page_log2;
    const int per_page_log2 = p.page_log2 - 3 + groups_log2;      // threads per page: 16 to 512
    const int item = tid & ((1 << per_page_log2) - 1);
    const int h = blockIdx.y * (kWriteThreads >> per_page_log2) + (tid >> per_page_log2);
    const Span span = span_of(a, b, p.page_log2);
    const int slot = (span.start >> p.page_log2) + blockIdx.x;    // entry of the sequence's row
    if (slot >= a.W)
        return;
    const int p0 = slot << p.page_log2;
    if (p0 >= span.end || span.end <= span.start)
        return;
    const int id = a.table[b * a.table_stride + slot];
    const bool mine = h < p.H;
    const int from = span.start > p0 ? span.start - p0 : 0;       // tokens [from, to) of the page are new, [0, from) are kept
    const int to = span.end - p0 < page ? span.end - p0 : page;
    const int octet = item >> groups_log2, t0 = octet * 8, col = (item & (groups - 1)) * CW;
    const bool fresh = mine && t0 < to && t0 + 8 > from, whole = t0 >= from && t0 + 8 <= to;
    const FT *rows = static_cast<const FT *>(a.values) + ((int64_t)b * p.H + h) * a.value_stride + (p0 - span.first) * DK + col;

    u32x4 raw[8];
    if (fresh) {
        // (rows outside the new ones repeat the nearest new one: no branch between the loads, and the maximum does not mind)
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const int at = t0 + t < from ? from : t0 + t >= to ? to - 1 : t0 + t;
            raw[t] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(rows + (int64_t)at * DK));
        }
    } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
            raw[t] = (u32x4){0, 0, 0, 0};
    }
    if ((uint32_t)id >= (uint32_t)p.pages)
        return;
    const int64_t place = (int64_t)id * p.H + h;
    u32x4 *bytes = reinterpret_cast<u32x4 *>(p.values + place * ((int64_t)page * DK) + (t0 * DK + col * 8));
    int old_e = kLowExponent;
    if (mine && from > 0)
        old_e = p.exponents[place];
    float top = 0.f;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        float x[CW];
        to_f32<FT>(raw[t], x);
#pragma unroll
        for (int k = 0; k < CW; ++k)
            top = fmaxf(top, fabsf(x[k]));                        // (a NaN is not the larger one)
    }
    top = group_top(top, per_page_log2);
    if (per_page_log2 > 6) {
        // (the old exponent goes through shared memory too: every wavefront has it before one of them writes the new one)
        __shared__ float tops[kWriteThreads / kWave];
        __shared__ int olds[kWriteThreads / kWave];
        if ((tid & (kWave - 1)) == 0) {
            tops[tid / kWave] = top;
            olds[tid / kWave] = old_e;
        }
        __syncthreads();
        const int waves = 1 << (per_page_log2 - 6), w0 = (tid / kWave) & ~(waves - 1);
        for (int w = 0; w < waves; ++w)
            top = fmaxf(top, tops[w0 + w]);
        old_e = olds[tid / kWave];
    }
    if (!mine)
        return;
    int e = exponent_of<FP8>(top);
    e = from > 0 && old_e > e ? old_e : e;
    if (item == 0)
        p.exponents[place] = (int8_t)e;
    const bool again = t0 < from && e != old_e;                   // kept tokens of this octet get the new exponent
    if (fresh || again) {
        const float down = two_to(-e), back = rescale(old_e, e);
        u32x4 out[CW / 2];
#pragma unroll
        for (int t = 0; t < 8; t += 4) {
            float x[4][CW];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                to_f32<FT>(raw[t + i], x[i]);
#pragma unroll
            for (int c = 0; c < CW; ++c)
                out[c / 2][2 * (c % 2) + t / 4] = pack4<FP8>(x[0][c] * down, x[1][c] * down, x[2][c] * down, x[3][c] * down);
        }
        if (!whole) {
            // kept tokens, in the new exponent, and what lies behind the last token, as it was
            uint32_t is_new[2], is_kept[2];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                is_new[w] = is_kept[w] = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int token = t0 + 4 * w + i;
                    is_kept[w] |= token < from ? 0xffu << (8 * i) : 0u;
                    is_new[w] |= token >= from && token < to ? 0xffu << (8 * i) : 0u;
                }
            }
#pragma unroll
            for (int k = 0; k < CW / 2; ++k) {
                const u32x4 was = bytes[k];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t kept = was[j];
                    if (again) {
                        float x[4];
                        unpack4<FP8>(was[j], x);
                        kept = pack4<FP8>(x[0] * back, x[1] * back, x[2] * back, x[3] * back);
                    }
                    out[k][j] = (out[k][j] & is_new[j & 1]) | (kept & is_kept[j & 1]) | (was[j] & ~(is_new[j & 1] | is_kept[j & 1]));
                }
            }
        }
#pragma unroll
        for (int k = 0; k < CW / 2; ++k)
            bytes[k] = out[k];
    }
    // codes: m bytes a token, one after another on both sides
    const uint8_t *src = a.codes + ((int64_t)b * p.H + h) * a.code_stride + (p0 - span.first) * p.m;
    uint8_t *dst = p.codes + (place << p.page_log2) * p.m;
    for (int t = from + item; t < to; t += 1 << per_page_log2)
        copy_code(dst, src, p.m, t);
}

// One token per sequence: a wavefront per head, a lane per DK / 64 coordinates; nothing but the token is touched unless the exponent grows.
constexpr int kTokenThreads = 256;
template <int DK, typename FT, bool FP8>
__global__ __launch_bounds__(kTokenThreads) void pages_write_token_kernel(PoolArgs p, WriteArgs a)
{
    constexpr int CL = DK / kWave;
    const int lane = threadIdx.x & (kWave - 1), b = blockIdx.y, h = blockIdx.x * (kTokenThreads / kWave) + threadIdx.x / kWave;
    if (h >= p.H)
        return;
    const int64_t head = (int64_t)b * p.H + h;
    float x[CL];
#pragma unroll
    for (int c = 0; c < CL; ++c)
        x[c] = (float)(static_cast<const FT *>(a.values)[head * a.value_stride + lane * CL + c]);
    const Span span = span_of(a, b, p.page_log2);
    if (span.end <= span.start || span.first < 0)                 // (first < 0: row 0 is not among the tokens that have a place)
        return;
    const int pos = span.start;
    const int id = a.table[b * a.table_stride + (pos >> p.page_log2)];
    if ((uint32_t)id >= (uint32_t)p.pages)
        return;
    const int page = 1 << p.page_log2, t = pos & (page - 1);
    const int64_t place = (int64_t)id * p.H + h;
    uint8_t *bytes = p.values + place * ((int64_t)page * DK);
    const int old_e = p.exponents[place];
    if (lane == 0)
        copy_code(p.codes + ((place << p.page_log2) + t) * p.m, a.codes + head * a.code_stride, p.m, 0);
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < CL; ++c)
        top = fmaxf(top, fabsf(x[c]));
    int e = exponent_of<FP8>(wave_max(top));
    e = t > 0 && old_e > e ? old_e : e;
    const float down = two_to(-e);
    if (t > 0 && e != old_e) {
        // the tokens that the page holds, in the new exponent: an octet's bytes in pieces of two coordinates
        const float back = rescale(old_e, e);
        const int pieces = ((t + 7) >> 3) * (DK / 2);
        for (int j = lane; j < pieces; j += kWave) {
            u32x4 w = reinterpret_cast<u32x4 *>(bytes)[j];
            const int t0 = j / (DK / 2) * 8;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float y[4];
                unpack4<FP8>(w[k], y);
                const uint32_t again = pack4<FP8>(y[0] * back, y[1] * back, y[2] * back, y[3] * back);
                const int n = t - t0 - 4 * (k & 1);               // kept tokens among these four
                const uint32_t kept = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
                w[k] = (again & kept) | (w[k] & ~kept);
            }
            reinterpret_cast<u32x4 *>(bytes)[j] = w;
        }
        // (the token's own bytes lie in words that other lanes have just written: after them)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_wave_barrier();
    }
    if (lane == 0)
        p.exponents[place] = (int8_t)e;
    uint8_t *own = bytes + (t >> 3) * (DK * 8) + (t & 7);
#pragma unroll
    for (int c = 0; c < CL; ++c)
        own[(lane * CL + c) * 8] = (uint8_t)pack4<FP8>(x[c] * down, 0.f, 0.f, 0.f);
}

template <int DK, typename FT, bool FP8>
static void launch_write(const PoolArgs &p, const WriteArgs &a, int B, int64_t touched, hipStream_t st)
{
    if (a.N == 1) {
        const int heads = kTokenThreads / kWave;
        hipLaunchKernelGGL((pages_write_token_kernel<DK, FT, FP8>), dim3((unsigned)((p.H + heads - 1) / heads), (unsigned)B), dim3(kTokenThreads), 0, st, p, a);
        return;
    }
    const int per_page = (1 << p.page_log2) / 8 * (DK / (16 / (int)sizeof(FT))), heads = kWriteThreads / per_page;
    hipLaunchKernelGGL((pages_write_kernel<DK, FT, FP8>), dim3((unsigned)touched, (unsigned)((p.H + heads - 1) / heads), (unsigned)B), dim3(kWriteThreads),
                       0, st, p, a);
}
template <typename FT>
static void launch_write_any(const PoolArgs &p, const WriteArgs &a, bool fp8, int B, int64_t touched, hipStream_t st)
{
    if (p.d_k == 64)
        fp8 ? launch_write<64, FT, true>(p, a, B, touched, st) : launch_write<64, FT, false>(p, a, B, touched, st);
    else
        fp8 ? launch_write<128, FT, true>(p, a, B, touched, st) : launch_write<128, FT, false>(p, a, B, touched, st);
}

}  // namespace lookat

extern "C" int lookat_pages_write(const lookat_page_pool *pool, int32_t B, int64_t N, const uint8_t *codes, int64_t code_stride_bh,
                                  const void *values, lookat_dtype value_dtype, int64_t value_stride_bh, const int32_t *table, int32_t W,
                                  int64_t table_stride, const int32_t *lengths, const int32_t *counts, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_pool(pool))
        return rc;
    if (N < 0)
        return fail(LOOKAT_ERR_SHAPE, "N=%lld must not be negative", (long long)N);
    if (value_dtype != LOOKAT_F16 && value_dtype != LOOKAT_F32)
        return fail(LOOKAT_ERR_DTYPE, "value_dtype=%d is neither LOOKAT_F16 nor LOOKAT_F32", (int)value_dtype);
    if (int rc = check_table(pool, "B", B, table, W, table_stride))
        return rc;
    if (N == 0)
        return LOOKAT_OK;
    if (!codes || !values || !lengths)
        return fail(LOOKAT_ERR_NULL, "codes, values and lengths must be non-NULL");
    if (N > (1 << 30))
        return fail(LOOKAT_ERR_UNSUPPORTED, "N=%lld: at most 2^30 rows", (long long)N);
    if (code_stride_bh < N * pool->m || value_stride_bh < N * pool->d_k)
        return fail(LOOKAT_ERR_SHAPE, "code_stride_bh=%lld / value_stride_bh=%lld smaller than one (b,h) slab", (long long)code_stride_bh,
                    (long long)value_stride_bh);
    const int64_t bytes = value_dtype == LOOKAT_F16 ? 2 : 4;
    if (!aligned16(values) || (value_stride_bh * bytes) % 16)
        return fail(LOOKAT_ERR_ALIGN, "values and value_stride_bh must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(codes) % pool->m) || (code_stride_bh % pool->m))
        return fail(LOOKAT_ERR_ALIGN, "codes and code_stride_bh must be multiples of m=%d bytes", pool->m);
    if ((reinterpret_cast<uintptr_t>(lengths) | reinterpret_cast<uintptr_t>(counts)) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "lengths and counts must be 4-byte aligned");
    const PoolArgs p = pool_args(pool);
    WriteArgs a;
    a.codes = codes;
    a.values = values;
    a.table = table;
    a.lengths = lengths;
    a.counts = counts;
    a.code_stride = code_stride_bh;
    a.value_stride = value_stride_bh;
    a.table_stride = table_stride;
    a.N = N;
    a.W = W;
    int64_t touched = (N + pool->page - 2) / pool->page + 1;      // N tokens from anywhere in a page on
    touched = touched < W ? touched : W;
    if (!fits_launch(touched, kWriteThreads))
        return fail(LOOKAT_ERR_UNSUPPORTED, "N=%lld: %lld pages of a sequence exceed one launch", (long long)N, (long long)touched);
    const bool fp8 = pool->value_type == LOOKAT_VALUES_E4M3;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (value_dtype == LOOKAT_F16)
        launch_write_any<__half>(p, a, fp8, B, touched, st);
    else
        launch_write_any<float>(p, a, fp8, B, touched, st);
    return check_launch("lookat_pages_write");
}
