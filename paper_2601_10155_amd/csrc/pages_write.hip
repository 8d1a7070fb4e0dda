// Tokens into the pages of an 8-bit cache: codes copied, values quantised with one power-of-two exponent per page and head.
//
//   e = min { e : max |v| <= Q 2^e } (Q = 127 or 448),   q = round(v 2^-e)      (kept tokens: q' = round(q 2^(e_old - e)))
//
// v 2^-e is exact in fp32, so every stored number is one rounding (to nearest, ties to even) away from its value, whatever computes it.
// Memory-bound: each value is read once (2 or 4 bytes) and written once (1 byte).  A thread owns 8 tokens x 8 coordinates: it
// loads 8 rows of 16 (fp16) or 32 (fp32) bytes, all requested before the first is used, keeps them in registers while the page's
// threads agree on the exponent, and writes the 64 bytes that those numbers occupy in the page ([octet][coordinate][token]) as
// four 16-byte stores: the transposition costs no shared memory.
#include "pages.h"

namespace lookat {

struct WriteArgs {
    const uint8_t *codes;
    const void *values;
    const int32_t *table, *lengths, *counts;
    int64_t code_stride, value_stride, table_stride;
    int64_t N;
    int32_t W;
};

typedef float v2f __attribute__((ext_vector_type(2)));

template <bool FP8>
__device__ __forceinline__ int exponent_of(float top)
{
    const uint32_t bits = __float_as_uint(top);
    const int e = (int)(bits >> 23) - 127;
    const uint32_t mant = bits & 0x7fffffu;
    // largest stored number: 127 = 1.984375 * 2^6, 448 = 1.75 * 2^8
    const int x = FP8 ? e - 8 + (mant > 0x600000u) : e - 6 + (mant > 0x7e0000u);
    return x < kLowExponent ? kLowExponent : x > kHighExponent ? kHighExponent : x;   // (zero and fp32's subnormals: the lowest)
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // e in [-126, 127]

// Four scaled numbers to four stored bytes.
template <bool FP8>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d)
{
    constexpr float top = FP8 ? 448.f : 127.f;
    const float x[4] = {a, b, c, d};
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float r = FP8 ? x[i] : rintf(x[i]);
        y[i] = r != r ? 0.f : fminf(fmaxf(r, -top), top);
    }
    if constexpr (FP8) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    } else {
        return ((uint32_t)(int)y[0] & 0xffu) | ((uint32_t)(int)y[1] & 0xffu) << 8 | ((uint32_t)(int)y[2] & 0xffu) << 16 |
               (uint32_t)(int)y[3] << 24;
    }
}
template <bool FP8>
__device__ __forceinline__ void unpack4(uint32_t w, float (&x)[4])
{
    if constexpr (FP8) {
        const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo.x, x[1] = lo.y, x[2] = hi.x, x[3] = hi.y;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = (float)(int8_t)(w >> (8 * i));
    }
}

constexpr int kWriteThreads = 256;

// grid: (touched page of the sequence, group of heads, sequence)
template <int DK, typename FT, bool FP8>
__global__ __launch_bounds__(kWriteThreads) void pages_write_kernel(PoolArgs p, WriteArgs a)
{
    const int b = blockIdx.z, tid = threadIdx.x;
    const int page = 1 << p.page_log2;
    // threads per page: (page / 8) octets x (DK / 8) coordinate groups, 16 to 256
    const int per_page_log2 = p.page_log2 - 3 + (DK == 128 ? 4 : 3);
    const int item = tid & ((1 << per_page_log2) - 1);
    const int h = blockIdx.y * (kWriteThreads >> per_page_log2) + (tid >> per_page_log2);
    const int most = a.W << p.page_log2;
    // all positions in 64 bits: lengths and counts may be any 32-bit numbers
    const int64_t given = a.lengths[b] < 0 ? 0 : a.lengths[b];
    int64_t count = a.counts ? a.counts[b] : a.N;
    count = count < 0 ? 0 : count;
    const int64_t first = given - count;                          // position of row 0
    int64_t end = first + (count < a.N ? count : a.N);            // behind the last row's
    end = end < most ? end : most;
    const int start = (int)(first > 0 ? first : 0);
    if (end <= start)
        return;
    const int slot = (start >> p.page_log2) + blockIdx.x;         // entry of the sequence's row
    const int p0 = slot << p.page_log2;
    if (p0 >= end)
        return;
    const int id = a.table[b * a.table_stride + slot];
    if ((uint32_t)id >= (uint32_t)p.pages)
        return;
    const bool mine = h < p.H;
    const int from = start > p0 ? start - p0 : 0;                 // tokens [from, to) of the page are new, [0, from) are kept
    const int to = (int)(end - p0 < page ? end - p0 : page);
    const int octet = item / (DK / 8), col = (item % (DK / 8)) * 8;
    const int64_t place = (int64_t)id * p.H + h;
    const FT *rows = static_cast<const FT *>(a.values) + ((int64_t)b * p.H + h) * a.value_stride + (p0 - first + octet * 8) * DK + col;

    float v[8][8];                                                // [token][coordinate]
    float top = 0.f;
    const bool fresh = mine && octet * 8 < to && octet * 8 + 8 > from;
    uint4 raw[8][sizeof(FT) / 2];
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
        for (int k = 0; k < (int)sizeof(FT) / 2; ++k) {
            raw[t][k] = make_uint4(0, 0, 0, 0);
            if (fresh && octet * 8 + t >= from && octet * 8 + t < to)
                raw[t][k] = reinterpret_cast<const uint4 *>(rows + (int64_t)t * DK)[k];
        }
    int old_e = kLowExponent;
    if (mine && from > 0)
        old_e = p.exponents[place];
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        if constexpr (sizeof(FT) == 2) {
            const __half2 *x = reinterpret_cast<const __half2 *>(&raw[t][0]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = __half22float2(x[k]);
                v[t][2 * k] = f.x;
                v[t][2 * k + 1] = f.y;
            }
        } else {
            const float *x = reinterpret_cast<const float *>(&raw[t][0]);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                v[t][k] = x[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            top = fmaxf(top, fabsf(v[t][k]));                     // (a NaN is not the larger one)
    }
    // the page's threads are 16, 32 or 64 lanes of a wavefront, or 2 or 4 wavefronts
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const float other = __shfl_xor(top, d);
        top = d < (1 << per_page_log2) ? fmaxf(top, other) : top;
    }
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
    const bool again = from > octet * 8 && e != old_e;            // kept tokens of this octet get the new exponent
    if (fresh || again) {
        uint4 *bytes = reinterpret_cast<uint4 *>(p.values + place * ((int64_t)page * DK) + (octet * DK + col) * 8);
        uint4 was[4];
        const bool partly = octet * 8 < from || octet * 8 + 8 > to;
        if (partly) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                was[k] = bytes[k];
        }
        // (an exponent that this kernel did not write may be any int8: 2^(old - e) down to 2^-168, the lowest rounds everything to zero too)
        const float down = two_to(-e), back = two_to(old_e - e < -126 ? -126 : old_e - e);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t w[4];
#pragma unroll
            for (int c2 = 0; c2 < 2; ++c2) {
                const int c = 2 * k + c2;
#pragma unroll
                for (int t4 = 0; t4 < 2; ++t4) {
                    const int t = 4 * t4;
                    w[2 * c2 + t4] = pack4<FP8>(v[t][c] * down, v[t + 1][c] * down, v[t + 2][c] * down, v[t + 3][c] * down);
                    if (partly) {
                        const uint32_t old = reinterpret_cast<const uint32_t *>(&was[k])[2 * c2 + t4];
                        uint32_t kept = old;
                        if (again) {
                            float x[4];
                            unpack4<FP8>(old, x);
                            kept = pack4<FP8>(x[0] * back, x[1] * back, x[2] * back, x[3] * back);
                        }
                        uint32_t out = 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int token = octet * 8 + t + i;
                            const uint32_t from_which = token < from ? kept : token < to ? w[2 * c2 + t4] : old;
                            out |= from_which & (0xffu << (8 * i));
                        }
                        w[2 * c2 + t4] = out;
                    }
                }
            }
            bytes[k] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    // codes: m bytes a token, one after another on both sides
    const int m = p.m;
    const uint8_t *src = a.codes + ((int64_t)b * p.H + h) * a.code_stride + (p0 - first) * m;
    uint8_t *dst = p.codes + (place << p.page_log2) * m;
    for (int t = from + item; t < to; t += 1 << per_page_log2) {
        if (m == 2)
            reinterpret_cast<uint16_t *>(dst)[t] = reinterpret_cast<const uint16_t *>(src)[t];
        else if (m == 4)
            reinterpret_cast<uint32_t *>(dst)[t] = reinterpret_cast<const uint32_t *>(src)[t];
        else if (m == 8)
            reinterpret_cast<uint2 *>(dst)[t] = reinterpret_cast<const uint2 *>(src)[t];
        else
            reinterpret_cast<uint4 *>(dst)[t] = reinterpret_cast<const uint4 *>(src)[t];
    }
}

template <typename FT>
static void launch_write(const PoolArgs &p, const WriteArgs &a, bool fp8, dim3 grid, hipStream_t st)
{
    const dim3 block(kWriteThreads);
    if (p.d_k == 64) {
        if (fp8)
            hipLaunchKernelGGL((pages_write_kernel<64, FT, true>), grid, block, 0, st, p, a);
        else
            hipLaunchKernelGGL((pages_write_kernel<64, FT, false>), grid, block, 0, st, p, a);
    } else {
        if (fp8)
            hipLaunchKernelGGL((pages_write_kernel<128, FT, true>), grid, block, 0, st, p, a);
        else
            hipLaunchKernelGGL((pages_write_kernel<128, FT, false>), grid, block, 0, st, p, a);
    }
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
    const int per_page = pool->page / 8 * (pool->d_k / 8), heads = kWriteThreads / per_page;
    const dim3 grid((unsigned)touched, (unsigned)((p.H + heads - 1) / heads), (unsigned)B);
    const bool fp8 = pool->value_type == LOOKAT_VALUES_E4M3;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (value_dtype == LOOKAT_F16)
        launch_write<__half>(p, a, fp8, grid, st);
    else
        launch_write<float>(p, a, fp8, grid, st);
    return check_launch("lookat_pages_write");
}
