// Shared pieces of the paged 8-bit cache: geometry, argument checks, how a page's bytes are addressed.
#pragma once

#include "common.h"
#include "lookat_pages.h"

namespace lookat {

// Geometry of a pool as the kernels take it.
struct PoolArgs {
    uint8_t *codes;
    uint8_t *values;
    int8_t *exponents;
    int32_t pages, H, d_k, m;
    int32_t page_log2;
};

// Checks a pool (host).  Returns LOOKAT_OK or a failure.
int check_pool(const lookat_page_pool *p);
// Checks a table of `rows` rows (host).
int check_table(const lookat_page_pool *p, const char *rows_name, int32_t rows, const int32_t *table, int32_t W, int64_t stride);
PoolArgs pool_args(const lookat_page_pool *p);

// Why not the whole of int8: attention adds a page's exponent to its logits (base 2) and takes it off the weight again for the softmax sum, in
// fp32.  A token of the lowest exponent beside one of the highest keeps its weight down to 2^-126 + 80 - 15 = 2^-61 of the largest.
constexpr int kLowExponent = -40, kHighExponent = 40;

#if defined(__HIPCC__)

__device__ __forceinline__ int clamp_length(int length, int W, int page_log2)
{
    const int most = W << page_log2;      // (at most 2^30)
    return length < 0 ? 0 : length < most ? length : most;
}

// 16-byte units of one page: its codes, then its values (the exponents go apart: H bytes).
__host__ __device__ __forceinline__ uint32_t page_units(const PoolArgs &p)
{
    return ((uint32_t)p.H << p.page_log2) * (uint32_t)(p.m + p.d_k) / 16u;
}
constexpr int kCopyThreads = 256;
constexpr int kCopyUnits = 4;             // 16-byte units per thread and part, all requested before the first is stored
constexpr uint32_t kCopyPart = kCopyThreads * kCopyUnits;
__host__ __device__ __forceinline__ uint32_t page_parts(const PoolArgs &p) { return (page_units(p) + kCopyPart - 1) / kCopyPart; }

// One workgroup of kCopyThreads copies part `part` of page src onto page dst (both in range, src != dst).
__device__ __forceinline__ void copy_page_part(const PoolArgs &p, int src, int dst, uint32_t part)
{
    const uint32_t units = page_units(p);
    const uint32_t code_units = ((uint32_t)p.H << p.page_log2) * (uint32_t)p.m / 16u;
    const uint32_t value_units = units - code_units;
    const uint4 *codes = reinterpret_cast<const uint4 *>(p.codes), *values = reinterpret_cast<const uint4 *>(p.values);
    const int64_t code_from = (int64_t)src * code_units, code_to = (int64_t)dst * code_units;
    const int64_t value_from = (int64_t)src * value_units, value_to = (int64_t)dst * value_units;
    uint4 x[kCopyUnits];
#pragma unroll
    for (int k = 0; k < kCopyUnits; ++k) {
        const uint32_t u = part * kCopyPart + k * kCopyThreads + threadIdx.x;
        if (u < units)
            x[k] = u < code_units ? codes[code_from + u] : values[value_from + (u - code_units)];
    }
#pragma unroll
    for (int k = 0; k < kCopyUnits; ++k) {
        const uint32_t u = part * kCopyPart + k * kCopyThreads + threadIdx.x;
        if (u < units) {
            if (u < code_units)
                reinterpret_cast<uint4 *>(p.codes)[code_to + u] = x[k];
            else
                reinterpret_cast<uint4 *>(p.values)[value_to + (u - code_units)] = x[k];
        }
    }
    if (part == 0)
        for (int h = threadIdx.x; h < p.H; h += kCopyThreads)
            p.exponents[(int64_t)dst * p.H + h] = p.exponents[(int64_t)src * p.H + h];
}

#endif  // __HIPCC__

}  // namespace lookat
