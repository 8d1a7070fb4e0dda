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

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// A page is copied in parts of one region, codes or values, kCopyPart 16-byte units each (the exponents, H bytes, go with part 0).
constexpr int kCopyThreads = 256;
constexpr int kCopyUnits = 4;             // per thread, all requested before the first is stored
constexpr uint32_t kCopyPart = kCopyThreads * kCopyUnits;
__host__ __device__ __forceinline__ uint32_t code_units(const PoolArgs &p) { return ((uint32_t)p.H << p.page_log2) * (uint32_t)p.m / 16u; }
__host__ __device__ __forceinline__ uint32_t value_units(const PoolArgs &p) { return ((uint32_t)p.H << p.page_log2) * (uint32_t)p.d_k / 16u; }
__host__ __device__ __forceinline__ uint32_t parts_of(uint32_t units) { return (units + kCopyPart - 1) / kCopyPart; }
__host__ __device__ __forceinline__ uint32_t page_parts(const PoolArgs &p) { return parts_of(code_units(p)) + parts_of(value_units(p)); }

// One workgroup of kCopyThreads copies part `part` of page src onto page dst (both in range, src != dst).  A thread's last units repeat the
// region's last one instead of being skipped, so that all loads go out together, without a branch between them.
__device__ __forceinline__ void copy_page_part(const PoolArgs &p, int src, int dst, uint32_t part)
{
    const uint32_t code_parts = parts_of(code_units(p));
    const bool values = part >= code_parts;
    const uint32_t units = values ? value_units(p) : code_units(p);
    const uint32_t u0 = (values ? part - code_parts : part) * kCopyPart + threadIdx.x;
    u32x4 *base = reinterpret_cast<u32x4 *>(values ? p.values : p.codes);
    const u32x4 *from = base + (int64_t)src * units;
    u32x4 *to = base + (int64_t)dst * units;
    int8_t e = 0;
    const bool exponents = part == 0 && (int)threadIdx.x < p.H;
    if (exponents)
        e = p.exponents[(int64_t)src * p.H + threadIdx.x];
    u32x4 x[kCopyUnits];
#pragma unroll
    for (int k = 0; k < kCopyUnits; ++k) {
        const uint32_t u = u0 + k * kCopyThreads;
        x[k] = from[u < units ? u : units - 1];
    }
#pragma unroll
    for (int k = 0; k < kCopyUnits; ++k) {
        const uint32_t u = u0 + k * kCopyThreads;
        if (u < units)
            to[u] = x[k];
    }
    if (exponents) {
        p.exponents[(int64_t)dst * p.H + threadIdx.x] = e;
        for (int h = threadIdx.x + kCopyThreads; h < p.H; h += kCopyThreads)
            p.exponents[(int64_t)dst * p.H + h] = p.exponents[(int64_t)src * p.H + h];
    }
}

#endif  // __HIPCC__

}  // namespace lookat
