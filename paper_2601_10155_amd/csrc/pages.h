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
// One launch counts its threads along x in 32 bits.
inline bool fits_launch(int64_t groups, int threads) { return groups * threads <= 0xffffffffLL; }

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

// A page is copied in parts of kCopyPart 16-byte units, its codes first, then its values (the exponents, H bytes, go with part 0).
constexpr int kCopyThreads = 256;
constexpr int kCopyUnits = 4;             // per thread, all requested before the first is stored
constexpr uint32_t kCopyPart = kCopyThreads * kCopyUnits;
__host__ __device__ __forceinline__ uint32_t code_units(const PoolArgs &p) { return ((uint32_t)p.H << p.page_log2) * (uint32_t)p.m / 16u; }
__host__ __device__ __forceinline__ uint32_t value_units(const PoolArgs &p) { return ((uint32_t)p.H << p.page_log2) * (uint32_t)p.d_k / 16u; }
__host__ __device__ __forceinline__ uint32_t page_parts(const PoolArgs &p) { return (code_units(p) + value_units(p) + kCopyPart - 1) / kCopyPart; }

// One workgroup of kCopyThreads copies part `part` of page src onto page dst (both in range, src != dst).  A thread's units behind the page's
// last one repeat that one instead of being skipped, so that all loads go out together, without a branch between them.
// Stores carry the non-temporal hint: the copy is not read again by this kernel, and a plain store takes cache room from the pages still
// to be read.  us for 1024 pages of 70 KB: plain 32.5, hint on stores 23.7 (6.0 TB/s), on loads 25.4, on both 29.4; 8 units a thread 33.7, 2 32.3.
__device__ __forceinline__ void copy_page_part(const PoolArgs &p, int src, int dst, uint32_t part)
{
    const uint32_t codes = code_units(p), values = value_units(p), units = codes + values;
    const uint32_t u0 = part * kCopyPart + threadIdx.x;
    u32x4 *code_base = reinterpret_cast<u32x4 *>(p.codes), *value_base = reinterpret_cast<u32x4 *>(p.values);
    // (the values' bases are moved back by the codes' units, so that one index serves both)
    const u32x4 *from_codes = code_base + (int64_t)src * codes, *from_values = value_base + ((int64_t)src * values - codes);
    u32x4 *to_codes = code_base + (int64_t)dst * codes, *to_values = value_base + ((int64_t)dst * values - codes);
    int8_t e = 0;
    const bool exponents = part == 0 && (int)threadIdx.x < p.H;
    if (exponents)
        e = p.exponents[(int64_t)src * p.H + threadIdx.x];
    u32x4 x[kCopyUnits];
#pragma unroll
    for (int k = 0; k < kCopyUnits; ++k) {
        uint32_t u = u0 + k * kCopyThreads;
        u = u < units ? u : units - 1;
        x[k] = (u < codes ? from_codes : from_values)[u];
    }
#pragma unroll
    for (int k = 0; k < kCopyUnits; ++k) {
        const uint32_t u = u0 + k * kCopyThreads;
        if (u < units)
            __builtin_nontemporal_store(x[k], (u < codes ? to_codes : to_values) + u);
    }
    if (exponents) {
        p.exponents[(int64_t)dst * p.H + threadIdx.x] = e;
        for (int h = threadIdx.x + kCopyThreads; h < p.H; h += kCopyThreads)
            p.exponents[(int64_t)dst * p.H + h] = p.exponents[(int64_t)src * p.H + h];
    }
}

#endif  // __HIPCC__

}  // namespace lookat
