// Upkeep of the paged cache: copying, forking, freeing, reserving and compacting pages.
//
// The books (tables, lengths, counts) stay on the device: a decode loop captured in a graph reserves its next tokens without a trip
// to the host.  Every result is a function of the books alone: free pages are taken in ascending order by rank (a prefix sum over
// the counts), never by an atomic race; the only atomics are integer additions to counts, whose order does not matter.
//
// What bounds these kernels is the launch and a few dependent memory round trips (the books are tens of kilobytes): free 3.4 us, fork 3.5, reserve
// 3.6 + 4.1 (16 of 32 sequences) and 4.6 + 5.5 (192 of 384, 26 MB of shared last pages); where pages are copied, their bytes once read and once
// written: 1024 pages of 70 KB 22.4 us (6.4 TB/s), compacting a pool of 16000 pages with 4000 moves 5.2 + 28.8 us (5.1 TB/s).
#include "pages.h"

namespace lookat {

int check_pool(const lookat_page_pool *p)
{
    if (!p)
        return fail(LOOKAT_ERR_NULL, "pool is NULL");
    if (p->pages <= 0 || p->H <= 0 || p->d_k <= 0 || p->m <= 0 || p->page <= 0)
        return fail(LOOKAT_ERR_SHAPE, "pages, H, d_k, m and page must be positive (pages=%d H=%d d_k=%d m=%d page=%d)", p->pages,
                    p->H, p->d_k, p->m, p->page);
    if (p->value_type != LOOKAT_VALUES_I8 && p->value_type != LOOKAT_VALUES_E4M3)
        return fail(LOOKAT_ERR_DTYPE, "value type %d is neither LOOKAT_VALUES_I8 nor LOOKAT_VALUES_E4M3", (int)p->value_type);
    if ((p->d_k != 64 && p->d_k != 128) || (p->m != 2 && p->m != 4 && p->m != 8 && p->m != 16))
        return fail(LOOKAT_ERR_UNSUPPORTED, "paged caches handle d_k in {64,128} with m in {2,4,8,16}; got d_k=%d m=%d", p->d_k, p->m);
    if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128)
        return fail(LOOKAT_ERR_UNSUPPORTED, "page=%d: pages hold 16, 32, 64 or 128 tokens", p->page);
    if (p->pages > (1 << 30) || p->H > 4096)
        return fail(LOOKAT_ERR_UNSUPPORTED, "pages=%d, H=%d: at most 2^30 pages and 4096 heads", p->pages, p->H);
    if (!p->codes || !p->values || !p->exponents)
        return fail(LOOKAT_ERR_NULL, "the pool's codes, values and exponents must be non-NULL");
    if (!aligned16(p->codes) || !aligned16(p->values))
        return fail(LOOKAT_ERR_ALIGN, "the pool's codes and values must be 16-byte aligned");
    return LOOKAT_OK;
}

int check_table(const lookat_page_pool *p, const char *rows_name, int32_t rows, const int32_t *table, int32_t W, int64_t stride)
{
    if (rows <= 0 || W <= 0)
        return fail(LOOKAT_ERR_SHAPE, "%s=%d and W=%d must be positive", rows_name, rows, W);
    if (!table)
        return fail(LOOKAT_ERR_NULL, "table must be non-NULL");
    if (stride < W)
        return fail(LOOKAT_ERR_SHAPE, "table_stride=%lld smaller than a row of %d", (long long)stride, W);
    if (reinterpret_cast<uintptr_t>(table) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "table must be 4-byte aligned");
    if ((int64_t)W * p->page > (1 << 30))
        return fail(LOOKAT_ERR_UNSUPPORTED, "W=%d pages of %d tokens: rows of at most 2^30 tokens", W, p->page);
    if (rows > 65535)
        return fail(LOOKAT_ERR_UNSUPPORTED, "%s=%d: at most 65535 sequences", rows_name, rows);
    return LOOKAT_OK;
}

PoolArgs pool_args(const lookat_page_pool *p)
{
    PoolArgs a;
    a.codes = p->codes;
    a.values = static_cast<uint8_t *>(p->values);
    a.exponents = p->exponents;
    a.pages = p->pages;
    a.H = p->H;
    a.d_k = p->d_k;
    a.m = p->m;
    a.page_log2 = __builtin_ctz((unsigned)p->page);
    return a;
}

struct BookArgs {
    int32_t *table;
    int64_t stride;
    int32_t *lengths, *refs;
    int32_t S, W, pages, page_log2;
};

__device__ __forceinline__ int pages_of(int length, const BookArgs &a)
{
    const int n = clamp_length(length, a.W, a.page_log2);
    return (n + (1 << a.page_log2) - 1) >> a.page_log2;
}

constexpr int kBookThreads = 256;

// Sums over the workgroup of two numbers; every thread ends with them.  `s`: two ints per wavefront in LDS.
template <int THREADS>
__device__ __forceinline__ int2 block_sums(int x, int y, int *s)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        x += __shfl_xor(x, d);
        y += __shfl_xor(y, d);
    }
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0)
        reinterpret_cast<int2 *>(s)[threadIdx.x / kWave] = make_int2(x, y);
    __syncthreads();
    int2 t = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) {
        const int2 v = reinterpret_cast<const int2 *>(s)[w];
        t.x += v.x;
        t.y += v.y;
    }
    return t;
}
template <int THREADS>
__device__ __forceinline__ int block_sum(int v, int *s)
{
    return block_sums<THREADS>(v, 0, s).x;
}
// Sum over the threads before this one in the workgroup; *total = over all.
template <int THREADS>
__device__ __forceinline__ int block_before(int v, int *s, int *total)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    int up = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int t = __shfl_up(up, d);
        up += lane >= d ? t : 0;
    }
    __syncthreads();
    if (lane == kWave - 1)
        s[wave] = up;
    __syncthreads();
    int before = up - v, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) {
        before += w < wave ? s[w] : 0;
        all += s[w];
    }
    *total = all;
    return before;
}

// For two numbers of every thread: the sum of x over the threads before this one, and the sums of both over the workgroup.  `s`: two numbers
// per wavefront in LDS, not in use yet.
struct Sums {
    long long before, x, y;
};
template <int THREADS>
__device__ __forceinline__ Sums block_before_and_sums(long long x, long long y, long long *s)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    long long up = x;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const long long t = __shfl_up(up, d);
        up += lane >= d ? t : 0;
        y += __shfl_xor(y, d);
    }
    if (lane == kWave - 1) {
        s[2 * wave] = up;
        s[2 * wave + 1] = y;
    }
    __syncthreads();
    Sums r = {up - x, 0, 0};
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) {
        r.before += w < wave ? s[2 * w] : 0;
        r.x += s[2 * w];
        r.y += s[2 * w + 1];
    }
    return r;
}

// ---- copy -------------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(PoolArgs p, const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                                  int n, uint32_t parts)
{
    const uint32_t pair = blockIdx.x / parts, part = blockIdx.x % parts;
    const int from = src[pair], to = dst[pair];
    if ((uint32_t)from >= (uint32_t)p.pages || (uint32_t)to >= (uint32_t)p.pages || from == to)
        return;
    copy_page_part(p, from, to, part);
}

// Lists of slots: every workgroup of a fork or free looks through the call's list for its own slot, so the work grows with the
// square of it (us for 1500 / 16384 / 65535 entries: fork 14 / 90 / 1100, free 8 / 44 / 490).  A list as long as there can be sequences
// names everything that can take effect.
constexpr int kMostListed = 65535;

// ---- fork -------------------------------------------------------------------------------------------------------
// One workgroup per pair.  Which pairs count is decided from the call's own arguments and from lengths that no other pair of the call
// writes: a source that is somebody's destination is out, a destination belongs to the first pair that names it.
__global__ __launch_bounds__(kBookThreads) void pages_fork_kernel(BookArgs a, int n, const int32_t *__restrict__ src, const int32_t *__restrict__ dst)
{
    __shared__ __align__(8) int s[2 * kBookThreads / kWave];
    const int i = blockIdx.x, tid = threadIdx.x;
    const int from = src[i], to = dst[i];
    if ((uint32_t)from >= (uint32_t)a.S || (uint32_t)to >= (uint32_t)a.S)
        return;
    int out = 0;
    for (int j = tid; j < n; j += kBookThreads) {
        const int d = dst[j];
        out |= (d == from) | (j < i && d == to);
    }
    if (block_sum<kBookThreads>(out, s))
        return;
    // (what is read here no other workgroup writes; this one writes after all of its threads have read: block_sum's barriers)
    const int length = a.lengths[from], there = a.lengths[to];
    if (block_sum<kBookThreads>(there > 0 || length <= 0, s))
        return;
    const int pages = pages_of(length, a);
    const int32_t *row = a.table + from * a.stride;
    int32_t *row_to = a.table + to * a.stride;
    for (int w = tid; w < pages; w += kBookThreads) {
        const int id = row[w];
        row_to[w] = id;
        if ((uint32_t)id < (uint32_t)a.pages)
            atomicAdd(a.refs + id, 1);
    }
    if (tid == 0)
        a.lengths[to] = length;
}

// ---- free -------------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(kBookThreads) void pages_free_kernel(BookArgs a, const int32_t *__restrict__ slots)
{
    __shared__ __align__(8) int s[2 * kBookThreads / kWave];
    const int i = blockIdx.x, tid = threadIdx.x;
    const int slot = slots[i];
    if ((uint32_t)slot >= (uint32_t)a.S)
        return;
    int out = 0;
    for (int j = tid; j < i; j += kBookThreads)
        out |= slots[j] == slot;
    const int length = a.lengths[slot];
    if (block_sum<kBookThreads>(out, s))     // (its barriers: every thread has read the length before one writes it)
        return;
    const int pages = pages_of(length, a);
    int32_t *row = a.table + slot * a.stride;
    for (int w = tid; w < pages; w += kBookThreads) {
        const int id = row[w];
        row[w] = -1;
        if ((uint32_t)id < (uint32_t)a.pages)
            atomicSub(a.refs + id, 1);
    }
    if (tid == 0)
        a.lengths[slot] = 0;
}

// ---- reserve ----------------------------------------------------------------------------------------------------
// Two launches.  The first ranks: its page workgroups write the free pages' ids in ascending order (each counts the free pages
// ahead of its segment by itself: the counts are read from L2 a few times over instead of a chain of launches), its slot workgroups what each
// sequence needs, summed up within kRankThreads sequences.  The second adds up those at most 64 sums and gives the pages out, a workgroup per
// sequence and part of a page to copy.
struct ReservePlan {
    int32_t *free_ids;   // [pages]
    int32_t *need;       // [S] pages
    int32_t *shared;     // [S] the page to copy, or -1
    int32_t *before;     // [S] pages needed by the sequences ahead in the same kRankThreads (right where no page is missing)
    long long *sums;     // [S / kRankThreads, rounded up][2] pages needed, entries that rows are short of
    int32_t *count;      // [0]: free pages
    int32_t *copies;     // [2][S] for the caller, or NULL
};

constexpr int kRankThreads = 1024;
constexpr int kSegments = 64;            // workgroups over the pages, at most

// Which pages are in use, for a whole workgroup of kRankThreads: bit k of a thread's word is page kRankThreads * k + its index.  One pass of
// independent loads, and everything below is counted from registers: a pool of up to PIECES * kRankThreads pages.
template <int PIECES>
__device__ __forceinline__ uint64_t pages_in_use(const int32_t *__restrict__ refs, int pages)
{
    uint64_t bits = 0;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int j = k * kRankThreads + (int)threadIdx.x;
        const int r = refs[j < pages ? j : pages - 1];
        bits |= (uint64_t)(j < pages && r > 0) << k;
    }
    return bits;
}
// Those of a thread's pages in use that lie below `end`.
__device__ __forceinline__ int in_use_below(uint64_t bits, int end)
{
    const int k = end / kRankThreads, r = end % kRankThreads;
    const uint64_t whole = k >= 64 ? bits : bits & ((1ull << k) - 1);
    return __popcll(whole) + (k < 64 && (int)threadIdx.x < r ? (int)(bits >> k & 1) : 0);
}
// A thread's pages in use below `end` in a pool of any size, by a loop.
__device__ __forceinline__ int in_use_below(const int32_t *__restrict__ refs, int end)
{
    int n = 0;
    for (int j = threadIdx.x; j < end; j += kRankThreads)
        n += refs[j] > 0;
    return n;
}

// PIECES: 1, 4, 16 or 64 (pools of up to 65536 pages), 0: any size.
template <int PIECES>
__global__ __launch_bounds__(kRankThreads) void pages_reserve_rank_kernel(BookArgs a, const int32_t *__restrict__ new_lengths, ReservePlan plan,
                                                                          int segments, int segment)
{
    __shared__ __align__(8) int s[2 * kRankThreads / kWave];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= segments) {
        __shared__ long long sums[2 * kRankThreads / kWave];
        const int group = (int)blockIdx.x - segments, slot = group * kRankThreads + tid;
        const bool there = slot < a.S;
        const int page = 1 << a.page_log2;
        const int length = there && a.lengths[slot] > 0 ? a.lengths[slot] : 0, wanted = there ? new_lengths[slot] : 0;
        int need = 0, shared = -1;
        long long over = 0;                                       // entries that the row is short of
        if (wanted > length) {
            // (64-bit: lengths up to 2^31 - 1)
            const int64_t has = ((int64_t)length + page - 1) >> a.page_log2, needs = ((int64_t)wanted + page - 1) >> a.page_log2;
            need = (int)(needs - has);
            if ((length & (page - 1)) && (length >> a.page_log2) < a.W) {
                const int id = a.table[slot * a.stride + (length >> a.page_log2)];
                if ((uint32_t)id < (uint32_t)a.pages && a.refs[id] > 1) {
                    shared = id;
                    ++need;
                }
            }
            over = need > 0 && needs > a.W ? needs - a.W : 0;
        }
        const Sums t = block_before_and_sums<kRankThreads>(need, over, sums);
        if (tid == 0) {
            plan.sums[2 * group] = t.x;
            plan.sums[2 * group + 1] = t.y;
        }
        if (!there)
            return;
        plan.need[slot] = need;
        plan.shared[slot] = shared;
        plan.before[slot] = (int32_t)t.before;
        if (plan.copies) {
            plan.copies[slot] = -1;
            plan.copies[a.S + slot] = -1;
        }
        return;
    }
    const int begin = blockIdx.x * segment, end = begin + segment < a.pages ? begin + segment : a.pages;
    uint64_t bits = 0;
    int used;
    if constexpr (PIECES != 0) {
        bits = pages_in_use<PIECES>(a.refs, a.pages);
        used = in_use_below(bits, begin);
    } else {
        used = in_use_below(a.refs, begin);
    }
    int free_before = begin - block_sum<kRankThreads>(used, s);
    for (int j0 = begin; j0 < end; j0 += kRankThreads) {
        const int j = j0 + tid;
        const bool is_free = j < end && (PIECES != 0 ? !(bits >> (j0 / kRankThreads) & 1) : a.refs[j] <= 0);
        int total;
        const int rank = block_before<kRankThreads>(is_free, s, &total);
        if (is_free)
            plan.free_ids[free_before + rank] = j;
        free_before += total;
    }
    if (end == a.pages && begin < end && tid == 0)
        plan.count[0] = free_before;
}

__global__ __launch_bounds__(kBookThreads) void pages_reserve_kernel(PoolArgs p, BookArgs a, const int32_t *__restrict__ new_lengths, ReservePlan plan,
                                                                     int32_t *__restrict__ missing)
{
    const int slot = blockIdx.x, part = blockIdx.y, tid = threadIdx.x;
    const int need = plan.need[slot], shared = plan.shared[slot];
    const int wanted = new_lengths[slot];
    const int length = part > 0 || a.lengths[slot] < 0 ? 0 : a.lengths[slot];        // (the first part's workgroup alone writes it)
    const bool report = slot == 0 && part == 0;
    if (!report && (part > 0 ? shared < 0 : need == 0 && wanted <= 0))
        return;
    // pages needed ahead of this sequence, and by all; how far rows are short
    long long before = plan.before[slot], all, over;
    const int groups = (a.S + kRankThreads - 1) / kRankThreads;          // (at most 64: a lane each)
    if (groups == 1) {
        all = plan.sums[0];
        over = plan.sums[1];
    } else {
        const int lane = tid & (kWave - 1);
        all = lane < groups ? plan.sums[2 * lane] : 0;
        over = lane < groups ? plan.sums[2 * lane + 1] : 0;
        long long ahead = lane < slot / kRankThreads ? all : 0;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            ahead += __shfl_xor(ahead, d);
            all += __shfl_xor(all, d);
            over += __shfl_xor(over, d);
        }
        before += ahead;
    }
    const int free_pages = plan.count[0];
    const long long short_of = (all > free_pages ? all - free_pages : 0) + over;
    if (report && tid == 0)
        missing[0] = short_of > 0x7fffffff ? 0x7fffffff : (int)short_of;
    if (short_of || (part > 0 && shared < 0))
        return;
    if (shared >= 0)
        copy_page_part(p, shared, plan.free_ids[before], part);
    if (part > 0 || wanted <= length)
        return;
    __syncthreads();                       // every thread has read the length
    int32_t *row = a.table + slot * a.stride;
    const int page = 1 << a.page_log2;
    const int first = shared >= 0 ? length >> a.page_log2 : (length + page - 1) >> a.page_log2;
    for (int k = tid; k < need; k += kBookThreads) {
        const int id = plan.free_ids[before + k];
        row[first + k] = id;
        a.refs[id] = 1;
    }
    if (tid == 0) {
        a.lengths[slot] = wanted;
        if (shared >= 0) {
            atomicSub(a.refs + shared, 1);
            if (plan.copies) {
                plan.copies[slot] = shared;
                plan.copies[a.S + slot] = plan.free_ids[before];
            }
        }
    }
}

// ---- compact ----------------------------------------------------------------------------------------------------
// Two launches.  The first ranks: with n pages in use, free page i < n is hole number i - live(i), page i >= n in use is mover number
// live(i) - live(n), live(i) = pages in use below i; mover k goes to hole k.  The second moves the pages (a set of workgroups that
// take moves in turn: how many there are is known on the device alone) and rewrites the books.
struct CompactPlan {
    int32_t *holes, *movers, *rank;   // [pages] each; rank[i] for movers
    int32_t *count;                   // [0]: moves, [1]: pages in use
};

template <int PIECES>
__global__ __launch_bounds__(kRankThreads) void pages_compact_rank_kernel(const int32_t *__restrict__ refs, int pages, CompactPlan plan, int segment,
                                                                          int32_t *__restrict__ live)
{
    __shared__ __align__(8) int s[2 * kRankThreads / kWave];
    const int tid = threadIdx.x;
    const int begin = blockIdx.x * segment, end = begin + segment < pages ? begin + segment : pages;
    uint64_t bits = 0;
    int n, below, before;
    if constexpr (PIECES != 0) {
        bits = pages_in_use<PIECES>(refs, pages);
        const int2 sums = block_sums<kRankThreads>(__popcll(bits), in_use_below(bits, begin), s);
        n = sums.x;
        before = sums.y;
        below = block_sum<kRankThreads>(in_use_below(bits, n), s);
    } else {
        const int2 sums = block_sums<kRankThreads>(in_use_below(refs, pages), in_use_below(refs, begin), s);
        n = sums.x;
        before = sums.y;
        below = block_sum<kRankThreads>(in_use_below(refs, n), s);
    }
    if (blockIdx.x == 0 && tid == 0) {
        plan.count[0] = n - below;
        plan.count[1] = n;
        live[0] = n;
    }
    for (int j0 = begin; j0 < end; j0 += kRankThreads) {
        const int j = j0 + tid;
        const bool used = j < end && (PIECES != 0 ? bits >> (j0 / kRankThreads) & 1 : refs[j] > 0);
        int total;
        const int at = before + block_before<kRankThreads>(used, s, &total);
        before += total;
        if (j < end) {
            if (j < n && !used)
                plan.holes[j - at] = j;
            if (j >= n && used) {
                plan.movers[at - below] = j;
                plan.rank[j] = at - below;
            }
        }
    }
}

__global__ __launch_bounds__(kCopyThreads) void pages_compact_kernel(PoolArgs p, BookArgs a, CompactPlan plan, int32_t *__restrict__ table_out,
                                                                     int64_t out_stride, int32_t *__restrict__ refs_out, uint32_t parts, int move_groups)
{
    const int moves = plan.count[0], n = plan.count[1];
    if ((int)blockIdx.x < move_groups) {
        const int64_t all = (int64_t)moves * parts;
        for (int64_t k = blockIdx.x; k < all; k += move_groups) {
            const int move = (int)(k / parts);
            copy_page_part(p, plan.movers[move], plan.holes[move], (uint32_t)(k % parts));
        }
        return;
    }
    const int64_t entries = (int64_t)a.S * a.W, step = (int64_t)(gridDim.x - move_groups) * kCopyThreads;
    for (int64_t k = (int64_t)(blockIdx.x - move_groups) * kCopyThreads + threadIdx.x; k < entries + a.pages; k += step) {
        if (k < entries) {
            const int slot = (int)(k / a.W), w = (int)(k % a.W);
            int id = -1;
            if (w < pages_of(a.lengths[slot], a)) {
                id = a.table[slot * a.stride + w];
                // (an id that no count stands behind has no new place)
                if ((uint32_t)id >= (uint32_t)a.pages || a.refs[id] <= 0)
                    id = -1;
                else if (id >= n)
                    id = plan.holes[plan.rank[id]];
            }
            table_out[slot * out_stride + w] = id;
        } else {
            // a place below n keeps its count or gets that of the page that moves there; the rank of a hole among the holes is found
            // from the side of the mover, so movers write for both
            const int i = (int)(k - entries);
            const int r = a.refs[i];
            if (i < n) {
                if (r > 0)
                    refs_out[i] = r;
            } else {
                refs_out[i] = 0;
                if (r > 0)
                    refs_out[plan.holes[plan.rank[i]]] = r;
            }
        }
    }
}

static int segments_of(int pages, int *segment)
{
    // a multiple of the workgroup, at most kSegments of them
    int64_t each = ((int64_t)pages + kSegments - 1) / kSegments;
    each = (each + kRankThreads - 1) / kRankThreads * kRankThreads;
    *segment = (int)each;
    return (int)((pages + each - 1) / each);
}

static BookArgs book_args(const lookat_page_pool *pool, int32_t S, const int32_t *table, int32_t W, int64_t stride, const int32_t *lengths,
                          const int32_t *refs)
{
    BookArgs a;
    a.table = const_cast<int32_t *>(table);
    a.stride = stride;
    a.lengths = const_cast<int32_t *>(lengths);
    a.refs = const_cast<int32_t *>(refs);
    a.S = S;
    a.W = W;
    a.pages = pool->pages;
    a.page_log2 = __builtin_ctz((unsigned)pool->page);
    return a;
}

static int check_books(const lookat_page_pool *pool, int32_t S, const int32_t *table, int32_t W, int64_t stride, const int32_t *lengths,
                       const int32_t *refs)
{
    if (int rc = check_pool(pool))
        return rc;
    if (int rc = check_table(pool, "S", S, table, W, stride))
        return rc;
    if (!lengths || !refs)
        return fail(LOOKAT_ERR_NULL, "lengths and refs must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(lengths) | reinterpret_cast<uintptr_t>(refs)) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "lengths and refs must be 4-byte aligned");
    return LOOKAT_OK;
}

static int check_workspace(size_t need, const void *workspace, size_t bytes)
{
    if (!workspace || bytes < need)
        return fail(LOOKAT_ERR_WORKSPACE, "workspace of %zu bytes needed, got %zu", need, workspace ? bytes : (size_t)0);
    if (!aligned16(workspace))
        return fail(LOOKAT_ERR_ALIGN, "workspace must be 16-byte aligned");
    return LOOKAT_OK;
}

static int check_list(int32_t n, const void *x, const void *y)
{
    if (n < 0)
        return fail(LOOKAT_ERR_SHAPE, "n=%d must not be negative", n);
    if (n > 0 && (!x || !y))
        return fail(LOOKAT_ERR_NULL, "the lists of pages or slots must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "the lists of pages or slots must be 4-byte aligned");
    return LOOKAT_OK;
}

}  // namespace lookat

extern "C" int lookat_pages_copy(const lookat_page_pool *pool, int32_t n, const int32_t *src, const int32_t *dst, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_pool(pool))
        return rc;
    if (int rc = check_list(n, src, dst))
        return rc;
    if (n == 0)
        return LOOKAT_OK;
    const PoolArgs p = pool_args(pool);
    const int64_t groups = (int64_t)n * page_parts(p);
    if (!fits_launch(groups, kCopyThreads))
        return fail(LOOKAT_ERR_UNSUPPORTED, "n=%d pages of %u parts exceed one launch", n, page_parts(p));
    hipLaunchKernelGGL(pages_copy_kernel, dim3((unsigned)groups), dim3(kCopyThreads), 0, static_cast<hipStream_t>(stream), p, src, dst, n,
                       page_parts(p));
    return check_launch("lookat_pages_copy");
}

extern "C" int lookat_pages_fork(const lookat_page_pool *pool, int32_t S, int32_t *table, int32_t W, int64_t table_stride, int32_t *lengths,
                                 int32_t *refs, int32_t n, const int32_t *src, const int32_t *dst, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_books(pool, S, table, W, table_stride, lengths, refs))
        return rc;
    if (int rc = check_list(n, src, dst))
        return rc;
    if (n == 0)
        return LOOKAT_OK;
    if (n > kMostListed)
        return fail(LOOKAT_ERR_UNSUPPORTED, "n=%d: one launch takes at most %d slots", n, kMostListed);
    hipLaunchKernelGGL(pages_fork_kernel, dim3((unsigned)n), dim3(kBookThreads), 0, static_cast<hipStream_t>(stream),
                       book_args(pool, S, table, W, table_stride, lengths, refs), n, src, dst);
    return check_launch("lookat_pages_fork");
}

extern "C" int lookat_pages_free(const lookat_page_pool *pool, int32_t S, int32_t *table, int32_t W, int64_t table_stride, int32_t *lengths,
                                 int32_t *refs, int32_t n, const int32_t *slots, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_books(pool, S, table, W, table_stride, lengths, refs))
        return rc;
    if (int rc = check_list(n, slots, slots))
        return rc;
    if (n == 0)
        return LOOKAT_OK;
    if (n > kMostListed)
        return fail(LOOKAT_ERR_UNSUPPORTED, "n=%d: one launch takes at most %d slots", n, kMostListed);
    hipLaunchKernelGGL(pages_free_kernel, dim3((unsigned)n), dim3(kBookThreads), 0, static_cast<hipStream_t>(stream),
                       book_args(pool, S, table, W, table_stride, lengths, refs), slots);
    return check_launch("lookat_pages_free");
}

extern "C" size_t lookat_pages_reserve_workspace_bytes(const lookat_page_pool *pool, int32_t S)
{
    using namespace lookat;
    clear_error();
    if (check_pool(pool) != LOOKAT_OK || S <= 0)
        return 0;
    // (count, sums, need, shared, before, free_ids)
    return ((size_t)pool->pages + 3 * (size_t)S + 4) * sizeof(int32_t) + ((size_t)S + kRankThreads - 1) / kRankThreads * 2 * sizeof(long long);
}

extern "C" int lookat_pages_reserve(const lookat_page_pool *pool, int32_t S, int32_t *table, int32_t W, int64_t table_stride, int32_t *lengths,
                                    int32_t *refs, const int32_t *new_lengths, int32_t *missing, int32_t *copies, void *workspace,
                                    size_t workspace_bytes, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_books(pool, S, table, W, table_stride, lengths, refs))
        return rc;
    if (!new_lengths || !missing)
        return fail(LOOKAT_ERR_NULL, "new_lengths and missing must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(new_lengths) | reinterpret_cast<uintptr_t>(missing) | reinterpret_cast<uintptr_t>(copies)) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "new_lengths, missing and copies must be 4-byte aligned");
    if (new_lengths < lengths + S && lengths < new_lengths + S)
        return fail(LOOKAT_ERR_SHAPE, "new_lengths and lengths must not overlap");
    if (int rc = check_workspace(lookat_pages_reserve_workspace_bytes(pool, S), workspace, workspace_bytes))
        return rc;
    const PoolArgs p = pool_args(pool);
    const BookArgs a = book_args(pool, S, table, W, table_stride, lengths, refs);
    ReservePlan plan;
    plan.count = static_cast<int32_t *>(workspace);
    const int groups = (S + kRankThreads - 1) / kRankThreads;
    plan.sums = reinterpret_cast<long long *>(plan.count + 4);
    plan.need = reinterpret_cast<int32_t *>(plan.sums + 2 * groups);
    plan.shared = plan.need + S;
    plan.before = plan.shared + S;
    plan.free_ids = plan.before + S;
    plan.copies = copies;
    int segment;
    const int segments = segments_of(p.pages, &segment);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int pieces = (p.pages + kRankThreads - 1) / kRankThreads;
    const auto rank = pieces <= 1 ? &pages_reserve_rank_kernel<1> : pieces <= 4 ? &pages_reserve_rank_kernel<4> : pieces <= 16 ? &pages_reserve_rank_kernel<16>
                    : pieces <= 64 ? &pages_reserve_rank_kernel<64> : &pages_reserve_rank_kernel<0>;
    hipLaunchKernelGGL(rank, dim3((unsigned)(segments + groups)), dim3(kRankThreads), 0, st, a, new_lengths, plan,
                       segments, segment);
    if (int rc = check_launch("lookat_pages_reserve (ranks)"))
        return rc;
    hipLaunchKernelGGL(pages_reserve_kernel, dim3((unsigned)S, page_parts(p)), dim3(kBookThreads), 0, st, p, a, new_lengths, plan, missing);
    return check_launch("lookat_pages_reserve");
}

extern "C" size_t lookat_pages_compact_workspace_bytes(const lookat_page_pool *pool)
{
    using namespace lookat;
    clear_error();
    if (check_pool(pool) != LOOKAT_OK)
        return 0;
    return (3 * (size_t)pool->pages + 4) * sizeof(int32_t);
}

extern "C" int lookat_pages_compact(const lookat_page_pool *pool, int32_t S, const int32_t *table, int32_t W, int64_t table_stride,
                                    const int32_t *lengths, const int32_t *refs, int32_t *table_out, int64_t table_out_stride,
                                    int32_t *refs_out, int32_t *live, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace lookat;
    clear_error();
    if (int rc = check_books(pool, S, table, W, table_stride, lengths, refs))
        return rc;
    if (!table_out || !refs_out || !live)
        return fail(LOOKAT_ERR_NULL, "table_out, refs_out and live must be non-NULL");
    if (table_out_stride < W)
        return fail(LOOKAT_ERR_SHAPE, "table_out_stride=%lld smaller than a row of %d", (long long)table_out_stride, W);
    if ((reinterpret_cast<uintptr_t>(table_out) | reinterpret_cast<uintptr_t>(refs_out) | reinterpret_cast<uintptr_t>(live)) & 3u)
        return fail(LOOKAT_ERR_ALIGN, "table_out, refs_out and live must be 4-byte aligned");
    const uintptr_t t0 = reinterpret_cast<uintptr_t>(table), t1 = t0 + ((size_t)(S - 1) * table_stride + W) * 4;
    const uintptr_t u0 = reinterpret_cast<uintptr_t>(table_out), u1 = u0 + ((size_t)(S - 1) * table_out_stride + W) * 4;
    const uintptr_t r0 = reinterpret_cast<uintptr_t>(refs), r1 = r0 + (size_t)pool->pages * 4;
    const uintptr_t q0 = reinterpret_cast<uintptr_t>(refs_out), q1 = q0 + (size_t)pool->pages * 4;
    if ((t0 < u1 && u0 < t1) || (r0 < q1 && q0 < r1))
        return fail(LOOKAT_ERR_SHAPE, "table_out and refs_out must not overlap table and refs");
    if (int rc = check_workspace(lookat_pages_compact_workspace_bytes(pool), workspace, workspace_bytes))
        return rc;
    const PoolArgs p = pool_args(pool);
    const BookArgs a = book_args(pool, S, table, W, table_stride, lengths, refs);
    CompactPlan plan;
    plan.count = static_cast<int32_t *>(workspace);
    plan.holes = plan.count + 4;
    plan.movers = plan.holes + p.pages;
    plan.rank = plan.movers + p.pages;
    int segment;
    const int segments = segments_of(p.pages, &segment);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int pieces = (p.pages + kRankThreads - 1) / kRankThreads;
    const auto rank = pieces <= 1 ? &pages_compact_rank_kernel<1> : pieces <= 4 ? &pages_compact_rank_kernel<4> : pieces <= 16 ? &pages_compact_rank_kernel<16>
                    : pieces <= 64 ? &pages_compact_rank_kernel<64> : &pages_compact_rank_kernel<0>;
    hipLaunchKernelGGL(rank, dim3((unsigned)segments), dim3(kRankThreads), 0, st, refs, p.pages, plan, segment, live);
    if (int rc = check_launch("lookat_pages_compact (ranks)"))
        return rc;
    const int64_t most = ((int64_t)p.pages / 2 + 1) * page_parts(p);     // at most half of the pages move
    const int move_groups = (int)(most < 16384 ? most : 16384);
    const int64_t book = ((int64_t)S * W + p.pages + kCopyThreads - 1) / kCopyThreads;
    hipLaunchKernelGGL(pages_compact_kernel, dim3((unsigned)(move_groups + (book < 1024 ? book : 1024))), dim3(kCopyThreads), 0, st, p, a, plan,
                       table_out, table_out_stride, refs_out, page_parts(p), move_groups);
    return check_launch("lookat_pages_compact");
}
