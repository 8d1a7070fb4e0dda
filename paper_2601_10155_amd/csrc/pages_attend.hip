// Attention decode over the paged cache: product-quantised keys, 8-bit values with a power-of-two scale per page and head.
//
//   s_l = sum_i lut_i[code_l,i],   out = sum_l softmax_l(scale s) q_l 2^e(l)
//
// computed in one pass with the page's exponent added to the logit: y_l = scale log2(e) s_l + e(l), R a running reference near max y,
//   w_l = 2^(y_l - R),   out = sum_l w_l q_l / sum_l w_l 2^-e(l).
// So the stored integers enter the product as they are (exact in fp16), the weights are as precise as the largest contribution to the result
// needs whatever the pages' exponents are, and no per-page rescaling is done.
//
// Bound: the stream of codes and values from HBM, m + d_k bytes per token and key/value head, where there is much of it: 8 x 32 x 32768
// tokens (d_k = 128, m = 8, int8; 1.14 GB, fetched once) take 165 us in the kernel, 6.9 TB/s (a plain read of 1 GiB: 7.0 to 7.1), 169 a call.
// Below some 50 MB the chain of dependent steps counts instead: lengths, page id, codes and values, reduction, merge.  12 x 1024 tokens
// (0.8 MB) 5.2 us in the kernel: 0.4 until the range is known, 0.3 until the first tile is requested, 1.5 until it is weighted, 1.2 for the
// results.  12 x 8 x up to 8191 in groups of 8 (52 MB) 16.9 us and 3.8 for the merge: 224 ranges, one of eight wavefronts to a compute unit, whose
// wavefronts take four tiles one after the other and wait for them during 61% of their cycles; vector issue (270 instructions a tile) is 5 us of it.
//
// Weighted sums on the matrix cores at every group, also for one query head: 1 + 1/2 vector instructions a stored value (int8; 1/2 in e4m3)
// instead of 2.  What was tried and not kept: four or sixteen wavefronts to a workgroup (long contexts 178.9 / 179.8 us, eight 177.4, groups of 8
// 30.6 / 41.0, eight 27.7, at an earlier stage), a second tile in registers at d_k = 64 (16 x 12 x 4096 14.8 -> 17.1 us: fewer wavefronts fit),
// ranges of whole steps of eight tiles (no change), a product with integer weights (the tables' scores need 22 bits), tables loaded straight into
// LDS (a lane names one word where heads are interleaved: groups of 8 20.1 / 22.2, of 4 17.5 / 18.8, one head 15.9 / 16.6 us).  Neither side of the
// tables' LDS traffic counts: without bank conflicts in the stores 20.2, in the look-ups 19.7 instead of 20.1.
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
typedef float v2f __attribute__((ext_vector_type(2)));

struct AttendArgs {
    const float *lut;
    const int32_t *table, *lengths;
    float *part, *out;
    int2 *plan;                           // ranges by length: (first range, ranges) of every sequence, for the merge
    int64_t table_stride;
    int32_t W, B, units;                  // units = sequences * key/value heads
    int32_t splits, chunk;                // equal ranges: their number and their tokens (a multiple of 64)
    int32_t per_head;                     // ranges by length: how many there should be for each key/value head; 0: equal ranges
    int32_t least;                        // ... of at least this many tokens
    float scale_log2e;
};

constexpr float kRefLag = 8.f;            // the reference moves when a logit exceeds it by more (log2 units)
constexpr float kNoReference = -3.402823466e38f;   // before the first token: fp32's lowest, so no logit is below it, and finite: -inf less it is -inf
constexpr float kRefLift = 7.f;           // weights are 2^7 at the reference, below 2^15: fp16's range, its subnormals far below
// Wavefronts of a workgroup: eight of 128 registers, two workgroups to a compute unit.  Four where no sequence is longer than four tiles: the
// others would only take room from the next workgroups (us, eight / four: 42 x 32 x 157 tokens in groups of 2 15.0 / 10.7, 64 x 32 x 250
// 14.1 / 11.2, 27 x 32 x 2 in groups of 4 12.3 / 9.9, a few heads the same), unless there are 64 KB of tables to fetch (32 x 8 x 200 in
// groups of 8, m = 8: 9.2 / 10.9).
constexpr int kAttendWaves = 8, kShortWaves = 4;
__host__ __device__ constexpr bool few_waves(int G, int m, int64_t longest) { return G * m < 64 && longest <= kShortWaves * kTile; }
// Wavefronts to a SIMD that the registers have to allow.  Six (80 registers) at d_k = 64 for one or two query heads, whose instances fit, but for
// two heads at m = 8: those spill 2 to 6 registers and gain all the same.  us, four / six: groups of 2 x 32 x 6 x 4096, m = 8 int8 18.1 / 17.0,
// e4m3 18.1 / 16.6, 16 x 12 x 4096, m = 16 e4m3 18.9 / 17.0, m = 4 14.9 / 14.9.  Not two heads at m = 16, which would spill up to 8 (x 32 x 6 x 4096
// 21.9 / 22.2, x 8 x 6 x 32768 34.4 / 35.6, x 32 x 6 x 700 7.3 / 7.8), nor four heads (16 x 4 x 8192 13.4 / 13.8).
// Two where 128 KB of tables leave room for one workgroup only: the other registers hold look-ups in flight (8 x 4 x 65536 84.5 / 81.6).
// (At four, 128 registers, two heads at d_k = 128, m = 16 spill 3 or 4; with more registers one workgroup would have the compute unit to itself.)
__host__ __device__ constexpr int min_waves(int d_k, int m, int G) { return G * m >= 128 ? 2 : d_k == 64 && G <= 2 && G * m <= 16 ? 6 : 4; }
// Tables of 32 KB and more: every range fetches them, so there are as many ranges as the chip holds at once and no second round (see cut_of).
__host__ __device__ constexpr bool one_round(int m, int G) { return G * m >= 32; }
constexpr int kMostPlanned = 1024;        // sequences whose ranges are cut by their lengths

// Ranges by length.  Sequences of unequal length cut into equally many ranges leave most of the chip waiting for the longest one, and the host
// does not know the lengths.  So every workgroup looks at all of them: with c tokens per range, c such that all sequences
// together make about `per_head` ranges for each head, sequence b gets ceil(length_b / c) ranges of nearly equal size, and the ranges of all
// (sequence, head) pairs are dealt to the workgroups in order.  At most per_head + 1 + B per head: a workgroup that has none leaves.
struct Range {
    int b, h, split, splits, k0, k1, index;
};
__device__ __forceinline__ int range_tokens(float total, int per_head, int least)
{
    // (rounded the same in every workgroup; 2^-20 of a range more or less is what the extra range per head is for)
    const float want = total / (float)per_head;
    return want < (float)least ? least : want > 1073741824.f ? 1 << 30 : ((int)want + kTile) / kTile * kTile;
}
// a / b rounded down, for a quotient below 2^20
__device__ __forceinline__ int quotient(int a, int b)
{
    int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b));      // off by one at most
    q -= q * b > a;
    q += a - q * b >= b;
    return q;
}
__device__ __forceinline__ int ranges_of(int length, int c) { return length > c ? quotient(length - 1, c) + 1 : 1; }
__device__ __forceinline__ void set_range(Range &r, int b, int place, int splits, int length, int c, int index)
{
    r.b = b;
    r.splits = splits;
    r.h = quotient(place, splits);
    r.split = place - r.h * splits;
    r.index = index;
    // no less than length / splits (2^-20 more than its product with the reciprocal), and at most c: no range is empty
    int size = ((int)((float)length * __builtin_amdgcn_rcpf((float)splits) * 1.000001f) + kTile) / kTile * kTile;
    size = size < c ? size : c;
    r.k0 = r.split * size;
    r.k1 = r.split == splits - 1 ? length : r.k0 + size;
}
// Sum over the lanes up to this one.
__device__ __forceinline__ int upto_lane(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);       // row_shr:1, 2, 4, 8: within 16 lanes
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast:15 into rows 1 and 3
    return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);    // row_bcast:31 into rows 2 and 3
}
// (all threads of the workgroup; s: 36 ints of LDS; B <= kMostPlanned; false: no range)
template <bool ONE_ROUND>
__device__ __forceinline__ bool range_by_length(const AttendArgs &a, int H, int page_log2, int *s, Range &r)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, waves = blockDim.x / kWave;
    const int die = blockIdx.x % kXcds, nth = blockIdx.x / kXcds;
    if (a.B <= kWave) {
        // a lane per sequence, every wavefront for itself
        const int length = lane < a.B ? clamp_length(a.lengths[lane], a.W, page_log2) : 0;
        const float total = wave_sum((float)length);
        int c = range_tokens(total, a.per_head, a.least);
        int n = lane < a.B ? ranges_of(length, c) : 0;
        int upto = upto_lane(n);
        const int extra = ONE_ROUND ? __builtin_amdgcn_readlane(upto, kWave - 1) - a.per_head : 0;
        if (extra > 0 && 2 * extra < a.per_head) {
            // (longer ones instead of as many more as the sequences' last ranges made: a few too many wait for a round of their own)
            c = range_tokens(total, a.per_head - extra, a.least);
            n = lane < a.B ? ranges_of(length, c) : 0;
            upto = upto_lane(n);
        }
        const int ranges = __builtin_amdgcn_readlane(upto, kWave - 1) * H, per_die = (ranges + kXcds - 1) / kXcds, index = die * per_die + nth;
        if (nth >= per_die || index >= ranges)
            return false;
        if (index == 0 && wave == 0 && lane < a.B)
            a.plan[lane] = make_int2((upto - n) * H, n);
        const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(index < upto * H));
        set_range(r, at, index - __builtin_amdgcn_readlane(upto - n, at) * H, __builtin_amdgcn_readlane(n, at), __builtin_amdgcn_readlane(length, at), c, index);
        return true;
    }
    const int each = (a.B + (int)blockDim.x - 1) / (int)blockDim.x;       // consecutive sequences of a thread: 1 to 16
    const int b0 = tid * each;
    float total = 0.f;
    for (int j = 0; j < each; ++j)
        if (b0 + j < a.B)
            total += (float)clamp_length(a.lengths[b0 + j], a.W, page_log2);
    total = wave_sum(total);
    float *f = reinterpret_cast<float *>(s);
    if (lane == 0)
        f[wave] = total;
    __syncthreads();
    total = 0.f;
    for (int w = 0; w < waves; ++w)
        total += f[w];
    const int c = range_tokens(total, a.per_head, a.least);
    int n = 0;
    for (int j = 0; j < each; ++j)
        if (b0 + j < a.B) {
            const int length = clamp_length(a.lengths[b0 + j], a.W, page_log2);
            n += ranges_of(length, c);
        }
    int before = upto_lane(n);
    if (lane == kWave - 1)
        s[16 + wave] = before;
    before -= n;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < waves; ++w) {
        before += w < wave ? s[16 + w] : 0;
        all += s[16 + w];
    }
    // consecutive ranges on one die: those of a (sequence, head) share its tables
    const int ranges = all * H, per_die = (ranges + kXcds - 1) / kXcds;
    const int index = die * per_die + nth;
    if (nth >= per_die || index >= ranges)
        return false;
    for (int j = 0; j < each; ++j)
        if (b0 + j < a.B) {
            const int length = clamp_length(a.lengths[b0 + j], a.W, page_log2);
            const int mine = ranges_of(length, c);
            if (index == 0)
                a.plan[b0 + j] = make_int2(before * H, mine);
            if (index >= before * H && index < (before + mine) * H) {
                s[32] = b0 + j;
                s[33] = index - before * H;
                s[34] = mine;
                s[35] = length;
            }
            before += mine;
        }
    __syncthreads();
    const int at = s[32], place = s[33], mine = s[34], length = s[35];
    __syncthreads();                                      // (s is free again)
    set_range(r, at, place, mine, length, c, index);
    return true;
}

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

template <int CTRL>
__device__ __forceinline__ float lane_of(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_value(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }
// Maxima or sums over the wavefront of G values at once, as scalars: every exchange serves two values, so that eight take 28 instructions.
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
template <typename Op>
__device__ __forceinline__ float over_row(float x, Op op)          // 16 lanes
{
    x = op(x, lane_of<0xB1>(x));
    x = op(x, lane_of<0x4E>(x));
    x = op(x, lane_of<0x141>(x));
    return op(x, lane_of<0x140>(x));
}
// Lanes 0-31: over x's halves, 32-63: over y's.
template <typename Op>
__device__ __forceinline__ float over_halves(float x, float y, Op op)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Rows 0 and 2: over x's rows 0, 1 and 2, 3; rows 1 and 3: over y's.
template <typename Op>
__device__ __forceinline__ float over_rows(float x, float y, Op op)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int G, typename Op>
__device__ __forceinline__ void over_wave(const float (&y)[G], float (&m)[G], Op op)
{
    if constexpr (G == 1) {
        const float h = over_halves(y[0], y[0], op);
        m[0] = lane_value(over_row(over_rows(h, h, op), op), 0);
    } else if constexpr (G == 2) {
        const float h = over_halves(y[0], y[1], op), a = over_row(over_rows(h, h, op), op);
        m[0] = lane_value(a, 0);
        m[1] = lane_value(a, 32);
    } else if constexpr (G == 4) {
        const float a = over_row(over_rows(over_halves(y[0], y[2], op), over_halves(y[1], y[3], op), op), op);
#pragma unroll
        for (int g = 0; g < 4; ++g)
            m[g] = lane_value(a, 16 * g);
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float a = over_row(over_rows(over_halves(y[k], y[k + 4], op), over_halves(y[k + 2], y[k + 6], op), op), op);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                m[k + 2 * r] = lane_value(a, 16 * r);
        }
    }
}

// LDS of a workgroup: tables (afterwards the wavefronts' results), then the wavefronts' staged weights (afterwards their references and sums).
__host__ __device__ constexpr size_t attend_front_bytes(int G, int M, int d_k, int waves)
{
    const size_t tables = (size_t)G * M * kCentroids * 4, results = (size_t)waves * G * (d_k + 2) * 4;
    return tables > results ? tables : results;
}
__host__ __device__ constexpr size_t attend_lds_bytes(int G, int M, int d_k, int waves)
{
    return attend_front_bytes(G, M, d_k, waves) + (size_t)waves * 2 * G * kTile * 2;
}

template <int DK, int M, int G, bool FP8, int WAVES>
__global__ __launch_bounds__(WAVES *kWave, min_waves(DK, M, G)) void attend_pages_kernel(PoolArgs p, AttendArgs a)
{
    constexpr int threads = WAVES * kWave;
    constexpr size_t front = attend_front_bytes(G, M, DK, WAVES);
    extern __shared__ __align__(16) char lds[];
    constexpr int GP = G < 4 ? G : 4;                     // query heads whose tables are interleaved
    typedef float vg __attribute__((ext_vector_type(GP)));
    constexpr int CB = DK / 32;                           // 16-byte loads per lane and 32 tokens
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    Range r;
    if (a.per_head) {
        if (!range_by_length<one_round(M, G)>(a, p.H, p.page_log2, reinterpret_cast<int *>(lds), r))
            return;
    } else {
        // ranges of one (sequence, head) on one die: its tables are fetched into one L2
        const int unit = (int)(blockIdx.x / kXcds) / a.splits * kXcds + blockIdx.x % kXcds;
        if (unit >= a.units)
            return;
        r.b = unit / p.H;
        r.h = unit - r.b * p.H;
        r.split = (int)(blockIdx.x / kXcds) % a.splits;
        r.splits = a.splits;
        r.index = unit * a.splits + r.split;
        const int length = clamp_length(a.lengths[r.b], a.W, p.page_log2);
        r.k0 = r.split * a.chunk;
        r.k1 = r.split == a.splits - 1 || length - r.k0 < a.chunk ? length : r.k0 + a.chunk;
        if (r.k0 >= r.k1 && r.split > 0)
            return;                                       // (the merge knows the length)
    }
    const int b = r.b, h = r.h, k0 = r.k0, k1 = r.k1, unit = b * p.H + h;
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
        }
    };

    int t = k0 + wave * kWave;
    const int step = threads;
    int id = page_of(t + lane);
    float *tables = reinterpret_cast<float *>(lds);
    // Tables [query head][i][c] -> [plane of GP heads][i][c][head], scaled; a thread takes four entries of GP heads at a time.  The first tile is
    // requested between the tables' loads and their use.
    constexpr int quads = G / GP * M * (kCentroids / 4), rounds = (quads + threads - 1) / threads;
    constexpr int early = rounds * GP <= 8 ? rounds : 8 / GP;         // (rounds is a multiple of it: both are powers of two)
    const v4f *lut = reinterpret_cast<const v4f *>(a.lut + (int64_t)unit * G * M * kCentroids);
    v4f x[early][GP];
    auto table_load = [&](int round, int n) {
        const int j = tid + round * threads, at = quads % threads && j >= quads ? quads - 1 : j;
        const int plane = at / (M * (kCentroids / 4)), entry = at % (M * (kCentroids / 4));
#pragma unroll
        for (int g = 0; g < GP; ++g)
            x[n][g] = lut[(plane * GP + g) * (M * (kCentroids / 4)) + entry];
    };
    auto table_store = [&](int round, int n) {
        const int j = tid + round * threads;
        if (quads % threads == 0 || j < quads) {
#pragma unroll
            for (int k = 0; k < GP; ++k) {                // GP * 4 floats as GP 16-byte stores, ordered entry, head
                v4f y;
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    y[w] = x[n][(4 * k + w) % GP][(4 * k + w) / GP] * a.scale_log2e;
                reinterpret_cast<v4f *>(tables)[j * GP + k] = y;
            }
        }
    };
#pragma unroll
    for (int n = 0; n < early; ++n)
        table_load(n, n);
    __builtin_amdgcn_sched_barrier(0);
    if (t < k1)
        request(t, id);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < early; ++n)
        table_store(n, n);
#pragma unroll
    for (int r0 = early; r0 < rounds; r0 += early) {
#pragma unroll
        for (int n = 0; n < early; ++n)
            if (r0 + n < rounds)
                table_load(r0 + n, n);
#pragma unroll
        for (int n = 0; n < early; ++n)
            if (r0 + n < rounds)
                table_store(r0 + n, n);
    }
    int id_next = page_of(t + step + lane);
    __syncthreads();

    // staged weights: a row of 64 tokens per column, 128 bytes; its 16-byte pieces are permuted (xor with the row) so that neither side conflicts
    constexpr int staged = 2 * G * kTile * 2;
    char *weights = lds + front + wave * staged;
    int w_at = (lane >> 3) << 4 | (lane & 7) << 1;
    auto weight = [&](int row) -> _Float16 & { return *reinterpret_cast<_Float16 *>(weights + row * (kTile * 2) + (w_at ^ ((row & 7) << 4))); };
    v4f acc[2 * CB];
#pragma unroll
    for (int c = 0; c < 2 * CB; ++c)
        acc[c] = (v4f){0.f, 0.f, 0.f, 0.f};
    float lift[G], z[G];                                  // the reference less kRefLift (one value for the wavefront), the sum
#pragma unroll
    for (int g = 0; g < G; ++g) {
        lift[g] = kNoReference;
        z[g] = 0.f;
    }

    while (t < k1) {
        // logits, above the reference
        float y[G];
        exponent = id < 0 ? 0 : exponent;                 // (a lane without a token has read some page's)
#pragma unroll
        for (int g = 0; g < G; ++g)
            y[g] = (float)exponent;
        // (LDS reads in flight at once: 16 registers of them, 8 where the others take what is left: groups of 8 x 8191 tokens 20.4 / 19.7 us; 32
        // where one workgroup has the compute unit: 8 / 16 / 32 / 64 84.2 / 81.9 / 81.5 / 81.5 us for 128 KB of tables x 4 heads x 8 x 65536)
        constexpr int planes = G / GP, most_reads = (G * M >= 128 ? 32 : DK == 128 && (G == 8 || M == 16) ? 8 : 16) / GP;
        constexpr int together = M * planes < most_reads ? M * planes : most_reads;
#pragma unroll
        for (int n0 = 0; n0 < M * planes; n0 += together) {
            vg x[together];
#pragma unroll
            for (int n = 0; n < together; ++n) {
                const int i = (n0 + n) / planes, plane = (n0 + n) % planes;
                x[n] = reinterpret_cast<const vg *>(tables)[(plane * M + i) * kCentroids + ((codes[i / 4] >> (8 * (i % 4))) & 0xffu)];
            }
#pragma unroll
            for (int n = 0; n < together; ++n)
#pragma unroll
                for (int g = 0; g < GP; ++g)
                    y[(n0 + n) % planes * GP + g] += x[n][g];
        }
        float most = -INFINITY;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            y[g] = id < 0 ? -INFINITY : y[g];
            most = fmaxf(most, y[g] - lift[g]);
        }
        if (__builtin_amdgcn_ballot_w64(most > kRefLift + kRefLag)) {
            float fix_n = 1.f, top[G];                    // fix_n: for the column that this lane accumulates
            over_wave(y, top, Max());
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float to = fmaxf(lift[g], top[g] - kRefLift);
                const float fix = fast_exp2(lift[g] - to);
                lift[g] = lane_value(to, 0);
                z[g] *= fix;
                fix_n = (lane & (G - 1)) == g ? fix : fix_n;
            }
#pragma unroll
            for (int c = 0; c < 2 * CB; ++c)
                acc[c] *= fix_n;
        }
        asm volatile("" : "+v"(w_at));                    // (the rows' places are computed here: kept from tile to tile they take eight registers)
        const float unscale = __uint_as_float((uint32_t)(127 - exponent) << 23);      // 2^-e
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float w = fast_exp2(y[g] - lift[g]);
            z[g] = fmaf(w, unscale, z[g]);
            const _Float16 hi = (_Float16)w;
            weight(g) = hi;
            weight(G + g) = (_Float16)(w - (float)hi);
        }
        if constexpr (FP8) {
            // bytes without a token behind them may be NaN: zeros in their place
            if (__builtin_amdgcn_ballot_w64(id < 0)) {
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const int first = kk * 32 + quad * 8;
                    const int n = __shfl(id, first) < 0 ? 0 : k1 - t - first;
                    const uint32_t lo = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
                    const uint32_t hi = n >= 8 ? ~0u : n <= 4 ? 0u : (1u << (8 * (n - 4))) - 1;
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        v[kk][cb].x &= lo, v[kk][cb].y &= hi;
                        v[kk][cb].z &= lo, v[kk][cb].w &= hi;
                    }
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const int row = col & (2 * G - 1);
            const v8h wt = *reinterpret_cast<const v8h *>(weights + row * (kTile * 2) + (((kk * 4 + quad) ^ (row & 7)) << 4));
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const v4u x = v[kk][cb];
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

    // The wavefronts' results: references and sums first, so that every wavefront brings its own to the common reference before they are added.
    float sums[G];
    over_wave(z, sums, Sum());
    if (lane == 0) {
#pragma unroll
        for (int g = 0; g < G; ++g)
            reinterpret_cast<v2f *>(weights)[g] = (v2f){lift[g], sums[g]};
    }
    __syncthreads();                                      // and every wavefront is done with the tables
    const int mine = col & (G - 1);
    v2f stat[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
        stat[w] = *reinterpret_cast<const v2f *>(lds + front + w * staged + mine * 8);
    float top = stat[0].x, sum = 0.f, own = lift[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w)
        top = fmaxf(top, stat[w].x);
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
        sum = fmaf(fast_exp2(stat[w].x - top), stat[w].y, sum);
#pragma unroll
    for (int g = 1; g < G; ++g)
        own = mine == g ? lift[g] : own;
    // one range: results are divided by the sum here; several: the merge does it
    float f = fast_exp2(own - top);
    if (r.splits == 1)
        f = sum == 0.f ? 0.f : f / sum;                   // (nothing to sum: zeros; a sum that is NaN stays one)
    float *results = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int c = 0; c < 2 * CB; c += 2)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            // columns n and n + G: the two terms of a weight; row 4 quad + k of an instruction's result is coordinate 2 (4 quad + k) of the 32
            // that a load covers, the next instruction's the coordinate behind it
            v2f both;
            both.x = (acc[c][k] + lane_of<0x120 + G>(acc[c][k])) * f;
            both.y = (acc[c + 1][k] + lane_of<0x120 + G>(acc[c + 1][k])) * f;
            if (col < G)
                *reinterpret_cast<v2f *>(results + (wave * G + col) * (DK + 2) + c * 16 + 2 * (4 * quad + k)) = both;
        }
    __syncthreads();
    float *to = r.splits == 1 ? a.out + (int64_t)unit * G * DK : a.part + (int64_t)r.index * G * (DK + 2);
    const int row_to = r.splits == 1 ? DK : DK + 2;
#pragma unroll
    for (int j = tid; j < G * DK / 2; j += threads) {
        const int g = j / (DK / 2), d = j % (DK / 2) * 2;
        v2f o = {0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            o += *reinterpret_cast<const v2f *>(results + (w * G + g) * (DK + 2) + d);
        *reinterpret_cast<v2f *>(to + g * row_to + d) = o;
    }
    if (r.splits > 1 && tid < G)                          // (lanes 0 to G - 1 of the first wavefront: mine == tid)
        *reinterpret_cast<v2f *>(to + tid * row_to + DK) = (v2f){top, sum};
}

// Merges the ranges of one (sequence, query head): a thread per coordinate, the ranges' loads issued eight at a time.
__global__ __launch_bounds__(128) void attend_pages_merge_kernel(AttendArgs a, int H, int G, int d_k, int page_log2)
{
    constexpr int GR = 8;
    const int unit = blockIdx.x, b = unit / H, h = unit - b * H;
    int n;
    int64_t first;
    if (a.per_head) {
        const int2 plan = a.plan[b];
        n = plan.y;
        first = plan.x + (int64_t)h * n;
        if (n == 1)
            return;                                       // written already
    } else {
        n = (clamp_length(a.lengths[b], a.W, page_log2) + a.chunk - 1) / a.chunk;
        n = n < 1 ? 1 : n > a.splits ? a.splits : n;
        first = (int64_t)unit * a.splits;
    }
    const int row = d_k + 2, g = blockIdx.y, d = threadIdx.x;
    const float *x = a.part + (first * G + g) * row;
    float top = kNoReference, o = 0.f, z = 0.f;
    for (int s0 = 0; s0 < n; s0 += GR) {
        float m_[GR], z_[GR], o_[GR];
#pragma unroll
        for (int k = 0; k < GR; ++k) {
            const float *y = x + (int64_t)(s0 + k < n ? s0 + k : s0) * G * row;
            m_[k] = y[d_k];
            z_[k] = y[d_k + 1];
            o_[k] = y[d];
        }
        float to = top;
#pragma unroll
        for (int k = 0; k < GR; ++k)
            to = fmaxf(to, m_[k]);
        const float fix = fast_exp2(top - to);
        o *= fix;
        z *= fix;
#pragma unroll
        for (int k = 0; k < GR; ++k) {
            const float f = s0 + k < n ? fast_exp2(m_[k] - to) : 0.f;
            o = fmaf(f, o_[k], o);
            z = fmaf(f, z_[k], z);
        }
        top = to;
    }
    a.out[((int64_t)unit * G + g) * d_k + d] = z == 0.f ? 0.f : o / z;
}

// ---- host -------------------------------------------------------------------------------------------------------
// Ranges by length: how many, and from how many tokens on.  us a call (int8, d_k = 128, m = 8 unless said) for 512 / 1024 / 2048 / 4096 ranges in all,
// not under 1024 tokens each: 8 x 32 heads x 32768 tokens 174.7 / 171.8 / 169.0 / 171.2 (the more, the less the last ones run alone; two
// workgroups on a compute unit do not share it evenly); 32 x 8 x up to 8192 34.0 / 34.2 / 33.4 / 35.0; 16 x 12 x 4096 (d_k = 64, m = 4)
// 16.1 / 14.6 / 15.3 / 17.4; 28 x 25 x up to 4859 (same) 30.5 / 28.7 / 30.4 / 30.7; 1 x 8 x 32768 in groups of 4 15.4 / 15.3 / 15.8 / 18.3.
// So 1024, and 2048 where those still have 4096 tokens.  Least range of 512 / 1024 / 2048 tokens (1024 ranges): 2 heads in groups of 8 x 3000
// 10.3 / 11.6 / 13.6; 1 x 32 x 8192 13.5 / 13.4 / 15.5; 8 x 32 x up to 1500 16.7 / 14.8 / 14.0; 64 KB of tables (groups of 8, m = 8), which every
// range fetches: 12 x 8 x up to 8191 25.3 / 21.1 / 20.3, 64 x 4 x up to 2048 27.6 / 23.0 / 21.9.  So 1024, and 2048 from 64 KB on.
// Tables of 32 KB and more (G m >= 32): 512 ranges, two for each compute unit, and 256 from 128 KB on, of which one workgroup fills a
// compute unit; the target is not passed (range_by_length; for up to 64 sequences), so that nothing waits for a second round.  us, 1024 or 2048 ranges / so:
// groups of 8 x 4 heads, m = 16, 8 x 65536 81.6 / 57.6, 16 x up to 65536 104.9 / 72.3, m = 8 59.5 / 54.4 and 76.1 / 64.2; groups of 4 x 8, m = 8,
// 8 x 32768 52.9 / 51.2, 16 x up to 32768 66.8 / 61.9; groups of 8 x 8, d_k = 64, m = 4, 16 x up to 16384 31.4 / 24.0.  With 16 KB it costs: one
// head, m = 16, 16 x 32 x up to 16384 114.9 / 119.9; d_k = 64, 16 x 12 x 4096 17.0 / 18.8.
// Sequences of up to 2048 tokens are not cut at all: the merge is a launch more (8 x 32 x up to 1500 14.0 whole, 14.8 cut).  Where 1024 tokens a
// range would make fewer than 128 ranges, 512.
constexpr int kWholeLength = 2048;
static int least_range(int G, int m, int64_t units, int64_t room)
{
    return G * m >= 64 ? 2048 : units * room < 128 * 1024 ? 512 : 1024;
}

// How a call is cut up.
struct Cut {
    int per_head;     // ranges by length: ranges per head, or 0
    int least;        // ... of at least so many tokens
    int splits;       // equal ranges
    int64_t groups;   // workgroups
    int64_t ranges;   // ranges whose results the workspace holds (0: none)
};
static Cut cut_of(const lookat_page_pool *p, int32_t B, int32_t G, int32_t W, int64_t longest, int32_t num_splits)
{
    const int64_t units = (int64_t)B * p->H;
    Cut c;
    c.per_head = c.least = 0;
    c.splits = num_splits ? num_splits : 1;
    if (num_splits == 0 && longest > kWholeLength && B <= kMostPlanned) {
        // (from the rows' room where the number of ranges has to hold them all: a sequence may be longer than the caller knows)
        const int64_t room = (int64_t)W * p->page;
        if (one_round(p->m, G)) {
            const int target = G * p->m >= 128 ? 256 : 512;
            c.per_head = target > p->H ? target / p->H : 1;
        } else {
            const int64_t target = units * longest >= 2048LL * 4096 ? 2048 : 1024;
            c.per_head = (int)((target + p->H - 1) / p->H);
        }
        c.least = least_range(G, p->m, units, longest);
        const int64_t fit = (int64_t)B * ((room + c.least - 1) / c.least), most = c.per_head + 1 + B;
        c.ranges = p->H * (fit < most ? fit : most);
        c.groups = (c.ranges + kXcds - 1) / kXcds * kXcds;
        return c;
    }
    c.ranges = c.splits == 1 ? 0 : units * c.splits;
    c.groups = (units + kXcds - 1) / kXcds * kXcds * c.splits;
    return c;
}
static size_t cut_bytes(const lookat_page_pool *p, int32_t B, int32_t G, const Cut &c)
{
    const size_t plan = c.per_head ? ((size_t)B * sizeof(int2) + 15) / 16 * 16 : 0;
    return plan + (size_t)c.ranges * G * (p->d_k + 2) * sizeof(float);
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
static int launch_attend(const PoolArgs &p, const AttendArgs &a, bool fp8, bool brief, dim3 grid, hipStream_t st)
{
    constexpr int brief_waves = few_waves(G, M, 0) ? kShortWaves : kAttendWaves;
    const int waves = brief ? brief_waves : kAttendWaves;
    const size_t lds = attend_lds_bytes(G, M, DK, waves);
    const auto f = brief ? (fp8 ? &attend_pages_kernel<DK, M, G, true, brief_waves> : &attend_pages_kernel<DK, M, G, false, brief_waves>)
                         : (fp8 ? &attend_pages_kernel<DK, M, G, true, kAttendWaves> : &attend_pages_kernel<DK, M, G, false, kAttendWaves>);
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(f), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess)
            return fail(LOOKAT_ERR_HIP, "lookat_attend_pages: %s", hipGetErrorString(e));
    }
    hipLaunchKernelGGL(f, grid, dim3(waves * kWave), lds, st, p, a);
    return check_launch("lookat_attend_pages");
}
template <int DK, int M>
static int launch_attend_g(int G, const PoolArgs &p, const AttendArgs &a, bool fp8, bool brief, dim3 grid, hipStream_t st)
{
    switch (G) {
    case 1: return launch_attend<DK, M, 1>(p, a, fp8, brief, grid, st);
    case 2: return launch_attend<DK, M, 2>(p, a, fp8, brief, grid, st);
    case 4: return launch_attend<DK, M, 4>(p, a, fp8, brief, grid, st);
    default: return launch_attend<DK, M, 8>(p, a, fp8, brief, grid, st);
    }
}
template <int DK>
static int launch_attend_m(int G, const PoolArgs &p, const AttendArgs &a, bool fp8, bool brief, dim3 grid, hipStream_t st)
{
    switch (p.m) {
    case 2: return launch_attend_g<DK, 2>(G, p, a, fp8, brief, grid, st);
    case 4: return launch_attend_g<DK, 4>(G, p, a, fp8, brief, grid, st);
    case 8: return launch_attend_g<DK, 8>(G, p, a, fp8, brief, grid, st);
    default: return launch_attend_g<DK, 16>(G, p, a, fp8, brief, grid, st);
    }
}

}  // namespace lookat

extern "C" size_t lookat_attend_pages_workspace_bytes(const lookat_page_pool *pool, int32_t B, int32_t group, int32_t W, int64_t max_length,
                                                      int32_t num_splits)
{
    using namespace lookat;
    clear_error();
    if (check_attend(pool, B, group, W, max_length, num_splits) != LOOKAT_OK)
        return 0;
    return cut_bytes(pool, B, group, cut_of(pool, B, group, W, longest_of(pool, W, max_length), num_splits));
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
    const Cut cut = cut_of(pool, B, group, W, longest, num_splits);
    const size_t need = cut_bytes(pool, B, group, cut);
    if (need) {
        if (!workspace || workspace_bytes < need)
            return fail(LOOKAT_ERR_WORKSPACE, "workspace of %zu bytes needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
        if (!aligned16(workspace))
            return fail(LOOKAT_ERR_ALIGN, "workspace must be 16-byte aligned");
    }
    const int64_t units = (int64_t)B * pool->H;
    if (!fits_launch(cut.groups, kAttendWaves * kWave) || !fits_launch(units, pool->d_k))
        return fail(LOOKAT_ERR_UNSUPPORTED, "B*H*num_splits: %lld workgroups exceed one launch", (long long)cut.groups);
    const PoolArgs p = pool_args(pool);
    AttendArgs a;
    a.lut = lut;
    a.table = table;
    a.lengths = lengths;
    const size_t plan_bytes = cut.per_head ? ((size_t)B * sizeof(int2) + 15) / 16 * 16 : 0;
    a.plan = static_cast<int2 *>(workspace);
    a.part = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan_bytes);
    a.out = out;
    a.table_stride = table_stride;
    a.W = W;
    a.B = B;
    a.units = (int32_t)units;
    a.per_head = cut.per_head;
    a.least = cut.least;
    a.splits = cut.splits;
    a.chunk = (int32_t)(((longest + cut.splits - 1) / cut.splits + kTile - 1) / kTile * kTile);
    a.scale_log2e = scale * kLog2e;
    const bool fp8 = pool->value_type == LOOKAT_VALUES_E4M3;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)cut.groups);
    const bool brief = cut.splits == 1 && cut.per_head == 0 && few_waves(group, p.m, longest);
    const int rc = p.d_k == 64 ? launch_attend_m<64>(group, p, a, fp8, brief, grid, st) : launch_attend_m<128>(group, p, a, fp8, brief, grid, st);
    if (rc != LOOKAT_OK || !need)
        return rc;
    hipLaunchKernelGGL(attend_pages_merge_kernel, dim3((unsigned)units, group), dim3(p.d_k), 0, st, a, pool->H, group, p.d_k, p.page_log2);
    return check_launch("lookat_attend_pages (merge)");
}
