// The token that a row of logits gives for a random number, behind temperature, top-k, top-p and min-p.
//
// With M the row's largest logit and t its temperature, logit l_i has the weight w_i = 2^44 exp((l_i - M) / t), rounded to a whole number:
// sums of whole numbers do not depend on their order, so a row's token is the same in every run however the work is shared.
// (2^18 weights of at most 2^44 stay within 64 bits; what rounds to 0 has less than 2^-45 of the largest weight.)  In the order of
// falling logits, equal ones by place, a filter keeps the first logits: top-k the first k, top-p, of these, those with less
// than p of their sum in front of them.  So what is kept is one logit value, the threshold, and a place: everything above the value,
// and of its equals those up to the place.  min-p is a bound on w itself.
//
// sample_scan_kernel reads the logits, all blocks at the rate of the memory: the largest of every 64 or 16 (a group), and of every 4096 (a
// tile) also the sum of the weights against the tile's own largest, where the row needs a sum over all.
// sample_row_kernel, a block to a row, then reads little more of it:
//   * nothing filtered: the tiles' sums give the tile that the random number falls into, which is read;
//   * otherwise the groups' maxima (for a large k the logits themselves, counted) bound the threshold from below: the k-th largest of them
//     is no larger than the k-th largest logit.  The groups that reach the bound are read and the logits above it listed, up to 2048, and filtered.  For top-p
//     alone the bound is that of 128 groups, and the list will do if it has p of the sum;
//   * where it has not, the row is left to three more kernels, in which many blocks share it: a histogram of the weights by
//     (M - l) / t; the bin where their sum passes p, whose logits are listed, and the sums of each tile's logits above it; the draw.
//     So are rows of which more than 256 groups have to be read, for the list or, with min-p alone, the draw;
//   * where a list does not do, the block goes over the row by itself: the threshold digit by digit of the logit's bits (11, 11, 10 from the
//     top, as unsigned numbers in the logits' order), a histogram of each digit's values among what agrees in the digits before.  That
//     is slow, by one logit to a load, and happens
//       - with thousands of equal logits, or a k of some 2000 or more;
//       - with a k of up to half of the groups that is more than the groups with a logit above -inf: masked rows (5 rows of 128000 fp32 with 30 such logits,
//         us a call: k = 50 377, k = 20 18.3, no k 16.3; of 32000 107, 13.7, 11.7);
//       - with top-p alone, where one bin of the histogram, 1/32 of a temperature wide, has more than 2048 logits, as wide rows have at high temperatures
//         (5 rows of N(0, 2.5), top-p 0.95: 262144 fp32 t 1 51, t 1.6 635, t 3 818; 200003 t 2 49.5, t 3 566; 128000 t 3 46).
//
// One block to a row for all of it, by digits from memory, took 64 us for 5 rows of 32000 bf16, 556 for 320 of 128000 fp32 (a quarter of them
// top-p alone) and 111 for 80 of 200003 bf16, nothing filtered.  Now 20 to 32 (a row with k = 1000 is the
// slowest of such a call), 102 and 23.2.  The scan is bound by memory (164 MB in 28 us, 5.9 TB/s) or, with sums, by vector instructions (16 million
// fp64 exponentials in 18 us: 31 instructions a logit, a third of them fp64, issue in 12.7 of these); the row kernel by latency, some twenty steps
// between barriers (7 us where nothing is filtered, 14 with k = 50 and p, 20 over 320 rows); the three kernels behind it by their start, their loads and the list's (12, 23 and 17).
#pragma once

#include <type_traits>

#include "internal.h"
#include "scan64.h"

namespace fka {

constexpr int kSampleThreads = 512;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kSampleBins = 2048;
constexpr int kSampleFew = kSampleThreads / 4;
// Groups whose maxima bound the list of top-p alone.  (48 made no difference: a row whose kept logits are few is done either way, and one of thousands
// is left to many blocks or read by its own.)
constexpr int kSampleFirst = 128;
constexpr double kSampleUnit = 17592186044416.0;  // 2^44
constexpr uint32_t kNoLogit = 0x007fffffu;        // the key of -inf (NaN counts as that)

typedef unsigned long long u64;

// 2^(44 + j / 64), to nearest
__device__ const double kSampleTable[64] = {
    0x1.0000000000000p+44, 0x1.02c9a3e778061p+44, 0x1.059b0d3158574p+44, 0x1.0874518759bc8p+44,
    0x1.0b5586cf9890fp+44, 0x1.0e3ec32d3d1a2p+44, 0x1.11301d0125b51p+44, 0x1.1429aaea92de0p+44,
    0x1.172b83c7d517bp+44, 0x1.1a35beb6fcb75p+44, 0x1.1d4873168b9aap+44, 0x1.2063b88628cd6p+44,
    0x1.2387a6e756238p+44, 0x1.26b4565e27cddp+44, 0x1.29e9df51fdee1p+44, 0x1.2d285a6e4030bp+44,
    0x1.306fe0a31b715p+44, 0x1.33c08b26416ffp+44, 0x1.371a7373aa9cbp+44, 0x1.3a7db34e59ff7p+44,
    0x1.3dea64c123422p+44, 0x1.4160a21f72e2ap+44, 0x1.44e086061892dp+44, 0x1.486a2b5c13cd0p+44,
    0x1.4bfdad5362a27p+44, 0x1.4f9b2769d2ca7p+44, 0x1.5342b569d4f82p+44, 0x1.56f4736b527dap+44,
    0x1.5ab07dd485429p+44, 0x1.5e76f15ad2148p+44, 0x1.6247eb03a5585p+44, 0x1.6623882552225p+44,
    0x1.6a09e667f3bcdp+44, 0x1.6dfb23c651a2fp+44, 0x1.71f75e8ec5f74p+44, 0x1.75feb564267c9p+44,
    0x1.7a11473eb0187p+44, 0x1.7e2f336cf4e62p+44, 0x1.82589994cce13p+44, 0x1.868d99b4492edp+44,
    0x1.8ace5422aa0dbp+44, 0x1.8f1ae99157736p+44, 0x1.93737b0cdc5e5p+44, 0x1.97d829fde4e50p+44,
    0x1.9c49182a3f090p+44, 0x1.a0c667b5de565p+44, 0x1.a5503b23e255dp+44, 0x1.a9e6b5579fdbfp+44,
    0x1.ae89f995ad3adp+44, 0x1.b33a2b84f15fbp+44, 0x1.b7f76f2fb5e47p+44, 0x1.bcc1e904bc1d2p+44,
    0x1.c199bdd85529cp+44, 0x1.c67f12e57d14bp+44, 0x1.cb720dcef9069p+44, 0x1.d072d4a07897cp+44,
    0x1.d5818dcfba487p+44, 0x1.da9e603db3285p+44, 0x1.dfc97337b9b5fp+44, 0x1.e502ee78b3ff6p+44,
    0x1.ea4afa2a490dap+44, 0x1.efa1bee615a27p+44, 0x1.f50765b6e4540p+44, 0x1.fa7c1819e90d8p+44,
};

// Bits in the order of the logits; -0 equals 0.
__device__ inline uint32_t sample_key(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return x == x ? u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u) : kNoLogit;
}
__device__ inline float sample_logit(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// exp(x) in 64 bits as 2^(n / 64) times the series of the rest, |rest| <= ln 2 / 128: its next term is 4e-17 of the result.
struct SampleWeight {
    const double *table;  // kSampleTable, in LDS
    double max, step;     // M, 64 / (t ln 2)

    __device__ inline SampleWeight(const double *table_, uint32_t max_key, float t)
        : table(table_), max((double)sample_logit(max_key)), step(64 * 1.4426950408889634074 / (double)t)
    {
    }
    // what exp is of, in units of ln 2 / 64; no less than `least`, as which NaN counts (an infinite M beside another logit)
    __device__ inline double times64(float x, double least) const { return fmax(((double)x - max) * step, least); }
    __device__ static inline double series(double r)  // 2^(r / 64)
    {
        constexpr double L = 0.69314718055994530942 / 64;
        double p = __builtin_fma(r, L * L * L * L * L / 120, L * L * L * L / 24);
        p = __builtin_fma(r, p, L * L * L / 6);
        p = __builtin_fma(r, p, L * L / 2);
        p = __builtin_fma(r, p, L);
        return __builtin_fma(r, p, 1.0);
    }
    __device__ inline double exact(uint32_t key) const
    {
        const float x = sample_logit(key);
        if ((double)x == max) return kSampleUnit;
        const double z = times64(x, -64.0 * 1000), n = rint(z);
        const int m = (int)n;
        return ldexp(table[m & 63] * series(z - n), m >> 6);
    }
    // The weight + kMark.  What is below 2^-60 of the largest rounds to 0.
    static constexpr u64 kMark = 0x4330000000000000ull;
    __device__ inline u64 marked(float x) const
    {
        const double z = times64(x, -64.0 * 60), n = rint(z), p = series(z - n);
        const int m = (int)n;
        const double y = table[m & 63] * p;
        const double scaled = __hiloint2double(__double2hiint(y) + (int)((uint32_t)(m & ~63) << 14), __double2loint(y));  // 2^(m / 64), below
        // 2^52 added rounds to a whole number in the lowest bits
        return (u64)__double_as_longlong(scaled + 4503599627370496.0);
    }
    __device__ inline u64 operator()(uint32_t key) const
    {
        const float x = sample_logit(key);
        return (double)x == max ? (u64)kSampleUnit : marked(x) - kMark;
    }
};

template <class T>
struct SampleRow;
template <>
struct SampleRow<float> {
    static constexpr int VEC = 4;
    static constexpr uint32_t kNone = 0xff800000u;
    __device__ static float get(const uint32_t (&w)[4], int i) { return __uint_as_float(w[i]); }
    __device__ static float one(const float *p) { return *p; }
};
template <>
struct SampleRow<uint16_t> {
    static constexpr int VEC = 8;
    static constexpr uint32_t kNone = 0xff80ff80u;
    __device__ static float get(const uint32_t (&w)[4], int i) { return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
    __device__ static float one(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
};

// The VEC logits from place i on, 16 bytes, as they lie in memory (rows may start anywhere); `whole`: none is past the row's end, otherwise those
// that are count as -inf.
template <class T>
__device__ inline void sample_load(const T *row, int i, int n, bool whole, uint32_t (&w)[4])
{
    using R = SampleRow<T>;
    if (whole || i + R::VEC <= n) {
        __builtin_memcpy(w, row + i, 16);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = R::kNone;
            if constexpr (R::VEC == 4) {
                if (i + j < n) w[j] = __float_as_uint(R::one(row + i + j));
            } else {
                if (i + 2 * j < n) w[j] = (R::kNone << 16) | row[i + 2 * j];
                if (i + 2 * j + 1 < n) w[j] = (w[j] & 0xffffu) | (uint32_t)row[i + 2 * j + 1] << 16;
            }
        }
    }
}

template <class T>
__device__ inline void sample_keys(const T *row, int i, int n, uint32_t (&key)[SampleRow<T>::VEC])
{
    uint32_t w[4];
    sample_load(row, i, n, false, w);
#pragma unroll
    for (int j = 0; j < SampleRow<T>::VEC; ++j) key[j] = sample_key(SampleRow<T>::get(w, j));
}

// f(keys, place of the first) for the row, the block's threads side by side, all lanes of a wave at once (past the row's end: kNoLogit), and the loads of
// several steps on their way.
constexpr int kSampleAhead = 4;
template <class T, class F>
__device__ inline void sample_walk(const T *row, int n, F &&f)
{
    constexpr int VEC = SampleRow<T>::VEC, STEP = kSampleThreads * VEC;
    for (int i0 = 0; i0 < n; i0 += kSampleAhead * STEP) {
        const int at = i0 + (int)threadIdx.x * VEC;
        uint32_t w[kSampleAhead][4];
#pragma unroll
        for (int e = 0; e < kSampleAhead; ++e) sample_load(row, max(0, min(at + e * STEP, n - VEC)), n, n >= VEC, w[e]);
#pragma unroll
        for (int e = 0; e < kSampleAhead; ++e) {
            if (i0 + e * STEP >= n) break;  // (uniform)
            const int i = at + e * STEP;
            if (i + VEC > n) sample_load(row, i, n, false, w[e]);
            uint32_t key[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) key[j] = sample_key(SampleRow<T>::get(w[e], j));
            f(key, i);
        }
    }
}

__device__ inline bool sample_all(const SampleArgs &a, int r)  // whether row r needs the sum over all its logits
{
    const float t = a.temperature ? a.temperature[r] : 1.f, p = a.top_p ? a.top_p[r] : 1.f, m = a.min_p ? a.min_p[r] : 0.f;
    const int k = a.top_k ? a.top_k[r] : 0;
    return t > 0.f && !(k > 0 && k < a.n_vocab) && (p < 1.f || !(m > 0.f));
}

// Steps across lanes in the vector ALU (a shuffle is a round trip to LDS).
template <int CTRL, int ROWS = 0xf>
__device__ inline uint32_t sample_dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS = 0xf>
__device__ inline u64 sample_dpp(u64 x)
{
    return (u64)sample_dpp<CTRL, ROWS>((uint32_t)(x >> 32)) << 32 | sample_dpp<CTRL, ROWS>((uint32_t)x);
}
// f over the lanes up to each (0 where f(0, x) = x): row shifts, then the rows' last lanes.
template <class X, class F>
__device__ inline X sample_wave_scan(X x, F &&f)
{
    x = f(sample_dpp<0x111>(x), x);
    x = f(sample_dpp<0x112>(x), x);
    x = f(sample_dpp<0x114>(x), x);
    x = f(sample_dpp<0x118>(x), x);
    x = f(sample_dpp<0x142, 0xa>(x), x);
    return f(sample_dpp<0x143, 0xc>(x), x);
}
__device__ inline uint32_t sample_last(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); }
__device__ inline u64 sample_last(u64 x) { return (u64)sample_last((uint32_t)(x >> 32)) << 32 | sample_last((uint32_t)x); }
template <class X>
__device__ inline X sample_wave_max(X x)
{
    return sample_last(sample_wave_scan(x, [](X a, X b) { return a > b ? a : b; }));
}
__device__ inline u64 sample_wave_sum(u64 x)
{
    return sample_last(sample_wave_scan(x, [](u64 a, u64 b) { return a + b; }));
}

// Largest over the LANES lanes of a group.
template <int LANES>
__device__ inline float sample_group_max(float x)
{
    auto step = [](float v, auto ctrl) {
        return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)));
    };
    x = step(x, std::integral_constant<int, 0xb1>{});  // quad_perm 1,0,3,2
    if constexpr (LANES >= 4) x = step(x, std::integral_constant<int, 0x4e>{});  // quad_perm 2,3,0,1
    if constexpr (LANES >= 8) x = step(x, std::integral_constant<int, 0x141>{});  // row_half_mirror
    if constexpr (LANES == 16) x = step(x, std::integral_constant<int, 0x140>{});  // row_mirror
    return x;
}

// A block takes a tile: its groups' maxima, its maximum and its sum.
template <class T, int GROUP>
__global__ __launch_bounds__(256) void sample_scan_kernel(SampleArgs a)
{
    using R = SampleRow<T>;
    constexpr int VEC = R::VEC, LOADS = kSampleTile / (256 * VEC), GL = GROUP / VEC;  // lanes of a group
    __shared__ double table[64];
    __shared__ uint32_t top[4];
    __shared__ u64 part[4];
    const int tid = threadIdx.x, n = a.n_vocab;
    const int tiles = (n + kSampleTile - 1) / kSampleTile, groups = (n + GROUP - 1) / GROUP;
    const int r = blockIdx.x / tiles, tile = blockIdx.x - r * tiles, i0 = tile * kSampleTile + tid * VEC;
    const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.stride;
    if (blockIdx.x == 0 && tid == 0) *a.n_left = 0;
    uint32_t w[LOADS][4];
    if ((tile + 1) * kSampleTile <= n) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) sample_load(row, i0 + j * 256 * VEC, n, true, w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) sample_load(row, i0 + j * 256 * VEC, n, false, w[j]);
    }
    const bool all = sample_all(a, r);
    if (all && tid < 64) table[tid] = kSampleTable[tid];
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < VEC; ++i) m = fmaxf(m, __builtin_canonicalizef(R::get(w[j], i)));  // (drops a quiet NaN; a signalling one wins)
        m = sample_group_max<GL>(m);
        const int g = (i0 + j * 256 * VEC) / GROUP;
        if (tid % GL == 0 && g < groups) a.group_max[(size_t)r * groups + g] = sample_key(m);
        most = fmaxf(most, m);
    }
    if (!all) return;  // (uniform)
    const uint32_t wave_max = sample_wave_max(sample_key(most));
    if ((tid & 63) == 0) top[tid >> 6] = wave_max;
    __syncthreads();
    const uint32_t max_key = max(max(top[0], top[1]), max(top[2], top[3]));
    u64 sum = 0;
    if (max_key != kNoLogit) {
        const SampleWeight weight(table, max_key, a.temperature ? a.temperature[r] : 1.f);
        if (sample_logit(max_key) < INFINITY) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum += weight.marked(R::get(w[j], i));
            sum -= LOADS * VEC * SampleWeight::kMark;
        } else {
#pragma unroll
            for (int j = 0; j < LOADS; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum += R::get(w[j], i) == INFINITY ? (u64)kSampleUnit : 0;
        }
    }
    sum = sample_wave_sum(sum);
    if ((tid & 63) == 0) part[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) {
        a.tile_max[(size_t)r * tiles + tile] = max_key;
        a.tile_sum[(size_t)r * tiles + tile] = part[0] + part[1] + part[2] + part[3];
    }
}

struct SampleShared {
    double table[64];
    u64 hist[kSampleBins];
    u64 list[kSampleList], weight[kSampleList];  // (key << 32 | ~place): a larger one comes first
    uint16_t few[kSampleFew];
    uint16_t groups[kSampleGroups];
    u64 part[2 * kSampleWaves];
    u64 tile[kMaxVocab / (kSampleThreads * 4)];
    u64 result[4];
    int count, n_few;
};

// Sum over the block's threads before this one; `total` gets the sum of all.
template <int WAVES = kSampleWaves>
__device__ inline u64 sample_scan(u64 x, u64 *part, u64 &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const u64 y = sample_wave_scan(x, [](u64 a, u64 b) { return a + b; });
    __syncthreads();
    if (lane == 63) part[wave] = y;
    __syncthreads();
    u64 before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        if (i == wave) before = total;
        total += part[i];
    }
    return before + y - x;
}

// The last filled bin for whose front (`front`, and what is in the bins before it) takes(front) holds, and that front.  takes() holds up to
// some sum and not past it, so this is the bin whose own content leads past it, or the last that is filled.
template <int BINS, int THREADS, class F>
__device__ inline int sample_bin(const u64 *hist, u64 *part, u64 *result, u64 front, u64 &before, F &&takes)
{
    constexpr int EACH = BINS / THREADS;
    u64 x[EACH], sum = 0, total;
#pragma unroll
    for (int e = 0; e < EACH; ++e) sum += x[e] = hist[threadIdx.x * EACH + e];
    u64 in_front = sample_scan<THREADS / 64>(sum, part, total) + front;
    total += front;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const u64 next = in_front + x[e];
        if (x[e] && takes(in_front) && (next == total || !takes(next))) {
            result[0] = (u64)(threadIdx.x * EACH + e);
            result[1] = in_front;
        }
        in_front = next;
    }
    __syncthreads();
    before = result[1];
    return (int)result[0];
}
__device__ inline int sample_bin(double limit, u64 front, SampleShared &s, u64 &before)
{
    return sample_bin<kSampleBins, kSampleThreads>(s.hist, s.part, s.result, front, before, [=](u64 x) { return (double)x < limit; });
}

__device__ inline void sample_clear(SampleShared &s)
{
    __syncthreads();
    for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) s.hist[i] = 0;
    __syncthreads();
}

// The filters' threshold so far: kept are the keys above `key` and those equal to it at places up to `last`.
struct SampleKept {
    uint32_t key;
    int last;
    __device__ inline bool operator()(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

// f(key, place) for every logit of the row.  (One to a load: this is the way of rare rows, and wide loads make its code eight times as long.)
template <class T, class F>
__device__ inline void sample_each(const T *row, int n, F &&f)
{
#pragma unroll 2
    for (int i = threadIdx.x; i < n; i += kSampleThreads) f(sample_key(SampleRow<T>::one(row + i)), i);
}

// The last group of equal keys, among those that `kept` keeps, with less than `limit` in front of it (counts, or the sum of
// weights), and how much that is.
template <bool MASS, class T>
__device__ inline void sample_select(const T *row, int n, const SampleKept &kept, const SampleWeight &weight, double limit, SampleShared &s,
                                     uint32_t &key, u64 &before)
{
    uint32_t prefix = 0;
    before = 0;
    for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
        sample_clear(s);
        sample_each(row, n, [&](uint32_t k, int i) {
            if (!kept(k, i) || (digit && k >> (shift + bits) != prefix)) return;
            const u64 add = MASS ? weight(k) : 1;
            if (add) atomicAdd(&s.hist[kSampleBins - 1 - (k >> shift & ((1u << bits) - 1))], add);
        });
        __syncthreads();
        prefix = prefix << bits | (uint32_t)(kSampleBins - 1 - sample_bin(limit, before, s, before));
    }
    key = prefix;
}

// The place of the r-th (from 1) key equal to `key`; n if there are fewer.
template <class T>
__device__ inline int sample_place(const T *row, int n, uint32_t key, u64 r, SampleShared &s)
{
    u64 seen = 0;
    for (int at = 0; at < n; at += kSampleThreads) {
        const int i = at + threadIdx.x;
        const bool here = i < n && sample_key(SampleRow<T>::one(row + i)) == key;
        u64 total;
        const u64 rank = seen + sample_scan((u64)here, s.part, total);
        if (seen + total >= r) {
            if (here && rank + 1 == r) s.result[2] = (u64)i;
            __syncthreads();
            return (int)s.result[2];
        }
        seen += total;
    }
    return n;
}

// The place of the last of the keys equal to `key` that top-p keeps, with `before` in front of the first: that one, and each further one
// with less than `limit` in front of it.
template <class T>
__device__ inline int sample_mass_place(const T *row, int n, uint32_t key, u64 w, u64 before, double limit, SampleShared &s)
{
    u64 more = 1;
    for (u64 by = (u64)1 << 18; by; by >>= 1)
        if ((double)(before + (more + by - 1) * w) < limit) more += by;
    return sample_place(row, n, key, more, s);
}

// Appends the logits that each lane takes, bit j of `take` for key[j] at place + j, a wave at once; `count` counts them all, also those
// that do not fit.
template <int N>
__device__ inline void sample_append(u64 *list, int *count, uint32_t take, const uint32_t (&key)[N], int place)
{
    if (!__builtin_amdgcn_ballot_w64(take != 0)) return;
    const int mine = __popc(take), up_to = scan64(mine);
    int base = 0;
    if ((threadIdx.x & 63) == 63) base = atomicAdd(count, up_to);
    int at = __builtin_amdgcn_readlane(base, 63) + up_to - mine;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (take >> j & 1) {
            if (at < kSampleList) list[at] = (u64)key[j] << 32 | (uint32_t)~(place + j);
            ++at;
        }
}

// The part where the sum of up to 128 parts' sums passes the mark, and what is left of the mark in it.
struct SamplePart {
    int part;
    u64 mark, total;
};
template <class F>
__device__ inline SamplePart sample_part(const u64 *sums, int parts, F &&mark_of)
{
    const int lane = threadIdx.x & 63;
    const u64 a = 2 * lane < parts ? sums[2 * lane] : 0, b = 2 * lane + 1 < parts ? sums[2 * lane + 1] : 0;
    const u64 up_to = sample_wave_scan(a + b, [](u64 x, u64 y) { return x + y; }), total = sample_last(up_to), mark = mark_of(total);
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(up_to > mark));
    const u64 front = __shfl(up_to - a - b, at), first = __shfl(a, at);
    const bool second = mark - front >= first;
    return SamplePart{2 * at + (second ? 1 : 0), mark - front - (second ? first : 0), total};
}

// Of the n entries of s.list, those from `from` on in falling order (they differ, by their places): the last with less than `limit`
// in front of it, in what q(i) says of entry i, on top of `front`.  A histogram by the entries' upper bits finds a bin; its entries, where they
// are few, are compared with each other, otherwise their own range is cut into bins again.
template <class Q>
__device__ inline u64 sample_list_select(int n, u64 from, double limit, u64 front, SampleShared &s, Q &&q)
{
    const int tid = threadIdx.x;
    u64 low = 0, hi = 0;  // ~ the lowest, the highest
    for (int i = tid; i < n; i += kSampleThreads) {
        const u64 x = s.list[i];
        if (x >= from) {
            low = ~x > low ? ~x : low;
            hi = x > hi ? x : hi;
        }
    }
    for (;;) {  // [~low, hi] holds the entry; each round keeps less than a 1024th of it
        low = sample_wave_max(low);
        hi = sample_wave_max(hi);
        __syncthreads();
        if ((tid & 63) == 0) {
            s.part[tid >> 6] = hi;
            s.part[kSampleWaves + (tid >> 6)] = low;
        }
        if (tid == 0) s.n_few = 0;
        sample_clear(s);
#pragma unroll
        for (int i = 0; i < kSampleWaves; ++i) {
            hi = s.part[i] > hi ? s.part[i] : hi;
            low = s.part[kSampleWaves + i] > low ? s.part[kSampleWaves + i] : low;
        }
        const u64 top = hi, bottom = ~low, width = (top - bottom) >> 11;
        const int shift = width ? 64 - __builtin_clzll(width) : 0;
        for (int i = tid; i < n; i += kSampleThreads) {
            const u64 x = s.list[i];
            if (x >= bottom && x <= top) {
                const u64 add = q(i);
                if (add) atomicAdd(&s.hist[(top - x) >> shift], add);
            }
        }
        __syncthreads();
        const u64 b = (u64)sample_bin(limit, front, s, front);
        low = hi = 0;
        for (int i = tid; i < n; i += kSampleThreads) {
            const u64 x = s.list[i];
            if (x >= bottom && x <= top && (top - x) >> shift == b && q(i)) {
                const int at = atomicAdd(&s.n_few, 1);
                if (at < kSampleFew) s.few[at] = (uint16_t)i;
                low = ~x > low ? ~x : low;
                hi = x > hi ? x : hi;
            }
        }
        if (tid == 0) s.result[3] = ~0ull;
        __syncthreads();
        if (s.n_few <= kSampleFew) break;
    }
    // four lanes an entry share the others
    const int few = s.n_few, i = tid / 4;
    if (i < few) {
        const u64 x = s.list[s.few[i]];
        u64 before = 0;
        for (int j = tid % 4; j < few; j += 4) before += s.list[s.few[j]] > x ? q(s.few[j]) : 0;
        before += __shfl_xor(before, 1);
        before += __shfl_xor(before, 2);
        if ((double)(front + before) < limit) atomicMin(&s.result[3], x);
    }
    __syncthreads();
    return s.result[3];
}

// What is drawn from: the row's parameters.
struct SampleDraw {
    float t, p, u;
    int k;      // 0: no top-k
    u64 least;  // the smallest weight that min-p keeps

    __device__ inline SampleDraw(const SampleArgs &a, int r)
        : t(a.temperature ? a.temperature[r] : 1.f), p(a.top_p ? a.top_p[r] : 1.f), u(a.u[r]), k(a.top_k ? a.top_k[r] : 0)
    {
        if (k < 0 || k >= a.n_vocab) k = 0;
        const float m = a.min_p ? a.min_p[r] : 0.f;
        least = m > 0.f ? (u64)ceil(fmin((double)m, 1.0) * kSampleUnit) : 0;
    }
    __device__ inline u64 mark(u64 total) const
    {
        const double at = floor((u > 0.f ? (double)u : 0.0) * (double)total);
        const u64 m = at < (double)total ? (u64)at : total - 1;  // (a double may be past the sum that it was made from)
        return m < total ? m : total - 1;
    }
};

__device__ inline void sample_answer(const SampleArgs &a, int r, int token, double logprob)
{
    a.tokens[r] = token;
    if (a.logprob) a.logprob[r] = (float)logprob;
}

// The same as sample_from_list for up to 64 entries, by one wave: an entry's rank is the number of those above it, and with the entries
// in that order sums across lanes take the place of histograms.
__device__ inline bool sample_from_few(const SampleArgs &a, int r, const SampleDraw &draw, const SampleWeight &weight, int n, double sum,
                                       SampleShared &s)
{
    const int lane = threadIdx.x & 63;
    u64 x = lane < n ? s.list[lane] : 0;
    auto entry = [](u64 v, int i) {
        return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, i);
    };
    int rank = lane < n ? 0 : lane;
    for (int i = 0; i < n; ++i) rank += lane < n && entry(x, i) > x ? 1 : 0;
    x = (u64)(uint32_t)__builtin_amdgcn_ds_permute(4 * rank, (int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_ds_permute(4 * rank, (int)x);
    if (draw.k) n = min(n, draw.k);
    auto add = [](u64 p, u64 q) { return p + q; };
    u64 w = lane < n ? weight((uint32_t)(x >> 32)) : 0;
    const u64 up_to = sample_wave_scan(w, add), total = sample_last(up_to);
    bool in = w > 0 && w >= draw.least;
    if (draw.p < 1.f) {
        const double limit = fmax((double)draw.p * (draw.k ? (double)total : sum), 0.5);  // the first is always kept
        if (!draw.k && (double)total < limit) return false;
        in = in && (double)(up_to - w) < limit;
    }
    w = in ? w : 0;
    const u64 kept = sample_wave_sum(w), mark = draw.mark(kept);
    u64 before = 0;  // the kept weights of lower places
    for (int i = 0; i < n; ++i) {
        const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, i);  // ~place
        before += at > (uint32_t)x ? entry(w, i) : 0;
    }
    if (w && mark >= before && mark < before + w) sample_answer(a, r, (int)~(uint32_t)x, log((double)w / (double)kept));
    return true;
}

// Filters and draws from the n entries of s.list, which hold all that is kept.  `sum`: of all the row's weights, where the list is
// not known to hold what top-p keeps; false if it does not.
__device__ inline bool sample_from_list(const SampleArgs &a, int r, const SampleDraw &draw, const SampleWeight &weight, int n, double sum,
                                        SampleShared &s)
{
    const int tid = threadIdx.x;
    __syncthreads();
    for (int i = tid; i < n; i += kSampleThreads) s.weight[i] = weight((uint32_t)(s.list[i] >> 32));
    __syncthreads();
    u64 from = 0, total = 0;  // kept are the entries from `from` on
    if (draw.k && draw.k < n) from = sample_list_select(n, 0, (double)draw.k, 0, s, [](int) { return (u64)1; });
    if (draw.p < 1.f) {
        u64 mine = 0;
        for (int i = tid; i < n; i += kSampleThreads) mine += s.list[i] >= from ? s.weight[i] : 0;
        sample_scan(mine, s.part, total);
        const double limit = fmax((double)draw.p * (draw.k ? (double)total : sum), 0.5);  // the first is always kept
        if (!draw.k && (double)total < limit) return false;  // (uniform)
        from = sample_list_select(n, from, limit, 0, s, [&](int i) { return s.weight[i]; });
    }
    // in the vocabulary's order: the kept weights of equal stretches of it, the stretch where their sum passes the mark, its entries
    const int width = (a.n_vocab - 1) >> 11, shift = width ? 32 - __builtin_clz(width) : 0;
    auto kept = [&](int i) -> u64 { return s.list[i] >= from && s.weight[i] >= draw.least ? s.weight[i] : 0; };
    sample_clear(s);
    u64 mine = 0;
    for (int i = tid; i < n; i += kSampleThreads) {
        const u64 w = kept(i);
        mine += w;
        if (w) atomicAdd(&s.hist[~(uint32_t)s.list[i] >> shift], w);
    }
    if (tid == 0) s.n_few = 0;
    sample_scan(mine, s.part, total);
    const u64 mark = draw.mark(total);
    u64 front;
    const uint32_t stretch = (uint32_t)sample_bin<kSampleBins, kSampleThreads>(s.hist, s.part, s.result, 0, front, [=](u64 x) { return x <= mark; });
    for (int i = tid; i < n; i += kSampleThreads)
        if (kept(i) && ~(uint32_t)s.list[i] >> shift == stretch) s.few[atomicAdd(&s.n_few, 1)] = (uint16_t)i;
    __syncthreads();
    static_assert(kSampleFew >= kMaxVocab / kSampleBins, "a stretch's entries");
    const int few = s.n_few, e = tid / 4;
    if (e < few) {
        const uint32_t at = (uint32_t)s.list[s.few[e]];  // ~place
        u64 before = 0;
        for (int j = tid % 4; j < few; j += 4) before += (uint32_t)s.list[s.few[j]] > at ? s.weight[s.few[j]] : 0;
        before += __shfl_xor(before, 1);
        before += __shfl_xor(before, 2);
        const u64 here = s.weight[s.few[e]];
        if (tid % 4 == 0 && mark >= front + before && mark < front + before + here)
            sample_answer(a, r, (int)~at, log((double)here / (double)total));
    }
    return true;
}

// The place where the sum of the kept weights of COUNT logits, `first` on, passes mark_of(their sum).
template <int COUNT, class T, class F>
__device__ inline void sample_from_part(const SampleArgs &a, int r, const T *row, int first, F &&mark_of, double total, SampleShared &s,
                                        const SampleDraw &draw, const SampleKept &kept, const SampleWeight &weight)
{
    constexpr int EACH = COUNT / kSampleThreads;
    const int i = first + (int)threadIdx.x * EACH;
    u64 w[EACH], sum = 0, here;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        w[j] = 0;
        if (i + j < a.n_vocab) {
            const uint32_t key = sample_key(SampleRow<T>::one(row + i + j));
            const u64 x = kept(key, i + j) ? weight(key) : 0;
            w[j] = x >= draw.least ? x : 0;
        }
        sum += w[j];
    }
    u64 before = sample_scan(sum, s.part, here);
    const u64 mark = mark_of(here);
    if (mark >= before && mark < before + sum) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            if (mark >= before && mark < before + w[j]) sample_answer(a, r, i + j, log((double)w[j] / total));
            before += w[j];
        }
    }
}

// The part, by the kept weights of each in s.tile, then the thread and the place where their sum passes the mark.
template <class T>
__device__ inline void sample_from_parts(const SampleArgs &a, int r, const T *row, const SampleDraw &draw, const SampleKept &kept,
                                         const SampleWeight &weight, SampleShared &s)
{
    constexpr int PART = kSampleThreads * SampleRow<T>::VEC;
    const SamplePart at = sample_part(s.tile, (a.n_vocab + PART - 1) / PART, [&](u64 total) { return draw.mark(total); });
    sample_from_part<PART>(a, r, row, at.part * PART, [&](u64) { return at.mark; }, (double)at.total, s, draw, kept, weight);
}

// Draws from all that the threshold and min-p keep: the kept weights of each part of the row, then as above.
template <class T>
__device__ inline void sample_from_row(const SampleArgs &a, int r, const T *row, const SampleDraw &draw, const SampleKept &kept,
                                       const SampleWeight &weight, SampleShared &s)
{
    constexpr int VEC = SampleRow<T>::VEC, PART = kSampleThreads * VEC;
    const int n = a.n_vocab, tid = threadIdx.x, parts = (n + PART - 1) / PART;
    __syncthreads();
    if (tid < parts) s.tile[tid] = 0;
    __syncthreads();
    sample_walk(row, n, [&](const uint32_t(&x)[VEC], int i) {
        u64 sum = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const u64 w = i + j < n && kept(x[j], i + j) ? weight(x[j]) : 0;
            sum += w >= draw.least ? w : 0;
        }
        sum = sample_wave_sum(sum);
        if ((tid & 63) == 0 && sum) atomicAdd(&s.tile[i / PART], sum);
    });
    __syncthreads();
    sample_from_parts(a, r, row, draw, kept, weight, s);
}

// Lane i: tile i's share of the sum of all weights, in units of the largest one's 2^-44: 0 for a tile whose largest rounds to 0 there.
__device__ inline double sample_tile_sum(const SampleArgs &a, int r, const SampleWeight &weight)
{
    const int tiles = (a.n_vocab + kSampleTile - 1) / kSampleTile, lane = threadIdx.x & 63;
    if (lane >= tiles) return 0;
    const uint32_t key = a.tile_max[(size_t)r * tiles + lane];
    return weight(key) ? (double)a.tile_sum[(size_t)r * tiles + lane] * (weight.exact(key) / kSampleUnit) : 0;
}

// Nothing filtered: the tile that the random number falls into, by the tiles' sums, and the place in it by the weights against M (in a tile
// with a share one at least is no 0).
template <class T>
__device__ inline void sample_from_tiles(const SampleArgs &a, int r, const T *row, const SampleDraw &draw, const SampleWeight &weight,
                                         SampleShared &s)
{
    const int n = a.n_vocab, lane = threadIdx.x & 63;
    const double sum = sample_tile_sum(a, r, weight);
    double up_to = sum;  // the sums up to the lane's tile
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double z = __shfl_up(up_to, d);
        if (lane >= d) up_to += z;
    }
    const double total = __shfl(up_to, 63), mark = (draw.u > 0.f ? fmin((double)draw.u, 1.0) : 0.0) * total;
    const u64 past = __builtin_amdgcn_ballot_w64(sum > 0 && up_to > mark), any = __builtin_amdgcn_ballot_w64(sum > 0);
    const int tile = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any);
    const double here = __shfl(sum, tile), front = __shfl(up_to, tile) - here;
    const double part = fmin(fmax((mark - front) / here, 0.0), 1.0);
    sample_from_part<kSampleTile>(
        a, r, row, tile * kSampleTile, [=](u64 all) { return min((u64)(part * (double)all), all - 1); }, total, s, draw,
        SampleKept{0, n}, weight);
}

// (M - l) / t in bins of 1/32 (a weight of more than 2^-45 is in the first 999).
struct SampleNucleusBin {
    float max, step;
    __device__ inline SampleNucleusBin(uint32_t max_key, float t) : max(sample_logit(max_key)), step(32.f / t) {}
    __device__ inline int operator()(float x) const { return x == max ? 0 : (int)fminf((max - x) * step, (float)(kSampleLeftBins - 1)); }
};

// top-p alone, by one block: the histogram of the weights; the list of the bin where their sum passes the limit, and the sums of each part's
// weights above it; the draw.  False where the list does not fit.
template <class T>
__device__ inline bool sample_nucleus(const SampleArgs &a, int r, const T *row, const SampleDraw &draw, const SampleWeight &weight,
                                      uint32_t max_key, double limit, SampleShared &s)
{
    constexpr int VEC = SampleRow<T>::VEC, PART = kSampleThreads * VEC;
    const int tid = threadIdx.x, n = a.n_vocab, parts = (n + PART - 1) / PART;
    const SampleNucleusBin bin(max_key, draw.t);
    sample_clear(s);
    if (tid == 0) s.count = 0;
    if (tid < parts) s.tile[tid] = 0;
    sample_walk(row, n, [&](const uint32_t(&x)[VEC], int) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const u64 w = weight(x[j]);
            if (w) atomicAdd(&s.hist[bin(sample_logit(x[j]))], w);
        }
    });
    __syncthreads();
    u64 front;
    const int border = sample_bin(limit, 0, s, front);
    sample_walk(row, n, [&](const uint32_t(&x)[VEC], int i) {
        uint32_t take = 0;
        u64 sum = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int b = x[j] > kNoLogit ? bin(sample_logit(x[j])) : kSampleLeftBins;
            take |= b == border ? 1u << j : 0;
            const u64 w = b < border ? weight(x[j]) : 0;
            sum += w >= draw.least ? w : 0;
        }
        sum = sample_wave_sum(sum);
        if ((tid & 63) == 0 && sum) atomicAdd(&s.tile[i / PART], sum);
        sample_append(s.list, &s.count, take, x, i);
    });
    __syncthreads();
    const int count = s.count;
    if (count > kSampleList) return false;  // (uniform)
    for (int i = tid; i < count; i += kSampleThreads) s.weight[i] = weight((uint32_t)(s.list[i] >> 32));
    __syncthreads();
    const u64 last = sample_list_select(count, 0, limit, front, s, [&](int i) { return s.weight[i]; });
    for (int i = tid; i < count; i += kSampleThreads)
        if (s.list[i] >= last && s.weight[i] >= draw.least) atomicAdd(&s.tile[~(uint32_t)s.list[i] / PART], s.weight[i]);
    __syncthreads();
    sample_from_parts(a, r, row, draw, SampleKept{(uint32_t)(last >> 32), (int)~(uint32_t)last}, weight, s);
    return true;
}

// Top-k, and top-p behind it or alone, over the whole row.  limit: top-p's, where it is alone.
template <class T>
__device__ inline SampleKept sample_whole_row(const T *row, int n, const SampleWeight &weight, const SampleDraw &draw, double limit,
                                              SampleShared &s)
{
    SampleKept kept{0, n};
    uint32_t key;
    u64 before;
    if (draw.k) {
        sample_select<false>(row, n, kept, weight, (double)draw.k, s, key, before);
        kept.last = sample_place(row, n, key, (u64)draw.k - before, s);
        kept.key = key;
    }
    if (!(draw.p < 1.f)) return kept;
    if (draw.k) {
        u64 sum = 0, total;
        sample_each(row, n, [&](uint32_t x, int i) { sum += kept(x, i) ? weight(x) : 0; });
        sample_scan(sum, s.part, total);
        limit = fmax((double)draw.p * (double)total, 0.5);  // the first is always kept
    }
    sample_select<true>(row, n, kept, weight, limit, s, key, before);
    const int last = sample_mass_place(row, n, key, weight(key), before, limit, s);
    return SampleKept{key, key == kept.key ? min(kept.last, last) : last};
}

// Leaves the row to many blocks, where there is a place.
__device__ inline bool sample_leave(const SampleArgs &a, SampleShared &s, const SampleLeft &left)
{
    if (a.max_left == 0) return false;
    __syncthreads();
    if (threadIdx.x == 0) {
        const int at = atomicAdd(a.n_left, 1);
        s.result[0] = (u64)(at < a.max_left);
        if (at < a.max_left) a.left[at] = left;
    }
    __syncthreads();
    return s.result[0] != 0;
}

template <class T, int GROUP>
__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(SampleArgs a)
{
    constexpr int VEC = SampleRow<T>::VEC, GL = GROUP / VEC, EACH = kSampleGroups / kSampleThreads, AHEAD = 4;
    __shared__ SampleShared s;
    const int r = blockIdx.x, n = a.n_vocab, tid = threadIdx.x, groups = (n + GROUP - 1) / GROUP;
    const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.stride;
    if (tid < 64) s.table[tid] = kSampleTable[tid];
    const SampleDraw draw(a, r);

    // the groups' maxima; the largest, in the first group that has it, and the lowest that is a number
    uint32_t most[EACH], low = 0;  // ~ the lowest
    u64 best = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int g = tid + e * kSampleThreads;
        most[e] = g < groups ? a.group_max[(size_t)r * groups + g] : kNoLogit;
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const u64 x = (u64)most[e] << 32 | (uint32_t)~(tid + e * kSampleThreads);
        best = x > best ? x : best;
        if (most[e] > kNoLogit) low = max(low, ~most[e]);
    }
    best = sample_wave_max(best);
    low = sample_wave_max(low);
    if ((tid & 63) == 0) {
        s.part[tid >> 6] = best;
        s.part[kSampleWaves + (tid >> 6)] = low;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSampleWaves; ++i) {
        best = s.part[i] > best ? s.part[i] : best;
        low = max(low, (uint32_t)s.part[kSampleWaves + i]);
    }
    const uint32_t max_key = (uint32_t)(best >> 32);
    if (max_key == kNoLogit || !(draw.t > 0.f)) {
        if (max_key == kNoLogit) {
            if (tid == 0) {
                sample_answer(a, r, -1, -INFINITY);
                if (a.err) atomicOr(a.err, kErrNoToken);
            }
        } else if (tid < 64) {
            const int i = (int)~(uint32_t)best * GROUP + tid;
            const u64 equal = __builtin_amdgcn_ballot_w64(tid < GROUP && i < n && sample_key(SampleRow<T>::one(row + min(i, n - 1))) == max_key);
            if (tid == 0) sample_answer(a, r, i + __builtin_ctzll(equal), 0.0);
        }
        return;
    }
    const SampleWeight weight(s.table, max_key, draw.t);
    const bool nucleus = draw.p < 1.f && !draw.k;
    if (!draw.k && !nucleus && !draw.least) {
        sample_from_tiles(a, r, row, draw, weight, s);
        return;
    }

    // the list of the logits above a bound that is below the threshold
    double sum = nucleus ? sample_tile_sum(a, r, weight) : 0;
    if (nucleus) {
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    }
    const double limit = fmax((double)draw.p * sum, 0.5);
    const float top = sample_logit(max_key), range = top - sample_logit(~low);
    const bool by_rank = draw.k || nucleus;
    // k so large that the groups' maxima say little about the k-th logit: the bins count the logits themselves (over twice the maxima's range; what
    // is below is in the last one).  us a call of 5 rows, maxima / logits: 17000 (1063 groups of 16) k 300 17.4 / 21.1, 600 20.8 / 22.6, 1000
    // 60 / 25; 24000 k 600 20.2 / 24.2, 1000 24.9 / 26.6; 32000 k 1000 24.1 / 28.3, 1500 158 / 35; 128000 (groups of 64) k 1500 506 / 55.
    const bool ranks = draw.k > groups / 2;
    int bound = 0;
    const float step = range > 0.f ? (kSampleBins - 1) / (ranks ? 2 * range : range) : 0.f;
    auto bin = [&](uint32_t k) -> int { return (int)fminf((top - sample_logit(k)) * step, (float)(kSampleBins - 1)); };
    auto above = [&](uint32_t k) -> bool { return k > kNoLogit && (by_rank ? bin(k) <= bound : weight(k) >= draw.least); };
    const bool listed = !by_rank || (range < 1.5e38f && step < 3e38f);  // (uniform)
    if (listed) {
        if (tid == 0) s.count = s.n_few = 0;
        if (by_rank) {
            sample_clear(s);
            if (ranks) {
                sample_walk(row, n, [&](const uint32_t(&x)[VEC], int) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        if (x[j] > kNoLogit) atomicAdd(&s.hist[bin(x[j])], 1ull);
                });
            } else {
#pragma unroll
                for (int e = 0; e < EACH; ++e)
                    if (most[e] > kNoLogit) atomicAdd(&s.hist[bin(most[e])], 1ull);
            }
            __syncthreads();
            u64 unused;
            bound = sample_bin((double)(draw.k ? draw.k : kSampleFirst), 0, s, unused);
        } else {
            __syncthreads();
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (above(most[e])) s.groups[atomicAdd(&s.n_few, 1)] = (uint16_t)(tid + e * kSampleThreads);
        __syncthreads();
        const int picked = s.n_few;
        // Shared by many blocks / read by this one, us a call, fp32, all rows with the same k: 5 rows of 128000 k 100 22.3 / 25.4, 400 23.5 / 31, 1000
        // 26.9 / 48; 40 rows k 300 30.0 / 30.0, 600 31.2 / 38.9; 320 rows k 100 76 / 50, 400 80 / 61, 1000 87 / 83; 5 rows of 65536 (groups of
        // 16) k 100 22.5 / 20.5, 1000 26.4 / 29.0.  Where only some of many rows share, theirs cost less.
        if (picked > 256 && !nucleus && (ranks || picked >= draw.k) &&
            sample_leave(a, s, SampleLeft{limit, 0, r, max_key, 0, by_rank ? bound : SampleLeft::kAll, step}))
            return;
        for (int e0 = 0; e0 < picked * GL; e0 += AHEAD * kSampleThreads) {  // AHEAD loads of a thread on their way
            uint32_t w[AHEAD][4];
            int place[AHEAD];
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const int at = e0 + e * kSampleThreads + tid;
                if (at - tid >= picked * GL) break;  // (uniform)
                place[e] = at < picked * GL ? s.groups[at / GL] * GROUP + at % GL * VEC : n;
                sample_load(row, max(0, min(place[e], n - VEC)), n, n >= VEC, w[e]);
            }
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                if (e0 + e * kSampleThreads >= picked * GL) break;
                if (place[e] + VEC > n) sample_load(row, place[e], n, false, w[e]);
                uint32_t x[VEC], take = 0;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    x[j] = sample_key(SampleRow<T>::get(w[e], j));
                    take |= above(x[j]) ? 1u << j : 0;  // (past the row's end: kNoLogit)
                }
                sample_append(s.list, &s.count, take, x, place[e]);
            }
        }
        __syncthreads();
        const int count = s.count;
        // (fewer groups than k: a logit below all of them may be among the first k)
        if ((ranks || picked >= draw.k) && count <= kSampleList &&
            (count <= 64 ? sample_from_few(a, r, draw, weight, count, sum, s) : sample_from_list(a, r, draw, weight, count, sum, s)))
            return;
        __syncthreads();
    }
    if (nucleus && sample_leave(a, s, SampleLeft{limit, 0, r, max_key, 0, SampleLeft::kNucleus, 0.f})) return;
    if (nucleus && sample_nucleus(a, r, row, draw, weight, max_key, limit, s)) return;
    sample_from_row(a, r, row, draw, by_rank ? sample_whole_row(row, n, weight, draw, limit, s) : SampleKept{0, n}, weight, s);
}

// The rows that are left: block c of the a.shares of a row takes every a.shares-th tile of it.
struct SampleShare {
    const SampleLeft *left;
    int share;
    bool on;
    __device__ inline explicit SampleShare(const SampleArgs &a)
    {
        const int at = (int)blockIdx.x / a.shares;
        share = (int)blockIdx.x - at * a.shares;
        on = at < min(*a.n_left, a.max_left);
        left = a.left + at;
    }
};

// f(logits, place of the first) for the tiles of a share, all of a wave's lanes at once (those past the row's end: -inf).
template <class T, class F, class G>
__device__ inline void sample_share_tiles(const SampleArgs &a, int r, int share, F &&f, G &&after)
{
    using R = SampleRow<T>;
    constexpr int VEC = R::VEC, LOADS = kSampleTile / (256 * VEC);
    const int n = a.n_vocab, tiles = (n + kSampleTile - 1) / kSampleTile;
    const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.stride;
    for (int tile = share; tile < tiles; tile += a.shares) {
        const int i0 = tile * kSampleTile + (int)threadIdx.x * VEC;
        uint32_t w[LOADS][4];
        if ((tile + 1) * kSampleTile <= n) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) sample_load(row, i0 + j * 256 * VEC, n, true, w[j]);
        } else {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) sample_load(row, i0 + j * 256 * VEC, n, false, w[j]);
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            float x[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] = R::get(w[j], i);
            f(x, i0 + j * 256 * VEC);
        }
        after(tile);
    }
}

template <class T>
__global__ __launch_bounds__(256) void sample_hist_kernel(SampleArgs a)
{
    constexpr int VEC = SampleRow<T>::VEC;
    __shared__ double table[64];
    __shared__ u64 hist[kSampleLeftBins];
    const SampleShare mine(a);
    if (!mine.on || mine.left->bound != SampleLeft::kNucleus) return;
    const int tid = threadIdx.x, r = mine.left->row;
    const uint32_t max_key = mine.left->max_key;
    if (tid < 64) table[tid] = kSampleTable[tid];
    for (int i = tid; i < kSampleLeftBins; i += 256) hist[i] = 0;
    __syncthreads();
    const float t = a.temperature ? a.temperature[r] : 1.f;
    const SampleWeight weight(table, max_key, t);
    const SampleNucleusBin bin(max_key, t);
    const float max = sample_logit(max_key);
    sample_share_tiles<T>(
        a, r, mine.share,
        [&](const float(&x)[VEC], int) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const u64 w = x[j] == max ? (u64)kSampleUnit : weight.marked(x[j]) - SampleWeight::kMark;
                if (w) atomicAdd(&hist[bin(x[j])], w);
            }
        },
        [](int) {});
    __syncthreads();
    for (int i = tid; i < kSampleLeftBins; i += 256) a.hist[(size_t)blockIdx.x * kSampleLeftBins + i] = hist[i];
}

template <class T>
__global__ __launch_bounds__(256) void sample_cut_kernel(SampleArgs a)
{
    constexpr int VEC = SampleRow<T>::VEC;
    __shared__ double table[64];
    __shared__ u64 hist[kSampleLeftBins];
    __shared__ u64 part[4], result[2], list[kSampleList];
    __shared__ int count, base;
    const SampleShare mine(a);
    if (!mine.on) return;
    const int tid = threadIdx.x, at = mine.left - a.left, r = mine.left->row, tiles = (a.n_vocab + kSampleTile - 1) / kSampleTile;
    const uint32_t max_key = mine.left->max_key;
    const double limit = mine.left->limit;
    const int bound = mine.left->bound;
    if (tid == 0) count = 0;
    auto pass_on = [&]() {
        __syncthreads();
        if (tid == 0) base = atomicAdd(&a.left[at].count, count);  // (one to a block: a wave's would be a round trip to memory each)
        __syncthreads();
        for (int i = tid; i < min(count, kSampleList); i += 256)
            if (base + i < kSampleList) a.list[(size_t)at * kSampleList + base + i] = list[i];
    };
    if (bound >= 0) {  // the list of the logits up to a bound, as sample_row_kernel makes it
        const float top = sample_logit(max_key), step = mine.left->step;
        __syncthreads();
        sample_share_tiles<T>(
            a, r, mine.share,
            [&](const float(&x)[VEC], int i) {
                uint32_t key[VEC], take = 0;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    key[j] = sample_key(x[j]);
                    take |= key[j] > kNoLogit && (int)fminf((top - x[j]) * step, (float)(kSampleBins - 1)) <= bound ? 1u << j : 0;
                }
                sample_append(list, &count, take, key, i);
            },
            [](int) {});
        pass_on();
        return;
    }
    if (tid < 64) table[tid] = kSampleTable[tid];
    int border = kSampleLeftBins;
    u64 front = 0;
    if (bound == SampleLeft::kNucleus) {
        // four bins a thread, the loads of several shares on their way at a time
        static_assert(kSampleLeftBins == 4 * 256, "four bins a thread");
        ulonglong2 sum[2] = {};
        const ulonglong2 *from = reinterpret_cast<const ulonglong2 *>(a.hist + (size_t)at * a.shares * kSampleLeftBins) + 2 * tid;
#pragma unroll 8
        for (int c = 0; c < a.shares; ++c) {
            const ulonglong2 x = from[0], y = from[1];
            from += kSampleLeftBins / 2;
            sum[0].x += x.x, sum[0].y += x.y, sum[1].x += y.x, sum[1].y += y.y;
        }
        hist[4 * tid] = sum[0].x, hist[4 * tid + 1] = sum[0].y, hist[4 * tid + 2] = sum[1].x, hist[4 * tid + 3] = sum[1].y;
        __syncthreads();
        border = sample_bin<kSampleLeftBins, 256>(hist, part, result, 0, front, [=](u64 x) { return (double)x < limit; });
    }
    __syncthreads();
    if (mine.share == 0 && tid == 0) a.left[at].front = front;
    const SampleDraw draw(a, r);
    const SampleWeight weight(table, max_key, draw.t);
    const SampleNucleusBin bin(max_key, draw.t);
    const float max = sample_logit(max_key);
    u64 sum = 0;
    sample_share_tiles<T>(
        a, r, mine.share,
        [&](const float(&x)[VEC], int i) {
            uint32_t key[VEC], take = 0;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int b = bin(fmaxf(x[j], -INFINITY));  // (fmaxf drops a NaN)
                if (b < border) {
                    const u64 w = x[j] == max ? (u64)kSampleUnit : weight.marked(x[j]) - SampleWeight::kMark;
                    sum += w >= draw.least ? w : 0;
                }
                take |= b == border ? 1u << j : 0;
                key[j] = sample_key(x[j]);
            }
            sample_append(list, &count, take, key, i);
        },
        [&](int tile) {
            sum = sample_wave_sum(sum);
            __syncthreads();
            if ((tid & 63) == 0) part[tid >> 6] = sum;
            __syncthreads();
            if (tid == 0) a.tile_sum[(size_t)r * tiles + tile] = part[0] + part[1] + part[2] + part[3];
            sum = 0;
        });
    pass_on();
}

template <class T>
__global__ __launch_bounds__(kSampleThreads) void sample_left_kernel(SampleArgs a)
{
    __shared__ SampleShared s;
    const int at = blockIdx.x, tid = threadIdx.x, n = a.n_vocab, tiles = (n + kSampleTile - 1) / kSampleTile;
    if (at >= min(*a.n_left, a.max_left)) return;
    const SampleLeft left = a.left[at];
    const int r = left.row, count = left.count;
    const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.stride;
    if (tid < 64) s.table[tid] = kSampleTable[tid];
    if (tid < tiles && left.bound < 0) s.tile[tid] = a.tile_sum[(size_t)r * tiles + tid];
    __syncthreads();
    const SampleDraw draw(a, r);
    const SampleWeight weight(s.table, left.max_key, draw.t);
    if (count > kSampleList) {  // (not min-p alone)
        sample_from_row(a, r, row, draw, sample_whole_row(row, n, weight, draw, left.limit, s), weight, s);
        return;
    }
    for (int i = tid; i < count; i += kSampleThreads) {
        s.list[i] = a.list[(size_t)at * kSampleList + i];
        s.weight[i] = weight((uint32_t)(s.list[i] >> 32));
    }
    if (left.bound >= 0) {
        (void)sample_from_list(a, r, draw, weight, count, 0, s);  // (top-k: it holds all that is kept)
        return;
    }
    __syncthreads();
    u64 last = 0;  // (nothing listed: min-p alone)
    if (left.bound == SampleLeft::kNucleus)
        last = sample_list_select(count, 0, left.limit, left.front, s, [&](int i) { return s.weight[i]; });
    for (int i = tid; i < count; i += kSampleThreads)
        if (s.list[i] >= last && s.weight[i] >= draw.least) atomicAdd(&s.tile[~(uint32_t)s.list[i] / kSampleTile], s.weight[i]);
    __syncthreads();
    const SamplePart in = sample_part(s.tile, tiles, [&](u64 total) { return draw.mark(total); });
    sample_from_part<kSampleTile>(a, r, row, in.part * kSampleTile, [&](u64) { return in.mark; }, (double)in.total, s, draw,
                                  SampleKept{(uint32_t)(last >> 32), (int)~(uint32_t)last}, weight);
}

template <class T, int GROUP>
void launch_sample_group(const SampleArgs &a, hipStream_t s)
{
    const unsigned tiles = (a.n_vocab + kSampleTile - 1) / kSampleTile;
    sample_scan_kernel<T, GROUP><<<dim3(a.n_rows * tiles), dim3(256), 0, s>>>(a);
    sample_row_kernel<T, GROUP><<<dim3(a.n_rows), dim3(kSampleThreads), 0, s>>>(a);
}

template <class T>
void launch_sample_type(const SampleArgs &a, hipStream_t s)
{
    if (sample_group_of(a.n_vocab) == 16)
        launch_sample_group<T, 16>(a, s);
    else
        launch_sample_group<T, 64>(a, s);
    if (a.max_left == 0) return;
    sample_hist_kernel<T><<<dim3(a.max_left * a.shares), dim3(256), 0, s>>>(a);
    sample_cut_kernel<T><<<dim3(a.max_left * a.shares), dim3(256), 0, s>>>(a);
    sample_left_kernel<T><<<dim3(a.max_left), dim3(kSampleThreads), 0, s>>>(a);
}

inline hipError_t launch_sample_kernels(const SampleArgs &a, hipStream_t s)
{
    if (a.n_rows <= 0) return hipSuccess;
    if (a.bf16)
        launch_sample_type<uint16_t>(a, s);
    else
        launch_sample_type<float>(a, s);
    return hipGetLastError();
}

}  // namespace fka
