// The token that a row of logits gives for a random number, behind temperature, top-k, top-p and min-p.
//
// With M the row's largest logit and t its temperature, logit l_i has the weight w_i = 2^44 exp((l_i - M) / t), rounded to a whole number:
// sums of whole numbers do not depend on their order, so a row's token is the same in every run however the work is shared.
// (2^18 weights of at most 2^44 stay within 64 bits; what rounds to 0 has less than 2^-45 of the largest weight.)  In the order of
// falling logits, equal ones by place, a filter keeps the first logits: top-k the first k, top-p, of these, those with less
// than p of their sum in front of them.  So what is kept is one logit value, the threshold, and a place: everything above the value,
// and of its equals those up to the place.  min-p is a bound on w itself.
//
// Two kernels.  sample_scan_kernel reads the logits, all blocks at the rate of the memory: the largest of every 64 (a
// group), and of every 4096 (a tile) also the sum of the weights against the tile's own largest, where the row needs a sum over all.
// sample_row_kernel, a block to a row, then reads little more of it:
//   * nothing filtered: the tiles' sums give the tile that the random number falls into, which is read;
//   * otherwise the groups' maxima bound the threshold from below: the k-th largest of them is no larger than the k-th largest
//     logit.  The groups that reach the bound are read and the logits above it listed, up to 2048, ranked, and filtered.  For top-p
//     alone the bound is that of 256 groups, and the list will do if it has p of the sum;
//   * where it does not, a histogram of the weights by (M - l) / t, then the list of the bin where the sum passes p;
//   * where a list does not fit: the threshold digit by digit of the logit's bits (11, 11, 10 from the top, as unsigned numbers in the
//     logits' order), a histogram of each digit's values among what agrees in the digits before.
#pragma once

#include "internal.h"

namespace fka {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kSampleBins = 2048;
constexpr int kSampleList = 2048;
constexpr double kSampleUnit = 17592186044416.0;  // 2^44
constexpr uint32_t kNoLogit = 0x007fffffu;        // the key of -inf (NaN counts as that)

typedef unsigned long long u64;

// 2^(j / 64), to nearest
__device__ const double kSampleTable[64] = {
    0x1.0000000000000p+0, 0x1.02c9a3e778061p+0, 0x1.059b0d3158574p+0, 0x1.0874518759bc8p+0,
    0x1.0b5586cf9890fp+0, 0x1.0e3ec32d3d1a2p+0, 0x1.11301d0125b51p+0, 0x1.1429aaea92de0p+0,
    0x1.172b83c7d517bp+0, 0x1.1a35beb6fcb75p+0, 0x1.1d4873168b9aap+0, 0x1.2063b88628cd6p+0,
    0x1.2387a6e756238p+0, 0x1.26b4565e27cddp+0, 0x1.29e9df51fdee1p+0, 0x1.2d285a6e4030bp+0,
    0x1.306fe0a31b715p+0, 0x1.33c08b26416ffp+0, 0x1.371a7373aa9cbp+0, 0x1.3a7db34e59ff7p+0,
    0x1.3dea64c123422p+0, 0x1.4160a21f72e2ap+0, 0x1.44e086061892dp+0, 0x1.486a2b5c13cd0p+0,
    0x1.4bfdad5362a27p+0, 0x1.4f9b2769d2ca7p+0, 0x1.5342b569d4f82p+0, 0x1.56f4736b527dap+0,
    0x1.5ab07dd485429p+0, 0x1.5e76f15ad2148p+0, 0x1.6247eb03a5585p+0, 0x1.6623882552225p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6dfb23c651a2fp+0, 0x1.71f75e8ec5f74p+0, 0x1.75feb564267c9p+0,
    0x1.7a11473eb0187p+0, 0x1.7e2f336cf4e62p+0, 0x1.82589994cce13p+0, 0x1.868d99b4492edp+0,
    0x1.8ace5422aa0dbp+0, 0x1.8f1ae99157736p+0, 0x1.93737b0cdc5e5p+0, 0x1.97d829fde4e50p+0,
    0x1.9c49182a3f090p+0, 0x1.a0c667b5de565p+0, 0x1.a5503b23e255dp+0, 0x1.a9e6b5579fdbfp+0,
    0x1.ae89f995ad3adp+0, 0x1.b33a2b84f15fbp+0, 0x1.b7f76f2fb5e47p+0, 0x1.bcc1e904bc1d2p+0,
    0x1.c199bdd85529cp+0, 0x1.c67f12e57d14bp+0, 0x1.cb720dcef9069p+0, 0x1.d072d4a07897cp+0,
    0x1.d5818dcfba487p+0, 0x1.da9e603db3285p+0, 0x1.dfc97337b9b5fp+0, 0x1.e502ee78b3ff6p+0,
    0x1.ea4afa2a490dap+0, 0x1.efa1bee615a27p+0, 0x1.f50765b6e4540p+0, 0x1.fa7c1819e90d8p+0,
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
    uint32_t max_key;

    __device__ inline SampleWeight(const double *table_, uint32_t max_key_, float t)
        : table(table_), max((double)sample_logit(max_key_)), step(64 * 1.4426950408889634074 / (double)t), max_key(max_key_)
    {
    }
    __device__ inline double exact(uint32_t key) const
    {
        if (key == max_key) return kSampleUnit;
        const double z = ((double)sample_logit(key) - max) * step;
        if (!(z > -64.0 * 1000) || key == kNoLogit) return 0;  // (also infinities: -inf, or all but those of an infinite M)
        const double n = rint(z), r = (z - n) * (0.69314718055994530942 / 64);
        const int m = (int)n;
        double p = __builtin_fma(r, 1.0 / 120, 1.0 / 24);
        p = __builtin_fma(r, p, 1.0 / 6);
        p = __builtin_fma(r, p, 0.5);
        p = __builtin_fma(r, p, 1.0);
        p = __builtin_fma(r, p, 1.0);
        return ldexp(table[m & 63] * p, (m >> 6) + 44);
    }
    __device__ inline u64 operator()(uint32_t key) const
    {
        // 2^52 added rounds to a whole number in the lowest bits
        return (u64)__double_as_longlong(exact(key) + 4503599627370496.0) & 0xfffffffffffffull;
    }
};

template <class T>
struct SampleRow;
template <>
struct SampleRow<float> {
    static constexpr int VEC = 4;
    __device__ static float get(const uint32_t (&w)[4], int i) { return __uint_as_float(w[i]); }
    __device__ static float one(const float *p) { return *p; }
};
template <>
struct SampleRow<uint16_t> {
    static constexpr int VEC = 8;
    __device__ static float get(const uint32_t (&w)[4], int i) { return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
    __device__ static float one(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
};

// The keys of the VEC logits from place i on (those past the row's end: kNoLogit).
template <class T>
__device__ inline void sample_keys(const T *row, int i, int n, uint32_t (&key)[SampleRow<T>::VEC])
{
    using R = SampleRow<T>;
    if (i + R::VEC <= n) {
        uint32_t w[4];
        __builtin_memcpy(w, row + i, 16);  // rows may start anywhere
#pragma unroll
        for (int j = 0; j < R::VEC; ++j) key[j] = sample_key(R::get(w, j));
    } else {
#pragma unroll
        for (int j = 0; j < R::VEC; ++j) key[j] = i + j < n ? sample_key(R::one(row + i + j)) : kNoLogit;
    }
}

__device__ inline bool sample_all(const SampleArgs &a, int r)  // whether row r needs the sum over all its logits
{
    const float t = a.temperature ? a.temperature[r] : 1.f, p = a.top_p ? a.top_p[r] : 1.f, m = a.min_p ? a.min_p[r] : 0.f;
    const int k = a.top_k ? a.top_k[r] : 0;
    return t > 0.f && !(k > 0 && k < a.n_vocab) && (p < 1.f || !(m > 0.f));
}

__device__ inline u64 sample_wave_sum(u64 x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// A block takes a tile: its groups' maxima, its maximum and its sum.
template <class T>
__global__ __launch_bounds__(256) void sample_scan_kernel(SampleArgs a)
{
    constexpr int VEC = SampleRow<T>::VEC, LOADS = kSampleTile / (256 * VEC), GL = kSampleGroup / VEC;  // lanes of a group
    __shared__ double table[64];
    __shared__ uint32_t top[4];
    __shared__ u64 part[4];
    const int tid = threadIdx.x, n = a.n_vocab;
    const int tiles = (n + kSampleTile - 1) / kSampleTile, groups = (n + kSampleGroup - 1) / kSampleGroup;
    const int r = blockIdx.x / tiles, tile = blockIdx.x - r * tiles;
    const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.stride;
    uint32_t key[LOADS][VEC], most = 0;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) sample_keys(row, tile * kSampleTile + j * 256 * VEC + tid * VEC, n, key[j]);
    const bool all = sample_all(a, r);
    if (all && tid < 64) table[tid] = kSampleTable[tid];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        uint32_t m = key[j][0];
#pragma unroll
        for (int i = 1; i < VEC; ++i) m = max(m, key[j][i]);
#pragma unroll
        for (int d = 1; d < GL; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
        const int g = (tile * kSampleTile + j * 256 * VEC + tid * VEC) / kSampleGroup;
        if (tid % GL == 0 && g < groups) a.group_max[(size_t)r * groups + g] = m;
        most = max(most, m);
    }
    if (!all) return;  // (uniform)
#pragma unroll
    for (int d = GL; d < 64; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    if ((tid & 63) == 0) top[tid >> 6] = most;
    __syncthreads();
    most = max(max(top[0], top[1]), max(top[2], top[3]));
    u64 sum = 0;
    if (most != kNoLogit) {
        const SampleWeight weight(table, most, a.temperature ? a.temperature[r] : 1.f);
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum += weight(key[j][i]);
    }
    sum = sample_wave_sum(sum);
    if ((tid & 63) == 0) part[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) {
        a.tile_max[(size_t)r * tiles + tile] = most;
        a.tile_sum[(size_t)r * tiles + tile] = part[0] + part[1] + part[2] + part[3];
    }
}

struct SampleShared {
    double table[64];
    u64 hist[kSampleBins];
    u64 list[kSampleList], ranked[kSampleList];  // (key << 32 | ~place): a larger one comes first
    uint16_t groups[kMaxVocab / kSampleGroup];
    u64 part[kSampleWaves];
    u64 tile[kMaxVocab / kSampleTile];
    u64 result[4];
    int count;
};

// Sum over the block's threads before this one; `total` gets the sum of all.
__device__ inline u64 sample_scan(u64 x, SampleShared &s, u64 &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 y = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const u64 z = __shfl_up(y, d);
        if (lane >= d) y += z;
    }
    __syncthreads();
    if (lane == 63) s.part[wave] = y;
    __syncthreads();
    u64 before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kSampleWaves; ++i) {
        if (i == wave) before = total;
        total += s.part[i];
    }
    return before + y - x;
}

// The last filled bin, from the top, with less than `limit` in front of it, and what is in front.
__device__ inline int sample_bin(double limit, u64 front, SampleShared &s, u64 &before)
{
    static_assert(kSampleBins == 2 * kSampleThreads, "two bins a thread");
    const int tid = threadIdx.x;
    const u64 a = s.hist[2 * tid], b = s.hist[2 * tid + 1];
    u64 total;
    const u64 in_front = sample_scan(a + b, s, total) + front;
    if (tid == 0) s.result[0] = 0;
    __syncthreads();
    u64 mine = 0;
    if (a && (double)in_front < limit) mine = (u64)tid * 2 + 1;
    if (b && (double)(in_front + a) < limit) mine = (u64)tid * 2 + 2;
    if (mine) atomicMax(&s.result[0], mine);
    __syncthreads();
    if (mine && s.result[0] == mine) s.result[1] = (mine & 1) ? in_front : in_front + a;
    __syncthreads();
    before = s.result[1];
    return (int)s.result[0] - 1;
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

// f(key, place) for every logit of the row.
template <class T, class F>
__device__ inline void sample_each(const T *row, int n, F &&f)
{
    constexpr int VEC = SampleRow<T>::VEC;
    for (int i = threadIdx.x * VEC; i < n; i += kSampleThreads * VEC) {
        uint32_t k[VEC];
        sample_keys(row, i, n, k);
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (i + j < n) f(k[j], i + j);
    }
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
    constexpr int VEC = SampleRow<T>::VEC;
    u64 seen = 0;
    for (int at = 0; at < n; at += kSampleThreads * VEC) {
        const int i = at + threadIdx.x * VEC;
        uint32_t k[VEC];
        sample_keys(row, i, n, k);
        u64 here = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) here += i + j < n && k[j] == key;
        u64 total;
        u64 rank = seen + sample_scan(here, s, total);
        if (seen + total >= r) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (i + j < n && k[j] == key && ++rank == r) s.result[2] = (u64)(i + j);
            __syncthreads();
            return (int)s.result[2];
        }
        seen += total;
    }
    return n;
}

// Appends the logits that take() accepts to the list; s.count counts them all, also those that do not fit.
__device__ inline void sample_append(SampleShared &s, uint32_t key, int place)
{
    const int at = atomicAdd(&s.count, 1);
    if (at < kSampleList) s.list[at] = (u64)key << 32 | (uint32_t)~place;
}

// s.ranked: the n entries of s.list in falling order (they differ, by their places).
__device__ inline void sample_rank(SampleShared &s, int n)
{
    const int tid = threadIdx.x;
    if (n <= 512) {  // an entry's rank is the number of those above it; the threads of an entry share the others
        const int shares = n <= 64 ? 16 : n <= 128 ? 8 : n <= 256 ? 4 : 2;  // neighbouring lanes
        const int i = tid / shares, share = tid % shares;
        const u64 x = i < n ? s.list[i] : 0;
        int above = 0;
        for (int j = share; j < n; j += shares) above += s.list[j] > x;
        for (int d = 1; d < shares; d <<= 1) above += __shfl_xor(above, d);
        if (i < n && share == 0) s.ranked[above] = x;
        __syncthreads();
        return;
    }
    // a bitonic sort of 1024 or 2048 entries
    const int size = n <= 1024 ? 1024 : 2048;
    for (int i = tid; i < size; i += kSampleThreads) s.ranked[i] = i < n ? s.list[i] : 0;
    __syncthreads();
    for (int run = 2; run <= size; run <<= 1)
        for (int d = run >> 1; d; d >>= 1) {
            for (int e = tid; e < size / 2; e += kSampleThreads) {
                const int lo = (e & ~(d - 1)) * 2 + (e & (d - 1)), hi = lo + d;
                const u64 x = s.ranked[lo], y = s.ranked[hi];
                if ((x < y) == ((lo & run) == 0)) s.ranked[lo] = y, s.ranked[hi] = x;
            }
            __syncthreads();
        }
}

// What is drawn from: the row's parameters.
struct SampleDraw {
    float t, p, u;
    int k;      // 0: no top-k
    u64 least;  // the smallest weight that min-p keeps
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

// Filters and draws from the n entries of s.list, which hold all that is kept.  `sum`: of all the row's weights, where the list is
// not known to hold what top-p keeps; false if it does not.
__device__ inline bool sample_from_list(const SampleArgs &a, int r, const SampleDraw &draw, const SampleWeight &weight, int n, double sum,
                                        SampleShared &s)
{
    const int tid = threadIdx.x;
    sample_rank(s, n);
    if (draw.k) n = min(n, draw.k);
    // two entries a thread, in order
    u64 w[2], before[2], total;
    for (int e = 0; e < 2; ++e) w[e] = 2 * tid + e < n ? weight((uint32_t)(s.ranked[2 * tid + e] >> 32)) : 0;
    before[0] = sample_scan(w[0] + w[1], s, total);
    before[1] = before[0] + w[0];
    bool in[2];
    const double limit = (double)draw.p * (draw.k ? (double)total : sum);
    if (draw.p < 1.f && !draw.k && (double)total < limit) return false;  // (uniform)
    u64 mine = 0;
    for (int e = 0; e < 2; ++e) {
        const int i = 2 * tid + e;
        in[e] = i < n && (!(draw.p < 1.f) || i == 0 || (double)before[e] < limit) && w[e] >= draw.least && w[e] > 0;
        mine += in[e] ? 1 : 0;
    }
    // in the vocabulary's order: the sums up to each kept entry (kept ones are the first `kept`)
    u64 kept;
    sample_scan(mine, s, kept);
    for (int e = 0; e < 2; ++e)
        if (in[e]) s.list[2 * tid + e] = w[e];
    __syncthreads();
    u64 kept_sum;
    sample_scan((in[0] ? w[0] : 0) + (in[1] ? w[1] : 0), s, kept_sum);
    const u64 mark = draw.mark(kept_sum);
    const int shares = kept <= 64 ? 16 : kept <= 128 ? 8 : kept <= 256 ? 4 : kept <= 512 ? 2 : 1;
    for (int i = tid / shares; i < (int)kept; i += kSampleThreads / shares) {
        const uint32_t at = (uint32_t)s.ranked[i];  // ~place
        u64 front = 0;
        for (int j = tid % shares; j < (int)kept; j += shares) front += (uint32_t)s.ranked[j] > at ? s.list[j] : 0;
        for (int d = 1; d < shares; d <<= 1) front += __shfl_xor(front, d);
        const u64 here = s.list[i];
        if (tid % shares == 0 && mark >= front && mark < front + here)
            sample_answer(a, r, (int)~at, log((double)here / (double)kept_sum));
    }
    return true;
}

// Draws from all that the threshold and min-p keep: the kept weights of each part of the row, then the part, the thread and the place
// where the sum passes the mark.
template <class T>
__device__ inline void sample_from_row(const SampleArgs &a, int r, const T *row, const SampleDraw &draw, const SampleKept &kept,
                                       const SampleWeight &weight, SampleShared &s)
{
    constexpr int VEC = SampleRow<T>::VEC, PART = kSampleThreads * VEC;
    const int n = a.n_vocab, tid = threadIdx.x, parts = (n + PART - 1) / PART;
    __syncthreads();
    if (tid < parts) s.tile[tid] = 0;
    __syncthreads();
    auto kept_weight = [&](uint32_t key, int i) -> u64 {
        if (i >= n || !kept(key, i)) return 0;
        const u64 w = weight(key);
        return w >= draw.least ? w : 0;
    };
    for (int part = 0; part < parts; ++part) {
        const int i = part * PART + tid * VEC;
        uint32_t x[VEC];
        sample_keys(row, i, n, x);
        u64 sum = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum += kept_weight(x[j], i + j);
        sum = sample_wave_sum(sum);
        if ((tid & 63) == 0 && sum) atomicAdd(&s.tile[part], sum);
    }
    __syncthreads();
    u64 total = 0;
    for (int i = 0; i < parts; ++i) total += s.tile[i];
    u64 mark = draw.mark(total);
    int part = 0;
    while (mark >= s.tile[part]) mark -= s.tile[part++];
    const int i = part * PART + tid * VEC;
    uint32_t x[VEC];
    sample_keys(row, i, n, x);
    u64 w[VEC], sum = 0, unused;
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum += w[j] = kept_weight(x[j], i + j);
    u64 before = sample_scan(sum, s, unused);
    if (mark >= before && mark < before + sum) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if (mark >= before && mark < before + w[j]) sample_answer(a, r, i + j, log((double)w[j] / (double)total));
            before += w[j];
        }
    }
}

// Lane i: tile i's share of the sum of all weights, in units of the largest one's 2^-44.
__device__ inline double sample_tile_sum(const SampleArgs &a, int r, const SampleWeight &weight)
{
    const int tiles = (a.n_vocab + kSampleTile - 1) / kSampleTile, lane = threadIdx.x & 63;
    if (lane >= tiles) return 0;
    return (double)a.tile_sum[(size_t)r * tiles + lane] * (weight.exact(a.tile_max[(size_t)r * tiles + lane]) / kSampleUnit);
}

// Nothing filtered: the tile that the random number falls into, by the tiles' sums, and the place in it.
template <class T>
__device__ inline void sample_from_tiles(const SampleArgs &a, int r, const T *row, const SampleDraw &draw, const SampleWeight &against,
                                         SampleShared &s)
{
    const int n = a.n_vocab, tid = threadIdx.x, lane = tid & 63, tiles = (n + kSampleTile - 1) / kSampleTile;
    const double sum = sample_tile_sum(a, r, against);
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
    const uint32_t tile_key = a.tile_max[(size_t)r * tiles + tile];
    const double unit = against.exact(tile_key) / kSampleUnit;
    const SampleWeight weight(s.table, tile_key, draw.t);
    const int i = tile * kSampleTile + tid * 4;
    u64 w[4], mine = 0, all;
#pragma unroll
    for (int j = 0; j < 4; ++j) mine += w[j] = i + j < n ? weight(sample_key(SampleRow<T>::one(row + i + j))) : 0;
    u64 before = sample_scan(mine, s, all);
    const u64 at = min((u64)(fmin(fmax((mark - front) / here, 0.0), 1.0) * (double)all), all - 1);
    if (at >= before && at < before + mine) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (at >= before && at < before + w[j]) sample_answer(a, r, i + j, log((double)w[j] * unit / total));
            before += w[j];
        }
    }
}

// The threshold of top-p alone: the bin of (M - l) / t in which the sum passes the limit, and in it the last logit with less than the limit
// in front.
template <class T>
__device__ inline SampleKept sample_nucleus(const T *row, int n, const SampleWeight &weight, float t, double limit, SampleShared &s)
{
    const int tid = threadIdx.x;
    const float max = sample_logit(weight.max_key), step = 64.f / t;
    auto bin = [&](uint32_t k) -> int {
        return k == weight.max_key ? 0 : (int)fminf((max - sample_logit(k)) * step, (float)(kSampleBins - 1));
    };
    sample_clear(s);
    sample_each(row, n, [&](uint32_t k, int) {
        const u64 w = weight(k);
        if (w) atomicAdd(&s.hist[bin(k)], w);
    });
    __syncthreads();
    u64 front;
    const int b = sample_bin(limit, 0, s, front);
    if (tid == 0) s.count = 0;
    __syncthreads();
    sample_each(row, n, [&](uint32_t k, int i) {
        if (bin(k) == b) sample_append(s, k, i);
    });
    __syncthreads();
    const int count = s.count;
    if (count <= kSampleList) {
        sample_rank(s, count);
        u64 w[2], unused;
        for (int e = 0; e < 2; ++e) w[e] = 2 * tid + e < count ? weight((uint32_t)(s.ranked[2 * tid + e] >> 32)) : 0;
        const u64 before = front + sample_scan(w[0] + w[1], s, unused);
        // the last with less than the limit in front; the bin's first has
        if (tid == 0) s.result[3] = 0;
        __syncthreads();
        u64 mine = 0;
        if (w[0] && (double)before < limit) mine = 2 * tid;
        if (w[1] && (double)(before + w[0]) < limit) mine = 2 * tid + 1;
        if (mine) atomicMax(&s.result[3], mine);
        __syncthreads();
        const u64 last = s.ranked[s.result[3]];
        return SampleKept{(uint32_t)(last >> 32), (int)~(uint32_t)last};
    }
    SampleKept kept{0, n};
    uint32_t key;
    u64 before;
    sample_select<true>(row, n, kept, weight, limit, s, key, before);
    // of its equals those with less than the limit in front: one, and each further one
    const u64 w = weight(key);
    u64 more = 1;
    for (u64 by = (u64)1 << 18; by; by >>= 1)
        if ((double)(before + (more + by - 1) * w) < limit) more += by;
    return SampleKept{key, sample_place(row, n, key, more, s)};
}

// Top-k, and top-p behind it, over the whole row.
template <class T>
__device__ inline SampleKept sample_first_k(const T *row, int n, const SampleWeight &weight, int k, float p, SampleShared &s)
{
    SampleKept kept{0, n};
    uint32_t key;
    u64 before;
    sample_select<false>(row, n, kept, weight, (double)k, s, key, before);
    kept.last = sample_place(row, n, key, (u64)k - before, s);
    kept.key = key;
    if (!(p < 1.f)) return kept;
    u64 sum = 0, total;
    sample_each(row, n, [&](uint32_t x, int i) { sum += kept(x, i) ? weight(x) : 0; });
    sample_scan(sum, s, total);
    const double limit = fmax((double)p * (double)total, 0.5);  // the first is always kept
    sample_select<true>(row, n, kept, weight, limit, s, key, before);
    const u64 w = weight(key);
    u64 more = 1;
    for (u64 by = (u64)1 << 18; by; by >>= 1)
        if ((double)(before + (more + by - 1) * w) < limit) more += by;
    const int last = sample_place(row, n, key, more, s);
    return SampleKept{key, key == kept.key ? min(kept.last, last) : last};
}

template <class T>
__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(SampleArgs a)
{
    constexpr int VEC = SampleRow<T>::VEC, GL = kSampleGroup / VEC, EACH = kMaxVocab / kSampleGroup / kSampleThreads;
    __shared__ SampleShared s;
    const int r = blockIdx.x, n = a.n_vocab, tid = threadIdx.x, groups = (n + kSampleGroup - 1) / kSampleGroup;
    const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.stride;
    if (tid < 64) s.table[tid] = kSampleTable[tid];

    // the groups' maxima; the largest, in the first group that has it, and the lowest that is a number
    uint32_t most[EACH], low = ~0u;
    u64 best = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int g = tid + e * kSampleThreads;
        most[e] = g < groups ? a.group_max[(size_t)r * groups + g] : kNoLogit;
        const u64 x = (u64)most[e] << 32 | (uint32_t)~g;
        best = x > best ? x : best;
        if (most[e] > kNoLogit) low = min(low, most[e]);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const u64 x = __shfl_xor(best, d);
        best = x > best ? x : best;
        low = min(low, (uint32_t)__shfl_xor((int)low, d));
    }
    if ((tid & 63) == 0) {
        s.part[tid >> 6] = best;
        s.tile[tid >> 6] = low;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSampleWaves; ++i) {
        best = s.part[i] > best ? s.part[i] : best;
        low = min(low, (uint32_t)s.tile[i]);
    }
    const uint32_t max_key = (uint32_t)(best >> 32);
    SampleDraw draw;
    draw.t = a.temperature ? a.temperature[r] : 1.f;
    if (max_key == kNoLogit || !(draw.t > 0.f)) {
        if (max_key == kNoLogit) {
            if (tid == 0) {
                sample_answer(a, r, -1, -INFINITY);
                if (a.err) atomicOr(a.err, kErrNoToken);
            }
        } else if (tid < 64) {
            const int i = (int)~(uint32_t)best * kSampleGroup + tid;
            const u64 equal = __builtin_amdgcn_ballot_w64(i < n && sample_key(SampleRow<T>::one(row + min(i, n - 1))) == max_key);
            if (tid == 0) sample_answer(a, r, i + __builtin_ctzll(equal), 0.0);
        }
        return;
    }
    const SampleWeight weight(s.table, max_key, draw.t);
    const float min_p = a.min_p ? a.min_p[r] : 0.f;
    draw.p = a.top_p ? a.top_p[r] : 1.f;
    draw.u = a.u[r];
    draw.k = a.top_k ? a.top_k[r] : 0;
    if (draw.k < 0 || draw.k >= n) draw.k = 0;
    draw.least = min_p > 0.f ? (u64)ceil(fmin((double)min_p, 1.0) * kSampleUnit) : 0;
    const bool nucleus = draw.p < 1.f && !draw.k;
    if (!draw.k && !nucleus && !draw.least) {
        sample_from_tiles(a, r, row, draw, weight, s);
        return;
    }

    // the list of the logits above a bound that is below the threshold
    double sum = nucleus ? sample_tile_sum(a, r, weight) : 0;
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    const float max = sample_logit(max_key), range = max - sample_logit(low);
    const bool by_rank = draw.k || nucleus;
    int bound = 0;
    const float step = range > 0.f ? (kSampleBins - 1) / range : 0.f;
    auto bin = [&](uint32_t k) -> int { return (int)fminf((max - sample_logit(k)) * step, (float)(kSampleBins - 1)); };
    auto above = [&](uint32_t k) -> bool { return k > kNoLogit && (by_rank ? bin(k) <= bound : weight(k) >= draw.least); };
    bool listed = !by_rank || (range < 3e38f && step < 3e38f && draw.k <= groups);  // (uniform)
    if (listed) {
        if (by_rank) {
            sample_clear(s);
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (most[e] > kNoLogit) atomicAdd(&s.hist[bin(most[e])], 1ull);
            __syncthreads();
            u64 unused;
            bound = sample_bin((double)(draw.k ? draw.k : 256), 0, s, unused);
        }
        if (tid == 0) s.count = 0;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (above(most[e])) s.groups[atomicAdd(&s.count, 1)] = (uint16_t)(tid + e * kSampleThreads);
        __syncthreads();
        const int picked = s.count;
        __syncthreads();
        if (tid == 0) s.count = 0;
        __syncthreads();
        for (int e = tid; e < picked * GL; e += kSampleThreads) {
            const int i = s.groups[e / GL] * kSampleGroup + e % GL * VEC;
            uint32_t x[VEC];
            sample_keys(row, i, n, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (above(x[j])) sample_append(s, x[j], i + j);  // (past the row's end: kNoLogit)
        }
        __syncthreads();
        const int count = s.count;
        // (fewer groups than k: a logit below all of them may be among the first k)
        if (picked >= draw.k && count <= kSampleList && sample_from_list(a, r, draw, weight, count, sum, s)) return;
        __syncthreads();
    }
    SampleKept kept{0, n};
    if (draw.k)
        kept = sample_first_k(row, n, weight, draw.k, draw.p, s);
    else if (nucleus)
        kept = sample_nucleus(row, n, weight, draw.t, fmax((double)draw.p * sum, 0.5), s);
    sample_from_row(a, r, row, draw, kept, weight, s);
}

inline hipError_t launch_sample_kernels(const SampleArgs &a, hipStream_t s)
{
    if (a.n_rows <= 0) return hipSuccess;
    const unsigned tiles = (a.n_vocab + kSampleTile - 1) / kSampleTile;
    if (a.bf16) {
        sample_scan_kernel<uint16_t><<<dim3(a.n_rows * tiles), dim3(256), 0, s>>>(a);
        sample_row_kernel<uint16_t><<<dim3(a.n_rows), dim3(kSampleThreads), 0, s>>>(a);
    } else {
        sample_scan_kernel<float><<<dim3(a.n_rows * tiles), dim3(256), 0, s>>>(a);
        sample_row_kernel<float><<<dim3(a.n_rows), dim3(kSampleThreads), 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace fka
