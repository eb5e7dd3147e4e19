// The token that a row of logits gives for a random number, behind temperature, top-k, top-p and min-p.
//
// With M the row's largest logit and t its temperature, logit l_i has the weight w_i = round(2^44 exp((l_i - M) / t)), a whole number:
// sums of them do not depend on their order, so a row's token is the same in every run however the work is shared.
// (2^18 weights of at most 2^44 stay within 64 bits; what rounds to 0 has less than 2^-45 of the largest weight.)  In the order of
// falling logits, equal ones by place, a filter keeps the first logits: top-k the first k, top-p, of these, those with less
// than p of their sum in front of them.  So what is kept is one logit value, the threshold, and a place: everything above the value,
// and of its equals those up to the place.  min-p is a bound on w itself.
// The threshold is found digit by digit of the logit's bits (11, 11, 10 from the top, as unsigned numbers in the logits' order): a
// histogram of the counts, or of the weights, of a digit's values among what agrees in the digits before.
//
// One block takes a row.
#pragma once

#include "internal.h"

namespace fka {

constexpr int kSampleThreads = 1024;
constexpr int kSampleBins = 2048;
constexpr double kSampleUnit = 17592186044416.0;  // 2^44
constexpr uint32_t kNoLogit = 0x007fffffu;        // the key of -inf (NaN counts as that)

typedef unsigned long long u64;

// Bits in the order of the logits; -0 equals 0.
__device__ inline uint32_t sample_key(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return x == x ? u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u) : kNoLogit;
}
__device__ inline float sample_logit(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// exp(x) in 64 bits as 2^(n / 64) times the series of the rest, |rest| <= ln 2 / 128: its next term is 4e-17 of the result.
struct SampleWeight {
    const double *table;  // 2^(j / 64), LDS
    double max, step;     // M, 64 / (t ln 2)
    uint32_t max_key;

    __device__ inline u64 operator()(uint32_t key) const
    {
        if (key == max_key) return (u64)kSampleUnit;
        const double z = ((double)sample_logit(key) - max) * step;
        if (!(z > -64.0 * 46) || key == kNoLogit) return 0;  // (also infinities: -inf, or all but those of an infinite M)
        const double n = rint(z), r = (z - n) * (0.69314718055994530942 / 64);
        const int m = (int)n;
        double p = __builtin_fma(r, 1.0 / 120, 1.0 / 24);
        p = __builtin_fma(r, p, 1.0 / 6);
        p = __builtin_fma(r, p, 0.5);
        p = __builtin_fma(r, p, 1.0);
        p = __builtin_fma(r, p, 1.0);
        // 2^52 added rounds to a whole number in the lowest bits
        const double w = ldexp(table[m & 63] * p, (m >> 6) + 44) + 4503599627370496.0;
        return (u64)__double_as_longlong(w) & 0xfffffffffffffull;
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

struct SampleShared {
    double table[64];
    u64 hist[kSampleBins];
    u64 part[kSampleThreads / 64];
    u64 tile[64];
    u64 result[4];
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
    for (int i = 0; i < kSampleThreads / 64; ++i) {
        if (i == wave) before = total;
        total += s.part[i];
    }
    return before + y - x;
}

// The filters' threshold so far: kept are the keys above `key` and those equal to it at places up to `last`.
struct SampleKept {
    uint32_t key;
    int last;
    __device__ inline bool operator()(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

// The last group of equal keys, among those that `kept` keeps, with less than `limit` in front of it (counts, or the sum of
// weights), and how much that is.
template <bool MASS, class T>
__device__ inline void sample_select(const T *row, int n, const SampleKept &kept, const SampleWeight &weight, double limit, SampleShared &s,
                                     uint32_t &key, u64 &before)
{
    constexpr int VEC = SampleRow<T>::VEC;
    uint32_t prefix = 0;
    u64 front = 0;
    for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
        __syncthreads();
        for (int i = threadIdx.x; i < kSampleBins; i += kSampleThreads) s.hist[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x * VEC; i < n; i += kSampleThreads * VEC) {
            uint32_t k[VEC];
            sample_keys(row, i, n, k);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (i + j >= n || !kept(k[j], i + j) || (digit && k[j] >> (shift + bits) != prefix)) continue;
                const u64 add = MASS ? weight(k[j]) : 1;
                if (add) atomicAdd(&s.hist[k[j] >> shift & ((1u << bits) - 1)], add);
            }
        }
        __syncthreads();
        // thread i has the bins 2047 - 2 i and the one below
        const int top = kSampleBins - 1 - 2 * (int)threadIdx.x;
        const u64 a = s.hist[top], b = s.hist[top - 1];
        u64 total;
        const u64 in_front = sample_scan(a + b, s, total) + front;
        // of the bins with something in them and less than the limit in front, the last: bins' fronts rise, so one
        // thread has it, the one whose next filled bin is past the limit
        if (threadIdx.x == 0) s.result[0] = 0;
        __syncthreads();
        u64 mine = 0;
        if (a && (double)in_front < limit) mine = (u64)threadIdx.x * 2 + 1;
        if (b && (double)(in_front + a) < limit) mine = (u64)threadIdx.x * 2 + 2;
        if (mine) atomicMax(&s.result[0], mine);
        __syncthreads();
        if (mine && s.result[0] == mine) s.result[1] = (mine & 1) ? in_front : in_front + a;
        __syncthreads();
        front = s.result[1];
        prefix = prefix << bits | (uint32_t)(kSampleBins - (int)s.result[0]);
    }
    key = prefix;
    before = front;
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

template <class T>
__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(SampleArgs a)
{
    constexpr int VEC = SampleRow<T>::VEC, TILE = kSampleThreads * VEC;
    __shared__ SampleShared s;
    const int r = blockIdx.x, n = a.n_vocab, tid = threadIdx.x;
    const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.stride;
    if (tid < 64) s.table[tid] = exp2((double)tid / 64);

    // the largest logit and its lowest place
    u64 best = 0;
    for (int i = tid * VEC; i < n; i += TILE) {
        uint32_t k[VEC];
        sample_keys(row, i, n, k);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const u64 x = (u64)k[j] << 32 | (uint32_t)~(i + j);
            best = x > best ? x : best;
        }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const u64 x = __shfl_xor(best, d);
        best = x > best ? x : best;
    }
    if ((tid & 63) == 0) s.part[tid >> 6] = best;
    __syncthreads();
    best = s.part[0];
#pragma unroll
    for (int i = 1; i < kSampleThreads / 64; ++i) best = s.part[i] > best ? s.part[i] : best;
    const uint32_t max_key = (uint32_t)(best >> 32);
    const float t = a.temperature ? a.temperature[r] : 1.f;
    if (max_key == kNoLogit || !(t > 0.f)) {
        if (tid == 0) {
            const bool none = max_key == kNoLogit;
            a.tokens[r] = none ? -1 : (int)~(uint32_t)best;
            if (a.logprob) a.logprob[r] = none ? -INFINITY : 0.f;
            if (none && a.err) atomicOr(a.err, kErrNoToken);
        }
        return;
    }
    const SampleWeight weight{s.table, (double)sample_logit(max_key), 64 * 1.4426950408889634074 / (double)t, max_key};

    SampleKept kept{0, n};
    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.f;
    if (k > 0 && k < n) {
        uint32_t key;
        u64 before;
        sample_select<false>(row, n, kept, weight, (double)k, s, key, before);
        kept.last = sample_place(row, n, key, (u64)k - before, s);
        kept.key = key;
    }
    if (p < 1.f) {
        // the sum of what is kept so far
        u64 sum = 0, total;
        for (int i = tid * VEC; i < n; i += TILE) {
            uint32_t x[VEC];
            sample_keys(row, i, n, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (i + j < n && kept(x[j], i + j)) sum += weight(x[j]);
        }
        sample_scan(sum, s, total);
        const double limit = fmax((double)p * (double)total, 0.5);  // the first is always kept
        uint32_t key;
        u64 before;
        sample_select<true>(row, n, kept, weight, limit, s, key, before);
        // of its equals those with less than the limit in front: one, and each further one
        const u64 w = weight(key);
        u64 more = 1;
        for (u64 step = (u64)1 << 18; step; step >>= 1)
            if ((double)(before + (more + step - 1) * w) < limit) more += step;
        const int last = sample_place(row, n, key, more, s);
        kept.last = key == kept.key ? min(kept.last, last) : last;
        kept.key = key;
    }
    const float min_p = a.min_p ? a.min_p[r] : 0.f;
    const u64 least = min_p > 0.f ? (u64)ceil(fmin((double)min_p, 1.0) * kSampleUnit) : 0;

    // the kept weights of each tile, then the tile, the thread and the place where the sum passes the mark
    const int tiles = (n + TILE - 1) / TILE;
    if (tid < 64) s.tile[tid] = 0;
    __syncthreads();
    auto kept_weight = [&](uint32_t key, int i) -> u64 {
        if (i >= n || !kept(key, i)) return 0;
        const u64 w = weight(key);
        return w >= least ? w : 0;
    };
    for (int tile = 0; tile < tiles; ++tile) {
        const int i = tile * TILE + tid * VEC;
        u64 sum = 0;
        if (i < n) {
            uint32_t x[VEC];
            sample_keys(row, i, n, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum += kept_weight(x[j], i + j);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        if ((tid & 63) == 0 && sum) atomicAdd(&s.tile[tile], sum);
    }
    __syncthreads();
    u64 total = 0;
    for (int i = 0; i < tiles; ++i) total += s.tile[i];
    const float u = a.u[r];
    const double at = floor((u > 0.f ? (double)u : 0.0) * (double)total);
    u64 mark = at < (double)total ? (u64)at : total - 1;  // (a double may be past the sum that it was made from)
    mark = mark < total ? mark : total - 1;
    int tile = 0;
    while (mark >= s.tile[tile]) mark -= s.tile[tile++];
    const int i = tile * TILE + tid * VEC;
    u64 w[VEC], sum = 0;
    {
        uint32_t x[VEC];
        sample_keys(row, i, n, x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) sum += w[j] = kept_weight(x[j], i + j);
    }
    u64 unused;
    u64 before = sample_scan(sum, s, unused);
    if (mark >= before && mark < before + sum) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if (mark >= before && mark < before + w[j]) {
                a.tokens[r] = i + j;
                if (a.logprob) a.logprob[r] = (float)log((double)w[j] / (double)total);
            }
            before += w[j];
        }
    }
}

inline hipError_t launch_sample_kernels(const SampleArgs &a, hipStream_t s)
{
    if (a.n_rows <= 0) return hipSuccess;
    if (a.bf16)
        sample_row_kernel<uint16_t><<<dim3(a.n_rows), dim3(kSampleThreads), 0, s>>>(a);
    else
        sample_row_kernel<float><<<dim3(a.n_rows), dim3(kSampleThreads), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace fka
