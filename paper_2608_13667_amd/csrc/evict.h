// The attention weight of each prefix key, and the prefix shortened to its heaviest keys.
//
// key_weights: w[g][j] = decay w[g][j] + sum over the query rows r of KV head g of exp(scale q_r . k_j - lse_r),
// lse_r being the row's log-sum-exp over all its keys (a decode's or prefill's out_lse): the softmax weights,
// summed.  Bound by the read of K where the rows are few, by the products and exponentials where they are many.
//
// evict: of the positions [0, len) of each KV head, the first n_first and the last n_last, and of those between
// the ones with the largest weights (equal ones: the lowest positions), `keep` in all; their K and V rows and
// weights are copied in order.  The threshold is found digit by digit (11, 11 and 10 bits of an order-preserving
// integer of the weight) from histograms, so the choice is exact and does not depend on the order of the atomics;
// a kept position's place is the count of kept ones in front of it.
#pragma once

#include "internal.h"
#include "mx_attend.h"
#include "scan64.h"

namespace fka {

// Both kernels hold 64 keys per wave as the products' A operands (keys on M), so a lane sums its rows' weights of 16 keys over all
// row tiles, and the 16 lanes of a key are summed once at the end; query rows (N) are read from LDS, for all waves of a block.
constexpr int kWeightsKeys = 64;   // keys of a wave
// Query rows of a KV head that the few-rows kernel holds in LDS.  8 heads of 128, 128k keys: 32 rows 44.0 us and 50.7 by the kernel for many,
// 32k keys 14.4 and 15.8; 8192 keys of 2 heads 5.7 and 5.7.  With room for 48 rows (another block's LDS still fits), 40 rows over 128k
// keys 45.2 us and 50.6, 32k 15.5 and 15.7, 8192 of 2 heads 6.5 and 5.6: not taken so far.
constexpr int kWeightsFew = 32;

// 1 / log of the exponentials' base in the rows' -lse; -inf: a row past the end or without keys, weight 0.
__device__ inline float weights_offset(float lse) { return lse != -INFINITY ? -lse * 1.44269504088896341f : -INFINITY; }

// Row r (of a KV head's n_rows) in q and lse.
__device__ inline size_t weights_row(const WeightsArgs &a, int head, int32_t r)
{
    const int32_t seq = r / a.by_group;
    return (size_t)seq * a.n_q_heads + head * a.group + (r - seq * a.group);
}

// The weights of one 16-row tile, in LDS chunk order c ^ row mod CPR, added to the lane's sums.
template <int HD>
__device__ __attribute__((always_inline)) inline void weights_tile(const uint4 *qs, float nl, int r, int q4, const mx_bf16x8 (&kb)[4][HD / 32],
                                                                   float scale_log2, float (&w)[4][4])
{
    constexpr int NC = HD / 32, CPR = HD / 8;
    mx_f32x4 s[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) s[u] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
    // the four key tiles' chains side by side: a product of a chain waits for the one before
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const mx_bf16x8 qb = __builtin_bit_cast(mx_bf16x8, qs[r * CPR + ((4 * c + q4) ^ (r & (CPR - 1)))]);
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] = mx_mfma(kb[u][c], qb, s[u]);
    }
    mx_result_wait();
    const bool live = nl != -INFINITY;
    if (__builtin_amdgcn_ballot_w64(!live) == 0) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[u][i] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], scale_log2, nl));
    } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], scale_log2, nl));
                w[u][i] += live ? p : 0.f;
            }
    }
}

// The key of a wave's 64 whose sum lane (l16, q4) ends up with.
__device__ inline int weights_key(int l16, int q4) { return 16 * (l16 >> 2) + 4 * q4 + (l16 & 3); }

// The weight this lane will update, requested ahead (0 where it is not read: decay 0, or no such key).
__device__ __attribute__((always_inline)) inline float weights_old(const WeightsArgs &a, int head, int key)
{
    return a.decay != 0.f && key < a.len ? a.weights[(size_t)head * a.w_cap + key] : 0.f;
}

// The sums over the 16 lanes of each key, one to a lane (weights_key).  Four exchanges, each of which halves the values a lane holds (with
// lane ^ 15, ^ 7, ^ 3, ^ 1: DPP mirrors), leave one sum to each lane, so that the weights are read and written in one piece.
__device__ __attribute__((always_inline)) inline float weights_sum(int l16, const float (&w)[4][4])
{
    auto partner = [](float v, auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = w[i / 4][i % 4];
    auto halve = [&](auto N, auto ctrl) {  // of the first 2 N values, by this lane's bit N
        constexpr int n = decltype(N)::value;
        const bool up = (l16 & n) != 0;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float keep = up ? x[n + i] : x[i], send = up ? x[i] : x[n + i];
            x[i] = keep + partner(send, ctrl);
        }
    };
    halve(std::integral_constant<int, 8>{}, std::integral_constant<int, 0x140>{});  // row_mirror
    halve(std::integral_constant<int, 4>{}, std::integral_constant<int, 0x141>{});  // row_half_mirror
    halve(std::integral_constant<int, 2>{}, std::integral_constant<int, 0x1b>{});   // quad_perm 3,2,1,0
    halve(std::integral_constant<int, 1>{}, std::integral_constant<int, 0xb1>{});   // quad_perm 1,0,3,2
    return x[0];
}

__device__ __attribute__((always_inline)) inline void weights_store(const WeightsArgs &a, int head, int key, float sum, float old)
{
    if (key < a.len) a.weights[(size_t)head * a.w_cap + key] = a.decay == 0.f ? sum : __builtin_fmaf(a.decay, old, sum);
}

// A wave's 64 keys from key0 on; keys at or past len read as zeros.
template <int HD>
__device__ __attribute__((always_inline)) inline void weights_keys(const WeightsArgs &a, int head, int key0, int l16, int q4,
                                                                   mx_bf16x8 (&kb)[4][HD / 32])
{
    const int n = min(max(a.len - key0, 0), kWeightsKeys);
    const __amdgpu_buffer_rsrc_t rs = mx_rsrc(a.k + ((size_t)head * a.k_cap + (n > 0 ? key0 : 0)) * HD, n * HD * 2);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int c = 0; c < HD / 32; ++c)
            kb[u][c] = __builtin_bit_cast(
                mx_bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, (16 * u + l16) * HD * 2 + 64 * c + 16 * q4, 0, 2));
}

// Few query rows (n_rows <= kWeightsFew): bound by the read of K.  grid (blocks per head, Hkv): the rows pass into LDS once, and
// each wave takes every gridDim 4-th group of 64 keys, the next one loading meanwhile.  A load instruction reads 1 KiB in one
// piece, and the keys pass through the wave's own LDS into the operands' layout: read there directly, 64 bytes of each of 16 rows at
// a time, K came at 3.8 TB/s (one row over 128k keys of 8 heads of 128, 269 MB: 72 us; this way 42.6, 6.5 TB/s).  25 rows over
// 32k keys 14.7 us.
template <int HD>
__global__ __launch_bounds__(256, 2) void key_weights_few_kernel(WeightsArgs a)
{
    constexpr int CPR = HD / 8, KL = kWeightsKeys * CPR / 64;
    __shared__ uint4 qs[kWeightsFew * CPR];
    __shared__ float nls[kWeightsFew];
    __shared__ uint4 ks[4][kWeightsKeys * CPR];  // chunk c of row r at r CPR + (c ^ r mod CPR), as the query rows
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, q4 = lane >> 4, head = blockIdx.y;
    const int n_rows = (int)a.n_rows, tiles = (n_rows + 15) / 16;
    const int step = gridDim.x * 4 * kWeightsKeys;
    int key0 = (blockIdx.x * 4 + wave) * kWeightsKeys;
    uint4 kr[KL];
    float old_next;
    auto load = [&](int key) {  // keys at or past len read as zeros
        old_next = weights_old(a, head, key + weights_key(l16, q4));  // (read behind the group, it waited for the keys behind it)
        const int n = min(max(a.len - key, 0), kWeightsKeys);
        const __amdgpu_buffer_rsrc_t rs = mx_rsrc(a.k + ((size_t)head * a.k_cap + (n > 0 ? key : 0)) * HD, n * HD * 2);
#pragma unroll
        for (int i = 0; i < KL; ++i) kr[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, (64 * i + lane) * 16, 0, 2));
    };
    load(key0);
    for (int i = tid; i < 16 * tiles * CPR; i += 256) {
        const int r = i / CPR, c = i % CPR;
        qs[r * CPR + (c ^ (r & (CPR - 1)))] =
            r < n_rows ? *reinterpret_cast<const uint4 *>(a.q + weights_row(a, head, r) * HD + 8 * c) : uint4{0, 0, 0, 0};
    }
    if (tid < 16 * tiles) nls[tid] = tid < n_rows ? weights_offset(a.lse[weights_row(a, head, tid)]) : -INFINITY;
    __syncthreads();
    for (; key0 < a.len; key0 += step) {
#pragma unroll
        for (int i = 0; i < KL; ++i) {
            const int r = (64 * i + lane) / CPR, c = lane % CPR;
            ks[wave][r * CPR + (c ^ (r & (CPR - 1)))] = kr[i];
        }
        const float old = old_next;
        load(min(key0 + step, a.len));
        mx_bf16x8 kb[4][HD / 32];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int c = 0; c < HD / 32; ++c)
                kb[u][c] = __builtin_bit_cast(mx_bf16x8, ks[wave][(16 * u + l16) * CPR + ((4 * c + q4) ^ (l16 & (CPR - 1)))]);
        float w[4][4] = {};
        for (int t = 0; t < tiles; ++t) weights_tile<HD>(qs, nls[16 * t + l16], 16 * t + l16, q4, kb, a.scale_log2, w);
        weights_store(a, head, key0 + weights_key(l16, q4), weights_sum(l16, w), old);
    }
}

typedef __attribute__((address_space(3))) void weights_lds;
typedef const __attribute__((address_space(1))) void weights_global;

// 16 bytes per lane from global memory into LDS at dst + 16 lane, past the registers.
__device__ inline void weights_dma16(const void *src, void *dst)
{
    __builtin_amdgcn_global_load_lds((weights_global *)src, (weights_lds *)dst, 16, 0, 0);
}

// Many query rows: bound by the products and the exponentials, which three waves of a SIMD overlap (one wave that computes a
// tile's exponentials beside the next one's products, at two waves a SIMD, was slower: 190 us against 168).  The rows pass
// through LDS 64 at a time, the next ones on their way meanwhile: 512 rows over 128k keys x 8 heads 165 us (832 TF/s; by way of
// registers, 32 at a time, 176; read from L2 by each wave 289).  grid (ceil(len / 256), Hkv); SPLIT, for few keys:
// (ceil(len / 64), Hkv), where the four waves of a block have the same 64 keys and every fourth 16-row tile each, joined at the end.
template <int HD, bool SPLIT>
__global__ __launch_bounds__(256, 3) void key_weights_kernel(WeightsArgs a)
{
    constexpr int CPR = HD / 8, QR = 64, QL = QR * CPR / 256;
    __shared__ uint4 qs[2][QR * CPR];  // chunk c of row r at r CPR + (c ^ r mod CPR): a read of 16 rows touches every bank
    __shared__ float nls[2][QR];
    __shared__ float part[SPLIT ? 4 : 1][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, q4 = lane >> 4, head = blockIdx.y;
    const int key0 = (SPLIT ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave) * kWeightsKeys;
    float nl_next = 0.f;
    auto fetch = [&](int64_t r0, int buf) {
#pragma unroll
        for (int i = 0; i < QL; ++i) {
            const int r = (tid + 256 * i) / CPR, c = tid % CPR;
            const int64_t row = min(r0 + r, a.n_rows - 1);  // (rows past the end have weight 0)
            weights_dma16(a.q + weights_row(a, head, (int32_t)row) * HD + (c ^ (r & (CPR - 1))) * 8, &qs[buf][256 * i + 64 * wave]);
        }
        nl_next = -INFINITY;
        if (tid < QR && r0 + tid < a.n_rows) nl_next = weights_offset(a.lse[weights_row(a, head, (int32_t)(r0 + tid))]);
    };
    auto put = [&](int buf) {
        if (tid < QR) nls[buf][tid] = nl_next;
        __builtin_amdgcn_s_waitcnt(0xf70);  // vmcnt(0): this wave's rows are in LDS
    };
    float w[4][4] = {};
    fetch(0, 0);
    mx_bf16x8 kb[4][HD / 32];
    weights_keys<HD>(a, head, key0, l16, q4, kb);
    const int key = key0 + weights_key(l16, q4);
    const float old = weights_old(a, head, key);
    put(0);
    __syncthreads();
    for (int64_t r0 = 0; r0 < a.n_rows; r0 += QR) {
        const int buf = (int)(r0 / QR) & 1;
        if (r0 + QR < a.n_rows) fetch(r0 + QR, buf ^ 1);  // whose readers are a barrier behind
        if constexpr (SPLIT) {
            weights_tile<HD>(qs[buf], nls[buf][16 * wave + l16], 16 * wave + l16, q4, kb, a.scale_log2, w);
        } else {
#pragma unroll
            for (int t = 0; t < QR / 16; ++t)
                weights_tile<HD>(qs[buf], nls[buf][16 * t + l16], 16 * t + l16, q4, kb, a.scale_log2, w);
        }
        if (r0 + QR < a.n_rows) put(buf ^ 1);
        __syncthreads();
    }
    float sum = weights_sum(l16, w);
    if constexpr (SPLIT) {
        part[wave][lane] = sum;
        __syncthreads();
        if (wave > 0) return;
        sum = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    }
    weights_store(a, head, key, sum, old);
}

// An integer in the order of the weights: -0 is 0, a NaN is above all.
__device__ inline uint32_t evict_key(float w)
{
    uint32_t b = __float_as_uint(w);
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    if (b == 0x80000000u) b = 0;
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__device__ inline int evict_shift(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }
__device__ inline uint32_t evict_mask(int digit) { return digit == 2 ? 1023u : 2047u; }

constexpr int kEvictThreads = 1024;

struct EvictLds {
    uint32_t bins[kEvictBins];
    int32_t wave[kEvictThreads / 64];
    int32_t bin, want;
    int32_t sums[3];
    uint32_t ranks[16 * kEvictThreads / 64];  // per (load, wave): keys above the threshold << 16, keys at it
};

// The bin that holds the want-th largest key: thread t has the counts of bins 2047 - 2 t and 2046 - 2 t.
// want goes on among the keys of that bin.
__device__ inline void evict_find(EvictLds &l, int c0, int c1, int &bin, int &want)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int sum = scan64(c0 + c1);
    if (lane == 63) l.wave[wave] = sum;
    __syncthreads();
    int before = sum - c0 - c1;
    for (int w = 0; w < kEvictThreads / 64; ++w) before += w < wave ? l.wave[w] : 0;
    if (before < want && want <= before + c0) {
        l.bin = kEvictBins - 1 - 2 * tid;
        l.want = want - before;
    } else if (before + c0 < want && want <= before + c0 + c1) {
        l.bin = kEvictBins - 2 - 2 * tid;
        l.want = want - before - c0;
    }
    __syncthreads();
    bin = l.bin;
    want = l.want;
}

// The histogram of a digit among this block's keys that share the digits before it (key), in LDS.  Keys out of the
// choice are 0 with `in` unset.
template <int E>
__device__ inline void evict_hist(EvictLds &l, const uint32_t (&k)[E], uint32_t in, int digit, uint32_t key)
{
    const int tid = threadIdx.x;
    l.bins[2 * tid] = l.bins[2 * tid + 1] = 0;
    __syncthreads();
    const int above = digit == 0 ? 31 : evict_shift(digit - 1);  // the digits before it start here
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if (!(in >> i & 1) || (digit != 0 && (k[i] >> above) != (key >> above))) continue;
        const uint32_t bin = (k[i] >> evict_shift(digit)) & evict_mask(digit);
        // one bin's lanes together: many equal keys (a fresh cache's zeros) would follow one another on its address
        // (8192 equal ones 31 us, 13 so)
        const bool first = bin == (uint32_t)__builtin_amdgcn_readfirstlane((int)bin);
        const uint64_t same = __builtin_amdgcn_ballot_w64(first);
        if (!first || (tid & 63) == __builtin_ctzll(same)) atomicAdd(&l.bins[bin], first ? (uint32_t)__builtin_popcountll(same) : 1u);
    }
    __syncthreads();
}

// The block's keys: position p0 + i 1024 + tid; returns which lie between the first n_first and the last n_last.
template <int E>
__device__ inline uint32_t evict_load(const EvictArgs &a, int head, int p0, uint32_t (&k)[E])
{
    const float *w = a.weights + (size_t)head * a.w_cap;
    float x[E];
    uint32_t in = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int p = p0 + i * kEvictThreads + (int)threadIdx.x;
        const bool mid = p >= a.n_first && p < a.len - a.n_last;
        x[i] = mid ? w[p] : 0.f;
        in |= mid ? 1u << i : 0u;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) k[i] = evict_key(x[i]);
    return in;
}

// The block's kept positions to their places in the index.  above0 and at0: keys above the threshold `key` and at it in the
// blocks in front; of those at it the first `want` are kept (want = 0: none, and none above).
template <int E>
__device__ inline void evict_write(EvictLds &l, const EvictArgs &a, int head, int p0, const uint32_t (&k)[E], uint32_t in, uint32_t key,
                                   int want, int above0, int at0)
{
    constexpr int NW = kEvictThreads / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint64_t above[E], at[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const bool mid = (in >> i & 1) && want > 0;
        above[i] = __builtin_amdgcn_ballot_w64(mid && k[i] > key);
        at[i] = __builtin_amdgcn_ballot_w64(mid && k[i] == key);
        if (lane == 0) l.ranks[i * NW + wave] = (uint32_t)__builtin_popcountll(above[i]) << 16 | (uint32_t)__builtin_popcountll(at[i]);
    }
    __syncthreads();
    // exclusive sums in the order of the positions, by the first wave
    if (wave == 0) {
        constexpr int PER = E * NW / 64;
        uint32_t c[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            c[i] = l.ranks[lane * PER + i];
            sum += c[i];
        }
        uint32_t run = (uint32_t)scan64((int)sum) - sum;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            l.ranks[lane * PER + i] = run;
            run += c[i];
        }
    }
    __syncthreads();
    const uint64_t below = lane == 0 ? 0 : ~0ull >> (64 - lane);
    int32_t *index = a.index + (size_t)head * a.keep;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int p = p0 + i * kEvictThreads + tid;
        if (p >= a.len) continue;
        const uint32_t r = l.ranks[i * NW + wave];
        const int ab = above0 + (int)(r >> 16) + __builtin_popcountll(above[i] & below);
        const int eq = at0 + (int)(r & 0xffff) + __builtin_popcountll(at[i] & below);
        int out = -1;
        if (p < a.n_first)
            out = p;
        else if (p >= a.len - a.n_last)
            out = a.keep - (a.len - p);
        else if ((above[i] >> lane & 1) || ((at[i] >> lane & 1) && eq < want))
            out = a.n_first + ab + min(eq, want);
        if (out >= 0 && out < a.keep) index[out] = p;
    }
}

// grid (Hkv): a head's positions all in one block's registers (len <= 1024 E).
template <int E>
__global__ __launch_bounds__(kEvictThreads) void evict_one_kernel(EvictArgs a)
{
    __shared__ EvictLds l;
    const int head = blockIdx.x, tid = threadIdx.x;
    uint32_t k[E], key = 0;
    const uint32_t in = evict_load<E>(a, head, 0, k);
    int want = a.keep - a.n_first - a.n_last;
    if (want > 0)
        for (int d = 0; d < 3; ++d) {
            int bin;
            evict_hist<E>(l, k, in, d, key);
            evict_find(l, l.bins[kEvictBins - 1 - 2 * tid], l.bins[kEvictBins - 2 - 2 * tid], bin, want);
            key |= (uint32_t)bin << evict_shift(d);
            __syncthreads();
        }
    evict_write<E>(l, a, head, 0, k, in, key, want, 0, 0);
}

// Longer prefixes: a kernel per digit, grid (chunks, Hkv).  Each leaves its chunk's histogram; the next finds
// the digit in their sum, and what the chunk has above it.
//
// The sums over the chunks of this thread's two bins of a digit: all, this chunk's own and those in front.
__device__ inline void evict_sum(const EvictArgs &a, int head, int digit, int (&all)[2], int (&own)[2], int (&front)[2])
{
    const uint2 *h = reinterpret_cast<const uint2 *>(a.hist) +
                     ((size_t)digit * a.n_kv_heads + head) * a.chunks * (kEvictBins / 2) + (kEvictBins / 2 - 1 - threadIdx.x);
    all[0] = all[1] = own[0] = own[1] = front[0] = front[1] = 0;
#pragma unroll 16
    for (int c = 0; c < a.chunks; ++c) {
        const uint2 v = h[(size_t)c * (kEvictBins / 2)];  // the higher bin is y
        all[0] += v.y;
        all[1] += v.x;
        if (c < (int)blockIdx.x) front[0] += v.y, front[1] += v.x;
        if (c == (int)blockIdx.x) own[0] = v.y, own[1] = v.x;
    }
}

// Adds x over the block into l.sums[i] (cleared before, read behind a barrier).
__device__ inline void evict_add(EvictLds &l, int i, int x)
{
    const int s = scan64(x);
    if ((threadIdx.x & 63) == 63 && s) atomicAdd(&l.sums[i], s);
}

// Digit DIGIT's histogram; behind the first, the digit before it is found first.
template <int E, int DIGIT>
__global__ __launch_bounds__(kEvictThreads) void evict_hist_kernel(EvictArgs a)
{
    __shared__ EvictLds l;
    const int tid = threadIdx.x, head = blockIdx.y, chunk = blockIdx.x;
    const int per = a.chunk_blocks;  // groups of 1024 E positions to a chunk
    uint32_t key = 0, k[E];
    uint32_t in = evict_load<E>(a, head, chunk * per * E * kEvictThreads, k);
    if constexpr (DIGIT > 0) {
        int want = a.keep - a.n_first - a.n_last, bin, all[2], own[2], front[2];
        int32_t *state = a.state + (size_t)head * 4;
        if (DIGIT > 1) {
            key = state[0];
            want = state[1];
        }
        if (tid < 3) l.sums[tid] = 0;
        evict_sum(a, head, DIGIT - 1, all, own, front);
        evict_find(l, all[0], all[1], bin, want);
        key |= (uint32_t)bin << evict_shift(DIGIT - 1);
        // each digit's state in a place of its own: other blocks may still read the one before
        if (chunk == 0 && tid == 0) {
            state[2 * (DIGIT - 1)] = (int32_t)key;
            state[2 * (DIGIT - 1) + 1] = want;
        }
        const int b0 = kEvictBins - 1 - 2 * tid;
        evict_add(l, 0, (b0 > bin ? own[0] : 0) + (b0 - 1 > bin ? own[1] : 0));
        __syncthreads();
        if (tid == 0) a.counts[((size_t)head * a.chunks + chunk) * 2 + DIGIT - 1] = l.sums[0];
    }
    uint32_t mine[2] = {0, 0};
    for (int g = 0;;) {
        evict_hist<E>(l, k, in, DIGIT, key);
        mine[0] += l.bins[2 * tid];
        mine[1] += l.bins[2 * tid + 1];
        if (++g == per) break;
        in = evict_load<E>(a, head, (chunk * per + g) * E * kEvictThreads, k);
        __syncthreads();
    }
    reinterpret_cast<uint2 *>(a.hist)[(((size_t)DIGIT * a.n_kv_heads + head) * a.chunks + chunk) * (kEvictBins / 2) + tid] =
        uint2{mine[0], mine[1]};
}

// The last digit, the chunk's place among the kept, and its part of the index.
template <int E>
__global__ __launch_bounds__(kEvictThreads) void evict_index_kernel(EvictArgs a)
{
    __shared__ EvictLds l;
    const int tid = threadIdx.x, head = blockIdx.y, chunk = blockIdx.x;
    const int per = a.chunk_blocks;
    uint32_t k[E], key = 0;
    uint32_t in = evict_load<E>(a, head, chunk * per * E * kEvictThreads, k);
    int want = a.keep - a.n_first - a.n_last, above0 = 0, at0 = 0;
    if (want > 0) {
        int bin, all[2], own[2], front[2];
        const int32_t *state = a.state + (size_t)head * 4;
        key = state[2];
        want = state[3];
        if (tid < 3) l.sums[tid] = 0;
        evict_sum(a, head, 2, all, own, front);
        evict_find(l, all[0], all[1], bin, want);
        key |= (uint32_t)bin;
        const int b0 = kEvictBins - 1 - 2 * tid;
        int above = (b0 > bin ? front[0] : 0) + (b0 - 1 > bin ? front[1] : 0);
        for (int c = tid; c < 2 * chunk; c += kEvictThreads) above += a.counts[(size_t)head * a.chunks * 2 + c];
        evict_add(l, 0, above);
        evict_add(l, 1, (b0 == bin ? front[0] : 0) + (b0 - 1 == bin ? front[1] : 0));
        __syncthreads();
        above0 = l.sums[0];
        at0 = l.sums[1];
    }
    for (int g = 0;;) {
        const int p0 = (chunk * per + g) * E * kEvictThreads;
        evict_write<E>(l, a, head, p0, k, in, key, want, above0, at0);
        if (++g == per) break;
        // the group's own keys above the threshold and at it, for the next group
        int above = 0, at = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            above += (in >> i & 1) && want > 0 && k[i] > key;
            at += (in >> i & 1) && want > 0 && k[i] == key;
        }
        __syncthreads();
        if (tid < 3) l.sums[tid] = 0;
        __syncthreads();
        evict_add(l, 0, above);
        evict_add(l, 1, at);
        in = evict_load<E>(a, head, p0 + E * kEvictThreads, k);
        __syncthreads();
        above0 += l.sums[0];
        at0 += l.sums[1];
    }
}

// grid (ceil(keep / rows per block), Hkv): the kept rows and weights.
__global__ __launch_bounds__(256) void evict_gather_kernel(EvictArgs a)
{
    const int cpr = a.head_dim / 8, per = 256 / cpr * 4, head = blockIdx.y;
    const int c = threadIdx.x % cpr;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int i = blockIdx.x * per + u * (256 / cpr) + threadIdx.x / cpr;
        if (i >= a.keep) continue;
        const size_t out = (size_t)head * a.keep + i;
        const int p = min(max(a.index[out], 0), a.len - 1);  // (weights that another stream changes meanwhile leave gaps)
        const size_t src = ((size_t)head * a.kv_cap + p) * cpr + c;
        reinterpret_cast<uint4 *>(a.k_out)[out * cpr + c] = reinterpret_cast<const uint4 *>(a.k)[src];
        reinterpret_cast<uint4 *>(a.v_out)[out * cpr + c] = reinterpret_cast<const uint4 *>(a.v)[src];
        if (a.weights_out && c == 0) a.weights_out[out] = a.weights[(size_t)head * a.w_cap + p];
    }
}

inline hipError_t launch_key_weights_kernel(const WeightsArgs &a, int head_dim, hipStream_t s)
{
    if (a.len <= 0) return hipSuccess;
    if (head_dim != 64 && head_dim != 128) return hipErrorInvalidValue;
    const int groups = (a.len + 4 * kWeightsKeys - 1) / (4 * kWeightsKeys);  // of a block's keys
    if (a.n_rows <= kWeightsFew) {
        // two blocks on each of 256 compute units
        const int per_head = (512 + a.n_kv_heads - 1) / a.n_kv_heads;
        const dim3 grid(groups < per_head ? groups : per_head, a.n_kv_heads);
        head_dim == 128 ? key_weights_few_kernel<128><<<grid, dim3(256), 0, s>>>(a) : key_weights_few_kernel<64><<<grid, dim3(256), 0, s>>>(a);
    } else {
        // fewer blocks than CUs leave CUs idle: 512 rows, 4096 keys x 2 heads 20.9 us whole and 10.4 split, x 8 heads 22.3 and
        // 14.1; 8192 x 8, as many blocks as CUs, 22.6 and 25.7
        const bool split = (int64_t)groups * a.n_kv_heads < 256;
        const dim3 grid(split ? (a.len + kWeightsKeys - 1) / kWeightsKeys : groups, a.n_kv_heads), block(256);
        if (head_dim == 128)
            split ? key_weights_kernel<128, true><<<grid, block, 0, s>>>(a) : key_weights_kernel<128, false><<<grid, block, 0, s>>>(a);
        else
            split ? key_weights_kernel<64, true><<<grid, block, 0, s>>>(a) : key_weights_kernel<64, false><<<grid, block, 0, s>>>(a);
    }
    return hipGetLastError();
}

inline hipError_t launch_evict_kernels(const EvictArgs &a, hipStream_t s)
{
    if (a.keep <= 0) return hipSuccess;
    const dim3 block(kEvictThreads), chunks(a.chunks, a.n_kv_heads), heads(a.n_kv_heads);
    // one block's registers (1024 threads) or a kernel per digit, 8 heads, with 256 rows' copies: 8192 positions 13.3 and 22.1 us,
    // 16384 at 16 a thread 19.5 and 23.6, 32768 at 32 a thread 31.3 and 25.7
    if (a.len <= 8 * kEvictThreads) {
        evict_one_kernel<8><<<heads, block, 0, s>>>(a);
    } else if (a.len <= 16 * kEvictThreads) {
        evict_one_kernel<16><<<heads, block, 0, s>>>(a);
    } else {
        if (a.keep > a.n_first + a.n_last) {
            evict_hist_kernel<8, 0><<<chunks, block, 0, s>>>(a);
            evict_hist_kernel<8, 1><<<chunks, block, 0, s>>>(a);
            evict_hist_kernel<8, 2><<<chunks, block, 0, s>>>(a);
        }
        evict_index_kernel<8><<<chunks, block, 0, s>>>(a);
    }
    const int per = 256 / (a.head_dim / 8) * 4;
    evict_gather_kernel<<<dim3((a.keep + per - 1) / per, a.n_kv_heads), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace fka
