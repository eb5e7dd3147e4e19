// The attention weight of each prefix key, and the prefix shortened to its heaviest keys.
//
// key_weights: w[g][j] = decay w[g][j] + sum over the query rows r of KV head g of exp(scale q_r . k_j - lse_r),
// lse_r being the row's log-sum-exp over all its keys (a decode's or prefill's out_lse): the softmax weights,
// summed.  Bound by the read of K where the rows are few, by the products and exponentials where they are many.
//
// evict: of the positions [0, len) of each KV head, the first n_first and the last n_last, and of those between
// the ones with the largest weights (equal ones: the lowest positions), `keep` in all; their K and V rows and
// weights are copied in order.  The threshold is found digit by digit (11, 11 and 10 bits of an order-preserving
// integer of the weight) from histograms, so the choice is exact and does not depend on the order of the atomics.
#pragma once

#include "internal.h"
#include "mx_attend.h"

namespace fka {

// grid (ceil(len / 256), Hkv), four waves of 64 keys: K on M, query rows on N, so a lane sums its rows'
// weights of 16 keys over all row tiles and the 16 lanes of a key are summed once at the end.
template <int HD>
__global__ __launch_bounds__(256, 2) void key_weights_kernel(WeightsArgs a)
{
    constexpr int NC = HD / 32, KT = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, q4 = lane >> 4, head = blockIdx.y;
    const int key0 = (blockIdx.x * 4 + wave) * 16 * KT;
    if (key0 >= a.len) return;
    const uint16_t *k = a.k + ((size_t)head * a.k_cap + key0) * HD;
    mx_bf16x8 kb[KT][NC];
#pragma unroll
    for (int u = 0; u < KT; ++u)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            kb[u][c] = mx_bf16x8{};
            if (key0 + 16 * u + l16 < a.len)
                kb[u][c] = *reinterpret_cast<const mx_bf16x8 *>(k + (size_t)(16 * u + l16) * HD + 32 * c + 8 * q4);
        }
    float w[KT][4] = {};
    for (int64_t r0 = 0; r0 < a.n_rows; r0 += 16) {
        const int64_t r = r0 + l16;
        mx_bf16x8 qb[NC];
        float nl = -INFINITY;  // a row past the end, or one without keys: weight 0
#pragma unroll
        for (int c = 0; c < NC; ++c) qb[c] = mx_bf16x8{};
        if (r < a.n_rows) {
            const int64_t seq = (int32_t)r / a.by_group;
            const size_t row = (size_t)seq * a.n_q_heads + head * a.group + (r - seq * a.group);
#pragma unroll
            for (int c = 0; c < NC; ++c) qb[c] = *reinterpret_cast<const mx_bf16x8 *>(a.q + row * HD + 32 * c + 8 * q4);
            const float l = a.lse[row];
            if (l != -INFINITY) nl = -l * 1.44269504088896341f;
        }
        mx_f32x4 s[KT];
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            s[u] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NC; ++c) s[u] = mx_mfma(kb[u][c], qb[c], s[u]);
        }
        mx_result_wait();
        const bool live = nl != -INFINITY;
#pragma unroll
        for (int u = 0; u < KT; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], a.scale_log2, nl));
                w[u][i] += live ? p : 0.f;
            }
    }
    auto ror = [](float v, auto n) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + decltype(n)::value, 0xf, 0xf, false));
    };
#pragma unroll
    for (int u = 0; u < KT; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = w[u][i];
            x += ror(x, std::integral_constant<int, 8>{});
            x += ror(x, std::integral_constant<int, 4>{});
            x += ror(x, std::integral_constant<int, 2>{});
            x += ror(x, std::integral_constant<int, 1>{});
            const int key = key0 + 16 * u + 4 * q4 + i;
            if (l16 == 0 && key < a.len) {
                float *dst = a.weights + (size_t)head * a.w_cap + key;
                *dst = a.decay == 0.f ? x : __builtin_fmaf(a.decay, *dst, x);
            }
        }
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

// The threshold's first `digits` digits, from their histograms, by a block of 256 threads: the `want`-th largest key has
// the prefix `key` (in its place), and `want` counts on among those that share it.
__device__ inline void evict_threshold(const EvictArgs &a, int head, int digits, uint32_t &key, int &want)
{
    __shared__ int32_t s_sum[256], s_bin, s_want;
    key = 0;
    want = a.keep - a.n_first - a.n_last;
    const int tid = threadIdx.x;
    for (int d = 0; d < digits; ++d) {
        const uint32_t *h = a.hist + ((size_t)d * a.n_kv_heads + head) * kEvictBins;
        // thread t has bins [2048 - 8 (t + 1), 2048 - 8 t), from the top
        uint32_t c[8];
        int32_t sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c[i] = h[kEvictBins - 1 - 8 * tid - i];
            sum += c[i];
        }
        __syncthreads();
        s_sum[tid] = sum;
        if (tid == 0) s_bin = 0, s_want = 0;
        __syncthreads();
        for (int o = 1; o < 256; o *= 2) {
            const int32_t x = tid >= o ? s_sum[tid - o] : 0;
            __syncthreads();
            s_sum[tid] += x;
            __syncthreads();
        }
        int32_t before = s_sum[tid] - sum;  // keys above this thread's bins
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (before < want && want <= before + (int32_t)c[i]) {
                s_bin = kEvictBins - 1 - 8 * tid - i;
                s_want = want - before;
            }
            before += c[i];
        }
        __syncthreads();
        if (want == 0) {  // nothing to take: above every key
            key = 0xffffffffu;
            return;
        }
        key |= (uint32_t)s_bin << evict_shift(d);
        want = s_want;
    }
}

__global__ __launch_bounds__(256) void evict_clear_kernel(uint32_t *hist, int n)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) hist[i] = 0;
}

// grid (chunks, Hkv): the histogram of one digit among the keys that share the digits before it.
__global__ __launch_bounds__(256) void evict_hist_kernel(EvictArgs a, int digit)
{
    __shared__ uint32_t bins[kEvictBins];
    const int tid = threadIdx.x, head = blockIdx.y;
    uint32_t key;
    int want;
    evict_threshold(a, head, digit, key, want);
    if (want == 0) return;
    for (int i = tid; i < kEvictBins; i += 256) bins[i] = 0;
    __syncthreads();
    const float *w = a.weights + (size_t)head * a.w_cap;
    const int p0 = blockIdx.x * kEvictChunk, p1 = min(p0 + kEvictChunk, a.len - a.n_last);
    const int above = digit == 0 ? 32 : evict_shift(digit - 1);  // the digits before it start here
    for (int p = max(p0, a.n_first) + tid; p < p1; p += 256) {
        const uint32_t k = evict_key(w[p]);
        if (digit == 0 || (k >> above) == (key >> above)) atomicAdd(&bins[(k >> evict_shift(digit)) & evict_mask(digit)], 1u);
    }
    __syncthreads();
    uint32_t *h = a.hist + ((size_t)digit * a.n_kv_heads + head) * kEvictBins;
    for (int i = tid; i < kEvictBins; i += 256)
        if (bins[i]) atomicAdd(&h[i], bins[i]);
}

// grid (chunks, Hkv): how many of the chunk's keys are above the threshold and at it.
__global__ __launch_bounds__(256) void evict_count_kernel(EvictArgs a)
{
    __shared__ int32_t n[2];
    const int tid = threadIdx.x, head = blockIdx.y;
    uint32_t key;
    int want;
    evict_threshold(a, head, 3, key, want);
    if (tid < 2) n[tid] = 0;
    __syncthreads();
    const float *w = a.weights + (size_t)head * a.w_cap;
    const int p0 = blockIdx.x * kEvictChunk, p1 = min(p0 + kEvictChunk, a.len - a.n_last);
    int above = 0, at = 0;
    for (int p = max(p0, a.n_first) + tid; p < p1; p += 256) {
        const uint32_t k = evict_key(w[p]);
        above += k > key;
        at += k == key;
    }
    atomicAdd(&n[0], above);
    atomicAdd(&n[1], at);
    __syncthreads();
    if (tid < 2) a.counts[((size_t)head * a.chunks + blockIdx.x) * 2 + tid] = n[tid];
}

// grid (chunks, Hkv): the chunk's kept positions, in order, to their places in the index.
__global__ __launch_bounds__(256) void evict_index_kernel(EvictArgs a)
{
    __shared__ int32_t s_before[2], s_at[256], s_kept[256];
    const int tid = threadIdx.x, head = blockIdx.y, chunk = blockIdx.x;
    uint32_t key;
    int want;
    evict_threshold(a, head, 3, key, want);
    const int m = a.keep - a.n_first - a.n_last;
    if (tid < 2) s_before[tid] = 0;
    __syncthreads();
    int above = 0, at = 0;
    for (int c = tid; c < chunk; c += 256) {
        above += a.counts[((size_t)head * a.chunks + c) * 2];
        at += a.counts[((size_t)head * a.chunks + c) * 2 + 1];
    }
    atomicAdd(&s_before[0], above);
    atomicAdd(&s_before[1], at);
    __syncthreads();
    const int at_before = s_before[1];
    const int p0 = chunk * kEvictChunk, mid1 = a.len - a.n_last;
    // kept before the chunk: the first n_first, the middle's, the last n_last
    int out = min(p0, a.n_first) + s_before[0] + min(at_before, want) + max(p0 - mid1, 0);
    // eight consecutive positions per thread, so that the order is kept
    constexpr int E = kEvictChunk / 256;
    const float *w = a.weights + (size_t)head * a.w_cap;
    uint32_t k[E];
    int n_at = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int p = p0 + E * tid + i;
        const bool mid = p >= a.n_first && p < mid1;
        k[i] = mid ? evict_key(w[p]) : 0;
        n_at += mid && m > 0 && k[i] == key;
    }
    s_at[tid] = n_at;
    __syncthreads();
    for (int o = 1; o < 256; o *= 2) {
        const int32_t x = tid >= o ? s_at[tid - o] : 0;
        __syncthreads();
        s_at[tid] += x;
        __syncthreads();
    }
    int rank = at_before + s_at[tid] - n_at;  // keys at the threshold before this thread's
    bool take[E];
    int n_take = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int p = p0 + E * tid + i;
        const bool mid = p >= a.n_first && p < mid1;
        take[i] = p < a.len && !mid;
        if (mid && m > 0) {
            if (k[i] == key)
                take[i] = rank++ < want;
            else
                take[i] = k[i] > key;
        }
        n_take += take[i];
    }
    s_kept[tid] = n_take;
    __syncthreads();
    for (int o = 1; o < 256; o *= 2) {
        const int32_t x = tid >= o ? s_kept[tid - o] : 0;
        __syncthreads();
        s_kept[tid] += x;
        __syncthreads();
    }
    out += s_kept[tid] - n_take;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (take[i]) {
            if (out < a.keep) a.index[(size_t)head * a.keep + out] = p0 + E * tid + i;
            ++out;
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
    const dim3 grid((a.len + 255) / 256, a.n_kv_heads);
    if (head_dim == 128)
        key_weights_kernel<128><<<grid, dim3(256), 0, s>>>(a);
    else if (head_dim == 64)
        key_weights_kernel<64><<<grid, dim3(256), 0, s>>>(a);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

inline hipError_t launch_evict_kernels(const EvictArgs &a, hipStream_t s)
{
    if (a.keep <= 0) return hipSuccess;
    const dim3 chunks(a.chunks, a.n_kv_heads), block(256);
    const int n = 3 * a.n_kv_heads * kEvictBins;
    evict_clear_kernel<<<dim3((n + 255) / 256), block, 0, s>>>(a.hist, n);
    for (int d = 0; d < 3; ++d) evict_hist_kernel<<<chunks, block, 0, s>>>(a, d);
    evict_count_kernel<<<chunks, block, 0, s>>>(a);
    evict_index_kernel<<<chunks, block, 0, s>>>(a);
    const int per = 256 / (a.head_dim / 8) * 4;
    evict_gather_kernel<<<dim3((a.keep + per - 1) / per, a.n_kv_heads), block, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace fka
