// Per-head RMS norm, position rotation and cache store of new tokens, in one pass.
//
// For a query or key head x of d channels at position m, with a norm weight w (optional):
//   y_c = x_c w_c / sqrt(mean(x^2) + eps)
//   (z_a, z_b) = (y_a cos t - y_b sin t, y_b cos t + y_a sin t),   t = m freq[p]
// for the pairs p of channels (a, b) = (p, p + R/2), or (2p, 2p + 1) interleaved, p < R/2; channels from R
// on are passed through.  Everything is computed in fp32 and rounded once to bf16; the angle is reduced to
// a turn in fp64 first (at position 100000 an fp32 product is off by 0.004 rad).  Queries go to q_out, keys
// to their cache rows, values are copied there bit for bit.
//
// A head is held by d / 16 lanes, 16 channels each: the two 8-channel chunks whose pairs it rotates, so
// that the pairs stay within a lane and the norm's sum is two or three steps across lanes.  A wave takes
// 1024 / d heads at a time (a unit).
//
// Bound by the bytes for many tokens: 32768 of 40 + 8 + 8 heads of 128 (0.94 GB read and written) 187 us, 5.0 TB/s, the
// rate of a large copy; by latency for few, five tokens 4.5 us.
#pragma once

#include "internal.h"

namespace fka {

typedef float rot_f32x8 __attribute__((ext_vector_type(8)));

__device__ inline rot_f32x8 rot_widen(uint4 x)
{
    auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
    auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
    return rot_f32x8{lo(x.x), hi(x.x), lo(x.y), hi(x.y), lo(x.z), hi(x.z), lo(x.w), hi(x.w)};
}

__device__ inline uint4 rot_round(rot_f32x8 x)  // to nearest, ties to even
{
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(uint4, __builtin_convertvector(x, bf16x8));
}

// The sum over each group of LANES (4 or 8) neighbouring lanes.
template <int LANES>
__device__ inline float rot_sum(float x)
{
    auto dpp = [](float v, auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    x += dpp(x, std::integral_constant<int, 0xb1>{});  // quad_perm 1,0,3,2
    x += dpp(x, std::integral_constant<int, 0x4e>{});  // quad_perm 2,3,0,1
    if constexpr (LANES == 8) x += dpp(x, std::integral_constant<int, 0x141>{});  // row_half_mirror
    return x;
}

// Where the token's rows go: K/V row of head h at dst + h * head_step (elements).
struct RotateRow {
    bool ok;
    size_t dst, head_step;
};

template <int HD>
__device__ inline RotateRow rotate_row(const RotateArgs &a, int seq, int t, int len)
{
    RotateRow r;
    const int row = (int)((uint32_t)len + (uint32_t)t);
    r.ok = len >= 0 && (int64_t)len + a.n_tokens <= a.max_len;
    if (a.page_table) {
        int page = -1;
        if (r.ok) {
            const int64_t pidx = ((int64_t)max(a.seq_prefix_len[seq], 0) + kPageSize - 1) / kPageSize + row / kPageSize;
            if (pidx < a.max_pages) page = a.page_table[(size_t)seq * a.max_pages + pidx];
        }
        r.ok = page >= 0 && page < a.n_pool_pages;
        r.dst = ((size_t)(r.ok ? page : 0) * a.n_kv_heads * kPageSize + (r.ok ? row % kPageSize : 0)) * HD;
        r.head_step = (size_t)kPageSize * HD;
    } else {
        r.dst = ((size_t)seq * a.n_kv_heads * a.suffix_cap + (r.ok ? row : 0)) * HD;
        r.head_step = (size_t)a.suffix_cap * HD;
    }
    return r;
}

// WHOLE: a wave takes a whole token, its angles computed once (many tokens); else a block takes a token and
// each wave every blockDim / 64-th unit of it (few tokens: latency).
template <int HD, bool INTERLEAVED, bool WHOLE>
__global__ void rotate_kernel(RotateArgs a)
{
    constexpr int LPH = HD / 16, HPU = 64 / LPH;  // lanes per head, heads per unit
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const int token = WHOLE ? (int)blockIdx.x * waves + wave : (int)blockIdx.x;
    if (token >= a.n_seqs * a.n_tokens) return;  // (only waves of a WHOLE block: no barrier below for them)
    const int seq = token / a.by_tokens, t = token - seq * a.n_tokens;
    const int sub = lane % LPH, hu = lane / LPH;
    const int R = a.rotary_dim;
    const bool turns = 16 * sub < R;
    const int c1 = INTERLEAVED ? 16 * sub : (turns ? 8 * sub : 16 * sub);
    const int c2 = INTERLEAVED || !turns ? c1 + 8 : R / 2 + 8 * sub;
    const int qu = (a.n_q_heads + HPU - 1) / HPU, ku = (a.n_kv_heads + HPU - 1) / HPU;
    const int u0 = WHOLE ? 0 : wave, step = WHOLE ? 1 : waves;

    const int len = a.suffix_len ? a.suffix_len[seq] : 0;
    const RotateRow dst = rotate_row<HD>(a, seq, t, len);
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = 1.f, sn[i] = 0.f;
    if (turns && u0 < qu + ku) {
        const double pos = (double)a.positions[token] * 0.15915494309189533577;  // 1 / (2 pi)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double x = pos * a.freq[8 * sub + i];
            const float r = (float)(x - rint(x));
            sincospif(2.f * r, &sn[i], &cs[i]);
        }
    }
    for (int u = u0; u < qu + 2 * ku; u += step) {
        const bool is_q = u < qu, is_k = !is_q && u < qu + ku;
        const int h = (is_q ? u : is_k ? u - qu : u - qu - ku) * HPU + hu;
        const bool on = h < (is_q ? a.n_q_heads : a.n_kv_heads);
        const uint16_t *src = is_q ? a.q + token * a.q_stride : is_k ? a.k + token * a.k_stride : a.v + token * a.v_stride;
        uint4 x1 = {0, 0, 0, 0}, x2 = {0, 0, 0, 0};
        if (on) {
            x1 = *reinterpret_cast<const uint4 *>(src + (size_t)h * HD + c1);
            x2 = *reinterpret_cast<const uint4 *>(src + (size_t)h * HD + c2);
        }
        if (is_q || is_k) {
            rot_f32x8 y1 = rot_widen(x1), y2 = rot_widen(x2);
            const uint16_t *w = is_q ? a.q_weight : a.k_weight;
            if (w) {
                auto mean = [&](float eps) {
                    float ss = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(y1[i], y1[i], __builtin_fmaf(y2[i], y2[i], ss));
                    return rot_sum<LPH>(ss) * (1.f / HD) + eps;
                };
                float ms = mean(a.eps);
                // a head whose squares leave fp32's range (values past 2^50, or eps next to nothing and values below 2^-50) is
                // normed times 2^-100 or 2^100: exact, and gone again in the quotient
                const bool far = !(ms > 0x1p-100f && ms < 0x1p100f);
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(far) != 0, 0)) {
                    const float s = !far ? 1.f : ms <= 0x1p-100f ? 0x1p100f : 0x1p-100f;
                    y1 *= s;
                    y2 *= s;
                    ms = mean(a.eps * s * s);
                }
                const float inv = 1.f / sqrtf(ms);
                y1 *= rot_widen(*reinterpret_cast<const uint4 *>(w + c1)) * inv;
                y2 *= rot_widen(*reinterpret_cast<const uint4 *>(w + c2)) * inv;
            }
            if (turns) {
                if constexpr (INTERLEAVED) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        rot_f32x8 &y = i < 4 ? y1 : y2;
                        const int j = 2 * (i & 3);
                        const float p = y[j], q = y[j + 1];
                        y[j] = __builtin_fmaf(p, cs[i], -(q * sn[i]));
                        y[j + 1] = __builtin_fmaf(q, cs[i], p * sn[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float p = y1[i], q = y2[i];
                        y1[i] = __builtin_fmaf(p, cs[i], -(q * sn[i]));
                        y2[i] = __builtin_fmaf(q, cs[i], p * sn[i]);
                    }
                }
            }
            if (w || turns) {  // (a head that neither changes keeps its bits)
                x1 = rot_round(y1);
                x2 = rot_round(y2);
            }
        }
        if (!on || (!is_q && !dst.ok)) continue;
        uint16_t *out = is_q ? a.q_out + ((size_t)token * a.n_q_heads + h) * HD
                             : (is_k ? a.k_dst : a.v_dst) + dst.dst + h * dst.head_step;
        *reinterpret_cast<uint4 *>(out + c1) = x1;
        *reinterpret_cast<uint4 *>(out + c2) = x2;
    }
    if constexpr (!WHOLE) __syncthreads();  // every wave has read the length
    if (lane == 0 && (WHOLE || wave == 0)) {
        if (!dst.ok && a.err) atomicOr(a.err, kErrAppendNoRoom);
        if (dst.ok && a.advance && a.n_tokens == 1) a.suffix_len[seq] = len + 1;
    }
}

// Several tokens per sequence: the lengths advance behind the kernel above, which reads them in every block.
// A sequence of which a page is missing keeps its length.
__global__ __launch_bounds__(64) void rotate_advance_kernel(RotateArgs a)
{
    const int seq = blockIdx.x, lane = threadIdx.x;
    const int len = a.suffix_len[seq];
    bool ok = len >= 0 && (int64_t)len + a.n_tokens <= a.max_len;
    if (ok && a.page_table) {
        const int64_t p0 = ((int64_t)max(a.seq_prefix_len[seq], 0) + kPageSize - 1) / kPageSize;
        for (int64_t i = p0 + len / kPageSize + lane; i <= p0 + (len + a.n_tokens - 1) / kPageSize; i += 64) {
            const int page = i < a.max_pages ? a.page_table[(size_t)seq * a.max_pages + i] : -1;
            ok = ok && page >= 0 && page < a.n_pool_pages;
        }
    }
    if (__builtin_amdgcn_ballot_w64(!ok) == 0 && lane == 0) a.suffix_len[seq] = len + a.n_tokens;
}

template <int HD, bool INTERLEAVED>
void launch_rotate_hd(const RotateArgs &a, hipStream_t s)
{
    const int tokens = a.n_seqs * a.n_tokens;
    const int per = 1024 / HD, units = (a.n_q_heads + per - 1) / per + 2 * ((a.n_kv_heads + per - 1) / per);
    // a wave to a token computes its angles once, but only many tokens fill the GPU that way; 40 + 8 + 8 heads of 128: one
    // token 6.6 us by wave and 3.6 by block, 1024 tokens 9.2 and 8.1, 2048 13.1 and 14.2, 8192 37.6 and 43.1
    if (tokens >= 2048)
        rotate_kernel<HD, INTERLEAVED, true><<<dim3((tokens + 3) / 4), dim3(256), 0, s>>>(a);
    else
        rotate_kernel<HD, INTERLEAVED, false><<<dim3(tokens), dim3(64 * (units < 16 ? units : 16)), 0, s>>>(a);
    if (a.advance && a.n_tokens > 1) rotate_advance_kernel<<<dim3(a.n_seqs), dim3(64), 0, s>>>(a);
}

inline hipError_t launch_rotate_kernels(const RotateArgs &a, int head_dim, bool interleaved, hipStream_t s)
{
    if (a.n_seqs <= 0 || a.n_tokens <= 0) return hipSuccess;
    if (head_dim == 128)
        interleaved ? launch_rotate_hd<128, true>(a, s) : launch_rotate_hd<128, false>(a, s);
    else if (head_dim == 64)
        interleaved ? launch_rotate_hd<64, true>(a, s) : launch_rotate_hd<64, false>(a, s);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace fka
