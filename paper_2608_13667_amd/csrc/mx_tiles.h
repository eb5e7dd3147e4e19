// 4-bit K/V tiles: layout, packing from bf16 and unpacking to it.
//
// A block of 32 values shares a power-of-two scale (one byte b, scale 2^(b - 127)); a value is a 4-bit code
// e2m1: sign, then 0, 0.5, 1, 1.5, 2, 3, 4 or 6.  K blocks are 32 channels of one token and V blocks 32 tokens
// of one channel, in both cases along the axis that the attention's product sums over.  With amax the block's
// largest magnitude,
//   2^E = the power of two at or below amax, over 4; twice that where amax > 7 2^E (6 2^E would cut it by more
//   than an eighth; measured on normal values 19.0 dB signal to noise, 18.8 without),  -125 <= E <= 125,
// and each value is x / 2^E rounded to the nearest code, ties to the even one, at most 6.  The limits of E keep
// every value an ordinary bf16 number (0.5 2^-125 is the smallest normal one), so a tile unpacks exactly; a block of
// zeros has the lowest one.  A block with an infinity or a NaN becomes all NaN (scale byte 255).
//
// A tile holds 128 tokens of one KV head, 136 d bytes: K codes, V codes (64 d each), K scales, V scales
// (4 d each), in the order in which the attention kernel's lanes read them (mx_attend.h).  With token
// 32 a + 8 j + 4 x + b of the tile (a, j, b in 0..3, x in 0..1):
//   K codes   d = 128: [j][x][q][a][b] 16 bytes, channels 32 q ..; d = 64: [j][q][a][b][x] 8 bytes, channels 16 q ..
//   V codes   [channel / 16][a][channel % 16] 16 bytes: tokens 32 a ..
//   K scales  [channel / 32][a][b][j][x]
//   V scales  [a][channel % 16][channel / 16]
// The earlier of two values in a byte is its low half.  Tile ids index a pool [tiles][Hkv][136 d].
//
// Packing and unpacking are bound by the bytes, 2.53 a value: 131000 tokens of 8 heads of 128 (0.68 GB) take 154 and 157 us,
// 4.4 and 4.3 TB/s; 8192 tokens 9.8 and 12.3 us.
#pragma once

#include "internal.h"

namespace fka {

template <int HD>
constexpr int mx_tile_bytes()
{
    return 136 * HD;
}

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));

// The scale byte of a block whose largest magnitude has these bf16 bits.
__device__ inline uint32_t mx_scale_byte(uint32_t amax)
{
    const int e = (int)(amax >> 7) - 2 + ((amax & 0x7f) > 0x60 ? 1 : 0);  // mantissa past 1.75
    return amax >= 0x7f80u ? 255u : (uint32_t)min(max(e, 2), 252);
}

__device__ inline uint32_t mx_amax2(uint32_t a, uint32_t w)  // over both halves of w
{
    return max(a, max(w & 0x7fffu, (w >> 16) & 0x7fffu));
}

// Eight codes of four words (two bf16 each), the first in the low bits.
__device__ inline uint32_t mx_codes8(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, uint32_t scale_byte)
{
    if (scale_byte == 255u) return 0;
    const float s = __uint_as_float(scale_byte << 23);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, w0), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, w1), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, w2), s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(mx_bf16x2, w3), s, 3);
    return r;
}

// Values of byte B of a word of codes, as two bf16.
template <int B>
__device__ inline uint32_t mx_value2(uint32_t codes, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}

__device__ inline uint4 mx_value8(uint32_t codes, float scale)
{
    return uint4{mx_value2<0>(codes, scale), mx_value2<1>(codes, scale), mx_value2<2>(codes, scale), mx_value2<3>(codes, scale)};
}

// The tile's place in the pool, or null for an id outside it (flagged by the block's first thread).
template <int HD>
__device__ inline uint8_t *mx_tile_at(const MxCopyArgs &a, int tile, int head)
{
    const int id = a.tile_row ? a.tile_row[tile] : tile;
    if (id < 0 || id >= a.n_pool_tiles) {
        if (threadIdx.x == 0 && a.err) atomicOr(a.err, kErrBadPage);
        return nullptr;
    }
    return a.tiles + ((size_t)id * a.n_kv_heads + head) * mx_tile_bytes<HD>();
}

// grid (tiles, Hkv), 256 threads: packs one tile.  Bound by HBM: 4 d bytes read per token and head, 1.06 d
// written.  K blocks lie along a row and are packed by a thread each, straight from memory; V blocks run
// across the rows, so the tile's V passes through LDS and a thread packs two neighbouring channels.
template <int HD>
__global__ __launch_bounds__(256) void mx_pack_kernel(MxCopyArgs a)
{
    constexpr int CPR = HD / 8, WPR = HD / 2;  // 16-byte chunks, 4-byte words per row
    __shared__ uint4 v_rows[kMxTile * CPR];
    __shared__ uint8_t scales[8 * HD];  // K's, then V's
    const int tid = threadIdx.x, head = blockIdx.y, tile = a.from / kMxTile + blockIdx.x;
    uint8_t *dst = mx_tile_at<HD>(a, tile, head);
    if (!dst) return;
    const int pos0 = tile * kMxTile, left = a.len - pos0;  // tokens of this tile and after
    const size_t row0 = (size_t)head * a.cap + (pos0 - a.from);
    const uint4 *vs = reinterpret_cast<const uint4 *>(a.v_src + row0 * HD);
    const uint4 *ks = reinterpret_cast<const uint4 *>(a.k_src + row0 * HD);
#pragma unroll
    for (int i = tid; i < kMxTile * CPR; i += 256) v_rows[i] = i / CPR < left ? vs[i] : uint4{0, 0, 0, 0};

    constexpr int GR = HD / kMxBlock;  // blocks per row
#pragma unroll
    for (int i = tid; i < kMxTile * GR; i += 256) {  // i = [j][x][g][a][b]
        const int b = i & 3, ta = (i >> 2) & 3, g = (i >> 4) % GR, jx = (i >> 4) / GR;
        const int token = 32 * ta + 4 * jx + b;
        uint4 w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = token < left ? ks[token * CPR + 4 * g + c] : uint4{0, 0, 0, 0};
        uint32_t amax = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) amax = mx_amax2(mx_amax2(mx_amax2(mx_amax2(amax, w[c].x), w[c].y), w[c].z), w[c].w);
        const uint32_t sb = mx_scale_byte(amax);
        uint4 codes;
        codes.x = mx_codes8(w[0].x, w[0].y, w[0].z, w[0].w, sb);
        codes.y = mx_codes8(w[1].x, w[1].y, w[1].z, w[1].w, sb);
        codes.z = mx_codes8(w[2].x, w[2].y, w[2].z, w[2].w, sb);
        codes.w = mx_codes8(w[3].x, w[3].y, w[3].z, w[3].w, sb);
        if constexpr (HD == 128) {
            reinterpret_cast<uint4 *>(dst)[(jx * 4 + g) * 16 + ta * 4 + b] = codes;
        } else {  // the block is the channels of q = 2 g and 2 g + 1
            uint2 *d2 = reinterpret_cast<uint2 *>(dst);
            const int at = ((((jx >> 1) * 4 + 2 * g) * 4 + ta) * 4 + b) * 2 + (jx & 1);
            d2[at] = uint2{codes.x, codes.y};
            d2[at + 32] = uint2{codes.z, codes.w};
        }
        scales[((g * 4 + ta) * 4 + b) * 8 + jx] = (uint8_t)sb;
    }
    __syncthreads();
    const uint32_t *vw = reinterpret_cast<const uint32_t *>(v_rows);
#pragma unroll
    for (int i = tid; i < 4 * WPR; i += 256) {  // i = [a][channel pair]: lanes along the row, no bank conflicts
        const int ta = i / WPR, c = 2 * (i % WPR);
        uint32_t w[32], m0 = 0, m1 = 0;
#pragma unroll
        for (int t = 0; t < 32; ++t) {
            w[t] = vw[(32 * ta + t) * WPR + c / 2];
            m0 = max(m0, w[t] & 0x7fffu);
            m1 = max(m1, (w[t] >> 16) & 0x7fffu);
        }
        const uint32_t s0 = mx_scale_byte(m0), s1 = mx_scale_byte(m1);
        uint32_t c0[4], c1[4];
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            uint32_t p0[4], p1[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {  // one channel's two tokens in a word
                p0[e] = __builtin_amdgcn_perm(w[8 * o + 2 * e + 1], w[8 * o + 2 * e], 0x05040100u);
                p1[e] = __builtin_amdgcn_perm(w[8 * o + 2 * e + 1], w[8 * o + 2 * e], 0x07060302u);
            }
            c0[o] = mx_codes8(p0[0], p0[1], p0[2], p0[3], s0);
            c1[o] = mx_codes8(p1[0], p1[1], p1[2], p1[3], s1);
        }
        uint4 *vd = reinterpret_cast<uint4 *>(dst + 64 * HD) + (c / 16 * 4 + ta) * 16 + c % 16;
        vd[0] = uint4{c0[0], c0[1], c0[2], c0[3]};
        vd[1] = uint4{c1[0], c1[1], c1[2], c1[3]};
        scales[4 * HD + (ta * 16 + c % 16) * (HD / 16) + c / 16] = (uint8_t)s0;
        scales[4 * HD + (ta * 16 + c % 16 + 1) * (HD / 16) + c / 16] = (uint8_t)s1;
    }
    __syncthreads();
    for (int i = tid; i < 8 * HD / 4; i += 256)
        reinterpret_cast<uint32_t *>(dst + 128 * HD)[i] = reinterpret_cast<const uint32_t *>(scales)[i];
}

// grid (tiles, Hkv), 256 threads: unpacks the positions [from, len) of one tile; V turned through LDS.
template <int HD>
__global__ __launch_bounds__(256) void mx_unpack_kernel(MxCopyArgs a)
{
    constexpr int CPR = HD / 8, WPR = HD / 2, GR = HD / kMxBlock;
    __shared__ uint4 v_rows[kMxTile * CPR];
    const int tid = threadIdx.x, head = blockIdx.y, tile = a.from / kMxTile + blockIdx.x;
    const uint8_t *src = mx_tile_at<HD>(a, tile, head);
    const int pos0 = tile * kMxTile;
    const int lo = max(a.from - pos0, 0), hi = min(a.len - pos0, kMxTile);  // the tile's tokens asked for
    const int64_t row0 = (int64_t)head * a.cap + (pos0 - a.from);           // of the tile's first token
    uint4 *vd = reinterpret_cast<uint4 *>(a.v_dst), *kd = reinterpret_cast<uint4 *>(a.k_dst);
    if (!src) {  // an id outside the pool reads as zeros
        for (int i = tid + lo * CPR; i < hi * CPR; i += 256) kd[row0 * CPR + i] = vd[row0 * CPR + i] = uint4{0, 0, 0, 0};
        return;
    }
    const uint8_t *ksc = src + 128 * HD, *vsc = src + 132 * HD;
    uint32_t *vw = reinterpret_cast<uint32_t *>(v_rows);
#pragma unroll
    for (int i = tid; i < 4 * WPR; i += 256) {  // [a][channel pair]
        const int ta = i / WPR, c = 2 * (i % WPR);
        const uint4 *vc = reinterpret_cast<const uint4 *>(src + 64 * HD) + (c / 16 * 4 + ta) * 16 + c % 16;
        const uint4 x0 = vc[0], x1 = vc[1];
        const float s0 = __uint_as_float((uint32_t)vsc[(ta * 16 + c % 16) * (HD / 16) + c / 16] << 23);
        const float s1 = __uint_as_float((uint32_t)vsc[(ta * 16 + c % 16 + 1) * (HD / 16) + c / 16] << 23);
        const uint32_t w0[4] = {x0.x, x0.y, x0.z, x0.w}, w1[4] = {x1.x, x1.y, x1.z, x1.w};
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            const uint4 p0 = mx_value8(w0[o], s0), p1 = mx_value8(w1[o], s1);
            const uint32_t q0[4] = {p0.x, p0.y, p0.z, p0.w}, q1[4] = {p1.x, p1.y, p1.z, p1.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                vw[(32 * ta + 8 * o + 2 * e) * WPR + c / 2] = __builtin_amdgcn_perm(q1[e], q0[e], 0x05040100u);
                vw[(32 * ta + 8 * o + 2 * e + 1) * WPR + c / 2] = __builtin_amdgcn_perm(q1[e], q0[e], 0x07060302u);
            }
        }
    }
#pragma unroll
    for (int i = tid; i < kMxTile * GR; i += 256) {  // [j][x][g][a][b], as packed
        const int b = i & 3, ta = (i >> 2) & 3, g = (i >> 4) % GR, jx = (i >> 4) / GR;
        const int token = 32 * ta + 4 * jx + b;
        uint32_t w[4];
        if constexpr (HD == 128) {
            const uint4 c = reinterpret_cast<const uint4 *>(src)[(jx * 4 + g) * 16 + ta * 4 + b];
            w[0] = c.x, w[1] = c.y, w[2] = c.z, w[3] = c.w;
        } else {
            const uint2 *s2 = reinterpret_cast<const uint2 *>(src);
            const int at = ((((jx >> 1) * 4 + 2 * g) * 4 + ta) * 4 + b) * 2 + (jx & 1);
            const uint2 c0 = s2[at], c1 = s2[at + 32];
            w[0] = c0.x, w[1] = c0.y, w[2] = c1.x, w[3] = c1.y;
        }
        const float s = __uint_as_float((uint32_t)ksc[((g * 4 + ta) * 4 + b) * 8 + jx] << 23);
        if (token < lo || token >= hi) continue;
#pragma unroll
        for (int c = 0; c < 4; ++c) kd[(row0 + token) * CPR + 4 * g + c] = mx_value8(w[c], s);
    }
    __syncthreads();
    for (int i = tid + lo * CPR; i < hi * CPR; i += 256) vd[row0 * CPR + i] = v_rows[i];
}

inline hipError_t launch_mx_pack_kernel(const MxCopyArgs &a, int head_dim, hipStream_t s)
{
    if (a.len <= a.from) return hipSuccess;
    const dim3 grid((a.len + kMxTile - 1) / kMxTile - a.from / kMxTile, a.n_kv_heads);
    if (head_dim == 128)
        mx_pack_kernel<128><<<grid, dim3(256), 0, s>>>(a);
    else if (head_dim == 64)
        mx_pack_kernel<64><<<grid, dim3(256), 0, s>>>(a);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

inline hipError_t launch_mx_unpack_kernel(const MxCopyArgs &a, int head_dim, hipStream_t s)
{
    if (a.len <= a.from) return hipSuccess;
    const dim3 grid((a.len + kMxTile - 1) / kMxTile - a.from / kMxTile, a.n_kv_heads);
    if (head_dim == 128)
        mx_unpack_kernel<128><<<grid, dim3(256), 0, s>>>(a);
    else if (head_dim == 64)
        mx_unpack_kernel<64><<<grid, dim3(256), 0, s>>>(a);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace fka
