// Partial attention over a prefix in 4-bit tiles (mx_tiles.h) and bf16 suffixes: the streaming stage of a
// decode step whose prefix is held in 4 bits.
//
// Rows, as in the bf16 decode: all sequences of a group (one prefix) x the G query heads of a KV head read
// that head's prefix tiles, so each is fetched once for all of them; a sequence's suffix is read by its G rows.
// A block of four waves takes one job, fixed by the plan: a range of prefix tiles of one (group, KV head), or
// one of R equal shares of one (sequence, KV head)'s suffix, by the length found on the device.  Its waves deal
// the job's tiles (128 keys) or slices (32 keys) in turn, each with an online softmax of its own, and are joined
// through LDS into one normalised partial (o, lse) per row, which the merge kernel joins over the jobs.
//
// Both products run on v_mfma_f32_16x16x32_bf16 with keys on M, S^T = K Q^T and O^T += V^T P^T, so a lane owns
// one query row.  The tile's layout is made for the operands: a lane's 16 bytes of K are 32 channels of the key
// in its M row, its 16 bytes of V 32 keys of the channel in its M row, and the keys of S^T that a lane gets in two
// products (x = 0, 1) are the eight that it has to supply as P in the one with its V bytes: nothing crosses lanes
// and no tile passes through LDS.  Codes become bf16 (K) and fp16 (V) by v_cvt_scalef32_pk_*_fp4, exactly.  p enters
// the second product as two fp16 terms (mx_split16; two bf16 terms left 2e-6 in the output, one 1e-3), times
// 2^7 so that the second term is a normal number down to p = 2^-9 of the reference.  A tile with a V scale outside fp16's exact
// range, [2^-23, 2^8], takes bf16 and three terms instead, as do the suffixes, whose values are bf16.  The
// running maximum is a reference only: it moves when a score passes it by 2^8.
//
// Up to 16 rows bound by the tiles' bytes (128k keys of 8 heads of 128, 143 MB: 5 rows 26.1 us and 4.5 of the merge), past them by the
// vector instructions and the products: 20 rows 31.6 us, 40 rows 49.1.  In a 32k step of 25 rows 18.3 us, the bf16 kernel 29.
#pragma once

#include <type_traits>

#include "internal.h"
#include "mx_tiles.h"

namespace fka {

typedef __bf16 mx_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 mx_f16x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x4 __attribute__((ext_vector_type(4)));
typedef short mx_s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) mx_s16x4 mx_lds_s16x4;

__device__ inline mx_f32x4 mx_mfma(mx_bf16x8 a, mx_bf16x8 b, mx_f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ inline mx_f32x4 mx_mfma(mx_f16x8 a, mx_f16x8 b, mx_f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight values of a word of codes as fp16.
__device__ inline mx_f16x8 mx_value8h(uint32_t codes, float scale)
{
    const uint4 r = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3))};
    return __builtin_bit_cast(mx_f16x8, r);
}

// Raw buffer resource over [base, base + bytes), wave-uniform.
__device__ inline __amdgpu_buffer_rsrc_t mx_rsrc(const void *base, int bytes)
{
    const uint64_t b = (uint64_t)base;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void *)(((uint64_t)hi << 32) | lo), 0, __builtin_amdgcn_readfirstlane(bytes),
                                             0x00020000);
}

// 16 bytes per lane, non-temporal where they are read once (POLICY 2), else kept for the pair's other wave (0).
template <int POLICY = 2>
__device__ inline uint4 mx_load16(__amdgpu_buffer_rsrc_t r, uint32_t off)
{
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, POLICY));
}

// Sixteen wait states between products and the first vector read of their results: what the compiler counts
// there has fallen short for this instruction on gfx950 (see partials.hip).
__device__ inline void mx_result_wait()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 7\n\ts_nop 7" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A product's result, read behind mx_result_wait: held in the registers where the product left it, so that no copy is made
// in front of the wait.
__device__ __attribute__((always_inline)) inline void mx_result(mx_f32x4 &x) { asm volatile("" : "+v"(x)); }

// The four lanes that hold one query row: l, l ^ 16, l ^ 32, l ^ 48.
__device__ inline float mx_row_max(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float mx_row_sum(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Moves the rows' references of all NT tiles where a score has passed one by more than 2^8; mx: the largest of
// each lane's own raw scores.  The four lanes of a row are looked at together only then.
template <int NT, int NE>
__device__ __attribute__((always_inline)) inline void mx_move(const float (&mx)[NT], float scale_log2, float (&m_ref)[NT],
                                                              float (&l_run)[NT], mx_f32x4 (&acc)[NT][NE])
{
    constexpr float kGap = 8.f;
    bool any = false;
#pragma unroll
    for (int t = 0; t < NT; ++t) any |= mx[t] * scale_log2 > m_ref[t] + kGap;  // the scale is positive: the order is kept
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(any) == 0, 1)) return;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float m = mx_row_max(mx[t]) * scale_log2;
        const bool move = m > m_ref[t] + kGap;
        // exactly 1 for a row that keeps its reference; 0 when that was -inf
        const float alpha = move ? __builtin_amdgcn_exp2f(m_ref[t] - m) : 1.f;
        l_run[t] *= alpha;
#pragma unroll
        for (int e = 0; e < NE; ++e) acc[t][e] *= alpha;
        m_ref[t] = move ? m : m_ref[t];
    }
}

template <int N>
__device__ __attribute__((always_inline)) inline float mx_max(const float (&x)[N])
{
    float m = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, x[i]);
    return m;
}

// x becomes p = 2^(scaled x - reference + kMxShift), summed into l_run.  The shift keeps the second fp16
// term of p from the subnormals down to 2^-9 of the reference; with the gap of 2^8 a p is at most 2^15.
constexpr float kMxShift = 7.f;
template <int N>
__device__ __attribute__((always_inline)) inline void mx_exp(float (&x)[N], float scale_log2, float m_ref, float &l_run)
{
    const float nm = m_ref == -INFINITY ? 0.f : kMxShift - m_ref;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], scale_log2, nm));
        sum += x[i];
    }
    l_run += sum;
}

// p less one half of a word of two fp16 values, in one instruction.
template <int HALF>
__device__ __attribute__((always_inline)) inline float mx_rest(uint32_t h, float p)
{
    float r;
    if constexpr (HALF == 0)
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(p));
    else
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(p));
    return r;
}

// Eight p as two fp16 terms, both to nearest (v_cvt_pk_f16_f32 takes two values, as the instruction that cuts does): within 2^-23 of p
// down to 2^-9 of the reference, below it, where the second term is a subnormal, within 2^-32 of the reference.  To nearest, since a second
// term that is never negative is lost one way: added to a sum 2^24 times as large it rounds to nothing, and 2^19 keys of value 1
// with some 2^-16 of the largest weight each came out 2.4e-4 short, 1e-7 this way (the mean of 128 rows).
__device__ __attribute__((always_inline)) inline void mx_split16(const float *p, mx_f16x8 &hi, mx_f16x8 &lo)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    auto pair = [](float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2)); };
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[i] = pair(p[2 * i], p[2 * i + 1]);
        l[i] = pair(mx_rest<0>(h[i], p[2 * i]), mx_rest<1>(h[i], p[2 * i + 1]));
    }
    hi = __builtin_bit_cast(mx_f16x8, h);
    lo = __builtin_bit_cast(mx_f16x8, l);
}

// Eight p as three bf16 terms, to nearest: all of p's 24 bits.
__device__ __attribute__((always_inline)) inline void mx_split3(const float *p, mx_bf16x8 (&t)[3])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        t[0][i] = (__bf16)p[i];
        const float r = p[i] - (float)t[0][i];
        t[1][i] = (__bf16)r;
        t[2][i] = (__bf16)(r - (float)t[1][i]);
    }
}

// A wave goes first while it feeds the matrix cores, and last in its softmax, so that its neighbour's softmax runs beside its
// products: 8 forks of 20 rows at 32k 92.9 -> 90.7 us, 40 rows at 128k without suffixes 64.6 -> 62.8; d 64, whose products are half as
// long, 50.7 -> 51.8, and stays without.
template <int HD, int P>
__device__ __attribute__((always_inline)) inline void mx_prio()
{
    if constexpr (HD == 128) __builtin_amdgcn_s_setprio(P);
}

// A wave takes NT 16-row tiles, one or two: with three or four, its registers would leave one wave to a SIMD, and a
// lone wave issues a vector instruction every 8 cycles at best (two together every 4; measured with chains of eight).  So
// with more than 32 rows the waves of a block work in pairs (RS = 2), each pair on one tile, half of the rows each.
template <int HD, int NT, int RS>
__global__ __launch_bounds__(256, 2) void mx_partials_kernel(MxArgs a)
{
    constexpr int NW = 4, NG = NW / RS, NC = HD / 32, NE = HD / 16, CPR = HD / 8, ROWB = 2 * HD;
    constexpr int kTileB = mx_tile_bytes<HD>();
    // the waves' V slices of a suffix, then their accumulators
    __shared__ __attribute__((aligned(16))) float stage[NW][NT * 16 * HD];
    __shared__ __attribute__((aligned(16))) float red_m[NT * 16][NW], red_l[NT * 16][NW];
    static_assert(sizeof(stage[0]) >= (size_t)kSlice * ROWB, "a V slice fits");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, q4 = lane >> 4;
    const MxJob job = a.jobs[blockIdx.x];
    const bool suffix = job.suffix != 0;
    // a prefix job's waves: wave group wg takes every NG-th tile, row half rh of it (rows from 16 NT rh on)
    const int wg = suffix ? wave : wave / RS, rh = suffix ? 0 : wave % RS, row_lo = 16 * NT * rh;
    const int G = a.group, rows = job.rows, nt_act = (rows - row_lo + 15) / 16;

    if (blockIdx.x == 0) {  // what the merge appends at
        for (int s = tid; s < a.n_seqs; s += 256) {
            const int raw = a.suffix_len[s], L = min(max(raw, 0), a.max_suffix_len);
            a.lens[s] = L;
            if (L != raw) atomicOr(a.err, kErrSuffixClamped);
        }
    }

    // query rows (B operand): lane holds row 16 t + l16; its channels are those of the K operand
    mx_bf16x8 qb[NT][NC];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = row_lo + 16 * t + l16;
#pragma unroll
        for (int c = 0; c < NC; ++c) qb[t][c] = mx_bf16x8{};
        if (r < rows) {
            const int ri = job.first + r, rq = div_magic(ri, G, a.group_magic);
            const uint16_t *qp = a.q + ((size_t)(job.seq0 + rq) * a.n_q_heads + job.head * G + ri - rq * G) * HD;
#pragma unroll
            for (int c = 0; c < NC; ++c)
                qb[t][c] = *reinterpret_cast<const mx_bf16x8 *>(qp + (suffix ? 32 * c + 8 * q4 : (HD / 4) * q4 + 8 * c));
        }
    }
    mx_f32x4 acc[NT][NE];
    float m_ref[NT], l_run[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m_ref[t] = -INFINITY;
        l_run[t] = 0.f;
#pragma unroll
        for (int e = 0; e < NE; ++e) acc[t][e] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
    }

    bool any = true;  // the job has keys
    if (!suffix) {
        constexpr int KL = HD / 16;  // K loads of 16 bytes
        uint4 kr[KL], vr[NE];
        uint32_t ks[2], vs[2] = {0, 0};
        // the resource of one of the job's tiles; an id outside the pool is not read: an empty resource gives zeros
        auto tile_rsrc = [&](int tile) {
            int id = job.tile0 + tile;
            if (a.tile_table && tile < job.end) id = a.tile_table[(size_t)job.group * a.max_tiles + tile];
            id = __builtin_amdgcn_readfirstlane(id);
            const bool in = tile < job.end, bad = in && (id < 0 || id >= a.n_pool_tiles);
            if (bad && lane == 0) atomicOr(a.err, kErrBadPage);
            const bool read = in && !bad;
            return mx_rsrc(a.tiles + ((size_t)(read ? id : 0) * a.n_kv_heads + job.head) * kTileB, read ? kTileB : 0);
        };
        auto load_k = [&](__amdgpu_buffer_rsrc_t rs) {
#pragma unroll
            for (int i = 0; i < KL; ++i) kr[i] = mx_load16<RS == 1 ? 2 : 0>(rs, i * 1024 + lane * 16);
            const auto w = __builtin_amdgcn_raw_buffer_load_b64(rs, 128 * HD + ((HD == 128 ? q4 : q4 >> 1) * 16 + l16) * 8, 0, 2);
            ks[0] = w[0], ks[1] = w[1];
        };
        auto load_v = [&](__amdgpu_buffer_rsrc_t rs) {
#pragma unroll
            for (int e = 0; e < NE; ++e) vr[e] = mx_load16<RS == 1 ? 2 : 0>(rs, 64 * HD + e * 1024 + lane * 16);
            if constexpr (HD == 128) {
                const auto w = __builtin_amdgcn_raw_buffer_load_b64(rs, 132 * HD + lane * 8, 0, 2);
                vs[0] = w[0], vs[1] = w[1];
            } else {
                vs[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, 132 * HD + lane * 4, 0, 2);
            }
        };
        int tile = job.begin + wg;
        const __amdgpu_buffer_rsrc_t rs = tile_rsrc(tile);
        load_k(rs);
        load_v(rs);
        for (; tile < job.end; tile += NG) {
            const int valid = job.prefix_len - tile * kMxTile;
            const __amdgpu_buffer_rsrc_t next = tile_rsrc(tile + NG);
            // V scales 2^-23 .. 2^8, as bytes 104 .. 135: exact in fp16 (a byte below 104 borrows, and shows so itself).  A block of
            // zeros has byte 2 and counts as outside, though its scale does not matter: see the loop behind
            uint32_t odd = (vs[0] - 0x68686868u) & 0xe0e0e0e0u;
            if constexpr (HD == 128) odd |= (vs[1] - 0x68686868u) & 0xe0e0e0e0u;
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd != 0) != 0, 0)) break;  // the loop behind takes the rest
            // J steps of 32 keys at a time: their scores, their softmax, their p.v.  With one row tile all four, whose first two
            // parts need K only, so that V arrives behind them; with two, two and two, which the registers hold.  Product (j, x) has keys 32 a + 8 j + 4 x + b in M row 4 a + b.
            constexpr int J = NT == 1 ? 4 : 2;
#pragma unroll
            for (int j0 = 0; j0 < 4; j0 += J) {
                mx_prio<HD, 1>();
                mx_f32x4 s[NT][2 * J];
                // two products' chains (x = 0, 1) of each row tile side by side: a product of a chain waits for the one before
#pragma unroll
                for (int i = 0; i < 2 * J; i += 2) {
                    const int jx = 2 * j0 + i;
                    float ksc[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        ksc[u] = __uint_as_float(((ks[jx >> 2] >> (8 * ((jx & 3) + u))) & 0xff) << 23);
#pragma unroll
                        for (int t = 0; t < NT; ++t) s[t][i + u] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
                    }
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const uint4 w = HD == 128 ? kr[jx + u] : kr[jx >> 1];
                            const int n = HD == 128 ? c : 2 * u + c;
                            const mx_bf16x8 kb =
                                __builtin_bit_cast(mx_bf16x8, mx_value8(n == 0 ? w.x : n == 1 ? w.y : n == 2 ? w.z : w.w, ksc[u]));
#pragma unroll
                            for (int t = 0; t < NT; ++t) s[t][i + u] = mx_mfma(kb, qb[t][c], s[t][i + u]);
                        }
                    __builtin_amdgcn_sched_barrier(0);  // (conversions far ahead would leave the registers)
                }
                mx_result_wait();
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 2 * J; ++i) mx_result(s[t][i]);
                if (j0 + J == 4) load_k(next);  // its time: the softmax and p.v
                if (__builtin_expect(valid < kMxTile, 0)) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int i = 0; i < 8 * J; ++i)
                            s[t][i / 4][i % 4] = 32 * q4 + 8 * j0 + i < valid ? s[t][i / 4][i % 4] : -INFINITY;
                }
                mx_prio<HD, 0>();
                float mx[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    mx[t] = s[t][0][0];
#pragma unroll
                    for (int i = 1; i < 8 * J; ++i) mx[t] = fmaxf(mx[t], s[t][i / 4][i % 4]);
                }
                mx_move(mx, a.scale_log2, m_ref, l_run, acc);
                mx_f16x8 ph[NT][J], pl[NT][J];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        float x[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = s[t][2 * j + i / 4][i % 4];
                        mx_exp(x, a.scale_log2, m_ref[t], l_run[t]);
                        mx_split16(x, ph[t][j], pl[t][j]);
                    }
                __builtin_amdgcn_sched_barrier(0);
                mx_prio<HD, 1>();
                // two channel tiles side by side, the first terms of p in front of the second
#pragma unroll
                for (int e = 0; e < NE; e += 2) {
                    float vsc[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) vsc[u] = __uint_as_float(((vs[e >> 2] >> (8 * ((e & 3) + u))) & 0xff) << 23);
#pragma unroll
                    for (int i = 0; i < J; ++i) {
                        const int j = j0 + i;
                        mx_f16x8 vb[2];
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            vb[u] = mx_value8h(j == 0 ? vr[e + u].x : j == 1 ? vr[e + u].y : j == 2 ? vr[e + u].z : vr[e + u].w, vsc[u]);
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int t = 0; t < NT; ++t) acc[t][e + u] = mx_mfma(vb[u], ph[t][i], acc[t][e + u]);
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int t = 0; t < NT; ++t) acc[t][e + u] = mx_mfma(vb[u], pl[t][i], acc[t][e + u]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            load_v(next);  // its time: the next tile's scores and first softmax
        }
        // the same with V in bf16 and three terms of p, from the first tile with another scale on: 32 keys at a time straight from
        // memory.  What comes here, with the rest of its wave's tiles: a block whose largest value is past 7 2^8 or at most 7 2^-24;
        // a prefix's last tile of at most 96 tokens (25 rows over 32668 keys 19.6 us, 32767 or 32768 17.9); and a V channel of
        // zeros (25 rows over 32k keys 27.0 us, 40 rows over 128k 148 against 69)
        for (; tile < job.end; tile += NG) {
            const int valid = job.prefix_len - tile * kMxTile;
            const __amdgpu_buffer_rsrc_t rt = tile_rsrc(tile);
#pragma unroll 1
            for (int j = 0; j < 4; ++j) {
                const uint32_t kw = __builtin_amdgcn_raw_buffer_load_b16(
                    rt, 128 * HD + ((HD == 128 ? q4 : q4 >> 1) * 16 + l16) * 8 + 2 * j, 0, 0);
                uint4 w[2];
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    w[u] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rt, (HD == 128 ? 2 * j + u : j) * 1024 + lane * 16, 0, 0));
                mx_f32x4 s[NT][2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float ksc = __uint_as_float(((kw >> (8 * u)) & 0xff) << 23);
                    mx_bf16x8 kb[NC];
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        const int n = HD == 128 ? c : 2 * u + c;
                        kb[c] = __builtin_bit_cast(mx_bf16x8, mx_value8(n == 0 ? w[u].x : n == 1 ? w[u].y : n == 2 ? w[u].z : w[u].w, ksc));
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        s[t][u] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int c = 0; c < NC; ++c) s[t][u] = mx_mfma(kb[c], qb[t][c], s[t][u]);
                    }
                }
                mx_result_wait();
                float x[NT][8], mx[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    mx_result(s[t][0]), mx_result(s[t][1]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[t][i] = 32 * q4 + 8 * j + i < valid ? s[t][i / 4][i % 4] : -INFINITY;
                    mx[t] = mx_max(x[t]);
                }
                mx_move(mx, a.scale_log2, m_ref, l_run, acc);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    mx_exp(x[t], a.scale_log2, m_ref[t], l_run[t]);
                    mx_bf16x8 p3[3];
                    mx_split3(x[t], p3);
#pragma unroll
                    for (int e = 0; e < NE; ++e) {
                        const uint32_t vw = __builtin_amdgcn_raw_buffer_load_b32(rt, 64 * HD + e * 1024 + lane * 16 + 4 * j, 0, 0);
                        const uint32_t vb8 = __builtin_amdgcn_raw_buffer_load_b8(rt, 132 * HD + lane * NE + e, 0, 0);
                        const mx_bf16x8 vb = __builtin_bit_cast(mx_bf16x8, mx_value8(vw, __uint_as_float(vb8 << 23)));
#pragma unroll
                        for (int n = 0; n < 3; ++n) acc[t][e] = mx_mfma(vb, p3[n], acc[t][e]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    } else {
        const int L = __builtin_amdgcn_readfirstlane(min(max(a.suffix_len[job.seq0], 0), a.max_suffix_len));
        const int n = slices_of(L), begin = mul_div(job.begin, n, job.end), end = mul_div(job.begin + 1, n, job.end);
        any = end > begin;
        const size_t base = ((size_t)job.seq0 * a.n_kv_heads + job.head) * a.suffix_cap * ROWB;
        uint4 *ring = reinterpret_cast<uint4 *>(&stage[wave][0]);
        constexpr int VL = kSlice * CPR / 64;  // V loads per lane of a slice
        const int jt = l16 >> 2, m4 = l16 & 3, T0 = 4 * q4 + jt;
        uint4 kr[2][NC], vr[VL];
        auto load = [&](int sl) {
            const int bytes = sl < end ? min(L - sl * kSlice, kSlice) * ROWB : 0;  // rows at or past L read as zeros
            const size_t off = base + (size_t)(sl < end ? sl : 0) * kSlice * ROWB;
            const __amdgpu_buffer_rsrc_t rk = mx_rsrc(reinterpret_cast<const char *>(a.suffix_k) + off, bytes);
            const __amdgpu_buffer_rsrc_t rv = mx_rsrc(reinterpret_cast<const char *>(a.suffix_v) + off, bytes);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int c = 0; c < NC; ++c) kr[u][c] = mx_load16(rk, (16 * u + l16) * ROWB + 64 * c + 16 * q4);
#pragma unroll
            for (int i = 0; i < VL; ++i) vr[i] = mx_load16(rv, (64 * i + lane) * 16);
        };
        load(begin + wave);
        for (int sl = begin + wave; sl < end; sl += NW) {
            const int valid = L - sl * kSlice;
            mx_f32x4 s[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                s[u] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NC; ++c) s[u] = mx_mfma(__builtin_bit_cast(mx_bf16x8, kr[u][c]), qb[0][c], s[u]);
            }
            // V through the wave's own LDS, read back transposed: chunk c of token T at T CPR + (c ^ 2 T mod CPR),
            // so that a column read touches every bank (a wave's LDS operations run in order: no barrier)
#pragma unroll
            for (int i = 0; i < VL; ++i) {
                const int p = 64 * i + lane, T = p / CPR, c = p % CPR;
                ring[T * CPR + (c ^ ((2 * T) & (CPR - 1)))] = vr[i];
            }
            mx_result_wait();
            mx_result(s[0]), mx_result(s[1]);
            load(sl + NW);  // its time: the softmax and p.v
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = s[i / 4][i % 4];
                if (valid < kSlice) x[i] = 16 * (i / 4) + 4 * q4 + i % 4 < valid ? x[i] : -INFINITY;
            }
            const float mx[1] = {mx_max(x)};
            mx_move(mx, a.scale_log2, reinterpret_cast<float(&)[1]>(m_ref), reinterpret_cast<float(&)[1]>(l_run),
                    reinterpret_cast<mx_f32x4(&)[1][NE]>(acc));
            mx_exp(x, a.scale_log2, m_ref[0], l_run[0]);
            mx_bf16x8 p3[3];
            mx_split3(x, p3);
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                // lane (q4, 4 j + m): tokens 4 q4 + j and 16 + 4 q4 + j, channels 16 e + 4 m ..
                const int slot = (2 * e + (m4 >> 1)) ^ ((2 * T0) & (CPR - 1));
                char *at = reinterpret_cast<char *>(ring) + T0 * ROWB + slot * 16 + (m4 & 1) * 8;
                const mx_s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mx_lds_s16x4 *)at);
                const mx_s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mx_lds_s16x4 *)(at + 16 * ROWB));
                const short __attribute__((ext_vector_type(8))) v = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
#pragma unroll
                for (int n = 0; n < 3; ++n) acc[0][e] = mx_mfma(__builtin_bit_cast(mx_bf16x8, v), p3[n], acc[0][e]);
            }
        }
        // An infinite value has met the three terms of p, of either sign or zero: NaN, where the result is that infinity (of both
        // signs: NaN).  So where a sum is not finite (products of pairs tell in few steps), the channel's values are looked up.
        mx_result_wait();
        float fold = 0.f;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
            mx_result(acc[0][e]);
            fold = __builtin_fmaf(acc[0][e][0], acc[0][e][1], fold);
            fold = __builtin_fmaf(acc[0][e][2], acc[0][e][3], fold);
        }
        // (a row with a NaN sum is NaN whatever its values are)
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(l_run[0] < INFINITY && !(__builtin_fabsf(fold) < INFINITY)) != 0, 0)) {
            // lane l looks at channels CL l .. of this wave's keys; bits 3 i of `seen`: channel CL l + i has +inf, -inf, a NaN
            constexpr int CL = HD / 64;
            const uint16_t *v = reinterpret_cast<const uint16_t *>(reinterpret_cast<const char *>(a.suffix_v) + base);
            uint32_t seen = 0;
            for (int sl = begin + wave; sl < end; sl += NW)
                for (int k = sl * kSlice; k < min(L, (sl + 1) * kSlice); ++k)
#pragma unroll
                    for (int i = 0; i < CL; ++i) {
                        const uint32_t x = v[(size_t)k * HD + CL * lane + i];
                        seen |= (x == 0x7f80u ? 1u : x == 0xff80u ? 2u : (x & 0x7fffu) > 0x7f80u ? 4u : 0u) << (3 * i);
                    }
#pragma unroll
            for (int e = 0; e < NE; ++e)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = 16 * e + 4 * q4 + j;
                    const uint32_t f = (uint32_t)__shfl((int)seen, c / CL) >> (3 * (c % CL)) & 7u;
                    if (f == 1 || f == 2) acc[0][e][j] = f == 1 ? INFINITY : -INFINITY;
                }
        }
    }

    // ---- the waves' (max, sum, accumulator) into one partial per row
    const size_t row_out = (size_t)job.slot * a.slot_rows + job.row0;
    if (!any) {
        for (int r = tid; r < rows; r += 256) a.part_lse[row_out + r] = -INFINITY;
        return;
    }
    mx_result_wait();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float sum = mx_row_sum(l_run[t]);
        if (q4 == 0) {
            red_m[16 * t + l16][wave] = m_ref[t];
            red_l[16 * t + l16][wave] = sum;
        }
        // chunk c of row r at c ^ r mod 16: a store covers 16 rows at one chunk (a suffix's slices in the ring are read)
#pragma unroll
        for (int e = 0; e < NE; ++e)
            if (t < nt_act) *reinterpret_cast<mx_f32x4 *>(&stage[wave][(16 * t + l16) * HD + 4 * ((4 * e + q4) ^ l16)]) = acc[t][e];
    }
    __syncthreads();
    // a thread takes one chunk of 4 channels of every 256 / (HD / 4)-th row
    constexpr int CH = HD / 4;
    const int c = tid % CH;
    for (int row = tid / CH; row < rows; row += 256 / CH) {
        // the row in its half, whose waves are every RS-th (a suffix: all four have all rows)
        const int half = row / (16 * NT), r = row - 16 * NT * half;
        float m[NW], w[NW], M = -INFINITY, W = 0.f;
        mx_f32x4 v[NW], o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const bool has = RS == 1 || suffix || i % RS == half;
            m[i] = has ? red_m[r][i] : -INFINITY;
            w[i] = has ? red_l[r][i] : 0.f;
            v[i] = *reinterpret_cast<const mx_f32x4 *>(&stage[i][r * HD + 4 * (c ^ (r & 15))]);
        }
#pragma unroll
        for (int i = 0; i < NW; ++i) M = fmaxf(M, m[i]);
        const float Mu = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float e = __builtin_amdgcn_exp2f(m[i] - Mu);  // a wave without keys: 0
            W = __builtin_fmaf(e, w[i], W);
            if (RS == 1 || suffix || i % RS == half) o += e * v[i];  // (the other half's may be NaN)
        }
        *reinterpret_cast<mx_f32x4 *>(a.part_o + (row_out + row) * HD + 4 * c) = o * (W == 0.f ? 0.f : 1.f / W);
        if (c == 0) a.part_lse[row_out + row] = W == 0.f ? -INFINITY : (Mu - kMxShift + log2f(W)) * 0.693147180559945309f;
    }
}

template <int HD>
const void *mx_kernel_of(int row_tiles)
{
    if (row_tiles == 1) return reinterpret_cast<const void *>(&mx_partials_kernel<HD, 1, 1>);
    if (row_tiles == 2) return reinterpret_cast<const void *>(&mx_partials_kernel<HD, 2, 1>);
    return reinterpret_cast<const void *>(&mx_partials_kernel<HD, 2, 2>);
}

// Resident blocks per compute unit (0 on error).
inline int mx_blocks_per_cu_of(int head_dim, int row_tiles)
{
    if ((head_dim != 64 && head_dim != 128) || row_tiles < 1 || row_tiles > 4) return 0;
    int n = 0;
    const void *f = head_dim == 128 ? mx_kernel_of<128>(row_tiles) : mx_kernel_of<64>(row_tiles);
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, f, 256, 0) != hipSuccess) return 0;
    return n;
}

template <int HD>
hipError_t launch_mx_hd(const MxArgs &a, int n_jobs, int row_tiles, hipStream_t s)
{
    if (row_tiles < 1 || row_tiles > 4) return hipErrorInvalidValue;
    if (row_tiles == 1)
        mx_partials_kernel<HD, 1, 1><<<dim3(n_jobs), dim3(256), 0, s>>>(a);
    else if (row_tiles == 2)
        mx_partials_kernel<HD, 2, 1><<<dim3(n_jobs), dim3(256), 0, s>>>(a);
    else
        mx_partials_kernel<HD, 2, 2><<<dim3(n_jobs), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace fka
