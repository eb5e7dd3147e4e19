// Drafted trees: which nodes each node reads, and what stays of a tree once the tokens are chosen.
//
// tree_layout: with a(i) the parent of node i, a(i) < i, the nodes that node i reads are itself, a(i), a(a(i)), .. to the
// root.  One wave takes a tree, lane i node i.  Six doublings replace up to 63 steps: with m_i the nodes found so far
// and r_i the node behind them, m_i |= m[r_i], r_i = r[r_i].  Bound by the launch: the kernel takes 1.9 us for 5 trees of 16 nodes and 2.4 us
// for 512 of 64, a call from Python 6.
//
// tree_accept: node i is right where its token is the one chosen behind its parent, and no node before it has the same parent
// and token.  It is accepted where all the nodes that it reads are right: one comparison of bit sets a lane.  The
// accepted nodes i_0 < i_1 < .. are a path from the root (a node reads lower ones only), and their K/V rows move to the front,
// row L + i_j to row L + j.  i_j >= j, so a wave that moves a head's rows in ascending chunks, each read whole before it is
// written, never writes a row that is still to be read.
// One block takes a branch, so that the length is written behind every read of it; its waves share the K and V heads.  Bound by
// latency: the tree, the pages, the rows, one after the other.  3.9 us for 5 branches of 16 nodes, 8 KV heads of 128; 7.2 us for 80 of 64 nodes
// in pages (12 MB at the copy rate would be 2.4).
#pragma once

#include "internal.h"

namespace fka {

__global__ __launch_bounds__(256) void tree_layout_kernel(LayoutArgs a)
{
    const int lane = threadIdx.x & 63, b = (int)blockIdx.x * 4 + (threadIdx.x >> 6), n = a.n_nodes;
    if (b >= a.n_branches) return;
    const size_t at = (size_t)b * n + lane;
    const int parent = lane < n ? a.parents[at] : -1, base = a.base[b];
    const bool valid = parent >= 0 && parent < lane;
    if (!valid && parent != -1 && a.err) atomicOr(a.err, kErrBadTree);
    uint64_t m = 1ull << lane;
    int behind = valid ? parent : lane;
#pragma unroll
    for (int i = 0; i < 6; ++i) {
        m |= (uint64_t)(uint32_t)__shfl((int)(uint32_t)m, behind) | (uint64_t)(uint32_t)__shfl((int)(uint32_t)(m >> 32), behind) << 32;
        behind = __shfl(behind, behind);
    }
    if (lane >= n) return;
    a.masks[at] = m;
    a.positions[at] = (int)((uint32_t)base + (uint32_t)__popcll(m) - 1u);
}

// Element offset of head 0's row of suffix position u, and from one head's row to the next; false where there is no such page.
template <int HD>
__device__ inline bool tree_row(const AcceptArgs &a, int b, int64_t u, size_t &at)
{
    if (!a.page_table) {
        at = ((size_t)b * a.n_kv_heads * a.suffix_cap + (size_t)u) * HD;
        return true;
    }
    const int64_t i = ((int64_t)max(a.seq_prefix_len[b], 0) + kPageSize - 1) / kPageSize + u / kPageSize;
    const int page = i < a.max_pages ? a.page_table[(size_t)b * a.max_pages + i] : -1;
    const bool ok = page >= 0 && page < a.n_pool_pages;
    at = ok ? ((size_t)page * a.n_kv_heads * kPageSize + (size_t)(u % kPageSize)) * HD : 0;
    return ok;
}

template <int HD>
__global__ __launch_bounds__(1024) void tree_accept_kernel(AcceptArgs a)
{
    constexpr int LPR = HD / 8, RPI = 64 / LPR, UN = 4, CHUNK = UN * RPI;  // lanes a row, rows an instruction, rows a chunk
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int b = blockIdx.x, n = a.n_nodes;
    const size_t node = (size_t)b * n + lane;
    const bool on = lane < n;
    const int len = a.suffix_len[b];
    const int parent = on ? a.parents[node] : -1, token = on ? a.tokens[node] : 0, target = on ? a.targets[node] : 0;
    const uint64_t reads = on ? a.masks[node] & ~0ull >> (64 - n) : 0;

    const int chosen = __shfl(target, parent & 63);
    const bool fits = parent >= 0 && parent < lane && token == chosen;  // (no lane past the tree has a parent)
    uint64_t right = __builtin_amdgcn_ballot_w64(fits);
    for (uint64_t left = right; left;) {  // of those with one parent, which all have its chosen token, the first
        const int i = __builtin_ctzll(left);
        const int same = __builtin_amdgcn_readlane(parent, i);
        const uint64_t twins = __builtin_amdgcn_ballot_w64(fits && parent == same && lane > i);
        right &= ~twins;
        left &= (left - 1) & ~twins;
    }
    right |= 1;
    uint64_t accepted = __builtin_amdgcn_ballot_w64(lane == 0 || (on && ((reads | 1ull << lane) & ~right) == 0));

    const int last = __builtin_amdgcn_readlane(target, 63 - __builtin_clzll(accepted));  // the pending token

    // lane j: the path's node j, and the offsets of its row and of where that goes
    int count = __popcll(accepted), at = -1;
    {
        const int rank = __popcll(accepted & ((1ull << lane) - 1));
        // the j-th accepted lane sends its number to lane j
        const int to = (accepted >> lane & 1) ? rank : 63;
        const int sent = __builtin_amdgcn_ds_permute(4 * to, lane);
        if (lane < count) at = count == 64 ? lane : sent;
    }
    bool room = len >= 0 && (int64_t)len + n <= a.max_len;
    size_t from = 0, dest = 0;
    if (room && lane < count) {
        const bool ok = tree_row<HD>(a, b, (int64_t)len + at, from);
        room = tree_row<HD>(a, b, (int64_t)len + lane, dest) && ok;
    }
    room = __builtin_amdgcn_ballot_w64(!room) == 0;
    if (wave == 0) {
        if (on) a.path[node] = room ? at : -1;
        if (lane == 0) {
            a.count[b] = room ? count : 0;
            a.next[b] = room ? last : -1;
            if (!room && a.err) atomicOr(a.err, kErrAppendNoRoom);
        }
    }
    __syncthreads();  // every wave has read the length
    if (!room) return;
    if (threadIdx.x == 0 && a.advance) a.suffix_len[b] = len + count;

    const size_t head_step = (size_t)(a.page_table ? kPageSize : a.suffix_cap) * HD;
    const int j_first = accepted == ~0ull ? 64 : __builtin_ctzll(~accepted);  // the rows in front are where they belong
    const int sub = lane % LPR, row = lane / LPR;
    for (int p = wave; p < 2 * a.n_kv_heads; p += waves) {
        uint16_t *cache = (p & 1 ? a.v : a.k) + (p >> 1) * head_step + 8 * sub;
        for (int j0 = j_first; j0 < count; j0 += CHUNK) {
            uint4 x[UN];
            uint16_t *to[UN];
#pragma unroll
            for (int i = 0; i < UN; ++i) {
                const int j = j0 + i * RPI + row;
                const int src = j & 63;
                const size_t f = (size_t)__shfl((unsigned long long)from, src), d = (size_t)__shfl((unsigned long long)dest, src);
                to[i] = j < count ? cache + d : nullptr;
                x[i] = uint4{0, 0, 0, 0};
                if (j < count) x[i] = *reinterpret_cast<const uint4 *>(cache + f);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the chunk is read whole before any of it is written
#pragma unroll
            for (int i = 0; i < UN; ++i)
                if (to[i]) *reinterpret_cast<uint4 *>(to[i]) = x[i];
        }
    }
}

inline hipError_t launch_tree_layout_kernel(const LayoutArgs &a, hipStream_t s)
{
    tree_layout_kernel<<<dim3((a.n_branches + 3) / 4), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

inline hipError_t launch_tree_accept_kernel(const AcceptArgs &a, int head_dim, hipStream_t s)
{
    const dim3 block(64 * (2 * a.n_kv_heads < 16 ? 2 * a.n_kv_heads : 16));
    if (head_dim == 128)
        tree_accept_kernel<128><<<dim3(a.n_branches), block, 0, s>>>(a);
    else if (head_dim == 64)
        tree_accept_kernel<64><<<dim3(a.n_branches), block, 0, s>>>(a);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace fka
