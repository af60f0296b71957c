// The small kernels around attention of drafted tokens: what a tree's tokens see and where they stand, accepted tokens moved up in the
// caches of all layers, pages copied in them.
#pragma once

#include "fa_paged_common.cuh"

namespace fa {

// ------------------------------------------------------------------ tree layout

struct LayoutParams {
    const int* parents;
    const int* cu_seqlens;
    const int* seq_lens;
    int total, B, max_tokens;
    uint32_t* mask;
    long long mask_stride;
    int* positions;
    uint32_t* status;
};

// seen(i) = {i} + seen(parent(i)): a thread per token, the paths doubled in every round (a token's words, in registers, take in those of
// the token that it has come to; both then look from where that one looks), so a chain of n tokens takes log2(n) rounds and a tree of
// depth 8 three.  One CTA per sequence.  Bound by the launch and a chain of three loads (offsets, parents and length, result): 4 bytes
// in and 8 to 36 out a token are nothing.
template <int kWords>
__global__ void __launch_bounds__(32 * kWords)
fa_tree_layout_kernel(const LayoutParams p) {
    __shared__ uint32_t seen[32 * kWords][kWords + (kWords > 1 ? 1 : 0)];
    __shared__ int look[32 * kWords];
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int b = blockIdx.x, i = threadIdx.x;
    const DraftRows d = draft_rows(p.cu_seqlens, b, p.B, p.total, p.max_tokens, i == 0 ? p.status : nullptr);
    if (d.count == 0) return;         // (uniform)
    const int len = p.positions ? p.seq_lens[b] : 0;
    int at = -1;                      // the ancestor that is looked at next
    if (i < d.count) {
        at = p.parents[d.first + i];
        if (at < -1 || at >= i) {
            report_bad_input(p.status, kSiteBadParent);
            at = -1;
        }
    }
    uint32_t mine[kWords];
#pragma unroll
    for (int w = 0; w < kWords; ++w) mine[w] = i >> 5 == w ? 1u << (i & 31) : 0u;
    while (__syncthreads_or(at >= 0)) {
#pragma unroll
        for (int w = 0; w < kWords; ++w) seen[i][w] = mine[w];
        look[i] = at;
        __syncthreads();
        if (at >= 0) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) mine[w] |= seen[at][w];
            at = look[at];
        }
    }
    if (i >= d.count) return;
    int depth = -1;
#pragma unroll
    for (int w = 0; w < kWords; ++w) depth += __popc(mine[w]);
    const long long row = d.first + i;
    if (p.mask) {
        const int words = (p.max_tokens + 31) >> 5;
#pragma unroll
        for (int w = 0; w < kWords; ++w)
            if (w < words) p.mask[row * p.mask_stride + w] = mine[w];
    }
    if (p.positions) p.positions[row] = len - d.count + depth;
}

// ------------------------------------------------------------------ caches of several layers

constexpr int kMostCaches = 128;      // of a launch: their pointers travel with its parameters

struct Caches {
    void* k[kMostCaches];
    void* v[kMostCaches];
    int layers;
    int Hkv, page_size, num_pages;
    int k_vecs, v_vecs;               // 16-byte vectors of a head's row
    long long k_stride[3], v_stride[3];          // page, head, slot, in vectors
};

// ------------------------------------------------------------------ accepted drafts

struct CompactParams {
    const int* block_table;
    long long table_stride;
    const int* seq_lens;
    const int* cu_seqlens;
    int B, max_pages, total;
    const int* keep;
    long long keep_stride;
    const int* keep_counts;
    int max_keep;
    int* new_lens;
    int columns;                      // 16-byte vectors of a token in one layer
    int rounds, ctas;                 // of 256 columns a CTA takes, CTAs of a sequence
    uint32_t* status;
};

// Token m of the kept ones goes from slot first + keep[m] to slot first + m; keep rises, so keep[m] >= m, and a slot that is written has
// been read before or is not read at all.  A thread owns one 16-byte column of one sequence and layer and takes it through the moves in
// order, kDeep loads ahead of their stores: no two threads touch the same bytes, so nothing has to wait for anything else, and the
// move is in place.  Bytes are all there is to it; with a few tokens a sequence it is the chain of look-ups before the first load that
// shows: three loads one after the other, for which a CTA takes columns of several layers (64 sequences, 32 layers: 8.0 us with one layer
// a CTA, two waves of 2048, 6.1 with all in one wave).  The moves of a sequence (tokens that stay where they are left out) are found by the
// CTA's threads, one each.
constexpr int kCompactThreads = 256, kMostKeep = 256;

__global__ void __launch_bounds__(kCompactThreads)
fa_compact_kernel(const __grid_constant__ Caches c, const CompactParams p) {
    constexpr int kDeep = 8;
    __shared__ long long from_k[kMostKeep], from_v[kMostKeep], to_k[kMostKeep], to_v[kMostKeep];
    __shared__ int warp_moves[kCompactThreads / 32];
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int b = blockIdx.x / p.ctas, part = blockIdx.x - b * p.ctas;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const bool reports = part == 0 && t == 0;
    // (the kept tokens' numbers are loaded beside their count)
    int src = 0, prev = -1;
    if (t < p.max_keep) {
        src = p.keep[b * p.keep_stride + t];
        if (t > 0) prev = p.keep[b * p.keep_stride + t - 1];
    }
    const DraftRows d = draft_rows(p.cu_seqlens, b, p.B, p.total, kMostKeep, reports ? p.status : nullptr);
    const int len = clamped_len(p.seq_lens[b], p.max_pages, c.page_size, reports ? p.status : nullptr);
    int count = p.keep_counts[b];
    bool bad = count < 0 || count > d.count || count > p.max_keep;
    if (bad) count = 0;
    const int first = len - d.count;
    bad = bad || (t < count && (src <= prev || src >= d.count));
    bad = __syncthreads_or(bad) != 0;
    if (reports) {
        if (bad) report_bad_input(p.status, kSiteBadKeep);
        if (p.new_lens) p.new_lens[b] = bad ? len : max(0, first + count);
    }
    if (bad) return;
    // (drafts in front of position 0 were never stored)
    bool move = t < count && src != t && first + t >= 0;
    long long k0 = 0, v0 = 0, k1 = 0, v1 = 0;
    if (move) {
        const int* table = p.block_table + b * p.table_stride;
        const int a0 = (first + src) / c.page_size, a1 = (first + t) / c.page_size;
        const int s0 = first + src - a0 * c.page_size, s1 = first + t - a1 * c.page_size;
        const int p0 = table[a0], p1 = table[a1];
        if (p0 < 0 || p0 >= c.num_pages || p1 < 0 || p1 >= c.num_pages) {
            report_bad_input(p.status, kSiteBadPage);
            move = false;
        }
        k0 = p0 * c.k_stride[0] + s0 * c.k_stride[2];
        v0 = p0 * c.v_stride[0] + s0 * c.v_stride[2];
        k1 = p1 * c.k_stride[0] + s1 * c.k_stride[2];
        v1 = p1 * c.v_stride[0] + s1 * c.v_stride[2];
    }
    const uint32_t moving = __ballot_sync(0xffffffffu, move);
    if (lane == 0) warp_moves[warp] = __popc(moving);
    __syncthreads();
    int at = __popc(moving & ((1u << lane) - 1u)), moves = 0;
#pragma unroll
    for (int w = 0; w < kCompactThreads / 32; ++w) {
        if (w < warp) at += warp_moves[w];
        moves += warp_moves[w];
    }
    if (move) {
        from_k[at] = k0; from_v[at] = v0;
        to_k[at] = k1; to_v[at] = v1;
    }
    __syncthreads();
    const int k_all = c.Hkv * c.k_vecs;
#pragma unroll 1
    for (int r = 0; r < p.rounds; ++r) {
        const unsigned int at_all = (part * p.rounds + r) * kCompactThreads + t;      // (128 layers of 65535 heads of 40 vectors at most)
        const int layer = at_all / static_cast<unsigned int>(p.columns), col = at_all - layer * p.columns;
        if (layer >= c.layers) return;
        const bool is_v = col >= k_all;
        const int in = is_v ? col - k_all : col, vecs = is_v ? c.v_vecs : c.k_vecs, head = in / vecs;
        uint4* const base = static_cast<uint4*>(is_v ? c.v[layer] : c.k[layer]) + head * (is_v ? c.v_stride[1] : c.k_stride[1]) + (in - head * vecs);
        const long long* const from = is_v ? from_v : from_k;
        const long long* const to = is_v ? to_v : to_k;
        for (int m = 0; m < moves; m += kDeep) {
            uint4 x[kDeep];
#pragma unroll
            for (int q = 0; q < kDeep; ++q)
                if (m + q < moves) x[q] = base[from[m + q]];
#pragma unroll
            for (int q = 0; q < kDeep; ++q)
                if (m + q < moves) base[to[m + q]] = x[q];
        }
    }
}

// ------------------------------------------------------------------ pages

struct CopyParams {
    const int* src;
    const int* dst;
    const int* slots;                 // nullptr: whole pages
    int n;
    // A page is `outer` runs of vectors, `run` for each filled slot long, the next one `step` vectors behind (K, V): heads where a head's
    // slots lie together, one run where a slot's heads do; else heads * slots of one row each
    int k_outer, v_outer, k_run, v_run;
    long long k_step, v_step;
    int scattered;                    // runs are single rows: (head, slot) by their strides
    int k_chunks, v_chunks;           // CTAs of a page
    uint32_t* status;
};

// A copy: read once, written once.  A CTA takes kCopyDeep * 256 vectors of one page of one layer, all loads ahead of the stores.
constexpr int kCopyThreads = 256, kCopyDeep = 4;

__global__ void __launch_bounds__(kCopyThreads)
fa_copy_pages_kernel(const __grid_constant__ Caches c, const CopyParams p) {
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int chunks = p.k_chunks + p.v_chunks;
    const int chunk = blockIdx.x % chunks, rest = blockIdx.x / chunks, i = rest % p.n, layer = rest / p.n;
    const int from = p.src[i], to = p.dst[i];
    if (from < 0 || to < 0) return;
    if (from >= c.num_pages || to >= c.num_pages) {
        if (chunk == 0 && layer == 0 && threadIdx.x == 0) report_bad_input(p.status, kSiteBadPage);
        return;
    }
    const int slots = p.slots ? max(0, min(p.slots[i], c.page_size)) : c.page_size;
    const bool is_v = chunk >= p.k_chunks;
    const int run = (is_v ? p.v_run : p.k_run) * (p.scattered ? 1 : slots), outer = (is_v ? p.v_outer : p.k_outer) * (p.scattered ? slots : 1);
    const int all = run * outer, first = (is_v ? chunk - p.k_chunks : chunk) * (kCopyThreads * kCopyDeep);
    if (first >= all) return;
    const long long* const stride = is_v ? c.v_stride : c.k_stride;
    uint4* const base = static_cast<uint4*>(is_v ? c.v[layer] : c.k[layer]);
    const uint4* const src = base + from * stride[0];
    uint4* const dst = base + to * stride[0];
    uint4 x[kCopyDeep];
    long long at[kCopyDeep];
#pragma unroll
    for (int q = 0; q < kCopyDeep; ++q) {
        const int v = first + q * kCopyThreads + threadIdx.x;
        if (v < all) {
            const int o = outer == 1 ? 0 : v / run, in = v - o * run;
            if (p.scattered) {
                const int head = o / slots;
                at[q] = head * stride[1] + (o - head * slots) * stride[2] + in;
            } else {
                at[q] = o * (is_v ? p.v_step : p.k_step) + in;
            }
            x[q] = src[at[q]];
        }
    }
#pragma unroll
    for (int q = 0; q < kCopyDeep; ++q)
        if (first + q * kCopyThreads + threadIdx.x < all) dst[at[q]] = x[q];
}

}  // namespace fa
