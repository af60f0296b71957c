// Attention of drafted tokens over a paged cache, the plain way: the cross-check of the kernel in fa_tree.cuh
// (FA_FLAG_SERIAL_KERNEL), built like fa_paged_simple.cuh.  One CTA per (token, query head); its four warps take every fourth key, a lane
// holds DQK/32 of a key's dimensions and DV/32 of the accumulator's, everything in fp32 (P too), online softmax per key, and the
// four states are merged at the end.  Bound by the dependent loads and shuffles of a key.
#pragma once

#include <math.h>

#include "fa_paged_common.cuh"

namespace fa {

template <int DQK, int DV, bool kE4m3>
__global__ void __launch_bounds__(128)
fa_tree_simple_kernel(const PagedParams p, const TreeParams tp) {
    constexpr int NQ = DQK / 32, NV = DV / 32;
    __shared__ float sm_m[4], sm_l[4], sm_o[4][DV];
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t* const status = warp == 0 && lane == 0 ? p.status : nullptr;
    const int hq = blockIdx.x % p.Hq, row = blockIdx.x / p.Hq, kvh = hq / (p.Hq / p.Hkv);
    int b = -1;
    DraftRows d{0, 0};
    if (!tp.cu_seqlens) {
        d = draft_rows(nullptr, b = row / (tp.total / p.B), p.B, tp.total, tp.max_tokens, status);
    } else {
        for (int i = 0; i < p.B; ++i) {
            const DraftRows x = draft_rows(tp.cu_seqlens, i, p.B, tp.total, tp.max_tokens, status);
            if (row >= x.first && row < x.first + x.count) { b = i; d = x; break; }
        }
    }
    if (b < 0) return;
    const int i = row - d.first;
    const int len = clamped_len(p.seq_lens[b], p.max_pages, p.page_size, status);
    const __nv_bfloat16* q_row = p.Q + row * p.q_st + hq * p.q_sh;

    float q[NQ], m = -INFINITY, l = 0.f, o[NV];
    const float kq = (kE4m3 && p.k_scale ? p.k_scale[kvh] : 1.f) * p.scale_log2;
#pragma unroll
    for (int e = 0; e < NQ; ++e) q[e] = __bfloat162float(q_row[lane * NQ + e]) * kq;
#pragma unroll
    for (int e = 0; e < NV; ++e) o[e] = 0.f;
    for (int j = warp; j < len; j += 4) {
        const int draft = j - (len - d.count);
        if (draft >= 0 && !((draft_word(tp, row, i, d.count, draft >> 5) >> (draft & 31)) & 1u)) continue;
        const int page = p.block_table[b * p.table_stride + j / p.page_size];
        if (page < 0 || page >= p.num_pages) {
            if (lane == 0) report_bad_input(p.status, kSiteBadPage);
            continue;
        }
        const int slot = j % p.page_size;
        const long long ka = page * p.k_stride[0] + kvh * p.k_stride[1] + slot * p.k_stride[2] + lane * NQ;
        const long long va = page * p.v_stride[0] + kvh * p.v_stride[1] + slot * p.v_stride[2] + lane * NV;
        float s = 0.f, v[NV];
#pragma unroll
        for (int e = 0; e < NQ; ++e)
            s = fmaf(q[e], kE4m3 ? e4m3_to_float(static_cast<const uint8_t*>(p.k)[ka + e])
                                 : __bfloat162float(static_cast<const __nv_bfloat16*>(p.k)[ka + e]), s);
#pragma unroll
        for (int e = 0; e < NV; ++e)
            v[e] = kE4m3 ? e4m3_to_float(static_cast<const uint8_t*>(p.v)[va + e])
                         : __bfloat162float(static_cast<const __nv_bfloat16*>(p.v)[va + e]);
#pragma unroll
        for (int sh = 16; sh > 0; sh >>= 1) s += __shfl_xor_sync(0xffffffffu, s, sh);
        const float mn = fmaxf(m, s);
        // (a score of -inf with nothing before it: weight 0, not exp2(nan))
        const float base = mn == -INFINITY ? 0.f : mn;
        const float r = exp2f(m - base), w = exp2f(s - base);
        m = mn;
        l = l * r + w;
#pragma unroll
        for (int e = 0; e < NV; ++e) o[e] = o[e] * r + w * v[e];
    }
    if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
#pragma unroll
    for (int e = 0; e < NV; ++e) sm_o[warp][lane * NV + e] = o[e];
    __syncthreads();
    const int c = threadIdx.x;
    float mx = -INFINITY, sum = 0.f, acc = 0.f;
    for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm_m[w]);
    const float base = mx == -INFINITY ? 0.f : mx;
    for (int w = 0; w < 4; ++w) {
        const float f = exp2f(sm_m[w] - base);
        sum += f * sm_l[w];
        if (c < DV) acc += f * sm_o[w][c];
    }
    const bool any = sum > 0.f || sum != sum;        // (a NaN goes through)
    const float y = any ? acc / sum * (kE4m3 && p.v_scale ? p.v_scale[kvh] : 1.f) : 0.f;
    if (p.lse && c == 0) p.lse[static_cast<long long>(hq) * tp.total + row] = any ? (mx + log2f(sum)) * 0.6931471805599453f : -INFINITY;
    if (c < DV) p.O[row * p.o_st + hq * p.o_sh + c] = __float2bfloat16(y);
}

}  // namespace fa
