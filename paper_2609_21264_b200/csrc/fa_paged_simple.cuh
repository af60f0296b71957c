// Attention of the last tokens of every sequence over a paged cache, the plain way: the cross-check of the kernel in
// fa_paged.cuh (FA_FLAG_SERIAL_KERNEL).  One CTA per (token, query head); its four warps take every fourth key, a lane holds
// DQK/32 of a key's dimensions and DV/32 of the accumulator's, everything in fp32 (P too), online softmax per key, and
// the four states are merged at the end.  Every row of K and V is read by each query head that uses it: bound by the dependent
// loads and shuffles of a key (about 1 us per 4 keys and warp), not by memory.
#pragma once

#include <math.h>

#include "fa_paged_common.cuh"

namespace fa {

template <int DQK, int DV, bool kE4m3, bool kDiff>
__global__ void __launch_bounds__(128)
fa_paged_simple_kernel(const PagedParams p) {
    constexpr int kMaps = kDiff ? 2 : 1, NQ = DQK / 32, NV = DV / 32;
    __shared__ float sm_m[4][kMaps], sm_l[4][kMaps], sm_o[4][kMaps][DV], sm_sq[4];
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int hq = blockIdx.x % p.Hq, t = blockIdx.x / p.Hq;
    const int b = t / p.Sq, i = t - b * p.Sq, kvh = hq / (p.Hq / p.Hkv);
    const int len = p.seq_lens ? clamped_len(p.seq_lens[b], p.max_pages, p.page_size, warp == 0 && lane == 0 ? p.status : nullptr)
                               : p.fixed_len;
    int n_keys = len;                                           // visible keys (may be negative)
    if (p.causal && len - p.Sq + i + 1 < n_keys) n_keys = len - p.Sq + i + 1;
    const __nv_bfloat16* q_row = p.Q + b * p.q_sb + i * p.q_st + hq * p.q_sh;

    // lane l holds dimensions [l*NQ, (l+1)*NQ): with two maps lanes 0-15 hold the first, 16-31 the second
    float q[NQ], m[kMaps], l[kMaps], o[kMaps][NV];
    const float kq = (kE4m3 && p.k_scale ? p.k_scale[kvh] : 1.f) * p.scale_log2;
#pragma unroll
    for (int e = 0; e < NQ; ++e) q[e] = __bfloat162float(q_row[lane * NQ + e]) * kq;
#pragma unroll
    for (int a = 0; a < kMaps; ++a) {
        m[a] = -INFINITY;
        l[a] = 0.f;
#pragma unroll
        for (int e = 0; e < NV; ++e) o[a][e] = 0.f;
    }
    for (int j = warp; j < n_keys; j += 4) {
        const int page = p.block_table ? p.block_table[b * p.table_stride + j / p.page_size] : b;
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
        for (int sh = kDiff ? 8 : 16; sh > 0; sh >>= 1) s += __shfl_xor_sync(0xffffffffu, s, sh);
#pragma unroll
        for (int a = 0; a < kMaps; ++a) {
            const float sa = kDiff ? __shfl_sync(0xffffffffu, s, 16 * a) : s;
            const float mn = fmaxf(m[a], sa);
            // (a score of -inf with nothing before it: weight 0, not exp2(nan))
            const float base = mn == -INFINITY ? 0.f : mn;
            const float r = exp2f(m[a] - base), w = exp2f(sa - base);
            m[a] = mn;
            l[a] = l[a] * r + w;
#pragma unroll
            for (int e = 0; e < NV; ++e) o[a][e] = o[a][e] * r + w * v[e];
        }
    }
#pragma unroll
    for (int a = 0; a < kMaps; ++a) {
        if (lane == 0) { sm_m[warp][a] = m[a]; sm_l[warp][a] = l[a]; }
#pragma unroll
        for (int e = 0; e < NV; ++e) sm_o[warp][a][lane * NV + e] = o[a][e];
    }
    __syncthreads();
    const int c = threadIdx.x;
    const float vs = kE4m3 && p.v_scale ? p.v_scale[kvh] : 1.f;
    float y = 0.f;
#pragma unroll
    for (int a = 0; a < kMaps; ++a) {
        float mx = -INFINITY, sum = 0.f, acc = 0.f;
        for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm_m[w][a]);
        const float base = mx == -INFINITY ? 0.f : mx;
        for (int w = 0; w < 4; ++w) {
            const float f = exp2f(sm_m[w][a] - base);
            sum += f * sm_l[w][a];
            if (c < DV) acc += f * sm_o[w][a][c];
        }
        const bool any = sum > 0.f || sum != sum;        // (a NaN goes through)
        const float part = any ? acc / sum * vs : 0.f;
        y += a == 0 ? part : -p.lambda[hq] * part;
        if (!kDiff && p.lse && c == 0)
            p.lse[static_cast<long long>(hq) * p.B * p.Sq + t] = any ? (mx + log2f(sum)) * 0.6931471805599453f : -INFINITY;
    }
    if constexpr (kDiff) {
        float f = p.out_scale;
        if (p.weight) {
            float sq = y * y;
#pragma unroll
            for (int sh = 16; sh > 0; sh >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, sh);
            if (lane == 0) sm_sq[warp] = sq;
            __syncthreads();
            f *= p.weight[c] * rsqrtf((sm_sq[0] + sm_sq[1] + sm_sq[2] + sm_sq[3]) * (1.f / DV) + p.eps);
        }
        y *= f;
    }
    if (c < DV) p.O[b * p.o_sb + i * p.o_st + hq * p.o_sh + c] = __float2bfloat16(y);
}

}  // namespace fa
