// New keys and values into a paged cache, the keys (and the queries of the same tokens) rotated by their positions.
#pragma once

#include "fa_paged_common.cuh"

namespace fa {

struct AppendParams {
    const __nv_bfloat16 *K, *V, *Q;          // element (t, h, c) at K + t*k_st + h*k_sh + c
    __nv_bfloat16* Q_out;
    long long k_st, k_sh, v_st, v_sh, q_st, q_sh, qo_st, qo_sh;
    void* k_cache;
    void* v_cache;
    long long k_stride[3], v_stride[3];
    const float* k_scale;
    const float* v_scale;
    const int* block_table;
    long long table_stride;
    const int* seq_lens;
    const int* cu_seqlens;                   // nullptr: every sequence has `per_seq` new tokens
    int B, max_pages, num_pages, page_size, total, per_seq;
    int Hq, Hkv, dqk, dv;                    // Hq = 0: no queries
    const float* cos_sin;                    // nullptr: no rotation
    int max_pos, rot_dim, rot_offset, span, interleaved;
    // 16-byte work units of a token: `head_units` per head of K and Q, dv/8 per head of V; K first, then V, then Q
    int span_units, head_units, k_units, v_units, q_units;
    uint32_t* status;
};

// Eight neighbouring values of a row.
struct Vec8 { float x[8]; };

FA_DEVI Vec8 unpack8(uint4 r) {
    Vec8 v;
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v.x[2 * i] = __uint_as_float(w[i] << 16);
        v.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    return v;
}
FA_DEVI uint4 pack8(const Vec8& v) {
    return make_uint4(ptx::pack_bf16x2(v.x[0], v.x[1]), ptx::pack_bf16x2(v.x[2], v.x[3]), ptx::pack_bf16x2(v.x[4], v.x[5]),
                      ptx::pack_bf16x2(v.x[6], v.x[7]));
}

// A vector into the cache: bf16, or value / scale rounded once to e4m3 (an exact division: a product with the reciprocal
// would round twice).
template <bool kE4m3>
FA_DEVI void store_cache8(void* base, long long at, const Vec8& v, float scale) {
    if constexpr (kE4m3) {
        Vec8 s;
#pragma unroll
        for (int i = 0; i < 8; ++i) s.x[i] = __fdiv_rn(v.x[i], scale);
        uint2 o;
        o.x = ptx::pack_e4m3x4(s.x[0], s.x[1], s.x[2], s.x[3]);
        o.y = ptx::pack_e4m3x4(s.x[4], s.x[5], s.x[6], s.x[7]);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(base) + at) = o;
    } else {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + at) = pack8(v);
    }
}

// One thread per 16-byte unit; a unit of a half-split rotation is the pair of vectors whose values turn into each other,
// so that every value is read and written by one thread alone (Q_out may be Q).
template <bool kE4m3>
__global__ void __launch_bounds__(256)
fa_append_paged_kernel(const AppendParams p) {
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int t = blockIdx.x;
    // the token's sequence and position: the last b with cu_seqlens[b] <= t
    int b, pos;
    {
        int first, count;
        if (p.cu_seqlens) {
            if (t >= p.cu_seqlens[p.B]) return;          // a row behind the last sequence
            int lo = 0, hi = p.B;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.cu_seqlens[mid] <= t) lo = mid; else hi = mid;
            }
            b = lo;
            first = p.cu_seqlens[b];
            count = p.cu_seqlens[b + 1] - first;
        } else {
            b = t / p.per_seq;
            first = b * p.per_seq;
            count = p.per_seq;
        }
        pos = p.seq_lens[b] - count + (t - first);
    }
    if (pos < 0) return;
    const int page_at = pos / p.page_size;
    if (page_at >= p.max_pages) { if (threadIdx.x == 0) report_bad_input(p.status, kSiteBadLength); return; }
    if (p.cos_sin && pos >= p.max_pos) { if (threadIdx.x == 0) report_bad_input(p.status, kSiteBadPosition); return; }
    const int page = p.block_table[b * p.table_stride + page_at];
    if (page < 0 || page >= p.num_pages) { if (threadIdx.x == 0) report_bad_input(p.status, kSiteBadPage); return; }
    const int slot = pos - page_at * p.page_size;
    const float* row = p.cos_sin ? p.cos_sin + static_cast<long long>(pos) * p.rot_dim : nullptr;

    for (int u = threadIdx.x; u < p.k_units + p.v_units + p.q_units; u += blockDim.x) {
        if (u >= p.k_units && u < p.k_units + p.v_units) {
            const int w = u - p.k_units, per = p.dv >> 3, h = w / per, c = (w - h * per) * 8;
            const uint4 r = *reinterpret_cast<const uint4*>(p.V + t * p.v_st + h * p.v_sh + c);
            store_cache8<kE4m3>(p.v_cache, page * p.v_stride[0] + h * p.v_stride[1] + slot * p.v_stride[2] + c, unpack8(r),
                                kE4m3 && p.v_scale ? p.v_scale[h] : 1.f);
            continue;
        }
        const bool is_q = u >= p.k_units;
        const int w = is_q ? u - p.k_units - p.v_units : u;
        const int h = w / p.head_units, in_head = w - h * p.head_units;
        const int sub = in_head / p.span_units, i = in_head - sub * p.span_units;
        // unit i of a span: vectors before the rotated part, its pairs (or vectors), vectors behind it
        const int before = p.rot_offset >> 3, turned = p.interleaved ? p.rot_dim >> 3 : p.rot_dim >> 4;
        const bool rotated = row && i >= before && i < before + turned;
        const bool pair = rotated && !p.interleaved;
        const int c = sub * p.span + (i < before + turned || p.interleaved ? i : i + (p.rot_dim >> 4)) * 8;
        const __nv_bfloat16* src = is_q ? p.Q + t * p.q_st + h * p.q_sh + c : p.K + t * p.k_st + h * p.k_sh + c;
        Vec8 x = unpack8(*reinterpret_cast<const uint4*>(src)), y;
        if (pair) {
            const int half = p.rot_dim >> 1, j = (i - before) * 8;
            y = unpack8(*reinterpret_cast<const uint4*>(src + half));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float cs = row[j + e], sn = row[half + j + e];
                const float a = x.x[e], d = y.x[e];
                x.x[e] = a * cs - d * sn;
                y.x[e] = d * cs + a * sn;
            }
        } else if (rotated) {
            const int half = p.rot_dim >> 1, j = (i - before) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float cs = row[j + e], sn = row[half + j + e];
                const float a = x.x[2 * e], d = x.x[2 * e + 1];
                x.x[2 * e] = a * cs - d * sn;
                x.x[2 * e + 1] = d * cs + a * sn;
            }
        }
        if (is_q) {
            __nv_bfloat16* dst = p.Q_out + t * p.qo_st + h * p.qo_sh + c;
            *reinterpret_cast<uint4*>(dst) = pack8(x);
            if (pair) *reinterpret_cast<uint4*>(dst + (p.rot_dim >> 1)) = pack8(y);
        } else {
            const long long at = page * p.k_stride[0] + h * p.k_stride[1] + slot * p.k_stride[2] + c;
            const float scale = kE4m3 && p.k_scale ? p.k_scale[h] : 1.f;
            store_cache8<kE4m3>(p.k_cache, at, x, scale);
            if (pair) store_cache8<kE4m3>(p.k_cache, at + (p.rot_dim >> 1), y, scale);
        }
    }
}

}  // namespace fa
