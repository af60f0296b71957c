// New keys and values into a paged cache, the keys (and the queries of the same tokens) rotated by their positions.
//
// Bytes are all there is to it: every value is read once and written once (2 + 2 or 2 + 1 bytes), the rotation adds three
// operations a value.  What a plain kernel spends its time on is the chain of dependent loads in front of the store: offsets ->
// length -> block table -> (rotation row, slot).  So a block takes `tokens` tokens; while its threads' first loads of values,
// which depend on none of that, are under way, one warp finds the tokens' sequences, pages and slots (a lane each) and leaves
// them in shared memory.  A thread then works on units of 16 bytes (of a half-split rotation: pairs of them) across all
// tokens of the block, kDeep units' loads in flight at a time.
#pragma once

#include "fa_paged_common.cuh"

namespace fa {

constexpr int kMostAxes = 4, kMostPairs = 96;

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
    // Work units of a token, of one or two 16-byte vectors: `head_units` per head of K and Q (`span_units` per span), dv/16 per head of
    // V; K, then V, then Q.  The vectors of a span before its turned part, the turned ones and those behind it are cut into units
    // apart: pairs that turn into each other in a half-split rotation, else neighbours where their number is even.
    int before_units, turned_units, span_units, head_units, k_units, v_units, units;
    int before_step, behind_step;                   // vectors of a unit outside the turned part (1 or 2)
    uint32_t head_magic, span_magic, v_magic;       // ceil(2^32 / divisor): exact quotients of numbers below 2^16
    int tokens;                                     // of a block
    uint32_t* status;
    // Positions given for every token (kAt): row `pos[axis * pos_stride + token]` of the table turns the pairs of `axis`; two bits a pair
    const int* pos;
    long long pos_stride;
    int axes;
    uint32_t axis_bits[kMostPairs / 16];
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

// A vector into the cache: bf16, or value * recip rounded to e4m3, recip = 1 / scale in fp32.  (The product's own rounding, 2^-24 of it,
// can move only values within that distance of the middle between two e4m3 numbers; an exact quotient, five operations a
// value, took 38.8 us where this takes 33.2, 2753 tokens of 32 heads 192/128.)
template <bool kE4m3>
FA_DEVI void store_cache8(void* base, long long at, const Vec8& v, float recip) {
    if constexpr (kE4m3) {
        Vec8 s;
#pragma unroll
        for (int i = 0; i < 8; ++i) s.x[i] = v.x[i] * recip;
        uint2 o;
        o.x = ptx::pack_e4m3x4(s.x[0], s.x[1], s.x[2], s.x[3]);
        o.y = ptx::pack_e4m3x4(s.x[4], s.x[5], s.x[6], s.x[7]);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(base) + at) = o;
    } else {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + at) = pack8(v);
    }
}

// floor(x / d) from ceil(2^32 / d), for x < 2^16 (d = 1 has no such number of 32 bits)
FA_DEVI int magic_quot(int x, uint32_t magic) { return magic == 0 ? x : static_cast<int>(__umulhi(static_cast<uint32_t>(x), magic)); }

constexpr int kAppendThreads = 256, kAppendMaxTokens = 16;

// A unit of a half-split rotation is the pair of vectors whose values turn into each other, so that every value is read and written by
// one thread alone (Q_out may be Q).
//
// kAt: the table's rows are given, one per token and axis.  The block puts every token's angles together in shared memory, once for all of its
// heads (40 heads, 7312 tokens of 128 dimensions, three axes: 38 us, against 56 where every unit picks its pairs' rows itself).
template <bool kE4m3, bool kAt = false>
__global__ void __launch_bounds__(kAppendThreads)
fa_append_paged_kernel(const AppendParams p) {
    constexpr int kDeep = 2;
    struct Token { long long k_at, v_at; int pos, live; };      // offsets of its slot in the two caches
    __shared__ Token token[kAppendMaxTokens];
    __shared__ int token_row[kAt ? kAppendMaxTokens : 1][kMostAxes];
    __shared__ alignas(16) float angles[kAt ? kAppendMaxTokens : 1][kAt ? 2 * kMostPairs : 4];
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int t0 = blockIdx.x * p.tokens, n_tokens = min(p.tokens, p.total - t0);

    struct Unit {
        int t, kind, h, c, d, j;     // token of the block, 0 K / 1 V / 2 Q, head, first column, columns to the second vector (0: none),
        uint4 a, b;                  // first angle (-1: not turned); the vectors
    };
    const bool half_split = p.rot_dim != 0 && !p.interleaved;
    auto load_unit = [&](int t, int u, Unit& x) {
        x.t = t;
        x.j = -1;
        const long long row = t0 + t;
        const __nv_bfloat16* src;
        if (u >= p.k_units && u < p.k_units + p.v_units) {
            const int w = u - p.k_units;
            x.kind = 1;
            x.h = magic_quot(w, p.v_magic);
            x.c = (w - x.h * (p.dv >> 4)) * 16;
            x.d = 8;
            src = p.V + row * p.v_st + x.h * p.v_sh + x.c;
        } else {
            x.kind = u < p.k_units ? 0 : 2;
            const int w = x.kind == 2 ? u - p.k_units - p.v_units : u;
            x.h = magic_quot(w, p.head_magic);
            const int in_head = w - x.h * p.head_units, sub = magic_quot(in_head, p.span_magic), i = in_head - sub * p.span_units;
            x.c = sub * p.span;
            if (i < p.before_units) {
                x.c += i * p.before_step * 8;
                x.d = p.before_step == 2 ? 8 : 0;
            } else if (i < p.before_units + p.turned_units) {
                const int r = i - p.before_units;
                x.c += p.rot_offset + r * (half_split ? 8 : 16);
                x.d = half_split ? p.rot_dim >> 1 : 8;
                x.j = r * 8;
            } else {
                x.c += p.rot_offset + p.rot_dim + (i - p.before_units - p.turned_units) * p.behind_step * 8;
                x.d = p.behind_step == 2 ? 8 : 0;
            }
            src = x.kind == 2 ? p.Q + row * p.q_st + x.h * p.q_sh + x.c : p.K + row * p.k_st + x.h * p.k_sh + x.c;
        }
        x.a = *reinterpret_cast<const uint4*>(src);
        if (x.d) x.b = *reinterpret_cast<const uint4*>(src + x.d);
    };
    auto store_unit = [&](const Unit& x) {
        const Token tk = token[x.t];
        if (!tk.live) return;
        Vec8 v = unpack8(x.a), w;
        if (x.d) w = unpack8(x.b);
        if (x.j >= 0) {
            const float* cs = p.cos_sin + static_cast<long long>(tk.pos) * p.rot_dim + x.j;
            const float* sn = cs + (p.rot_dim >> 1);
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                float4 c4, s4;
                if constexpr (kAt) {
                    c4 = *reinterpret_cast<const float4*>(&angles[x.t][x.j + e]);
                    s4 = *reinterpret_cast<const float4*>(&angles[x.t][x.j + (p.rot_dim >> 1) + e]);
                } else {
                    c4 = __ldg(reinterpret_cast<const float4*>(cs + e));
                    s4 = __ldg(reinterpret_cast<const float4*>(sn + e));
                }
                const float cc[4] = {c4.x, c4.y, c4.z, c4.w}, ss[4] = {s4.x, s4.y, s4.z, s4.w};
                Vec8& z = e == 0 ? v : w;            // interleaved: four pairs of each vector
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float& first = half_split ? v.x[e + q] : z.x[2 * q];
                    float& second = half_split ? w.x[e + q] : z.x[2 * q + 1];
                    const float a = first, d = second;
                    first = a * cc[q] - d * ss[q];
                    second = d * cc[q] + a * ss[q];
                }
            }
        }
        if (x.kind == 2) {
            __nv_bfloat16* dst = p.Q_out + (t0 + x.t) * p.qo_st + x.h * p.qo_sh + x.c;
            *reinterpret_cast<uint4*>(dst) = pack8(v);
            if (x.d) *reinterpret_cast<uint4*>(dst + x.d) = pack8(w);
        } else {
            const bool is_v = x.kind == 1;
            const long long at = (is_v ? tk.v_at + x.h * p.v_stride[1] : tk.k_at + x.h * p.k_stride[1]) + x.c;
            const float* scales = is_v ? p.v_scale : p.k_scale;
            // (the reciprocal of a number below the normal ones would be infinite, and 0 times that no number)
            const float recip = kE4m3 && scales ? fminf(__frcp_rn(scales[x.h]), 3.402823466e38f) : 1.f;
            void* base = is_v ? p.v_cache : p.k_cache;
            store_cache8<kE4m3>(base, at, v, recip);
            if (x.d) store_cache8<kE4m3>(base, at + x.d, w, recip);
        }
    };

    // this thread's units: items threadIdx.x, + kAppendThreads, ... as (token, unit)
    int t = 0, u = threadIdx.x;
    auto step = [&]() {
        u += kAppendThreads;
        while (u >= p.units) { u -= p.units; ++t; }
    };
    while (u >= p.units) { u -= p.units; ++t; }
    Unit x[kDeep];
    int have = 0;
#pragma unroll
    for (int q = 0; q < kDeep; ++q) {
        if (t < n_tokens) {
            load_unit(t, u, x[q]);
            have = q + 1;
            step();
        }
    }
    // the tokens' sequences (the last b with cu_seqlens[b] <= row), positions, pages and slots: a lane each
    if (threadIdx.x < n_tokens) {
        const int row = t0 + threadIdx.x;
        Token tk{0, 0, 0, 0};
        int b = -1, first = 0, count = 0;
        if (!p.cu_seqlens) {
            b = row / p.per_seq;
            first = b * p.per_seq;
            count = p.per_seq;
        } else if (row < p.cu_seqlens[p.B]) {        // (else: a row behind the last sequence)
            int lo = 0, hi = p.B;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.cu_seqlens[mid] <= row) lo = mid; else hi = mid;
            }
            b = lo;
            first = p.cu_seqlens[b];
            count = p.cu_seqlens[b + 1] - first;
        }
        if (b >= 0) {
            const int len = p.seq_lens[b];
            tk.pos = len - count + (row - first);
            const int at = tk.pos / p.page_size;
            if (len < 0) {
                report_bad_input(p.status, kSiteBadLength);
            } else if (tk.pos < 0) {
                // (the padding of a batch)
            } else if (at >= p.max_pages) {
                report_bad_input(p.status, kSiteBadLength);
            } else if (!kAt && p.rot_dim && tk.pos >= p.max_pos) {
                report_bad_input(p.status, kSiteBadPosition);
            } else {
                bool rows_ok = true;
                if constexpr (kAt) {
                    for (int a = 0; a < p.axes; ++a) {
                        const int r = p.pos[a * p.pos_stride + row];
                        rows_ok = rows_ok && r >= 0 && r < p.max_pos;
                        token_row[threadIdx.x][a] = r;
                    }
                    if (!rows_ok) report_bad_input(p.status, kSiteBadPosition);
                }
                const int page = p.block_table[b * p.table_stride + at], slot = tk.pos - at * p.page_size;
                if (page < 0 || page >= p.num_pages) {
                    report_bad_input(p.status, kSiteBadPage);
                } else {
                    tk.k_at = page * p.k_stride[0] + slot * p.k_stride[2];
                    tk.v_at = page * p.v_stride[0] + slot * p.v_stride[2];
                    tk.live = rows_ok ? 1 : 0;
                }
            }
        }
        token[threadIdx.x] = tk;
    }
    __syncthreads();
    if constexpr (kAt) {
        for (int i = threadIdx.x; i < n_tokens * p.rot_dim; i += kAppendThreads) {
            const int at = i / p.rot_dim, j = i - at * p.rot_dim, pair = j < (p.rot_dim >> 1) ? j : j - (p.rot_dim >> 1);
            const int axis = (p.axis_bits[pair >> 4] >> (2 * (pair & 15))) & 3;
            if (token[at].live) angles[at][j] = p.cos_sin[static_cast<long long>(token_row[at][axis]) * p.rot_dim + j];
        }
        __syncthreads();
    }
    for (;;) {
#pragma unroll
        for (int q = 0; q < kDeep; ++q)
            if (q < have) store_unit(x[q]);
        if (t >= n_tokens) break;
        have = 0;
#pragma unroll
        for (int q = 0; q < kDeep; ++q) {
            if (t < n_tokens) {
                load_unit(t, u, x[q]);
                have = q + 1;
                step();
            }
        }
    }
}

}  // namespace fa
