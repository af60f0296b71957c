// Types shared by the kernels that work on a paged key/value cache and by their launcher.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "fa_common.cuh"
#include "ptx.cuh"

namespace fa {

// Contents that only the device sees and that a call may not have: reported as FA_ERR_INVALID_ARG with one of these.
constexpr uint32_t kSiteBadLength = 0x0901, kSiteBadPage = 0x0902, kSiteBadPosition = 0x0903, kSiteBadRows = 0x0904,
                   kSiteBadParent = 0x0905, kSiteBadKeep = 0x0906;

struct PagedParams {
    const __nv_bfloat16* Q;       // token i of sequence b: element (hq, c) at Q + b*q_sb + i*q_st + hq*q_sh + c
    __nv_bfloat16* O;
    float* lse;                   // [Hq, B*Sq] or nullptr
    long long q_sb, q_st, q_sh, o_sb, o_st, o_sh;
    const void* k;                // cache tensors (the serial kernel; the other one goes through tensor maps)
    const void* v;
    long long k_stride[3], v_stride[3];      // page, head, slot, in elements
    const float* k_scale;         // [Hkv] or nullptr
    const float* v_scale;
    const int* block_table;       // nullptr (serial kernel on dense tensors): sequence b is page b
    long long table_stride;
    const int* seq_lens;          // nullptr: every length is `fixed_len`
    int B, max_pages, num_pages, page_size, fixed_len;
    int Hq, Hkv, Sq;
    int causal;                   // 0 (dense tensors only): every token sees every key
    float scale_log2;             // scale * log2(e)
    const float* lambda;          // differential attention: [Hq]
    const float* weight;          // [dv] or nullptr (no normalisation)
    float eps, out_scale;
    int row_blocks;               // blocks of query rows that a (sequence, K/V head) is cut into
    int box_rows;                 // rows of a page box: the largest power of two that divides the page size, at most 128
    int least_units;              // tiles that a CTA takes at least
    int part_cost, long_tiles;    // units that a row block takes in the list beside its tiles, where they are fewer than long_tiles on average
    float* part;                  // partial results: two slots per CTA
    unsigned int* arrivals;       // pieces finished, per (sequence, K/V head, row block) with more than one; zero between launches
    uint32_t* status;
    unsigned long long wait_limit_ns;
    int debug_drop_v_load;
    // drafted tokens: token i of sequence b is row cu_seqlens[b] + i of Q, O and lse, Sq the largest number of them
    const int* cu_seqlens;        // nullptr: total / B tokens each
    const uint32_t* mask;         // as in TreeParams
    long long mask_stride;
    int total;
};

// The place is the report (one store, so that reports of several CTAs cannot mix), in a word of its own behind the code and place of a
// launch that gave up: bad contents concern their own sequences alone and must not hide one whose results are all invalid.
__host__ __device__ inline void report_bad_input(uint32_t* status, uint32_t site) {
    if (!status) return;
    volatile uint32_t* sw = status;       // mapped host memory: plain stores
    sw[2] = site;                         // FA_ERR_INVALID_ARG
}

// Length of sequence b as the kernels use it: what the block table can hold, and never negative.
__host__ __device__ inline int clamped_len(int len, int max_pages, int page_size, uint32_t* status) {
    const long long most = static_cast<long long>(max_pages) * page_size;
    if (len < 0 || len > most) {
        report_bad_input(status, kSiteBadLength);
        return len < 0 ? 0 : static_cast<int>(most);
    }
    return len;
}

// The drafted tokens of sequence b: its rows of the call's tensors.  A sequence whose rows do not lie in [0, total], or that has
// more than `most`, counts as one without.
struct DraftRows { int first, count; };
__host__ __device__ inline DraftRows draft_rows(const int* cu_seqlens, int b, int B, int total, int most, uint32_t* status) {
    DraftRows r;
    if (!cu_seqlens) {
        r.count = total / B;
        r.first = b * r.count;
        return r;
    }
    r.first = cu_seqlens[b];
    const long long n = static_cast<long long>(cu_seqlens[b + 1]) - r.first;
    r.count = static_cast<int>(n);
    if (r.first < 0 || n < 0 || n > most || r.first + n > total) {
        report_bad_input(status, kSiteBadRows);
        r.first = r.count = 0;
    }
    return r;
}

// What the kernels on drafted tokens take beside PagedParams (whose Sq, q_sb and o_sb they do not use).
struct TreeParams {
    const int* cu_seqlens;        // nullptr: total / B tokens each
    int total, max_tokens;
    const uint32_t* mask;         // nullptr: causal among the drafts
    long long mask_stride;
};

// Word w of what token i of n sees among the drafts: bits 32 w .. 32 w + 31 (none from n on).
FA_DEVI uint32_t draft_word(const TreeParams& tp, int row, int i, int n, int w) {
    if (w < 0 || 32 * w >= n) return 0u;
    const int here = n - 32 * w;                                  // drafts from this word on
    const uint32_t in_range = here >= 32 ? 0xffffffffu : (1u << here) - 1u;
    if (tp.mask) return tp.mask[row * tp.mask_stride + w] & in_range;
    const int upto = i - 32 * w;
    return upto < 0 ? 0u : upto >= 31 ? in_range : in_range & ((2u << upto) - 1u);
}

FA_DEVI float e4m3_to_float(uint8_t code) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(code, __NV_E4M3)));
}

}  // namespace fa
