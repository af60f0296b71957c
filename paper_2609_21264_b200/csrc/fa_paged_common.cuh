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
constexpr uint32_t kSiteBadLength = 0x0901, kSiteBadPage = 0x0902, kSiteBadPosition = 0x0903;

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

FA_DEVI float e4m3_to_float(uint8_t code) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(code, __NV_E4M3)));
}

}  // namespace fa
