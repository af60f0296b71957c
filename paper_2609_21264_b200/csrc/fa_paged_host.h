// Argument checks and the launch that the entry points on paged caches share.
#pragma once

#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/fa.h"
#include "fa_handle.h"

namespace fa_host {

// Units that a list of work can have at most, by either kernel's count: they are counted in 32 bits, and blocks whose tiles are rounded up to
// a share can count twice their tiles.
constexpr long long kMostUnits = 1ll << 30;

inline bool head_sizes_ok(int dqk, int dv) {
    return (dqk == 64 && dv == 64) || (dqk == 128 && dv == 128) || (dqk == 192 && dv == 128);
}

inline fa_status check_cache(const fa_paged_cache* c) {
    if (!c || c->struct_size != sizeof(fa_paged_cache) || c->reserved != 0) return FA_ERR_INVALID_ARG;
    if (c->type != FA_CACHE_BF16 && c->type != FA_CACHE_E4M3) return FA_ERR_INVALID_ARG;
    if (!c->k || !c->v || misaligned(c->k, 16) || misaligned(c->v, 16)) return FA_ERR_INVALID_ARG;
    if (c->num_pages <= 0 || c->page_size <= 0 || c->Hkv <= 0 || c->dqk <= 0 || c->dv <= 0) return FA_ERR_INVALID_ARG;
    if (!head_sizes_ok(c->dqk, c->dv)) return FA_ERR_UNSUPPORTED;
    if (c->page_size % 16 != 0 || c->page_size > 65536 || c->Hkv > 65535) return FA_ERR_UNSUPPORTED;
    const int64_t unit = c->type == FA_CACHE_E4M3 ? 16 : 8;      // 16 bytes
    for (int i = 0; i < 3; ++i)
        if (c->k_strides[i] <= 0 || c->v_strides[i] <= 0 || c->k_strides[i] % unit != 0 || c->v_strides[i] % unit != 0)
            return FA_ERR_INVALID_ARG;
    if (c->k_strides[2] < c->dqk || c->v_strides[2] < c->dv) return FA_ERR_INVALID_ARG;
    if (c->type == FA_CACHE_BF16 && (c->k_scale || c->v_scale)) return FA_ERR_INVALID_ARG;
    if ((c->k_scale && misaligned(c->k_scale, 4)) || (c->v_scale && misaligned(c->v_scale, 4))) return FA_ERR_INVALID_ARG;
    return FA_OK;
}

inline fa_status check_seqs(const fa_paged_seqs* s, const fa_paged_cache* c) {
    if (!s || s->struct_size != sizeof(fa_paged_seqs) || s->reserved != 0) return FA_ERR_INVALID_ARG;
    if (s->B < 0 || s->max_pages < 0 || s->table_stride < s->max_pages) return FA_ERR_INVALID_ARG;
    if (s->B > 0 && (s->max_pages == 0 || !s->block_table || !s->seq_lens)) return FA_ERR_INVALID_ARG;
    if (misaligned(s->block_table, 4) || misaligned(s->seq_lens, 4)) return FA_ERR_INVALID_ARG;
    // positions are 32-bit
    if (static_cast<int64_t>(s->max_pages) * c->page_size > 0x7fffff00LL) return FA_ERR_UNSUPPORTED;
    return FA_OK;
}

// {token, head} strides of a row-major [tokens, heads, d] tensor
inline bool row_strides_ok(const int64_t* s, int d) { return s && s[0] > 0 && s[1] >= d && ((s[0] | s[1]) & 7) == 0; }

// Rows of one head that lie apart (a [pages, slots, heads, d] pool) are fetched into L2 as they are; with the default of 256 bytes
// their neighbours, other heads' rows, would be fetched too, long before or after their own turn (head size 64,
// 2 K/V heads, 402 MB: 75 us, against 97 with the default).
inline int map_promotion(int d, int elem_bytes, const int64_t* strides) {
    const int64_t row = static_cast<int64_t>(d) * elem_bytes;
    if (strides[2] * elem_bytes == row || row % 256 == 0) return CU_TENSOR_MAP_L2_PROMOTION_L2_256B;
    return row % 128 == 0 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_64B;
}

// Launch with programmatic stream serialisation (see FA_FLAG_NO_DEPENDENT_LAUNCH).
template <typename... Params, typename... Args>
fa_status launch(fa_handle* h, void (*kernel)(Params...), long long blocks, int threads, int smem, cudaStream_t st, const Args&... args) {
    if (blocks <= 0 || blocks > 0x7fffffffLL) return FA_ERR_UNSUPPORTED;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks), 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = (h->flags & FA_FLAG_NO_DEPENDENT_LAUNCH) ? 0 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) {
        cudaGetLastError();
        return FA_ERR_CUDA;
    }
    h->launches += 1;
    return FA_OK;
}

}  // namespace fa_host
