// Host side of fa_forward_paged_tree (include/fa.h): argument checks, tensor maps, launch.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "../../include/fa.h"
#include "fa_handle.h"
#include "fa_paged_common.cuh"
#include "fa_paged_host.h"
#include "fa_tree_simple.cuh"

namespace {

using namespace fa_host;

template <bool kE4m3>
fa_status launch_simple(fa_handle* h, int dqk, const fa::PagedParams& p, const fa::TreeParams& tp, cudaStream_t st) {
    const long long blocks = static_cast<long long>(tp.total) * p.Hq;
    h->last_kernel = "fa_tree_simple";
    h->last_splits = 1;
    if (dqk == 64) return launch(h, fa::fa_tree_simple_kernel<64, 64, kE4m3>, blocks, 128, 0, st, p, tp);
    if (dqk == 192) return launch(h, fa::fa_tree_simple_kernel<192, 128, kE4m3>, blocks, 128, 0, st, p, tp);
    return launch(h, fa::fa_tree_simple_kernel<128, 128, kE4m3>, blocks, 128, 0, st, p, tp);
}

}  // namespace

extern "C" {

fa_status fa_forward_paged_tree(fa_handle* h, const fa_paged_cache* cache, const fa_paged_seqs* seqs, const fa_tree* tree, int total,
                                const void* Q, void* O, float* lse, int Hq, float scale, const int64_t* q_strides, const int64_t* o_strides,
                                void* stream) {
    if (!h) return FA_ERR_INVALID_ARG;
    fa_status s = check_cache(cache);
    if (s != FA_OK) return s;
    if ((s = check_seqs(seqs, cache)) != FA_OK) return s;
    if (!tree || tree->struct_size != sizeof(fa_tree) || tree->max_tokens <= 0 || total < 0) return FA_ERR_INVALID_ARG;
    if (misaligned(tree->cu_seqlens, 4) || misaligned(tree->mask, 4)) return FA_ERR_INVALID_ARG;
    if (tree->mask && tree->mask_stride < (tree->max_tokens + 31) / 32) return FA_ERR_INVALID_ARG;
    const bool empty = seqs->B == 0 || total == 0;
    if ((!empty && (!Q || !O)) || misaligned(Q, 16) || misaligned(O, 16) || misaligned(lse, 4)) return FA_ERR_INVALID_ARG;
    if (Hq <= 0 || Hq % cache->Hkv != 0 || !isfinite(scale) || scale < 0.f) return FA_ERR_INVALID_ARG;
    if (!row_strides_ok(q_strides, cache->dqk) || !row_strides_ok(o_strides, cache->dv)) return FA_ERR_INVALID_ARG;
    if (tree->max_tokens > FA_TREE_MAX_TOKENS || Hq > 65535 || seqs->B > 65535) return FA_ERR_UNSUPPORTED;
    if (empty) return FA_OK;
    if (!tree->cu_seqlens && (total % seqs->B != 0 || total / seqs->B > tree->max_tokens)) return FA_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok()) return FA_ERR_CUDA;
    if (scale == 0.f) scale = 1.f / sqrtf(static_cast<float>(cache->dqk));

    fa::PagedParams p;
    memset(&p, 0, sizeof p);
    p.Q = static_cast<const __nv_bfloat16*>(Q);
    p.O = static_cast<__nv_bfloat16*>(O);
    p.lse = lse;
    p.q_st = q_strides[0]; p.q_sh = q_strides[1];
    p.o_st = o_strides[0]; p.o_sh = o_strides[1];
    p.k = cache->k; p.v = cache->v;
    for (int i = 0; i < 3; ++i) { p.k_stride[i] = cache->k_strides[i]; p.v_stride[i] = cache->v_strides[i]; }
    p.k_scale = cache->k_scale; p.v_scale = cache->v_scale;
    p.block_table = seqs->block_table; p.table_stride = seqs->table_stride; p.seq_lens = seqs->seq_lens;
    p.B = seqs->B; p.max_pages = seqs->max_pages; p.num_pages = cache->num_pages; p.page_size = cache->page_size;
    p.Hq = Hq; p.Hkv = cache->Hkv;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.status = h->status_dev;
    p.wait_limit_ns = h->wait_limit_ns;
    p.debug_drop_v_load = (h->flags & FA_FLAG_DEBUG_DROP_V_LOAD) ? 1 : 0;
    const fa::TreeParams tp{tree->cu_seqlens, total, tree->max_tokens, tree->mask, tree->mask_stride};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cache->type == FA_CACHE_E4M3 ? launch_simple<true>(h, cache->dqk, p, tp, st) : launch_simple<false>(h, cache->dqk, p, tp, st);
}

}  // extern "C"
