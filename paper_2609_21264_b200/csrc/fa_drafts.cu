// Host side of the entry points around attention of drafted tokens declared in include/fa.h (tree layout, compaction, page
// copies): argument checks and launch.
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/fa.h"
#include "fa_drafts.cuh"
#include "fa_handle.h"
#include "fa_paged_host.h"

namespace {

using namespace fa_host;

// The caches of a call's layers: each one sound, all of one geometry.
fa_status check_caches(const fa_paged_cache* caches, int num_caches) {
    if (!caches || num_caches <= 0) return FA_ERR_INVALID_ARG;
    for (int i = 0; i < num_caches; ++i) {
        const fa_paged_cache &a = caches[i], &b = caches[0];
        const fa_status s = check_cache(&a);
        if (s != FA_OK) return s;
        if (a.type != b.type || a.num_pages != b.num_pages || a.page_size != b.page_size || a.Hkv != b.Hkv || a.dqk != b.dqk || a.dv != b.dv)
            return FA_ERR_INVALID_ARG;
        for (int j = 0; j < 3; ++j)
            if (a.k_strides[j] != b.k_strides[j] || a.v_strides[j] != b.v_strides[j]) return FA_ERR_INVALID_ARG;
    }
    return FA_OK;
}

// Geometry in 16-byte vectors, and the pointers of caches [first, first + layers).
void set_caches(fa::Caches& c, const fa_paged_cache* caches, int first, int layers) {
    const fa_paged_cache& a = caches[first];
    const int per_vec = a.type == FA_CACHE_E4M3 ? 16 : 8;
    c.layers = layers;
    c.Hkv = a.Hkv; c.page_size = a.page_size; c.num_pages = a.num_pages;
    c.k_vecs = a.dqk / per_vec; c.v_vecs = a.dv / per_vec;
    for (int j = 0; j < 3; ++j) { c.k_stride[j] = a.k_strides[j] / per_vec; c.v_stride[j] = a.v_strides[j] / per_vec; }
    for (int i = 0; i < layers; ++i) { c.k[i] = caches[first + i].k; c.v[i] = caches[first + i].v; }
}

template <int kWords>
fa_status launch_layout(fa_handle* h, const fa::LayoutParams& p, cudaStream_t st) {
    return launch(h, fa::fa_tree_layout_kernel<kWords>, p.B, 32 * kWords, 0, st, p);
}

}  // namespace

extern "C" {

fa_status fa_tree_layout(fa_handle* h, const int32_t* parents, const int32_t* cu_seqlens, int total, int B, const int32_t* seq_lens,
                         int max_tokens, uint32_t* mask, int64_t mask_stride, int32_t* positions, void* stream) {
    if (!h || total < 0 || B < 0 || max_tokens <= 0) return FA_ERR_INVALID_ARG;
    if (max_tokens > FA_TREE_MAX_TOKENS) return FA_ERR_UNSUPPORTED;
    if (misaligned(parents, 4) || misaligned(cu_seqlens, 4) || misaligned(seq_lens, 4) || misaligned(mask, 4) || misaligned(positions, 4))
        return FA_ERR_INVALID_ARG;
    if (mask && mask_stride < (max_tokens + 31) / 32) return FA_ERR_INVALID_ARG;
    if (total == 0 || B == 0 || (!mask && !positions)) return FA_OK;
    if (!parents || (positions && !seq_lens)) return FA_ERR_INVALID_ARG;
    if (!cu_seqlens && (total % B != 0 || total / B > max_tokens)) return FA_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok()) return FA_ERR_CUDA;
    fa::LayoutParams p;
    memset(&p, 0, sizeof p);
    p.parents = parents; p.cu_seqlens = cu_seqlens; p.seq_lens = seq_lens;
    p.total = total; p.B = B; p.max_tokens = max_tokens;
    p.mask = mask; p.mask_stride = mask_stride; p.positions = positions;
    p.status = h->status_dev;
    h->last_kernel = "fa_tree_layout";
    h->last_splits = 1;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // a thread per token and a word per 32: the smallest of the four sizes that holds the trees
    if (max_tokens <= 32) return launch_layout<1>(h, p, st);
    if (max_tokens <= 64) return launch_layout<2>(h, p, st);
    if (max_tokens <= 128) return launch_layout<4>(h, p, st);
    return launch_layout<8>(h, p, st);
}

fa_status fa_compact_paged(fa_handle* h, const fa_paged_cache* caches, int num_caches, const fa_paged_seqs* seqs, const int32_t* cu_seqlens,
                           int total, const int32_t* keep, int64_t keep_stride, const int32_t* keep_counts, int max_keep, int32_t* new_lens,
                           void* stream) {
    if (!h) return FA_ERR_INVALID_ARG;
    fa_status s = check_caches(caches, num_caches);
    if (s != FA_OK) return s;
    if ((s = check_seqs(seqs, caches)) != FA_OK) return s;
    if (total < 0 || max_keep <= 0 || keep_stride < max_keep) return FA_ERR_INVALID_ARG;
    if (misaligned(cu_seqlens, 4) || misaligned(keep, 4) || misaligned(keep_counts, 4) || misaligned(new_lens, 4)) return FA_ERR_INVALID_ARG;
    if (max_keep > FA_TREE_MAX_TOKENS) return FA_ERR_UNSUPPORTED;
    if (seqs->B == 0) return FA_OK;
    if (!keep || !keep_counts) return FA_ERR_INVALID_ARG;
    // (the CTAs of a sequence read all of these, each in its own time)
    if (new_lens && (new_lens == seqs->seq_lens || new_lens == keep_counts || new_lens == keep || new_lens == cu_seqlens)) return FA_ERR_INVALID_ARG;
    if (!cu_seqlens && (total % seqs->B != 0)) return FA_ERR_INVALID_ARG;
    if (!cu_seqlens && total / seqs->B > FA_TREE_MAX_TOKENS) return FA_ERR_UNSUPPORTED;
    DeviceGuard guard(h->device);
    if (!guard.ok()) return FA_ERR_CUDA;
    fa::CompactParams p;
    memset(&p, 0, sizeof p);
    p.block_table = seqs->block_table; p.table_stride = seqs->table_stride; p.seq_lens = seqs->seq_lens;
    p.cu_seqlens = cu_seqlens;
    p.B = seqs->B; p.max_pages = seqs->max_pages; p.total = total;
    p.keep = keep; p.keep_stride = keep_stride; p.keep_counts = keep_counts; p.max_keep = max_keep;
    p.status = h->status_dev;
    h->last_kernel = "fa_compact_paged";
    h->last_splits = 1;
    for (int i = 0; i < num_caches; i += fa::kMostCaches) {
        fa::Caches c;
        memset(&c, 0, sizeof c);
        set_caches(c, caches, i, num_caches - i < fa::kMostCaches ? num_caches - i : fa::kMostCaches);
        p.new_lens = i == 0 ? new_lens : nullptr;
        p.columns = c.Hkv * (c.k_vecs + c.v_vecs);                  // (at most 65535 heads of 40)
        // As many columns a CTA as put all CTAs into one wave of four an SM (60 registers a thread), so that look-ups are not waited for twice.
        const long long all = static_cast<long long>(c.layers) * p.columns, blocks = (all + fa::kCompactThreads - 1) / fa::kCompactThreads;
        const long long rounds = (blocks * p.B + 4ll * h->num_sms - 1) / (4ll * h->num_sms);
        p.rounds = static_cast<int>(rounds < 1 ? 1 : rounds > 16 ? 16 : rounds);
        p.ctas = static_cast<int>((blocks + p.rounds - 1) / p.rounds);
        s = launch(h, fa::fa_compact_kernel, static_cast<long long>(p.ctas) * p.B, fa::kCompactThreads, 0,
                   static_cast<cudaStream_t>(stream), c, p);
        if (s != FA_OK) return s;
    }
    return FA_OK;
}

fa_status fa_copy_pages(fa_handle* h, const fa_paged_cache* caches, int num_caches, const int32_t* src, const int32_t* dst, const int32_t* slots,
                        int n, void* stream) {
    if (!h) return FA_ERR_INVALID_ARG;
    fa_status s = check_caches(caches, num_caches);
    if (s != FA_OK) return s;
    if (n < 0 || misaligned(src, 4) || misaligned(dst, 4) || misaligned(slots, 4)) return FA_ERR_INVALID_ARG;
    if (n == 0) return FA_OK;
    if (!src || !dst) return FA_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok()) return FA_ERR_CUDA;
    h->last_kernel = "fa_copy_pages";
    h->last_splits = 1;
    for (int i = 0; i < num_caches; i += fa::kMostCaches) {
        fa::Caches c;
        memset(&c, 0, sizeof c);
        set_caches(c, caches, i, num_caches - i < fa::kMostCaches ? num_caches - i : fa::kMostCaches);
        fa::CopyParams p;
        memset(&p, 0, sizeof p);
        p.src = src; p.dst = dst; p.slots = slots; p.n = n;
        p.status = h->status_dev;
        // (vectors of a page are counted in 32 bits)
        const long long k_page = static_cast<long long>(c.Hkv) * c.page_size * c.k_vecs, v_page = static_cast<long long>(c.Hkv) * c.page_size * c.v_vecs;
        if (k_page > 0x3fffffffLL || v_page > 0x3fffffffLL) return FA_ERR_UNSUPPORTED;
        const bool one = c.Hkv == 1;
        const bool slots_together = (c.k_stride[2] == c.k_vecs && c.v_stride[2] == c.v_vecs);
        const bool heads_together = !one && c.k_stride[1] == c.k_vecs && c.v_stride[1] == c.v_vecs && c.k_stride[2] == static_cast<long long>(c.Hkv) * c.k_vecs &&
                                    c.v_stride[2] == static_cast<long long>(c.Hkv) * c.v_vecs;
        p.scattered = !slots_together && !heads_together;
        p.k_outer = p.v_outer = heads_together ? 1 : c.Hkv;
        p.k_run = heads_together ? c.Hkv * c.k_vecs : c.k_vecs;
        p.v_run = heads_together ? c.Hkv * c.v_vecs : c.v_vecs;
        p.k_step = c.k_stride[1]; p.v_step = c.v_stride[1];
        const int per = fa::kCopyThreads * fa::kCopyDeep;
        p.k_chunks = static_cast<int>((k_page + per - 1) / per);
        p.v_chunks = static_cast<int>((v_page + per - 1) / per);
        s = launch(h, fa::fa_copy_pages_kernel, static_cast<long long>(p.k_chunks + p.v_chunks) * n * c.layers, fa::kCopyThreads, 0,
                   static_cast<cudaStream_t>(stream), c, p);
        if (s != FA_OK) return s;
    }
    return FA_OK;
}

}  // extern "C"
