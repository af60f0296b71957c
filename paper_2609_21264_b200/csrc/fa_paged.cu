// Host side of the paged-cache and differential-attention entry points declared in include/fa.h: argument checks,
// tensor maps, kernel selection and launch.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "../../include/fa.h"
#include "fa_append_paged.cuh"
#include "fa_common.cuh"
#include "fa_fwd_diff.cuh"
#include "fa_handle.h"
#include "fa_paged_common.cuh"
#include "fa_paged_host.h"
#include "fa_paged_list.h"
#include "fa_paged_simple.cuh"

namespace {

using namespace fa_host;

fa_status check_diff(const fa_diff* d) {
    if (!d || d->struct_size != sizeof(fa_diff) || d->reserved != 0.f) return FA_ERR_INVALID_ARG;
    if (!d->lambda || misaligned(d->lambda, 4)) return FA_ERR_INVALID_ARG;
    if (d->weight && (misaligned(d->weight, 16) || !isfinite(d->eps) || d->eps <= 0.f)) return FA_ERR_INVALID_ARG;
    if (!isfinite(d->out_scale)) return FA_ERR_INVALID_ARG;
    return FA_OK;
}

template <bool kE4m3, bool kDiff>
fa_status launch_simple(fa_handle* h, int dqk, const fa::PagedParams& p, cudaStream_t st) {
    const long long blocks = static_cast<long long>(p.B) * p.Sq * p.Hq;
    h->last_kernel = "fa_paged_simple";
    h->last_splits = 1;
    if constexpr (!kDiff) {
        if (dqk == 64) return launch(h, fa::fa_paged_simple_kernel<64, 64, kE4m3, kDiff>, blocks, 128, 0, st, p);
        if (dqk == 192) return launch(h, fa::fa_paged_simple_kernel<192, 128, kE4m3, kDiff>, blocks, 128, 0, st, p);
    }
    return launch(h, fa::fa_paged_simple_kernel<128, 128, kE4m3, kDiff>, blocks, 128, 0, st, p);
}

template <int DQK, int DV, bool kE4m3, bool kDiff>
fa_status launch_paged_rows(fa_handle* h, int block, const CUtensorMap& mk, const CUtensorMap& mv, fa::PagedParams& p, cudaStream_t st) {
    if constexpr (!kE4m3 && !kDiff && DQK != 192) {
        if (block == 64) return launch_paged<DQK, DV, kE4m3, kDiff, 64>(h, mk, mv, p, st);
    }
    if constexpr (!kDiff) {
        if (block == 32) return launch_paged<DQK, DV, kE4m3, kDiff, 32>(h, mk, mv, p, st);
    }
    return launch_paged<DQK, DV, kE4m3, kDiff, 16>(h, mk, mv, p, st);
}

fa_status forward_paged(fa_handle* h, const fa_paged_cache* cache, const fa_paged_seqs* seqs, const void* Q, void* O, float* lse,
                        int Hq, int Sq, float scale, const fa_diff* diff, const int64_t* q_strides, const int64_t* o_strides,
                        void* stream) {
    fa_status s = check_cache(cache);
    if (s != FA_OK) return s;
    if ((s = check_seqs(seqs, cache)) != FA_OK) return s;
    if ((seqs->B > 0 && (!Q || !O)) || misaligned(Q, 16) || misaligned(O, 16) || (lse && misaligned(lse, 4))) return FA_ERR_INVALID_ARG;
    if (Hq <= 0 || Sq <= 0 || Hq % cache->Hkv != 0 || !isfinite(scale) || scale < 0.f) return FA_ERR_INVALID_ARG;
    if (!row_strides_ok(q_strides, cache->dqk) || !row_strides_ok(o_strides, cache->dv)) return FA_ERR_INVALID_ARG;
    if (Sq > FA_PAGED_MAX_SQ || Hq > 65535 || seqs->B > 65535) return FA_ERR_UNSUPPORTED;
    if (diff && (cache->dqk != 128 || cache->dv != 128)) return FA_ERR_UNSUPPORTED;
    if (seqs->B == 0) return FA_OK;
    DeviceGuard guard(h->device);
    if (!guard.ok()) return FA_ERR_CUDA;
    if (scale == 0.f) scale = 1.f / sqrtf(static_cast<float>(diff ? 64 : cache->dqk));

    fa::PagedParams p;
    memset(&p, 0, sizeof p);
    p.Q = static_cast<const __nv_bfloat16*>(Q);
    p.O = static_cast<__nv_bfloat16*>(O);
    p.lse = lse;
    p.q_st = q_strides[0]; p.q_sh = q_strides[1]; p.q_sb = Sq * q_strides[0];
    p.o_st = o_strides[0]; p.o_sh = o_strides[1]; p.o_sb = Sq * o_strides[0];
    p.k = cache->k; p.v = cache->v;
    for (int i = 0; i < 3; ++i) { p.k_stride[i] = cache->k_strides[i]; p.v_stride[i] = cache->v_strides[i]; }
    p.k_scale = cache->k_scale; p.v_scale = cache->v_scale;
    p.block_table = seqs->block_table; p.table_stride = seqs->table_stride; p.seq_lens = seqs->seq_lens;
    p.B = seqs->B; p.max_pages = seqs->max_pages; p.num_pages = cache->num_pages; p.page_size = cache->page_size;
    p.Hq = Hq; p.Hkv = cache->Hkv; p.Sq = Sq;
    p.causal = 1;
    p.scale_log2 = scale * 1.4426950408889634f;
    if (diff) { p.lambda = diff->lambda; p.weight = diff->weight; p.eps = diff->eps; p.out_scale = diff->out_scale; }
    p.status = h->status_dev;
    p.wait_limit_ns = h->wait_limit_ns;
    p.debug_drop_v_load = (h->flags & FA_FLAG_DEBUG_DROP_V_LOAD) ? 1 : 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool e4m3 = cache->type == FA_CACHE_E4M3;
    if (h->flags & FA_FLAG_SERIAL_KERNEL) {
        if (e4m3) return diff ? launch_simple<true, true>(h, cache->dqk, p, st) : launch_simple<true, false>(h, cache->dqk, p, st);
        return diff ? launch_simple<false, true>(h, cache->dqk, p, st) : launch_simple<false, false>(h, cache->dqk, p, st);
    }
    p.box_rows = 16;
    while (p.box_rows < 128 && cache->page_size % (2 * p.box_rows) == 0) p.box_rows *= 2;
    set_list(p, cache->dqk, cache->dv, e4m3);
    const int rows = Hq / cache->Hkv * Sq, block = rows_per_block(rows, cache->dqk, e4m3, diff != nullptr);
    p.row_blocks = (rows + block - 1) / block;
    if (most_units(p) > kMostUnits) return FA_ERR_UNSUPPORTED;
    const int eb = e4m3 ? 1 : 2;
    const CUtensorMap* m = nullptr;
    auto promotion = [&](int d, const int64_t* strides) { return map_promotion(d, eb, strides); };
    if ((s = get_map(h, cache->k, cache->dqk, cache->page_size, cache->Hkv, cache->num_pages, cache->k_strides[0], cache->k_strides[1],
                     cache->k_strides[2], p.box_rows, &m, eb, 1, 128, promotion(cache->dqk, cache->k_strides))) != FA_OK) return s;
    const CUtensorMap mk = *m;       // a copy: the next insertion may move the cache's entries
    if ((s = get_map(h, cache->v, cache->dv, cache->page_size, cache->Hkv, cache->num_pages, cache->v_strides[0], cache->v_strides[1],
                     cache->v_strides[2], p.box_rows, &m, eb, 1, 128, promotion(cache->dv, cache->v_strides))) != FA_OK) return s;
    const CUtensorMap mv = *m;
    if (diff) return e4m3 ? launch_paged_rows<128, 128, true, true>(h, block, mk, mv, p, st) : launch_paged_rows<128, 128, false, true>(h, block, mk, mv, p, st);
    if (cache->dqk == 64) return e4m3 ? launch_paged_rows<64, 64, true, false>(h, block, mk, mv, p, st) : launch_paged_rows<64, 64, false, false>(h, block, mk, mv, p, st);
    if (cache->dqk == 192) return e4m3 ? launch_paged_rows<192, 128, true, false>(h, block, mk, mv, p, st) : launch_paged_rows<192, 128, false, false>(h, block, mk, mv, p, st);
    return e4m3 ? launch_paged_rows<128, 128, true, false>(h, block, mk, mv, p, st) : launch_paged_rows<128, 128, false, false>(h, block, mk, mv, p, st);
}

}  // namespace

extern "C" {

fa_status fa_append_paged(fa_handle* h, const fa_paged_cache* cache, const fa_paged_seqs* seqs, const int32_t* cu_seqlens, int total,
                          const void* K, const void* V, const void* Q, void* Q_out, int Hq, const int64_t* k_strides,
                          const int64_t* v_strides, const int64_t* q_strides, const int64_t* qo_strides, const fa_rope* rope,
                          void* stream) {
    return fa_append_paged_at(h, cache, seqs, cu_seqlens, total, K, V, Q, Q_out, Hq, k_strides, v_strides, q_strides, qo_strides, rope, nullptr,
                              stream);
}

fa_status fa_append_paged_at(fa_handle* h, const fa_paged_cache* cache, const fa_paged_seqs* seqs, const int32_t* cu_seqlens, int total,
                             const void* K, const void* V, const void* Q, void* Q_out, int Hq, const int64_t* k_strides,
                             const int64_t* v_strides, const int64_t* q_strides, const int64_t* qo_strides, const fa_rope* rope,
                             const fa_positions* positions, void* stream) {
    if (!h) return FA_ERR_INVALID_ARG;
    fa_status s = check_cache(cache);
    if (s != FA_OK) return s;
    if ((s = check_seqs(seqs, cache)) != FA_OK) return s;
    if (total < 0 || (cu_seqlens && misaligned(cu_seqlens, 4))) return FA_ERR_INVALID_ARG;
    if (total == 0 || seqs->B == 0) return FA_OK;
    if (!cu_seqlens && total % seqs->B != 0) return FA_ERR_INVALID_ARG;
    if (!K || !V || misaligned(K, 16) || misaligned(V, 16)) return FA_ERR_INVALID_ARG;
    if (!row_strides_ok(k_strides, cache->dqk) || !row_strides_ok(v_strides, cache->dv)) return FA_ERR_INVALID_ARG;
    if (!Q != !Q_out) return FA_ERR_INVALID_ARG;
    if (Q) {
        if (misaligned(Q, 16) || misaligned(Q_out, 16) || Hq <= 0) return FA_ERR_INVALID_ARG;
        if (Hq > 65535) return FA_ERR_UNSUPPORTED;
        if (!row_strides_ok(q_strides, cache->dqk) || !row_strides_ok(qo_strides, cache->dqk)) return FA_ERR_INVALID_ARG;
    }
    if (rope) {
        if (rope->struct_size != sizeof(fa_rope) || !rope->cos_sin || misaligned(rope->cos_sin, 16)) return FA_ERR_INVALID_ARG;
        if (rope->max_pos <= 0 || rope->dim <= 0 || rope->offset < 0 || rope->span <= 0) return FA_ERR_INVALID_ARG;
        if (rope->dim % 16 != 0 || rope->span % 16 != 0 || rope->offset % 8 != 0) return FA_ERR_UNSUPPORTED;
        if (cache->dqk % rope->span != 0 || rope->dim > rope->span || rope->offset > rope->span - rope->dim) return FA_ERR_INVALID_ARG;
    }
    if (positions) {
        if (!rope || positions->struct_size != sizeof(fa_positions) || !positions->pos || misaligned(positions->pos, 4)) return FA_ERR_INVALID_ARG;
        if (positions->axes <= 0 || (positions->axes > 1 && positions->stride < total)) return FA_ERR_INVALID_ARG;
        if (positions->axes > FA_MAX_AXES) return FA_ERR_UNSUPPORTED;
        for (int i = 0; positions->axis_of_pair && i < rope->dim / 2; ++i)
            if (positions->axis_of_pair[i] >= positions->axes) return FA_ERR_INVALID_ARG;
    }
    DeviceGuard guard(h->device);
    if (!guard.ok()) return FA_ERR_CUDA;
    fa::AppendParams p;
    memset(&p, 0, sizeof p);
    p.K = static_cast<const __nv_bfloat16*>(K);
    p.V = static_cast<const __nv_bfloat16*>(V);
    p.k_st = k_strides[0]; p.k_sh = k_strides[1];
    p.v_st = v_strides[0]; p.v_sh = v_strides[1];
    if (Q) {
        p.Q = static_cast<const __nv_bfloat16*>(Q);
        p.Q_out = static_cast<__nv_bfloat16*>(Q_out);
        p.q_st = q_strides[0]; p.q_sh = q_strides[1];
        p.qo_st = qo_strides[0]; p.qo_sh = qo_strides[1];
        p.Hq = Hq;
    }
    p.k_cache = cache->k; p.v_cache = cache->v;
    for (int i = 0; i < 3; ++i) { p.k_stride[i] = cache->k_strides[i]; p.v_stride[i] = cache->v_strides[i]; }
    p.k_scale = cache->k_scale; p.v_scale = cache->v_scale;
    p.block_table = seqs->block_table; p.table_stride = seqs->table_stride; p.seq_lens = seqs->seq_lens;
    p.cu_seqlens = cu_seqlens;
    p.B = seqs->B; p.max_pages = seqs->max_pages; p.num_pages = cache->num_pages; p.page_size = cache->page_size;
    p.total = total;
    p.per_seq = cu_seqlens ? 0 : total / seqs->B;
    p.Hkv = cache->Hkv; p.dqk = cache->dqk; p.dv = cache->dv;
    p.span = cache->dqk;
    if (rope) {
        p.cos_sin = rope->cos_sin;
        p.max_pos = rope->max_pos; p.rot_dim = rope->dim; p.rot_offset = rope->offset; p.span = rope->span;
        p.interleaved = rope->interleaved ? 1 : 0;
    }
    if (positions) {
        static_assert(fa::kMostAxes == FA_MAX_AXES, "axis numbers are two bits");
        p.pos = positions->pos;
        p.pos_stride = positions->stride;
        p.axes = positions->axes;
        for (int i = 0; positions->axis_of_pair && i < rope->dim / 2; ++i)       // (dim is at most the head size, 192)
            p.axis_bits[i / 16] |= static_cast<uint32_t>(positions->axis_of_pair[i]) << (2 * (i % 16));
    }
    // the span's vectors before, in and behind its turned part, and the units that they are cut into
    const int before = p.rot_offset / 8, behind = (p.span - p.rot_offset - p.rot_dim) / 8;
    p.before_step = before % 2 == 0 ? 2 : 1;
    p.behind_step = behind % 2 == 0 ? 2 : 1;
    p.before_units = before / p.before_step;
    p.turned_units = p.rot_dim / 16;
    p.span_units = p.before_units + p.turned_units + behind / p.behind_step;
    p.head_units = p.span_units * (p.dqk / p.span);
    p.k_units = p.Hkv * p.head_units;
    p.v_units = p.Hkv * (p.dv / 16);
    p.units = p.k_units + p.v_units + p.Hq * p.head_units;
    if (p.units > 65535) return FA_ERR_UNSUPPORTED;          // (the quotients below are exact up to there)
    auto magic = [](int d) -> uint32_t { return d == 1 ? 0u : static_cast<uint32_t>((0x100000000ull + d - 1) / d); };
    p.head_magic = magic(p.head_units);
    p.span_magic = magic(p.span_units);
    p.v_magic = magic(p.dv / 16);
    p.status = h->status_dev;
    // Tokens of a block: whole rounds of blocks over the four places of every SM (64 registers a thread), as few as
    // kAppendMaxTokens allows, so that a block's look-ups are paid once for many tokens and no round is left half empty.
    const long long places = 4ll * h->num_sms;
    const long long rounds = (total + places * fa::kAppendMaxTokens - 1) / (places * fa::kAppendMaxTokens);
    p.tokens = static_cast<int>((total + places * rounds - 1) / (places * rounds));
    h->last_kernel = "fa_append_paged";
    h->last_splits = 1;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const long long blocks = (static_cast<long long>(total) + p.tokens - 1) / p.tokens;
    if (positions) {
        if (cache->type == FA_CACHE_E4M3) return launch(h, fa::fa_append_paged_kernel<true, true>, blocks, fa::kAppendThreads, 0, st, p);
        return launch(h, fa::fa_append_paged_kernel<false, true>, blocks, fa::kAppendThreads, 0, st, p);
    }
    if (cache->type == FA_CACHE_E4M3) return launch(h, fa::fa_append_paged_kernel<true>, blocks, fa::kAppendThreads, 0, st, p);
    return launch(h, fa::fa_append_paged_kernel<false>, blocks, fa::kAppendThreads, 0, st, p);
}

fa_status fa_forward_paged(fa_handle* h, const fa_paged_cache* cache, const fa_paged_seqs* seqs, const void* Q, void* O, float* lse,
                           int Hq, int Sq, float scale, const int64_t* q_strides, const int64_t* o_strides, void* stream) {
    if (!h) return FA_ERR_INVALID_ARG;
    return forward_paged(h, cache, seqs, Q, O, lse, Hq, Sq, scale, nullptr, q_strides, o_strides, stream);
}

fa_status fa_forward_paged_diff(fa_handle* h, const fa_paged_cache* cache, const fa_paged_seqs* seqs, const void* Q, void* O, int Hq,
                                int Sq, float scale, const fa_diff* diff, const int64_t* q_strides, const int64_t* o_strides,
                                void* stream) {
    if (!h) return FA_ERR_INVALID_ARG;
    const fa_status s = check_diff(diff);
    if (s != FA_OK) return s;
    return forward_paged(h, cache, seqs, Q, O, nullptr, Hq, Sq, scale, diff, q_strides, o_strides, stream);
}

fa_status fa_forward_diff(fa_handle* h, const void* Q, const void* K, const void* V, void* O, int B, int Hq, int Hkv, int Sq, int Sk,
                          int dqk, int dv, int causal, float scale, const fa_diff* diff, const int64_t* q_strides,
                          const int64_t* k_strides, const int64_t* v_strides, const int64_t* o_strides, void* stream) {
    if (!h) return FA_ERR_INVALID_ARG;
    fa_status s = check_diff(diff);
    if (s != FA_OK) return s;
    if (!Q || !K || !V || !O || misaligned(Q, 16) || misaligned(K, 16) || misaligned(V, 16) || misaligned(O, 16)) return FA_ERR_INVALID_ARG;
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Sk <= 0 || Hq % Hkv != 0 || !isfinite(scale) || scale < 0.f) return FA_ERR_INVALID_ARG;
    if (dqk != 128 || dv != 128) return dqk > 0 && dv > 0 ? FA_ERR_UNSUPPORTED : FA_ERR_INVALID_ARG;
    if (!q_strides || !k_strides || !v_strides || !o_strides) return FA_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i) {
        if (q_strides[i] <= 0 || k_strides[i] <= 0 || v_strides[i] <= 0 || o_strides[i] <= 0) return FA_ERR_INVALID_ARG;
        if ((q_strides[i] | k_strides[i] | v_strides[i] | o_strides[i]) & 7) return FA_ERR_INVALID_ARG;
    }
    if (q_strides[2] < dqk || k_strides[2] < dqk || v_strides[2] < dv || o_strides[2] < dv) return FA_ERR_INVALID_ARG;
    if (Hq > 65535 || B > 65535 || static_cast<int64_t>(B) * Hq > 0x7fffffffLL || Sq > 0x7fffff00 || Sk > 0x7fffff00) return FA_ERR_UNSUPPORTED;
    DeviceGuard guard(h->device);
    if (!guard.ok()) return FA_ERR_CUDA;
    if (scale == 0.f) scale = 0.125f;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!(h->flags & FA_FLAG_SERIAL_KERNEL)) {
        const CUtensorMap* m = nullptr;
        if ((s = get_map(h, Q, 128, Sq, Hq, B, q_strides[0], q_strides[1], q_strides[2], fa::kTileM, &m)) != FA_OK) return s;
        const CUtensorMap mq = *m;       // copies: a later insertion may move the cache's entries
        if ((s = get_map(h, K, 128, Sk, Hkv, B, k_strides[0], k_strides[1], k_strides[2], fa::kTileN, &m)) != FA_OK) return s;
        const CUtensorMap mk = *m;
        if ((s = get_map(h, V, 128, Sk, Hkv, B, v_strides[0], v_strides[1], v_strides[2], fa::kTileN, &m)) != FA_OK) return s;
        const CUtensorMap mv = *m;
        if ((s = get_map(h, O, 128, Sq, Hq, B, o_strides[0], o_strides[1], o_strides[2], fa::kTileM, &m)) != FA_OK) return s;
        const CUtensorMap mo = *m;
        fa::FwdParams f;
        memset(&f, 0, sizeof f);
        f.B = B; f.Hq = Hq; f.Hkv = Hkv; f.Sq = Sq; f.Sk = Sk;
        f.causal = causal ? 1 : 0;
        f.scale_log2 = scale * 1.4426950408889634f;
        f.n_q_tiles = (Sq + fa::kTileM - 1) / fa::kTileM;
        f.heads_per_group = heads_per_group(static_cast<long long>(Sk) * 512, B, Hq, Hkv);
        f.kv_splits = 1;
        f.sched_counter = h->sched_counter;
        f.status = h->status_dev;
        f.wait_limit_ns = h->wait_limit_ns;
        f.debug_drop_v_load = (h->flags & FA_FLAG_DEBUG_DROP_V_LOAD) ? 1 : 0;
        const fa::DiffParams dp{diff->lambda, diff->weight, diff->eps, diff->out_scale};
        constexpr int smem = fa::diff_smem_bytes();
        static_assert(smem <= 227 * 1024, "shared memory budget exceeded");
        if ((s = ensure_smem_attr(h, fa::fa_fwd_diff_kernel, smem)) != FA_OK) return s;
        h->last_kernel = "fa_fwd_diff";
        h->last_splits = 1;
        const long long items = static_cast<long long>(f.n_q_tiles) * Hq * B;
        if (items > 0x3fffffffLL) return FA_ERR_UNSUPPORTED;
        return launch(h, fa::fa_fwd_diff_kernel, items < h->num_sms ? items : h->num_sms, fa::DiffCfg::kThreads, smem, st, mq, mk, mv, mo, f, dp);
    }
    fa::PagedParams p;
    memset(&p, 0, sizeof p);
    p.Q = static_cast<const __nv_bfloat16*>(Q);
    p.O = static_cast<__nv_bfloat16*>(O);
    p.q_sb = q_strides[0]; p.q_sh = q_strides[1]; p.q_st = q_strides[2];
    p.o_sb = o_strides[0]; p.o_sh = o_strides[1]; p.o_st = o_strides[2];
    p.k = K; p.v = V;
    for (int i = 0; i < 3; ++i) { p.k_stride[i] = k_strides[i]; p.v_stride[i] = v_strides[i]; }
    p.B = B; p.num_pages = B; p.page_size = Sk; p.fixed_len = Sk;
    p.Hq = Hq; p.Hkv = Hkv; p.Sq = Sq;
    p.causal = causal ? 1 : 0;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.lambda = diff->lambda; p.weight = diff->weight; p.eps = diff->eps; p.out_scale = diff->out_scale;
    p.status = h->status_dev;
    return launch_simple<false, true>(h, 128, p, st);
}

fa_status fa_plan_paged(int num_sms, const fa_config* cfg, const fa_paged_cache* cache, const fa_paged_seqs* seqs, int Hq, int Sq,
                        int diff, fa_paged_plan_info* out, fa_paged_piece* pieces, int max_pieces) {
    if (num_sms <= 0 || !cache || !seqs || !out || cache->struct_size != sizeof(fa_paged_cache) || seqs->struct_size != sizeof(fa_paged_seqs))
        return FA_ERR_INVALID_ARG;
    if (cache->page_size <= 0 || cache->Hkv <= 0 || Hq <= 0 || Sq <= 0 || Hq % cache->Hkv != 0 || seqs->B <= 0 || seqs->max_pages <= 0 ||
        !seqs->seq_lens || max_pieces < 0 || (max_pieces > 0 && !pieces)) return FA_ERR_INVALID_ARG;
    if (!head_sizes_ok(cache->dqk, cache->dv) || cache->page_size % 16 != 0 || Sq > FA_PAGED_MAX_SQ || Hq > 65535 || seqs->B > 65535 ||
        (diff && (cache->dqk != 128 || cache->dv != 128)) || static_cast<int64_t>(seqs->max_pages) * cache->page_size > 0x7fffff00LL)
        return FA_ERR_UNSUPPORTED;
    uint64_t scratch = 32ull << 20;
    if (cfg) {
        if (cfg->struct_size < 16) return FA_ERR_INVALID_ARG;
        if (cfg->struct_size >= sizeof(fa_config) && cfg->scratch_bytes) scratch = cfg->scratch_bytes;
    }
    fa::PagedParams p;
    memset(&p, 0, sizeof p);
    p.seq_lens = seqs->seq_lens;
    p.B = seqs->B; p.max_pages = seqs->max_pages; p.page_size = cache->page_size; p.Hkv = cache->Hkv; p.Hq = Hq; p.Sq = Sq;
    return plan_paged(num_sms, static_cast<size_t>(scratch), p, cache->dqk, cache->dv, cache->type == FA_CACHE_E4M3, diff != 0, false, out, pieces, max_pieces);
}

}  // extern "C"
