// Host side of fa_forward_paged_tree (include/fa.h): argument checks, tensor maps, launch.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <memory>
#include <new>

#include "../../include/fa.h"
#include "fa_handle.h"
#include "fa_paged_common.cuh"
#include "fa_paged_host.h"
#include "fa_tree.cuh"
#include "fa_tree_simple.cuh"

namespace fa_host {      // (fa_tree_few.cu)

fa_status launch_tree_few(fa_handle* h, int dqk, int dv, bool e4m3, const CUtensorMap& mk, const CUtensorMap& mv, fa::PagedParams& p, cudaStream_t st);
fa_status plan_tree_few(int num_sms, size_t scratch, fa::PagedParams& p, int dqk, int dv, bool e4m3, fa_paged_plan_info* out, fa_paged_piece* pieces,
                        int max_pieces);

}  // namespace fa_host

namespace {

using namespace fa_host;

// Few rows are columns of turned products, many are lanes: a pass over the keys costs the streaming kernel's softmax warps what the rows
// are, and this one 128 rows whatever they are.  64 sequences of 300 keys, 64/8 heads of 128: 8 rows 17.2 us against 40.5, 32 rows 24.3
// against 38.0, 64 rows (forward_paged's time) 49.5 against 36.8; 48 of 4200 keys over e4m3 71.8 against 117.9, 79.8 against 126.2, 64 rows
// 140 against 125.  (The largest loss: one sequence of 8000 keys, 32/8 heads, 32 rows, 20.0 against 18.6.)
bool few_rows(int group, int max_tokens) { return static_cast<long long>(group) * max_tokens <= 32; }

template <bool kE4m3>
fa_status launch_simple(fa_handle* h, int dqk, const fa::PagedParams& p, const fa::TreeParams& tp, cudaStream_t st) {
    const long long blocks = static_cast<long long>(tp.total) * p.Hq;
    h->last_kernel = "fa_tree_simple";
    h->last_splits = 1;
    if (dqk == 64) return launch(h, fa::fa_tree_simple_kernel<64, 64, kE4m3>, blocks, 128, 0, st, p, tp);
    if (dqk == 192) return launch(h, fa::fa_tree_simple_kernel<192, 128, kE4m3>, blocks, 128, 0, st, p, tp);
    return launch(h, fa::fa_tree_simple_kernel<128, 128, kE4m3>, blocks, 128, 0, st, p, tp);
}

// How the list of work is made (fa_tree.cuh).  A row tile's tokens are as many as fit, and no more than a sequence can have.  A tile of keys
// counts what it takes: two row tiles have twice the exponentials.  What a block costs beside its tiles is some four tiles' time (16 sequences
// of 129 to 8192 keys, 64 drafts: 73.4 us counted as one unit, 69.2 as four, 67.0 as eight; 48 over e4m3 168.4, 168.8 and 171.6).
fa::TreeList make_list(int group, int max_tokens, int dqk, bool e4m3) {
    fa::TreeList li;
    li.row_heads = group < 128 ? group : 128;
    li.head_chunks = (group + li.row_heads - 1) / li.row_heads;
    li.row_tokens = 128 / li.row_heads < max_tokens ? 128 / li.row_heads : max_tokens;
    li.two = dqk != 192 && !e4m3;      // (as in TreeCfg)
    li.token_magic = li.row_tokens == 1 ? 0u : static_cast<uint32_t>((0x100000000ull + li.row_tokens - 1) / li.row_tokens);
    li.w1 = 1;
    li.w2 = li.two ? 2 : 1;
    li.cost = 4;
    li.least = 2 * li.w2;
    li.pad = 0;
    return li;
}

// Whether a call's list can have more units than are counted.  (With few rows too: the streaming kernel's has no more tiles, and three units
// beside them at most.)
bool too_long(const fa::TreeList& li, int B, int Hkv, int max_tokens, long long most_keys) {
    const long long row_tiles = fa::tree_row_tiles(li, max_tokens), most_tiles = (most_keys + fa::kTileN - 1) / fa::kTileN;
    return static_cast<long long>(B) * Hkv > kMostUnits / row_tiles / (most_tiles * li.w2 + li.cost);
}

// CTAs of a launch: one per SM, as far as the scratch has two partial results and an entry of the list of what is joined for each.
int tree_ctas(int num_sms, size_t scratch_bytes, int dv, bool two) {
    const long long fit = static_cast<long long>(scratch_bytes / (2 * sizeof(float) * fa::tree_slot_floats(dv, two) + sizeof(fa::TreeJoin)));
    return static_cast<int>(fit < num_sms ? fit : num_sms);
}

template <int DQK, int DV, bool kE4m3>
fa_status launch_tree(fa_handle* h, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const fa::PagedParams& p, fa::TreeArgs& a,
                      cudaStream_t st) {
    using Cfg = fa::TreeCfg<DQK, DV, kE4m3>;
    constexpr int smem = fa::tree_smem_bytes<DQK, DV, kE4m3>();
    static_assert(smem <= 227 * 1024, "shared memory budget exceeded");
    const int ctas = tree_ctas(h->num_sms, h->tree_scratch_bytes, DV, Cfg::kTwo);
    if (ctas < 1) return FA_ERR_UNSUPPORTED;
    a.part = static_cast<float*>(h->scratch);
    a.join = reinterpret_cast<fa::TreeJoin*>(a.part + 2ll * ctas * fa::tree_slot_floats(DV, Cfg::kTwo));
    auto kernel = fa::fa_tree_kernel<DQK, DV, kE4m3>;
    fa_status s = ensure_smem_attr(h, kernel, smem);
    if (s != FA_OK) return s;
    if ((s = launch(h, kernel, ctas, Cfg::kThreads, smem, st, mq, mk, mv, p, a)) != FA_OK) return s;
    return launch(h, fa::fa_tree_join_kernel<DV, Cfg::kTwo>, static_cast<long long>(ctas) * 4 * (Cfg::kTwo ? 2 : 1), 2 * DV, 0, st, p, a);
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
    const bool e4m3 = cache->type == FA_CACHE_E4M3;
    if (h->flags & FA_FLAG_SERIAL_KERNEL) return e4m3 ? launch_simple<true>(h, cache->dqk, p, tp, st) : launch_simple<false>(h, cache->dqk, p, tp, st);
    fa::TreeArgs a;
    memset(&a, 0, sizeof a);
    a.t = tp;
    a.group = Hq / cache->Hkv;
    a.list = make_list(a.group, tree->max_tokens, cache->dqk, e4m3);
    if (too_long(a.list, seqs->B, cache->Hkv, tree->max_tokens, static_cast<long long>(seqs->max_pages) * cache->page_size)) return FA_ERR_UNSUPPORTED;
    p.box_rows = 16;
    while (p.box_rows < 128 && cache->page_size % (2 * p.box_rows) == 0) p.box_rows *= 2;
    const int eb = e4m3 ? 1 : 2;
    const CUtensorMap* m = nullptr;
    const bool few = few_rows(a.group, tree->max_tokens);
    CUtensorMap mq = {};
    // (queries: heads in the place of rows, tokens in that of heads; one head may have any stride)
    if (!few) {
        if ((s = get_map(h, Q, cache->dqk, Hq, total, 1, q_strides[0], q_strides[0], q_strides[1], a.list.row_heads, &m, 2, a.list.row_tokens)) != FA_OK) return s;
        mq = *m;                     // copies: a later insertion may move the cache's entries
    }
    if ((s = get_map(h, cache->k, cache->dqk, cache->page_size, cache->Hkv, cache->num_pages, cache->k_strides[0], cache->k_strides[1],
                     cache->k_strides[2], p.box_rows, &m, eb, 1, 128, map_promotion(cache->dqk, eb, cache->k_strides))) != FA_OK) return s;
    const CUtensorMap mk = *m;
    if ((s = get_map(h, cache->v, cache->dv, cache->page_size, cache->Hkv, cache->num_pages, cache->v_strides[0], cache->v_strides[1],
                     cache->v_strides[2], p.box_rows, &m, eb, 1, 128, map_promotion(cache->dv, eb, cache->v_strides))) != FA_OK) return s;
    const CUtensorMap mv = *m;
    if (few) {
        p.Sq = tree->max_tokens;
        p.cu_seqlens = tree->cu_seqlens; p.mask = tree->mask; p.mask_stride = tree->mask_stride; p.total = total;
        return launch_tree_few(h, cache->dqk, cache->dv, e4m3, mk, mv, p, st);
    }
    h->last_kernel = e4m3 ? "fa_tree_e4m3" : "fa_tree";
    h->last_splits = 1;
    if (cache->dqk == 64) return e4m3 ? launch_tree<64, 64, true>(h, mq, mk, mv, p, a, st) : launch_tree<64, 64, false>(h, mq, mk, mv, p, a, st);
    if (cache->dqk == 192) return e4m3 ? launch_tree<192, 128, true>(h, mq, mk, mv, p, a, st) : launch_tree<192, 128, false>(h, mq, mk, mv, p, a, st);
    return e4m3 ? launch_tree<128, 128, true>(h, mq, mk, mv, p, a, st) : launch_tree<128, 128, false>(h, mq, mk, mv, p, a, st);
}

fa_status fa_plan_paged_tree(int num_sms, const fa_config* cfg, const fa_paged_cache* cache, const fa_paged_seqs* seqs, const fa_tree* tree, int total,
                             int Hq, fa_paged_plan_info* out, fa_paged_piece* pieces, int max_pieces) {
    if (num_sms <= 0 || !cache || !seqs || !tree || !out || cache->struct_size != sizeof(fa_paged_cache) || seqs->struct_size != sizeof(fa_paged_seqs) ||
        tree->struct_size != sizeof(fa_tree)) return FA_ERR_INVALID_ARG;
    if (cache->page_size <= 0 || cache->Hkv <= 0 || Hq <= 0 || Hq % cache->Hkv != 0 || seqs->B <= 0 || seqs->max_pages <= 0 || !seqs->seq_lens ||
        tree->max_tokens <= 0 || total <= 0 || max_pieces < 0 || (max_pieces > 0 && !pieces)) return FA_ERR_INVALID_ARG;
    if (!tree->cu_seqlens && (total % seqs->B != 0 || total / seqs->B > tree->max_tokens)) return FA_ERR_INVALID_ARG;
    if (!head_sizes_ok(cache->dqk, cache->dv) || cache->page_size % 16 != 0 || tree->max_tokens > FA_TREE_MAX_TOKENS || Hq > 65535 || seqs->B > 65535 ||
        static_cast<int64_t>(seqs->max_pages) * cache->page_size > 0x7fffff00LL) return FA_ERR_UNSUPPORTED;
    uint64_t scratch = 40ull << 20;
    if (cfg) {
        if (cfg->struct_size < 16) return FA_ERR_INVALID_ARG;
        if (cfg->struct_size >= sizeof(fa_config) && cfg->scratch_bytes) scratch = cfg->scratch_bytes;
    }
    fa::TreeList li = make_list(Hq / cache->Hkv, tree->max_tokens, cache->dqk, cache->type == FA_CACHE_E4M3);
    if (too_long(li, seqs->B, cache->Hkv, tree->max_tokens, static_cast<long long>(seqs->max_pages) * cache->page_size)) return FA_ERR_UNSUPPORTED;
    const int B = seqs->B;
    const fa::TreeSeqs seq_of{tree->cu_seqlens, seqs->seq_lens, B, total, tree->max_tokens, seqs->max_pages, cache->page_size};
    if (few_rows(Hq / cache->Hkv, tree->max_tokens)) {
        // (a sequence without drafts counts as one without keys)
        std::unique_ptr<int32_t[]> lens(new (std::nothrow) int32_t[B]);
        if (!lens) return FA_ERR_CUDA;
        for (int b = 0; b < B; ++b) {
            int n, row0, len;
            seq_of(b, n, row0, len);
            lens[b] = n > 0 ? len : 0;
        }
        fa::PagedParams p;
        memset(&p, 0, sizeof p);
        p.seq_lens = lens.get();
        p.B = B; p.max_pages = seqs->max_pages; p.page_size = cache->page_size; p.Hkv = cache->Hkv; p.Hq = Hq; p.Sq = tree->max_tokens;
        return plan_tree_few(num_sms, std::min(scratch, static_cast<uint64_t>(32) << 20), p, cache->dqk, cache->dv, cache->type == FA_CACHE_E4M3, out,
                             pieces, max_pieces);
    }
    const int ctas = tree_ctas(num_sms, scratch, cache->dv, li.two != 0);
    if (ctas < 1) return FA_ERR_UNSUPPORTED;
    auto units_of = [&](int b) {
        int n, row0, len;
        seq_of(b, n, row0, len);
        return cache->Hkv * fa::tree_head_units(fa::tree_units(li, n, len));
    };
    fa::TreeBatch batch{0, 0, 0, 0x7fffffff, 0};
    for (int b = 0; b < B; ++b) {
        int n, row0, len;
        seq_of(b, n, row0, len);
        const fa::TreeUnits u = fa::tree_units(li, n, len);
        batch.units += cache->Hkv * fa::tree_head_units(u);
        if (n == 0) continue;
        const int nt = fa::tree_tiles(len);
        batch.blocks += cache->Hkv * (u.pairs + (u.single ? 1 : 0));
        batch.longest = nt > batch.longest ? nt : batch.longest;
        batch.shortest = nt < batch.shortest ? nt : batch.shortest;
        batch.kinds |= (u.pairs ? 1 : 0) | (u.single ? 2 : 0);
    }
    int share = fa::tree_rules(li, batch, ctas), all = 0;
    for (int b = 0; b < B; ++b) all += units_of(b);
    if (share == 0) share = fa::tree_share(li, all, ctas);
    out->rows_per_block = li.row_tokens * li.row_heads;
    out->row_blocks = fa::tree_row_tiles(li, tree->max_tokens);
    out->ctas = ctas;
    out->part_cost = li.cost;
    out->units = all;
    out->units_per_cta = share;
    long long n_pieces = 0;
    int b0 = 0, base0 = 0;             // the sequence that the CTA's share begins in, and its first unit
    for (int c = 0; c < ctas && static_cast<long long>(c) * share < all; ++c) {
        while (c * share >= base0 + units_of(b0)) base0 += units_of(b0++);
        fa::TreeWalk w;
        seq_of(b0, w.n, w.row0, w.len);
        fa::tree_walk_begin(w, li, c, share, all, b0, base0);
        fa::TreePart e;
        while (fa::tree_walk_next(w, li, cache->Hkv, seq_of, e)) {
            if (n_pieces < max_pieces) {
                fa_paged_piece* x = pieces + n_pieces;
                x->cta = c;
                x->sequence = e.b;
                x->kv_head = e.kvh;
                x->row_block = e.row_tile;
                x->first_tile = e.t0;
                x->end_tile = e.t1;
                x->slot = e.slot;
                x->pieces = e.pieces;
                x->first_cta = e.first_cta;
            }
            ++n_pieces;
        }
    }
    out->pieces = n_pieces;
    return FA_OK;
}

}  // extern "C"
