// The streaming kernel's list of work, launch and plan (fa_paged.cuh), for the entry points that use it.
#pragma once

#include <stdint.h>

#include "fa_paged.cuh"
#include "fa_paged_host.h"

namespace fa_host {

// Units of 128 keys that a CTA of the streaming kernel takes at least: two softmax groups work on two tiles at once, and every piece of
// a row block more is one more to join (2000 keys, 8 K/V heads: 14.8 us, against 17.9 with one; 14.6 with four, but 100 to
// 400 keys lose 1.5 us there).
constexpr int kLeastUnits = 2;

// Query rows per block: 16 where they suffice, else 32 or 64, as far as the accumulators (S^T and O^T of both groups, three times the
// columns over an 8-bit cache, four times with two maps) and two stages of tiles fit.
inline int rows_per_block(int rows, int dqk, bool e4m3, bool diff) {
    if (rows <= 16 || diff) return 16;
    return rows > 32 && !e4m3 && dqk != 192 ? 64 : 32;
}

// Units that a call's list of work can have at most (kMostUnits).
inline long long most_units(const fa::PagedParams& p) {
    return static_cast<long long>(p.B) * p.Hkv * p.row_blocks *
           (fa::paged_tiles(static_cast<int>(static_cast<long long>(p.max_pages) * p.page_size)) + fa::kMostPartCost);
}

// CTAs of a launch: one per SM, as many as there can be units, and as many as the scratch has two partial results for.
inline int paged_ctas(int num_sms, size_t scratch_bytes, const fa::PagedParams& p, int dv, int states) {
    long long ctas = num_sms;
    if (ctas > most_units(p)) ctas = most_units(p);
    const long long fit = static_cast<long long>(scratch_bytes / (2 * fa::paged_slot_bytes(dv, states)));
    return static_cast<int>(ctas > fit ? fit : ctas);
}

// The list's constants (fa_paged.cuh): the units that a row block counts beside its tiles are what 128 KB of tiles are, and it
// counts them up to 768 KB.
inline void set_list(fa::PagedParams& p, int dqk, int dv, bool e4m3) {
    const int tile = 128 * (dqk + dv) * (e4m3 ? 1 : 2), units = (128 << 10) / tile;
    p.least_units = kLeastUnits;
    p.part_cost = units > fa::kMostPartCost ? fa::kMostPartCost : units;
    p.long_tiles = (768 << 10) / tile;
}

// The streaming kernel with blocks of kRows query rows.
template <int DQK, int DV, bool kE4m3, bool kDiff, int kRows, bool kTree = false>
fa_status launch_paged(fa_handle* h, const CUtensorMap& mk, const CUtensorMap& mv, fa::PagedParams& p, cudaStream_t st) {
    using Cfg = fa::PagedCfg<DQK, DV, kE4m3, kDiff, kRows>;
    constexpr int smem = fa::paged_smem_bytes<DQK, DV, kE4m3, kDiff, kRows, kTree>();
    static_assert(smem <= 227 * 1024, "shared memory budget exceeded");
    const int ctas = paged_ctas(h->num_sms, h->scratch_bytes, p, DV, Cfg::kStates);
    if (ctas < 1) return FA_ERR_UNSUPPORTED;
    p.part = static_cast<float*>(h->scratch);
    p.arrivals = h->arrivals;
    auto kernel = fa::fa_paged_kernel<DQK, DV, kE4m3, kDiff, kRows, kTree>;
    const fa_status s = ensure_smem_attr(h, kernel, smem);
    if (s != FA_OK) return s;
    h->last_kernel = kTree ? (kE4m3 ? "fa_tree_few_e4m3" : "fa_tree_few") : kE4m3 ? "fa_paged_e4m3" : "fa_paged";
    h->last_splits = 1;
    return launch(h, kernel, ctas, 512, smem, st, mk, mv, p);
}

// How a batch is dealt out (p: its lengths on the host, B, max_pages, page_size, Hq, Hkv, Sq).
inline fa_status plan_paged(int num_sms, size_t scratch, fa::PagedParams& p, int dqk, int dv, bool e4m3, bool diff, bool tree,
                            fa_paged_plan_info* out, fa_paged_piece* pieces, int max_pieces) {
    const int rows = p.Hq / p.Hkv * p.Sq, block = rows_per_block(rows, dqk, e4m3, diff);
    p.row_blocks = (rows + block - 1) / block;
    set_list(p, dqk, dv, e4m3);
    if (most_units(p) > kMostUnits) return FA_ERR_UNSUPPORTED;
    const int ctas = paged_ctas(num_sms, scratch, p, dv, (diff ? 2 : 1) * block);
    if (ctas < 1) return FA_ERR_UNSUPPORTED;
    int longest = 0, total = 0;
    for (int b = 0; b < p.B; ++b) {
        const int n = fa::paged_len(p, b, nullptr);
        longest = n > longest ? n : longest;
        total += fa::paged_units(p, n, fa::PagedCount{0, 0, 0});
    }
    const int least = fa::paged_least(p, tree, fa::paged_tiles(longest));
    const fa::PagedCount cnt = fa::paged_count(p, least, ctas, fa::paged_tiles(longest), total);
    auto units_of = [&](int b) { return fa::paged_units(p, fa::paged_len(p, b, nullptr), cnt); };
    total = 0;
    for (int b = 0; b < p.B; ++b) total += units_of(b);
    const int share = fa::paged_share(least, total, ctas, cnt);
    out->rows_per_block = block;
    out->row_blocks = p.row_blocks;
    out->ctas = ctas;
    out->part_cost = cnt.cost;
    out->units = total;
    out->units_per_cta = share;
    long long n = 0;
    int b0 = 0, base0 = 0;             // the sequence that the CTA's share begins in, and its first unit
    for (int c = 0; c < ctas && static_cast<long long>(c) * share < total; ++c) {
        const int u0 = c * share, u1 = total - u0 < share ? total : u0 + share;
        while (u0 >= base0 + units_of(b0)) base0 += units_of(b0++);
        for (int b = b0, base = base0; b < p.B && base < u1; base += units_of(b), ++b) {
            for (int hr = 0; hr < p.Hkv * p.row_blocks; ++hr) {
                fa::PagedEntry e;
                if (!fa::paged_entry(p, c, share, u0, u1, b, base, fa::paged_len(p, b, nullptr), cnt, hr, e)) continue;
                if (n < max_pieces) {
                    fa_paged_piece* x = pieces + n;
                    x->cta = c;
                    x->sequence = e.b;
                    x->kv_head = e.kvh;
                    x->row_block = e.rb;
                    x->first_tile = e.t0;
                    x->end_tile = e.t1;
                    x->slot = e.slot;
                    x->pieces = e.pieces;
                    x->first_cta = e.first_cta;
                }
                ++n;
            }
        }
    }
    out->pieces = n;
    return FA_OK;
}

}  // namespace fa_host
