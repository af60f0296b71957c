// Attention of drafted tokens over a paged key/value cache, for sm_100a.
//
// A tree of n drafts gives R = n * (Hq / Hkv) query rows per (sequence, K/V head), more than 32 here (fewer are the work of fa_paged.cuh),
// against thousands of keys that all of them see and n that a mask of bits decides about.  2 R (dqk + dv) flops stand against (dqk + dv) * bytes a key: up to 256
// rows over a 16-bit cache HBM is the bound, behind that the tensor cores and, as in every kernel here, the exponentials.  So a CTA
// takes up to 256 rows in one pass over the keys, as two tiles of 128 rows on the accumulator's lanes:
//
//   * Two streams t = 0, 1, each with scores S_t, probabilities P_t and accumulator O_t, the loop of fa_fwd_pair.cuh (read that file
//     first).  With more than 128 rows the streams are the two row tiles and share every K/V tile; with up to 128 they are the even
//     and the odd K/V tiles of the same rows, merged at the end.  Either way one stream's softmax runs under the other's MMAs.
//     (192/128 and e4m3 caches have no room for a second query tile: always the latter.)  P_t lies over S_t, or where there is room
//     (head size 64, e4m3 at 128) in shared memory, and the next scores need not wait for P_t V (e4m3 198 to 168 us).
//   * A row tile is tt tokens x ht heads of the group (ht = the group, tt = 128 / ht), which is one TMA box of Q: rows lie in the tile as
//     token, head.  Rows that the sequence does not have are computed and not stored.
//   * The tiles of all (sequence, K/V head, row block)s form one list that the CTAs cut into equal consecutive shares on the device, as
//     in fa_paged.cuh.  What several CTAs share is joined by a second kernel: its pieces are up to 130 KB each, which the CTA that
//     finishes last would read alone at the speed of one SM (up to three pieces joined that way: 71.4 us, against 68.6).
//   * The mask concerns the last tiles alone: a thread has one row, takes its bits for 32 keys out of the row's words by a funnel shift,
//     and hides keys past the length with the same bits.
//
// What bounds it.  16 sequences of 129 to 8192 keys, trees of 16 to 64 drafts, 32/8 heads of 128, bf16: 68.1 us, where 248 MB take 38 at the
// copy rate.  With 256 rows a tile of keys takes a CTA 3000 cycles, the chain softmax (2000) -> P V and next scores (1024 cycles of MMAs) of each
// stream; the list gives most CTAs 20 to 24 such tiles in one to three parts.  That is 60 to 72 thousand of this kernel's 110 (65.2 us at
// 1.70 GHz): the rest is 9000 from the launch to the first scores (list, block table, first loads), some 6000 from one part's last tile to
// the next one's first (result, barrier, first pass), and what has not been taken apart.  The join takes 5 us more.
// 48 sequences of 300 to 8192 keys over e4m3, 13 drafts, 64/8 heads: 153 us, where 521 MB take 80: two tiles take 3600 cycles, of which MMAs
// 2630 (8-bit scores in three terms, fp16 products).  Most CTAs have 105 to 113 tiles in three or four parts, 190 to 203 thousand of 266
// thousand cycles (158.6 us at 1.68 GHz): a quarter lies outside of the loop over the tiles, not taken apart yet.  (A part's beginning is
// a chain here: queries loaded when the last scores of the part before are done, turned into terms, then the first values into fp16.)
//
// Over an e4m3 cache K is multiplied as it is (kind::f8f6f4), the queries as three e5m2 terms like in fa_paged.cuh, added up in one
// accumulator (half as many MMAs again); P V is an fp16 product, since terms of P would be work of the softmax warps, which are the
// bound: four more warps turn V's codes into fp16, which holds them exactly, and P is scaled by 2^7.  (K through fp16 too: 255 us, 48
// sequences of 300 to 8192 keys, 13 drafts, 64/8 heads; the conversions slow the softmax down by what they share with it.)
//
// Roles: warps 0-3 / 4-7 softmax of stream 0 / 1 and results, warp 8 MMA issue, warp 9 loads of K, warp 10 of Q and V, warp 11 the list
// and the zeros behind a sequence's last value, over e4m3 caches warps 12-15 the terms of Q and the codes of V.
// TMEM: S_0 [0,128) S_1 [128,256) O_0 [256,384) O_1 [384,512); P_t over S_t[0,64), where it is not in shared memory.
#pragma once

#include <cuda_fp16.h>
#include <float.h>
#include <math.h>

#include "fa_common.cuh"
#include "fa_fwd_pair.cuh"
#include "fa_paged_common.cuh"
#include "fa_tree_simple.cuh"
#include "ptx.cuh"

namespace fa {

// ------------------------------------------------------------------ the list of work units and its shares

// A row block (up to two row tiles of a sequence and K/V head) has `cost` units for what it takes beside its tiles, and then `w2` or `w1` units
// per tile of 128 keys, as it has two row tiles or one; with `pad` it counts as many tiles at least.  A tile belongs to the CTA whose
// share its first unit is in.
struct TreeList {
    int row_tokens, row_heads;    // tokens and heads of a row tile
    uint32_t token_magic;         // ceil(2^32 / row_tokens): exact quotients of numbers below 2^16 (0: row_tokens is 1)
    int head_chunks;              // row tiles that a token's group is cut into
    int two;                      // blocks have two row tiles where there are two
    int cost, w1, w2, least, pad;
};
// Row tiles of n drafts.
__host__ __device__ inline int tree_row_tiles(const TreeList& li, int n) {
    const uint32_t x = static_cast<uint32_t>(n + li.row_tokens - 1);
    const int tiles = li.token_magic ? static_cast<int>((static_cast<unsigned long long>(x) * li.token_magic) >> 32) : static_cast<int>(x);
    return li.head_chunks == 1 ? tiles : tiles * li.head_chunks;
}
__host__ __device__ inline int tree_tiles(int len) { return (len + kTileN - 1) / kTileN; }
struct TreeUnits { int pairs, pair, single; };      // blocks of two row tiles, units of each, units of the one behind them (0: none)
__host__ __device__ inline TreeUnits tree_units(const TreeList& li, int n, int len) {
    const int rt = tree_row_tiles(li, n), nt = tree_tiles(len) > li.pad ? tree_tiles(len) : li.pad;
    TreeUnits u;
    if (li.two) {
        u.pairs = rt / 2;
        u.pair = li.cost + li.w2 * nt;
        u.single = rt % 2 ? li.cost + li.w1 * nt : 0;
    } else {
        u.pairs = rt;
        u.pair = li.cost + li.w1 * nt;
        u.single = 0;
    }
    return u;
}
__host__ __device__ inline int tree_head_units(const TreeUnits& u) { return u.pairs * u.pair + u.single; }

// What a batch is, as far as the rules below ask: row blocks, units, key tiles of its longest and shortest sequence, whether blocks of one and of
// two row tiles are among it.
struct TreeBatch { int blocks, units, longest, shortest, kinds; };
constexpr int kTreeSplitCost = 3;
// Tiles of a piece at least: a tile takes its CTA about four times what a piece takes the joining kernel, so pieces of s tiles cost
// s + tiles / (4 s), which is least where s is half the root of the tiles (one sequence of 17353 keys, one K/V head, 64 drafts of 8 heads: 53.3 us in pieces as small as the
// CTAs allow, 30.3 so; 100000 and 33333 keys, 13 drafts 66.7, 47.9).
__host__ __device__ inline int tree_root(int tiles) { return static_cast<int>(ceilf(0.5f * sqrtf(static_cast<float>(tiles)))); }
// Small batches.  Where there is a CTA for every block, the longest block, unsplit, is what the call takes; split, it takes an equal share and
// what the join of the pieces costs, about three tiles' time.  Where that is not less, all blocks count the same and nothing is split (16
// sequences of 1003 keys, 8 K/V heads, 9 drafts of 4 heads: 18.1 us, against 20.8 split; over e4m3, 5 drafts of 8 heads, 21.0 against 25.1; one
// of 500 keys, 26 drafts: 12.2 split, against 13.7).  Where
// there are two CTAs for every block at least and all are equally long, their pieces are equally long too, and a CTA has one.  No share
// is smaller than a piece of the longest sequence should be (tree_root).  Returns the share (0: what the total gives).
__host__ __device__ inline int tree_rules(TreeList& li, const TreeBatch& b, int ctas) {
    const int w = b.kinds & 1 ? li.w2 : li.w1;
    if (b.blocks <= ctas && li.cost + w * (b.longest - kTreeSplitCost) <= b.units / ctas) {
        li.w1 = li.w2 = w;
        li.pad = b.longest;
        return li.cost + li.w2 * li.pad;
    }
    if (2 * b.blocks <= ctas && b.longest == b.shortest && b.longest > 0 && b.kinds != 3) {
        const int pieces = ctas / b.blocks, per = (b.longest + pieces - 1) / pieces;
        li.cost = 0;
        li.w1 = li.w2 = 1;
        const int root = tree_root(b.longest), least = root < 2 ? 2 : root, share = per < least ? least : per;
        li.pad = (b.longest + share - 1) / share * share;
        return share;
    }
    if (w * tree_root(b.longest) > li.least) li.least = w * tree_root(b.longest);
    return 0;
}
__host__ __device__ inline int tree_share(const TreeList& li, int total, int ctas) {
    const int per = static_cast<int>((static_cast<unsigned>(total) + ctas - 1) / ctas);
    return per < li.least ? li.least : per;
}

// A part of the list as the roles of a CTA see it: tiles [t0, t1) of one row block.
struct TreePart {
    int b, kvh, row_tile, two;    // first row tile; whether the block has a second one
    int len, n, row0;             // keys, drafts and first row of the sequence
    int t0, t1;                   // t1 < 0: the end of the CTA's share
    int tile0;                    // index of the part's first tile in the CTA's share
    int slot;                     // of the partial result, -1: the part is whole
    int pieces, first_cta;        // of the whole block, and the CTA of its first piece
};
// A row block in several pieces as the joining kernel sees it, one per CTA (the one with the first piece; pieces = 0: none).  Piece 0
// is in slot 2 * CTA + 1, piece i in slot 2 * (CTA + i).
struct TreeJoin { int kvh, row_tile, two, n, row0, pieces, unused0, unused1; };

// Tiles [t0, t1) that units [u0, u1) hold of a block of nt tiles whose first unit is ub.
__host__ __device__ inline int tree_tile_at(int u, int ub, int cost, int w, int nt) {
    const int x = u - ub - cost;
    const int t = x <= 0 ? 0 : w == 1 ? x : (x + 1) >> 1;         // (w is 1 or 2)
    return t < nt ? t : nt;
}

// A sequence's drafts, its first row and its length, as the list takes them (and without reports).
struct TreeSeqs {
    const int* cu_seqlens;
    const int* seq_lens;
    int B, total, max_tokens, max_pages, page_size;
    __host__ __device__ void operator()(int b, int& n, int& row0, int& len) const {
        const DraftRows d = draft_rows(cu_seqlens, b, B, total, max_tokens, nullptr);
        n = d.count;
        row0 = d.first;
        len = clamped_len(seq_lens[b], max_pages, page_size, nullptr);
    }
};

// The list from the unit u0 on: the block that holds it, and the ones behind it.  `next` gives the next part, or false at the end.
struct TreeWalk {
    int u0, u1, share, cta;
    int seq, base, kvh, block;    // the block that is looked at, base: first unit of its K/V head
    int n, row0, len, tiles;      // of the sequence; tiles handed out
    TreeUnits u;
    bool ended;
};
// (n, row0 and len of the sequence that the share begins in have been set)
__host__ __device__ inline void tree_walk_begin(TreeWalk& w, const TreeList& li, int cta, int share, int total, int seq, int base) {
    w.cta = cta;
    w.share = share;
    w.u0 = static_cast<long long>(cta) * share < total ? cta * share : total;
    w.u1 = total - w.u0 < share ? total : w.u0 + share;
    w.ended = w.u0 >= total;
    w.seq = seq;
    w.tiles = 0;
    if (w.ended) return;
    w.u = tree_units(li, w.n, w.len);
    const int per = tree_head_units(w.u);
    w.kvh = (w.u0 - base) / per;
    w.base = base + w.kvh * per;
    const int in = w.u0 - w.base, at = in / w.u.pair;
    w.block = at < w.u.pairs ? at : w.u.pairs;
}
__host__ __device__ inline bool tree_walk_next(TreeWalk& w, const TreeList& li, int Hkv, const TreeSeqs& seq_of, TreePart& e) {
    while (!w.ended) {
        const int blocks = w.u.pairs + (w.u.single ? 1 : 0);
        const int ub = w.base + w.block * w.u.pair, nt = tree_tiles(w.len);
        const bool pair = w.block < w.u.pairs;
        const int wt = li.two && pair ? li.w2 : li.w1, end = ub + (pair ? w.u.pair : w.u.single);
        e.b = w.seq;
        e.kvh = w.kvh;
        e.two = li.two && pair ? 1 : 0;
        e.row_tile = li.two ? 2 * w.block : w.block;
        e.len = w.len;
        e.n = w.n;
        e.row0 = w.row0;
        e.t0 = tree_tile_at(w.u0, ub, li.cost, wt, nt);
        e.t1 = tree_tile_at(w.u1, ub, li.cost, wt, nt);
        e.tile0 = w.tiles;
        e.slot = -1;
        e.pieces = 1;
        e.first_cta = w.cta;
        const bool some = nt > 0 ? e.t0 < e.t1 : ub >= w.u0;
        if (some && e.t1 - e.t0 < nt) {
            e.slot = 2 * w.cta + (e.t0 == 0 ? 1 : 0);
            e.first_cta = (ub + li.cost) / w.share;
            e.pieces = (ub + li.cost + (nt - 1) * wt) / w.share - e.first_cta + 1;
        }
        w.tiles += some ? e.t1 - e.t0 : 0;
        // the block behind it
        if (end >= w.u1) {
            w.ended = true;
        } else if (++w.block == blocks) {
            w.block = 0;
            w.base += tree_head_units(w.u);
            if (++w.kvh == Hkv) {
                w.kvh = 0;
                do {
                    if (++w.seq >= seq_of.B) { w.ended = true; break; }      // (not reached: the share ends before)
                    seq_of(w.seq, w.n, w.row0, w.len);
                } while (w.n == 0);
                if (!w.ended) w.u = tree_units(li, w.n, w.len);
            }
        }
        if (some) return true;
    }
    return false;
}

// ------------------------------------------------------------------ configuration

template <int DQK, int DV, bool kE4m3>
struct TreeCfg {
    static constexpr bool kTwo = DQK != 192 && !kE4m3;          // room for a second query tile
    static constexpr int kQTiles = kTwo ? 2 : 1;
    static constexpr int kQChunks = DQK / kChunkCols, kVChunks = DV / kChunkCols;
    static constexpr int kQBytes = kQChunks * kChunkBytes;      // a query tile; a K tile alike
    // tiles of K as they are multiplied: 64 columns of bf16, or 128 codes, to a 128-byte row
    static constexpr int kKChunks = kE4m3 ? (DQK + 127) / 128 : kQChunks;
    static constexpr int kKBytes = kKChunks * kChunkBytes;
    static constexpr int kTerms = 3;                            // of the queries, over e4m3 caches
    static constexpr int kQSpace = kE4m3 ? kTerms * kKBytes : kQTiles * kQBytes;
    // where 64 columns of the queries are loaded to (over e4m3 caches, into the space of their terms)
    static __host__ __device__ constexpr int q_place(int chunk) {
        return (!kE4m3 ? chunk : DQK == 192 ? 2 * chunk + 1 : 2 * chunk) * kChunkBytes;
    }
    static_assert(kQSpace >= kQTiles * kQBytes, "the queries are loaded into the space of their terms");
    // P_t in shared memory, where there is room for two tiles of it: S_t is free as soon as it has been read, and the next scores are
    // there when a pass ends.  Else P_t lies over S_t.
    static constexpr bool kPSmem = DQK == 64 || (kE4m3 && DQK == 128);
    static constexpr int kPBytes = 2 * kChunkBytes;             // 128 keys of 128 rows
    // keys of a V stage: over e4m3 caches at 128 there is room for three halves of a tile of fp16 values
    static constexpr int kVKeys = kE4m3 && kPSmem ? 64 : 128, kVParts = 128 / kVKeys;
    static constexpr int kVChunk = kVKeys * 128, kVStage = kVChunks * kVChunk;
    static constexpr int kKStages = kE4m3 ? 2 : (DQK == 64 ? 4 : DQK == 128 ? 3 : 2);
    static constexpr int kVStages = kE4m3 ? (DQK == 192 ? 1 : DQK == 128 ? 3 : 4) : (DQK == 64 ? 4 : 2);
    static constexpr int kRaw = kE4m3 ? (DQK == 64 ? 3 : 2) : 0;      // tiles of V's codes
    static constexpr int kTileBytes = kQSpace + kKStages * kKBytes + kVStages * kVStage + kRaw * kChunkBytes + (kPSmem ? 2 * kPBytes : 0);
    static constexpr int kThreads = kE4m3 ? 512 : 384;
    // registers per thread: 256 x 216 + 128 x 72 of 384 x 168, or 256 x 184 + 256 x 72 of 512 x 128
    static constexpr int kRegsSoftmax = kE4m3 ? 184 : 216, kRegsOther = 72;
    static constexpr float kBias = kE4m3 ? 7.f : 0.f;           // P in fp16: below 2^(8 + 7), 11 bits down to 2^-21
    static constexpr int kParts = 4;
};

struct TreeWait {
    uint32_t abort_flag;
    uint32_t* status;
    unsigned long long limit_ns;
};

template <int DQK, int DV, bool kE4m3>
struct TreeShared {
    using Cfg = TreeCfg<DQK, DV, kE4m3>;
    uint64_t q_full, q_ready, q_empty;
    uint64_t k_full[Cfg::kKStages], k_empty[Cfg::kKStages], v_full[Cfg::kVStages], v_empty[Cfg::kVStages];
    uint64_t raw_full[kE4m3 ? Cfg::kRaw : 1], raw_empty[kE4m3 ? Cfg::kRaw : 1];      // codes of V
    uint64_t v_tail[kE4m3 ? 1 : Cfg::kVStages];       // the rows behind a sequence's last value are zeros
    uint64_t s_full[2], s_free[2], p_first[2], p_rest[2], o_final[2];      // (s_free, and o_final of every step, with P in shared memory)
    uint64_t part_full[Cfg::kParts], part_empty[Cfg::kParts];
    uint64_t mma_done;            // (only after a wait that ran out)
    TreePart part[Cfg::kParts];
    uint32_t tmem_base;
    TreeWait wait;
    int v_issued;                 // V tiles whose loads have been issued
    int loads[3];                 // of K and V tiles and of queries, at the end
    float stat_m[2][kTileM], stat_l[2][kTileM];       // (of two streams on the same rows; before a part's end stat_l: what far scores are relative to)
    uint8_t q_shift[2][kE4m3 ? kTileM : 4];      // of even and odd parts: 127 - exponent that a row was scaled by
};

template <int DQK, int DV, bool kE4m3>
constexpr int tree_smem_bytes() {
    return TreeCfg<DQK, DV, kE4m3>::kTileBytes + static_cast<int>(sizeof(TreeShared<DQK, DV, kE4m3>));
}
// Floats of a partial result: unnormalised O as [tile][column / 4][row][4], then every row's reference (log2 units) and sum.
__host__ __device__ constexpr int tree_slot_floats(int dv, bool two) { return (two ? 2 : 1) * kTileM * (dv + 2); }

struct TreeArgs {
    TreeParams t;
    TreeList list;
    int group;
    TreeJoin* join;               // one per CTA
    float* part;                  // two slots per CTA
};

__host__ __device__ constexpr uint32_t make_idesc_f16_f32(int m, int n, bool b_mn_major) {
    return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}

namespace ptx {

// Whether a phase is complete, without the wait that try_wait may take.
FA_DEVI bool mbar_test_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Two e4m3 codes (low byte first) -> two fp16, exactly (NaN stays NaN).
FA_DEVI uint32_t e4m3x2_to_f16x2(uint32_t codes) {
    uint32_t r;
    asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, lo; }" : "=r"(r) : "r"(codes));
    return r;
}
// probe3_mma_ss3 (fa_fwd_pair.cuh), or the same around three 8-bit products
template <bool kF8>
FA_DEVI uint32_t probe3_scores(uint32_t bar0, uint32_t par0, uint32_t bar1, uint32_t par1, uint32_t bar2, uint32_t par2, uint32_t d_tmem, uint64_t a0,
                               uint64_t b0, uint64_t a1, uint64_t b1, uint64_t a2, uint64_t b2, uint32_t idesc) {
    if constexpr (!kF8) {
        return probe3_mma_ss3(bar0, par0, bar1, par1, bar2, par2, d_tmem, a0, b0, a1, b1, a2, b2, idesc);
    } else {
        uint32_t r;
        asm volatile(
            "{\n"
            ".reg .pred p0, p1, p2, q;\n"
            ".reg .b32 t0, t1, t2;\n"
            "setp.ne.b32 q, 1, 0;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 p0, [%1], %2;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 p1, [%3], %4;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 p2, [%5], %6;\n"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%7], %8, %9, %14, q;\n"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%7], %10, %11, %14, q;\n"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%7], %12, %13, %14, q;\n"
            "selp.u32 t0, 1, 0, p0;\n"
            "selp.u32 t1, 2, 0, p1;\n"
            "selp.u32 t2, 4, 0, p2;\n"
            "or.b32 t0, t0, t1;\n"
            "or.b32 %0, t0, t2;\n"
            "}\n"
            : "=r"(r)
            : "r"(bar0), "r"(par0), "r"(bar1), "r"(par1), "r"(bar2), "r"(par2), "r"(d_tmem), "l"(a0), "l"(b0), "l"(a1), "l"(b1), "l"(a2),
              "l"(b2), "r"(idesc)
            : "memory");
        return r;
    }
}
FA_DEVI uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

}  // namespace ptx

// Bounded waits, as in fa_paged.cuh: the softmax warps wait, directly or in turn, for every other role and alone watch the clock; once one
// of their waits has run out, the abort flag ends everybody's.  (A clock in each of some twenty waits is code that the SM's instruction
// cache would have to hold: what is run once in a part, its list entry, masked tile and result, took 2000 to 7000 cycles each.)
FA_DEVI bool tree_wait(uint64_t& bar, uint32_t parity, const TreeWait* ctx) {
    const uint32_t at = ptx::smem_addr(&bar);
    if (ptx::mbar_try_wait(at, parity)) return true;
    do {
        if (*static_cast<const volatile uint32_t*>(&ctx->abort_flag)) return false;
    } while (!ptx::mbar_try_wait(at, parity));
    return true;
}
static __device__ __noinline__ bool tree_wait_long(uint64_t* bar, uint32_t parity, TreeWait* ctx, uint32_t who) {
    const uint32_t at = ptx::smem_addr(bar);
    volatile uint32_t* abort_flag = &ctx->abort_flag;
    uint64_t t0 = 0;
    for (uint32_t it = 1;; ++it) {
        if (ptx::mbar_try_wait(at, parity)) return true;
        if ((it & 63u) == 0u) {
            if (*abort_flag) return false;
            const uint64_t now = ptx::globaltimer_ns();
            if (t0 == 0) {
                t0 = now;
            } else if (now - t0 > ctx->limit_ns) {
                *abort_flag = 1u;
                if (ctx->status) {
                    volatile uint32_t* sw = ctx->status;      // mapped host memory: plain stores
                    sw[1] = who;
                    sw[0] = 4u;                               // FA_ERR_DEVICE_TIMEOUT
                    __threadfence_system();
                }
                return false;
            }
        }
    }
}
FA_DEVI bool tree_wait_timed(uint64_t& bar, uint32_t parity, TreeWait* ctx, uint32_t who) {
    return ptx::mbar_try_wait(ptx::smem_addr(&bar), parity) || tree_wait_long(&bar, parity, ctx, who);
}

// After a wait that ran out: the end of what a barrier counts, for 100 us at most (a load that was never issued does not end).
static __device__ __noinline__ void tree_settle(uint64_t& bar, uint32_t parity) {
    for (int i = 0; i < 1000 && !ptx::mbar_test_wait(ptx::smem_addr(&bar), parity); ++i) __nanosleep(100);
}
// The last of n loads in turn into each of `stages` stages.
static __device__ __noinline__ void tree_settle_ring(uint64_t* full, int stages, int n) {
    for (int i = 0; i < stages && i < n; ++i) tree_settle(full[i], static_cast<uint32_t>((n - 1 - i) / stages) & 1u);
}

// ------------------------------------------------------------------ softmax pass

// Scores that a row does not see become -inf in TMEM, 32 at a time (bit e of `seen`: the e-th of them), ahead of the pass: a loop of 50
// instructions for the few tiles that are masked, where 128 selections in the pass would be 4 KB of its code.
FA_DEVI void tree_hide(uint32_t tS, uint32_t seen) {
#pragma unroll 1
    for (int e = 0; e < 32; e += 16, seen >>= 16) {
        uint32_t s[16];
        ptx::tmem_ld_x16(tS + e, s);
        ptx::tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (!(seen & (1u << i))) s[i] = 0xff800000u;
        ptx::tmem_st_x16(tS + e, s);
    }
}

// Far scores.  s c + off is one rounding of the exact sum, but off itself is a rounded number, and from 2^22 on (log2 units) what it is off by
// moves all weights of a row by more than fp16 has room for, from 2^31 on by more than fp32.  So where references come to lie that far out, the
// scores of the rows' tiles from there on are taken relative to a `base` first, in TMEM, which costs them no more than their own
// rounding, and m_ref is relative to it too.  (Functions of their own, as code that hardly ever runs: see TreeWait.)
constexpr float kTreeFar = 4194304.f;      // 2^22
FA_DEVI bool tree_far(float m_ref, float c) { return m_ref != -INFINITY && fabsf(m_ref * c) > kTreeFar; }
// All scores of a tile less a number of each row's.
static __device__ __noinline__ void tree_shift(uint32_t tS, float by) {
#pragma unroll 1
    for (int e = 0; e < kTileN; e += 16) {
        uint32_t s[16];
        ptx::tmem_ld_x16(tS + e, s);
        ptx::tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __float_as_uint(__uint_as_float(s[i]) - by);
        ptx::tmem_st_x16(tS + e, s);
    }
    ptx::tc_wait_st();
}

// Over e4m3 caches scores are below 2^32, so a row's factor says ahead of its tiles whether they can be far: then the tile's largest score is looked
// for before the pass.  Returns the new base; m_ref follows it.
constexpr float kTreeFarFactor = 1.f / 1024;
static __device__ __noinline__ float tree_rebase(uint32_t tS, float c, float base, float* m_ref) {
    float mx = -INFINITY;
#pragma unroll 1
    for (int e = 0; e < kTileN; e += 16) {
        uint32_t s[16];
        ptx::tmem_ld_x16(tS + e, s);
        ptx::tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, __uint_as_float(s[i]));
    }
    const float up = (mx - base) * c;
    float by = 0.f;
    if (mx != -INFINITY && (*m_ref == -INFINITY ? fabsf(up) : up) > kTreeFar) by = mx - base;
    *m_ref -= by;
    tree_shift(tS, base + by);
    return base + by;
}

// The pass of fa_softmax_pass.cuh, over e4m3 caches with P as fp16 under a bias.  P = 2^(s c + off), off = bias - u c with the reference u; all
// exponentials on the special-function unit.
// Over bf16 caches the pass gives up where a reference has come out far (false: nothing has been handed over yet), and is made again on the
// moved scores, the largest of which is 0, so that no reference moves a second time.
// kPSmem: P goes to the row's bytes p_row of two swizzled chunks of 64 keys; `take` is called once the scores are in registers, and
// says when the product before (of P's space and O) is done, `arrive_first` is not.
template <int DV, bool kHalf, bool kPSmem, typename Take, typename ArriveFirst, typename ArriveRest>
FA_DEVI bool tree_pass(uint32_t tS, uint32_t tO, uint32_t p_row, float c, float tau_raw, float bias, bool first_tile, float& m_ref, float& l, float& alpha,
                       int lane, Take&& take, ArriveFirst&& arrive_first, ArriveRest&& arrive_rest) {
    using namespace ptx;
    const float2 c2 = make_float2(c, c);
    float2 off2;
    float2 sum_a = make_float2(0.f, 0.f), sum_b = make_float2(0.f, 0.f);
    uint32_t s[kTileN];
    auto exp_chunk = [&](int q) {
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(s[q * 32 + e]), __uint_as_float(s[q * 32 + e + 1])), c2, off2);
            s[q * 32 + e] = __float_as_uint(exp2_approx(x.x));
            s[q * 32 + e + 1] = __float_as_uint(exp2_approx(x.y));
        }
    };
    auto emit_chunk = [&](int q) {
        uint32_t pk[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float x = __uint_as_float(s[q * 32 + e]), y = __uint_as_float(s[q * 32 + e + 1]);
            pk[e / 2] = kHalf ? pack_f16x2(x, y) : pack_bf16x2(x, y);
        }
        if constexpr (kPSmem) {
            const uint32_t chunk = p_row + (q >> 1) * kChunkBytes;
            const uint32_t sw = (p_row >> 7 & 7u) << 4;               // (chunks are 1024-byte aligned, rows 128 bytes)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                st_shared_v4(chunk + ((((q & 1) * 4 + v) << 4) ^ sw), pk[4 * v], pk[4 * v + 1], pk[4 * v + 2], pk[4 * v + 3]);
        } else {
            tmem_st_x16(tS + q * 16, pk);
        }
    };
    auto sum_chunk = [&](int q) {
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
            sum_a = fadd2_ftz(sum_a, make_float2(__uint_as_float(s[q * 32 + e]), __uint_as_float(s[q * 32 + e + 1])));
            sum_b = fadd2_ftz(sum_b, make_float2(__uint_as_float(s[q * 32 + e + 2]), __uint_as_float(s[q * 32 + e + 3])));
        }
    };
#pragma unroll 1
    for (;;) {
        tmem_ld_x32(tS + 0, s + 0);
        tmem_ld_x32(tS + 32, s + 32);
        tmem_ld_x32(tS + 64, s + 64);
        tmem_ld_x32(tS + 96, s + 96);
        tc_wait_ld();
        auto set_off = [&]() {
            const float off = m_ref == -INFINITY ? bias : bias - m_ref * c;
            off2 = make_float2(off, off);
        };
        set_off();
        float a[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) a[q] = -INFINITY;
#pragma unroll
        for (int e = 0; e < kTileN; e += 16) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                a[q] = fmax3(a[q], __uint_as_float(s[e + 2 * q]), __uint_as_float(s[e + 2 * q + 1]));
        }
        if (!first_tile) exp_chunk(0);
        float mx = fmaxf(fmax3(a[0], a[1], a[2]), fmax3(a[3], a[4], a[5]));
        mx = fmax3(mx, a[6], a[7]);
        if (first_tile) {            // (nothing to guess with: the row's first reference is this maximum)
            m_ref = mx;
            if constexpr (!kHalf) {
                if (__any_sync(0xffffffffu, tree_far(m_ref, c))) return false;
            }
            set_off();
            exp_chunk(0);
            break;
        }
        const bool grow = mx > m_ref + tau_raw;
        if (!__any_sync(0xffffffffu, grow)) break;
        if (grow) {
            alpha = exp2_approx((m_ref - mx) * c);    // 0 where no key has been seen yet
            m_ref = mx;
        }
        if constexpr (!kHalf) {
            if (__any_sync(0xffffffffu, tree_far(m_ref, c))) return false;
        }
    }
    if constexpr (kPSmem) take();
    if (!first_tile && __any_sync(0xffffffffu, alpha != 1.f)) {
        if constexpr (kPSmem) tc_fence_after_sync();
#pragma unroll 1
        for (int cc = 0; cc < DV / 32; ++cc) {
            uint32_t r[32];
            tmem_ld_x32(tO + cc * 32, r);
            tc_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e)
                r[e] = __float_as_uint(__uint_as_float(r[e]) * alpha);
            tmem_st_x32(tO + cc * 32, reinterpret_cast<uint32_t(&)[32]>(r));
        }
        if constexpr (kPSmem) tc_wait_st();
    }
    // (the sums: under the exponentials where the hand-over can wait for them, else behind it, off the chain MMA -> softmax -> MMA)
    exp_chunk(1);
    emit_chunk(0);
    if constexpr (kPSmem) sum_chunk(0);
    exp_chunk(2);
    emit_chunk(1);
    if constexpr (kPSmem) sum_chunk(1);
    if constexpr (!kPSmem) emit_chunk(2);
    if constexpr (!kPSmem) {
        tc_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) arrive_first();
    }
    exp_chunk(3);
    if constexpr (kPSmem) {
        emit_chunk(2);
        sum_chunk(2);
    }
    emit_chunk(3);
    if constexpr (kPSmem) fence_proxy_async_smem();
    else tc_wait_st();
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) arrive_rest();
    if constexpr (!kPSmem) {
        sum_chunk(0);
        sum_chunk(1);
        sum_chunk(2);
    }
    sum_chunk(3);
    l = l * alpha + ((sum_a.x + sum_a.y) + (sum_b.x + sum_b.y));
    return true;
}

// ------------------------------------------------------------------ kernel

template <int DQK, int DV, bool kE4m3>
__global__ void __launch_bounds__((TreeCfg<DQK, DV, kE4m3>::kThreads), 1)
fa_tree_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
               const PagedParams p, const TreeArgs a) {
    using Cfg = TreeCfg<DQK, DV, kE4m3>;
    using Shared = TreeShared<DQK, DV, kE4m3>;
    using namespace ptx;
    constexpr int NK = Cfg::kKStages, NV = Cfg::kVStages, NR = kE4m3 ? Cfg::kRaw : 1, NP = Cfg::kParts;

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(smem_raw + Cfg::kTileBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t smem_base = smem_addr(smem_raw);
    const uint32_t sQ = smem_base, sK = sQ + Cfg::kQSpace, sV = sK + NK * Cfg::kKBytes, sRaw = sV + NV * Cfg::kVStage, sP = sRaw + Cfg::kRaw * kChunkBytes;

    grid_launch_dependents();
    if ((smem_base & 1023u) != 0u) {          // uniform over the CTA; nothing has been set up yet
        grid_dependency_wait();
        if (tid == 0) {
            a.join[blockIdx.x].pieces = 0;
            if (p.status) {
                volatile uint32_t* sw = p.status;
                sw[1] = kSiteSmemAlign;
                sw[0] = 3u;                   // FA_ERR_CUDA
                __threadfence_system();
            }
        }
        return;
    }
    if (tid == 0) {
        sh.wait.abort_flag = 0;
        sh.wait.status = p.status;
        sh.wait.limit_ns = p.wait_limit_ns;
        mbar_init(smem_addr(&sh.q_full), 1);
        mbar_init(smem_addr(&sh.q_empty), 1);
        mbar_init(smem_addr(&sh.mma_done), 1);
        sh.v_issued = 0;
#pragma unroll
        for (int s = 0; s < NK; ++s) {
            mbar_init(smem_addr(&sh.k_full[s]), 1);
            mbar_init(smem_addr(&sh.k_empty[s]), 1);
        }
#pragma unroll
        for (int s = 0; s < NV; ++s) {
            mbar_init(smem_addr(&sh.v_full[s]), kE4m3 ? 4 : 1);     // the four warps that convert, or the copy
            mbar_init(smem_addr(&sh.v_empty[s]), 1);
            if constexpr (!kE4m3) mbar_init(smem_addr(&sh.v_tail[s]), 1);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            mbar_init(smem_addr(&sh.s_full[t]), 1);
            mbar_init(smem_addr(&sh.s_free[t]), 4);
            mbar_init(smem_addr(&sh.p_first[t]), 4);      // 4 softmax warps
            mbar_init(smem_addr(&sh.p_rest[t]), 4);
            mbar_init(smem_addr(&sh.o_final[t]), 1);
        }
        if constexpr (kE4m3) {
            mbar_init(smem_addr(&sh.q_ready), 4);
#pragma unroll
            for (int s = 0; s < NR; ++s) {
                mbar_init(smem_addr(&sh.raw_full[s]), 1);
                mbar_init(smem_addr(&sh.raw_empty[s]), 4);
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            mbar_init(smem_addr(&sh.part_full[i]), 1);
            mbar_init(smem_addr(&sh.part_empty[i]), 8 + 3 + (kE4m3 ? 4 : 0));      // softmax warps, MMA thread, two loading warps, converting warps
        }
        fence_mbar_init();
        prefetch_tensormap(&tm_q);
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
    }
    if (warp == 8) {
        tmem_alloc(smem_addr(&sh.tmem_base), 512);
        tmem_relinquish_alloc_permit();
    }
    if (warp >= 9 && warp < 11) {
        // lengths, offsets and block table towards L2 (a line each; the streams of other calls have usually driven them out): list and loads
        // wait for one after the other
        const int per_row = (p.max_pages + 31) / 32, line = blockIdx.x * 32 + lane, b = line / per_row;
        if (warp == 9) {
            if (lane * 32 < p.B) {
                prefetch_l2(p.seq_lens + lane * 32);
                if (a.t.cu_seqlens) prefetch_l2(a.t.cu_seqlens + lane * 32);
            }
        } else if (b < p.B) {
            prefetch_l2(p.block_table + b * p.table_stride + (line - b * per_row) * 32);
        }
    }
    // Rows of the query tiles that no load fills count as zeros (see the softmax warps)
    for (int i = tid; i < Cfg::kQSpace / 16; i += Cfg::kThreads) st_shared_v4(sQ + 16 * i, 0, 0, 0, 0);
    fence_proxy_async_smem();
    grid_dependency_wait();

    const TreeSeqs seq_of{a.t.cu_seqlens, p.seq_lens, p.B, a.t.total, a.t.max_tokens, p.max_pages, p.page_size};
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem_base;
    auto wait = [&](uint64_t& bar, uint32_t parity) -> bool { return tree_wait(bar, parity, &sh.wait); };
    // Part k for a warp as a whole; false at the end of the list or after a wait that ran out.
    auto take_part = [&](int k, TreePart& e) -> bool {
        if (!__all_sync(0xffffffffu, wait(sh.part_full[k % NP], (k / NP) & 1))) return false;
        e = sh.part[k % NP];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&sh.part_empty[k % NP]));
        return e.t1 >= 0;
    };

    if (warp < 8) {
        // ============================================================ softmax of stream t
        setmaxnreg_inc<Cfg::kRegsSoftmax>();
        const int t = warp >> 2, row = tid & (kTileM - 1);
        const uint32_t lane_sel = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + 128 * t + lane_sel, tO = tmem + 256 + lane_sel;
        const uint32_t bar_pf = smem_addr(&sh.p_first[t]), bar_pr = smem_addr(&sh.p_rest[t]);
        const int row_token = row / a.list.row_heads, row_head = row - row_token * a.list.row_heads;
        int n_s = 0, n_q = 0, n_final[2] = {0, 0};       // score tiles, parts with queries, parts with a result of stream 0 / 1 so far
        bool ok = true;
        // All 256 threads meet at the barriers of a part, also after a wait that ran out (nothing is stored then), and leave together.
        for (int k = 0;; ++k) {
            TreePart e;
            e.t1 = -1;
            ok = ok && tree_wait_timed(sh.part_full[k % NP], (k / NP) & 1, &sh.wait, kSiteItem);
            if (named_barrier_or(1, 256, !ok)) break;
            e = sh.part[k % NP];
            if (e.t1 < 0) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.part_empty[k % NP]));
            const int nt = e.t1 - e.t0;
            const bool two = Cfg::kTwo && e.two;
            const int steps0 = two ? nt : (nt + 1) / 2, steps1 = two ? nt : nt / 2, steps = t == 0 ? steps0 : steps1;
            // the row: its token and head
            const int tile = e.row_tile + (two ? t : 0), tc = a.list.head_chunks == 1 ? tile : tile / a.list.head_chunks, hc = tile - tc * a.list.head_chunks;
            const int token = tc * a.list.row_tokens + row_token, head = hc * a.list.row_heads + row_head;
            const bool live = row_token < a.list.row_tokens && token < e.n && head < a.group;
            const bool warp_live = __any_sync(0xffffffffu, live);
            const int first_draft = e.len - e.n, q_row = e.row0 + (live ? token : 0);
            if (live && a.t.mask) asm volatile("prefetch.global.L1 [%0];" ::"l"(a.t.mask + q_row * a.t.mask_stride));
            float c = p.scale_log2;
            if constexpr (kE4m3) {
                c *= p.k_scale ? p.k_scale[e.kvh] : 1.f;
                n_q += nt > 0;
            }
            // Rows that are not the block's (zeros, or other sequences' queries) count as zeros with probabilities of zero: scores that rise from
            // tile to tile would have their warp move references all the time, and products of zeros take less of the power limit.
            if (!live) c = 0.f;
            const float bias = live ? Cfg::kBias : -INFINITY;
            float m_ref = -INFINITY, l = 0.f, tau_raw = kRescaleThresholdLog2 / c;
            bool far = false;            // scores of the warp's rows are relative to base (over e4m3 caches, which leave no register, where stat_l is free)
            float base_reg = 0.f;
            float& base = kE4m3 ? sh.stat_l[t][row] : base_reg;
            for (int j = 0; j < steps; ++j, ++n_s) {
                ok = __all_sync(0xffffffffu, ok && tree_wait_timed(sh.s_full[t], n_s & 1, &sh.wait, kSiteSoftmaxSFull));
                if (!ok) break;
                tc_fence_after_sync();
                if constexpr (kE4m3) {
                    if (j == 0) {
                        c *= __uint_as_float(static_cast<uint32_t>(sh.q_shift[(n_q - 1) & 1][row]) << 23);
                        // (hidden scores are -inf already, and -inf times a factor that has become 0 is no number; scores, 2^32 at most,
                        // times the smallest normal number are nothing all the same)
                        if (live && c < FLT_MIN) c = FLT_MIN;
                        tau_raw = kRescaleThresholdLog2 / c;
                        far = __any_sync(0xffffffffu, c > kTreeFarFactor);
                        if (far) base = 0.f;
                    }
                }
                // (P in shared memory: the scores are in registers; before P is written, the product of the step before has to be done)
                auto take = [&]() {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_addr(&sh.s_free[t]));
                    if (j > 0) ok = tree_wait_timed(sh.o_final[t], (n_s & 1) ^ 1, &sh.wait, kSiteSoftmaxPFree);
                    __syncwarp();
                };
                if (!warp_live) {            // (its rows are not stored)
                    if constexpr (Cfg::kPSmem) {
                        take();
                        if (j == 0) {
#pragma unroll
                            for (int v = 0; v < 16; ++v) st_shared_v4(sP + t * Cfg::kPBytes + (v >> 3) * kChunkBytes + row * 128 + (v & 7) * 16, 0, 0, 0, 0);
                            fence_proxy_async_smem();
                        }
                    } else {
                        const uint32_t zeros[16] = {};
#pragma unroll
                        for (int q = 0; q < 4; ++q) tmem_st_x16(tS + 16 * q, zeros);
                        tc_wait_st();
                    }
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (!Cfg::kPSmem) mbar_arrive(bar_pf);
                        mbar_arrive(bar_pr);
                    }
                    continue;
                }
                const int key0 = (e.t0 + (two ? j : 2 * j + t)) * kTileN;
                const bool masked = key0 + kTileN > first_draft;
                if (masked) {
#pragma unroll 1
                    for (int w = 0; w < 4; ++w) {
                        const int j0 = key0 + 32 * w - first_draft;          // the draft of these 32 keys' first
                        uint32_t seen = 0xffffffffu;
                        if (j0 > -32) {
                            const int at = j0 >> 5;                          // (from -1 on; there is no word -1: its bits, the keys before the drafts, are seen)
                            const uint32_t lo = at < 0 ? 0xffffffffu : draft_word(a.t, q_row, token, e.n, at), hi = draft_word(a.t, q_row, token, e.n, at + 1);
                            seen = __funnelshift_r(lo, hi, j0 & 31);
                        }
                        tree_hide(tS + 32 * w, seen);
                    }
                    tc_wait_st();
                }
                float alpha = 1.f;
                if (far) {
                    if constexpr (kE4m3) {
                        float ref = m_ref;
                        base = tree_rebase(tS, c, base, &ref);
                        m_ref = ref;
                    } else {
                        tree_shift(tS, base);
                    }
                }
                for (bool again = false; !tree_pass<DV, kE4m3, Cfg::kPSmem>(tS, tO + 128 * t, sP + t * Cfg::kPBytes + row * 128, c, tau_raw, bias,
                                                                            j == 0 && !again, m_ref, l, alpha, lane, take,
                                                                            [&]() { mbar_arrive(bar_pf); }, [&]() { mbar_arrive(bar_pr); });
                     again = true) {
                    const float by = tree_far(m_ref, c) ? m_ref : 0.f;
                    tree_shift(tS, by);
                    m_ref -= by;
                    base += by;
                    far = true;
                }
            }
            // ---- the part's result: sum and reference of a row that saw a key, O of one stream or of both
            const float off = m_ref == -INFINITY ? Cfg::kBias : Cfg::kBias - m_ref * c;
            float m = l > 0.f || l != l ? -off : -INFINITY;       // (a NaN goes through)
            if (far) m += base * c;
            const bool whole = e.slot < 0;
            const float vs = kE4m3 && p.v_scale ? p.v_scale[e.kvh] : 1.f;
            float f0 = 1.f, f1 = 0.f;
            if (!two) {
                sh.stat_m[t][row] = m;
                sh.stat_l[t][row] = l;
                named_barrier_sync(1, 256);
                const float m0 = sh.stat_m[0][row], m1 = sh.stat_m[1][row];
                m = fmaxf(m0, m1);
                f0 = m0 == -INFINITY ? 0.f : exp2_approx(m0 - m);
                f1 = m1 == -INFINITY ? 0.f : exp2_approx(m1 - m);
                l = f0 * sh.stat_l[0][row] + f1 * sh.stat_l[1][row];
            }
            const bool any = l > 0.f || l != l;
            const float norm = whole ? (any ? vs / l : 0.f) : 1.f;
            f0 *= norm;
            f1 *= norm;
            // (with P in shared memory the barrier's phases are the steps, else the parts)
            n_final[0] += Cfg::kPSmem ? steps0 : steps0 > 0;
            n_final[1] += Cfg::kPSmem ? steps1 : steps1 > 0;
            if (steps0 > 0 && (!two || t == 0)) ok = ok && tree_wait_timed(sh.o_final[0], (n_final[0] & 1) ^ 1, &sh.wait, kSiteEpiOFull);
            if (steps1 > 0 && (!two || t == 1)) ok = ok && tree_wait_timed(sh.o_final[1], (n_final[1] & 1) ^ 1, &sh.wait, kSiteEpiOFull);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after_sync();
            // columns [col0, col1) are this thread's: all of its own stream's, or half of both streams'
            const int col0 = two ? 0 : t * (DV / 2), col1 = two ? DV : col0 + DV / 2;
            const int hq = e.kvh * a.group + head;
            // Whole results: four neighbouring lanes exchange 16-byte pieces of their rows, so that they store 64 neighbouring bytes of one row
            // at a time (a lane's own row: 32 lines a store, which held up the next part's begin by 4000 cycles).
            __nv_bfloat16* const out = p.O + q_row * p.o_st + hq * p.o_sh;
            __nv_bfloat16* out4[4];
            uint32_t live4 = __ballot_sync(0xffffffffu, ok && live) >> (lane & 28);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                out4[i] = reinterpret_cast<__nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(out), (lane & 28) + i)) + (lane & 3) * 8;
            float* const slot = a.part + static_cast<long long>(whole ? 0 : e.slot) * tree_slot_floats(DV, Cfg::kTwo);
            float4* const slot_o = reinterpret_cast<float4*>(slot) + (two ? t : 0) * (DV / 4) * kTileM + row;
#pragma unroll 1
            for (int col = col0; col < col1; col += 32) {
                float y[32];
                if (nt > 0 && ok) {
                    uint32_t r0[32];
                    tmem_ld_x32(tO + (two ? 128 * t : 0) + col, r0);
                    if (!two && steps1 > 0) {
                        uint32_t r1[32];
                        tmem_ld_x32(tO + 128 + col, r1);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[i] = f0 * __uint_as_float(r0[i]) + f1 * __uint_as_float(r1[i]);
                    } else {
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[i] = f0 * __uint_as_float(r0[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[i] = 0.f;
                }
                if (whole) {
                    // (nothing seen: zeros, whatever the products of zero probabilities gave)
                    uint32_t v[4][4];
#pragma unroll
                    for (int i = 0; i < 32; i += 2) v[i / 8][i % 8 / 2] = any ? pack_bf16x2(y[i], y[i + 1]) : 0u;
#pragma unroll
                    for (int bit = 1; bit <= 2; bit <<= 1) {
                        const bool up = (lane & bit) != 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (i & bit) continue;
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? v[i][w] : v[i | bit][w], bit);
                                if (up) v[i][w] = got; else v[i | bit][w] = got;
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (live4 & (1u << i)) *reinterpret_cast<uint4*>(out4[i] + col) = make_uint4(v[i][0], v[i][1], v[i][2], v[i][3]);
                } else if (ok && live) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4) slot_o[(col + i) / 4 * kTileM] = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
                }
            }
            if (ok && live && (two || t == 0)) {
                if (whole) {
                    if (p.lse) p.lse[static_cast<long long>(hq) * a.t.total + q_row] = any ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
                } else {
                    float* const ml = slot + (Cfg::kTwo ? 2 : 1) * kTileM * DV + (two ? t : 0) * 2 * kTileM + row;
                    ml[0] = m;
                    ml[kTileM] = l;
                }
            }
            // (both groups have read both accumulators, and each other's sums, at the barrier that the next part begins with)
            tc_fence_before_sync();
        }
    } else if (warp == 8) {
        // ============================================================ MMA issue, one thread for both streams
        setmaxnreg_dec<Cfg::kRegsOther>();
        if (elect_one()) {
            constexpr uint32_t kIdescQK = kE4m3 ? (make_idesc_e4m3_f32(kTileM, kTileN, false, false) | (1u << 7))        // A: e5m2
                                                : make_idesc_bf16_f32(kTileM, kTileN, false, false);
            constexpr uint32_t kIdescPV = kE4m3 ? make_idesc_f16_f32(kTileM, DV, true) : make_idesc_bf16_f32(kTileM, DV, false, true);
            constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);   // sbo, version, swizzle
            constexpr int kPerTerm = kE4m3 ? DQK / 32 : DQK / 16, kSteps = kE4m3 ? Cfg::kTerms * kPerTerm : kPerTerm;      // of 32 bytes of a row
            const uint32_t q_lo0 = ((sQ & 0x3FFFFu) >> 4) | (1u << 16);
            const uint32_t k_lo0 = ((sK & 0x3FFFFu) >> 4) | (1u << 16);
            const uint32_t v_lo0 = ((sV & 0x3FFFFu) >> 4) | ((static_cast<uint32_t>(Cfg::kVChunk) >> 4) << 16);
            const uint32_t p_lo0 = ((sP & 0x3FFFFu) >> 4) | (1u << 16);
            auto desc = [](uint32_t lo) -> uint64_t { return (static_cast<uint64_t>(kDescHi) << 32) | lo; };
            auto koff = [](int ks) -> uint32_t { ks %= kPerTerm; return static_cast<uint32_t>(((ks / 4) * kChunkBytes + (ks % 4) * 32) >> 4); };
            auto qoff = [&](int ks) -> uint32_t { return koff(ks) + static_cast<uint32_t>(ks / kPerTerm * (Cfg::kKBytes >> 4)); };
            auto score = [&](uint32_t tS, uint32_t q, uint32_t k, int ks) {
                if constexpr (kE4m3) mma_ss_f8(tS, desc(q + qoff(ks)), desc(k + koff(ks)), kIdescQK, ks > 0 ? 1u : 0u);
                else mma_ss(tS, desc(q + qoff(ks)), desc(k + koff(ks)), kIdescQK, ks > 0 ? 1u : 0u);
            };
            int sk = 0, sv = 0, n_q = 0;       // stages, parts with queries so far
            uint32_t ph_k = 0, ph_v = 0, ph_tail = 0, ph_p = 0, ph_s = 0;   // (of the last tiles, a bit per stage; of the steps, a bit per stream)
            bool two = false, tail = false;
            int nt = 0, k_tile = 0, v_tile = 0;                             // of the part: tiles, tile that stage sk / sv holds
            uint32_t pre_p = 0, pre_v = 0, pre_k = 0;                       // probes that succeeded for the next block
            auto step_k = [&]() { ++k_tile; if (++sk == NK) { sk = 0; ph_k ^= 1u; } };
            auto step_v = [&]() { ++v_tile; if (++sv == NV) { sv = 0; ph_v ^= 1u; } };
            auto q_lo = [&](int t) -> uint32_t { return q_lo0 + (two ? t : 0) * (Cfg::kQBytes >> 4); };
            // Behind the score products of stream t with the K tile in stage sk: who may go on.
            auto scores_done = [&](int t) {
                tc_commit(smem_addr(&sh.s_full[t]));
                if (!two || t == 1) {
                    tc_commit(smem_addr(&sh.k_empty[sk]));
                    if (k_tile == nt - 1) tc_commit(smem_addr(&sh.q_empty));
                    step_k();
                }
            };
            // Stream t's block of step j: P_t V, then the next scores.  Barriers that the next block needs are probed from inside it.
            // (one body for both streams: see TreeWait on code)
            auto block = [&](int t, int j, int steps) -> bool {
                const bool fresh = !two || t == 0;                   // (the streams of two row tiles share the K/V tiles)
                const bool next = j + 1 < steps;
                if (fresh) {
                    if (!pre_v && !wait(sh.v_full[sv], ph_v)) return false;
                    if constexpr (!kE4m3) {
                        if (tail && v_tile == nt - 1) {
                            if (!wait(sh.v_tail[sv], (ph_tail >> sv) & 1u)) return false;
                            ph_tail ^= 1u << sv;
                        }
                    }
                    if (next && !pre_k && !wait(sh.k_full[sk], ph_k)) return false;
                }
                const uint32_t parity = (ph_p >> t) & 1u;
                const uint32_t tS = tmem + 128 * t, tO = tmem + 256 + 128 * t;
                const uint32_t vlo = v_lo0 + sv * (Cfg::kVStage >> 4), klo = k_lo0 + sk * (Cfg::kKBytes >> 4);
                if (!pre_p && !wait(sh.p_first[t], parity)) return false;
                pre_p = pre_v = pre_k = 0u;
                tc_fence_after_sync();
                mma_ts(tO, tS + 0, desc(vlo + 0 * (2048 >> 4)), kIdescPV, j > 0 ? 1u : 0u);
                mma_ts(tO, tS + 8, desc(vlo + 1 * (2048 >> 4)), kIdescPV, 1u);
                mma_ts(tO, tS + 16, desc(vlo + 2 * (2048 >> 4)), kIdescPV, 1u);
                mma_ts(tO, tS + 24, desc(vlo + 3 * (2048 >> 4)), kIdescPV, 1u);
                const uint32_t rest = probe_mma_ts2(smem_addr(&sh.p_rest[t]), parity, tO, tS + 32, desc(vlo + 4 * (2048 >> 4)),
                                                    tS + 40, desc(vlo + 5 * (2048 >> 4)), kIdescPV);
                if (!rest && !wait(sh.p_rest[t], parity)) return false;
                tc_fence_after_sync();
                mma_ts(tO, tS + 48, desc(vlo + 6 * (2048 >> 4)), kIdescPV, 1u);
                mma_ts(tO, tS + 56, desc(vlo + 7 * (2048 >> 4)), kIdescPV, 1u);
                ph_p ^= 1u << t;
                const bool v_done = !two || t == 1;
                if (v_done) tc_commit(smem_addr(&sh.v_empty[sv]));       // (here: behind the scores it would come 512 cycles later)
                if (next) {
                    // (the next block's: the other stream's probabilities; its V and K tile where they are not this block's)
                    const bool same = two && t == 0;
                    const int sv_n = sv + 1 == NV ? 0 : sv + 1, sk_n = sk + 1 == NK ? 0 : sk + 1;
                    const uint32_t ph_v_n = sv + 1 == NV ? ph_v ^ 1u : ph_v, ph_k_n = sk + 1 == NK ? ph_k ^ 1u : ph_k;
                    score(tS, q_lo(t), klo, 0);
                    const uint32_t got = probe3_scores<kE4m3>(smem_addr(&sh.p_first[1 - t]), (ph_p >> (1 - t)) & 1u, smem_addr(&sh.v_full[same ? sv : sv_n]), same ? ph_v : ph_v_n,
                                                        smem_addr(&sh.k_full[same ? sk : sk_n]), same ? ph_k : ph_k_n, tS,
                                                        desc(q_lo(t) + qoff(1)), desc(klo + koff(1)), desc(q_lo(t) + qoff(2)), desc(klo + koff(2)),
                                                        desc(q_lo(t) + qoff(3)), desc(klo + koff(3)), kIdescQK);
#pragma unroll
                    for (int ks = 4; ks < kSteps; ++ks) score(tS, q_lo(t), klo, ks);
                    pre_p = got & 1u;
                    pre_v = (got >> 1) & 1u;
                    pre_k = (got >> 2) & 1u;
                    scores_done(t);
                } else {
                    tc_commit(smem_addr(&sh.o_final[t]));
                }
                if (v_done) step_v();
                return true;
            };
            // With P in shared memory: scores and products are two sequences, each over the streams in turn, and whichever can go on does.
            auto ready = [&](uint64_t& bar, uint32_t parity) -> bool { return mbar_test_wait(smem_addr(&bar), parity); };
            auto scores = [&](int t) {
                ph_s ^= 1u << t;
                tc_fence_after_sync();
                const uint32_t klo = k_lo0 + sk * (Cfg::kKBytes >> 4);
#pragma unroll
                for (int ks = 0; ks < kSteps; ++ks) score(tmem + 128 * t, q_lo(t), klo, ks);
                scores_done(t);
            };
            auto product = [&](int t, bool first) -> bool {
                const uint32_t tO = tmem + 256 + 128 * t;
                if constexpr (!kE4m3) {
                    if ((!two || t == 0) && tail && v_tile == nt - 1) {
                        if (!wait(sh.v_tail[sv], (ph_tail >> sv) & 1u)) return false;
                        ph_tail ^= 1u << sv;
                    }
                }
#pragma unroll
                for (int part = 0; part < Cfg::kVParts; ++part) {
                    if (part > 0 && !wait(sh.v_full[sv], ph_v)) return false;
                    tc_fence_after_sync();
                    const uint32_t vlo = v_lo0 + sv * (Cfg::kVStage >> 4), plo = p_lo0 + t * (Cfg::kPBytes >> 4);
#pragma unroll
                    for (int ks = 0; ks < Cfg::kVKeys / 16; ++ks) {
                        const int at = part * (Cfg::kVKeys / 16) + ks;
                        mma_ss(tO, desc(plo + static_cast<uint32_t>(((at / 4) * kChunkBytes + (at % 4) * 32) >> 4)), desc(vlo + ks * (2048 >> 4)), kIdescPV,
                               at > 0 || !first ? 1u : 0u);
                    }
                    if (!two || t == 1) {
                        tc_commit(smem_addr(&sh.v_empty[sv]));
                        if (++sv == NV) { sv = 0; ph_v ^= 1u; }
                    }
                }
                ph_p ^= 1u << t;
                if (!two || t == 1) ++v_tile;
                tc_commit(smem_addr(&sh.o_final[t]));
                return true;
            };
            bool ok = true;
            for (int k = 0; ok; ++k) {
                ok = wait(sh.part_full[k % NP], (k / NP) & 1);
                if (!ok) break;
                const TreePart e = sh.part[k % NP];
                mbar_arrive(smem_addr(&sh.part_empty[k % NP]));
                if (e.t1 < 0) break;
                nt = e.t1 - e.t0;
                if (nt == 0) continue;
                two = Cfg::kTwo && e.two;
                tail = !kE4m3 && e.t1 * kTileN > e.len;
                k_tile = v_tile = 0;
                pre_p = pre_v = pre_k = 0u;
                const int steps0 = two ? nt : (nt + 1) / 2, steps1 = two ? nt : nt / 2;
                if constexpr (kE4m3) ok = wait(sh.q_ready, n_q & 1);
                else ok = wait(sh.q_full, n_q & 1);
                ++n_q;
                if constexpr (Cfg::kPSmem) {
                    // (a stage that both streams use is waited for once: it is still full for the second)
                    const int blocks = steps0 + steps1;
                    int n_scores = 0, n_products = 0;              // blocks (j, t): number 2 j + t
                    while (ok && n_products < blocks) {
                        const int ts = n_scores & 1, tp = n_products & 1;
                        if (n_products < n_scores && ready(sh.p_rest[tp], (ph_p >> tp) & 1u) && ready(sh.v_full[sv], ph_v)) {
                            ok = product(tp, n_products < 2);
                            ++n_products;
                        }
                        if (n_scores < blocks && ready(sh.s_free[ts], ((ph_s >> ts) & 1u) ^ 1u) && ready(sh.k_full[sk], ph_k)) {
                            scores(ts);
                            ++n_scores;
                        }
                        if (*static_cast<volatile uint32_t*>(&sh.wait.abort_flag)) ok = false;
                    }
                } else {
#pragma unroll 1
                    for (int t = 0; t < 2; ++t) {
                        if (!ok || (t == 1 && steps1 == 0)) break;
                        if (t == 0 || !two) ok = wait(sh.k_full[sk], ph_k);
                        if (!ok) break;
                        tc_fence_after_sync();
                        const uint32_t klo = k_lo0 + sk * (Cfg::kKBytes >> 4);
#pragma unroll
                        for (int ks = 0; ks < kSteps; ++ks) score(tmem + 128 * t, q_lo(t), klo, ks);
                        scores_done(t);
                    }
                    for (int j = 0; j < steps0 && ok; ++j) {
#pragma unroll 1
                        for (int t = 0; t < 2 && ok; ++t)
                            if (t == 0 || j < steps1) ok = block(t, j, t == 0 ? steps0 : steps1);
                    }
                }
            }
        }
    } else if (warp == 9 || warp == 10) {
        // ============================================================ TMA loads of K (warp 9), or of Q and V (warp 10)
        setmaxnreg_dec<Cfg::kRegsOther>();
        const bool is_v = warp == 10;
        constexpr int kVC = kE4m3 ? 1 : Cfg::kVChunks, kMaxChunks = Cfg::kKChunks > kVC ? Cfg::kKChunks : kVC;
        constexpr int kChunk = kE4m3 ? 128 : kChunkCols;             // columns of a 128-byte row
        const int chunks = is_v ? kVC : Cfg::kKChunks, stages = is_v ? (kE4m3 ? NR : NV) : NK;
        const int stage_bytes = is_v ? kVC * kChunkBytes : Cfg::kKBytes;
        const CUtensorMap* tm = is_v ? &tm_v : &tm_k;
        uint64_t* const full = is_v ? (kE4m3 ? sh.raw_full : sh.v_full) : sh.k_full;
        uint64_t* const empty = is_v ? (kE4m3 ? sh.raw_empty : sh.v_empty) : sh.k_empty;
        const uint32_t dst0 = is_v ? (kE4m3 ? sRaw : sV) : sK;
        const int box = p.box_rows, shift = __ffs(kTileN / box) - 1, boxes = 1 << shift, tiles_ahead = 32 >> shift;
        int n = 0, n_q = 0, s = 0;
        uint32_t parity = 1;
        bool ok = true;
        TreePart e;
        for (int k = 0; ok && take_part(k, e); ++k) {
            if (e.t0 == e.t1) continue;
            const int* const table = p.block_table + e.b * p.table_stride;
            if (is_v) {              // (its tiles are needed later than those of K)
                const bool two = Cfg::kTwo && e.two;
                ok = __all_sync(0xffffffffu, wait(sh.q_empty, (n_q & 1) ^ 1));
                if (!ok) break;
                ++n_q;
                if (lane == 0) {
                    const uint32_t bar = smem_addr(&sh.q_full);
                    mbar_arrive_expect_tx(bar, (two ? 2 : 1) * Cfg::kQChunks * a.list.row_tokens * a.list.row_heads * 128);
                    for (int t = 0; t < (two ? 2 : 1); ++t) {
                        const int tile = e.row_tile + t, tc = a.list.head_chunks == 1 ? tile : tile / a.list.head_chunks, hc = tile - tc * a.list.head_chunks;
#pragma unroll
                        for (int cc = 0; cc < Cfg::kQChunks; ++cc)
                            tma_load_4d(sQ + t * Cfg::kQBytes + Cfg::q_place(cc), &tm_q, bar, cc * kChunkCols, e.kvh * a.group + hc * a.list.row_heads,
                                        e.row0 + tc * a.list.row_tokens, 0);
                    }
                }
                __syncwarp();
            }
            int pages = 0, slots = 0;         // of tile `first` + lane / boxes, box lane % boxes
            int first = e.t0;
            for (int t = e.t0; t < e.t1; ++t, ++n) {
                if (t == e.t0 || t - first == tiles_ahead) {
                    first = t;
                    const int tile = t + (lane >> shift), key = tile * kTileN + (lane & (boxes - 1)) * box;
                    if (tile < e.t1 && key < e.len) {
                        const int at = key / p.page_size;
                        slots = key - at * p.page_size;
                        pages = table[at];
                        if (pages < 0 || pages >= p.num_pages) {
                            report_bad_input(p.status, kSiteBadPage);
                            pages = p.num_pages;       // behind the pool: reads as zeros
                        }
                    }
                }
                const int from = ((t - first) << shift) + lane;
                const int page = __shfl_sync(0xffffffffu, pages, from & 31), slot = __shfl_sync(0xffffffffu, slots, from & 31);
                ok = __all_sync(0xffffffffu, wait(empty[s], parity));
                if (!ok) break;
                const uint32_t bar = smem_addr(&full[s]);
                const int n_box = min(boxes, (e.len - t * kTileN + box - 1) / box);
                if (!(is_v && p.debug_drop_v_load && n == 0)) {
                    if (lane == 0) mbar_arrive_expect_tx(bar, n_box * box * 128 * chunks);
                    __syncwarp();
                    if (lane < n_box) {
#pragma unroll
                        for (int cc = 0; cc < kMaxChunks; ++cc)
                            if (cc < chunks) tma_load_4d(dst0 + s * stage_bytes + cc * kChunkBytes + lane * box * 128, tm, bar, cc * kChunk, slot, e.kvh, page);
                    }
                    __syncwarp();
                }
                if (!kE4m3 && is_v && lane == 0) {
                    __threadfence_block();
                    *static_cast<volatile int*>(&sh.v_issued) = n + 1;
                }
                if (++s == stages) { s = 0; parity ^= 1u; }
            }
        }
        if (lane == 0) {
            sh.loads[is_v ? 1 : 0] = n;
            if (is_v) sh.loads[2] = n_q;
        }
    } else if (warp == 11) {
        // ============================================================ the list of parts; zeros behind the last value of a sequence
        setmaxnreg_dec<Cfg::kRegsOther>();
        // its length, and where this CTA's share begins: a lane has `chunk` sequences
        TreeList li = a.list;
        const int chunk = (p.B + 31) >> 5, b_first = min(p.B, lane * chunk), b_last = min(p.B, b_first + chunk);
        int n_mine = 0, row_mine = 0, len_mine = 0;          // the lane's last sequence
        TreeBatch batch{0, 0, 0, 0x7fffffff, 0};
        int mine = 0;
#pragma unroll 4
        for (int b = b_first; b < b_last; ++b) {
            seq_of(b, n_mine, row_mine, len_mine);
            const TreeUnits u = tree_units(li, n_mine, len_mine);
            mine += p.Hkv * tree_head_units(u);
            if (n_mine > 0) {
                batch.blocks += p.Hkv * (u.pairs + (u.single ? 1 : 0));
                batch.longest = max(batch.longest, tree_tiles(len_mine));
                batch.shortest = min(batch.shortest, tree_tiles(len_mine));
                batch.kinds |= (u.pairs ? 1 : 0) | (u.single ? 2 : 0);
            }
        }
        batch.blocks = __reduce_add_sync(0xffffffffu, batch.blocks);
        batch.units = __reduce_add_sync(0xffffffffu, mine);
        batch.longest = __reduce_max_sync(0xffffffffu, batch.longest);
        batch.shortest = __reduce_min_sync(0xffffffffu, batch.shortest);
        batch.kinds = __reduce_or_sync(0xffffffffu, batch.kinds);
        int share = tree_rules(li, batch, gridDim.x);
        if (share > 0) {             // (few sequences: units are counted otherwise)
            mine = 0;
            for (int b = b_first; b < b_last; ++b) {
                if (chunk > 1) seq_of(b, n_mine, row_mine, len_mine);
                mine += p.Hkv * tree_head_units(tree_units(li, n_mine, len_mine));
            }
        }
        int before = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, before, d);
            if (lane >= d) before += o;
        }
        const int total = __shfl_sync(0xffffffffu, before, 31);
        before -= mine;
        if (share == 0) share = tree_share(li, total, gridDim.x);
        const long long u0 = static_cast<long long>(blockIdx.x) * share;
        int start_seq = b_first, start_base = before;
        const uint32_t holds = __ballot_sync(0xffffffffu, before <= u0 && u0 < before + mine);
        if (holds && lane == __ffs(holds) - 1 && chunk > 1) {
            for (;; ++start_seq) {
                seq_of(start_seq, n_mine, row_mine, len_mine);
                const int units = p.Hkv * tree_head_units(tree_units(li, n_mine, len_mine));
                if (u0 < start_base + units) break;
                start_base += units;
            }
        }
        const int from = holds ? __ffs(holds) - 1 : 0;
        start_seq = __shfl_sync(0xffffffffu, start_seq, from);
        start_base = __shfl_sync(0xffffffffu, start_base, from);
        TreeWalk w;
        w.n = __shfl_sync(0xffffffffu, n_mine, from);
        w.row0 = __shfl_sync(0xffffffffu, row_mine, from);
        w.len = __shfl_sync(0xffffffffu, len_mine, from);
        tree_walk_begin(w, li, blockIdx.x, share, total, start_seq, start_base);
        TreeJoin join{0, 0, 0, 0, 0, 0, 0, 0};
        TreePart cur, e;
        e.t1 = 0;
        bool ok = true;
        auto issued = [&](int count) -> bool {
            while (*static_cast<volatile int*>(&sh.v_issued) < count) {
                __nanosleep(100);
                if (*static_cast<volatile uint32_t*>(&sh.wait.abort_flag)) return false;
            }
            __threadfence_block();
            return true;
        };
        auto publish = [&](int k) {
            if (!tree_walk_next(w, li, p.Hkv, seq_of, e)) e.t1 = -1;
            ok = __all_sync(0xffffffffu, ok && wait(sh.part_empty[k % NP], ((k / NP) & 1) ^ 1));
            if (!ok) return;
            if (e.t1 >= 0 && e.slot >= 0 && e.t0 == 0) join = TreeJoin{e.kvh, e.row_tile, e.two, e.n, e.row0, e.pieces, 0, 0};
            if (lane == 0) {
                sh.part[k % NP] = e;
                mbar_arrive(smem_addr(&sh.part_full[k % NP]));
            }
            __syncwarp();
        };
        for (int k = 0; ok; ++k) {
            cur = e;
            publish(k);
            if (!ok) break;
            if (k == 0) {
                if (e.t1 < 0) break;
                continue;
            }
            // the part's last tile holds the sequence's last key: V rows behind it hold whatever the page held, or were not loaded,
            // and 0 * NaN is NaN
            if (!kE4m3 && cur.t1 > cur.t0 && cur.t1 * kTileN > cur.len) {
                const int at = cur.tile0 + cur.t1 - cur.t0 - 1, s = at % NV;
                // (The list runs ahead of the loads, by more than a turn of the ring where parts are short: a phase of v_full says that it
                // is this tile's only once its load has been issued.  From there on the stage waits for the zeros.)
                ok = __all_sync(0xffffffffu, issued(at + 1) && wait(sh.v_full[s], (at / NV) & 1));
                if (!ok) break;
                const int keys = cur.len - (cur.t1 - 1) * kTileN;
                for (int i = lane; i < (kTileN - keys) * 8; i += 32) {
                    const uint32_t to = sV + s * Cfg::kVStage + (keys + (i >> 3)) * 128 + (i & 7) * 16;
#pragma unroll
                    for (int cc = 0; cc < Cfg::kVChunks; ++cc) st_shared_v4(to + cc * kChunkBytes, 0, 0, 0, 0);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.v_tail[kE4m3 ? 0 : s]));
            }
            if (e.t1 < 0) break;
        }
        // (contents that the other reads of the list clamp are reported here, by one CTA)
        if (blockIdx.x == 0) {
            for (int b = lane; b < p.B; b += 32) {
                draft_rows(a.t.cu_seqlens, b, p.B, a.t.total, a.t.max_tokens, p.status);
                clamped_len(p.seq_lens[b], p.max_pages, p.page_size, p.status);
            }
            __syncwarp();
        }
        // (after a wait that ran out the pieces are not joined; the results are invalid either way)
        if (lane == 0) {
            if (!ok) join.pieces = 0;
            a.join[blockIdx.x] = join;
        }
        __syncwarp();
    } else {
        // ============================================================ queries into their terms, codes of V into fp16
        setmaxnreg_dec<Cfg::kRegsOther>();
        if constexpr (kE4m3) {
            const int mine = warp & 3;
            // A lane has one row of every fourth group of 8 and one 16-byte piece of codes in 64 columns, two of fp16.  Eight neighbouring lanes
            // have four pieces of two rows r and r ^ 5: under the swizzle they meet all banks in the load and in both stores, and all
            // addresses of a lane are its own constants plus multiples of 1024.
            const int row = lane & 4 ? (lane >> 3) ^ 5 : lane >> 3, piece = lane & 3;
            const uint32_t in_even = row * 128 + ((piece ^ row) << 4), in_odd = in_even ^ 64u;
            const uint32_t out0 = row * 128 + (((2 * piece) ^ row) << 4), out1 = out0 ^ 16u;
            const int q_row = tid & (kTileM - 1), row_token = q_row / a.list.row_heads, row_head = q_row - row_token * a.list.row_heads;
            int s = 0, r = 0, n_q = 0;
            uint32_t ph = 1, ph_r = 0;
            bool ok = true;
            TreePart e;
            for (int k = 0; ok && take_part(k, e); ++k) {
                if (e.t0 == e.t1) continue;
                // The row's queries, scaled by a power of two that puts the largest into [2^14, 2^15) (from 2^127 down to 2^-112; a
                // smaller row by 2^126, which makes its entries, multiples of 2^-133, exact too), as fp16 and then as three
                // e5m2 terms: top byte, remainder, top byte, remainder, top byte.  They go where the queries were loaded to: a thread's row
                // lies in its own bytes before and after, and its pieces are taken in an order in which none is overwritten unread
                // (128 columns: the last term of the first 64 waits in local memory).  (Here and not by the softmax warps, which are
                // still at the part before: the first scores of a part came 7000 cycles after its beginning.)
                ok = __all_sync(0xffffffffu, wait(sh.q_full, n_q & 1));
                const int tc = a.list.head_chunks == 1 ? e.row_tile : e.row_tile / a.list.head_chunks, hc = e.row_tile - tc * a.list.head_chunks;
                const bool live = row_token < a.list.row_tokens && tc * a.list.row_tokens + row_token < e.n && hc * a.list.row_heads + row_head < a.group;
                uint32_t top = 0;
#pragma unroll 1
                for (int cc = 0; cc < Cfg::kQChunks; ++cc) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) {
                        const uint4 x = ld_shared_v4(sQ + Cfg::q_place(cc) + q_row * 128 + ((v ^ (q_row & 7)) << 4));
                        const uint32_t w4[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) top = max(top, max((w4[i] & 0x7fffu) << 16, w4[i] & 0x7fff0000u));
                    }
                }
                int sft = top ? 14 - (static_cast<int>(top >> 23) - 127) : 0;
                sft = sft > 126 ? 126 : (sft < -113 ? -113 : sft);
                const float mult = __uint_as_float(static_cast<uint32_t>(sft + 127) << 23);
                uint4 held[4];
#pragma unroll 1
                for (int cc = 0; cc < Cfg::kQChunks; ++cc) {
#pragma unroll 1
                    for (int u0 = 0; u0 < 4; ++u0) {               // 16 values: 16 bytes of each term
                        const int u = DQK == 128 && cc == 1 ? 3 - u0 : u0;
                        const uint32_t in = sQ + Cfg::q_place(cc) + q_row * 128;
                        const uint4 lo = ld_shared_v4(in + (((2 * u) ^ (q_row & 7)) << 4)), hi = ld_shared_v4(in + (((2 * u + 1) ^ (q_row & 7)) << 4));
                        const uint32_t w8[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                        uint32_t h[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) h[i] = live ? pack_f16x2(__uint_as_float(w8[i] << 16) * mult, __uint_as_float(w8[i] & 0xffff0000u) * mult) : 0u;
                        const uint32_t at = sQ + (cc >> 1) * kChunkBytes + q_row * 128 + ((((cc & 1) * 4 + u) ^ (q_row & 7)) << 4);
#pragma unroll
                        for (int term = 0; term < Cfg::kTerms; ++term) {
                            const uint4 bytes = make_uint4(__byte_perm(h[0], h[1], 0x7531), __byte_perm(h[2], h[3], 0x7531),
                                                           __byte_perm(h[4], h[5], 0x7531), __byte_perm(h[6], h[7], 0x7531));
                            if (DQK == 128 && cc == 0 && term == 2) held[u] = bytes;
                            else st_shared_v4(at + term * Cfg::kKBytes, bytes.x, bytes.y, bytes.z, bytes.w);
                            if (term + 1 < Cfg::kTerms) {
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    const uint32_t bits = h[i] & 0xff00ff00u;
                                    const __half2 rest = __hsub2(*reinterpret_cast<const __half2*>(&h[i]), *reinterpret_cast<const __half2*>(&bits));
                                    h[i] = *reinterpret_cast<const uint32_t*>(&rest);
                                }
                            }
                        }
                    }
                }
                if constexpr (DQK == 128) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) st_shared_v4(sQ + 2 * Cfg::kKBytes + q_row * 128 + ((u ^ (q_row & 7)) << 4), held[u].x, held[u].y, held[u].z, held[u].w);
                }
                sh.q_shift[n_q & 1][q_row] = static_cast<uint8_t>(127 - sft);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.q_ready));
                ++n_q;
                for (int t = e.t0; ok && t < e.t1; ++t) {
                    ok = __all_sync(0xffffffffu, wait(sh.raw_full[r], ph_r));
                    const uint32_t src = sRaw + r * kChunkBytes + mine * 1024;
                    const int keys = e.len - t * kTileN;
                    // (values behind the sequence's end hold whatever the page held: 0 * NaN is NaN)
                    const bool zeros = keys < kTileN;
                    constexpr int kDeep = Cfg::kVKeys / 32;          // loads ahead of the conversions: all of 64 columns of a stage
#pragma unroll 1
                    for (int part = 0; ok && part < Cfg::kVParts; ++part) {
                        ok = __all_sync(0xffffffffu, wait(sh.v_empty[s], ph));
                        if (!ok) break;
                        const uint32_t dst = sV + s * Cfg::kVStage + mine * 1024;
#pragma unroll
                        for (int c = 0; c < DV / 64; ++c) {
                            const uint32_t from = src + part * Cfg::kVKeys * 128 + (c & 1 ? in_odd : in_even), to = dst + c * Cfg::kVChunk;
                            uint4 x[kDeep];
#pragma unroll
                            for (int g = 0; g < kDeep; ++g) x[g] = ld_shared_v4(from + g * 4096);
                            if (zeros) {
#pragma unroll
                                for (int g = 0; g < kDeep; ++g)
                                    if (part * Cfg::kVKeys + (4 * g + mine) * 8 + row >= keys) x[g] = make_uint4(0, 0, 0, 0);
                            }
#pragma unroll
                            for (int g = 0; g < kDeep; ++g) {
                                const uint32_t at = to + g * 4096;
                                st_shared_v4(at + out0, e4m3x2_to_f16x2(x[g].x), e4m3x2_to_f16x2(x[g].x >> 16), e4m3x2_to_f16x2(x[g].y),
                                             e4m3x2_to_f16x2(x[g].y >> 16));
                                st_shared_v4(at + out1, e4m3x2_to_f16x2(x[g].z), e4m3x2_to_f16x2(x[g].z >> 16), e4m3x2_to_f16x2(x[g].w),
                                             e4m3x2_to_f16x2(x[g].w >> 16));
                            }
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_addr(&sh.v_full[s]));
                        if (++s == NV) { s = 0; ph ^= 1u; }
                    }
                    if (lane == 0) mbar_arrive(smem_addr(&sh.raw_empty[r]));
                    if (++r == NR) { r = 0; ph_r ^= 1u; }
                }
            }
        }
    }

    // ---------------------------------------------------------------- teardown (all warps)
    tc_fence_before_sync();
    __syncthreads();
    if (sh.wait.abort_flag) {         // (uniform: it is set before the barrier or not at all)
        // copies and MMAs that are still under way end before their memory is given back
        if (warp == 8 && elect_one()) {
            tc_commit(smem_addr(&sh.mma_done));
            tree_settle(sh.mma_done, 0);
        }
        if (tid == 0) {
            tree_settle_ring(sh.k_full, NK, sh.loads[0]);
            if constexpr (kE4m3) tree_settle_ring(sh.raw_full, NR, sh.loads[1]);
            else tree_settle_ring(sh.v_full, NV, sh.loads[1]);
            tree_settle_ring(&sh.q_full, 1, sh.loads[2]);
        }
        __syncthreads();
    }
    if (warp == 8) tmem_dealloc(tmem, 512);
}

// ------------------------------------------------------------------ joining

// The pieces of a row block that several CTAs share, in their order: O = sum_c 2^(m_c - m) O_c / sum_c 2^(m_c - m) l_c.  32 rows a CTA (a
// lane each), 16 columns a warp, so that loads are 512 neighbouring bytes and a thread stores 32.  Bound by the pieces' bytes, which
// are in L2.
template <int DV, bool kTwo>
__global__ void __launch_bounds__(DV * 2)
fa_tree_join_kernel(const PagedParams p, const TreeArgs a) {
    constexpr int kRowBlocks = kTileM / 32;
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int cta = blockIdx.x / (kRowBlocks * (kTwo ? 2 : 1)), at = blockIdx.x - cta * (kRowBlocks * (kTwo ? 2 : 1));
    const TreeJoin e = a.join[cta];
    const int t = at / kRowBlocks, row = (at - t * kRowBlocks) * 32 + (threadIdx.x & 31);
    if (e.pieces == 0 || (t == 1 && !e.two)) return;
    const int tile = e.row_tile + t, tc = tile / a.list.head_chunks, hc = tile - tc * a.list.head_chunks;
    const int in = row / a.list.row_heads, token = tc * a.list.row_tokens + in, head = hc * a.list.row_heads + row - in * a.list.row_heads;
    if (in >= a.list.row_tokens || token >= e.n || head >= a.group) return;
    auto slot = [&](int c) { return a.part + (c == 0 ? 2ll * cta + 1 : 2ll * (cta + c)) * tree_slot_floats(DV, kTwo); };
    constexpr int kMl = (kTwo ? 2 : 1) * kTileM * DV, kBatch = 2;
    const int col = (threadIdx.x >> 5) * 16;
    float4 y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    // (under a running maximum, so that references, sums and values of two pieces are all loaded at once)
    float m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int c = 0; c < e.pieces; c += kBatch) {
        float mc[kBatch], lc[kBatch];
        float4 x[kBatch][4];
#pragma unroll
        for (int q = 0; q < kBatch; ++q) {
            mc[q] = -INFINITY;
            lc[q] = 0.f;
            if (c + q >= e.pieces) break;
            const float* const s = slot(c + q);
            mc[q] = __ldcg(s + kMl + t * 2 * kTileM + row);
            lc[q] = __ldcg(s + kMl + (t * 2 + 1) * kTileM + row);
            const float4* const o = reinterpret_cast<const float4*>(s) + (t * (DV / 4) + col / 4) * kTileM + row;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[q][i] = __ldcg(o + i * kTileM);
        }
        float top = m;
#pragma unroll
        for (int q = 0; q < kBatch; ++q) top = fmaxf(top, mc[q]);
        const float keep = m == -INFINITY ? 0.f : ptx::exp2_approx(m - top);
        m = top;
        l *= keep;
#pragma unroll
        for (int i = 0; i < 4; ++i) { y[i].x *= keep; y[i].y *= keep; y[i].z *= keep; y[i].w *= keep; }
#pragma unroll
        for (int q = 0; q < kBatch; ++q) {
            if (c + q >= e.pieces) break;
            const float f = mc[q] == -INFINITY ? 0.f : ptx::exp2_approx(mc[q] - top);
            l = fmaf(f, lc[q], l);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i].x = fmaf(f, x[q][i].x, y[i].x);
                y[i].y = fmaf(f, x[q][i].y, y[i].y);
                y[i].z = fmaf(f, x[q][i].z, y[i].z);
                y[i].w = fmaf(f, x[q][i].w, y[i].w);
            }
        }
    }
    const bool any = l > 0.f || l != l;
    const int hq = e.kvh * a.group + head;
    const long long q_row = e.row0 + token;
    const float f = (p.v_scale ? p.v_scale[e.kvh] : 1.f) / l;
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[2 * i] = any ? ptx::pack_bf16x2(f * y[i].x, f * y[i].y) : 0u;
        r[2 * i + 1] = any ? ptx::pack_bf16x2(f * y[i].z, f * y[i].w) : 0u;
    }
    uint4* const out = reinterpret_cast<uint4*>(p.O + q_row * p.o_st + hq * p.o_sh + col);
    out[0] = make_uint4(r[0], r[1], r[2], r[3]);
    out[1] = make_uint4(r[4], r[5], r[6], r[7]);
    if (threadIdx.x < 32 && p.lse) p.lse[static_cast<long long>(hq) * a.t.total + q_row] = any ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace fa
