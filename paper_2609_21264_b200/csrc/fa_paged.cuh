// Attention of the last few tokens of every sequence over a paged key/value cache, for sm_100a.
//
// Per (sequence, K/V head) there are R = (Hq / Hkv) * Sq query rows, one to a few dozen, against thousands of keys: a byte
// of K and V is read once for a block of rows (up to 16, 32 or 64 of them; more rows are more blocks, each with a pass over the keys of
// its own, next to one another in the list) and used for its R rows, 2 R (dqk + dv) / ((dqk + dv) * bytes) = R .. 2R flops a byte, far below the 250 that
// the tensor cores need to be the bound.  The kernel is built to stream HBM:
//
//   * The products are turned around, keys on the 128 lanes of the accumulator and query rows on its columns:
//         S^T [128 keys x rows]  = K_tile [128 x dqk] Q^T          (tcgen05.mma, M = 128, N = rows)
//         O^T [dv x rows]       += V_tile^T [dv x 128] P^T          (V read MN-major, P^T written by the softmax warps)
//     so an MMA of 16 rows costs 16 columns and not a padded tile of 128, and a thread exponentiates rows, not 128 keys, per tile.
//   * The tiles of all sequences and heads form one list; CTA c takes the c-th of equal consecutive shares (the lengths are read on
//     the device).  Lengths that differ by orders of magnitude cost nothing, and no SM waits for a wave.  A (sequence, head)
//     that several CTAs share is joined by the one that finishes last, in the order of the CTAs (equal calls give equal bits).
//   * A ring of K/V tiles (two to six stages, all that the shared memory holds) runs across the boundaries of sequences.
//
// Two groups of four softmax warps take the tiles in turn; each has its own scores (two buffers), probabilities (two), reference maximum,
// row sums and accumulator, so that no tile waits for the one before it.  A thread owns a key of the tile: the row maximum runs
// across lanes, so it is taken rarely: the reference of a row moves only when some score exceeds it by more than kTauLog2 (one
// barrier with a vote per tile; the reductions, and the rescaling of O^T, on the few tiles where the vote says so).
// When a part of the list ends (a sequence and head, or the CTA's share), a third group of warps merges the two accumulators and
// writes the result or the partial result, under the next part's tiles.
//
// e4m3 caches: K and V enter the 8-bit MMA as they are; the bf16 queries and the fp32 probabilities as sums of three e5m2 terms,
// each on columns of its own (N = 3 rows): x -> fp16, top byte, remainder, top byte, remainder, top byte, 9 significant bits.
// Nothing is dequantised and both sides keep at least bf16's precision.  The probabilities are scaled by 2^11 so that weights of
// 2^-19 of the largest still have 9 bits.
//
// Drafted tokens (kTree): as many rows as a block has at most, a number of tokens and a word of the mask for each of them that are the
// sequence's own.  (Rows that a sequence does not have end the loop over the stores; tested one by one they cost a part 1 us: 64 sequences of
// 300 keys, 64/8 heads, 32 rows 27.5 to 24.3 us, where equally many tokens without a mask take 23.7.)
//
// Differential attention: two maps are two groups of columns.  Map a's scores are the k-steps of its half of K, its
// probabilities meet the same V tile, and the epilogue subtracts and normalises: K and V are read once for both maps of a block, of
// 16 rows here (group * Sq = 64 rows read the cache four times).
//
// Roles (512 threads): warps 0 / 2 TMA loads of K / V (a lane per page box), warps 1 / 3 issue of the score / value products (one thread
// each: a tile costs an issuing thread 600 cycles of waits, descriptors and commits, as much as a tile of head size 64 has in
// all), warps 4-7 and 8-11 softmax groups 0 and 1 (thread = key of the tile = lane of S^T), warps 12-15 the list of parts, the
// query rows, and the results (thread = output column = lane of O^T).
#pragma once

#include <math.h>
#include <stddef.h>

#include <type_traits>

#include "fa_paged_common.cuh"

namespace fa {

namespace ptx {

FA_DEVI void st_shared_u64(uint32_t addr, uint32_t lo, uint32_t hi) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(lo), "r"(hi) : "memory");
}

}  // namespace ptx

// Bounded waits.  The result warps wait, directly or in turn, for every other role: they alone watch the clock.  Once one of their
// waits has run out, the abort flag ends everybody's, and all roles fall through to the common exit.  (Every wait with a
// clock of its own, as ptx::mbar_wait, in some twenty places would take more than the instruction cache holds.)
struct PagedWait {
    uint32_t abort_flag;
    uint32_t* status;
    unsigned long long limit_ns;
};
FA_DEVI bool paged_wait(uint64_t& bar, uint32_t parity, PagedWait* ctx) {
    const uint32_t at = ptx::smem_addr(&bar);
    if (ptx::mbar_try_wait(at, parity)) return true;
    do {
        if (*static_cast<volatile uint32_t*>(&ctx->abort_flag)) return false;
    } while (!ptx::mbar_try_wait(at, parity));
    return true;
}
static __device__ __noinline__ bool paged_wait_long(uint64_t* bar, uint32_t parity, PagedWait* ctx, uint32_t who) {
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

// (a call costs some 400 cycles, so the first look is taken here)
FA_DEVI bool paged_wait_timed(uint64_t* bar, uint32_t parity, PagedWait* ctx, uint32_t who) {
    return ptx::mbar_try_wait(ptx::smem_addr(bar), parity) || paged_wait_long(bar, parity, ctx, who);
}

// ------------------------------------------------------------------ the list of work units and its shares

// The list holds every (sequence, K/V head, block of rows) in that order, one unit per tile of 128 keys; a sequence without keys has
// one empty tile, so that its rows are written.  CTA c takes units [c * share, (c + 1) * share).
//
// What a row block costs beside its tiles (query rows, first maxima, result: about what 128 KB take to load) is counted in units
// too where there are row blocks for all CTAs and they are short, or the CTAs that got the batch's short sequences would
// finish last: 48 sequences of 65 to 1000 keys, 8 K/V heads, 25.2 us with two units for it, 27.7 with one, 34.5 without; over
// e4m3 23.2 with three, 36 without.  With more than 768 KB in a block on average most CTAs have equally many parts and the bytes
// alone decide (160 row blocks 192/128 of 10 tiles 29.8 us, with one unit 31.2; 64 sequences of 65 to 4096 keys level).
// (The host refuses calls whose list could be longer than 32 bits can count.)
//
// Small calls: joining the pieces of a row block costs 4 to 5 us, a tile 0.6 us of a CTA's time.  So where there is a CTA for every row
// block and no sequence has more than kWholeTiles tiles, all blocks count as many units as the longest (`pad` tiles), the shares
// fall on their borders, and nothing is split (400 keys, 8 K/V heads: 9.4 us, against 11.3).  The blocks of a single sequence
// count a multiple of the share, so that a CTA has one part (777 keys 11.1 us, against 12.3; 8000 keys 18.3, against 20.1).
constexpr int kMostPartCost = 3, kWholeTiles = 6;
__host__ __device__ inline int paged_tiles(int len) { return len > 0 ? (len + kTileN - 1) / kTileN : 1; }
__host__ __device__ inline int paged_len(const PagedParams& p, int b, uint32_t* status) {
    return clamped_len(p.seq_lens[b], p.max_pages, p.page_size, status);
}
// How a call's units are counted: tiles that every row block has at least (0: its own), units beside them, a CTA's share (0: what
// the total gives).
struct PagedCount { int pad, cost, share; };
// Units that a CTA takes at least.  Drafted tokens: a long sequence in few row blocks has a CTA's tiles (0.6 us each) on one side and its
// pieces, which one CTA joins (some 0.4 us each), on the other; tiles / s + s is least where s is their root.  One K/V head, 32 rows, one
// sequence of 17353 keys: 29.7 us in pieces of two tiles, 17.7 in 14 pieces; 2 of 100000 57 in 74 pieces each, 43 in 34; 8 heads, 8000 keys
// 20.0 in 18 pieces, 18.1 in 9.  (Other calls keep the shares, and so the bits, that they have.)
__host__ __device__ inline int paged_least(const PagedParams& p, bool tree, int most_tiles) {
    const int root = tree ? static_cast<int>(ceilf(sqrtf(static_cast<float>(most_tiles) * (2.f / 3.f)))) : 0;
    return root > p.least_units ? root : p.least_units;
}
__host__ __device__ inline PagedCount paged_count(const PagedParams& p, int least, int ctas, int most_tiles, int all_tiles) {
    const long long blocks = static_cast<long long>(p.B) * p.Hkv * p.row_blocks;
    PagedCount c{0, 0, 0};
    if (most_tiles <= kWholeTiles && blocks <= ctas) {
        c.pad = c.share = most_tiles;
    } else if (p.B == 1 && 2 * blocks <= ctas) {
        // (a block has less than one share more than its tiles fill: the shares do not outnumber the CTAs)
        const int spare = ctas - static_cast<int>(blocks), per = (all_tiles + spare - 1) / spare;
        c.share = per < least ? least : per;
        c.pad = (most_tiles + c.share - 1) / c.share * c.share;
    } else if (blocks >= ctas && all_tiles < p.long_tiles * blocks) {
        c.cost = p.part_cost;
    }
    return c;
}
// Units of a row block, and of a sequence, from its length.
__host__ __device__ inline int paged_block_units(int len, PagedCount c) {
    const int nt = paged_tiles(len);
    return (nt < c.pad ? c.pad : nt) + c.cost;
}
__host__ __device__ inline int paged_units(const PagedParams& p, int len, PagedCount c) { return paged_block_units(len, c) * p.Hkv * p.row_blocks; }
__host__ __device__ inline int paged_share(int least, int units, int ctas, PagedCount c) {
    if (c.share > 0) return c.share;
    const int per = static_cast<int>((static_cast<unsigned>(units) + ctas - 1) / ctas);
    return per < least ? least : per;
}

// A part of the list as the roles of a CTA see it: tiles [t0, t1) of one (sequence, K/V head, row block).
struct PagedEntry {
    int b, kvh, rb, len, t0, t1;  // t1 < 0: the end of the CTA's share
    int tile0;                    // index of the part's first tile in the CTA's share
    int slot;                     // of the partial result, -1: the part is whole
    int pieces, first_cta;        // of the whole (sequence, head, block), and the slot of its first piece
    int first_slot;
};

// What CTA `cta` with units [u0, u1) has of row block hr = head * row_blocks + block of sequence b, whose first unit is `base`;
// false where that is nothing.  A CTA leaves at most two parts unfinished, its first and its last: two slots for partial results.
__host__ __device__ inline bool paged_entry(const PagedParams& p, int cta, int share, int u0, int u1, int b, int base, int len, PagedCount c, int hr,
                                            PagedEntry& e) {
    const int nt = paged_tiles(len), ub = base + (hr + 1) * paged_block_units(len, c), ua = ub - nt;       // units of its tiles
    const int v0 = u0 > ua ? u0 : ua, v1 = u1 < ub ? u1 : ub;
    e.b = b;
    e.kvh = hr / p.row_blocks;
    e.rb = hr - e.kvh * p.row_blocks;
    e.len = len;
    e.t0 = v0 - ua;
    e.t1 = v1 - ua;
    e.slot = -1;
    e.pieces = 1;
    e.first_cta = cta;
    e.first_slot = -1;
    if (v1 - v0 < nt) {
        e.first_cta = ua / share;
        e.pieces = (ub - 1) / share - e.first_cta + 1;
        e.first_slot = 2 * e.first_cta + (ua > e.first_cta * share ? 1 : 0);
        e.slot = 2 * cta + (ua > u0 ? 1 : 0);
    }
    return v0 < v1;
}

// ------------------------------------------------------------------ configuration

constexpr int kPartRing = 8;
// pieces whose weights are found at a time (16 against 8: 8000 keys, 8 K/V heads, 18 pieces a row block, 18.7 to 18.2 us)
__host__ __device__ constexpr int paged_merge_pieces(int states) { return states <= 32 ? 16 : 8; }

// Registers per thread after the per-role reallocation (512 threads start with 128 each): 128 x 80 + 256 x 136 + 128 x 160 = 65536;
// with 64 states per softmax thread 256 x 152 and 128 x 128.
constexpr int kPagedRegsOther = 80;
__host__ __device__ constexpr int paged_regs_softmax(int states) { return states <= 32 ? 136 : 152; }

template <int kRows, int kMaps>
struct PagedShared {
    uint64_t k_full[6], k_empty[6], v_full[6], v_empty[6];
    uint64_t q_full[2], q_empty[2];
    uint64_t s_full[2][2], s_empty[2][2], p_full[2][2], pv_done[2][2];      // [group][buffer]
    uint64_t acc_full[2], acc_empty[2];                      // [accumulator buffer]
    uint64_t part_full[kPartRing], stat_full[kPartRing];
    PagedEntry part[kPartRing];
    uint32_t tmem_base;
    PagedWait wait;
    uint32_t is_last[2];          // of even and odd parts
    int start_b, start_base;
    int warp_sums[4], warp_longest[4];
    alignas(16) float c[2][kRows];                       // per query buffer: factor of a score (log2 units)
    int i[2][kRows];                                     // place among the new tokens
    // per group: bias - reference maximum, +inf where no key has been seen; and the same with 0 there
    alignas(16) float neg_m[2][kMaps * kRows];
    alignas(16) float neg_p[2][kMaps * kRows];
    alignas(16) float rescale[2][kMaps * kRows];
    float red[2][4][kMaps * kRows], red_l[2][4][kMaps * kRows];
    float stat_m[kPartRing][2][kMaps * kRows], stat_l[kPartRing][2][kMaps * kRows];      // [part][group]
    // of the result warps
    float factor[2][kMaps * kRows];
    static constexpr int kMergePieces = paged_merge_pieces(kMaps * kRows);
    float piece_m[kMergePieces][kMaps * kRows], piece_l[kMergePieces][kMaps * kRows];
    float sq[4][kRows];
    // The rows of a block, apart from the part's sequence and K/V head: offsets in Q and O (-1: a padding row), place among the new
    // tokens (Q: of the last one for padding), query head of the group.  They change with the block of rows alone.
    long long row_q[kRows], row_o[kRows];
    int row_place[kRows], row_i[kRows], row_h[kRows];
};
// Drafted tokens: those of a part's sequence, and the first one's row (PagedShared::i holds every row's word of the mask).
template <int kRows, int kMaps>
struct PagedTreeShared : PagedShared<kRows, kMaps> { int n[kPartRing], row0[kPartRing]; };

template <int DQK, int DV, bool kE4m3, bool kDiff, int kRows>
struct PagedCfg {
    static constexpr int kMaps = kDiff ? 2 : 1;
    static constexpr int kTerms = kE4m3 ? 3 : 1;                // of the queries
    // of the probabilities: the difference of two maps loses what they have in common, so these keep 16 bits over a bf16 cache too
    // (one bf16 term: 1.5 times the error of the rounded output alone; two: none that shows, at the same speed).  One map over a bf16
    // cache keeps one term, as the other kernels on 16-bit inputs do: 2.2e-3 of the result, where its rounding alone makes 1.7e-3.
    static constexpr int kPTerms = kE4m3 ? 3 : (kDiff ? 2 : 1);
    static constexpr int kStates = kMaps * kRows;               // softmax states of a group
    static constexpr int kSCols = kStates * kTerms, kCols = kStates * kPTerms;      // columns of S^T and of O^T
    static constexpr int kElem = kE4m3 ? 1 : 2;
    static constexpr int kChunk = 128 / kElem;                  // columns of a 128-byte row of a chunk
    static constexpr int kKChunks = (DQK + kChunk - 1) / kChunk;
    static constexpr int kVChunks = (DV + kChunk - 1) / kChunk;
    static constexpr int kKBytes = kKChunks * kChunkBytes;
    static constexpr int kVBytes = kVChunks * kChunkBytes;
    static constexpr int kQRows = kTerms * kRows;               // rows of the staged queries
    static constexpr int kQChunkBytes = kQRows * 128;
    static constexpr int kQBytes = kKChunks * kQChunkBytes;
    // P^T as it is multiplied: columns of O^T in groups of 16 bytes, a group is the 128 keys' 16 bytes one after the other
    static constexpr int kPGroupBytes = 128 * 16;
    static constexpr int kPBytes = kCols * kElem / 16 * kPGroupBytes;
    // bf16 values of 64: the upper 64 lanes of O^T multiply a block of zeros
    static constexpr bool kZeroBlock = !kE4m3 && DV == 64;
    static constexpr int kZeroBytes = kZeroBlock ? 2048 : 0;
    static constexpr int kBudget = 227 * 1024 - static_cast<int>(sizeof(PagedShared<kRows, kMaps>));
    // two probability buffers per group, one where that makes room for a second or third stage
    static constexpr int stages_with(int p_bufs) { return (kBudget - 2 * kQBytes - 2 * p_bufs * kPBytes - kZeroBytes) / (kKBytes + kVBytes); }
    static constexpr int kPBufs = stages_with(2) >= 3 || stages_with(2) == stages_with(1) ? 2 : 1;
    static constexpr int kFixedBytes = 2 * kQBytes + 2 * kPBufs * kPBytes + kZeroBytes;
    static constexpr int kFit = (kBudget - kFixedBytes) / (kKBytes + kVBytes);
    static constexpr int kStages = kFit > 6 ? 6 : kFit;
    static_assert(kStages >= 2, "shared memory budget exceeded");
    static constexpr int kTileBytes = kFixedBytes + kStages * (kKBytes + kVBytes);
    // score buffers of both groups (4 or 2) and accumulators of both groups (for 2 parts or 1), as TMEM has room
    static constexpr int kSBufs = 4 * kSCols + 2 * kCols <= 512 ? 4 : 2;
    static constexpr int kOBufs = kSBufs * kSCols + 4 * kCols <= 512 ? 2 : 1;
    static constexpr int kUsedCols = kSBufs * kSCols + 2 * kOBufs * kCols;
    static constexpr int kTmemCols = kUsedCols <= 64 ? 64 : kUsedCols <= 128 ? 128 : kUsedCols <= 256 ? 256 : 512;
    static_assert(kUsedCols <= 512 && kSCols % 16 == 0 && kCols <= 256, "accumulators");
    static constexpr int kKSteps = DQK * kElem / 32;            // k-steps of 32 bytes
    static constexpr int kPSteps = 128 * kElem / 32;
    // exponents above the reference that a score may reach before the reference moves, and the scaling of P
    static constexpr float kTauLog2 = kE4m3 ? 4.5f : 8.f;      // 2^15.5 is below e5m2's largest number, 57344
    static constexpr float kBias = kE4m3 ? 11.f : 0.f;
};

template <int DQK, int DV, bool kE4m3, bool kDiff, int kRows, bool kTree = false>
constexpr int paged_smem_bytes() {
    using Cfg = PagedCfg<DQK, DV, kE4m3, kDiff, kRows>;
    return Cfg::kTileBytes + static_cast<int>(kTree ? sizeof(PagedTreeShared<kRows, Cfg::kMaps>) : sizeof(PagedShared<kRows, Cfg::kMaps>));
}
// Bytes of a partial result: unnormalised O of every state (fp32) and its maximum and sum.
constexpr long long paged_slot_bytes(int dv, int states) { return states * (dv + 2) * 4ll; }

// ------------------------------------------------------------------ kernel

// Low word of a shared-memory matrix descriptor; the high word is the same for all operands with 128-byte swizzle (8-row groups
// 1024 bytes apart, version 1).  P^T is not swizzled: blocks of 8 keys x 16 bytes, 128 bytes apart along the keys (the low
// word's offset) and a group (128 keys) apart along the columns.
FA_DEVI uint32_t desc_lo(uint32_t saddr, uint32_t lbo_bytes) { return ((saddr & 0x3ffffu) >> 4) | ((lbo_bytes >> 4) << 16); }
template <bool kE4m3, bool kPlainB = false>
FA_DEVI void paged_mma(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    constexpr uint64_t kHi = static_cast<uint64_t>((1024u >> 4) | (1u << 14) | (2u << 29)) << 32;
    constexpr uint64_t kHiB = kPlainB ? static_cast<uint64_t>((2048u >> 4) | (1u << 14)) << 32 : kHi;
    if constexpr (kE4m3) ptx::mma_ss_f8(d, kHi | a_lo, kHiB | b_lo, idesc, accumulate);
    else ptx::mma_ss(d, kHi | a_lo, kHiB | b_lo, idesc, accumulate);
}

// kTree: drafted tokens, one block of rows (so 32 drafts at most: a word of the mask each).  Every sequence has a number of tokens of its own,
// and what it sees of them is in its row's word; a sequence without drafts counts as one without keys.
template <int DQK, int DV, bool kE4m3, bool kDiff, int kRows, bool kTree = false>
__global__ void __launch_bounds__(512, 1)
fa_paged_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const PagedParams p) {
    static_assert(!kTree || (!kDiff && kRows <= 32), "one map, one word of a mask");
    using Cfg = PagedCfg<DQK, DV, kE4m3, kDiff, kRows>;
    using PlainShared = PagedShared<kRows, Cfg::kMaps>;
    static_assert(offsetof(PlainShared, i) % 16 == 0, "read in pieces of 16 bytes");
    using Shared = std::conditional_t<kTree, PagedTreeShared<kRows, Cfg::kMaps>, PagedShared<kRows, Cfg::kMaps>>;
    using namespace ptx;
    constexpr int NS = Cfg::kStages, kMaps = Cfg::kMaps, kTerms = Cfg::kTerms, kPTerms = Cfg::kPTerms, kStates = Cfg::kStates, kCols = Cfg::kCols;
    constexpr int kBufs = Cfg::kSBufs / 2;        // score buffers of a group
    constexpr int kOBufs = Cfg::kOBufs, kPBufs = Cfg::kPBufs;

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(smem_raw + Cfg::kTileBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t smem_base = smem_addr(smem_raw);
    const uint32_t sK = smem_base, sV = sK + NS * Cfg::kKBytes, sQ = sV + NS * Cfg::kVBytes, sP = sQ + 2 * Cfg::kQBytes,
                   sZero = sP + 2 * Cfg::kPBufs * Cfg::kPBytes;

    grid_launch_dependents();
    if ((smem_base & 1023u) != 0u) {          // uniform over the CTA; nothing has been set up yet
        grid_dependency_wait();
        if (tid == 0 && p.status) {
            volatile uint32_t* sw = p.status;
            sw[1] = kSiteSmemAlign;
            sw[0] = 3u;                       // FA_ERR_CUDA
            __threadfence_system();
        }
        return;
    }
    if (tid == 0) {
        sh.wait.abort_flag = 0;
        sh.wait.status = p.status;
        sh.wait.limit_ns = p.wait_limit_ns;
        for (int s = 0; s < NS; ++s) {
            mbar_init(smem_addr(&sh.k_full[s]), 1);
            mbar_init(smem_addr(&sh.k_empty[s]), 1);
            mbar_init(smem_addr(&sh.v_full[s]), 1);
            mbar_init(smem_addr(&sh.v_empty[s]), 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(smem_addr(&sh.q_full[w]), 4);       // the four warps that stage the rows
            mbar_init(smem_addr(&sh.q_empty[w]), 3);      // the last score MMA and the two softmax groups
            for (int i = 0; i < 2; ++i) {
                mbar_init(smem_addr(&sh.s_full[w][i]), 1);
                mbar_init(smem_addr(&sh.s_empty[w][i]), 4);     // four warps
                mbar_init(smem_addr(&sh.p_full[w][i]), 4);      // four warps
                mbar_init(smem_addr(&sh.pv_done[w][i]), 1);
            }
            mbar_init(smem_addr(&sh.acc_full[w]), 1);
            mbar_init(smem_addr(&sh.acc_empty[w]), 1);
        }
        for (int i = 0; i < kPartRing; ++i) {
            mbar_init(smem_addr(&sh.part_full[i]), 1);
            mbar_init(smem_addr(&sh.stat_full[i]), 8);          // the softmax warps
        }
        fence_mbar_init();
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
    }
    if (warp == 1) {
        tmem_alloc(smem_addr(&sh.tmem_base), Cfg::kTmemCols);
        tmem_relinquish_alloc_permit();
    }
    if constexpr (Cfg::kZeroBlock) {
        if (tid < 128) st_shared_v4(sZero + tid * 16, 0, 0, 0, 0);
        fence_proxy_async_smem();
    }
    const int group = p.Hq / p.Hkv;
    auto rows_of_q = [&](int rb, int r) {
        const int rr = rb * kRows + r, i = rr / group;
        sh.row_q[r] = i < p.Sq ? i * p.q_st + (rr - i * group) * p.q_sh : -1;
        sh.row_place[r] = min(i, p.Sq - 1);
    };
    auto rows_of_o = [&](int rb, int r) {
        const int rr = rb * kRows + r, i = rr / group;
        sh.row_o[r] = i < p.Sq ? i * p.o_st + (rr - i * group) * p.o_sh : -1;
        sh.row_i[r] = i;
        sh.row_h[r] = rr - i * group;
    };
    if (warp >= 12) {
        if ((tid & 127) < kRows) {
            rows_of_q(0, tid & 127);
            rows_of_o(0, tid & 127);
        }
        // lengths and block table towards L2 (a line each; the streams of other calls have usually driven them out): list and loads
        // wait for one after the other
        const int at = tid & 127, per_row = (p.max_pages + 31) / 32, line = blockIdx.x * 128 + at, b = line / per_row;
        if (at * 32 < p.B) prefetch_l2(p.seq_lens + at * 32);
        if constexpr (kTree) {
            if (p.cu_seqlens && at * 32 < p.B) prefetch_l2(p.cu_seqlens + at * 32);
        }
        if (b < p.B) prefetch_l2(p.block_table + b * p.table_stride + (line - b * per_row) * 32);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem_base;
    // (everything so far ran beside the kernel before; from here on its results may be read)
    grid_dependency_wait();
    // TMEM: S^T of group w, buffer i; behind them O^T of accumulator buffer ob, group w
    auto s_col = [&](int w, int i) -> uint32_t { return (w * kBufs + i) * Cfg::kSCols; };
    auto o_col = [&](int ob, int w) -> uint32_t { return Cfg::kSBufs * Cfg::kSCols + (ob * 2 + w) * kCols; };
    PagedWait* const wait = &sh.wait;
    // length of sequence b in the list, and (d) its drafts
    auto seq_len = [&](int b, uint32_t* status, DraftRows& d) -> int {
        const int len = paged_len(p, b, status);
        if constexpr (!kTree) return len;
        d = draft_rows(p.cu_seqlens, b, p.B, p.total, p.Sq, status);
        return d.count > 0 ? len : 0;
    };
    auto wait_part = [&](int k) -> bool { return paged_wait(sh.part_full[k % kPartRing], (k / kPartRing) & 1, wait); };

    if (warp == 0 || warp == 2) {
        // ============================================================ TMA loads of K (warp 0) or V (warp 2)
        setmaxnreg_dec<kPagedRegsOther>();
        // (one piece of code for both: the instruction cache is what short sequences run into)
        {
            const bool is_v = warp == 2;
            constexpr int kMaxChunks = Cfg::kKChunks > Cfg::kVChunks ? Cfg::kKChunks : Cfg::kVChunks;
            const int chunks = is_v ? Cfg::kVChunks : Cfg::kKChunks, stage_bytes = is_v ? Cfg::kVBytes : Cfg::kKBytes;
            const CUtensorMap* tm = is_v ? &tm_v : &tm_k;
            uint64_t* const full = is_v ? sh.v_full : sh.k_full;
            uint64_t* const empty = is_v ? sh.v_empty : sh.k_empty;
            const uint32_t dst0 = is_v ? sV : sK;
            const int box = p.box_rows, shift = __ffs(kTileN / box) - 1, boxes = 1 << shift, tiles_ahead = 32 >> shift;
            int n = 0, s = 0;
            uint32_t parity = 1;
            bool ok = true;
            for (int k = 0; ok; ++k) {
                ok = __all_sync(0xffffffffu, wait_part(k));
                if (!ok) break;
                const PagedEntry e = sh.part[k % kPartRing];
                if (e.t1 < 0) break;
                const int* const table = p.block_table + e.b * p.table_stride;
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
                    ok = __all_sync(0xffffffffu, paged_wait(empty[s], parity, wait));
                    if (!ok) break;
                    const uint32_t bar = smem_addr(&full[s]);
                    const int n_box = min(boxes, (max(0, e.len - t * kTileN) + box - 1) / box);
                    if (!(is_v && p.debug_drop_v_load && n == 0)) {
                        if (lane == 0) mbar_arrive_expect_tx(bar, n_box * box * 128 * chunks);
                        __syncwarp();
                        if (lane < n_box) {
#pragma unroll
                            for (int c = 0; c < kMaxChunks; ++c)
                                if (c < chunks) tma_load_4d(dst0 + s * stage_bytes + c * kChunkBytes + lane * box * 128, tm, bar, c * Cfg::kChunk, slot, e.kvh, page);
                        }
                        __syncwarp();
                    }
                    if (++s == NS) { s = 0; parity ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        // ============================================================ score products, one thread
        setmaxnreg_dec<kPagedRegsOther>();
        if (elect_one()) {
            constexpr uint32_t kIdescQK = kE4m3 ? (make_idesc_e4m3_f32(128, Cfg::kQRows, false, false) | (1u << 10))      // B: e5m2
                                                : make_idesc_bf16_f32(128, Cfg::kQRows, false, false);
            constexpr int kPerMap = Cfg::kKSteps / kMaps;
            const uint32_t k_lo0 = desc_lo(sK, 16), q_lo0 = desc_lo(sQ, 16);
            int n = 0, s = 0;
            uint32_t k_parity = 0;
            bool ok = true;
            for (int k = 0; ok; ++k) {
                if (!wait_part(k)) break;
                const int tiles = sh.part[k % kPartRing].t1 - sh.part[k % kPartRing].t0;
                if (sh.part[k % kPartRing].t1 < 0) break;
                if (!paged_wait(sh.q_full[k & 1], (k >> 1) & 1, wait)) break;
                const uint32_t q_lo = q_lo0 + (k & 1) * (Cfg::kQBytes >> 4);
                for (int t = 0; t < tiles; ++t, ++n) {
                    const int w = n & 1, i = (n >> 1) % kBufs;
                    ok = paged_wait(sh.s_empty[w][i], (((n >> 1) / kBufs) & 1) ^ 1, wait) &&
                         paged_wait(sh.k_full[s], k_parity, wait);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t k_lo = k_lo0 + s * (Cfg::kKBytes >> 4), d = tmem + s_col(w, i);
#pragma unroll
                    for (int m = 0; m < kMaps; ++m)
#pragma unroll
                        for (int j = 0; j < kPerMap; ++j) {
                            const int ks = m * kPerMap + j;
                            paged_mma<kE4m3>(d + m * Cfg::kQRows, k_lo + (((ks / 4) * kChunkBytes + (ks % 4) * 32) >> 4),
                                             q_lo + (((ks / 4) * Cfg::kQChunkBytes + (ks % 4) * 32) >> 4), kIdescQK, j > 0 ? 1u : 0u);
                        }
                    tc_commit(smem_addr(&sh.s_full[w][i]));
                    tc_commit(smem_addr(&sh.k_empty[s]));
                    if (++s == NS) { s = 0; k_parity ^= 1u; }
                }
                if (ok) tc_commit(smem_addr(&sh.q_empty[k & 1]));
            }
        }
    } else if (warp == 3) {
        // ============================================================ value products: the warp waits together, one thread issues
        setmaxnreg_dec<kPagedRegsOther>();
        constexpr uint32_t kIdescPV = kE4m3 ? (make_idesc_e4m3_f32(128, kCols, true, true) | (1u << 10))      // (both operands with the
                                            : make_idesc_bf16_f32(128, kCols, true, true);                  // keys as the slow dimension)
        constexpr int kStepKeys = 32 / Cfg::kElem, kStep16 = (kStepKeys * 128) >> 4;
        const uint32_t v_lo0 = desc_lo(sV, Cfg::kZeroBlock ? 0 : kChunkBytes), p_lo0 = desc_lo(sP, 128);
        int n = 0, s = 0;
        uint32_t v_parity = 0;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            ok = __all_sync(0xffffffffu, wait_part(k));
            if (!ok) break;
            const PagedEntry e = sh.part[k % kPartRing];
            if (e.t1 < 0) break;
            ok = __all_sync(0xffffffffu, paged_wait(sh.acc_empty[k % kOBufs], ((k / kOBufs) & 1) ^ 1, wait));
            if (!ok) break;
            for (int t = e.t0; t < e.t1; ++t, ++n) {
                const int w = n & 1, i = (n >> 1) % kPBufs;
                ok = paged_wait(sh.v_full[s], v_parity, wait);
                // the sequence's last tile: only the k-steps that hold keys are multiplied (one at least).  V rows behind the
                // sequence's end, as far as the last of them reaches, hold whatever the page held, or were not loaded: zeros, since
                // 0 * NaN is NaN.  (Here, where the stage is known to be this tile's: the softmax warps may be a turn of the ring ahead.)
                const int keys = t == e.t1 - 1 ? min(kTileN, e.len - t * kTileN) : kTileN;
                const int steps_end = keys <= 0 ? kStepKeys : (keys + kStepKeys - 1) / kStepKeys * kStepKeys;
                if (max(keys, 0) < steps_end) {
                    __syncwarp();
                    for (int j = lane; j < (steps_end - max(keys, 0)) * 8; j += 32) {
                        const uint32_t row = sV + s * Cfg::kVBytes + (max(keys, 0) + (j >> 3)) * 128 + (j & 7) * 16;
#pragma unroll
                        for (int c = 0; c < Cfg::kVChunks; ++c) st_shared_v4(row + c * kChunkBytes, 0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                }
                ok = __all_sync(0xffffffffu, ok && paged_wait(sh.p_full[w][i], ((n >> 1) / kPBufs) & 1, wait));
                if (!ok) break;
                tc_fence_after_sync();
                if (elect_one()) {
                    const uint32_t v_lo = v_lo0 + s * (Cfg::kVBytes >> 4), p_lo = p_lo0 + (w * kPBufs + i) * (Cfg::kPBytes >> 4);
                    const uint32_t d = tmem + o_col(k % kOBufs, w);
                    const uint32_t acc = t >= e.t0 + 2 ? 1u : 0u;        // the group's first tile of the part overwrites
#pragma unroll
                    for (int ks = 0; ks < Cfg::kPSteps; ++ks) {
                        if (ks * kStepKeys >= steps_end) break;
                        // (values of 64: the second 64 rows of V^T are read from a block of zeros, wherever this k-step is)
                        const uint32_t lo = v_lo + ks * kStep16;
                        const uint32_t lbo = Cfg::kZeroBlock ? (((sZero >> 4) - (lo & 0x3fffu)) << 16) : 0u;
                        paged_mma<kE4m3, true>(d, lo + lbo, p_lo + ks * kStepKeys, kIdescPV, ks > 0 ? 1u : acc);
                    }
                    tc_commit(smem_addr(&sh.v_empty[s]));
                    tc_commit(smem_addr(&sh.pv_done[w][i]));
                    if (t == e.t1 - 1) tc_commit(smem_addr(&sh.acc_full[k % kOBufs]));
                }
                __syncwarp();
                if (++s == NS) { s = 0; v_parity ^= 1u; }
            }
        }
    } else if (warp < 12) {
        // ============================================================ softmax groups
        // The four warps of a group stay together through their barriers: after a wait that ran out they go on to the end of
        // the part without waiting (results are invalid then, every access stays in bounds) and leave together.
        setmaxnreg_inc<paged_regs_softmax(kStates)>();
        const int w = (warp >> 2) - 1, key = tid & 127, wq = warp & 3;
        const uint32_t lane_sel = static_cast<uint32_t>(wq * 32) << 16;
        int mine_n = 0;                                                  // tiles this group has done
        bool ok = true;
        for (int k = 0;; ++k) {
            const int qb = k & 1;
            ok = ok && wait_part(k);
            const PagedEntry& entry = sh.part[k % kPartRing];
            const int t0 = entry.t0, t1 = entry.t1, len = entry.len, tile0 = entry.tile0;
            int n_drafts = 0;
            if constexpr (kTree) n_drafts = sh.n[k % kPartRing];
            if (named_barrier_or(1 + w, 128, !ok) || t1 < 0) break;
            // (also by a group without a tile here: its arrival at q_empty must not run ahead into the buffer's next turn)
            ok = paged_wait(sh.q_full[qb], (k >> 1) & 1, wait);
            const int skip = (tile0 & 1) == w ? 0 : 1;                   // this group's first tile of the part: t0 + skip
            if (t0 + skip < t1) {
                float l[kStates];
#pragma unroll
                for (int r = 0; r < kStates; ++r) l[r] = 0.f;
                const int first_masked = kTree ? len - n_drafts : len - p.Sq + 1;      // the first key that some row does not see
                const uint32_t tO = tmem + o_col(k % kOBufs, w) + lane_sel;
#pragma unroll 1
                for (int t = t0 + skip; t < t1; t += 2, ++mine_n) {
                    const int sb = mine_n % kBufs, pb = mine_n % kPBufs;
                    const bool first = t == t0 + skip;
                    const uint32_t tS = tmem + s_col(w, sb) + lane_sel;
                    const uint32_t sPw = sP + (w * kPBufs + pb) * Cfg::kPBytes + key * 16;
                    ok = ok && paged_wait(sh.s_full[w][sb], (mine_n / kBufs) & 1, wait);
                    __syncwarp();
                    tc_fence_after_sync();
                    const int key_at = t * kTileN + key;
                    float x[kStates];                                    // scores in log2 units
#pragma unroll
                    for (int g = 0; g < kStates / 16; ++g) {
                        // column of (map, term, row) in S^T: (map * kTerms + term) * kRows + row
                        const int map = g * 16 / kRows, r0 = g * 16 % kRows;
                        uint32_t s0[16];
                        tmem_ld_x16(tS + map * kTerms * kRows + r0, s0);
                        if constexpr (kE4m3) {
                            uint32_t s1[16], s2[16];
                            tmem_ld_x16(tS + (map * kTerms + 1) * kRows + r0, s1);
                            tmem_ld_x16(tS + (map * kTerms + 2) * kRows + r0, s2);
                            tc_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; j += 4) {
                                const float4 c = *reinterpret_cast<const float4*>(&sh.c[qb][r0 + j]);
                                const float cc[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                                for (int q = 0; q < 4; ++q)
                                    x[g * 16 + j + q] = (__uint_as_float(s0[j + q]) +
                                                         (__uint_as_float(s1[j + q]) + __uint_as_float(s2[j + q]))) * cc[q];
                            }
                        } else {
                            tc_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; j += 2) {
                                const float2 y = __fmul2_rn(make_float2(__uint_as_float(s0[j]), __uint_as_float(s0[j + 1])),
                                                            make_float2(p.scale_log2, p.scale_log2));
                                x[g * 16 + j] = y.x;
                                x[g * 16 + j + 1] = y.y;
                            }
                        }
                    }
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_addr(&sh.s_empty[w][sb]));
                    if (t * kTileN + kTileN > first_masked) {
                        if constexpr (kTree) {
                            // (no row has a bit for keys behind the drafts; a key before them is seen by all)
                            const int draft = key_at - first_masked;
                            const uint32_t bit = draft < 0 ? 0u : draft < 32 ? 1u << draft : 0u;
                            if (draft >= 0) {
#pragma unroll
                                for (int r = 0; r < kStates; r += 4) {
                                    const uint4 seen = *reinterpret_cast<const uint4*>(&sh.i[qb][r]);
                                    if (!(seen.x & bit)) x[r] = -INFINITY;
                                    if (!(seen.y & bit)) x[r + 1] = -INFINITY;
                                    if (!(seen.z & bit)) x[r + 2] = -INFINITY;
                                    if (!(seen.w & bit)) x[r + 3] = -INFINITY;
                                }
                            }
                        } else {
#pragma unroll
                            for (int r = 0; r < kStates; ++r)
                                if (key_at >= first_masked + sh.i[qb][r % kRows]) x[r] = -INFINITY;
                        }
                    }
                    bool move = first;
                    if (!first) {
                        float top = -INFINITY;
#pragma unroll
                        for (int r = 0; r < kStates; r += 4) {
                            const float4 nm = *reinterpret_cast<const float4*>(&sh.neg_m[w][r]);
                            top = fmax3(top, x[r] + nm.x, x[r + 1] + nm.y);
                            top = fmax3(top, x[r + 2] + nm.z, x[r + 3] + nm.w);
                        }
                        move = named_barrier_or(1 + w, 128, top > Cfg::kTauLog2 + Cfg::kBias);
                    }
                    if (move) {
                        // maxima over the keys: 16 rows at a time, halved at each exchange (as the row sums below)
#pragma unroll
                        for (int g = 0; g < kStates / 16; ++g) {
                            float a[16];
#pragma unroll
                            for (int j = 0; j < 16; ++j) a[j] = x[g * 16 + j];
#pragma unroll
                            for (int d = 16, m = 8; d >= 2; d >>= 1, m >>= 1) {
                                const bool up = (lane & d) != 0;
#pragma unroll
                                for (int j = 0; j < m; ++j) {
                                    const float give = up ? a[j] : a[j + m], keep = up ? a[j + m] : a[j];
                                    a[j] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, d));
                                }
                            }
                            a[0] = fmaxf(a[0], __shfl_xor_sync(0xffffffffu, a[0], 1));
                            if ((lane & 1) == 0) sh.red[w][wq][g * 16 + (lane >> 1)] = a[0];
                        }
                        named_barrier_sync(1 + w, 128);
                        if (key < kStates) {
                            const float old = first ? -INFINITY : Cfg::kBias - sh.neg_m[w][key];
                            const float here = fmaxf(fmaxf(sh.red[w][0][key], sh.red[w][1][key]), fmaxf(sh.red[w][2][key], sh.red[w][3][key]));
                            float mx = fmaxf(here, old), neg = Cfg::kBias - mx;
                            // A score between 2^27 and 2^28 has a step of 16, to which the bias of 11 is rounded, and 2^16 is no number of
                            // fp16's: one step higher the reference leaves that score a bias of 0 (and its own negative gives it back).
                            if constexpr (kE4m3) {
                                if (here + neg > 15.f) {
                                    mx = Cfg::kBias + here;
                                    neg = Cfg::kBias - mx;
                                }
                            }
                            sh.neg_m[w][key] = neg;
                            sh.neg_p[w][key] = mx == -INFINITY ? 0.f : neg;
                            sh.rescale[w][key] = mx == -INFINITY ? 1.f : exp2_approx(old - mx);
                        }
                        if (!first)       // the group's product before: nothing else adds to this accumulator
                            ok = ok && paged_wait(sh.pv_done[w][(mine_n - 1) % kPBufs], ((mine_n - 1) / kPBufs) & 1, wait);
                        named_barrier_sync(1 + w, 128);
                        if (!first) {
#pragma unroll
                            for (int r = 0; r < kStates; ++r) l[r] *= sh.rescale[w][r];
                            tc_fence_after_sync();
#pragma unroll 1
                            for (int g = 0; g < kCols / 16; ++g) {
                                const int col = g * 16, st = col / (kPTerms * kRows) * kRows + col % kRows;
                                uint32_t o[16];
                                tmem_ld_x16(tO + col, o);
                                tc_wait_ld();
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * sh.rescale[w][st + j]);
                                tmem_st_x16(tO + col, o);
                            }
                            tc_wait_st();
                        }
                    }
                    // The sum of score and reference is rounded apart from the score's own scaling: the score that the reference was
                    // taken from comes out as the bias, however large it is (from 2^23 on as far as the score's step allows).
#pragma unroll
                    for (int r = 0; r < kStates; r += 4) {
                        const float4 np = *reinterpret_cast<const float4*>(&sh.neg_p[w][r]);
                        x[r] = exp2_approx(x[r] + np.x);
                        x[r + 1] = exp2_approx(x[r + 1] + np.y);
                        x[r + 2] = exp2_approx(x[r + 2] + np.z);
                        x[r + 3] = exp2_approx(x[r + 3] + np.w);
                    }
#pragma unroll
                    for (int r = 0; r < kStates; ++r) l[r] += x[r];
                    // the buffer's last reader: the product of the group's tile kPBufs before
                    if (mine_n >= kPBufs) ok = ok && paged_wait(sh.pv_done[w][pb], ((mine_n / kPBufs) & 1) ^ 1, wait);
                    // P^T: 16 bytes of this key at a time (8 columns of bf16, 16 of e5m2)
                    if constexpr (kE4m3) {
#pragma unroll
                        for (int r = 0; r < kStates; r += 16) {
                            uint32_t h[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const __half2 two = __floats2half2_rn(x[r + 2 * j], x[r + 2 * j + 1]);
                                h[j] = *reinterpret_cast<const uint32_t*>(&two);
                            }
#pragma unroll
                            for (int term = 0; term < 3; ++term) {
                                const int col = (r / kRows * kPTerms + term) * kRows + r % kRows;
                                st_shared_v4(sPw + col / 16 * Cfg::kPGroupBytes, __byte_perm(h[0], h[1], 0x7531), __byte_perm(h[2], h[3], 0x7531),
                                             __byte_perm(h[4], h[5], 0x7531), __byte_perm(h[6], h[7], 0x7531));      // the top bytes
                                if (term < 2) {
#pragma unroll
                                    for (int j = 0; j < 8; ++j) {
                                        const uint32_t top = h[j] & 0xff00ff00u;
                                        const __half2 rest = __hsub2(*reinterpret_cast<const __half2*>(&h[j]), *reinterpret_cast<const __half2*>(&top));
                                        h[j] = *reinterpret_cast<const uint32_t*>(&rest);
                                    }
                                }
                            }
                        }
                    } else {
#pragma unroll
                        for (int r = 0; r < kStates; r += 8) {
#pragma unroll
                            for (int term = 0; term < kPTerms; ++term) {
                                uint32_t h[4];
#pragma unroll
                                for (int j = 0; j < 4; ++j) h[j] = pack_bf16x2(x[r + 2 * j], x[r + 2 * j + 1]);
                                const int col = (r / kRows * kPTerms + term) * kRows + r % kRows;
                                st_shared_v4(sPw + col / 8 * Cfg::kPGroupBytes, h[0], h[1], h[2], h[3]);
                                if (term + 1 < kPTerms) {
#pragma unroll
                                    for (int j = 0; j < 4; ++j) {
                                        x[r + 2 * j] -= __uint_as_float(h[j] << 16);
                                        x[r + 2 * j + 1] -= __uint_as_float(h[j] & 0xffff0000u);
                                    }
                                }
                            }
                        }
                    }
                    fence_proxy_async_smem();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_addr(&sh.p_full[w][pb]));
                }

                // ---- end of the part: row sums over the 128 threads, 16 rows at a time, halved at each exchange
#pragma unroll
                for (int g = 0; g < kStates / 16; ++g) {
                    float a[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) a[j] = l[g * 16 + j];
#pragma unroll
                    for (int d = 16, m = 8; d >= 2; d >>= 1, m >>= 1) {
                        const bool up = (lane & d) != 0;
#pragma unroll
                        for (int j = 0; j < m; ++j) {
                            const float give = up ? a[j] : a[j + m], keep = up ? a[j + m] : a[j];
                            a[j] = keep + __shfl_xor_sync(0xffffffffu, give, d);
                        }
                    }
                    a[0] += __shfl_xor_sync(0xffffffffu, a[0], 1);
                    // lane bits 4, 3, 2, 1 chose the halves: row = bit4*8 + bit3*4 + bit2*2 + bit1
                    if ((lane & 1) == 0) sh.red_l[w][wq][g * 16 + (lane >> 1)] = a[0];
                }
                named_barrier_sync(1 + w, 128);
                if (key < kStates) {
                    sh.stat_l[k % kPartRing][w][key] = (sh.red_l[w][0][key] + sh.red_l[w][1][key]) + (sh.red_l[w][2][key] + sh.red_l[w][3][key]);
                    sh.stat_m[k % kPartRing][w][key] = Cfg::kBias - sh.neg_m[w][key];
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.stat_full[k % kPartRing]));
            if (key == 0) mbar_arrive(smem_addr(&sh.q_empty[qb]));       // (every thread of the group is past its last use: the barrier above)
        }
    } else {
        // ============================================================ list of parts, query rows, results (thread = output column)
        if constexpr (kStates <= 32) setmaxnreg_inc<160>();
        const int key = tid & 127, wq = warp & 3;
        const uint32_t lane_sel = static_cast<uint32_t>(wq * 32) << 16;
        constexpr uint32_t kBar = 3;
        bool ok = true;
        // the shares: every thread sums up the tiles of consecutive sequences, a scan over the group finds the total, which decides how
        // units are counted, and the sequence that the CTA's share begins in
        const int chunk = (p.B + 127) / 128;
        const int b_first = key * chunk, b_last = min(p.B, b_first + chunk);
        int mine = 0, longest = 0;
#pragma unroll 4
        for (int b = b_first; b < b_last; ++b) {
            DraftRows d;
            const int n = seq_len(b, nullptr, d);
            mine += paged_units(p, n, PagedCount{0, 0, 0});
            longest = max(longest, n);
        }
        longest = __reduce_max_sync(0xffffffffu, longest);
        if (lane == 0) sh.warp_longest[wq] = longest;
        int before = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, before, d);
            if (lane >= d) before += o;
        }
        if (lane == 31) sh.warp_sums[wq] = before;
        before -= mine;
        named_barrier_sync(kBar, 128);
        int total = 0;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int n = sh.warp_sums[v];
            if (v < wq) before += n;
            total += n;
        }
        longest = max(max(sh.warp_longest[0], sh.warp_longest[1]), max(sh.warp_longest[2], sh.warp_longest[3]));
        const int least = paged_least(p, kTree, paged_tiles(longest));
        const PagedCount cnt = paged_count(p, least, gridDim.x, paged_tiles(longest), total);
        const int b_mine = max(0, b_last - b_first), b_before = min(b_first, p.B);
        if (cnt.pad > 0) {           // all sequences count the same
            const int units = paged_units(p, longest, cnt);
            total = units * p.B;
            mine = b_mine * units;
            before = b_before * units;
        } else if (cnt.cost > 0) {
            const int more = cnt.cost * p.Hkv * p.row_blocks;
            total += more * p.B;
            mine += more * b_mine;
            before += more * b_before;
        }
        const int share = paged_share(least, total, gridDim.x, cnt);
        const int u0 = min(total, static_cast<int>(blockIdx.x) * share), u1 = min(total, u0 + share);
        if (before <= u0 && u0 < before + mine) {
            int b = b_first, base = before;
            for (;; ++b) {
                DraftRows d;
                const int n = paged_units(p, seq_len(b, nullptr, d), cnt);
                if (u0 < base + n) break;
                base += n;
            }
            sh.start_b = b;
            sh.start_base = base;
        }
        named_barrier_sync(kBar, 128);
        // The list, published by the group's last warp, a lane per row block of the sequence: every entry that is free when the
        // results of part k begin (those of the parts before have been stored).  A CTA without a share has the end mark alone.
        const int blocks = p.Hkv * p.row_blocks;
        int seq = 0, base = 0, len = 0, hr = 0, published = 0, tiles = 0;
        DraftRows drafts{0, 0};       // of the sequence
        bool ended = u0 >= total, marked = false;
        if (wq == 3 && !ended) {
            seq = sh.start_b;
            base = sh.start_base;
            len = seq_len(seq, lane == 0 ? p.status : nullptr, drafts);
            hr = (u0 - base) / paged_block_units(len, cnt);
        }
        auto publish = [&](int k) {
            while (!ended && published < k + kPartRing) {
                const int nt = paged_tiles(len);
                PagedEntry e;
                const bool some = hr + lane < blocks && paged_entry(p, blockIdx.x, share, u0, u1, seq, base, len, cnt, hr + lane, e);
                const uint32_t have = __ballot_sync(0xffffffffu, some);
                const int count = min(__popc(have), k + kPartRing - published);
                // tiles of the parts before this lane's: the first part of a share may lack some, the others here have them all
                const int first_tiles = __shfl_sync(0xffffffffu, e.t1 - e.t0, 0);
                if (lane < count) {
                    e.tile0 = tiles + (lane > 0 ? first_tiles + (lane - 1) * nt : 0);
                    const int at = (published + lane) % kPartRing;
                    sh.part[at] = e;
                    if constexpr (kTree) {
                        sh.n[at] = drafts.count;
                        sh.row0[at] = drafts.first;
                    }
                    mbar_arrive(smem_addr(&sh.part_full[at]));
                }
                const int last_tiles = __shfl_sync(0xffffffffu, e.t1 - e.t0, max(0, count - 1));
                if (count > 0) tiles += last_tiles + (count > 1 ? first_tiles + (count - 2) * nt : 0);
                published += count;
                hr += count;
                if (count == __popc(have)) {
                    if (hr < blocks) {
                        ended = true;                  // the share ends inside this sequence
                    } else {
                        base += blocks * paged_block_units(len, cnt);
                        hr = 0;
                        if (base < u1) {
                            ++seq;
                            len = seq_len(seq, lane == 0 ? p.status : nullptr, drafts);
                        } else {
                            ended = true;
                        }
                    }
                }
            }
            if (ended && !marked && published < k + kPartRing) {
                if (lane == 0) {
                    sh.part[published % kPartRing].t1 = -1;
                    mbar_arrive(smem_addr(&sh.part_full[published % kPartRing]));
                }
                marked = true;
                ++published;
            }
        };
        // the query rows of a part into buffer k & 1 (before k = 2: free; later: the part two before has ended)
        constexpr int kVecs = DQK / 8;                        // 16-byte pieces of a row
        constexpr int kLanes = kVecs == 24 ? 32 : kVecs;      // lanes of a row
        constexpr int kPass = 128 / kLanes;                   // rows of a pass over the group
        constexpr int kPasses = (kRows + kPass - 1) / kPass;
        const int row_in = key / kLanes, piece = key % kLanes;
        uint4 xs[kPasses];
        uint32_t seen[kTree ? kPasses : 1];      // what the rows see of the drafts
        float q_scale = 1.f;
        int q_rb = 0, o_rb = 0;       // the blocks whose rows sh.row_q and sh.row_o are
        auto load_queries = [&](int k) {
            const PagedEntry& e = sh.part[k % kPartRing];
            if (e.rb != q_rb) {       // (uniform)
                q_rb = e.rb;
                named_barrier_sync(kBar, 128);         // (the rows before have been stored)
                if (key < kRows) rows_of_q(q_rb, key);
                named_barrier_sync(kBar, 128);
            }
            int n = 0, row0 = 0;
            if constexpr (kTree) {
                n = sh.n[k % kPartRing];
                row0 = sh.row0[k % kPartRing];
            }
            const __nv_bfloat16* const q = p.Q + (kTree ? row0 * p.q_st : e.b * p.q_sb) + static_cast<long long>(e.kvh * group) * p.q_sh + piece * 8;
#pragma unroll
            for (int j = 0; j < kPasses; ++j) {
                const int r = j * kPass + row_in;
                xs[j] = make_uint4(0, 0, 0, 0);
                if constexpr (kTree) seen[j] = 0u;
                if (r < kRows && piece < kVecs) {
                    const long long at = sh.row_q[r];
                    if constexpr (kTree) {
                        const int i = sh.row_place[r];
                        if (at >= 0 && i < n) {
                            xs[j] = *reinterpret_cast<const uint4*>(q + at);
                            if (piece == 0) seen[j] = draft_word(TreeParams{nullptr, 0, 0, p.mask, p.mask_stride}, row0 + i, i, n, 0);
                        }
                    } else if (at >= 0) {
                        xs[j] = *reinterpret_cast<const uint4*>(q + at);
                    }
                }
            }
            q_scale = p.scale_log2 * (kE4m3 && p.k_scale ? p.k_scale[e.kvh] : 1.f);
        };
        auto store_queries = [&](int k) {
            const int qb = k & 1;
            const uint32_t sQb = sQ + qb * Cfg::kQBytes;
            ok = ok && paged_wait_timed(&sh.q_empty[qb], ((k >> 1) & 1) ^ 1, wait, kSiteLoadQEmpty);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kPasses; ++j) {
                const int r = j * kPass + row_in;
                float c = q_scale;
                if constexpr (!kE4m3) {
                    if (r < kRows && piece < kVecs)
                        st_shared_v4(sQb + (piece >> 3) * Cfg::kQChunkBytes + r * 128 + (((piece & 7) ^ (r & 7)) << 4), xs[j].x, xs[j].y, xs[j].z, xs[j].w);
                } else {
                    // scaled by a power of two so that the row's largest entry is in [2^14, 2^15), then three e5m2 terms: exact for
                    // entries of 2^-23 of the largest and more, below that to 2^-30 of it
                    const uint32_t w4[4] = {xs[j].x, xs[j].y, xs[j].z, xs[j].w};
                    uint32_t top = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = max(top, max((w4[i] & 0x7fffu) << 16, w4[i] & 0x7fff0000u));
#pragma unroll
                    for (int d = kLanes / 2; d > 0; d >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
                    // (from 2^127 down to 2^-112; a smaller row is scaled by 2^126, which makes its entries, multiples of 2^-133, exact too)
                    int sft = top ? 14 - (static_cast<int>(top >> 23) - 127) : 0;
                    sft = sft > 126 ? 126 : (sft < -113 ? -113 : sft);
                    const float mult = __uint_as_float(static_cast<uint32_t>(sft + 127) << 23);
                    c *= __uint_as_float(static_cast<uint32_t>(127 - sft) << 23);
                    uint32_t t8[3][2];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        __half2 h = __floats2half2_rn(__uint_as_float(w4[i] << 16) * mult, __uint_as_float(w4[i] & 0xffff0000u) * mult);
#pragma unroll
                        for (int t = 0; t < 3; ++t) {
                            uint32_t bits = *reinterpret_cast<uint32_t*>(&h) & 0xff00ff00u;
                            const uint32_t two = __byte_perm(bits, 0, 0x4431);       // the two top bytes
                            if (i & 1) t8[t][i >> 1] |= two << 16; else t8[t][i >> 1] = two;
                            h = __hsub2(h, *reinterpret_cast<__half2*>(&bits));
                        }
                    }
                    if (r < kRows && piece < kVecs) {
#pragma unroll
                        for (int t = 0; t < 3; ++t) {
                            const int rq = t * kRows + r, q16 = piece >> 1;
                            st_shared_u64(sQb + (q16 >> 3) * Cfg::kQChunkBytes + rq * 128 + (((q16 & 7) ^ (rq & 7)) << 4) + (piece & 1) * 8,
                                          t8[t][0], t8[t][1]);
                        }
                    }
                }
                if (r < kRows && piece == 0) {
                    if constexpr (kE4m3) sh.c[qb][r] = c;
                    sh.i[qb][r] = kTree ? static_cast<int>(seen[kTree ? j : 0]) : sh.row_place[r];
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.q_full[qb]));
        };
        // Round k stages the query rows of part k + 2 as soon as part k has ended, loads those of part k + 3, and brings out part k's
        // results; rounds -3 to -1 begin this.
        int end_at = 0x7fffffff;                   // the end mark's place, once seen
        for (int k = -3; k < end_at; ++k) {
            if (wq == 3 && !marked && published < max(k, 0) + kPartRing - 3) publish(max(k, 0));
            if (k + 3 < end_at) ok = ok && wait_part(k + 3);       // (which waits for nobody)
            // whether all other pieces of an unfinished row block are there already: then this one need not be announced
            if (k >= 0 && key == 0 && sh.part[k % kPartRing].slot >= 0) {
                const PagedEntry& mine_part = sh.part[k % kPartRing];
                const unsigned int got = *static_cast<volatile unsigned int*>(p.arrivals + mine_part.first_cta);
                const bool last = got == static_cast<unsigned int>(mine_part.pieces - 1);
                sh.is_last[k & 1] = last ? 1u : 0u;
                if (last) {
                    __threadfence();
                    p.arrivals[mine_part.first_cta] = 0u;
                }
            }
            if (k >= 0) ok = ok && paged_wait_timed(&sh.stat_full[k % kPartRing], (k / kPartRing) & 1, wait, kSiteEpiState);
            if (named_barrier_or(kBar, 128, !ok)) break;
            if (k > -3 && k + 2 < end_at) store_queries(k + 2);
            if (k + 3 < end_at && sh.part[(k + 3) % kPartRing].t1 < 0) end_at = k + 3;
            if (k + 3 < end_at) load_queries(k + 3);
            if (k < 0) continue;
            const PagedEntry e = sh.part[k % kPartRing];
            const int ob = k % kOBufs;
            const bool whole = e.slot < 0;
            if (e.rb != o_rb) {           // (uniform; the barrier that the round began with: nobody reads the old ones any more)
                o_rb = e.rb;
                if (key < kRows) rows_of_o(o_rb, key);
                named_barrier_sync(kBar, 128);
            }
            const int hq0 = e.kvh * group;
            int live_rows = kRows, row0 = 0;
            if constexpr (kTree) {
                live_rows = sh.n[k % kPartRing] * group;
                row0 = sh.row0[k % kPartRing];
            }
            auto row_out = [&](int r) -> long long { return !kTree || r < live_rows ? sh.row_o[r] : -1; };
            __nv_bfloat16* const out = p.O + (kTree ? row0 * p.o_st : e.b * p.o_sb) + hq0 * p.o_sh;
            const float vs = kE4m3 && p.v_scale ? p.v_scale[e.kvh] : 1.f;
            float* const slot_o = p.part + static_cast<long long>(whole ? 0 : e.slot) * kStates * (DV + 2);
            float* const slot_ml = slot_o + kStates * DV;
            // A row block of two pieces: the CTA that joins them takes its own from registers, and where the other's is known to be there
            // its loads run under the last products.  (Other blocks are joined from memory, further below.)
            const bool two = !whole && e.pieces == 2, own_first = static_cast<int>(blockIdx.x) == e.first_cta;
            const bool known = two && sh.is_last[k & 1] != 0u;
            const float* const other_o = p.part + (own_first ? 2ll * (e.first_cta + 1) : e.first_slot) * kStates * (DV + 2);
            float other[kStates <= 16 ? kStates : 1], other_m = -INFINITY, other_l = 0.f, own_m = -INFINITY, own_l = 0.f;
            auto load_other = [&]() {
                if (key < kStates) {
                    other_m = __ldcg(other_o + kStates * DV + key);
                    other_l = __ldcg(other_o + kStates * DV + kStates + key);
                }
                if constexpr (kStates <= 16) {
#pragma unroll
                    for (int r = 0; r < kStates; ++r) other[r] = key < DV ? __ldcg(other_o + r * DV + key) : 0.f;
                }
            };
            if (known) load_other();
            // log-sum-exp of a row (natural units) from its maximum (log2 units) and sum
            auto store_lse = [&](int r, float m, float sum) {
                if (kDiff || !p.lse || row_out(r) < 0) return;
                const long long tokens = kTree ? p.total : static_cast<long long>(p.B) * p.Sq, first = kTree ? row0 : static_cast<long long>(e.b) * p.Sq;
                p.lse[(hq0 + sh.row_h[r]) * tokens + first + sh.row_i[r]] =
                    sum > 0.f || sum != sum ? (m - Cfg::kBias + log2f(sum)) * 0.6931471805599453f : -INFINITY;
            };
            // (uniform) whether a group had a tile of this part
            const bool had[2] = {e.t1 - e.t0 > 1 || (e.tile0 & 1) == 0, e.t1 - e.t0 > 1 || (e.tile0 & 1) == 1};
            // (the first two warps the factors, the other two the log-sum-exps: each takes some 300 cycles)
            const int st = key & 63;
            if (st < kStates) {
                float f[2], sum[2], mx[2];
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    mx[v] = had[v] ? sh.stat_m[k % kPartRing][v][st] : -INFINITY;
                    sum[v] = had[v] ? sh.stat_l[k % kPartRing][v][st] : 0.f;
                }
                const float m = fmaxf(mx[0], mx[1]);
#pragma unroll
                for (int v = 0; v < 2; ++v) f[v] = mx[v] == -INFINITY ? 0.f : exp2_approx(mx[v] - m);
                const float all = f[0] * sum[0] + f[1] * sum[1];
                if (key >= 64) {
                    if (whole) store_lse(st % kRows, m, all);
                } else {
                    const float norm = !whole ? 1.f : (all > 0.f || all != all ? 1.f / all : 0.f);
                    sh.factor[0][st] = f[0] * norm;
                    sh.factor[1][st] = f[1] * norm;
                    if (!whole) {
                        own_m = m;
                        own_l = all;
                        if (!known) {
                            slot_ml[st] = m;
                            slot_ml[kStates + st] = all;
                        }
                    }
                }
            }
            ok = ok && paged_wait_timed(&sh.acc_full[ob], (k / kOBufs) & 1, wait, kSiteEpiOFull);
            named_barrier_sync(kBar, 128);
            tc_fence_after_sync();
            float y[kStates];
#pragma unroll
            for (int r = 0; r < kStates; ++r) y[r] = 0.f;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                if (!had[v]) continue;
                // (48 columns in flight)
                constexpr int kGroup = kCols <= 48 ? kCols / 16 : 2;
#pragma unroll
                for (int g0 = 0; g0 < kCols / 16; g0 += kGroup) {
                    uint32_t o[kGroup][16];
#pragma unroll
                    for (int g = 0; g < kGroup; ++g) tmem_ld_x16(tmem + o_col(ob, v) + lane_sel + (g0 + g) * 16, o[g]);
                    tc_wait_ld();
#pragma unroll
                    for (int g = 0; g < kGroup; ++g) {
                        const int col = (g0 + g) * 16, st = col / (kPTerms * kRows) * kRows + col % kRows;
#pragma unroll
                        for (int j = 0; j < 16; ++j) y[st + j] = fmaf(sh.factor[v][st + j], __uint_as_float(o[g][j]), y[st + j]);
                    }
                }
            }
            tc_fence_before_sync();
            named_barrier_sync(kBar, 128);
            if (key == 0) mbar_arrive(smem_addr(&sh.acc_empty[ob]));
            // the rows' results (map 0, then map 1) to O: the result itself, or the difference and its norm
            auto store_rows = [&]() {
                if constexpr (kDiff) {
#pragma unroll
                    for (int r = 0; r < kRows; ++r) y[r] = vs * (y[r] - p.lambda[hq0 + sh.row_h[r]] * y[kRows + r]);
                    if (p.weight) {
#pragma unroll
                        for (int r = 0; r < kRows; ++r) {
                            float q = y[r] * y[r];
#pragma unroll
                            for (int d = 16; d > 0; d >>= 1) q += __shfl_xor_sync(0xffffffffu, q, d);
                            if (lane == 0) sh.sq[wq][r] = q;
                        }
                        named_barrier_sync(kBar, 128);
                        const float wt = p.weight[key];
#pragma unroll
                        for (int r = 0; r < kRows; ++r) {
                            const float q = (sh.sq[0][r] + sh.sq[1][r]) + (sh.sq[2][r] + sh.sq[3][r]);
                            y[r] *= wt * rsqrtf(q * (1.f / DV) + p.eps);
                        }
                    }
#pragma unroll
                    for (int r = 0; r < kRows; ++r) y[r] *= p.out_scale;
                } else {
#pragma unroll
                    for (int r = 0; r < kRows; ++r) y[r] *= vs;
                }
                if (key < DV) {
#pragma unroll
                    for (int r = 0; r < kRows; ++r) {
                        if (kTree && r >= live_rows) break;
                        const long long at = row_out(r);
                        if (at >= 0) out[at + key] = __float2bfloat16(y[r]);
                    }
                }
            };
            if (whole) {
                store_rows();
                continue;
            }
            if (!known) {
                if (key < DV) {
#pragma unroll
                    for (int r = 0; r < kStates; ++r) slot_o[r * DV + key] = y[r];
                }
                named_barrier_sync(kBar, 128);
                if (key == 0 && !sh.is_last[k & 1]) {
                    // (the fence covers the stores of all threads of the group: the barrier orders them before it)
                    __threadfence();
                    const bool last = atomicAdd(p.arrivals + e.first_cta, 1u) == static_cast<unsigned int>(e.pieces - 1);
                    sh.is_last[k & 1] = last ? 1u : 0u;
                    if (last) p.arrivals[e.first_cta] = 0u;
                    __threadfence();
                }
                named_barrier_sync(kBar, 128);
            }
            if (!sh.is_last[k & 1]) continue;
            if (two) {
                // the two pieces' sum, in the order of the CTAs whichever of them has it
                if (!known) load_other();
                if (key < kStates) {
                    const float m = fmaxf(own_m, other_m);
                    const float f_own = own_m == -INFINITY ? 0.f : exp2_approx(own_m - m), f_other = other_m == -INFINITY ? 0.f : exp2_approx(other_m - m);
                    const float l0 = own_first ? f_own * own_l : f_other * other_l;
                    const float sum = own_first ? fmaf(f_other, other_l, l0) : fmaf(f_own, own_l, l0);
                    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                    sh.factor[0][key] = f_own * inv;
                    sh.factor[1][key] = f_other * inv;
                    store_lse(key % kRows, m, sum);
                }
                named_barrier_sync(kBar, 128);
#pragma unroll
                for (int r = 0; r < kStates; ++r) {
                    const float x = kStates <= 16 ? other[kStates <= 16 ? r : 0] : key < DV ? __ldcg(other_o + r * DV + key) : 0.f;
                    const float f_own = sh.factor[0][r], f_other = sh.factor[1][r];
                    y[r] = own_first ? fmaf(f_other, x, f_own * y[r]) : fmaf(f_own, y[r], f_other * x);
                }
                store_rows();
            } else {
                // This CTA finished last: all pieces, in the order of the CTAs, kMergePieces at a time under a running maximum.  A
                // thread has four columns of every kGroups-th state (both maps of a row are its own); the first loads go out
                // before the weights that they wait for.  (The pieces behind the first are the first parts of their CTAs.)
                constexpr int kMergePieces = Shared::kMergePieces;
                constexpr int kGroups = 128 / (DV / 4), kMine = kStates / kGroups, kBatch = kMine <= 4 ? 2 : 1;
                static_assert(kRows % kGroups == 0, "both maps of a row in one thread");
                const int col = key % (DV / 4) * 4, g0 = key / (DV / 4);
                auto piece = [&](int c) {
                    return p.part + (c == 0 ? e.first_slot : 2ll * (e.first_cta + c)) * kStates * (DV + 2);
                };
                float4 z[kMine], v[kBatch][kMine];
#pragma unroll
                for (int j = 0; j < kMine; ++j) z[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                auto load_batch = [&](int c) {
#pragma unroll
                    for (int q = 0; q < kBatch; ++q) {
                        if (c + q >= e.pieces) break;
                        const float* po = piece(c + q) + g0 * DV + col;
#pragma unroll
                        for (int j = 0; j < kMine; ++j) v[q][j] = __ldcg(reinterpret_cast<const float4*>(po + j * kGroups * DV));
                    }
                };
                float run_m = -INFINITY, run_l = 0.f;
#pragma unroll 1
                for (int c0 = 0; c0 < e.pieces; c0 += kMergePieces) {
                    const int nc = min(kMergePieces, e.pieces - c0);
                    load_batch(c0);
                    for (int j = key; j < nc * kStates; j += 128) {
                        const float* ml = piece(c0 + j / kStates) + kStates * DV + j % kStates;
                        sh.piece_m[j / kStates][j % kStates] = __ldcg(ml);
                        sh.piece_l[j / kStates][j % kStates] = __ldcg(ml + kStates);
                    }
                    named_barrier_sync(kBar, 128);
                    if (key < kStates) {
                        float m = run_m;
                        for (int c = 0; c < nc; ++c) m = fmaxf(m, sh.piece_m[c][key]);
                        const float keep = run_m == -INFINITY ? 0.f : exp2_approx(run_m - m);
                        float sum = run_l * keep;
                        for (int c = 0; c < nc; ++c) {
                            const float mc = sh.piece_m[c][key];
                            const float f = mc == -INFINITY ? 0.f : exp2_approx(mc - m);
                            // (a piece without a finite score counts nothing, but a NaN of its sum goes through)
                            sum += f * sh.piece_l[c][key];
                            sh.piece_m[c][key] = f;
                        }
                        sh.factor[0][key] = keep;
                        run_m = m;
                        run_l = sum;
                        // (read after the last round)
                        sh.factor[1][key] = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                    }
                    named_barrier_sync(kBar, 128);
#pragma unroll
                    for (int j = 0; j < kMine; ++j) {
                        const float keep = sh.factor[0][g0 + j * kGroups];
                        z[j].x *= keep; z[j].y *= keep; z[j].z *= keep; z[j].w *= keep;
                    }
#pragma unroll 1
                    for (int c = 0; c < nc; c += kBatch) {
                        if (c > 0) load_batch(c0 + c);
#pragma unroll
                        for (int q = 0; q < kBatch; ++q) {
                            if (c + q >= nc) break;
#pragma unroll
                            for (int j = 0; j < kMine; ++j) {
                                const float f = sh.piece_m[c + q][g0 + j * kGroups];
                                z[j].x = fmaf(f, v[q][j].x, z[j].x);
                                z[j].y = fmaf(f, v[q][j].y, z[j].y);
                                z[j].z = fmaf(f, v[q][j].z, z[j].z);
                                z[j].w = fmaf(f, v[q][j].w, z[j].w);
                            }
                        }
                    }
                    if (c0 + kMergePieces < e.pieces) named_barrier_sync(kBar, 128);
                }
#pragma unroll
                for (int j = 0; j < kRows / kGroups; ++j) {
                    const int r = g0 + j * kGroups;
                    const float f0 = vs * sh.factor[1][r];
                    float4 o = make_float4(f0 * z[j].x, f0 * z[j].y, f0 * z[j].z, f0 * z[j].w);
                    if constexpr (kDiff) {
                        const float4 o1 = z[j + kRows / kGroups];
                        const float f1 = vs * sh.factor[1][kRows + r] * p.lambda[hq0 + sh.row_h[r]];
                        o.x -= f1 * o1.x; o.y -= f1 * o1.y; o.z -= f1 * o1.z; o.w -= f1 * o1.w;
                        float f = p.out_scale;
                        float4 w = make_float4(1.f, 1.f, 1.f, 1.f);
                        if (p.weight) {
                            float q = o.x * o.x + o.y * o.y + o.z * o.z + o.w * o.w;        // (a row is a warp's)
#pragma unroll
                            for (int d = 16; d > 0; d >>= 1) q += __shfl_xor_sync(0xffffffffu, q, d);
                            f *= rsqrtf(q * (1.f / DV) + p.eps);
                            w = __ldg(reinterpret_cast<const float4*>(p.weight + col));
                        }
                        o.x *= f * w.x; o.y *= f * w.y; o.z *= f * w.z; o.w *= f * w.w;
                    }
                    const long long at = row_out(r);
                    if (at >= 0)
                        *reinterpret_cast<uint2*>(out + at + col) = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
                }
                if (key < kStates) store_lse(key % kRows, run_m, run_l);
            }
            // (the barrier at the head of the loop comes before anything that is read here is overwritten)
        }
    }

    // ---------------------------------------------------------------- teardown (all warps)
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, Cfg::kTmemCols);
}

}  // namespace fa
