// Attention of the last few tokens of every sequence over a paged key/value cache, for sm_100a.
//
// Per (sequence, K/V head) there are R = (Hq / Hkv) * Sq query rows, one to a few dozen, against thousands of keys: every byte
// of K and V is read once and used for R rows, 2 R (dqk + dv) / ((dqk + dv) * bytes) = R .. 2R flops a byte, far below the 250 that
// the tensor cores need to be the bound.  The kernel is built to stream HBM:
//
//   * The products are turned around, keys on the 128 lanes of the accumulator and query rows on its columns:
//         S^T [128 keys x rows]  = K_tile [128 x dqk] Q^T          (tcgen05.mma, M = 128, N = rows)
//         O^T [dv x rows]       += V_tile^T [dv x 128] P^T          (V read MN-major, P^T written by the softmax warps)
//     so an MMA of 16 rows costs 16 columns and not a padded tile of 128, and a thread exponentiates rows, not 128 keys, per tile.
//   * The tiles of all sequences and heads form one list; CTA c takes the c-th of equal consecutive shares (the lengths are read on
//     the device).  Lengths that differ by orders of magnitude cost nothing, and no SM waits for a wave.  A (sequence, head)
//     that several CTAs share is joined by the one that finishes last, in the order of the CTAs (equal calls give equal bits).
//   * A ring of K/V tiles (two to five stages, all that the shared memory holds) runs across the boundaries of sequences.
//
// Two groups of four softmax warps take the tiles in turn; each has its own scores, probabilities, reference maximum, row
// sums and accumulator (merged when a piece of the list ends), so that one group's exponentials run under the other's MMAs
// and no tile waits for the one before it.  A thread owns a key of the tile: the row maximum runs across lanes, so it is
// taken rarely: the reference of a row moves only when some score exceeds it by more than kTauLog2 (one barrier with a
// vote per tile; the reductions, and the rescaling of O^T, on the few tiles where the vote says so).
//
// e4m3 caches: K and V enter the 8-bit MMA as they are; the bf16 queries and the fp32 probabilities as sums of three e5m2 terms,
// each on columns of its own (N = 3 rows): x -> fp16, top byte, remainder, top byte, remainder, top byte, 9 significant bits.
// Nothing is dequantised and both sides keep at least bf16's precision.  The probabilities are scaled by 2^13 so that weights of
// 2^-20 of the largest still have 9 bits.
//
// Differential attention: two maps are two groups of columns.  Map a's scores are the k-steps of its half of K, its
// probabilities meet the same V tile, and the epilogue subtracts and normalises: K and V are read once for both.
//
// Roles (384 threads): warp 0 TMA loads (a lane per page box), warp 1 MMA issue, warps 2-3 query rows into shared memory,
// warps 4-7 and 8-11 softmax groups 0 and 1 (thread = key of the tile = lane of S^T, and output column = lane of O^T).
#pragma once

#include <math.h>

#include "fa_paged_common.cuh"

namespace fa {

namespace ptx {

// OR of a predicate over the `nthreads` threads that meet at a named barrier.
FA_DEVI bool named_barrier_or(uint32_t id, uint32_t nthreads, bool x) {
    uint32_t r;
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.u32 p, %1, 0;\n"
        "barrier.cta.red.or.pred q, %2, %3, p;\n"
        "selp.u32 %0, 1, 0, q;\n"
        "}\n"
        : "=r"(r) : "r"(x ? 1u : 0u), "r"(id), "r"(nthreads) : "memory");
    return r != 0;
}
FA_DEVI float warp_max(float x) {
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
FA_DEVI void st_shared_u16(uint32_t addr, uint32_t x) {
    asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"(static_cast<uint16_t>(x)) : "memory");
}
FA_DEVI void st_shared_u8(uint32_t addr, uint32_t x) {
    asm volatile("st.shared.u8 [%0], %1;" ::"r"(addr), "r"(x) : "memory");
}
FA_DEVI void st_shared_u64(uint32_t addr, uint32_t lo, uint32_t hi) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(lo), "r"(hi) : "memory");
}

}  // namespace ptx

// ------------------------------------------------------------------ the list of work units and its shares

// A unit is one tile of 128 keys of one (sequence, K/V head, block of rows); a sequence without keys has one empty tile per
// head, so that its rows are written.  Units are ordered by sequence, head, row block, tile.
__host__ __device__ inline int paged_tiles(int len) { return len > 0 ? (len + kTileN - 1) / kTileN : 1; }
__host__ __device__ inline long long paged_units(const PagedParams& p, int b) {
    return static_cast<long long>(paged_tiles(clamped_len(p.seq_lens[b], p.max_pages, p.page_size, nullptr))) * p.Hkv * p.row_blocks;
}
__host__ __device__ inline long long paged_share(long long units, int ctas, int least) {
    const long long per = (units + ctas - 1) / ctas;
    return per < least ? least : per;
}
// First CTA of the (sequence, head, row block) whose units are [ua, ub), the number of CTAs that have a part of it, and the
// partial-result slot of CTA c's part (a CTA leaves at most two parts unfinished: its first and its last).
__host__ __device__ inline int paged_first_cta(long long ua, long long share) { return static_cast<int>(ua / share); }
__host__ __device__ inline int paged_pieces(long long ua, long long ub, long long share) {
    return static_cast<int>((ub - 1) / share - ua / share) + 1;
}
__host__ __device__ inline int paged_slot(int cta, long long ua, long long share) { return 2 * cta + (ua > cta * share ? 1 : 0); }

// Position in the unit list: the part [t0, t1) of the tiles of (b, hr), hr = K/V head * row_blocks + row block.
struct PagedPart {
    long long u, u1;              // next unit, end of the CTA's share
    long long base;               // first unit of sequence b
    int b, len, nt;
    int hr, t0, t1;
    bool report;
    __host__ __device__ void load_len(const PagedParams& p) {
        len = clamped_len(p.seq_lens[b], p.max_pages, p.page_size, report ? p.status : nullptr);
        nt = paged_tiles(len);
    }
    __host__ __device__ void begin(const PagedParams& p, int b0, long long base0, long long first, long long end, bool rep) {
        u = first; u1 = end; b = b0; base = base0; report = rep;
        load_len(p);
        set();
    }
    __host__ __device__ void set() {
        const long long local = u - base;
        hr = static_cast<int>(local / nt);
        t0 = static_cast<int>(local - static_cast<long long>(hr) * nt);
        t1 = (u1 - u < nt - t0) ? t0 + static_cast<int>(u1 - u) : nt;
    }
    __host__ __device__ bool next(const PagedParams& p) {
        u += t1 - t0;
        if (u >= u1) return false;
        if (t1 == nt && hr + 1 == p.Hkv * p.row_blocks) {
            base = u;
            ++b;
            load_len(p);
        }
        set();
        return true;
    }
    __host__ __device__ long long first_unit() const { return base + static_cast<long long>(hr) * nt; }     // of (b, hr)
};

// ------------------------------------------------------------------ configuration

template <int DQK, int DV, bool kE4m3, bool kDiff, int kRows>
struct PagedCfg {
    static constexpr int kMaps = kDiff ? 2 : 1;
    static constexpr int kTerms = kE4m3 ? 3 : 1;
    static constexpr int kStates = kMaps * kRows;               // softmax states of a group
    static constexpr int kCols = kStates * kTerms;              // columns of S^T and of O^T
    static constexpr int kElem = kE4m3 ? 1 : 2;
    static constexpr int kChunk = 128 / kElem;                  // columns of a 128-byte row of a chunk
    static constexpr int kKChunks = (DQK + kChunk - 1) / kChunk;
    static constexpr int kVChunks = (DV + kChunk - 1) / kChunk;
    static constexpr int kKBytes = kKChunks * kChunkBytes;
    static constexpr int kVBytes = kVChunks * kChunkBytes;
    static constexpr int kQRows = kTerms * kRows;               // rows of the staged queries
    static constexpr int kQChunkBytes = kQRows * 128;
    static constexpr int kQBytes = kKChunks * kQChunkBytes;
    static constexpr int kPChunks = kE4m3 ? 1 : 2;              // 128 keys of 1 or 2 bytes in rows of 128
    static constexpr int kPChunkBytes = kCols * 128;
    static constexpr int kPBytes = kPChunks * kPChunkBytes;
    // bf16 values of 64: the upper 64 lanes of O^T multiply a block of zeros
    static constexpr bool kZeroBlock = !kE4m3 && DV == 64;
    static constexpr int kZeroBytes = kZeroBlock ? 2048 : 0;
    static constexpr int kFixedBytes = 2 * kQBytes + 2 * kPBytes + kZeroBytes;
    static constexpr int kBudget = 227 * 1024 - 12 * 1024;      // the rest is for PagedShared
    static constexpr int kFit = (kBudget - kFixedBytes) / (kKBytes + kVBytes);
    static constexpr int kStages = kFit > 6 ? 6 : kFit;
    static_assert(kStages >= 2, "shared memory budget exceeded");
    static constexpr int kTileBytes = kFixedBytes + kStages * (kKBytes + kVBytes);
    static constexpr int kTmemCols = 4 * kCols <= 64 ? 64 : 4 * kCols <= 128 ? 128 : 4 * kCols <= 256 ? 256 : 512;
    static_assert(4 * kCols <= 512 && kCols % 16 == 0 && kCols <= 256, "accumulators");
    static constexpr int kKSteps = DQK * kElem / 32;            // k-steps of 32 bytes
    static constexpr int kPSteps = 128 * kElem / 32;
    // exponents above the reference that a score may reach before the reference moves, and the scaling of P
    static constexpr float kTauLog2 = kE4m3 ? 2.f : 8.f;
    static constexpr float kBias = kE4m3 ? 13.f : 0.f;
};

template <int kRows, int kMaps>
struct PagedShared {
    uint64_t k_full[6], k_empty[6], v_full[6], v_empty[6];
    uint64_t q_full[2], q_empty[2];
    uint64_t s_full[2], p_full[2], pv_done[2];
    uint32_t tmem_base;
    uint32_t abort_flag;
    uint32_t is_last;
    int start_b;
    long long start_base, total_units;
    long long warp_sums[12];
    struct Row { float c; int i; } row[2][kRows];        // factor of a score (log2 units), place among the new tokens
    long long out_at[2][kRows];                          // offset of the row in O (-1: a padding row)
    int out_hq[2][kRows];
    float m[2][kMaps * kRows];                           // reference maximum per group and state
    float rescale[2][kMaps * kRows];
    float red[2][4][kMaps * kRows];                      // per group and warp: maxima, or row sums
    float factor[2][kMaps * kRows];                      // weights of the two groups' accumulators
    float sq[2][4][kRows];
};

template <int DQK, int DV, bool kE4m3, bool kDiff, int kRows>
constexpr int paged_smem_bytes() {
    using Cfg = PagedCfg<DQK, DV, kE4m3, kDiff, kRows>;
    return Cfg::kTileBytes + static_cast<int>(sizeof(PagedShared<kRows, Cfg::kMaps>));
}
// Bytes of a partial result: unnormalised O of every state (fp32) and its maximum and sum.
constexpr long long paged_slot_bytes(int dv, int states) { return states * (dv + 2) * 4ll; }

// ------------------------------------------------------------------ kernel

template <int DQK, int DV, bool kE4m3, bool kDiff, int kRows>
__global__ void __launch_bounds__(384, 1)
fa_paged_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const PagedParams p) {
    using Cfg = PagedCfg<DQK, DV, kE4m3, kDiff, kRows>;
    using Shared = PagedShared<kRows, Cfg::kMaps>;
    using namespace ptx;
    constexpr int NS = Cfg::kStages, kMaps = Cfg::kMaps, kTerms = Cfg::kTerms, kStates = Cfg::kStates, kCols = Cfg::kCols;

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(smem_raw + Cfg::kTileBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t smem_base = smem_addr(smem_raw);
    const uint32_t sK = smem_base, sV = sK + NS * Cfg::kKBytes, sQ = sV + NS * Cfg::kVBytes, sP = sQ + 2 * Cfg::kQBytes,
                   sZero = sP + 2 * Cfg::kPBytes;

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
        sh.abort_flag = 0;
        for (int s = 0; s < NS; ++s) {
            mbar_init(smem_addr(&sh.k_full[s]), 1);
            mbar_init(smem_addr(&sh.k_empty[s]), 1);
            mbar_init(smem_addr(&sh.v_full[s]), 1);
            mbar_init(smem_addr(&sh.v_empty[s]), 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(smem_addr(&sh.q_full[w]), 2);       // the two query warps
            mbar_init(smem_addr(&sh.q_empty[w]), 3);      // the last score MMA and the two softmax groups
            mbar_init(smem_addr(&sh.s_full[w]), 1);
            mbar_init(smem_addr(&sh.p_full[w]), 4);       // four warps
            mbar_init(smem_addr(&sh.pv_done[w]), 1);
        }
        fence_mbar_init();
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
    }
    if constexpr (Cfg::kZeroBlock) {
        if (tid < 128) st_shared_v4(sZero + tid * 16, 0, 0, 0, 0);
    }
    grid_dependency_wait();

    // ---- the shares: every thread sums up the units of consecutive sequences, a scan over the CTA finds the total
    const int chunk = (p.B + 383) / 384;
    const int b_first = tid * chunk, b_last = min(p.B, b_first + chunk);
    long long mine = 0;
    for (int b = b_first; b < b_last; ++b) mine += paged_units(p, b);
    long long before = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before += o;
    }
    if (lane == 31) sh.warp_sums[warp] = before;
    before -= mine;
    if constexpr (Cfg::kZeroBlock) fence_proxy_async_smem();
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < 12; ++w) {
        const long long x = sh.warp_sums[w];
        if (w < warp) before += x;
        total += x;
    }
    const long long share = paged_share(total, gridDim.x, p.least_units);
    const long long u0 = blockIdx.x * share, u1 = min(total, u0 + share);
    if (u0 >= total) return;                  // uniform; no TMEM allocated yet
    if (before <= u0 && u0 < before + mine) {
        int b = b_first;
        long long base = before;
        for (;; ++b) {
            const long long n = paged_units(p, b);
            if (u0 < base + n) break;
            base += n;
        }
        sh.start_b = b;
        sh.start_base = base;
    }
    if (warp == 1) {
        tmem_alloc(smem_addr(&sh.tmem_base), Cfg::kTmemCols);
        tmem_relinquish_alloc_permit();
    }
    if (tid < 2 * kStates) sh.m[tid / kStates][tid % kStates] = -INFINITY;
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem_base;       // S^T of group w at w*kCols, O^T at (2 + w)*kCols
    WaitCtx wctx{&sh.abort_flag, p.status, p.wait_limit_ns};
    const int group = p.Hq / p.Hkv;
    PagedPart part;

    if (warp == 0) {
        // ============================================================ TMA loads: lane i takes the i-th page box of a tile
        part.begin(p, sh.start_b, sh.start_base, u0, u1, lane == 0);
        const int box = p.box_rows, boxes = kTileN / box;
        int n = 0;
        bool ok = true;
        do {
            const int kvh = part.hr / p.row_blocks;
            const long long row = part.b * p.table_stride;
            // the box of this lane in tile t: its page (the pool's end, which reads as zeros, for a page that is none) and slot
            auto look_up = [&](int t, int& page, int& slot) {
                const int key = t * kTileN + lane * box;
                page = -1;
                if (lane < boxes && key < part.len) {
                    const int at = key / p.page_size;
                    slot = key - at * p.page_size;
                    page = p.block_table[row + at];
                    if (page < 0 || page >= p.num_pages) {
                        report_bad_input(p.status, kSiteBadPage);
                        page = p.num_pages;
                    }
                }
            };
            int page, slot = 0, next_page = -1, next_slot = 0;
            look_up(part.t0, page, slot);
            for (int t = part.t0; t < part.t1 && ok; ++t, ++n) {
                if (t + 1 < part.t1) look_up(t + 1, next_page, next_slot);
                const int s = n % NS;
                const uint32_t parity = ((n / NS) & 1) ^ 1;
                const int n_box = min(boxes, (max(0, part.len - t * kTileN) + box - 1) / box);
                const uint32_t kb = smem_addr(&sh.k_full[s]), vb = smem_addr(&sh.v_full[s]);
                ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&sh.k_empty[s]), parity, wctx, kSiteLoadKvEmpty));
                if (!ok) break;
                if (lane == 0) mbar_arrive_expect_tx(kb, n_box * box * 128 * Cfg::kKChunks);
                __syncwarp();
                if (page >= 0)
#pragma unroll
                    for (int c = 0; c < Cfg::kKChunks; ++c)
                        tma_load_4d(sK + s * Cfg::kKBytes + c * kChunkBytes + lane * box * 128, &tm_k, kb, c * Cfg::kChunk, slot, kvh, page);
                __syncwarp();
                if (!(p.debug_drop_v_load && n == 0)) {
                    ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&sh.v_empty[s]), parity, wctx, kSiteLoadKvEmpty));
                    if (!ok) break;
                    if (lane == 0) mbar_arrive_expect_tx(vb, n_box * box * 128 * Cfg::kVChunks);
                    __syncwarp();
                    if (page >= 0)
#pragma unroll
                        for (int c = 0; c < Cfg::kVChunks; ++c)
                            tma_load_4d(sV + s * Cfg::kVBytes + c * kChunkBytes + lane * box * 128, &tm_v, vb, c * Cfg::kChunk, slot, kvh, page);
                    __syncwarp();
                }
                page = next_page;
                slot = next_slot;
            }
        } while (ok && part.next(p));
    } else if (warp == 1) {
        // ============================================================ MMA issue, one thread
        if (elect_one()) {
            part.begin(p, sh.start_b, sh.start_base, u0, u1, false);
            const int n_total = static_cast<int>(u1 - u0);
            constexpr uint32_t kIdescQK = kE4m3 ? (make_idesc_e4m3_f32(128, Cfg::kQRows, false, false) | (1u << 10))
                                                : make_idesc_bf16_f32(128, Cfg::kQRows, false, false);
            constexpr uint32_t kIdescPV = kE4m3 ? (make_idesc_e4m3_f32(128, kCols, true, false) | (1u << 10))
                                                : make_idesc_bf16_f32(128, kCols, true, false);
            auto mma = [](uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
                if constexpr (kE4m3) mma_ss_f8(d, a, b, idesc, acc);
                else mma_ss(d, a, b, idesc, acc);
            };
            bool ok = true;
            int seg = 0, left = part.t1 - part.t0;           // of the score products: segment and its tiles to come
            auto scores = [&](int n) -> bool {
                const int w = n & 1, s = n % NS, qb = seg & 1;
                if (left == part.t1 - part.t0 && !mbar_wait(smem_addr(&sh.q_full[qb]), (seg >> 1) & 1, wctx, kSiteMmaQFull)) return false;
                if (!mbar_wait(smem_addr(&sh.k_full[s]), (n / NS) & 1, wctx, kSiteMmaKvFull)) return false;
                tc_fence_after_sync();
                const uint32_t a0 = sK + s * Cfg::kKBytes, b0 = sQ + qb * Cfg::kQBytes;
                constexpr int kPerMap = Cfg::kKSteps / kMaps;
#pragma unroll
                for (int m = 0; m < kMaps; ++m)
#pragma unroll
                    for (int j = 0; j < kPerMap; ++j) {
                        const int k = m * kPerMap + j;
                        mma(tmem + w * kCols + m * Cfg::kQRows,
                            make_smem_desc_sw128(a0 + (k / 4) * kChunkBytes + (k % 4) * 32, 16, 1024),
                            make_smem_desc_sw128(b0 + (k / 4) * Cfg::kQChunkBytes + (k % 4) * 32, 16, 1024), kIdescQK, j > 0 ? 1u : 0u);
                    }
                tc_commit(smem_addr(&sh.s_full[w]));
                tc_commit(smem_addr(&sh.k_empty[s]));
                if (--left == 0) {
                    tc_commit(smem_addr(&sh.q_empty[qb]));
                    ++seg;
                    if (part.next(p)) left = part.t1 - part.t0;
                }
                return true;
            };
            // the same walk again for the second products: a group's accumulator starts anew with each part
            PagedPart pv;
            pv.begin(p, sh.start_b, sh.start_base, u0, u1, false);
            int pv_done = 0, pv_tiles = pv.t1 - pv.t0;
            ok = scores(0);
            if (ok && n_total > 1) ok = scores(1);
            for (int n = 0; n < n_total && ok; ++n) {
                const int w = n & 1, s = n % NS;
                ok = mbar_wait(smem_addr(&sh.v_full[s]), (n / NS) & 1, wctx, kSiteMmaKvFull) &&
                     mbar_wait(smem_addr(&sh.p_full[w]), (n >> 1) & 1, wctx, kSiteMmaPFull);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t a0 = sV + s * Cfg::kVBytes, b0 = sP + w * Cfg::kPBytes;
#pragma unroll
                for (int k = 0; k < Cfg::kPSteps; ++k) {
                    constexpr int kStepBytes = (32 / Cfg::kElem) * 128;        // keys of a k-step x 128 bytes
                    const uint32_t a = a0 + k * kStepBytes;
                    const uint32_t lbo = Cfg::kZeroBlock ? sZero - a : static_cast<uint32_t>(kChunkBytes);
                    mma(tmem + (2 + w) * kCols, make_smem_desc_sw128(a, lbo, 1024),
                        make_smem_desc_sw128(b0 + (k / 4) * Cfg::kPChunkBytes + (k % 4) * 32, 16, 1024), kIdescPV,
                        (pv_done >= 2 || k > 0) ? 1u : 0u);
                }
                tc_commit(smem_addr(&sh.v_empty[s]));
                tc_commit(smem_addr(&sh.pv_done[w]));
                if (++pv_done == pv_tiles && pv.next(p)) {
                    pv_done = 0;
                    pv_tiles = pv.t1 - pv.t0;
                }
                if (n + 2 < n_total) ok = scores(n + 2);
            }
        }
    } else if (warp < 4) {
        // ============================================================ query rows -> shared memory, and what is known of each
        part.begin(p, sh.start_b, sh.start_base, u0, u1, false);
        int seg = 0;
        bool ok = true;
        do {
            const int qb = seg & 1;
            ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&sh.q_empty[qb]), ((seg >> 1) & 1) ^ 1, wctx, kSiteLoadQEmpty));
            if (!ok) break;
            const int kvh = part.hr / p.row_blocks, rb = part.hr - kvh * p.row_blocks;
            constexpr int kVecs = DQK / 8;                        // 16-byte pieces of a row
            const float ks = kE4m3 && p.k_scale ? p.k_scale[kvh] : 1.f;
            // a warp takes every other row, a lane a piece of it
            constexpr int kBatch = kRows / 2 < 8 ? kRows / 2 : 8;
#pragma unroll 1
            for (int r0 = 0; r0 < kRows / 2; r0 += kBatch) {
                uint4 x[kBatch];
#pragma unroll
                for (int e = 0; e < kBatch; ++e) {
                    const int r = 2 * (r0 + e) + (warp - 2), rr = rb * kRows + r, i = rr / group, hq = kvh * group + rr - i * group;
                    const bool live = i < p.Sq;
                    x[e] = make_uint4(0, 0, 0, 0);
                    if (live && lane < kVecs)
                        x[e] = *reinterpret_cast<const uint4*>(p.Q + part.b * p.q_sb + i * p.q_st + hq * p.q_sh + lane * 8);
                    if (lane == 0) {
                        sh.row[qb][r].i = live ? i : p.Sq - 1;
                        sh.row[qb][r].c = p.scale_log2 * ks;
                        sh.out_at[qb][r] = live ? part.b * p.o_sb + i * p.o_st + hq * p.o_sh : -1;
                        sh.out_hq[qb][r] = hq;
                    }
                }
#pragma unroll
                for (int e = 0; e < kBatch; ++e) {
                    const int r = 2 * (r0 + e) + (warp - 2);
                    if constexpr (!kE4m3) {
                        if (lane < kVecs)
                            st_shared_v4(sQ + qb * Cfg::kQBytes + (lane >> 3) * Cfg::kQChunkBytes + r * 128 + (((lane & 7) ^ (r & 7)) << 4),
                                         x[e].x, x[e].y, x[e].z, x[e].w);
                    } else {
                        // scaled by a power of two so that the row's largest entry is in [2^14, 2^15), then three e5m2 terms: exact for
                        // entries of 2^-24 of the largest and more, below that to 2^-31 of it
                        const uint32_t w4[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
                        uint32_t top = 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            top = max(top, (w4[i] & 0x7fffu) << 16);
                            top = max(top, w4[i] & 0x7fff0000u);
                        }
                        top = __reduce_max_sync(0xffffffffu, top);
                        int sft = top ? 14 - (static_cast<int>(top >> 23) - 127) : 0;
                        sft = sft > 100 ? 100 : (sft < -100 ? -100 : sft);
                        const float mult = __uint_as_float(static_cast<uint32_t>(sft + 127) << 23);
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
                        if (lane < kVecs) {
#pragma unroll
                            for (int t = 0; t < 3; ++t) {
                                const int rq = t * kRows + r, piece = lane >> 1;
                                st_shared_u64(sQ + qb * Cfg::kQBytes + (piece >> 3) * Cfg::kQChunkBytes + rq * 128 +
                                                  (((piece & 7) ^ (rq & 7)) << 4) + (lane & 1) * 8, t8[t][0], t8[t][1]);
                            }
                        }
                        if (lane == 0) sh.row[qb][r].c = p.scale_log2 * ks * __uint_as_float(static_cast<uint32_t>(127 - sft) << 23);
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.q_full[qb]));
            ++seg;
        } while (part.next(p));
    } else {
        // ============================================================ softmax groups
        // No thread leaves this branch early: after a wait that ran out every later wait returns at once, and the groups go on
        // through their barriers (results are invalid then, every access stays in bounds).
        const int w = (warp >> 2) - 1, key = tid & 127, wq = warp & 3;
        const uint32_t lane_sel = static_cast<uint32_t>(wq * 32) << 16;
        const uint32_t tS = tmem + w * kCols + lane_sel, tO = tmem + (2 + w) * kCols + lane_sel;
        const uint32_t sPw = sP + w * Cfg::kPBytes + (kE4m3 ? 0 : (key >> 6) * Cfg::kPChunkBytes);
        const uint32_t p_byte = kE4m3 ? key : (key & 63) * 2;            // of this key in a row of P
        part.begin(p, sh.start_b, sh.start_base, u0, u1, false);
        float l[kStates];
#pragma unroll
        for (int r = 0; r < kStates; ++r) l[r] = 0.f;
        int n = 0, seg = 0;
        bool ok = true;
        do {
            const int qb = seg & 1;
            ok = ok && mbar_wait(smem_addr(&sh.q_full[qb]), (seg >> 1) & 1, wctx, kSiteMmaQFull);
            bool any_tile = false;
            const int first_masked = part.len - p.Sq + 1;                // the first key that some row does not see
#pragma unroll 1
            for (int t = part.t0; t < part.t1; ++t, ++n) {
                if ((n & 1) != w) continue;
                ok = ok && mbar_wait(smem_addr(&sh.s_full[w]), (n >> 1) & 1, wctx, kSiteSoftmaxSFull);
                __syncwarp();
                tc_fence_after_sync();
                float x[kStates];
#pragma unroll
                for (int g = 0; g < kStates / 16; ++g) {
                    // column of (map, term, row): (map * kTerms + term) * kRows + row
                    const int map = g * 16 / kRows, r0 = g * 16 % kRows;
                    uint32_t s0[16];
                    tmem_ld_x16(tS + map * kTerms * kRows + r0, s0);
                    if constexpr (kE4m3) {
                        uint32_t s1[16], s2[16];
                        tmem_ld_x16(tS + (map * kTerms + 1) * kRows + r0, s1);
                        tmem_ld_x16(tS + (map * kTerms + 2) * kRows + r0, s2);
                        tc_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            x[g * 16 + e] = __uint_as_float(s0[e]) + (__uint_as_float(s1[e]) + __uint_as_float(s2[e]));
                    } else {
                        tc_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[g * 16 + e] = __uint_as_float(s0[e]);
                    }
                }
                const int key_at = t * kTileN + key;
                if (kE4m3) {
#pragma unroll
                    for (int r = 0; r < kStates; ++r) x[r] *= sh.row[qb][r % kRows].c;
                } else {
#pragma unroll
                    for (int r = 0; r < kStates; ++r) x[r] *= p.scale_log2;
                }
                if (t * kTileN + kTileN > first_masked) {
#pragma unroll
                    for (int r = 0; r < kStates; ++r)
                        if (key_at >= first_masked + sh.row[qb][r % kRows].i) x[r] = -INFINITY;
                }
                bool over = false;
#pragma unroll
                for (int r = 0; r < kStates; ++r) over |= x[r] > sh.m[w][r] + Cfg::kTauLog2;
                if (named_barrier_or(1 + w, 128, over)) {
#pragma unroll
                    for (int r = 0; r < kStates; ++r) {
                        const float mx = warp_max(x[r]);
                        if (lane == 0) sh.red[w][wq][r] = mx;
                    }
                    named_barrier_sync(1 + w, 128);
                    if (key < kStates) {
                        const float old = sh.m[w][key];
                        const float mx = fmaxf(fmaxf(fmaxf(sh.red[w][0][key], sh.red[w][1][key]), fmaxf(sh.red[w][2][key], sh.red[w][3][key])), old);
                        sh.m[w][key] = mx;
                        sh.rescale[w][key] = mx == -INFINITY ? 1.f : exp2_approx(old - mx);
                    }
                    named_barrier_sync(1 + w, 128);
#pragma unroll
                    for (int r = 0; r < kStates; ++r) l[r] *= sh.rescale[w][r];
                    if (any_tile) {
                        // PV of this group's tile before is complete (these scores were issued after it), the next one waits for us
#pragma unroll 1
                        for (int g = 0; g < kCols / 16; ++g) {
                            const int col = g * 16, st = col / (kTerms * kRows) * kRows + col % kRows;
                            uint32_t o[16];
                            tmem_ld_x16(tO + col, o);
                            tc_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * sh.rescale[w][st + e]);
                            tmem_st_x16(tO + col, o);
                        }
                        tc_wait_st();
                    }
                }
#pragma unroll
                for (int r = 0; r < kStates; ++r) {
                    const float m = sh.m[w][r];
                    x[r] = exp2_approx(x[r] - ((m == -INFINITY ? 0.f : m) - Cfg::kBias));
                    l[r] += x[r];
                }
                // P^T: row = column of O^T, 128 keys of 1 or 2 bytes, 16-byte pieces swizzled
                if constexpr (kE4m3) {
#pragma unroll
                    for (int r = 0; r < kStates; r += 2) {
                        __half2 h = __floats2half2_rn(x[r], x[r + 1]);
#pragma unroll
                        for (int term = 0; term < 3; ++term) {
                            uint32_t bits = *reinterpret_cast<uint32_t*>(&h) & 0xff00ff00u;
                            const int col = (r / kRows * kTerms + term) * kRows + r % kRows;
                            st_shared_u8(sPw + col * 128 + (p_byte ^ ((col & 7) << 4)), (bits >> 8) & 0xffu);
                            st_shared_u8(sPw + (col + 1) * 128 + (p_byte ^ (((col + 1) & 7) << 4)), bits >> 24);
                            h = __hsub2(h, *reinterpret_cast<__half2*>(&bits));
                        }
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < kStates; r += 2) {
                        const uint32_t two = pack_bf16x2(x[r], x[r + 1]);
                        st_shared_u16(sPw + r * 128 + (p_byte ^ ((r & 7) << 4)), two);
                        st_shared_u16(sPw + (r + 1) * 128 + (p_byte ^ (((r + 1) & 7) << 4)), two >> 16);
                    }
                }
                if (t * kTileN + kTileN > part.len) {
                    // V rows behind the sequence's end hold whatever the page held, or were not loaded: zeros, since 0 * NaN is NaN
                    const int s = n % NS;
                    ok = ok && mbar_wait(smem_addr(&sh.v_full[s]), (n / NS) & 1, wctx, kSiteSoftmaxPFree);
                    if (key_at >= part.len) {
#pragma unroll
                        for (int c = 0; c < Cfg::kVChunks * 8; ++c)
                            st_shared_v4(sV + s * Cfg::kVBytes + (c >> 3) * kChunkBytes + key * 128 + (c & 7) * 16, 0, 0, 0, 0);
                    }
                }
                any_tile = true;
                fence_proxy_async_smem();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.p_full[w]));
            }

            // ---- end of a part: the groups' accumulators become one
            // row sums over the 128 threads of the group: 16 columns at a time, halved at each exchange
#pragma unroll
            for (int g = 0; g < kStates / 16; ++g) {
                float a[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) a[e] = l[g * 16 + e];
#pragma unroll
                for (int d = 16, m = 8; d >= 2; d >>= 1, m >>= 1) {
                    const bool up = (lane & d) != 0;
#pragma unroll
                    for (int e = 0; e < m; ++e) {
                        const float give = up ? a[e] : a[e + m], keep = up ? a[e + m] : a[e];
                        a[e] = keep + __shfl_xor_sync(0xffffffffu, give, d);
                    }
                }
                a[0] += __shfl_xor_sync(0xffffffffu, a[0], 1);
                // lane bits 4, 3, 2, 1 chose the halves: column = bit4*8 + bit3*4 + bit2*2 + bit1
                if ((lane & 1) == 0) sh.red[w][wq][g * 16 + (lane >> 1)] = a[0];
            }
            if (any_tile) {
                const int last = ((n - 1) & 1) == w ? n - 1 : n - 2;       // this group's last tile
                ok = ok && mbar_wait(smem_addr(&sh.pv_done[w]), (last >> 1) & 1, wctx, kSiteEpiOFull);
            }
            __syncwarp();
            tc_fence_before_sync();
            named_barrier_sync(3, 256);
            tc_fence_after_sync();
            const long long ua = part.first_unit();
            const bool whole = part.t1 - part.t0 == part.nt;
            const int gt = tid - 128;                                     // 0..255
            const int slot = whole ? 0 : paged_slot(blockIdx.x, ua, share);
            float* const slot_o = p.part + static_cast<long long>(slot) * kStates * (DV + 2);
            float* const slot_ml = slot_o + kStates * DV;
            // log-sum-exp of a row (natural units) from its maximum (log2 units) and sum, and where it goes
            auto store_lse = [&](int r, float m, float sum) {
                if (kDiff || !p.lse || sh.out_at[qb][r] < 0) return;
                p.lse[static_cast<long long>(sh.out_hq[qb][r]) * p.B * p.Sq + static_cast<long long>(part.b) * p.Sq + sh.row[qb][r].i] =
                    sum > 0.f ? (m - Cfg::kBias + log2f(sum)) * 0.6931471805599453f : -INFINITY;
            };
            if (gt < kStates) {
                float sum[2], mx[2];
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    mx[v] = sh.m[v][gt];
                    sum[v] = sh.red[v][0][gt] + sh.red[v][1][gt] + sh.red[v][2][gt] + sh.red[v][3][gt];
                }
                const float m = fmaxf(mx[0], mx[1]);
                float f[2];
#pragma unroll
                for (int v = 0; v < 2; ++v) f[v] = mx[v] == -INFINITY ? 0.f : exp2_approx(mx[v] - m);
                const float all = f[0] * sum[0] + f[1] * sum[1];
                const float norm = !whole ? 1.f : (all > 0.f || all != all ? 1.f / all : 0.f);
                sh.factor[0][gt] = f[0] * norm;
                sh.factor[1][gt] = f[1] * norm;
                if (whole) {
                    store_lse(gt % kRows, m, all);
                } else {
                    slot_ml[gt] = m;
                    slot_ml[kStates + gt] = all;
                }
            }
            named_barrier_sync(3, 256);
            // thread = output column; group w takes its half of the rows
            constexpr int kHalf = kRows / 2;
            const float vs = kE4m3 && p.v_scale ? p.v_scale[part.hr / p.row_blocks] : 1.f;
            // the rows' results [map][row] to O: the difference and its norm, or the result itself
            auto store_rows = [&](float (&y)[kMaps][kHalf]) {
                if constexpr (kDiff) {
#pragma unroll
                    for (int e = 0; e < kHalf; ++e)
                        y[0][e] = vs * (y[0][e] - p.lambda[sh.out_hq[qb][w * kHalf + e]] * y[1][e]);
                    if (p.weight) {
#pragma unroll
                        for (int e = 0; e < kHalf; ++e) {
                            float q = y[0][e] * y[0][e];
#pragma unroll
                            for (int d = 16; d > 0; d >>= 1) q += __shfl_xor_sync(0xffffffffu, q, d);
                            if (lane == 0) sh.sq[w][wq][e] = q;
                        }
                        named_barrier_sync(1 + w, 128);
                        const float wt = p.weight[key];
#pragma unroll
                        for (int e = 0; e < kHalf; ++e) {
                            const float q = sh.sq[w][0][e] + sh.sq[w][1][e] + sh.sq[w][2][e] + sh.sq[w][3][e];
                            y[0][e] *= wt * rsqrtf(q * (1.f / DV) + p.eps);
                        }
                        named_barrier_sync(1 + w, 128);
                    }
#pragma unroll
                    for (int e = 0; e < kHalf; ++e) y[0][e] *= p.out_scale;
                } else {
#pragma unroll
                    for (int e = 0; e < kHalf; ++e) y[0][e] *= vs;
                }
                if (key < DV) {
#pragma unroll
                    for (int e = 0; e < kHalf; ++e) {
                        const long long at = sh.out_at[qb][w * kHalf + e];
                        if (at >= 0) p.O[at + key] = __float2bfloat16(y[0][e]);
                    }
                }
            };
            const bool had0 = part.t1 - part.t0 > 1 || ((n - 1) & 1) == 0, had1 = part.t1 - part.t0 > 1 || ((n - 1) & 1) == 1;
            float y[kMaps][kHalf];
#pragma unroll
            for (int a = 0; a < kMaps; ++a) {
#pragma unroll
                for (int e = 0; e < kHalf; ++e) y[a][e] = 0.f;
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    if (!(v == 0 ? had0 : had1)) continue;                // (uniform) nothing of this part in that accumulator
#pragma unroll
                    for (int term = 0; term < kTerms; ++term)
#pragma unroll
                        for (int e0 = 0; e0 < kHalf; e0 += 8) {
                            uint32_t o[8];
                            tmem_ld_x8(tmem + (2 + v) * kCols + lane_sel + (a * kTerms + term) * kRows + w * kHalf + e0, o);
                            tc_wait_ld();
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float f = sh.factor[v][a * kRows + w * kHalf + e0 + e];
                                // (a row that saw no key in this group's tiles: its accumulator is all zeros)
                                y[a][e0 + e] = fmaf(f, __uint_as_float(o[e]), y[a][e0 + e]);
                            }
                        }
                }
            }
            if (whole) {
                store_rows(y);
            } else {
                if (key < DV) {
#pragma unroll
                    for (int a = 0; a < kMaps; ++a)
#pragma unroll
                        for (int e = 0; e < kHalf; ++e) slot_o[(a * kRows + w * kHalf + e) * DV + key] = y[a][e];
                }
                __threadfence();
                named_barrier_sync(3, 256);
                const int pieces = paged_pieces(ua, ua + part.nt, share), c0 = paged_first_cta(ua, share);
                if (gt == 0) {
                    const unsigned int got = atomicAdd(p.arrivals + c0, 1u);
                    sh.is_last = got == static_cast<unsigned int>(pieces - 1) ? 1u : 0u;
                    if (sh.is_last) p.arrivals[c0] = 0u;
                    __threadfence();
                }
                named_barrier_sync(3, 256);
                if (sh.is_last) {
                    __threadfence();
                    auto piece = [&](int c) { return p.part + static_cast<long long>(paged_slot(c0 + c, ua, share)) * kStates * (DV + 2); };
                    if (gt < kStates) {
                        float m = -INFINITY, sum = 0.f;
                        for (int c = 0; c < pieces; ++c) m = fmaxf(m, __ldcg(piece(c) + kStates * DV + gt));
                        for (int c = 0; c < pieces; ++c) {
                            const float mc = __ldcg(piece(c) + kStates * DV + gt);
                            // (a piece without a finite score counts nothing, but a NaN of its sum goes through)
                            sum += (mc == -INFINITY ? 0.f : exp2_approx(mc - m)) * __ldcg(piece(c) + kStates * DV + kStates + gt);
                        }
                        store_lse(gt % kRows, m, sum);
                        sh.factor[0][gt] = m;
                        sh.factor[1][gt] = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                    }
                    named_barrier_sync(3, 256);
#pragma unroll
                    for (int a = 0; a < kMaps; ++a)
#pragma unroll
                        for (int e = 0; e < kHalf; ++e) y[a][e] = 0.f;
                    if (key < DV) {
                        for (int c = 0; c < pieces; ++c) {
                            const float* po = piece(c);
#pragma unroll
                            for (int a = 0; a < kMaps; ++a)
#pragma unroll
                                for (int e = 0; e < kHalf; ++e) {
                                    const int st = a * kRows + w * kHalf + e;
                                    const float mc = __ldcg(po + kStates * DV + st);
                                    const float f = mc == -INFINITY ? 0.f : exp2_approx(mc - sh.factor[0][st]) * sh.factor[1][st];
                                    y[a][e] = fmaf(f, __ldcg(po + st * DV + key), y[a][e]);
                                }
                        }
                    }
                    store_rows(y);
                }
            }
            // both groups have read the accumulators, factors and rows: the next part may begin
            if (key < kStates) sh.m[w][key] = -INFINITY;
#pragma unroll
            for (int r = 0; r < kStates; ++r) l[r] = 0.f;
            tc_fence_before_sync();
            named_barrier_sync(3, 256);
            tc_fence_after_sync();
            if (key == 0) mbar_arrive(smem_addr(&sh.q_empty[qb]));
            ++seg;
        } while (part.next(p));
    }

    // ---------------------------------------------------------------- teardown (all warps)
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, Cfg::kTmemCols);
}

}  // namespace fa
