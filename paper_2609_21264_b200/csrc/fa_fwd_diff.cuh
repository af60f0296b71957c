// Differential attention over whole prompts for sm_100a, two maps of 64 over values of 128:
//     Y = (softmax(s Q1 K1^T) - lambda softmax(s Q2 K2^T)) V,   O = out_scale * weight (*) Y / sqrt(mean(Y^2) + eps)
//
// The loop of fa_fwd_pair.cuh (read that file first), with the two MAPS of one query tile in the place of two query tiles: S_t is
// the product of the t-th halves of Q and K (four k-steps of 16 and not eight), both maps' probabilities multiply the same
// V tile, and Q, K and V are loaded once for both.  Run as two heads of ordinary attention (zeros in the other half of Q, the
// difference and the norm in a kernel of their own), the scores would cost twice the MMAs, O would be written and read once
// more in each map, and K and V would be read as often but for twice the heads.
//
// What bounds it: the chain softmax -> P V_j -> Q K_{j+1} -> softmax of each map, which has one S with P over it.  A K/V tile takes some
// 3400 cycles (4096 tokens causal, 114 tiles an SM), of which 24 MMAs of 64 cycles are 1536 (tensor pipe 46 % busy) and two thirds of
// 2 x 128 x 128 exponentials 1365 (special-function unit 45 %); 52 % of the issue slots are used, two warps a scheduler.
//
// P is rounded to bf16 once (error 2.5e-3 of the result; the output's own rounding makes 1.65e-3).  The second half of S has room for a
// second term, and that makes the error 1.65e-3, but its 16 MMAs a tile and its arithmetic lie on the chain: 327 us, against 237
// (4096 tokens causal, 32/8 heads, back to back), 26.1 against 20 (2 x 8 heads, 1001 tokens).
//
// Epilogue: both groups of softmax warps read BOTH accumulators (a warp reaches the same 32 TMEM lanes of every column), each for one
// half of the 128 columns; row sums, lambda and the halves' sums of squares cross through shared memory, and each group
// stages and stores its 64-column chunk.  Nothing but O leaves the SM.
//
// Persistent: one CTA per SM draws (query tile, head) items by ticket, in L2-sized groups of heads, longest first.  The set-up is
// paid once, the next item's query tile (two buffers) and its first K and V tiles load and its first scores are multiplied under
// the current item's epilogue.  Against one item per CTA: 4096 tokens causal, 32/8 heads, 217.6 us (231.6); 16 x 300 tokens 91.3
// (132.3); level on items of 128 tiles.
//
// Roles (384 threads), TMEM: as in fa_fwd_pair.cuh (warps 0-3 / 4-7 softmax of map 0 / 1, warp 8 MMA issue, warp 9 loads and tickets).
#pragma once

#include <math.h>

#include "fa_common.cuh"
#include "fa_fwd_pair.cuh"
#include "fa_softmax_pass.cuh"
#include "ptx.cuh"

namespace fa {

struct DiffParams {
    const float* lambda;          // [Hq]
    const float* weight;          // [128] or nullptr: no normalisation
    float eps, out_scale;
};

// Every third pair of exponentials is computed on the FMA pipe (exp2_poly2): with half of the score MMAs gone the special-function
// unit is what the two passes of a round wait for.  4096 tokens causal, 32/8 heads: 207.6 us, against 218.4 without, 211.1
// with every fourth and 218.7 with every second; 16 x 300 tokens 80.7 us, against 90.  (That masked scores come out as exact
// zeros costs 1 % of it: 211.9 us, against 209.5 in the same run.)
constexpr int kDiffPolyEvery = 3;

struct DiffCfg {
    static constexpr int kQBytes = 2 * kChunkBytes;     // a query tile, both maps (chunk t = map t); K and V tiles alike
    static constexpr int kKStages = 3, kVStages = 2;
    static constexpr int kTileBytes = (2 + kKStages + kVStages) * kQBytes;
    static constexpr int kItems = 4;                    // entries of the item ring
    static constexpr int kColS0 = 0, kColO0 = 256;      // S_t at 128 t, O_t at 256 + 128 t; bf16 P_t overlays S_t
    static constexpr int kThreads = 384;
};

struct DiffShared {
    uint64_t q_full[2], q_empty[2];
    uint64_t item_full[DiffCfg::kItems], item_empty[DiffCfg::kItems];
    int item[DiffCfg::kItems];       // index in the list, -1: no more
    uint64_t k_full[DiffCfg::kKStages], k_empty[DiffCfg::kKStages];
    uint64_t v_full[DiffCfg::kVStages], v_empty[DiffCfg::kVStages];
    uint64_t s_full[2], p_first[2], p_rest[2], o_final[2], o_staged[2];
    uint32_t tmem_base;
    uint32_t abort_flag;
    float inv_l[2][kTileM];
    alignas(16) float weight[128];
    float sum_sq[2][kTileM];
};

constexpr int diff_smem_bytes() { return DiffCfg::kTileBytes + static_cast<int>(sizeof(DiffShared)); }

__global__ void __launch_bounds__(384, 1)
fa_fwd_diff_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o, const FwdParams p,
                   const DiffParams dp) {
    using Cfg = DiffCfg;
    using namespace ptx;
    constexpr int NK = Cfg::kKStages, NV = Cfg::kVStages;

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    DiffShared& sh = *reinterpret_cast<DiffShared*>(smem_raw + Cfg::kTileBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    grid_launch_dependents();
    const uint32_t smem_base = smem_addr(smem_raw);
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
    const uint32_t sQ = smem_base, sK = sQ + 2 * Cfg::kQBytes, sV = sK + NK * Cfg::kQBytes;

    // items: (query tile, head), in L2-sized groups of heads, longest first (as in the other kernels)
    const int n_bh = p.B * p.Hq, hpg = p.heads_per_group;
    const int n_items = p.n_q_tiles * n_bh;
    struct Item { int i0, hq, b, nkv; };
    auto decode = [&](int item) -> Item {
        const int group = item / (p.n_q_tiles * hpg);
        const int bh0 = group * hpg;
        const int group_size = (n_bh - bh0 < hpg) ? (n_bh - bh0) : hpg;
        const int local = item - group * p.n_q_tiles * hpg;
        const int tile = local / group_size, bh = bh0 + local - tile * group_size;
        Item x;
        x.i0 = (p.n_q_tiles - 1 - tile) * kTileM;
        x.b = bh / p.Hq;
        x.hq = bh - x.b * p.Hq;
        x.nkv = kv_tiles_for_q_tile(x.i0, kTileM, p.Sq, p.Sk, p.causal);
        return x;
    };
    const int off = p.Sk - p.Sq;

    if (tid == 0) {
        sh.abort_flag = 0;
#pragma unroll
        for (int i = 0; i < Cfg::kItems; ++i) {
            mbar_init(smem_addr(&sh.item_full[i]), 1);
            mbar_init(smem_addr(&sh.item_empty[i]), 9);   // MMA thread, 8 softmax warps
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            mbar_init(smem_addr(&sh.q_full[t]), 1);
            mbar_init(smem_addr(&sh.q_empty[t]), 2);      // both chunks of the result, staged there, have been stored
            mbar_init(smem_addr(&sh.s_full[t]), 1);
            mbar_init(smem_addr(&sh.p_first[t]), 4);      // 4 softmax warps
            mbar_init(smem_addr(&sh.p_rest[t]), 4);
            mbar_init(smem_addr(&sh.o_final[t]), 1);
            mbar_init(smem_addr(&sh.o_staged[t]), 4);
        }
#pragma unroll
        for (int s = 0; s < NK; ++s) {
            mbar_init(smem_addr(&sh.k_full[s]), 1);
            mbar_init(smem_addr(&sh.k_empty[s]), 1);
        }
#pragma unroll
        for (int s = 0; s < NV; ++s) {
            mbar_init(smem_addr(&sh.v_full[s]), 1);
            mbar_init(smem_addr(&sh.v_empty[s]), 1);
        }
        fence_mbar_init();
    }
    if (warp == 8) {
        tmem_alloc(smem_addr(&sh.tmem_base), 512);
        tmem_relinquish_alloc_permit();
    }
    if (warp == 9 && lane == 0) {
        prefetch_tensormap(&tm_q);
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
        prefetch_tensormap(&tm_o);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    grid_dependency_wait();

    const uint32_t tmem_base = sh.tmem_base;
    WaitCtx wctx{&sh.abort_flag, p.status, p.wait_limit_ns};
    const float c = p.scale_log2;

    if (warp < 8) {
        // ============================================================ softmax of map t
        setmaxnreg_inc<kPairRegsSoftmax>();
        const int t = warp >> 2;
        const int row = tid & (kTileM - 1);
        const uint32_t lane_sel = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t tS = tmem_base + Cfg::kColS0 + 128 * t + lane_sel;
        const uint32_t tO = tmem_base + Cfg::kColO0 + lane_sel;
        const uint32_t bar_s = smem_addr(&sh.s_full[t]), bar_pf = smem_addr(&sh.p_first[t]), bar_pr = smem_addr(&sh.p_rest[t]);
        const float tau_raw = kRescaleThresholdLog2 / c;
        if (dp.weight && t == 0) sh.weight[row] = dp.weight[row];        // (read after the barriers of the first item)
        int n = 0, n_final = 0, stored_buf = -1;      // K/V tiles so far, items with one so far, buffer of a store not waited for
        bool ok = true;
        // the thread that stored the group's chunk of an item gives the buffer back once the store has read it
        auto release_buffer = [&]() {
            if (stored_buf >= 0 && (warp & 3) == 0 && lane == 0) {
                tma_store_wait_read_all();
                mbar_arrive(smem_addr(&sh.q_empty[stored_buf]));
            }
            stored_buf = -1;
        };
        // All 256 threads meet at the barriers of an item, also after a wait that ran out (nothing is stored then), and leave together.
        for (int it = 0;; ++it) {
            const int slot = it % Cfg::kItems, buf = it & 1;
            ok = ok && mbar_wait(smem_addr(&sh.item_full[slot]), (it / Cfg::kItems) & 1, wctx, kSiteItem);
            if (named_barrier_or(1, 256, !ok)) break;
            const int index = sh.item[slot];
            if (index < 0) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.item_empty[slot]));
            const Item x = decode(index);
            const float lambda = dp.lambda[x.hq];
            const int i_glob = x.i0 + row;
            int kmax_row = p.Sk - 1;
            if (p.causal && i_glob + off < kmax_row) kmax_row = i_glob + off;
            float m_ref = -INFINITY, l = 0.f;
            for (int j = 0; j < x.nkv; ++j, ++n) {
                ok = __all_sync(0xffffffffu, ok && mbar_wait(bar_s, n & 1, wctx, kSiteSoftmaxSFull));
                if (!ok) break;
                tc_fence_after_sync();
                softmax_pass_128<128, kDiffPolyEvery>(tS, tO + 128 * t, c, tau_raw, j * kTileN, kmax_row, j == 0, m_ref, l, lane,
                                      [&]() { mbar_arrive(bar_pf); }, [&]() { mbar_arrive(bar_pr); });
                if (j == 0) release_buffer();
            }
            release_buffer();
            // (a row that saw no key has a sum of exactly zero; the reference says nothing: at scales below 2.4e-38 tau_raw is infinite
            // and no reference is ever taken, all weights are 1; a NaN goes through)
            sh.inv_l[t][row] = l > 0.f || l != l ? (1.f / l) : 0.f;
            if (x.nkv > 0) {
                ok = ok && mbar_wait(smem_addr(&sh.o_final[0]), n_final & 1, wctx, kSiteEpiOFull) &&
                     mbar_wait(smem_addr(&sh.o_final[1]), n_final & 1, wctx, kSiteEpiOFull);
                ok = __all_sync(0xffffffffu, ok);
                ++n_final;
            }
            named_barrier_sync(1, 256);
            tc_fence_after_sync();
            // group t: columns [64 t, 64 t + 64) of both accumulators
            const float f0 = sh.inv_l[0][row], f1 = sh.inv_l[1][row] * lambda;
            float y[64];
            float sq = 0.f;
            if (x.nkv > 0) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t r0[32], r1[32];
                    tmem_ld_x32(tO + 64 * t + 32 * h, r0);
                    tmem_ld_x32(tO + 128 + 64 * t + 32 * h, r1);
                    tc_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const float v = f0 * __uint_as_float(r0[e]) - f1 * __uint_as_float(r1[e]);
                        y[32 * h + e] = v;
                        sq = fmaf(v, v, sq);
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 64; ++e) y[e] = 0.f;
            }
            sh.sum_sq[t][row] = sq;
            tc_fence_before_sync();
            named_barrier_sync(1, 256);             // both groups have read both accumulators: the next item's products may come
            float f = dp.out_scale;
            if (dp.weight) {                        // (uniform)
                f *= rsqrtf((sh.sum_sq[0][row] + sh.sum_sq[1][row]) * (1.f / 128.f) + dp.eps);
#pragma unroll
                for (int e = 0; e < 64; e += 4) {
                    const float4 w = *reinterpret_cast<const float4*>(&sh.weight[64 * t + e]);
                    y[e] *= f * w.x;
                    y[e + 1] *= f * w.y;
                    y[e + 2] *= f * w.z;
                    y[e + 3] *= f * w.w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 64; ++e) y[e] *= f;
            }
            if (ok) {
                // chunk t of the query tile's space (its last readers, the final score MMAs, are complete)
                const uint32_t chunk = sQ + buf * Cfg::kQBytes + t * kChunkBytes;
#pragma unroll
                for (int v = 0; v < 8; ++v)
                    st_shared_v4(chunk + row * 128 + (static_cast<uint32_t>(v ^ (row & 7)) << 4),
                                 pack_bf16x2(y[8 * v], y[8 * v + 1]), pack_bf16x2(y[8 * v + 2], y[8 * v + 3]),
                                 pack_bf16x2(y[8 * v + 4], y[8 * v + 5]), pack_bf16x2(y[8 * v + 6], y[8 * v + 7]));
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.o_staged[t]));
                if ((warp & 3) == 0 && lane == 0 && mbar_wait(smem_addr(&sh.o_staged[t]), it & 1, wctx, kSiteEpiStaged)) {
                    tma_store_4d(&tm_o, chunk, 64 * t, x.i0, x.hq, x.b);
                    tma_store_commit();
                    stored_buf = buf;
                }
                __syncwarp();
            }
        }
        if (stored_buf >= 0) tma_store_wait_read_all();     // the CTA's shared memory outlives the reads
    } else if (warp == 8) {
        // ============================================================ MMA issue, one thread for both maps
        setmaxnreg_dec<kPairRegsOther>();
        if (elect_one()) {
            constexpr uint32_t kIdescQK = make_idesc_bf16_f32(kTileM, kTileN, false, false);
            constexpr uint32_t kIdescPV = make_idesc_bf16_f32(kTileM, 128, false, true);
            constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);   // sbo, version, swizzle
            const uint32_t q_lo0 = ((sQ & 0x3FFFFu) >> 4) | (1u << 16);
            const uint32_t k_lo0 = ((sK & 0x3FFFFu) >> 4) | (1u << 16);
            const uint32_t v_lo0 = ((sV & 0x3FFFFu) >> 4) | ((static_cast<uint32_t>(kChunkBytes) >> 4) << 16);
            auto desc = [](uint32_t lo) -> uint64_t { return (static_cast<uint64_t>(kDescHi) << 32) | lo; };
            // k-step k of map t: chunk t, 32 bytes a step
            auto koff = [](int t, int k) -> uint32_t { return static_cast<uint32_t>((t * kChunkBytes + k * 32) >> 4); };
            bool ok = true;
            int n = 0, sv = 0, sk = 0;                // tiles so far, stage of V_j and of K_{j+1}
            uint32_t ph_v = 0, ph_k = 0, q_lo = 0;
            int nkv = 0;

            // One map's block of iteration j: PV_t(j), then QK_t(j+1); barriers to probe from inside the block as in the pair kernel.
            auto map_block = [&](auto tc, int j, uint32_t pre_first, uint32_t b0, uint32_t par0, uint32_t b1, uint32_t par1, uint32_t b2,
                                 uint32_t par2, uint32_t& probed) -> bool {
                constexpr int t = decltype(tc)::value;
                probed = 0u;
                const uint32_t tS = tmem_base + Cfg::kColS0 + 128 * t, tO = tmem_base + Cfg::kColO0 + 128 * t;
                const uint32_t vlo = v_lo0 + sv * (Cfg::kQBytes >> 4), klo = k_lo0 + sk * (Cfg::kQBytes >> 4);
                if (!pre_first && !mbar_wait(smem_addr(&sh.p_first[t]), n & 1, wctx, kSiteMmaPFull)) return false;
                tc_fence_after_sync();
                mma_ts(tO, tS + 0, desc(vlo + 0 * (2048 >> 4)), kIdescPV, j > 0 ? 1u : 0u);
                mma_ts(tO, tS + 8, desc(vlo + 1 * (2048 >> 4)), kIdescPV, 1u);
                mma_ts(tO, tS + 16, desc(vlo + 2 * (2048 >> 4)), kIdescPV, 1u);
                mma_ts(tO, tS + 24, desc(vlo + 3 * (2048 >> 4)), kIdescPV, 1u);
                const uint32_t rest = probe_mma_ts2(smem_addr(&sh.p_rest[t]), n & 1, tO, tS + 32, desc(vlo + 4 * (2048 >> 4)),
                                                    tS + 40, desc(vlo + 5 * (2048 >> 4)), kIdescPV);
                if (!rest && !mbar_wait(smem_addr(&sh.p_rest[t]), n & 1, wctx, kSiteMmaPFull)) return false;
                tc_fence_after_sync();
                mma_ts(tO, tS + 48, desc(vlo + 6 * (2048 >> 4)), kIdescPV, 1u);
                mma_ts(tO, tS + 56, desc(vlo + 7 * (2048 >> 4)), kIdescPV, 1u);
                if (j + 1 < nkv) {
                    mma_ss(tS, desc(q_lo + koff(t, 0)), desc(klo + koff(t, 0)), kIdescQK, 0u);
                    probed = probe3_mma_ss3(b0, par0, b1, par1, b2, par2, tS, desc(q_lo + koff(t, 1)), desc(klo + koff(t, 1)),
                                            desc(q_lo + koff(t, 2)), desc(klo + koff(t, 2)), desc(q_lo + koff(t, 3)), desc(klo + koff(t, 3)),
                                            kIdescQK);
                    tc_commit(smem_addr(&sh.s_full[t]));
                } else {
                    tc_commit(smem_addr(&sh.o_final[t]));
                }
                return true;
            };

            for (int it = 0; ok; ++it) {
                const int slot = it % Cfg::kItems, buf = it & 1;
                ok = mbar_wait(smem_addr(&sh.item_full[slot]), (it / Cfg::kItems) & 1, wctx, kSiteItem);
                if (!ok) break;
                const int index = sh.item[slot];
                if (index < 0) break;
                mbar_arrive(smem_addr(&sh.item_empty[slot]));
                nkv = decode(index).nkv;
                if (nkv == 0) continue;
                q_lo = q_lo0 + buf * (Cfg::kQBytes >> 4);
                // (the query tile's barrier has completed by the first probe and does not move before the item's end)
                const uint32_t bar_always = smem_addr(&sh.q_full[buf]), par_always = (it >> 1) & 1;
                ok = mbar_wait(bar_always, par_always, wctx, kSiteMmaQFull) && mbar_wait(smem_addr(&sh.k_full[sk]), ph_k, wctx, kSiteMmaKvFull);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int t = 0; t < 2; ++t) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        mma_ss(tmem_base + Cfg::kColS0 + 128 * t, desc(q_lo + koff(t, k)), desc(k_lo0 + sk * (Cfg::kQBytes >> 4) + koff(t, k)), kIdescQK, k > 0 ? 1u : 0u);
                    tc_commit(smem_addr(&sh.s_full[t]));
                }
                tc_commit(smem_addr(&sh.k_empty[sk]));
                if (++sk == NK) { sk = 0; ph_k ^= 1u; }
                uint32_t pre_p0 = 0u, pre_p1 = 0u, pre_v = 0u, pre_k = 0u;    // probes that succeeded: P_0 / P_1 first part, V_j, K_{j+1}
                for (int j = 0; j < nkv && ok; ++j, ++n) {
                    if (!pre_v) ok = mbar_wait(smem_addr(&sh.v_full[sv]), ph_v, wctx, kSiteMmaKvFull);
                    if (ok && j + 1 < nkv && !pre_k) ok = mbar_wait(smem_addr(&sh.k_full[sk]), ph_k, wctx, kSiteMmaKvFull);
                    if (!ok) break;
                    uint32_t probed;
                    ok = map_block(IntC<0>{}, j, pre_p0, smem_addr(&sh.p_first[1]), n & 1, bar_always, par_always, bar_always, par_always, probed);
                    if (!ok) break;
                    pre_p1 = probed & 1u;
                    int sv_n = sv + 1; uint32_t ph_v_n = ph_v; if (sv_n == NV) { sv_n = 0; ph_v_n ^= 1u; }
                    int sk_n = sk; uint32_t ph_k_n = ph_k;
                    const bool next = j + 1 < nkv, next_k = j + 2 < nkv;
                    if (next && ++sk_n == NK) { sk_n = 0; ph_k_n ^= 1u; }
                    ok = map_block(IntC<1>{}, j, pre_p1, next ? smem_addr(&sh.p_first[0]) : bar_always, next ? ((n + 1) & 1) : par_always,
                                   next ? smem_addr(&sh.v_full[sv_n]) : bar_always, next ? ph_v_n : par_always,
                                   next_k ? smem_addr(&sh.k_full[sk_n]) : bar_always, next_k ? ph_k_n : par_always, probed);
                    if (!ok) break;
                    pre_p0 = next ? (probed & 1u) : 0u;
                    pre_v = next ? ((probed >> 1) & 1u) : 0u;
                    pre_k = next_k ? ((probed >> 2) & 1u) : 0u;
                    tc_commit(smem_addr(&sh.v_empty[sv]));
                    if (next) tc_commit(smem_addr(&sh.k_empty[sk]));
                    sv = sv_n; ph_v = ph_v_n; sk = sk_n; ph_k = ph_k_n;
                }
            }
        }
    } else if (warp == 9) {
        // ============================================================ TMA loads
        setmaxnreg_dec<kPairRegsOther>();
        if (elect_one()) {
            auto load_tile = [&](uint32_t dst, const CUtensorMap* tm, uint64_t& full, int row0, int head, int b) {
                const uint32_t bar = smem_addr(&full);
                mbar_arrive_expect_tx(bar, Cfg::kQBytes);
#pragma unroll
                for (int cc = 0; cc < 2; ++cc) tma_load_4d(dst + cc * kChunkBytes, tm, bar, cc * kChunkCols, row0, head, b);
            };
            int n = 0;
            for (int it = 0;; ++it) {
                const int slot = it % Cfg::kItems, buf = it & 1;
                // a CTA's first item is its own number, the others are drawn; every CTA draws past the list once, and the last of all
                // draws (one per item in the end) puts the counter back
                unsigned int ticket = blockIdx.x;
                if (it > 0) {
                    const unsigned int drawn = atomicAdd(p.sched_counter, 1u);
                    if (drawn == static_cast<unsigned int>(n_items) - 1u) *p.sched_counter = 0u;
                    ticket = gridDim.x + drawn;
                }
                const bool more = ticket < static_cast<unsigned int>(n_items);
                if (!mbar_wait(smem_addr(&sh.item_empty[slot]), ((it / Cfg::kItems) & 1) ^ 1, wctx, kSiteItem)) break;
                if (more && !mbar_wait(smem_addr(&sh.q_empty[buf]), ((it >> 1) & 1) ^ 1, wctx, kSiteLoadQEmpty)) break;
                sh.item[slot] = more ? static_cast<int>(ticket) : -1;
                mbar_arrive(smem_addr(&sh.item_full[slot]));
                if (!more) break;
                const Item x = decode(static_cast<int>(ticket));
                const int kvh = x.hq / (p.Hq / p.Hkv);
                if (x.nkv > 0) load_tile(sQ + buf * Cfg::kQBytes, &tm_q, sh.q_full[buf], x.i0, x.hq, x.b);
                else mbar_arrive(smem_addr(&sh.q_full[buf]));           // keeps the barrier's phases in step with the items
                bool ok = true;
                for (int j = 0; j < x.nkv && ok; ++j, ++n) {
                    const int ks = n % NK, vs = n % NV;
                    ok = mbar_wait(smem_addr(&sh.k_empty[ks]), ((n / NK) & 1) ^ 1, wctx, kSiteLoadKvEmpty);
                    if (!ok) break;
                    load_tile(sK + ks * Cfg::kQBytes, &tm_k, sh.k_full[ks], j * kTileN, kvh, x.b);
                    if (p.debug_drop_v_load && n == 0) continue;
                    ok = mbar_wait(smem_addr(&sh.v_empty[vs]), ((n / NV) & 1) ^ 1, wctx, kSiteLoadKvEmpty);
                    if (!ok) break;
                    load_tile(sV + vs * Cfg::kQBytes, &tm_v, sh.v_full[vs], j * kTileN, kvh, x.b);
                }
                if (!ok) break;
            }
        }
    } else {
        setmaxnreg_dec<kPairRegsOther>();     // idle warps of the third warpgroup
    }

    // ---------------------------------------------------------------- teardown (all warps)
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem_base, 512);
}

}  // namespace fa
