// BF16 products grouped by expert and their weight gradients (the tiles, loads
// and stores of grouped.cu, one plane per operand, one product).
//
// A CTA pair's tile is 256 features by up to 512 columns, held as one or two
// halves of up to 256 columns, each with its own accumulator of the two that
// TMEM has.  The two halves share every load of the feature operand: with one
// half per tile the copies from L2 (32 KB per SM and K-block) were what a K-block
// took, whatever its columns.  At the start of a tile the MMAs run up to a ring's
// length ahead on the first half until the epilogue has read the second one of
// the tile before.
//
// A gradient's contraction runs over a group's rows, which end anywhere.  Where
// the rows are used as they stand (not as padded copies), the rows of a last
// K-block between the group's end and the next multiple of 16 belong to other
// groups; a warp of each CTA sets them to zero in shared memory, in both
// operands, before it passes the stage on to the MMAs (a zero times an infinity
// would not be zero).
//
// BF16 results take one accumulator over the whole contraction: the tensor cores
// truncate when they add to it, 9e-6 of a result over 8192 terms of either sign and
// 1.6e-4 over 32768 of one sign (2-norm), below the rounding to 8 bits (1.7e-3).  FP32
// results (SUM) read it every 256 terms, from two accumulators in turn while the MMAs
// go on in the other, and add in FP32 with rounding in registers: 2.3e-7 to 3.4e-7 for
// 512 to 32768 terms.  64 groups of 512 rows, 2048 x 4096: 418 us (368 without the sums,
// 333 for BF16 results).
//
// Bound by the copies from L2 into the SMs (41-45 bytes per clock and SM) where
// groups have hundreds of rows: 64 uneven groups of 512 rows on average, 2048 x 4096:
// 411 us (1.34 PFLOP/s), the rows' gradient 392, the weights' 455 (1.21; only 8
// K-blocks between two epilogues); by reading the weights with few: 32 groups
// of 4 to 64 rows 81-87 us (6.6-6.1 TB/s), one row of 4 groups 14 us.
#include <type_traits>

#include "grouped_tile.cuh"

namespace emu {

namespace {

template <int BC, bool PAIR>
struct Bf16Cfg {
    static constexpr int CTAS = PAIR ? 2 : 1;
    static constexpr int HALVES = BC > 256 ? 2 : 1, HCOLS = BC / HALVES;
    static constexpr int STEP = PAIR ? 32 : 16;                   // granularity of the MMA's N
    static constexpr int L_TILE = kLRows * kKB * 2;
    static constexpr int C_HALF = HCOLS / CTAS * kKB * 2;         // one half's rows in this CTA
    static constexpr int STAGE = L_TILE + HALVES * C_HALF;
    static constexpr int FIXED = 1024 + 512 + 2 * (kMaxGroups + 1) * 4;   // alignment, barriers, group tables
    static constexpr int FIT = (kSmemMax - FIXED) / STAGE;
    static constexpr int STAGES = FIT > 8 ? 8 : FIT;
    static constexpr int BAR_OFF = STAGES * STAGE;
    static constexpr int TAB_OFF = BAR_OFF + 512;
    static constexpr int SMEM = STAGES * STAGE + FIXED;
    static constexpr int EPI_WARPS = HALVES == 2 ? 16 : 8;
    static constexpr int THREADS = 64 + 32 * EPI_WARPS;
    static constexpr int WCOLS = HCOLS / (EPI_WARPS / 4);         // accumulator columns of one epilogue warp
    static_assert(WCOLS % 32 == 0, "columns of an epilogue warp");
};

struct HalfTile {
    int g, l0, c0, cols;       // features, columns of group g (its rows, or m)
    int n[2];                  // MMA columns of the halves (n[1] = 0: one half)
    int kl, kc, nk;            // first contraction element of the operands, length
};

template <int BC, bool PAIR, bool CMN>
__device__ __forceinline__ HalfTile half_tile(int t, const GroupedArgs &a, const int *starts, const int *tpre, int rank)
{
    using Cfg = Bf16Cfg<BC, PAIR>;
    constexpr int LT = kLRows * Cfg::CTAS;
    const int nlt = (a.L + LT - 1) / LT;
    HalfTile x;
    int local, n;
    if constexpr (CMN) {
        const int per = nlt * ((a.C + BC - 1) / BC);
        x.g = t / per;
        local = t - x.g * per;
        n = a.C;
    } else {
        x.g = find_group(tpre, a.G, t);
        local = t - tpre[x.g];
        n = starts[x.g + 1] - starts[x.g];
    }
    // column tiles of equal size; 8 of them walk the feature tiles together
    const int nct = (n + BC - 1) / BC;
    int ct, lt;
    tile_coords(local, nct, nlt, ct, lt);
    auto up = [](int v) { return (v + Cfg::STEP - 1) / Cfg::STEP * Cfg::STEP; };
    const int each = up((n + nct - 1) / nct);
    x.c0 = ct * each;
    x.cols = min(each, n - x.c0);
    x.n[0] = Cfg::HALVES == 1 || x.cols <= 256 ? up(x.cols) : up((x.cols + 1) / 2);
    x.n[1] = x.cols > x.n[0] ? up(x.cols - x.n[0]) : 0;
    x.l0 = lt * LT + rank * kLRows;
    if constexpr (CMN) {
        const int s = starts[x.g], p = (int)padded_start(s, x.g);
        x.kl = a.lpadded ? p : s;
        x.kc = a.padded ? p : s;
        x.nk = starts[x.g + 1] - s;
    } else {
        x.kl = x.kc = 0;
        x.nk = a.K;
    }
    return x;
}

// Sets rows [from, to) (at most 15) of `blocks` 64-column blocks of a stage to
// zero; a whole warp.
__device__ __forceinline__ void zero_rows_of(uint32_t at, int blocks, int from, int to)
{
    const uint32_t lane = lane_id();
    for (int b = 0; b < blocks; ++b)
        for (int r = from + (int)(lane >> 3); r < to; r += 4)
            st_shared_v4(at + (uint32_t)(b * 64 * kKB * 2 + r * 128) + (lane & 7u) * 16u, 0u, 0u, 0u, 0u);
}

// LMN / CMN: the feature / column operand is stored with its MN dimension
// contiguous (else with the contraction contiguous).  CMN is the gradient.  SUM:
// FP32 results, tiles of one half; else BF16.
template <int BC, bool PAIR, bool LMN, bool CMN, bool SUM>
__global__ void __launch_bounds__(Bf16Cfg<BC, PAIR>::THREADS + (CMN ? 32 : 0), 1)
grouped_bf16_kernel(const __grid_constant__ CUtensorMap tmL, const __grid_constant__ CUtensorMap tmC,
                    const __grid_constant__ CUtensorMap tmS, const GroupedArgs a)
{
    using Cfg = Bf16Cfg<BC, PAIR>;
    static_assert(!SUM || Cfg::HALVES == 1, "FP32 sums are held for one half");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *base_ptr = smem_raw + (base - raw);
    const uint32_t full0 = base + Cfg::BAR_OFF, empty0 = full0 + 8u * Cfg::STAGES;
    const uint32_t tfull0 = empty0 + 8u * Cfg::STAGES, tempty0 = tfull0 + 16u, done_bar = tempty0 + 16u, tail0 = done_bar + 24u;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(base_ptr + Cfg::BAR_OFF + 16 * Cfg::STAGES + 48);
    int *starts = reinterpret_cast<int *>(base_ptr + Cfg::TAB_OFF), *tpre = starts + a.G + 1;

    const int warp = uniform((int)threadIdx.x >> 5), lane = (int)lane_id();
    const int rank = PAIR ? (int)cluster_rank() : 0;
    uint32_t *flags = a.flags;
    // gradient: each CTA of the pair says on the leader's barrier that its part of
    // a stage is in order: its producer at once (the bytes are counted there too),
    // or for a ragged tail, counted on a barrier of its own, the warp that clears it

    if (threadIdx.x == 0) {
        for (int s = 0; s < Cfg::STAGES; ++s) { mbar_init(full0 + 8u * s, CMN ? 2 : 1); mbar_init(empty0 + 8u * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(tfull0 + 8u * b, 1); mbar_init(tempty0 + 8u * b, Cfg::EPI_WARPS * Cfg::CTAS); }
        mbar_init(done_bar, 1);
        for (int s = 0; s < Cfg::STAGES; ++s) mbar_init(tail0 + 8u * s, 1);
        fence_mbar_init();
        tma_prefetch_desc(&tmL);
        tma_prefetch_desc(&tmC);
    }
    if constexpr (PAIR) {
        __syncthreads();
        cluster_sync();                                   // both CTAs' barriers initialised
        if (warp == 1) tmem_alloc_pair(smem_u32((const void *)tmem_slot), 512);
    } else {
        if (warp == 1) { tmem_alloc(smem_u32((const void *)tmem_slot), 512); tmem_relinquish(); }
    }
    // the set-up above overlaps the end of the kernel before this one when it
    // is launched as its programmatic dependent
    griddep_wait();
    groups_and_flags(a, starts);
    constexpr int LT = kLRows * Cfg::CTAS;
    const int nlt = (a.L + LT - 1) / LT;
    int total;
    if constexpr (CMN) {
        total = a.G * nlt * ((a.C + BC - 1) / BC);
    } else {
        if (warp == 2) tile_prefix(starts, a.G, BC, nlt, tpre);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if constexpr (!CMN) total = uniform(tpre[a.G]);
    const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
    const int first = (int)blockIdx.x / Cfg::CTAS, step = (int)gridDim.x / Cfg::CTAS;
    auto tile = [&](int t) { return half_tile<BC, PAIR, CMN>(t, a, starts, tpre, rank); };
    // whether a tile's last K-block holds other groups' rows among its MMAs
    auto ragged = [&](int nk) { return CMN && !(a.lpadded && a.padded) && nk % 16 != 0; };

    if (warp == 0 && lane == 0) {
        // ---------------- TMA producer
        long issued = 0;
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (int t = first; t < total && ok; t += step) {
            const HalfTile x = tile(t);
            const int nkb = (x.nk + kKB - 1) / kKB;
            // per half: this CTA's rows (columns), as 64-row boxes, the last one also for a
            // part of them (rows past the tile's are not multiplied) unless that is 16
            // (32 groups of 40 rows, 2048 x 4096: 86 us against 90 with boxes of 16
            // for every rest; of 330: 140 and 148); a gradient's two 64-column blocks in one copy where they
            // start on whole blocks (also where the second is not needed)
            int row[2], big[2], small[2];
            uint32_t bytes = Cfg::L_TILE;
#pragma unroll
            for (int h = 0; h < Cfg::HALVES; ++h) {
                const int n = x.n[h] / Cfg::CTAS, rest = n % 64;
                row[h] = x.c0 + (h ? x.n[0] : 0) + rank * n;
                if (!CMN) row[h] += a.padded ? (int)padded_start(starts[x.g], x.g) : starts[x.g];
                big[h] = n / 64 + (rest > (CMN ? 0 : 16));
                small[h] = !CMN && rest == 16 ? 1 : 0;
                if (CMN && a.cwide && n > 0) big[h] = 2;
                bytes += (uint32_t)((big[h] * 64 + small[h] * 16) * kKB * 2);
            }
            int kl = x.kl, kc = x.kc;
            for (int kb = 0; kb < nkb; ++kb, kl += kKB, kc += kKB) {
                if (!(ok = mbar_wait(empty0 + 8u * s, ph ^ 1u, flags))) break;
                const uint32_t st = base + (uint32_t)(s * Cfg::STAGE), fb = full0 + 8u * s;
                uint32_t bar = PAIR ? peer_addr(fb, 0) : fb;
                if constexpr (CMN) {
                    if (kb == nkb - 1 && ragged(x.nk)) {
                        bar = peer_addr(tail0 + 8u * s, (uint32_t)rank);
                        mbar_arrive_expect_tx(tail0 + 8u * s, bytes);
                    } else if (rank == 0) {
                        mbar_arrive_expect_tx(fb, 2 * bytes);
                    } else {
                        mbar_arrive_peer(bar);
                    }
                } else {
                    if (rank == 0) mbar_arrive_expect_tx(fb, bytes * Cfg::CTAS);
                }
                if constexpr (LMN) {
                    // 128 features x 64 contraction rows (a weight matrix's rows, or token rows)
                    const int g = CMN ? 0 : x.g;
                    if (a.lwide) {
                        tma_load_5d<PAIR>(st, &tmL, bar, 0, kl, x.l0 >> 6, g, 0);
                    } else {
                        tma_load_5d<PAIR>(st, &tmL, bar, x.l0, kl, 0, g, 0);
                        tma_load_5d<PAIR>(st + Cfg::L_TILE / 2, &tmL, bar, x.l0 + 64, kl, 0, g, 0);
                    }
                } else {
                    tma_load_4d<PAIR>(st, &tmL, bar, kl, x.l0, x.g, 0);
                }
#pragma unroll
                for (int h = 0; h < Cfg::HALVES; ++h) {
                    const uint32_t dc = st + (uint32_t)(Cfg::L_TILE + h * Cfg::C_HALF);
                    if constexpr (CMN) {
                        if (a.cwide) {
                            if (big[h]) tma_load_5d<PAIR>(dc, &tmC, bar, 0, kc, row[h] >> 6, 0, 0);
                        } else {
                            for (int b = 0; b < big[h]; ++b)
                                tma_load_5d<PAIR>(dc + (uint32_t)(b * 64 * kKB * 2), &tmC, bar, row[h] + 64 * b, kc, 0, 0, 0);
                        }
                    } else {
                        for (int b = 0; b < big[h]; ++b)
                            tma_load_4d<PAIR>(dc + (uint32_t)(b * 64 * kKB * 2), &tmC, bar, kc, row[h] + 64 * b, 0, 0);
                        if (small[h])
                            tma_load_4d<PAIR>(dc + (uint32_t)(big[h] * 64 * kKB * 2), &tmS, bar, kc, row[h] + 64 * big[h], 0, 0);
                    }
                }
                ++issued;
                if (++s == Cfg::STAGES) { s = 0; ph ^= 1u; }
            }
        }
        if (!ok) {
            if (rank == 0) {
                drain_inflight(full0, Cfg::STAGES, issued, flags);
            } else {
                // the peer's copies complete on the leader's barriers, which it
                // cannot observe: give them 200 us before the CTA winds down
                const unsigned long long t0 = globaltimer_ns();
                while (globaltimer_ns() - t0 < 200000ull) {}
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ---------------- MMA issuer (a pair's leader)
        const uint32_t elected = elect_lane();
        uint32_t s = 0, ph = 0, uses = 0;             // uses: halves issued; half u is in accumulator u % 2
        bool ok = true;
        constexpr int kstepL = LMN ? 2048 : 32, kstepC = CMN ? 2048 : 32;
        constexpr uint64_t descL = group_desc(LMN ? 64u * kKB * 2u : 16u), descC = group_desc(CMN ? 64u * kKB * 2u : 16u);
        for (int t = first; t < total && ok; t += step) {
            const HalfTile x = tile(t);
            const int nk = uniform(x.nk), nkb = (nk + kKB - 1) / kKB;
            if (nkb == 0) continue;                   // an empty group: the epilogue writes zeros by itself
            const uint32_t n0 = (uint32_t)uniform(x.n[0]), n1 = Cfg::HALVES == 2 ? (uint32_t)uniform(x.n[1]) : 0u;
            constexpr uint32_t id0 = make_idesc_bf16(kLRows * Cfg::CTAS, 0) | (LMN ? 1u << 15 : 0u) | (CMN ? 1u << 16 : 0u);
            const uint32_t i0 = id0 | n0 >> 3 << 17, i1 = id0 | n1 >> 3 << 17;
            if constexpr (SUM) {
                for (int kb = 0; kb < nkb; ++kb) {
                    const uint32_t b = uses & 1u;
                    const int kc = kb % kChunkBlocks, left = nk - kb * kKB;
                    if (kc == 0) {                    // this accumulator's last sum has been read
                        if (!(ok = warp_wait(tempty0 + 8u * b, ((uses >> 1) & 1u) ^ 1u, flags))) break;
                        tc_fence_after();
                    }
                    if (!(ok = warp_wait(full0 + 8u * s, ph, flags))) break;
                    tc_fence_after();
                    const uint32_t st = (base + s * (uint32_t)Cfg::STAGE) >> 4;
#pragma unroll
                    for (int kk = 0; kk < kKB / 16; ++kk)
                        if (16 * kk < left)
                            mma_elected<PAIR>(elected, tmem + b * 256u, descL + (st + (uint32_t)((kk * kstepL) >> 4)),
                                              descC + (st + (uint32_t)((Cfg::L_TILE + kk * kstepC) >> 4)), i0, (kc | kk) != 0);
                    commit_elected<PAIR>(elected, empty0 + 8u * s);
                    if (kc == kChunkBlocks - 1 || kb == nkb - 1) { commit_elected<PAIR>(elected, tfull0 + 8u * b); ++uses; }
                    if (++s == Cfg::STAGES) { s = 0; ph ^= 1u; }
                }
                continue;
            }
            const uint32_t b0 = uses & 1u, b1 = b0 ^ 1u, d0 = tmem + b0 * 256u, d1 = tmem + b1 * 256u;
            const uint32_t p0 = ((uses >> 1) & 1u) ^ 1u, p1 = (((uses + 1u) >> 1) & 1u) ^ 1u;
            if (!(ok = warp_wait(tempty0 + 8u * b0, p0, flags))) break;
            tc_fence_after();
            // the MMAs of half h for the K-block in stage q
            auto issue = [&](int h, uint32_t q, int kb) {
                const uint32_t st = (base + q * (uint32_t)Cfg::STAGE) >> 4;
                // 16-wide steps that hold contraction elements (the rest of the stage may hold anything)
                const int left = nk - kb * kKB;
#pragma unroll
                for (int kk = 0; kk < kKB / 16; ++kk)
                    if (16 * kk < left)
                        mma_elected<PAIR>(elected, h ? d1 : d0, descL + (st + (uint32_t)((kk * kstepL) >> 4)),
                                          descC + (st + (uint32_t)((Cfg::L_TILE + h * Cfg::C_HALF + kk * kstepC) >> 4)),
                                          h ? i1 : i0, (kb | kk) != 0);
            };
            auto arrived = [&](uint32_t q, uint32_t parity) {
                if (!warp_wait(full0 + 8u * q, parity, flags)) return false;
                tc_fence_after();
                return true;
            };
            int ahead = 0;                            // K-blocks whose second half is still to be issued
            bool second = n1 == 0 || __all_sync(0xFFFFFFFFu, mbar_try_wait(tempty0 + 8u * b1, p1));
            if (second) tc_fence_after();
            uint32_t sa = s, pa = ph;                 // stage of the next K-block to look at
            for (int kb = 0; kb < nkb; ++kb) {
                if (!(ok = arrived(sa, pa))) break;
                issue(0, sa, kb);
                if (++sa == Cfg::STAGES) { sa = 0; pa ^= 1u; }
                ++ahead;
                if (!second) {
                    if (ahead < Cfg::STAGES && kb + 1 < nkb) continue;
                    if (!(ok = warp_wait(tempty0 + 8u * b1, p1, flags))) break;
                    tc_fence_after();
                    second = true;
                }
                for (; ahead > 0; --ahead) {          // in order: stage s holds K-block kb + 1 - ahead
                    if (n1) issue(1, s, kb + 1 - ahead);
                    commit_elected<PAIR>(elected, empty0 + 8u * s);
                    if (++s == Cfg::STAGES) { s = 0; ph ^= 1u; }
                }
            }
            if (ok) {
                commit_elected<PAIR>(elected, tfull0 + 8u * b0);
                if (n1) commit_elected<PAIR>(elected, tfull0 + 8u * b1);
            }
            uses += n1 ? 2u : 1u;
        }
        commit_elected<PAIR>(elected, done_bar);
        (void)mbar_wait(done_bar, 0, flags);
    } else if (CMN && warp == 2 + Cfg::EPI_WARPS) {
        // ---------------- clears this CTA's part of ragged tails
        uint32_t blocks = 0, phases = 0;              // phases: parity of every stage's tail barrier
        bool ok = true;
        for (int t = first; t < total && ok; t += step) {
            const HalfTile x = tile(t);
            const int nkb = (x.nk + kKB - 1) / kKB;
            blocks += (uint32_t)nkb;
            if (!ragged(x.nk)) continue;
            const uint32_t q = (blocks - 1u) % (uint32_t)Cfg::STAGES, st = base + q * (uint32_t)Cfg::STAGE;
            if (!(ok = warp_wait(tail0 + 8u * q, phases >> q & 1u, flags))) break;
            phases ^= 1u << q;
            const int from = x.nk - (nkb - 1) * kKB, to = (from + 15) / 16 * 16;
            zero_rows_of(st, 2, from, to);
            zero_rows_of(st + Cfg::L_TILE, (x.n[0] / Cfg::CTAS + 63) / 64, from, to);
            if (x.n[1]) zero_rows_of(st + Cfg::L_TILE + Cfg::C_HALF, (x.n[1] / Cfg::CTAS + 63) / 64, from, to);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0)
                asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];"
                             ::"r"(peer_addr(full0 + 8u * q, 0)) : "memory");
        }
    } else if (warp >= 2) {
        // ---------------- epilogue: this CTA's 128 features of each half; a warp
        // has a quarter of the lanes and WCOLS of the columns
        const int quarter = warp & 3, h0 = ((warp - 2) >> 2) * Cfg::WCOLS;
        constexpr int esize = SUM ? 4 : 2;
        const bool pairs_ok = (a.ldo & 1) == 0 && (a.strideo & 1) == 0 && (reinterpret_cast<uintptr_t>(a.out) & 3u) == 0;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)h0;
        if constexpr (!CMN) zero_rest(a, starts, (int)threadIdx.x - 64, 32 * Cfg::EPI_WARPS);
        auto release = [&](uint32_t bar) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR) mbar_arrive_peer(peer_addr(bar, 0));
                else mbar_arrive(bar);
            }
        };
        uint32_t uses = 0;
        bool ok = true;
        for (int t = first; t < total && ok; t += step) {
            const HalfTile x = tile(t);
            const int l = x.l0 + quarter * 32;
            if constexpr (SUM) {
                const int cols = x.cols - h0;             // columns from this warp's first on
                float acc[Cfg::WCOLS];
#pragma unroll
                for (int j = 0; j < Cfg::WCOLS; ++j) acc[j] = 0.0f;
                const int nch = (x.nk + kKChunk - 1) / kKChunk;
                for (int c = 0; c < nch; ++c, ++uses) {
                    const uint32_t b = uses & 1u;
                    if (!(ok = warp_wait(tfull0 + 8u * b, (uses >> 1) & 1u, flags))) break;
                    tc_fence_after();
#pragma unroll
                    for (int h = 0; h < Cfg::WCOLS; h += 16) {
                        if (h < cols) {
                            uint32_t v[16];
                            tmem_load16(lanes + b * 256u + (uint32_t)h, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) acc[h + j] = __fadd_rn(acc[h + j], __uint_as_float(v[j]));
                        }
                    }
                    release(tempty0 + 8u * b);
                }
                const int64_t row0 = (CMN ? 0 : (int64_t)starts[x.g]) + x.c0 + h0;
                float *o = static_cast<float *>(a.out) + row0 * a.ldo + (CMN ? x.g * a.strideo : 0);
                if (ok && l < a.L) {
#pragma unroll
                    for (int h = 0; h < Cfg::WCOLS; h += 32) {
                        float v[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = acc[h + j];
                        if (h < cols) store_columns(v, cols - h, o + (int64_t)h * a.ldo, a.ldo, l, a.L, true, false);
                    }
                }
            } else {
#pragma unroll 1
                for (int h = 0; h < (x.n[1] ? 2 : 1); ++h) {
                    const int c0 = (h ? x.n[0] : 0) + h0;                     // this warp's first column of the tile
                    const int cols = min(h ? x.cols - x.n[0] : x.n[0], x.cols) - h0;
                    const int64_t row0 = (CMN ? 0 : (int64_t)starts[x.g]) + x.c0 + c0;
                    char *o = static_cast<char *>(a.out) + (row0 * a.ldo + (CMN ? x.g * a.strideo : 0)) * esize;
                    const uint32_t b = uses & 1u;
                    // tcgen05.ld needs the whole warp, so a timeout in any lane ends the warp's work
                    if (x.nk > 0) {
                        if (!(ok = warp_wait(tfull0 + 8u * b, (uses >> 1) & 1u, flags))) break;
                        tc_fence_after();
                    }
#pragma unroll 1
                    for (int c = 0; c < Cfg::WCOLS; c += 32) {
                        if (c >= cols) break;
                        uint32_t v[32];
                        if (x.nk > 0) {
                            tmem_ld32(lanes + b * 256u + (uint32_t)c, v);
                            tmem_ld_wait();
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = 0u;
                        }
                        if (l < a.L)
                            store_columns(v, cols - c, o + (int64_t)c * a.ldo * esize, a.ldo, l, a.L, false, pairs_ok);
                    }
                    if (x.nk == 0) continue;
                    ++uses;
                    release(tempty0 + 8u * b);
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();               // the leader's MMAs are done with both CTAs
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        if constexpr (PAIR) tmem_dealloc_pair(tmem, 512);
        else tmem_dealloc(tmem, 512);
    }
}

template <int BC, bool PAIR, bool LMN, bool CMN, bool SUM>
cudaError_t run_bf16(const CUtensorMap &tl, const CUtensorMap &tc, const CUtensorMap &ts, const GroupedArgs &a, int64_t tiles,
                     cudaStream_t st)
{
    using Cfg = Bf16Cfg<BC, PAIR>;
    return launch_persistent<grouped_bf16_kernel<BC, PAIR, LMN, CMN, SUM>>(Cfg::SMEM, Cfg::THREADS + (CMN ? 32 : 0), Cfg::CTAS,
                                                                      tiles, st, tl, tc, ts, a);
}

// Columns of the tiles for G results of n columns x L features on average: pairs
// with 512 or 256, or single CTAs with 64, by waves times the clocks of a
// K-block (measured about 1050, 750 and 530).  64 uneven groups of 512 rows, 2048
// x 4096: 423 us with 512, 497 with 256; 32 groups of 256 rows: 120 and 109; of
// 64: 91 with 64.
int columns_for(int64_t n, int64_t L, int64_t G)
{
    auto waves = [](int64_t tiles, int64_t units) { return (tiles + units - 1) / units; };
    const int64_t sms = sm_count(), lp = (L + 255) / 256;
    const int64_t t512 = waves(G * ((n + 511) / 512) * lp, sms / 2) * (n > 256 ? 1050 : 820);
    const int64_t t256 = waves(G * ((n + 255) / 256) * lp, sms / 2) * 750;
    const int64_t t64 = waves(G * ((n + 63) / 64) * ((L + 127) / 128), sms) * 530;
    return t64 <= t256 && t64 <= t512 ? 64 : t256 <= t512 ? 256 : 512;
}

template <bool LMN>
cudaError_t product(const GroupedOperand &X, const GroupedOperand &W, GroupedArgs a, cudaStream_t st)
{
    CUtensorMap tl, tc, ts;
    const bool ok = LMN ? make_group_map(&tl, W.planes, a.L, a.K, a.G, 1, W.ld, W.stride, W.plane, kKB, &a.lwide)
                        : make_group_map(&tl, W.planes, a.K, a.L, a.G, 1, W.ld, W.stride, W.plane, kLRows);
    if (!ok || !make_group_map(&tc, X.planes, a.K, X.rows, 1, 1, X.ld, 0, X.plane, 64) ||
        !make_group_map(&ts, X.planes, a.K, X.rows, 1, 1, X.ld, 0, X.plane, 16))
        return cudaErrorInvalidValue;
    const int bc = columns_for((a.rows + a.G - 1) / a.G, a.L, a.G);
    auto run = [&](auto sum) {
        constexpr bool SUM = decltype(sum)::value;
        if constexpr (!SUM)
            if (bc == 512) return run_bf16<512, true, LMN, false, false>(tl, tc, ts, a, max_tiles(a.rows, a.G, a.L, 512, 2), st);
        if (bc >= 256) return run_bf16<256, true, LMN, false, SUM>(tl, tc, ts, a, max_tiles(a.rows, a.G, a.L, 256, 2), st);
        return run_bf16<64, false, LMN, false, SUM>(tl, tc, ts, a, max_tiles(a.rows, a.G, a.L, 64, 1), st);
    };
    return a.out_f32 ? run(std::true_type{}) : run(std::false_type{});
}

}  // namespace

cudaError_t launch_bf16_product(bool trans, const GroupedOperand &X, const GroupedOperand &W, const GroupedArgs &a, cudaStream_t st)
{
    return trans ? product<false>(X, W, a, st) : product<true>(X, W, a, st);
}

cudaError_t launch_bf16_gradient(const GroupedOperand &A, const GroupedOperand &B, GroupedArgs a, cudaStream_t st)
{
    CUtensorMap tl, tc;
    if (!make_group_map(&tl, B.planes, a.L, B.rows, 1, 1, B.ld, 0, B.plane, kKB, &a.lwide) ||
        !make_group_map(&tc, A.planes, a.C, A.rows, 1, 1, A.ld, 0, A.plane, kKB, &a.cwide, a.C <= 128 ? 128 : 256))
        return cudaErrorInvalidValue;
    a.lpadded = B.padded;
    a.padded = A.padded;
    // (512 columns: 547 us for 64 groups of 512 rows, 2048 x 4096, against 495; a
    // short contraction does not hide the reading of two halves)
    const int64_t tiles = (int64_t)a.G * ((a.L + 255) / 256) * ((a.C + 255) / 256);
    return a.out_f32 ? run_bf16<256, true, true, true, true>(tl, tc, tc, a, tiles, st)
                     : run_bf16<256, true, true, true, false>(tl, tc, tc, a, tiles, st);
}

}  // namespace emu
