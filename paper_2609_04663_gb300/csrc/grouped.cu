// FP32 matrix products grouped by expert and their weight gradients, on tcgen05
// BF16 MMAs with FP32 accumulators in tensor memory (BF16 operands:
// grouped_bf16.cu; few rows for each group: grouped_fused.cu).
//
//   product:   Y[r, n]    = sum_k X[r, k] W_g[k, n]   for the rows r of group g
//   gradient:  D_g[m, n]  = sum over the rows r of group g of A[r, m] B[r, n]
//
// Operands are sets of three BF16 planes (Eq. (fp32split)); the six products of
// Eq. (fp32six) are issued from one stage.
//
// Both forms compute tiles of the TRANSPOSED result: the contiguous output
// dimension n (the weights' features) lies on the 128 MMA rows = TMEM lanes,
// and the other dimension (a group's rows, or m) on the up to 256 MMA columns.
// A group's ragged row count then only changes the MMA's N, which goes in
// steps of 16 (32 on CTA pairs), so a group of 300 rows costs 320 columns and
// not 384 or 512 rows; a few rows for each expert cost little more than reading
// the weights; and an accumulator column is 32 consecutive output elements
// per warp, stored without staging and with any row pitch.
//
// The grid is persistent: one CTA (or CTA pair) per SM (pair) walks the tiles
// of all groups, which every CTA derives from `ends` on the device.  Warp 0
// issues TMA loads, warp 1 the MMAs, warps 2-9 read TMEM and store.  Every
// wait is bounded (EMU_FLAG_TIMEOUT).
//
// The tensor cores truncate when they add to an FP32
// accumulator, a bias of about 1.8e-8 of the result per 16-wide step; six
// products over K = 256 in one accumulator came out at 1.7e-6 (2-norm).  So
// the leading product A0B0 has an accumulator of its own that is read every
// 256 elements of K (the K-chunk of Section 6.1) and added, correctly rounded,
// to a running FP32 sum in registers; the five products with i + j > 0, 2^-8
// of it and less, share a second accumulator over all of K.  While the
// epilogue warps read a chunk's leading sum, the MMAs of the five others of
// the next K-block run.
//
// Bound by the tensor pipe (92 % active): 16 groups of 1024 rows, 2048 x 2048:
// product 435 us (1.90 PFLOP/s executed, six products), gradients 434 and 420 us; 7
// groups of 219 rows, 333 x 517, 12 to 17 us each, by latency.
#include "grouped_tile.cuh"

namespace emu {

namespace {

constexpr int S = 3;

// LMN / CMN: the feature / column operand is stored with its MN dimension
// contiguous (else with the contraction contiguous).  CMN is the gradient.
template <int BC, bool PAIR, bool LMN, bool CMN>
__global__ void __launch_bounds__(64 + 32 * kEpiWarps, 1)
grouped_kernel(const __grid_constant__ CUtensorMap tmL, const __grid_constant__ CUtensorMap tmC,
               const __grid_constant__ CUtensorMap tmS, const GroupedArgs a)
{
    using Cfg = GroupedCfg<S, BC, PAIR>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *base_ptr = smem_raw + (base - raw);
    const uint32_t full0 = base + Cfg::BAR_OFF, empty0 = full0 + 8u * Cfg::STAGES;
    // tfull[0], tempty[0]: the leading accumulator (per chunk); tempty[1]: the
    // other one (per tile)
    const uint32_t tfull0 = empty0 + 8u * Cfg::STAGES, tempty0 = tfull0 + 16u, done_bar = tempty0 + 16u;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(base_ptr + Cfg::BAR_OFF + 16 * Cfg::STAGES + 48);
    int *starts = reinterpret_cast<int *>(base_ptr + Cfg::TAB_OFF), *tpre = starts + a.G + 1;

    const int warp = uniform((int)threadIdx.x >> 5), lane = (int)lane_id();
    const int rank = PAIR ? (int)cluster_rank() : 0;
    uint32_t *flags = a.flags;

    if (threadIdx.x == 0) {
        for (int s = 0; s < Cfg::STAGES; ++s) { mbar_init(full0 + 8u * s, 1); mbar_init(empty0 + 8u * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(tfull0 + 8u * b, 1); mbar_init(tempty0 + 8u * b, kEpiWarps * Cfg::CTAS); }
        mbar_init(done_bar, 1);
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

    if (warp == 0 && lane == 0) {
        // ---------------- TMA producer
        long issued = 0;
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (int t = first; t < total && ok; t += step) {
            const Tile x = tile_at<S, BC, PAIR, LMN, CMN>(t, a, starts, tpre, rank);
            const int nkb = (x.nk + kKB - 1) / kKB, crows = x.csz / Cfg::CTAS, cfirst = rank * crows;
            // 64-row (or 64-column) boxes; a short rest in boxes of 16 rows
            const int rest = crows % 64, cbig = crows / 64 + (CMN ? rest > 0 : rest > 32), csmall = CMN || rest > 32 ? 0 : rest / 16;
            // two blocks of 64 columns in one copy, also where the second is not needed
            const bool ctwo = CMN && a.cwide != 0;
            const uint32_t bytes = (uint32_t)(S * (Cfg::L_TILE + ((ctwo ? 2 : cbig) * 64 + csmall * 16) * kKB * 2)) * Cfg::CTAS;
            const int crow0 = CMN ? x.c0 + cfirst
                                  : (a.padded ? (int)padded_start(starts[x.g], x.g) : starts[x.g]) + x.c0 + cfirst;
            int k = x.k0;
            for (int kb = 0; kb < nkb; ++kb, k += kKB) {
                if (!(ok = mbar_wait(empty0 + 8u * s, ph ^ 1u, flags))) break;
                const uint32_t st = base + (uint32_t)(s * Cfg::STAGE), fb = full0 + 8u * s;
                const uint32_t bar = PAIR ? peer_addr(fb, 0) : fb;
                if (rank == 0) mbar_arrive_expect_tx(fb, bytes);
#pragma unroll
                for (int r = 0; r < S; ++r) {
                    const uint32_t dl = st + (uint32_t)(r * Cfg::L_TILE);
                    if constexpr (LMN) {
                        // 128 features x 64 contraction rows (a weight matrix's rows, or token rows)
                        const int g = CMN ? 0 : x.g;
                        if (a.lwide) {
                            tma_load_5d<PAIR>(dl, &tmL, bar, 0, k, x.l0 >> 6, g, r);
                        } else {
                            tma_load_5d<PAIR>(dl, &tmL, bar, x.l0, k, 0, g, r);
                            tma_load_5d<PAIR>(dl + Cfg::L_TILE / 2, &tmL, bar, x.l0 + 64, k, 0, g, r);
                        }
                    } else {
                        tma_load_4d<PAIR>(dl, &tmL, bar, k, x.l0, x.g, r);
                    }
                    const uint32_t dc = st + (uint32_t)(S * Cfg::L_TILE + r * Cfg::C_TILE);
                    if constexpr (CMN) {
                        if (ctwo) {
                            tma_load_5d<PAIR>(dc, &tmC, bar, 0, k, crow0 >> 6, 0, r);
                        } else {
                            for (int b = 0; b < cbig; ++b)
                                tma_load_5d<PAIR>(dc + (uint32_t)(b * 64 * kKB * 2), &tmC, bar, crow0 + 64 * b, k, 0, 0, r);
                        }
                    } else {
                        for (int b = 0; b < cbig; ++b)
                            tma_load_4d<PAIR>(dc + (uint32_t)(b * 64 * kKB * 2), &tmC, bar, k, crow0 + 64 * b, 0, r);
                        for (int b = 0; b < csmall; ++b)
                            tma_load_4d<PAIR>(dc + (uint32_t)((cbig * 64 + b * 16) * kKB * 2), &tmS, bar, k,
                                              crow0 + 64 * cbig + 16 * b, 0, r);
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
        uint32_t s = 0, ph = 0, it = 0, cph = 0;      // it: tiles with a contraction, cph: chunks issued
        bool ok = true;
        constexpr int kstepL = LMN ? 2048 : 32, kstepC = CMN ? 2048 : 32;
        constexpr uint64_t descL = group_desc(LMN ? 64u * kKB * 2u : 16u), descC = group_desc(CMN ? 64u * kKB * 2u : 16u);
        for (int t = first; t < total && ok; t += step) {
            const Tile x = tile_at<S, BC, PAIR, LMN, CMN>(t, a, starts, tpre, rank);
            const int nk = uniform(x.nk), nkb = (nk + kKB - 1) / kKB;
            if (nkb == 0) continue;                   // an empty group: the epilogue writes zeros by itself
            const uint32_t csz = (uint32_t)uniform(x.csz);
            const uint32_t idesc = make_idesc_bf16(kLRows * Cfg::CTAS, 0) | csz >> 3 << 17 | (LMN ? 1u << 15 : 0u) |
                                   (CMN ? 1u << 16 : 0u);
            const uint32_t d = tmem, d2 = tmem + 256u;
            if (!(ok = warp_wait(tempty0 + 8u, (it & 1u) ^ 1u, flags))) break;
            ++it;
            tc_fence_after();
            for (int kb = 0; kb < nkb; ++kb) {
                if (!(ok = warp_wait(full0 + 8u * s, ph, flags))) break;
                tc_fence_after();
                const uint32_t st = (base + s * (uint32_t)Cfg::STAGE) >> 4;
                // 16-wide steps that hold contraction elements (the rest of the stage may hold anything)
                const int left = nk - kb * kKB;
                auto mma = [&](uint32_t acc, int il, int ic, int kk, bool add) {
                    mma_elected<PAIR>(elected, acc, descL + (st + (uint32_t)((il * Cfg::L_TILE + kk * kstepL) >> 4)),
                                      descC + (st + (uint32_t)((S * Cfg::L_TILE + ic * Cfg::C_TILE + kk * kstepC) >> 4)), idesc,
                                      add);
                };
                const int kc = kb % kChunkBlocks;
#pragma unroll
                for (int kk = 0; kk < kKB / 16; ++kk) {
                    if (16 * kk < left) {
                        mma(d2, 1, 1, kk, (kb | kk) != 0);
                        mma(d2, 1, 0, kk, true);
                        mma(d2, 2, 0, kk, true);
                        mma(d2, 0, 2, kk, true);
                        mma(d2, 0, 1, kk, true);
                    }
                }
                if (kc == 0) {                    // the last chunk's leading sum has been read
                    if (!(ok = warp_wait(tempty0, (cph & 1u) ^ 1u, flags))) break;
                    tc_fence_after();
                }
#pragma unroll
                for (int kk = 0; kk < kKB / 16; ++kk)
                    if (16 * kk < left) mma(d, 0, 0, kk, (kc | kk) != 0);
                commit_elected<PAIR>(elected, empty0 + 8u * s);
                if (kc == kChunkBlocks - 1 || kb == nkb - 1) { commit_elected<PAIR>(elected, tfull0); ++cph; }
                if (++s == Cfg::STAGES) { s = 0; ph ^= 1u; }
            }
        }
        commit_elected<PAIR>(elected, done_bar);
        (void)mbar_wait(done_bar, 0, flags);
    } else if (warp >= 2) {
        // ---------------- epilogue: this CTA's 128 features of each tile; a warp
        // has a quarter of the lanes and half of the columns
        const int quarter = warp & 3, h0 = ((warp - 2) >> 2) * Cfg::HALF;
        const int esize = a.out_f32 ? 4 : 2;
        const bool pairs_ok = (a.ldo & 1) == 0 && (a.strideo & 1) == 0 && (reinterpret_cast<uintptr_t>(a.out) & 3u) == 0;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)h0;
        if constexpr (!CMN) {
            zero_rest(a, starts, (int)threadIdx.x - 64, 32 * kEpiWarps);
        }
        auto release = [&](uint32_t bar) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR) mbar_arrive_peer(peer_addr(bar, 0));
                else mbar_arrive(bar);
            }
        };
        int it = 0;
        uint32_t cph = 0;
        bool ok = true;
        for (int t = first; t < total && ok; t += step, ++it) {
            const Tile x = tile_at<S, BC, PAIR, LMN, CMN>(t, a, starts, tpre, rank);
            const int l = x.l0 + quarter * 32;
            const int cols = x.cols - h0;             // columns from this warp's first on
            const int64_t row0 = (CMN ? 0 : (int64_t)starts[x.g]) + x.c0 + h0;
            char *o = static_cast<char *>(a.out) + (row0 * a.ldo + (CMN ? x.g * a.strideo : 0)) * esize;
            auto store32 = [&](const float (&v)[32], int c) {
                if (l < a.L && c < cols)
                    store_columns(v, cols - c, o + (int64_t)c * a.ldo * esize, a.ldo, l, a.L, a.out_f32 != 0, pairs_ok);
            };
            if (x.nk == 0) {
                --it;
                const float z[32] = {};
                for (int c = 0; c < Cfg::HALF; c += 32) store32(z, c);
                continue;
            }
            // tcgen05.ld needs the whole warp, so a timeout in any lane ends the warp's work
            float acc[Cfg::HALF];
#pragma unroll
            for (int j = 0; j < Cfg::HALF; ++j) acc[j] = 0.0f;
            const int nch = (x.nk + kKChunk - 1) / kKChunk;
            for (int c = 0; c <= nch; ++c) {      // the chunks' leading sums, then the other products
                if (c < nch) {
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(tfull0, cph & 1u, flags));
                    if (!ok) break;
                    ++cph;
                    tc_fence_after();
                }
#pragma unroll
                for (int h = 0; h < Cfg::HALF; h += 16) {
                    if (h < cols) {
                        uint32_t v[16];
                        tmem_load16(lanes + (uint32_t)(c < nch ? h : 256 + h), v);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[h + j] = __fadd_rn(acc[h + j], __uint_as_float(v[j]));
                    }
                }
                release(c < nch ? tempty0 : tempty0 + 8u);
            }
            if (ok) {
#pragma unroll
                for (int h = 0; h < Cfg::HALF; h += 32) {
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = acc[h + j];
                    store32(v, h);
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

template <int BC, bool PAIR, bool LMN, bool CMN>
cudaError_t run_grouped(const CUtensorMap &tl, const CUtensorMap &tc, const CUtensorMap &ts, const GroupedArgs &a,
                        int64_t tiles, cudaStream_t st)
{
    using Cfg = GroupedCfg<S, BC, PAIR>;
    return launch_persistent<grouped_kernel<BC, PAIR, LMN, CMN>>(Cfg::SMEM, Cfg::THREADS, Cfg::CTAS, tiles, st, tl, tc, ts, a);
}

// Whether 256 x 256 tiles on CTA pairs are estimated faster than 128 x 64 tiles
// for G results of n columns x L features.  A K-block takes a pair 12 clocks
// per MMA column (the products' time) and a single CTA about 1000 (a 128-row
// MMA no less than 41 clocks, whatever its columns): the pair is a quarter
// faster per SM where the tiles fill the GPU, and 4 times longer where one
// wave holds them all (7 groups of 219 rows, 333 x 517: product 23 us on pairs).
bool pairs_win(int64_t n, int64_t L, int64_t G)
{
    auto waves = [](int64_t tiles, int64_t units) { return (tiles + units - 1) / units; };
    const int64_t nct = (n + 255) / 256, cols = (n + nct - 1) / nct, sms = sm_count();
    const int64_t pair = waves(G * nct * ((L + 255) / 256), sms / 2) * 12 * (cols < 128 ? 128 : cols);
    const int64_t one = waves(G * ((n + 63) / 64) * ((L + 127) / 128), sms) * 1000;
    return pair <= one;
}

template <bool LMN>
cudaError_t product(const GroupedOperand &X, const GroupedOperand &W, GroupedArgs a, cudaStream_t st)
{
    CUtensorMap tl, tc, ts;
    const bool ok = LMN ? make_group_map(&tl, W.planes, a.L, a.K, a.G, S, W.ld, W.stride, W.plane, kKB, &a.lwide)
                        : make_group_map(&tl, W.planes, a.K, a.L, a.G, S, W.ld, W.stride, W.plane, kLRows);
    if (!ok || !make_group_map(&tc, X.planes, a.K, X.rows, 1, S, X.ld, 0, X.plane, 64) ||
        !make_group_map(&ts, X.planes, a.K, X.rows, 1, S, X.ld, 0, X.plane, 16))
        return cudaErrorInvalidValue;
    const int64_t each = (a.rows + a.G - 1) / a.G;    // rows of a group on average
    if (pairs_win(each, a.L, a.G))
        return run_grouped<256, true, LMN, false>(tl, tc, ts, a, max_tiles(a.rows, a.G, a.L, 256, 2), st);
    return run_grouped<64, false, LMN, false>(tl, tc, ts, a, max_tiles(a.rows, a.G, a.L, 64, 1), st);
}

cudaError_t gradient(const GroupedOperand &A, const GroupedOperand &B, GroupedArgs a, cudaStream_t st)
{
    CUtensorMap tl, tc;
    if (!make_group_map(&tl, B.planes, a.L, B.rows, 1, S, B.ld, 0, B.plane, kKB, &a.lwide) ||
        !make_group_map(&tc, A.planes, a.C, A.rows, 1, S, A.ld, 0, A.plane, kKB, &a.cwide, a.C <= 128 ? 128 : 256))
        return cudaErrorInvalidValue;
    if (pairs_win(a.C, a.L, a.G))
        return run_grouped<256, true, true, true>(tl, tc, tc, a, (int64_t)a.G * ((a.L + 255) / 256) * ((a.C + 255) / 256), st);
    // (a 64-column tile is one block: the map must not load two)
    if (!make_group_map(&tc, A.planes, a.C, A.rows, 1, S, A.ld, 0, A.plane, kKB, &a.cwide, 1 << 30)) return cudaErrorInvalidValue;
    return run_grouped<64, false, true, true>(tl, tc, tc, a, (int64_t)a.G * ((a.L + 127) / 128) * ((a.C + 63) / 64), st);
}

}  // namespace

cudaError_t launch_grouped_product(int nslices, bool trans, int64_t G, int64_t rows, int64_t N, int64_t K,
                                   const GroupedOperand &X, const GroupedOperand &W, const int32_t *ends, void *Y,
                                   bool y_f32, int64_t ldy, uint32_t *flags, bool own_flags, cudaStream_t st)
{
    GroupedArgs a = {};
    a.ends = ends; a.G = (int)G; a.rows = (int)rows; a.L = (int)N; a.K = (int)K; a.padded = X.padded ? 1 : 0;
    a.out = Y; a.ldo = ldy; a.out_f32 = y_f32 ? 1 : 0; a.flags = flags; a.own_flags = own_flags ? 1 : 0;
    if (nslices == 1) return launch_bf16_product(trans, X, W, a, st);
    return trans ? product<false>(X, W, a, st) : product<true>(X, W, a, st);
}

cudaError_t launch_grouped_gradient(int nslices, int64_t G, int64_t rows, int64_t M, int64_t N, const GroupedOperand &A,
                                    const GroupedOperand &B, const int32_t *ends, void *D, bool d_f32, int64_t ldd,
                                    int64_t strided, uint32_t *flags, bool own_flags, cudaStream_t st)
{
    GroupedArgs a = {};
    a.ends = ends; a.G = (int)G; a.rows = (int)rows; a.L = (int)N; a.C = (int)M;
    a.out = D; a.ldo = ldd; a.strideo = strided; a.out_f32 = d_f32 ? 1 : 0; a.flags = flags;
    a.own_flags = own_flags ? 1 : 0;
    return nslices == 1 ? launch_bf16_gradient(A, B, a, st) : gradient(A, B, a, st);
}

}  // namespace emu
