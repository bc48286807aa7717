// Products in 8-bit integers for many rows: tiles of 256 features by up to 256 columns on
// pairs of SMs (i8_tile.cuh has the arithmetic).  The token rows are turned into FP16 once,
// gathered, by a small kernel before, whose result is waited for only by the warps that read it.
//
// A tile's columns are two halves with accumulators of their own, of three that tensor memory holds
// beside two stages of weights; a sum's first half is read while the second one is still being multiplied.
// In a pair's CTA warps 0-7 read accumulators and store, 8-15 convert weights, 16 brings weights by TMA, 17
// (of the first CTA) issues the MMAs, 18 brings the rows.
//
// 16384 x 8192 x 4096 takes 630 us, 1.75 PFLOP/s, 61 of them before the products (bytes in, FP16 out, by HBM); the
// tensor pipe is 84 % active there at 8192 rows.  8192 rows over 32 experts, 2048 -> 4096: 120 us, tensor pipe 59 %
// active: groups' last tiles are not full, and each tile has only 16 stages between two read-outs.
// Tried: rows turned into FP16 by these CTAs (599 ns for 64 codes of 256 columns, 404-448 from FP16), two accumulators
// instead of three (742 us against 682), one converting group of four warps (353 ns against 253 with 16 columns).
#include <type_traits>

#include "i8_tile.cuh"

namespace emu {

namespace {

struct PairCfg {
    static constexpr int HC = 128, STEP = 32;                             // columns of a half, granularity of the MMA's N
    static constexpr int SLOTS = 3;                                       // accumulators of HC columns
    static constexpr int A0 = SLOTS * HC, NA = (512 - A0) / 64;           // A stages: 64 TMEM columns of 128 codes
    static constexpr int C_HALF = HC / 2 * kKB * 2, C_BLOCK = 2 * C_HALF; // this CTA's rows of one K-block
    static constexpr int C_STAGE = 2 * C_BLOCK, NC = 4;
    static constexpr int W_STAGE = kLRows * kWK, NW = 4;
    static constexpr int CONV = kDrainWarps, TMAW = CONV + kConvertWarps, MMA = TMAW + 1, TMAC = TMAW + 2;
    static constexpr int THREADS = 32 * (TMAW + 4);
    static constexpr int WC = HC / 2;                                     // columns of a half that a draining warp reads
    static constexpr int W_OFF = NC * C_STAGE, BAR_OFF = W_OFF + NW * W_STAGE, TAB_OFF = BAR_OFF + 512;
    static constexpr int SMEM = TAB_OFF + 2 * (kMaxGroups + 1) * 4 + 1024;
    static_assert(SMEM <= kSmemMax, "shared memory per CTA");
    static_assert(NA >= 2 && NA <= NC && C_HALF == 8192, "stages");
};

constexpr uint32_t kNoRow = 0xFFFFFFFFu;              // a NaN that no scale is handed over as

struct PairArgs {
    I8Product p;
    const float *xs;                  // [rows] the rows' scales in group order (the bits kNoRow: no such row)
    int copied;                       // the launch before also writes the weights that are read
};

__device__ __forceinline__ I8Tile pair_tile(int t, const I8Product &p, const int *starts, const int *tpre, int rank)
{
    using Cfg = PairCfg;
    const int nlt = (p.N + 2 * kLRows - 1) / (2 * kLRows);
    I8Tile x;
    x.g = find_group(tpre, p.G, t);
    const int local = t - tpre[x.g], n = starts[x.g + 1] - starts[x.g];
    const int nct = (n + 255) / 256;
    int ct = 0, lt = local, each = n;                 // (divisions are most of this function: none for one column of tiles)
    if (nct > 1) {
        tile_coords(local, nct, nlt, ct, lt);
        each = (n + nct - 1) / nct;
    }
    auto step = [](int v) { return (v + Cfg::STEP - 1) / Cfg::STEP * Cfg::STEP; };
    each = step(each);
    x.c0 = ct * each;
    x.cols = min(each, n - x.c0);
    x.n[0] = x.cols <= Cfg::HC ? step(x.cols) : step((x.cols + 1) / 2);
    x.n[1] = x.cols > x.n[0] ? step(x.cols - x.n[0]) : 0;
    x.l0 = lt * 2 * kLRows + rank * kLRows;
    x.k0 = 0;
    x.nk = p.K;
    return x;
}

// The registers' split: 640 threads with 96 each at launch.
constexpr int kSplitRegisters = 128 * (2 * 168 + 2 * 48 + 40);

__global__ void __launch_bounds__(PairCfg::THREADS, 1)
i8_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmC,
               const __grid_constant__ CUtensorMap tmS, const PairArgs a)
{
    using Cfg = PairCfg;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *base_ptr = smem_raw + (base - raw);
    const uint32_t cfull0 = base + Cfg::BAR_OFF, used0 = cfull0 + 8u * Cfg::NC;
    const uint32_t wfull0 = used0 + 8u * Cfg::NC, wempty0 = wfull0 + 8u * Cfg::NW;
    const uint32_t afull0 = wempty0 + 8u * Cfg::NW, tfull0 = afull0 + 8u * Cfg::NA, tempty0 = tfull0 + 8u * Cfg::SLOTS, done_bar = tempty0 + 8u * Cfg::SLOTS;
    static_assert(8 * (2 * (Cfg::NC + Cfg::NW + Cfg::SLOTS) + Cfg::NA + 1) <= 496, "barriers");
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(base_ptr + Cfg::BAR_OFF + 496);
    int *starts = reinterpret_cast<int *>(base_ptr + Cfg::TAB_OFF), *tpre = starts + a.p.G + 1;
    const int warp = uniform((int)threadIdx.x >> 5), lane = (int)lane_id();
    const int rank = (int)cluster_rank();
    uint32_t *flags = a.p.flags;

    if (threadIdx.x == 0) {
        for (int s = 0; s < Cfg::NC; ++s) { mbar_init(cfull0 + 8u * s, 1); mbar_init(used0 + 8u * s, 1); }
        for (int s = 0; s < Cfg::NW; ++s) { mbar_init(wfull0 + 8u * s, 1); mbar_init(wempty0 + 8u * s, kConvertWarps); }
        for (int s = 0; s < Cfg::NA; ++s) mbar_init(afull0 + 8u * s, 2 * kConvertWarps);
        for (int s = 0; s < Cfg::SLOTS; ++s) { mbar_init(tfull0 + 8u * s, 1); mbar_init(tempty0 + 8u * s, 2 * kDrainWarps); }
        mbar_init(done_bar, 1);
        fence_mbar_init();
        tma_prefetch_desc(&tmW);
        tma_prefetch_desc(&tmC);
        tma_prefetch_desc(&tmS);
    }
    __syncthreads();
    cluster_sync();                                   // both CTAs' barriers initialised
    if (warp == Cfg::MMA) tmem_alloc_pair(smem_u32((const void *)tmem_slot), 512);
    // launched as the programmatic dependent of the kernel that turns the rows into FP16, which
    // itself started after everything before it: only what that kernel writes has to be waited for
    if (a.p.ends) {
        (void)load_groups(a.p.ends, a.p.G, a.p.rows, starts);
    } else if (threadIdx.x == 0) {
        starts[0] = 0;
        starts[1] = a.p.rows;
    }
    __syncthreads();
    if (warp == 0) tile_prefix(starts, a.p.G, 256, (a.p.N + 2 * kLRows - 1) / (2 * kLRows), tpre);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const int total = uniform(tpre[a.p.G]);
    const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
    const int first = (int)blockIdx.x / 2, step = (int)gridDim.x / 2;
    auto tile = [&](int t) { return pair_tile(t, a.p, starts, tpre, rank); };

    if (warp < kDrainWarps) {
        // ---------------- accumulators -> integer sums -> results.  A warp has a quarter
        // of the lanes and WC of each half's columns
        asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
        griddep_wait();
        const int quarter = warp & 3, w0 = (warp >> 2) * Cfg::WC;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)w0;
        const bool f32 = a.p.ytype != EMU_BF16;
        const int esize = f32 ? 4 : 2;
        const bool pairs_ok = (a.p.ldy & 1) == 0 && (reinterpret_cast<uintptr_t>(a.p.Y) & 3u) == 0;
        for (int64_t r = (int64_t)starts[a.p.G] + blockIdx.x; r < a.p.rows; r += gridDim.x)      // rows of no group are zero
            for (int l = (int)threadIdx.x; l < a.p.N; l += 32 * kDrainWarps) store_value(a.p, r, l, 0.0f, 0);
        uint32_t u = 0;
        bool ok = true;
        for (int t = first; t < total && ok; t += step) {
            const I8Tile x = tile(t);
            const int l = x.l0 + quarter * 32, nch = (x.nk + kI8Chunk - 1) / kI8Chunk;
            int acc[2 * Cfg::WC];
#pragma unroll
            for (int j = 0; j < 2 * Cfg::WC; ++j) acc[j] = 0;
            for (int c = 0; c < nch && ok; ++c) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h && !x.n[1]) break;
                    const uint32_t s = u % Cfg::SLOTS;
                    if (!(ok = warp_wait(tfull0 + 8u * s, (u / Cfg::SLOTS) & 1u, flags))) break;
                    tc_fence_after();
                    const int cols = x.n[h] - w0;
#pragma unroll
                    for (int q = 0; q < Cfg::WC; q += 16) {
                        if (q < cols) {
                            uint32_t v[16];
                            tmem_load16(lanes + s * (uint32_t)Cfg::HC + (uint32_t)q, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) acc[h * Cfg::WC + q + j] += __float2int_rn(__uint_as_float(v[j]));
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_peer(peer_addr(tempty0 + 8u * s, 0));
                    ++u;
                }
            }
            if (!ok) break;
            const int64_t row0 = (int64_t)starts[x.g] + x.c0;
            if (l >= a.p.N) continue;
            const float ws = a.p.wscales && l + lane < a.p.N ? __ldg(a.p.wscales + (int64_t)x.g * a.p.N + l + lane) : 1.0f;
            uint32_t nowhere = 0;                     // this lane's columns (of four blocks of 32) without a source
            static_assert(Cfg::WC == 64, "two blocks of 32 columns a half");
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int q = 0; q < Cfg::WC; q += 32) {
                    const int cols = (h ? x.cols - x.n[0] : min(x.n[0], x.cols)) - w0 - q;
                    const int64_t r = row0 + (h ? x.n[0] : 0) + w0 + q;
                    if (cols <= 0) continue;
                    const float xs = lane < cols ? __ldcg(a.xs + r + lane) : 0.0f;
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const int s = acc[h * Cfg::WC + q + j];
                        v[j] = a.p.ytype == EMU_I32 ? __int_as_float(s) : scaled_sum(s, ws, __shfl_sync(0xFFFFFFFFu, xs, j));
                    }
                    store_columns(v, cols, static_cast<char *>(a.p.Y) + r * a.p.ldy * esize, a.p.ldy, l, a.p.N, f32, pairs_ok);
                    nowhere |= (uint32_t)(__float_as_uint(xs) == kNoRow) << (h * 2 + q / 32);
                }
            }
            if (__any_sync(0xFFFFFFFFu, nowhere != 0)) {
#pragma unroll 1
                for (int i = 0; i < 4; ++i) {
                    const int h = i >> 1, q = (i & 1) * 32;
                    clear_rows(a.p, row0 + (h ? x.n[0] : 0) + w0 + q, __ballot_sync(0xFFFFFFFFu, nowhere >> i & 1u), l + lane);
                }
            }
        }
    } else if (warp < Cfg::TMAW) {
        // ---------------- weights: bytes of shared memory -> FP16 in tensor memory.  Lane: one
        // feature; group b of four warps takes K-block b of a stage
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        const int quarter = warp & 3, mine = (warp - Cfg::CONV) >> 2, row = quarter * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)Cfg::A0;
        const uint32_t from = base + Cfg::W_OFF + (uint32_t)row * kWK;
        // i: stages before (of 128 codes; the MMAs tell by used0 which of them they are done with)
        uint32_t s = 0, ph = 0, i = 0;
        bool ok = true;
        for (int t = first; t < total && ok; t += step) {
            const int nk = uniform(tile(t).nk);
            for (int k = 0; k < nk; k += kWK, ++i) {
                if (!(ok = warp_wait(wfull0 + 8u * s, ph, flags))) break;
                const uint32_t q = i % Cfg::NA, before = i - Cfg::NA;
                ok = convert_weights(
                    from + s * (uint32_t)Cfg::W_STAGE, mine * 4, row, lanes + q * 64u + (uint32_t)mine * 32u, k + mine * kKB < nk,
                    [&] { if (lane == 0) mbar_arrive(wempty0 + 8u * s); },
                    [&] { return i < Cfg::NA || warp_wait(used0 + 8u * (before % Cfg::NC), (before / Cfg::NC) & 1u, flags); });
                if (!ok) break;
                if (++s == Cfg::NW) { s = 0; ph ^= 1u; }
                if (lane == 0) mbar_arrive_peer(peer_addr(afull0 + 8u * q, 0));
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == Cfg::TMAW && lane == 0) {
            // ---------------- TMA: the weights' bytes
            if (a.copied) griddep_wait();
            long issued = 0;
            uint32_t s = 0, ph = 0;
            bool ok = true;
            for (int t = first; t < total && ok; t += step) {
                const I8Tile x = tile(t);
                for (int k = 0; k < x.nk; k += kWK) {
                    if (!(ok = mbar_wait(wempty0 + 8u * s, ph ^ 1u, flags))) break;
                    mbar_arrive_expect_tx(wfull0 + 8u * s, Cfg::W_STAGE);
                    tma_load_3d(base + Cfg::W_OFF + s * Cfg::W_STAGE, &tmW, wfull0 + 8u * s, x.k0 + k, x.l0, x.g);
                    ++issued;
                    if (++s == Cfg::NW) { s = 0; ph ^= 1u; }
                }
            }
            if (!ok) drain_inflight(wfull0, Cfg::NW, issued, flags);
        } else if (warp == Cfg::TMAC && lane == 0) {
            // ---------------- TMA: the rows as FP16
            griddep_wait();
            long issued = 0;
            uint32_t s = 0, ph = 0;
            bool ok = true;
            for (int t = first; t < total && ok; t += step) {
                const I8Tile x = tile(t);
                int row[2];
                bool big[2];
                uint32_t bytes = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int n = x.n[h] / 2;
                    row[h] = starts[x.g] + x.c0 + (h ? x.n[0] : 0) + rank * n;
                    big[h] = n > 16;
                    bytes += n ? (uint32_t)((big[h] ? 64 : 16) * kKB * 2) : 0u;
                }
                for (int k = 0; k < x.nk; k += kWK) {
                    if (!(ok = mbar_wait(used0 + 8u * s, ph ^ 1u, flags))) break;
                    const uint32_t fb = cfull0 + 8u * s, bar = peer_addr(fb, 0);
                    const int blocks = k + kKB < x.nk ? 2 : 1;
                    if (rank == 0) mbar_arrive_expect_tx(fb, bytes * 2 * (uint32_t)blocks);
                    for (int b = 0; b < blocks; ++b)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            if (x.n[h])
                                tma_load_4d<true>(base + s * Cfg::C_STAGE + (uint32_t)(b * Cfg::C_BLOCK + h * Cfg::C_HALF),
                                                  big[h] ? &tmC : &tmS, bar, x.k0 + k + b * kKB, row[h], 0, 0);
                    ++issued;
                    if (++s == Cfg::NC) { s = 0; ph ^= 1u; }
                }
            }
            if (!ok) {
                if (rank == 0) {
                    drain_inflight(cfull0, Cfg::NC, issued, flags);
                } else {
                    // the peer's copies complete on the leader's barriers, which it
                    // cannot observe: give them 200 us before the CTA winds down
                    const unsigned long long t0 = globaltimer_ns();
                    while (globaltimer_ns() - t0 < 200000ull) {}
                }
            }
        } else if (warp == Cfg::MMA && rank == 0) {
            // ---------------- MMA issuer (a pair's leader)
            const uint32_t elected = elect_lane();
            // s0, s1: the next two accumulators; e0, e1: parities of their last reading.  Contraction
            // elements past K are zero in both operands, so that all K-blocks are whole
            uint32_t cs = 0, cph = 0, as = 0, aph = 0, s0 = 0, s1 = 1, e0 = 1, e1 = 1;
            bool ok = true;
            auto next = [&]() {
                s0 = s1;
                e0 = e1;
                if (++s1 == Cfg::SLOTS) { s1 = 0; e1 ^= 1u; }
            };
            for (int t = first; t < total && ok; t += step) {
                const I8Tile x = tile(t);
                const int nk = uniform(x.nk);
                const uint32_t n0 = (uint32_t)uniform(x.n[0]), n1 = (uint32_t)uniform(x.n[1]);
                const uint32_t i0 = idesc_f16(kLRows * 2) | n0 >> 3 << 17, i1 = idesc_f16(kLRows * 2) | n1 >> 3 << 17;
                for (int k = 0; k < nk; k += kWK) {
                    const int kc = k % kI8Chunk;
                    const bool two = k + kKB < nk;
                    if (!(ok = warp_wait(cfull0 + 8u * cs, cph, flags))) break;
                    if (kc == 0 && !(ok = warp_wait(tempty0 + 8u * s0, e0, flags))) break;
                    if (!(ok = warp_wait(afull0 + 8u * as, aph, flags))) break;
                    tc_fence_after();
                    const uint32_t st = (base + cs * (uint32_t)Cfg::C_STAGE) >> 4, at = tmem + (uint32_t)Cfg::A0 + as * 64u;
                    mma_block<true>(elected, tmem + s0 * (uint32_t)Cfg::HC, at, st, i0, kc != 0);
                    if (two) mma_block<true>(elected, tmem + s0 * (uint32_t)Cfg::HC, at + 32u, st + (uint32_t)(Cfg::C_BLOCK >> 4), i0, 1);
                    // a sum's last stage: the first half is read while the second one is still multiplied
                    const bool whole = kc == kI8Chunk - kWK || k + kWK >= nk;
                    if (n1) {
                        if (whole) commit_elected<true>(elected, tfull0 + 8u * s0);
                        if (kc == 0) {
                            if (!(ok = warp_wait(tempty0 + 8u * s1, e1, flags))) break;
                            tc_fence_after();
                        }
                        const uint32_t sh = st + (uint32_t)(Cfg::C_HALF >> 4);
                        mma_block<true>(elected, tmem + s1 * (uint32_t)Cfg::HC, at, sh, i1, kc != 0);
                        if (two) mma_block<true>(elected, tmem + s1 * (uint32_t)Cfg::HC, at + 32u, sh + (uint32_t)(Cfg::C_BLOCK >> 4), i1, 1);
                    }
                    commit_elected<true>(elected, used0 + 8u * cs);
                    if (++as == Cfg::NA) { as = 0; aph ^= 1u; }
                    if (++cs == Cfg::NC) { cs = 0; cph ^= 1u; }
                    if (whole) {
                        if (n1) next();
                        commit_elected<true>(elected, tfull0 + 8u * s0);
                        next();
                    }
                }
            }
            commit_elected<true>(elected, done_bar);
            (void)mbar_wait(done_bar, 0, flags);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync();                                   // the leader's MMAs are done with both CTAs
    if (warp == Cfg::MMA) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

// ------------------------------------------------------- the rows as FP16
struct ExpandArgs {
    I8Product p;
    uint16_t *plane;                  // [rows][ld], in group order
    int64_t ld;
    float *xs;                        // [rows]
    int chunks;                       // parts of a row, of 512 codes
    int own_flags;                    // block 0 looks at all rows and sets the flag word
    CopyArgs copy;                    // of weights, or none
};

// 16 codes a lane, 512 of a row a warp, most warps once.  Bound by HBM and L2: one byte read and two written an
// element (16384 x 8192 61 us, 6.6 TB/s; four such parts a warp, in 8 blocks an SM, took 75).
template <bool WIDE>
__global__ void __launch_bounds__(256, 8) i8_expand_kernel(const ExpandArgs a)
{
    griddep_launch_dependents();
    const I8Product &p = a.p;
    const int lane = (int)lane_id();
    bool bad = false;
    if (blockIdx.x == 0) {
        if (p.ends)
            for (int g = threadIdx.x; g < p.G; g += 256) {
                const int e = p.ends[g];
                bad |= e < 0 || e > p.rows || (g > 0 && p.ends[g - 1] > e);
            }
        if (a.own_flags && p.src)
            for (int r = threadIdx.x; r < p.rows; r += 256) bad |= p.src[r] < 0 || p.src[r] >= p.xrows;
        bad = __syncthreads_or(bad ? 1 : 0) != 0;
        if (threadIdx.x == 0) {
            if (a.own_flags) *p.flags = bad ? (uint32_t)EMU_FLAG_INDEX : 0u;
            else if (bad) atomicOr(p.flags, (uint32_t)EMU_FLAG_INDEX);
        }
    }
    const int64_t units = (int64_t)p.rows * a.chunks;
    for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < units + a.copy.wrows; i += (int64_t)gridDim.x * 8) {
        if (i >= units) {
            copy_row(p, a.copy, i - units, lane);
            continue;
        }
        const int64_t r = i / a.chunks;
        const int first = (int)(i - r * a.chunks) * 512, k = first + lane * 16;
        const int64_t t = p.src ? __ldg(p.src + r) : r;
        const bool there = t >= 0 && t < p.xrows;
        const bool start = lane == 0 && first == 0;
        float xs = 1.0f;                              // (looked at behind the row's loads: nothing waits for it before)
        if (start && there && p.xscales) xs = __ldg(p.xscales + t);
        const int8_t *x = p.X + (there ? t : 0) * p.ldx;
        uint16_t *out = a.plane + r * a.ld;
        if (k >= p.K) continue;
        const uint4 v = there ? load_codes<WIDE>(x + k, p.K - k) : make_uint4(0u, 0u, 0u, 0u);
        uint4 f[2];
        codes_f16(v.x, f[0].x, f[0].y);
        codes_f16(v.y, f[0].z, f[0].w);
        codes_f16(v.z, f[1].x, f[1].y);
        codes_f16(v.w, f[1].z, f[1].w);
        *reinterpret_cast<uint4 *>(out + k) = f[0];
        if (k + 8 < a.ld) *reinterpret_cast<uint4 *>(out + k + 8) = f[1];
        if (start) {                                  // (K > 0: this lane has codes)
            a.xs[r] = __uint_as_float(!there ? kNoRow : isnan(xs) ? 0x7FFFFFFFu : __float_as_uint(xs));
            if (!there && !a.own_flags) atomicOr(p.flags, (uint32_t)EMU_FLAG_INDEX);
        }
    }
}

// Behind the header: the rows as FP16, their scales, a copy of weights.
struct PairLayout {
    int64_t xs, copy, bytes, ld, ldcopy;
};
PairLayout pair_layout(int64_t G, int64_t rows, int64_t N, int64_t K, bool aligned)
{
    PairLayout y = {};
    y.ld = up(K, 8);
    y.ldcopy = up(K, 16);
    y.xs = up(rows * y.ld * 2, 256);
    y.copy = y.xs + up(rows * 4, 256);
    y.bytes = y.copy + (aligned ? 0 : G * N * y.ldcopy);
    return y;
}

}  // namespace

size_t i8_tile_scratch_bytes(int64_t G, int64_t rows, int64_t N, int64_t K, bool aligned)
{
    return (size_t)pair_layout(G, rows, N, K, aligned).bytes;
}

// scratch: i8_tile_scratch_bytes, 16-byte aligned.
cudaError_t launch_i8_tile(I8Product p, void *scratch, cudaStream_t st)
{
    const bool aligned = i8_tma_reads(p.W, p.G, p.N, p.ldw, p.stridew);
    const PairLayout y = pair_layout(p.G, p.rows, p.N, p.K, aligned);
    char *s = static_cast<char *>(scratch);
    // the warps' shares of the registers have to fit what the launch has, or they would be waited for without end
    static std::atomic<int> fit{0};
    if (fit.load(std::memory_order_relaxed) == 0) {
        cudaFuncAttributes at;
        const cudaError_t e = cudaFuncGetAttributes(&at, i8_pair_kernel);
        if (e != cudaSuccess) return e;
        fit.store(at.numRegs * PairCfg::THREADS >= kSplitRegisters ? 1 : -1, std::memory_order_relaxed);
    }
    if (fit.load(std::memory_order_relaxed) < 0) return cudaErrorLaunchOutOfResources;
    ExpandArgs e = {};
    e.p = p;
    PairArgs a = {};
    if (!aligned) {
        e.copy.wrows = (int64_t)p.G * p.N; e.copy.w = reinterpret_cast<int8_t *>(s + y.copy); e.copy.ld = y.ldcopy;
        p.W = e.copy.w;
        p.ldw = y.ldcopy;
        p.stridew = p.N * y.ldcopy;
        a.copied = 1;
    }
    a.p = p;
    a.xs = reinterpret_cast<float *>(s + y.xs);
    uint16_t *plane = reinterpret_cast<uint16_t *>(s);
    CUtensorMap tw, tc, ts;
    if (!make_code_map(&tw, p.W, p.K, p.N, p.G, p.ldw, p.stridew) ||
        !make_group_map(&tc, plane, p.K, p.rows, 1, 1, y.ld, 0, 0, 64) || !make_group_map(&ts, plane, p.K, p.rows, 1, 1, y.ld, 0, 0, 16))
        return cudaErrorInvalidValue;
    e.plane = plane; e.ld = y.ld; e.xs = reinterpret_cast<float *>(s + y.xs);
    e.own_flags = p.rows <= 4096;
    if (!e.own_flags) {
        const cudaError_t c = cudaMemsetAsync(p.flags, 0, sizeof(uint32_t), st);
        if (c != cudaSuccess) return c;
    }
    e.chunks = (p.K + 511) / 512;
    const int64_t blocks = ((int64_t)p.rows * e.chunks + e.copy.wrows + 7) / 8;
    const unsigned grid = (unsigned)(blocks > 152 * 1024 ? 152 * 1024 : blocks);
    if (aligned_codes(p.X, p.xrows > 1 ? p.ldx : 0, 0)) i8_expand_kernel<true><<<grid, 256, 0, st>>>(e);
    else i8_expand_kernel<false><<<grid, 256, 0, st>>>(e);
    const cudaError_t c = cudaGetLastError();
    if (c != cudaSuccess) return c;
    return launch_persistent<i8_pair_kernel>(PairCfg::SMEM, PairCfg::THREADS, 2, max_tiles(p.rows, p.G, p.N, 256, 2), st, tw, tc, ts, a);
}

}  // namespace emu
