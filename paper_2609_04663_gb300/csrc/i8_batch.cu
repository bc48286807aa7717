// Products in 8-bit integers for some rows of each group, in one launch: tiles of 128 features by
// up to 64 columns on one SM (i8_tile.cuh has the arithmetic).
//
// Warps 0-3 read the accumulators and store.  Warps 4-11 turn the token rows into FP16 in swizzled shared
// memory, gathered, two warps a stage of 128 codes in turn: a thread asks for its runs of 16 codes of its group's
// next stage once it has handed over the one before.  (The fence that shows a stage to the tensor cores, and the arrival
// behind it, wait for all loads from global memory that a thread has in flight, as measured; not for those from shared
// memory, see convert_weights: two stages ahead in two groups were none, 58.6 us for 256 rows over
// 32 experts of 2048 x 4096 against 51.)  Warps 12-19 convert weights, 20 brings them by TMA and looks for
// bad indexes, 21 issues the MMAs.
//
// While there are SMs left, K is split between the CTAs of a cluster; each adds and stores a share of the columns,
// whose other sums it reads from their shared memory.
//
// 48 rows x 5120 x 8192 take 18.2 us (HBM alone would 6.5): 1.2 us until all is set up, 3.5 until the first stage's rows and
// weights are there, 2.5 for the next four stages, 6.4 for the other 16 (0.39 each), 4 from the last
// accumulator until the two parts' sums have been handed over, added and stored, 0.6 to the end (a clock read by a CTA at
// each).  64 x 4096 x 4096 13.4, of which handing over to storing takes 3.9.  16 x 16384 x 16384, without parts, 52: 0.4 for each
// of 128 stages and 0.7 for storing.  256 rows over 32 experts of 2048 x 4096 51 (5.3 TB/s).  (Without loads of rows 16.9 and
// 49 us for the first and the last, without converting weights as well 15.5 and 47.)
// Tried: all eight row warps on each stage, with the bytes brought to L1 ahead, 64 us for the 256 rows; a third group of
// converting warps 60 against 58.6; the first CTA of a cluster adding and storing all columns 16 us for the 64 rows.
#include "i8_tile.cuh"

namespace emu {

namespace {

constexpr int kReadWarps = 4, kRowWarps = 8;
constexpr int kRowGroups = 4, kGroupWarps = kRowWarps / kRowGroups, kStepRows = 4 * kGroupWarps, kRuns = 64 / kStepRows;

struct BatchCfg {
    static constexpr int COLS = 64, STEP = 16;
    static constexpr int SLOTS = 4;                                       // accumulators of 64 columns
    static constexpr int A0 = SLOTS * COLS, NS = 4;                       // stages: 64 TMEM columns of 128 codes,
    static constexpr int C_BLOCK = COLS * kKB * 2, C_STAGE = 2 * C_BLOCK; // and as many of the rows
    static constexpr int W_STAGE = kLRows * kWK, NW = 7;
    static constexpr int ROWS = kReadWarps, CONV = ROWS + kRowWarps, TMAW = CONV + kConvertWarps, MMA = TMAW + 1;
    static constexpr int THREADS = 32 * (TMAW + 4);
    static constexpr int W_OFF = NS * C_STAGE, SUM_OFF = W_OFF + NW * W_STAGE, SUMS = kReadWarps * COLS * 32 * 4;
    static constexpr int BAR_OFF = SUM_OFF + SUMS, TAB_OFF = BAR_OFF + 512;
    static constexpr int SMEM = TAB_OFF + 2 * (kMaxGroups + 1) * 4 + 1024;
    static_assert(SMEM <= kSmemMax && A0 + NS * 64 <= 512, "shared and tensor memory");
};

// The registers' split: 768 threads with 80 each at launch.
constexpr int kBatchRegisters = 128 * (144 + 2 * 88 + 2 * 56 + 40);

struct BatchArgs {
    I8Product p;
    const int8_t *rows;               // token rows: X, or copies in group order
    int64_t ldr;
    int copied;
    int parts, shift;                 // CTAs of a cluster, each with a part of K; the number's logarithm
    int own_flags;                    // the first CTA clears the flag word and looks at all rows; else it is clear, and all CTAs look
    unsigned long long selftest_ns;   // not 0: nothing is multiplied, and a wait for weights runs out after so long
};

__device__ uint32_t unread_flags;     // of calls without a workspace

__device__ __forceinline__ I8Tile batch_tile(int t, const BatchArgs &a, const int *starts, const int *tpre, int part)
{
    const int nlt = (a.p.N + kLRows - 1) / kLRows;
    I8Tile x;
    x.g = find_group(tpre, a.p.G, t);
    const int local = t - tpre[x.g], n = starts[x.g + 1] - starts[x.g];
    const int nct = (n + BatchCfg::COLS - 1) / BatchCfg::COLS;
    int ct = 0, lt = local, each = n;                 // (divisions are most of this function: none for one column of tiles)
    if (nct > 1) {
        tile_coords(local, nct, nlt, ct, lt);
        each = (n + nct - 1) / nct;
    }
    auto step = [](int v) { return (v + BatchCfg::STEP - 1) / BatchCfg::STEP * BatchCfg::STEP; };
    each = step(each);
    x.c0 = ct * each;
    x.cols = min(each, n - x.c0);
    x.n[0] = step(x.cols);
    x.n[1] = 0;
    x.l0 = lt * kLRows;
    const int nw = (a.p.K + kWK - 1) / kWK, from = nw * part >> a.shift, to = nw * (part + 1) >> a.shift;      // (2^10 stages, 8 parts)
    x.k0 = from * kWK;
    x.nk = min(a.p.K, to * kWK) - x.k0;
    return x;
}

// The last, short run of a row.
__device__ __noinline__ uint4 load_tail(const int8_t *p, int n) { return load_codes<false>(p, n); }

__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar, int rank)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(peer_addr(bar, (uint32_t)rank)) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_cluster() { asm volatile("fence.acq_rel.cluster;" ::: "memory"); }

__global__ void __launch_bounds__(BatchCfg::THREADS, 1)
i8_batch_kernel(const __grid_constant__ CUtensorMap tmW, const BatchArgs a)
{
    using Cfg = BatchCfg;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *base_ptr = smem_raw + (base - raw);
    const uint32_t cfull0 = base + Cfg::BAR_OFF, afull0 = cfull0 + 8u * Cfg::NS, used0 = afull0 + 8u * Cfg::NS;
    const uint32_t wfull0 = used0 + 8u * Cfg::NS, wempty0 = wfull0 + 8u * Cfg::NW;
    const uint32_t tfull0 = wempty0 + 8u * Cfg::NW, tempty0 = tfull0 + 8u * Cfg::SLOTS;
    const uint32_t sfull0 = tempty0 + 8u * Cfg::SLOTS, sempty0 = sfull0 + 8u * kReadWarps, done_bar = sempty0 + 8u * kReadWarps;
    static_assert(8 * (3 * Cfg::NS + 2 * (Cfg::NW + Cfg::SLOTS + kReadWarps) + 1) <= 496, "barriers");
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(base_ptr + Cfg::BAR_OFF + 496);
    int *starts = reinterpret_cast<int *>(base_ptr + Cfg::TAB_OFF), *tpre = starts + a.p.G + 1;
    const int warp = uniform((int)threadIdx.x >> 5), lane = (int)lane_id();
    const int rank = a.parts > 1 ? (int)cluster_rank() : 0;
    uint32_t *flags = a.p.flags ? a.p.flags : &unread_flags;

    if (threadIdx.x == 0) {
        for (int s = 0; s < Cfg::NS; ++s) {
            mbar_init(cfull0 + 8u * s, kGroupWarps);
            mbar_init(afull0 + 8u * s, kConvertWarps);
            mbar_init(used0 + 8u * s, 1);
        }
        for (int s = 0; s < Cfg::NW; ++s) { mbar_init(wfull0 + 8u * s, 1); mbar_init(wempty0 + 8u * s, kConvertWarps); }
        for (int s = 0; s < Cfg::SLOTS; ++s) { mbar_init(tfull0 + 8u * s, 1); mbar_init(tempty0 + 8u * s, kReadWarps); }
        for (int w = 0; w < kReadWarps; ++w) { mbar_init(sfull0 + 8u * w, a.parts > 1 ? (uint32_t)a.parts - 1u : 1u); mbar_init(sempty0 + 8u * w, a.parts > 1 ? (uint32_t)a.parts - 1u : 1u); }
        mbar_init(done_bar, 1);
        fence_mbar_init();
        tma_prefetch_desc(&tmW);
    }
    if (warp == Cfg::MMA) { tmem_alloc(smem_u32((const void *)tmem_slot), 512); tmem_relinquish(); }
    // the set-up above overlaps the end of the kernel before this one where that allows it
    griddep_wait();
    // before any wait of this CTA can give up (those of others take seconds): flags are only added from here on
    if (threadIdx.x == 0 && blockIdx.x == 0 && a.own_flags && a.p.flags) *a.p.flags = 0u;
    if (a.p.ends) {
        (void)load_groups(a.p.ends, a.p.G, a.p.rows, starts);
    } else if (threadIdx.x == 0) {
        starts[0] = 0;
        starts[1] = a.p.rows;
    }
    __syncthreads();
    if (warp == 0) tile_prefix(starts, a.p.G, Cfg::COLS, (a.p.N + kLRows - 1) / kLRows, tpre);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (a.parts > 1) cluster_arrive();                // this CTA's barriers are initialised
    const int total = a.selftest_ns ? 0 : uniform(tpre[a.p.G]);
    const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
    const int first = (int)blockIdx.x >> a.shift, step = (int)gridDim.x >> a.shift;
    auto tile = [&](int t) { return batch_tile(t, a, starts, tpre, rank); };

    if (warp < kReadWarps) {
        // ---------------- accumulators -> integer sums -> results.  A warp has a quarter of the lanes
        asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
        const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
        const bool f32 = a.p.ytype != EMU_BF16;
        const int esize = f32 ? 4 : 2;
        const bool pairs_ok = (a.p.ldy & 1) == 0 && (reinterpret_cast<uintptr_t>(a.p.Y) & 3u) == 0;
        for (int64_t r = (int64_t)starts[a.p.G] + blockIdx.x; r < a.p.rows; r += gridDim.x)      // rows of no group are zero
            for (int l = (int)threadIdx.x; l < a.p.N; l += 32 * kReadWarps) store_value(a.p, r, l, 0.0f, 0);
        if (a.parts > 1) cluster_wait();              // the other CTAs' barriers are initialised
        uint32_t u = 0, par = 0;                      // accumulator; parity of the tiles before
        bool ok = true;
        for (int t = first; t < total && ok; t += step, par ^= 1u) {
            const I8Tile x = tile(t);
            const int l = x.l0 + warp * 32;
            const int64_t row0 = (int64_t)starts[x.g] + x.c0;
            // scales, while the products are under way
            float ws = 1.0f, xs[2] = {};
            uint32_t gone[2];                         // columns without a source
            if (a.p.wscales && l + lane < a.p.N) ws = __ldg(a.p.wscales + (int64_t)x.g * a.p.N + l + lane);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bool none = false;
                if (32 * h + lane < x.cols) {
                    const int64_t from = a.p.src ? __ldg(a.p.src + row0 + 32 * h + lane) : row0 + 32 * h + lane;
                    none = from < 0 || from >= a.p.xrows;
                    if (!none) xs[h] = a.p.xscales ? __ldg(a.p.xscales + from) : 1.0f;
                }
                gone[h] = __ballot_sync(0xFFFFFFFFu, none);
            }
            int acc[Cfg::COLS];
#pragma unroll
            for (int j = 0; j < Cfg::COLS; ++j) acc[j] = 0;
            for (int k = 0; k < x.nk; k += kI8Chunk, ++u) {
                const uint32_t s = u % Cfg::SLOTS;
                if (!(ok = warp_wait(tfull0 + 8u * s, (u / Cfg::SLOTS) & 1u, flags))) break;
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < Cfg::COLS; q += 16) {
                    if (q < x.cols) {
                        uint32_t v[16];
                        tmem_load16(lanes + s * (uint32_t)Cfg::COLS + (uint32_t)q, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[q + j] += __float2int_rn(__uint_as_float(v[j]));
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(tempty0 + 8u * s);
            }
            if (!ok) break;
            if (a.parts > 1) {
                // sums of this part of K to shared memory; then each CTA of the cluster adds and stores a share of
                // the columns, in blocks of eight
                const uint32_t mine = base + (uint32_t)(Cfg::SUM_OFF + warp * Cfg::COLS * 128 + lane * 4);
                if (!(ok = warp_wait(sempty0 + 8u * warp, par ^ 1u, flags))) break;
#pragma unroll
                for (int j = 0; j < Cfg::COLS; ++j)
                    if (j < x.cols) asm volatile("st.shared.b32 [%0], %1;" ::"r"(mine + (uint32_t)(j * 128)), "r"(acc[j]) : "memory");
                __syncwarp();
                if (lane < a.parts && lane != rank) arrive_cluster(sfull0 + 8u * warp, lane);
                if (!(ok = warp_wait(sfull0 + 8u * warp, par, flags))) break;
                fence_cluster();
                for (int c = 8 * rank; c < x.cols; c += 8 * a.parts) {
                    const uint32_t at = mine + (uint32_t)(c * 128);
                    int sum[8];                       // (columns past the tile's hold anything, and are not stored)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] = 0;
#pragma unroll 2
                    for (int r = 0; r < a.parts; ++r) {
                        const uint32_t from = peer_addr(at, (uint32_t)(rank ^ r));
                        uint32_t v[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = ld_cluster(from + (uint32_t)(j * 128));
#pragma unroll
                        for (int j = 0; j < 8; ++j) sum[j] += (int)v[j];
                    }
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        v[j] = a.p.ytype == EMU_I32 ? __int_as_float(sum[j])
                                                    : scaled_sum(sum[j], ws, __shfl_sync(0xFFFFFFFFu, c < 32 ? xs[0] : xs[1], (c & 31) + j));
                    if (l < a.p.N) {
                        store_columns(v, x.cols - c, static_cast<char *>(a.p.Y) + (row0 + c) * a.p.ldy * esize, a.p.ldy, l, a.p.N, f32, pairs_ok);
                        clear_rows(a.p, row0 + c, (c < 32 ? gone[0] : gone[1]) >> (c & 31) & 0xFFu, l + lane);
                    }
                }
                __syncwarp();
                if (lane < a.parts && lane != rank) arrive_cluster(sempty0 + 8u * warp, lane);
                continue;
            }
            if (l >= a.p.N) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int cols = x.cols - 32 * h;
                if (cols <= 0) break;
                float v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    v[j] = a.p.ytype == EMU_I32 ? __int_as_float(acc[32 * h + j])
                                                : scaled_sum(acc[32 * h + j], ws, __shfl_sync(0xFFFFFFFFu, xs[h], j));
                store_columns(v, cols, static_cast<char *>(a.p.Y) + (row0 + 32 * h) * a.p.ldy * esize, a.p.ldy, l, a.p.N, f32, pairs_ok);
                clear_rows(a.p, row0 + 32 * h, gone[h], l + lane);
            }
        }
    } else if (warp < Cfg::CONV) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 88;");
        const int group = (warp - Cfg::ROWS) / kGroupWarps;
        // ---- rows: this group's next stage (tile, K), its runs of 16 codes on their way
        const int gt = (int)threadIdx.x % (32 * kGroupWarps), chunk = gt & 7, xrow = gt >> 3;        // rows xrow + 8 j
        const uint32_t xput = base + (uint32_t)((chunk >> 2) * Cfg::C_BLOCK + xrow * 128 + ((((chunk & 3) * 2) ^ (xrow & 7)) << 4));
        int lt = first, lk = -kWK, lnk = 0, lk0 = 0, ln = 0;
        const int8_t *source[kRuns] = {};               // this thread's runs in the rows (none: NULL)
        uint32_t li = 0xFFFFFFFFu;                    // stage that was asked for last
        uint4 v[kRuns];
        // to the group's next stage; false behind the last
        auto advance = [&]() {
            do {
                lk += kWK;
                ++li;
                if (lk < lnk) continue;
                if (lnk) lt += step;
                if (lt >= total) { lnk = 0; return false; }
                const I8Tile x = tile(lt);
                lk = 0;
                lnk = x.nk;
                lk0 = x.k0 + chunk * 16;
                ln = x.n[0];
#pragma unroll
                for (int j = 0; j < kRuns; ++j) {
                    const int c = xrow + kStepRows * j;
                    source[j] = nullptr;
                    if (c < x.cols) {
                        const int64_t at = (int64_t)starts[x.g] + x.c0 + c;
                        const int64_t r = a.p.src && !a.copied ? (int64_t)__ldg(a.p.src + at) : at;
                        if (a.copied || (r >= 0 && r < a.p.xrows)) source[j] = a.rows + r * a.ldr + lk0;
                    }
                }
            } while (li % kRowGroups != (uint32_t)group);
            return true;
        };
        // the loads stand next to each other, so that all are on their way before the first is waited for
        auto ask = [&]() {
            const int n = a.p.K - lk0 - lk;
#pragma unroll
            for (int j = 0; j < kRuns; ++j)
                asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
                             "@p ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
                             : "=&r"(v[j].x), "=&r"(v[j].y), "=&r"(v[j].z), "=&r"(v[j].w)
                             : "l"(source[j] + lk), "r"((uint32_t)(source[j] != nullptr && n >= 16)));
            if (n > 0 && n < 16) {                    // the last run of a row
#pragma unroll
                for (int j = 0; j < kRuns; ++j)
                    if (source[j]) v[j] = load_tail(source[j] + lk, n);
            }
        };
        uint32_t i = (uint32_t)group;                 // the group's next stage
        bool have = advance();
        if (have) ask();
        while (have) {
            const uint32_t s = i % Cfg::NS;
            if (!warp_wait(used0 + 8u * s, ((i / Cfg::NS) & 1u) ^ 1u, flags)) break;
            const uint32_t to = xput + s * (uint32_t)Cfg::C_STAGE;
#pragma unroll
            for (int j = 0; j < kRuns; ++j) {
                if (kStepRows * j >= ln) break;
                uint32_t lo[4], hi[4];
                codes_f16(v[j].x, lo[0], lo[1]);
                codes_f16(v[j].y, lo[2], lo[3]);
                codes_f16(v[j].z, hi[0], hi[1]);
                codes_f16(v[j].w, hi[2], hi[3]);
                st_shared_v4(to + (uint32_t)(j * kStepRows * 128), lo[0], lo[1], lo[2], lo[3]);
                st_shared_v4((to + (uint32_t)(j * kStepRows * 128)) ^ 16u, hi[0], hi[1], hi[2], hi[3]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(cfull0 + 8u * s);
            i += kRowGroups;
            if ((have = advance())) ask();
        }
    } else if (warp < Cfg::TMAW) {
        // ---------------- weights: bytes of shared memory -> FP16 in tensor memory.  Lane: one
        // feature; group b of four warps takes K-block b of a stage
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        const int quarter = warp & 3, mine = (warp - Cfg::CONV) >> 2, row = quarter * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(Cfg::A0 + mine * 32);
        const uint32_t from = base + Cfg::W_OFF + (uint32_t)row * kWK;
        uint32_t ws = 0, wph = 0, s = 0, ph = 1;
        bool ok = true;
        for (int t = first; t < total && ok; t += step) {
            const int nk = uniform(tile(t).nk);
            for (int k = 0; k < nk; k += kWK) {
                if (!(ok = warp_wait(wfull0 + 8u * ws, wph, flags))) break;
                ok = convert_weights(from + ws * (uint32_t)Cfg::W_STAGE, mine * 4, row, lanes + s * 64u, k + mine * kKB < nk,
                                     [&] { if (lane == 0) mbar_arrive(wempty0 + 8u * ws); },
                                     [&] { return warp_wait(used0 + 8u * s, ph, flags); });
                if (!ok) break;
                if (lane == 0) mbar_arrive(afull0 + 8u * s);
                if (++ws == Cfg::NW) { ws = 0; wph ^= 1u; }
                if (++s == Cfg::NS) { s = 0; ph ^= 1u; }
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == Cfg::TMAW) {
            // ---------------- TMA: the weights' bytes
            if (lane == 0) {
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
                if (a.selftest_ns) (void)mbar_wait(wfull0, 0, flags, a.selftest_ns);
                if (!ok) drain_inflight(wfull0, Cfg::NW, issued, flags);
            }
            __syncwarp();
            if (a.p.flags && (!a.own_flags || blockIdx.x == 0)) {
                // ---------------- flags: group ends and row indexes out of range
                bool bad = false;
                const int cta = a.own_flags ? 0 : (int)blockIdx.x, ctas = a.own_flags ? 1 : (int)gridDim.x;
                if (a.p.ends && blockIdx.x == 0)
                    for (int g = lane; g < a.p.G; g += 32) {
                        const int e = __ldg(a.p.ends + g);
                        bad |= e < 0 || e > a.p.rows || (g > 0 && __ldg(a.p.ends + g - 1) > e);
                    }
                if (a.p.src) {
#pragma unroll 4
                    for (int64_t r = cta * 32 + lane; r < a.p.rows; r += ctas * 32) {
                        const int t = __ldg(a.p.src + r);
                        bad |= t < 0 || t >= a.p.xrows;
                    }
                }
                bad = __any_sync(0xFFFFFFFFu, bad);
                if (lane == 0 && bad) atomicOr(flags, (uint32_t)EMU_FLAG_INDEX);
            }
        } else if (warp == Cfg::MMA) {
            // ---------------- MMA issuer.  Contraction elements past K are zero in both operands, so
            // that all K-blocks are whole
            const uint32_t elected = elect_lane();
            uint32_t s = 0, ph = 0, u = 0, uph = 1;       // stage; accumulator, parity of its last reading
            bool ok = true;
            for (int t = first; t < total && ok; t += step) {
                const I8Tile x = tile(t);
                const int nk = uniform(x.nk);
                const uint32_t idesc = idesc_f16(kLRows) | (uint32_t)uniform(x.n[0]) >> 3 << 17;
                for (int k = 0; k < nk; k += kWK) {
                    const int kc = k % kI8Chunk;
                    if (kc == 0 && !(ok = warp_wait(tempty0 + 8u * u, uph, flags))) break;
                    if (!(ok = warp_wait(cfull0 + 8u * s, ph, flags))) break;
                    if (!(ok = warp_wait(afull0 + 8u * s, ph, flags))) break;
                    tc_fence_after();
                    const uint32_t st = (base + s * (uint32_t)Cfg::C_STAGE) >> 4, at = tmem + (uint32_t)Cfg::A0 + s * 64u;
                    const uint32_t d = tmem + u * (uint32_t)Cfg::COLS;
                    mma_block<false>(elected, d, at, st, idesc, kc != 0);
                    if (k + kKB < nk) mma_block<false>(elected, d, at + 32u, st + (uint32_t)(Cfg::C_BLOCK >> 4), idesc, 1);
                    commit_elected<false>(elected, used0 + 8u * s);
                    if (++s == Cfg::NS) { s = 0; ph ^= 1u; }
                    if (kc == kI8Chunk - kWK || k + kWK >= nk) {
                        commit_elected<false>(elected, tfull0 + 8u * u);
                        if (++u == Cfg::SLOTS) { u = 0; uph ^= 1u; }
                    }
                }
            }
            commit_elected<false>(elected, done_bar);
            (void)mbar_wait(done_bar, 0, flags);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (a.parts > 1 && warp >= kReadWarps) cluster_wait();
    if (a.parts > 1) cluster_sync();                  // the others have read this CTA's sums
    if (warp == Cfg::MMA) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

__global__ void __launch_bounds__(256) i8_copy_kernel(const I8Product p, const CopyArgs a)
{
    for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < a.wrows + a.trows; i += (int64_t)gridDim.x * 8)
        copy_row(p, a, i, (int)lane_id());
}

// Token rows and weights that cannot be read as they stand are copied to the scratch.
bool rows_direct(const I8Product &p) { return aligned_codes(p.X, p.xrows > 1 ? p.ldx : 0, 0); }

}  // namespace

// Behind the header: copies of the token rows and of the weights, or nothing.
size_t i8_batch_scratch_bytes(int64_t G, int64_t rows, int64_t N, int64_t K, bool aligned)
{
    return aligned ? 0 : (size_t)(up(rows * up(K, 16), 256) + G * N * up(K, 16));
}

// scratch: i8_batch_scratch_bytes, 16-byte aligned; NULL where X and W can be read as they stand.
cudaError_t launch_i8_batch(I8Product p, int parts, void *scratch, cudaStream_t st, unsigned long long selftest_ns)
{
    // the warps' shares of the registers have to fit what the launch has, or they would be waited for without end
    static std::atomic<int> fit{0};
    if (fit.load(std::memory_order_relaxed) == 0) {
        cudaFuncAttributes at;
        const cudaError_t e = cudaFuncGetAttributes(&at, i8_batch_kernel);
        if (e != cudaSuccess) return e;
        fit.store(at.numRegs * BatchCfg::THREADS >= kBatchRegisters ? 1 : -1, std::memory_order_relaxed);
    }
    if (fit.load(std::memory_order_relaxed) < 0) return cudaErrorLaunchOutOfResources;
    const bool weights = !i8_tma_reads(p.W, p.G, p.N, p.ldw, p.stridew), tokens = !rows_direct(p);
    const int64_t ld = up(p.K, 16);
    BatchArgs a = {};
    a.rows = p.X;
    a.ldr = p.ldx;
    if (weights || tokens) {
        CopyArgs c = {};
        c.ld = ld;
        c.t = static_cast<int8_t *>(scratch);
        c.w = c.t + up(p.rows * ld, 256);
        c.wrows = weights ? (int64_t)p.G * p.N : 0;
        c.trows = tokens ? p.rows : 0;
        const int64_t blocks = (c.wrows + c.trows + 7) / 8;
        i8_copy_kernel<<<(unsigned)(blocks > 152 * 16 ? 152 * 16 : blocks), 256, 0, st>>>(p, c);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        if (weights) { p.W = c.w; p.ldw = ld; p.stridew = p.N * ld; }
        if (tokens) { a.rows = c.t; a.ldr = ld; a.copied = 1; }
    }
    a.p = p;
    a.parts = parts;
    while (1 << a.shift < parts) ++a.shift;
    a.selftest_ns = selftest_ns;
    a.own_flags = p.rows <= 4096;
    if (p.flags && !a.own_flags) {
        const cudaError_t e = cudaMemsetAsync(p.flags, 0, sizeof(uint32_t), st);
        if (e != cudaSuccess) return e;
    }
    CUtensorMap tw;
    if (!make_code_map(&tw, p.W, p.K, p.N, p.G, p.ldw, p.stridew)) return cudaErrorInvalidValue;
    return launch_persistent<i8_batch_kernel>(BatchCfg::SMEM, BatchCfg::THREADS, parts, max_tiles(p.rows, p.G, p.N, BatchCfg::COLS, 1), st,
                                              tw, a);
}

}  // namespace emu
