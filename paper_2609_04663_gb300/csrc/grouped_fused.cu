// Products grouped by expert for FP32 weights that meet only a few rows each:
// the weights are read once, as FP32, and split (Eq. (fp32split)) on their way
// to the tensor cores, instead of being written and read again as planes (10
// bytes of traffic per element more than the 4 that are needed).  Bound by the
// way of a K-block through the split (HBM latency, 16 warps' splitting, MMAs) and
// by HBM's rate behind it.  16 matrices of 1024 x 2048 with the rows' split: 37 us
// for one row each, 38 for 16, 44 for 64, 115 for 256; 8 of 4096 x 4096 with 8 rows
// each: 125 us (4.3 TB/s).
//
// Tiles and products are those of grouped.cu with one CTA per tile (128
// features x up to 64 rows).  The leading products A0B0 of every 256 elements
// of K go to one of seven accumulators in turn, which the epilogue warps read
// and add in FP32 while the MMAs go on; the five other products share an
// eighth over all of K.  Warp 18 brings the FP32 weights into shared memory by
// TMA; warps 0-15 split them, two runs of 8 consecutive weights per thread and
// K-block, and write the three slices into the 128-byte-swizzled stage, free of
// bank conflicts.  (Loads to registers ahead of the split were no faster than
// one K-block per HBM latency, 62 us for 16 matrices of 1024 x 2048: the fence
// that shows the slices to the tensor cores waits for a thread's loads in
// flight.)  Warp 16 loads the rows' planes by TMA, warp 17 issues the MMAs,
// warps 19-26 read TMEM and store.
#include "grouped_tile.cuh"
#include "split_f32_pair.cuh"

namespace emu {

namespace {

constexpr int kSplitWarps = 16;
constexpr int kRuns = 1024 / (32 * kSplitWarps);      // runs of 8 weights per thread and K-block
constexpr int kLead = 7;                              // accumulators of the leading products

__device__ __forceinline__ float4 lds_f4(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
    return v;
}

constexpr int kCols = 64;                             // rows of X per tile at most

struct FusedCfg {
    static constexpr int STORE_WARPS = kCols / 8, THREADS = 32 * (kSplitWarps + 3 + STORE_WARPS);
    static constexpr int L_TILE = kLRows * kKB * 2, C_TILE = kCols * kKB * 2;
    static constexpr int STAGE = 3 * (L_TILE + C_TILE), STAGES = 2;
    static constexpr int W_TILE = kLRows * kKB * 4, W_STAGES = 2, W_OFF = STAGES * STAGE;
    static constexpr int BAR_OFF = W_OFF + W_STAGES * W_TILE, TAB_OFF = BAR_OFF + 256;
    static constexpr int SMEM = TAB_OFF + 1024 + 2 * (kMaxGroups + 1) * 4;
    static_assert(SMEM <= kSmemMax, "shared memory per CTA");
};

template <bool LMN>
__global__ void __launch_bounds__(FusedCfg::THREADS, 1)
grouped_fused_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmC,
                     const __grid_constant__ CUtensorMap tmS, const GroupedArgs a)
{
    using Cfg = FusedCfg;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *base_ptr = smem_raw + (base - raw);
    const uint32_t full0 = base + Cfg::BAR_OFF, empty0 = full0 + 8u * Cfg::STAGES;
    const uint32_t tfull0 = empty0 + 8u * Cfg::STAGES, tempty0 = tfull0 + 8u * kLead, cempty = tempty0 + 8u * kLead;
    const uint32_t wfull0 = cempty + 8u, wempty0 = wfull0 + 24u, done_bar = wempty0 + 24u;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(base_ptr + Cfg::BAR_OFF + 16 * Cfg::STAGES + 16 * kLead + 64);
    int *starts = reinterpret_cast<int *>(base_ptr + Cfg::TAB_OFF), *tpre = starts + a.G + 1;
    const int warp = uniform((int)threadIdx.x >> 5), lane = (int)lane_id();
    uint32_t *flags = a.flags;

    if (threadIdx.x == 0) {
        for (int s = 0; s < Cfg::STAGES; ++s) { mbar_init(full0 + 8u * s, 1 + kSplitWarps); mbar_init(empty0 + 8u * s, 1); }
        for (int b = 0; b < kLead; ++b) { mbar_init(tfull0 + 8u * b, 1); mbar_init(tempty0 + 8u * b, Cfg::STORE_WARPS); }
        mbar_init(cempty, Cfg::STORE_WARPS);
        for (int b = 0; b < Cfg::W_STAGES; ++b) { mbar_init(wfull0 + 8u * b, 1); mbar_init(wempty0 + 8u * b, kSplitWarps); }
        mbar_init(done_bar, 1);
        fence_mbar_init();
        tma_prefetch_desc(&tmW);
        tma_prefetch_desc(&tmC);
        tma_prefetch_desc(&tmS);
    }
    if (warp == kSplitWarps + 1) { tmem_alloc(smem_u32((const void *)tmem_slot), 512); tmem_relinquish(); }
    // launched as the programmatic dependent of the kernel that splits the rows,
    // which itself started after everything before it: only the rows' planes have
    // to be waited for (below)
    groups_and_flags(a, starts);
    const int nlt = (a.L + kLRows - 1) / kLRows;
    if (warp == kSplitWarps) tile_prefix(starts, a.G, kCols, nlt, tpre);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const int total = uniform(tpre[a.G]), nkb = (a.K + kKB - 1) / kKB;
    const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
    auto tile = [&](int t) { return tile_at<3, kCols, false, LMN, false>(t, a, starts, tpre, 0); };

    if (warp < kSplitWarps) {
        // ---------------- split: weights -> three slices of the stage.  LMN (W_g
        // is K x N): run i is k row 32 i + tid / 16, features 8 (tid % 16) ..; else
        // (N x K): feature 64 i + tid / 8, k 8 (tid % 8) ...
        const int tid = (int)threadIdx.x, c = tid & 7;
        const int row0 = LMN ? tid >> 4 : tid >> 3;
        constexpr int RSTEP = LMN ? 2 * kSplitWarps : 4 * kSplitWarps;
        // of a run's two 16-byte pieces the second half of each eight lanes reads
        // the second one first
        const bool swap = (lane >> 2) & 1;
        const uint32_t from = base + Cfg::W_OFF + (uint32_t)(LMN ? row0 * 512 + (tid & 15) * 32 : row0 * 256 + c * 32);
        // rows of all runs are the same modulo 8
        const uint32_t to = (uint32_t)((LMN ? ((tid >> 3) & 1) * (Cfg::L_TILE / 2) : 0) + row0 * 128 + ((c ^ (row0 & 7)) << 4));
        uint32_t amax = 0, s = 0, ph = 0, ws = 0, wph = 0;
        bool ok = true;
        const int mine = total > (int)blockIdx.x ? (total - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;
        const long blocks = (long)mine * nkb;
        for (long i = 0; i < blocks; ++i) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(wfull0 + 8u * ws, wph, flags));
            if (!ok) break;
            float4 w[kRuns][2];
#pragma unroll
            for (int r = 0; r < kRuns; ++r) {
                const uint32_t at = from + ws * Cfg::W_TILE + (uint32_t)(r * RSTEP * (LMN ? 512 : 256));
                const float4 u = lds_f4(at + (swap ? 16u : 0u)), v = lds_f4(at + (swap ? 0u : 16u));
                w[r][0] = swap ? v : u;
                w[r][1] = swap ? u : v;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(wempty0 + 8u * ws);
            if (++ws == Cfg::W_STAGES) { ws = 0; wph ^= 1u; }
            // split before the stage is waited for: between its release and the
            // next MMAs only the stores are left
            uint4 p[kRuns][3];
#pragma unroll
            for (int r = 0; r < kRuns; ++r) {
                const float4 u = w[r][0], v = w[r][1];
                amax = abs_bits_max(abs_bits_max(abs_bits_max(abs_bits_max(amax, u.x, u.y), u.z, u.w), v.x, v.y), v.z, v.w);
                split_pair(u.x, u.y, p[r][0].x, p[r][1].x, p[r][2].x);
                split_pair(u.z, u.w, p[r][0].y, p[r][1].y, p[r][2].y);
                split_pair(v.x, v.y, p[r][0].z, p[r][1].z, p[r][2].z);
                split_pair(v.z, v.w, p[r][0].w, p[r][1].w, p[r][2].w);
            }
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(empty0 + 8u * s, ph ^ 1u, flags));
            if (!ok) break;
            const uint32_t st = base + s * (uint32_t)Cfg::STAGE + to;
#pragma unroll
            for (int r = 0; r < kRuns; ++r)
#pragma unroll
                for (int q = 0; q < 3; ++q)
                    st_shared_v4(st + (uint32_t)(r * RSTEP * 128 + q * Cfg::L_TILE), p[r][q].x, p[r][q].y, p[r][q].z, p[r][q].w);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(full0 + 8u * s);
            if (++s == Cfg::STAGES) { s = 0; ph ^= 1u; }
        }
        publish_f32_flags(amax, flags);
    } else if (warp == kSplitWarps + 2 && lane == 0) {
        // ---------------- TMA: the weights
        long i = 0;
        uint32_t s = 0, ph = 0;
        bool ok = true;
        for (int t = (int)blockIdx.x; t < total && ok; t += (int)gridDim.x) {
            const Tile x = tile(t);
            for (int kb = 0; kb < nkb; ++kb, ++i) {
                const uint32_t fb = wfull0 + 8u * s;
                if (!(ok = mbar_wait(wempty0 + 8u * s, ph ^ 1u, flags))) break;
                mbar_arrive_expect_tx(fb, Cfg::W_TILE);
                tma_load_3d(base + Cfg::W_OFF + s * Cfg::W_TILE, &tmW, fb, LMN ? x.l0 : kb * kKB, LMN ? kb * kKB : x.l0, x.g);
                if (++s == Cfg::W_STAGES) { s = 0; ph ^= 1u; }
            }
        }
        if (!ok) drain_inflight(wfull0, Cfg::W_STAGES, i, flags);
    } else if (warp == kSplitWarps && lane == 0) {
        // ---------------- TMA: the rows' planes
        griddep_wait();
        long issued = 0;
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (int t = (int)blockIdx.x; t < total && ok; t += (int)gridDim.x) {
            const Tile x = tile(t);
            // one copy per plane, of 16 rows or a tile's (rows past the group's are not
            // multiplied): several short ones take longer than the bytes
            const bool big = x.csz > 16;
            const int row = (a.padded ? (int)padded_start(starts[x.g], x.g) : starts[x.g]) + x.c0;
            for (int kb = 0; kb < nkb; ++kb) {
                if (!(ok = mbar_wait(empty0 + 8u * s, ph ^ 1u, flags))) break;
                const uint32_t fb = full0 + 8u * s, dc = base + (uint32_t)(s * Cfg::STAGE + 3 * Cfg::L_TILE);
                mbar_arrive_expect_tx(fb, (uint32_t)(3 * (big ? kCols : 16) * kKB * 2));
                for (int r = 0; r < 3; ++r)
                    tma_load_4d<false>(dc + (uint32_t)(r * Cfg::C_TILE), big ? &tmC : &tmS, fb, kb * kKB, row, 0, r);
                ++issued;
                if (++s == Cfg::STAGES) { s = 0; ph ^= 1u; }
            }
        }
        // copies that no MMA has waited for may still be on their way
        if (!ok) drain_inflight(full0, Cfg::STAGES, issued, flags);
    } else if (warp == kSplitWarps + 1) {
        // ---------------- MMA issuer
        const uint32_t elected = elect_lane();
        uint32_t s = 0, ph = 0, cph = 0, it = 0;
        bool ok = true;
        constexpr int kstepL = LMN ? 2048 : 32, kstepC = 32;
        constexpr uint64_t descL = group_desc(LMN ? 64u * kKB * 2u : 16u), descC = group_desc(16u);
        const uint32_t rest = tmem;
        for (int t = (int)blockIdx.x; t < total && ok; t += (int)gridDim.x, ++it) {
            const uint32_t csz = (uint32_t)uniform(tile(t).csz);
            const uint32_t idesc = make_idesc_bf16(kLRows, 0) | csz >> 3 << 17 | (LMN ? 1u << 15 : 0u);
            if (!(ok = warp_wait(cempty, (it & 1u) ^ 1u, flags))) break;
            tc_fence_after();
            for (int kb = 0; kb < nkb; ++kb) {
                if (!(ok = warp_wait(full0 + 8u * s, ph, flags))) break;
                tc_fence_after();
                const uint32_t st = (base + s * (uint32_t)Cfg::STAGE) >> 4;
                const int left = a.K - kb * kKB, kc = kb % kChunkBlocks;
                auto mma = [&](uint32_t acc, int il, int ic, int kk, bool add) {
                    mma_elected<false>(elected, acc, descL + (st + (uint32_t)((il * Cfg::L_TILE + kk * kstepL) >> 4)),
                                       descC + (st + (uint32_t)((3 * Cfg::L_TILE + ic * Cfg::C_TILE + kk * kstepC) >> 4)), idesc,
                                       add);
                };
#pragma unroll
                for (int kk = 0; kk < kKB / 16; ++kk) {
                    if (16 * kk < left) {
                        mma(rest, 1, 1, kk, (kb | kk) != 0);
                        mma(rest, 1, 0, kk, true);
                        mma(rest, 2, 0, kk, true);
                        mma(rest, 0, 2, kk, true);
                        mma(rest, 0, 1, kk, true);
                    }
                }
                const uint32_t b = cph % kLead, lead = tmem + (b + 1u) * kCols;
                if (kc == 0) {                        // this accumulator's last sum has been read
                    if (!(ok = warp_wait(tempty0 + 8u * b, ((cph / kLead) & 1u) ^ 1u, flags))) break;
                    tc_fence_after();
                }
#pragma unroll
                for (int kk = 0; kk < kKB / 16; ++kk)
                    if (16 * kk < left) mma(lead, 0, 0, kk, (kc | kk) != 0);
                commit_elected<false>(elected, empty0 + 8u * s);
                if (kc == kChunkBlocks - 1 || kb == nkb - 1) { commit_elected<false>(elected, tfull0 + 8u * b); ++cph; }
                if (++s == Cfg::STAGES) { s = 0; ph ^= 1u; }
            }
        }
        commit_elected<false>(elected, done_bar);
        (void)mbar_wait(done_bar, 0, flags);
    } else if (warp >= kSplitWarps + 3) {
        // ---------------- epilogue: a quarter of the lanes, 32 columns
        constexpr int HALF = 32;                      // columns of a warp
        const int quarter = warp & 3, h0 = (warp - (kSplitWarps + 3)) / 4 * HALF;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)h0;
        zero_rest(a, starts, (int)threadIdx.x - 32 * (kSplitWarps + 3), 32 * Cfg::STORE_WARPS);
        uint32_t cph = 0;
        bool ok = true;
        const int nch = (a.K + kKChunk - 1) / kKChunk;
        for (int t = (int)blockIdx.x; t < total && ok; t += (int)gridDim.x) {
            const Tile x = tile(t);
            const int l = x.l0 + quarter * 32, cols = x.cols - h0;
            float acc[HALF];
#pragma unroll
            for (int j = 0; j < HALF; ++j) acc[j] = 0.0f;
            for (int c = 0; c <= nch; ++c) {          // the chunks' leading sums, then the other products
                const uint32_t b = cph % kLead;
                if (c < nch) {
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(tfull0 + 8u * b, (cph / kLead) & 1u, flags));
                    if (!ok) break;
                    ++cph;
                    tc_fence_after();
                }
#pragma unroll
                for (int h = 0; h < HALF; h += 16) {
                    if (h < cols) {
                        uint32_t v[16];
                        tmem_load16(lanes + (c < nch ? (b + 1u) * kCols : 0u) + (uint32_t)h, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[h + j] = __fadd_rn(acc[h + j], __uint_as_float(v[j]));
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(c < nch ? tempty0 + 8u * b : cempty);
            }
            if (ok && l < a.L && cols > 0)
                store_columns(acc, cols, static_cast<float *>(a.out) + ((int64_t)starts[x.g] + x.c0 + h0) * a.ldo, a.ldo, l,
                              a.L, true, false);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kSplitWarps + 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <bool LMN>
cudaError_t run_fused(const CUtensorMap &tw, const CUtensorMap &tc, const CUtensorMap &ts, const GroupedArgs &a,
                      int64_t tiles, cudaStream_t st)
{
    using Cfg = FusedCfg;
    return launch_persistent<grouped_fused_kernel<LMN>>(Cfg::SMEM, Cfg::THREADS, 1, tiles, st, tw, tc, ts, a);
}

// Tensor map over G FP32 matrices of rows x inner, box box_inner x box_rows.
bool make_weight_map(CUtensorMap *map, const float *W, int64_t inner, int64_t rows, int64_t G, int64_t ld, int64_t stride,
                     int box_inner, int box_rows)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)G};
    cuuint64_t strides[2] = {(cuuint64_t)ld * 4, (cuuint64_t)(G > 1 ? stride : rows * ld) * 4};
    cuuint32_t box[3] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<float *>(W), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

bool fused_takes(const float *W, int64_t G, int64_t ldw, int64_t stridew)
{
    return (reinterpret_cast<uintptr_t>(W) & 15u) == 0 && ldw % 4 == 0 && (G == 1 || (stridew % 4 == 0 && stridew > 0));
}

// Y = X op(W_g) for FP32 weights in memory; X: the rows' three planes.
cudaError_t launch_grouped_fused(bool trans, int64_t G, int64_t rows, int64_t N, int64_t K, const GroupedOperand &X,
                                 const float *W, int64_t ldw, int64_t stridew, const int32_t *ends, float *Y,
                                 int64_t ldy, uint32_t *flags, cudaStream_t st)
{
    GroupedArgs a = {};
    a.ends = ends; a.G = (int)G; a.rows = (int)rows; a.L = (int)N; a.K = (int)K;
    a.padded = X.padded ? 1 : 0; a.out = Y; a.ldo = ldy; a.out_f32 = 1; a.flags = flags;
    CUtensorMap tw, tc, ts;
    const bool ok = trans ? make_weight_map(&tw, W, K, N, G, ldw, stridew, kKB, kLRows)
                          : make_weight_map(&tw, W, N, K, G, ldw, stridew, kLRows, kKB);
    if (!ok || !make_group_map(&tc, X.planes, K, X.rows, 1, 3, X.ld, 0, X.plane, kCols) ||
        !make_group_map(&ts, X.planes, K, X.rows, 1, 3, X.ld, 0, X.plane, 16))
        return cudaErrorInvalidValue;
    const int64_t tiles = max_tiles(rows, G, N, kCols, 1);
    return trans ? run_fused<false>(tw, tc, ts, a, tiles, st) : run_fused<true>(tw, tc, ts, a, tiles, st);
}

}  // namespace emu
