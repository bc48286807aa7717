// Pieces shared by the kernels of the products grouped by expert: tile
// geometry, tensor maps and loads, shared-memory descriptors, TMEM reads and
// the stores of an epilogue warp.  Each translation unit gets its own copies
// (unnamed namespace).
#pragma once
#include <atomic>

#include "gemm_common.cuh"
#include "grouped_common.cuh"
#include "expert_launchers.cuh"
#include "pair_common.cuh"

#pragma nv_diag_suppress 177      // helpers a translation unit does not use

namespace emu {

struct GroupedArgs {
    const int32_t *ends;
    int G, rows;
    int L;                 // output features (the lane dimension)
    int C;                 // gradient: output rows m
    int K;                 // product: contraction length
    int padded, lpadded;   // rows at padded positions: X or the gradient's A, the gradient's B
    void *out;
    int64_t ldo, strideo;  // row pitch; gradient: distance between the groups' results
    int out_f32;
    int lwide, cwide;      // the MN-major operand's tensor map loads two blocks of 64 at once
    uint32_t *flags;
    int own_flags;         // the flag word is this kernel's alone: it is set, not added to
    uint32_t never;        // grouped_fused.cu: 2^32 - 1, as a number that the compiler does not know
};

// BF16 operands (grouped_bf16.cu).
cudaError_t launch_bf16_product(bool trans, const GroupedOperand &X, const GroupedOperand &W, const GroupedArgs &a, cudaStream_t st);
cudaError_t launch_bf16_gradient(const GroupedOperand &A, const GroupedOperand &B, GroupedArgs a, cudaStream_t st);

namespace {

constexpr int kLRows = 128;           // MMA rows (output features) per CTA
constexpr int kKB = 64;               // K-block: one 128-byte swizzle row of BF16
constexpr int kSmemMax = 232448;      // shared memory per CTA

constexpr int kChunkBlocks = kKChunk / kKB;   // K-blocks of one chunk of the leading product
constexpr int kEpiWarps = 8;

// S slices, BC MMA columns at most, PAIR: a tile's 256 features on two CTAs.
template <int S, int BC, bool PAIR>
struct GroupedCfg {
    static constexpr int CTAS = PAIR ? 2 : 1;
    static constexpr int CROWS = BC / CTAS;                       // column-operand rows staged per CTA
    static constexpr int STEP = PAIR ? 32 : 16;                   // granularity of the MMA's N
    static constexpr int L_TILE = kLRows * kKB * 2;
    static constexpr int C_TILE = CROWS * kKB * 2;
    static constexpr int STAGE = S * (L_TILE + C_TILE);
    static constexpr int FIXED = 1024 + 512 + 2 * (kMaxGroups + 1) * 4;   // alignment, barriers, group tables
    static constexpr int FIT = (kSmemMax - FIXED) / STAGE;
    static constexpr int STAGES = FIT > 8 ? 8 : FIT;
    static constexpr int BAR_OFF = STAGES * STAGE;
    static constexpr int TAB_OFF = BAR_OFF + 512;
    static constexpr int SMEM = STAGES * STAGE + FIXED;
    static constexpr int THREADS = 64 + 32 * kEpiWarps;
    static constexpr int HALF = BC >= 64 ? BC / 2 : 32;           // accumulator columns of one epilogue warp
    static_assert(STAGES >= 2, "stages");
    static_assert(BC <= 256 && CROWS % 64 == 0 || BC < 128, "column tile");
};

// Tile loads, counted on this CTA's barrier or (PAIR) on one of either CTA.
// 4-D: K-major operands (K, MN, group, slice).  5-D: MN-major operands with
// the MN dimension in blocks of 64 (MN % 64, K, MN / 64, group, slice).
template <bool PAIR>
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int32_t c0, int32_t c1,
                                            int32_t c2, int32_t c3)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                     " [%0], [%1, {%3, %4, %5, %6}], [%2];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                     " [%0], [%1, {%3, %4, %5, %6}], [%2];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
                     : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int32_t c0, int32_t c1,
                                            int32_t c2, int32_t c3, int32_t c4)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                     " [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                     " [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
                     : "memory");
}

// 16 FP32 accumulator columns of the warp's lanes.
__device__ __forceinline__ void tmem_load16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}

// Shared-memory descriptor of a 128-byte-swizzled tile at shared address 0:
// the address is added in units of 16 bytes.  K-major: rows of 64 K elements,
// 8-row groups 1024 bytes apart; the next 16 K elements start 32 bytes on.
// MN-major: blocks of 64 MN elements (one 128-byte row) by kKB rows of K, the
// blocks `lbo` bytes apart, 8-row groups of K 1024 bytes apart; the next 16 K
// rows start 2048 bytes on.
__host__ __device__ constexpr uint64_t group_desc(uint32_t lbo)
{
    return (uint64_t)(lbo >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1u << 46 | (uint64_t)2u << 61;
}

// The MMA warp runs converged, with every operand the same in all lanes, so
// that the compiler can keep descriptors in uniform registers (one thread in a
// branch of its own took 92 clocks per MMA, moving them there one by one); one
// elected lane issues.
__device__ __forceinline__ uint32_t elect_lane()
{
    uint32_t q;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(q));
    return q;
}
template <bool PAIR>
__device__ __forceinline__ void mma_elected(uint32_t elected, uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                            uint32_t accumulate)
{
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                     "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                     "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void commit_elected(uint32_t elected, uint32_t bar)
{
    if (elected) {
        if constexpr (PAIR) mma_commit_pair(bar);
        else mma_commit(bar);
    }
    __syncwarp();
}
// A wait of a whole warp: true when every lane saw the phase complete.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint32_t *flags)
{
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, flags));
}
// The warp's index as a value the compiler knows to be uniform, and any other
// value that is the same in all lanes.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }

// One output tile: features l0 .. (this CTA's 128), columns c0 .. c0 + cols
// of group g (rows of the group, or m), contraction of nk elements from k0.
struct Tile {
    int g, l0, c0, cols, csz, k0, nk;
};

template <int S, int BC, bool PAIR, bool LMN, bool CMN>
__device__ __forceinline__ Tile tile_at(int t, const GroupedArgs &a, const int *starts, const int *tpre, int rank)
{
    using Cfg = GroupedCfg<S, BC, PAIR>;
    constexpr int LT = kLRows * Cfg::CTAS;
    const int nlt = (a.L + LT - 1) / LT;
    Tile x;
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
    const int each = ((n + nct - 1) / nct + Cfg::STEP - 1) / Cfg::STEP * Cfg::STEP;
    x.c0 = ct * each;
    x.cols = min(each, n - x.c0);
    x.csz = (x.cols + Cfg::STEP - 1) / Cfg::STEP * Cfg::STEP;
    x.l0 = lt * LT + rank * kLRows;
    if constexpr (CMN) {
        x.k0 = (int)padded_start(starts[x.g], x.g);
        x.nk = starts[x.g + 1] - starts[x.g];
    } else {
        x.k0 = 0;
        x.nk = a.K;
    }
    return x;
}

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(uint32_t x) { return __uint_as_float(x); }

// C accumulator columns of this warp's lanes -> rows 0 .. cols - 1 of out:
// column j is output row j, lane i feature l + i.  BF16: two columns at a
// time, neighbouring lanes exchange values so that each stores two features
// of one row.  The usual case (C whole columns, 32 features, pairs that can be
// stored as words) has no test per element: these instructions, not the
// stores' bandwidth, are what the epilogue takes.
template <typename T, int C>
__device__ __forceinline__ void store_columns(const T (&v)[C], int cols, void *out, int64_t ldo, int l, int L,
                                              bool out_f32, bool pairs_ok)
{
    const int lane = (int)lane_id();
    const bool whole = cols >= C && l + 32 <= L;
    if (out_f32) {
        float *o = static_cast<float *>(out) + l + lane;
        if (whole) {
#pragma unroll
            for (int j = 0; j < C; ++j, o += ldo) *o = as_float(v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (l + lane < L && j < cols) o[(int64_t)j * ldo] = as_float(v[j]);
        }
    } else {
        const bool odd = lane & 1;
        const int i = lane & ~1;
        uint16_t *o = static_cast<uint16_t *>(out) + (odd ? ldo : 0) + l + i;
        uint32_t w[C / 2];                              // features i (low half) and i + 1 of row 2 j + odd
#pragma unroll
        for (int j = 0; j < C / 2; ++j) {
            const float keep = as_float(odd ? v[2 * j + 1] : v[2 * j]);
            const float got = __shfl_xor_sync(0xFFFFFFFFu, as_float(odd ? v[2 * j] : v[2 * j + 1]), 1);
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(odd ? keep : got), "f"(odd ? got : keep));
        }
        if (whole && pairs_ok) {
            char *p = reinterpret_cast<char *>(o);
            const int64_t two = 4 * ldo;
#pragma unroll
            for (int j = 0; j < C / 2; ++j, p += two) *reinterpret_cast<uint32_t *>(p) = w[j];
        } else {
#pragma unroll
            for (int j = 0; j < C / 2; ++j) {
                if (2 * j + (odd ? 1 : 0) >= cols) continue;
                uint16_t *p = o + (int64_t)(2 * j) * ldo;
                if (l + i < L) p[0] = (uint16_t)w[j];
                if (l + i + 1 < L) p[1] = (uint16_t)(w[j] >> 16);
            }
        }
    }
}

// The groups' bounds, and what their check says in the flag word.  All CTAs see
// the same bounds; one reports.  A kernel that owns the word clears it this way
// too: the only other flag, a wait that gave up, comes seconds later.
__device__ __forceinline__ void groups_and_flags(const GroupedArgs &a, int *starts)
{
    const bool bad = load_groups(a.ends, a.G, a.rows, starts);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (a.own_flags) *a.flags = bad ? (uint32_t)EMU_FLAG_INDEX : 0u;
        else if (bad) atomicOr(a.flags, (uint32_t)EMU_FLAG_INDEX);
    }
}

// First tile of every group (tpre[G]: all tiles), for groups of n rows in
// column tiles of bc rows and nlt feature tiles; one warp.
__device__ __forceinline__ void tile_prefix(const int *starts, int G, int bc, int nlt, int *tpre)
{
    const int lane = (int)lane_id();
    int carry = 0;
    for (int g0 = 0; g0 < G; g0 += 32) {
        const int g = g0 + lane;
        int v = g < G ? (starts[g + 1] - starts[g] + bc - 1) / bc * nlt : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(0xFFFFFFFFu, v, d);
            if (lane >= d) v += u;
        }
        if (g < G) tpre[g + 1] = carry + v;
        carry += __shfl_sync(0xFFFFFFFFu, v, 31);
    }
    if (lane == 0) tpre[0] = 0;
}

// Rows of no group (from starts[G] on) are zero: n threads of every CTA, tid
// 0 .. n - 1, set them.
__device__ __forceinline__ void zero_rest(const GroupedArgs &a, const int *starts, int tid, int n)
{
    for (int64_t r = (int64_t)starts[a.G] + blockIdx.x; r < a.rows; r += gridDim.x)
        for (int l = tid; l < a.L; l += n) {
            if (a.out_f32) static_cast<float *>(a.out)[r * a.ldo + l] = 0.0f;
            else static_cast<uint16_t *>(a.out)[r * a.ldo + l] = 0;
        }
}

// Tensor maps over a plane set [S][batch][rows][ld].  K-major: dims (inner,
// rows, batch, S), box (64, box_rows).  MN-major: dims (64, rows, inner / 64,
// batch, S) and two blocks per box where inner is a multiple of `tile`, so that
// tiles start on whole blocks (*wide), else (inner, rows, 1, batch, S) and one.
bool make_group_map(CUtensorMap *map, const uint16_t *p, int64_t inner, int64_t rows, int64_t batch, int S, int64_t ld,
                    int64_t stride, int64_t plane, int box_rows, int *wide = nullptr, int tile = 64)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    if (batch <= 1) stride = rows * ld;
    if (S <= 1) plane = batch * stride;
    const bool mn = wide != nullptr, two = mn && inner % tile == 0;
    if (mn) *wide = two ? 1 : 0;
    cuuint64_t dims[5] = {(cuuint64_t)(two ? 64 : inner), (cuuint64_t)rows}, strides[4] = {(cuuint64_t)ld * 2};
    cuuint32_t box[5] = {64, (cuuint32_t)box_rows, 1, 1, 1}, estr[5] = {1, 1, 1, 1, 1};
    int n = 2;
    if (mn) {
        dims[n] = (cuuint64_t)(two ? inner / 64 : 1);
        box[n] = two ? 2 : 1;
        strides[n - 1] = 128;
        ++n;
    }
    dims[n] = (cuuint64_t)batch;
    strides[n - 1] = (cuuint64_t)stride * 2;
    ++n;
    dims[n] = (cuuint64_t)S;
    strides[n - 1] = (cuuint64_t)plane * 2;
    ++n;
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)n, const_cast<uint16_t *>(p), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// SMs of the current device (asked for once per device).
int sm_count()
{
    static std::atomic<int> known[64];
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 152;
    if (dev >= 0 && dev < 64 && (sms = known[dev].load(std::memory_order_relaxed)) > 0) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 2) return 152;
    if (dev >= 0 && dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

// Lets a kernel take `smem` bytes of dynamic shared memory (set once per device).
template <auto KERN>
cudaError_t allow_smem(int smem)
{
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(KERN, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// A persistent launch: one CTA (or cluster of `ctas`) per SM (pair), no more
// than there are tiles, as a programmatic dependent of the kernel before it.
template <auto KERN, typename... Args>
cudaError_t launch_persistent(int smem, int threads, int ctas, int64_t tiles, cudaStream_t st, const Args &...args)
{
    cudaError_t e = allow_smem<KERN>(smem);
    if (e != cudaSuccess) return e;
    int64_t units = sm_count() / ctas;
    if (units > tiles) units = tiles < 1 ? 1 : tiles;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * ctas));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ctas;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, KERN, args...);
    if (e != cudaSuccess) return e;
    return cudaGetLastError();
}

// Tiles at most (the host does not know the groups' sizes): every group may
// end in a partial column tile.
int64_t max_tiles(int64_t rows, int64_t G, int64_t L, int bc, int ctas)
{
    const int64_t groups = G < rows ? G : rows, lt = kLRows * ctas;
    return (rows / bc + groups) * ((L + lt - 1) / lt);
}

}  // namespace

}  // namespace emu
