// Products in 8-bit integers on the tensor cores, dense or grouped by expert.
//
// This GPU's integer tensor rate is a small part of its FP16 rate, so the codes are
// multiplied as FP16 numbers: a code has at most 8 significant bits, a product 15, and while
// a sum has at most 1024 terms it stays within 2^24, where FP32 holds every integer.  The
// accumulators are read every 1024 terms and added as 32-bit integers in registers: all sums
// are exact.
//
// Output features lie on the MMA's rows, token rows on its columns (as in grouped.cu).  The
// weights cross HBM and L2 as bytes; warps turn them into FP16 and write them to tensor memory, from
// which the MMA takes its first operand: the byte u = code + 128 in the mantissa of
// 1024 + u, less 1152 (five instructions for four codes).  The token rows are turned into FP16
// once, gathered, by a small kernel before.  Its result is waited for only by the warps that
// read it.
#include <type_traits>

#include "grouped_tile.cuh"
#include "i8_common.cuh"

namespace emu {

namespace {

constexpr int kI8Chunk = 1024;                        // terms of a sum that FP32 holds exactly: 2^14 each, 2^24 in all
constexpr int kWK = 128;                              // codes of a weight row per stage (two K-blocks)
constexpr int kDrainWarps = 8;                        // warps that read accumulators and store

template <int BC, bool PAIR>
struct I8Cfg {
    static constexpr int CTAS = PAIR ? 2 : 1;
    static constexpr int HALVES = BC > 128 ? 2 : 1, HC = BC / HALVES;     // halves of a tile's columns
    static constexpr int STEP = PAIR ? 32 : 16;
    static constexpr int SLOTS = HALVES == 2 ? 3 : 4;                     // accumulators of HC columns
    static constexpr int A0 = SLOTS * HC, NA = (512 - A0) / 64;           // A stages: 64 TMEM columns of 128 codes
    static constexpr int C_HALF = HC / CTAS * kKB * 2, C_BLOCK = HALVES * C_HALF;     // rows of one K-block
    static constexpr int C_STAGE = 2 * C_BLOCK, NC = 4;
    static constexpr int W_STAGE = kLRows * kWK, NW = HALVES == 2 ? 4 : 8;
    static constexpr int GROUPS = 2;                                      // groups of four converting warps
    static constexpr int CONV = kDrainWarps, TMAW = CONV + 4 * GROUPS, MMA = TMAW + 1, TMAC = TMAW + 2;
    static constexpr int THREADS = 32 * (TMAW + 4);
    static constexpr int WC = HC / 2;                                     // columns of a half that a draining warp reads
    static constexpr int W_OFF = NC * C_STAGE, BAR_OFF = W_OFF + NW * W_STAGE, TAB_OFF = BAR_OFF + 512;
    static constexpr int SMEM = TAB_OFF + 2 * (kMaxGroups + 1) * 4 + 1024;
    static_assert(SMEM <= kSmemMax, "shared memory per CTA");
    static_assert(NA >= 2 && NC % NA == 0 && C_HALF == 8192, "stages");
};

struct I8TileArgs {
    I8Product p;
    const float *xs;                  // [rows] the rows' scales in group order (0: no such row)
    int32_t *sums;                    // [rows][N], zero: sums over parts of K, where they are split
    uint32_t *tickets;                // [tiles][kDrainWarps], zero
    int parts;                        // parts of K
};

struct I8Tile {
    int tile, g, l0, c0, cols, n[2], k0, nk;
};

template <int BC, bool PAIR>
__device__ __forceinline__ I8Tile i8_tile_at(int t, const I8TileArgs &a, const int *starts, const int *tpre, int rank)
{
    using Cfg = I8Cfg<BC, PAIR>;
    constexpr int LT = kLRows * Cfg::CTAS;
    const int nlt = (a.p.N + LT - 1) / LT;
    I8Tile x;
    x.tile = t / a.parts;
    const int part = t - x.tile * a.parts;
    x.g = find_group(tpre, a.p.G, x.tile);
    const int local = x.tile - tpre[x.g], n = starts[x.g + 1] - starts[x.g];
    const int nct = (n + BC - 1) / BC;
    int ct, lt;
    tile_coords(local, nct, nlt, ct, lt);
    auto up = [](int v) { return (v + Cfg::STEP - 1) / Cfg::STEP * Cfg::STEP; };
    const int each = up((n + nct - 1) / nct);
    x.c0 = ct * each;
    x.cols = min(each, n - x.c0);
    x.n[0] = Cfg::HALVES == 1 || x.cols <= Cfg::HC ? up(x.cols) : up((x.cols + 1) / 2);
    x.n[1] = x.cols > x.n[0] ? up(x.cols - x.n[0]) : 0;
    x.l0 = lt * LT + rank * kLRows;
    const int nw = (a.p.K + kWK - 1) / kWK;           // (64 bits: 2^10 stages times parts)
    const int from = (int)((int64_t)nw * part / a.parts), to = (int)((int64_t)nw * (part + 1) / a.parts);
    x.k0 = from * kWK;
    x.nk = min(a.p.K, to * kWK) - x.k0;
    return x;
}

// D (+)= A B^T over one K-block (four MMAs of 16) with A in tensor memory: rows on lanes, two
// FP16 a column, so 8 columns an MMA; B's next 16 start 32 bytes on.  One block of assembly: with an MMA
// each, their operands' way into uniform registers took longer than the MMAs (60 clocks for one of 64).
template <bool PAIR>
__device__ __forceinline__ void mma_block(uint32_t elected, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    constexpr uint64_t desc = group_desc(16u);
#define EMU_MMA_BLOCK(CG)                                                                                              \
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b32 l;\n\t.reg .b32 c;\n\t.reg .b64 b;\n\t"                              \
                 "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"                                                  \
                 "mov.b64 b, {%2, %6};\n\t"                                                                            \
                 "@q tcgen05.mma.cta_group::" CG ".kind::f16 [%0], [%1], b, %3, p;\n\t"                                \
                 "add.u32 l, %2, 2;\n\tadd.u32 c, %1, 8;\n\tmov.b64 b, {l, %6};\n\t"                                  \
                 "@q tcgen05.mma.cta_group::" CG ".kind::f16 [%0], [c], b, %3, 1;\n\t"                                 \
                 "add.u32 l, %2, 4;\n\tadd.u32 c, %1, 16;\n\tmov.b64 b, {l, %6};\n\t"                                 \
                 "@q tcgen05.mma.cta_group::" CG ".kind::f16 [%0], [c], b, %3, 1;\n\t"                                 \
                 "add.u32 l, %2, 6;\n\tadd.u32 c, %1, 24;\n\tmov.b64 b, {l, %6};\n\t"                                 \
                 "@q tcgen05.mma.cta_group::" CG ".kind::f16 [%0], [c], b, %3, 1;\n\t}"                                \
                 ::"r"(d), "r"(a), "r"((uint32_t)desc + b), "r"(idesc), "r"(accumulate), "r"(elected), "n"((uint32_t)(desc >> 32)) \
                 : "memory")
    if constexpr (PAIR) EMU_MMA_BLOCK("2");
    else EMU_MMA_BLOCK("1");
#undef EMU_MMA_BLOCK
}

// Instruction descriptor, kind::f16: D FP32 (bits 4-5 = 1), A and B FP16 (bits 7-12 = 0),
// both K-major; N >> 3 in bits 17-22, M >> 4 in bits 24-28.
__host__ __device__ constexpr uint32_t idesc_f16(int M) { return (1u << 4) | ((uint32_t)(M >> 4) << 24); }

__device__ __forceinline__ void tmem_store16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
                 "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                 "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint4 lds_u4(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

// Four codes (bytes, the lowest first) -> four FP16 numbers in two words.
__device__ __forceinline__ void codes_f16(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    w ^= 0x80808080u;                                 // code + 128
    const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));      // - (1024 + 128), exact
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
}

// 32 codes of a weight row -> 16 columns of tensor memory.
__device__ __forceinline__ void half_block(const uint4 &u, const uint4 &v, uint32_t (&f)[16])
{
    codes_f16(u.x, f[0], f[1]);
    codes_f16(u.y, f[2], f[3]);
    codes_f16(u.z, f[4], f[5]);
    codes_f16(u.w, f[6], f[7]);
    codes_f16(v.x, f[8], f[9]);
    codes_f16(v.y, f[10], f[11]);
    codes_f16(v.z, f[12], f[13]);
    codes_f16(v.w, f[14], f[15]);
}

template <bool PAIR>
__device__ __forceinline__ void registers_drain() { if constexpr (PAIR) asm volatile("setmaxnreg.inc.sync.aligned.u32 168;"); }
template <bool PAIR>
__device__ __forceinline__ void registers_convert() { if constexpr (PAIR) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;"); }
template <bool PAIR>
__device__ __forceinline__ void registers_issue() { if constexpr (PAIR) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;"); }
constexpr int kSplitRegisters = 128 * (2 * 168 + 2 * 48 + 40);     // of the 640 threads of a pair's CTA

template <int BC, bool PAIR>
__global__ void __launch_bounds__(I8Cfg<BC, PAIR>::THREADS, 1)
i8_tile_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmC,
               const __grid_constant__ CUtensorMap tmS, const I8TileArgs a)
{
    using Cfg = I8Cfg<BC, PAIR>;
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
    const int rank = PAIR ? (int)cluster_rank() : 0;
    uint32_t *flags = a.p.flags;

    if (threadIdx.x == 0) {
        for (int s = 0; s < Cfg::NC; ++s) { mbar_init(cfull0 + 8u * s, 1); mbar_init(used0 + 8u * s, 1); }
        for (int s = 0; s < Cfg::NW; ++s) { mbar_init(wfull0 + 8u * s, 1); mbar_init(wempty0 + 8u * s, 4 * Cfg::GROUPS); }
        for (int s = 0; s < Cfg::NA; ++s) mbar_init(afull0 + 8u * s, 4 * Cfg::GROUPS * Cfg::CTAS);
        for (int s = 0; s < Cfg::SLOTS; ++s) { mbar_init(tfull0 + 8u * s, 1); mbar_init(tempty0 + 8u * s, kDrainWarps * Cfg::CTAS); }
        mbar_init(done_bar, 1);
        fence_mbar_init();
        tma_prefetch_desc(&tmW);
        tma_prefetch_desc(&tmC);
        tma_prefetch_desc(&tmS);
    }
    if constexpr (PAIR) {
        __syncthreads();
        cluster_sync();                               // both CTAs' barriers initialised
        if (warp == Cfg::MMA) tmem_alloc_pair(smem_u32((const void *)tmem_slot), 512);
    } else {
        if (warp == Cfg::MMA) { tmem_alloc(smem_u32((const void *)tmem_slot), 512); tmem_relinquish(); }
    }
    // launched as the programmatic dependent of the kernel that turns the rows into FP16, which
    // itself started after everything before it: only what that kernel writes has to be waited for
    if (a.p.ends) {
        (void)load_groups(a.p.ends, a.p.G, a.p.rows, starts);
    } else if (threadIdx.x == 0) {
        starts[0] = 0;
        starts[1] = a.p.rows;
    }
    __syncthreads();
    constexpr int LT = kLRows * Cfg::CTAS;
    if (warp == 0) tile_prefix(starts, a.p.G, BC, (a.p.N + LT - 1) / LT, tpre);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const int total = uniform(tpre[a.p.G]) * a.parts;
    const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
    const int first = (int)blockIdx.x / Cfg::CTAS, step = (int)gridDim.x / Cfg::CTAS;
    auto tile = [&](int t) { return i8_tile_at<BC, PAIR>(t, a, starts, tpre, rank); };

    if (warp < kDrainWarps) {
        // ---------------- accumulators -> integer sums -> results.  A warp has a quarter
        // of the lanes and WC of each half's columns
        registers_drain<PAIR>();
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
            int acc[Cfg::HALVES * Cfg::WC];
#pragma unroll
            for (int j = 0; j < Cfg::HALVES * Cfg::WC; ++j) acc[j] = 0;
            for (int c = 0; c < nch && ok; ++c) {
#pragma unroll
                for (int h = 0; h < Cfg::HALVES; ++h) {
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
                    if (lane == 0) {
                        if constexpr (PAIR) mbar_arrive_peer(peer_addr(tempty0 + 8u * s, 0));
                        else mbar_arrive(tempty0 + 8u * s);
                    }
                    ++u;
                }
            }
            if (!ok) break;
            const int64_t row0 = (int64_t)starts[x.g] + x.c0;
            if (a.parts > 1) {
                // sums of the parts: integer additions, the same in any order; the warp that adds
                // the last part goes on with the whole
#pragma unroll
                for (int h = 0; h < Cfg::HALVES; ++h) {
                    int32_t *to = a.sums + (row0 + (h ? x.n[0] : 0) + w0) * a.p.N + l + lane;
                    const int cols = (h ? x.cols - x.n[0] : min(x.n[0], x.cols)) - w0;
#pragma unroll
                    for (int j = 0; j < Cfg::WC; ++j)
                        if (j < cols && l + lane < a.p.N) atomicAdd(to + (int64_t)j * a.p.N, acc[h * Cfg::WC + j]);
                }
                __threadfence();
                __syncwarp();
                uint32_t before = 0;
                if (lane == 0) before = atomicAdd(a.tickets + (int64_t)x.tile * (kDrainWarps * Cfg::CTAS) + rank * kDrainWarps + warp, 1u);
                if (__shfl_sync(0xFFFFFFFFu, before, 0) != (uint32_t)a.parts - 1u) continue;
                __threadfence();
#pragma unroll
                for (int h = 0; h < Cfg::HALVES; ++h) {
                    const int32_t *from = a.sums + (row0 + (h ? x.n[0] : 0) + w0) * a.p.N + l + lane;
                    const int cols = (h ? x.cols - x.n[0] : min(x.n[0], x.cols)) - w0;
#pragma unroll
                    for (int j = 0; j < Cfg::WC; ++j)
                        if (j < cols && l + lane < a.p.N) acc[h * Cfg::WC + j] = __ldcg(from + (int64_t)j * a.p.N);
                }
            }
            if (l >= a.p.N) continue;
            const float ws = a.p.wscales && l + lane < a.p.N ? __ldg(a.p.wscales + (int64_t)x.g * a.p.N + l + lane) : 1.0f;
#pragma unroll
            for (int h = 0; h < Cfg::HALVES; ++h) {
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
                }
            }
        }
    } else if (warp < Cfg::TMAW) {
        // ---------------- weights: bytes of shared memory -> FP16 in tensor memory.  Lane: one
        // feature; group b of four warps takes K-block b of a stage
        registers_convert<PAIR>();
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
                const bool there = k + mine * kKB < nk;
                uint4 w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = lds_u4(from + s * (uint32_t)Cfg::W_STAGE + (uint32_t)(((mine * 4 + j) ^ (row & 7)) << 4));
                __syncwarp();
                if (lane == 0) mbar_arrive(wempty0 + 8u * s);
                if (++s == Cfg::NW) { s = 0; ph ^= 1u; }
                const uint32_t to = lanes + i % Cfg::NA * 64u + (uint32_t)mine * 32u, before = i - Cfg::NA;
                uint32_t f[16];
                half_block(w[0], w[1], f);
                if (i >= Cfg::NA && !(ok = warp_wait(used0 + 8u * (before % Cfg::NC), (before / Cfg::NC) & 1u, flags))) break;
                tc_fence_after();
                if (there) {
                    tmem_store16(to, f);
                    half_block(w[2], w[3], f);
                    tmem_store16(to + 16u, f);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) mbar_arrive_peer(peer_addr(afull0 + 8u * (i % Cfg::NA), 0));
                    else mbar_arrive(afull0 + 8u * (i % Cfg::NA));
                }
            }
        }
    } else {
        registers_issue<PAIR>();
        if (warp == Cfg::TMAW && lane == 0) {
            // ---------------- TMA: the weights' bytes
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
                for (int h = 0; h < Cfg::HALVES; ++h) {
                    const int n = x.n[h] / Cfg::CTAS;
                    row[h] = starts[x.g] + x.c0 + (h ? x.n[0] : 0) + rank * n;
                    big[h] = n > 16;
                    bytes += n ? (uint32_t)((big[h] ? 64 : 16) * kKB * 2) : 0u;
                }
                for (int k = 0; k < x.nk; k += kWK) {
                    if (!(ok = mbar_wait(used0 + 8u * s, ph ^ 1u, flags))) break;
                    const uint32_t fb = cfull0 + 8u * s, bar = PAIR ? peer_addr(fb, 0) : fb;
                    const int blocks = k + kKB < x.nk ? 2 : 1;
                    if (rank == 0) mbar_arrive_expect_tx(fb, bytes * Cfg::CTAS * (uint32_t)blocks);
                    for (int b = 0; b < blocks; ++b)
#pragma unroll
                        for (int h = 0; h < Cfg::HALVES; ++h)
                            if (x.n[h])
                                tma_load_4d<PAIR>(base + s * Cfg::C_STAGE + (uint32_t)(b * Cfg::C_BLOCK + h * Cfg::C_HALF),
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
            uint32_t cs = 0, cph = 0, as = 0, aph = 0, s0 = 0, s1 = 1 % Cfg::SLOTS, e0 = 1, e1 = 1;
            bool ok = true;
            auto next = [&]() {
                s0 = s1;
                e0 = e1;
                if (++s1 == Cfg::SLOTS) { s1 = 0; e1 ^= 1u; }
            };
            for (int t = first; t < total && ok; t += step) {
                const I8Tile x = tile(t);
                const int nk = uniform(x.nk);
                const uint32_t n0 = (uint32_t)uniform(x.n[0]), n1 = Cfg::HALVES == 2 ? (uint32_t)uniform(x.n[1]) : 0u;
                const uint32_t i0 = idesc_f16(kLRows * Cfg::CTAS) | n0 >> 3 << 17, i1 = idesc_f16(kLRows * Cfg::CTAS) | n1 >> 3 << 17;
                for (int k = 0; k < nk; k += kWK) {
                    const int kc = k % kI8Chunk;
                    const bool two = k + kKB < nk;
                    if (!(ok = warp_wait(cfull0 + 8u * cs, cph, flags))) break;
                    if (kc == 0 && !(ok = warp_wait(tempty0 + 8u * s0, e0, flags))) break;
                    if (!(ok = warp_wait(afull0 + 8u * as, aph, flags))) break;
                    tc_fence_after();
                    const uint32_t st = (base + cs * (uint32_t)Cfg::C_STAGE) >> 4, at = tmem + (uint32_t)Cfg::A0 + as * 64u;
                    mma_block<PAIR>(elected, tmem + s0 * (uint32_t)Cfg::HC, at, st, i0, kc != 0);
                    if (two) mma_block<PAIR>(elected, tmem + s0 * (uint32_t)Cfg::HC, at + 32u, st + (uint32_t)(Cfg::C_BLOCK >> 4), i0, 1);
                    // a sum's last stage: the first half is read while the second one is still multiplied
                    const bool whole = kc == kI8Chunk - kWK || k + kWK >= nk;
                    if (n1) {
                        if (whole) commit_elected<PAIR>(elected, tfull0 + 8u * s0);
                        if (kc == 0) {
                            if (!(ok = warp_wait(tempty0 + 8u * s1, e1, flags))) break;
                            tc_fence_after();
                        }
                        const uint32_t sh = st + (uint32_t)(Cfg::C_HALF >> 4);
                        mma_block<PAIR>(elected, tmem + s1 * (uint32_t)Cfg::HC, at, sh, i1, kc != 0);
                        if (two) mma_block<PAIR>(elected, tmem + s1 * (uint32_t)Cfg::HC, at + 32u, sh + (uint32_t)(Cfg::C_BLOCK >> 4), i1, 1);
                    }
                    commit_elected<PAIR>(elected, used0 + 8u * cs);
                    if (++as == Cfg::NA) { as = 0; aph ^= 1u; }
                    if (++cs == Cfg::NC) { cs = 0; cph ^= 1u; }
                    if (whole) {
                        if (n1) next();
                        commit_elected<PAIR>(elected, tfull0 + 8u * s0);
                        next();
                    }
                }
            }
            commit_elected<PAIR>(elected, done_bar);
            (void)mbar_wait(done_bar, 0, flags);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();               // the leader's MMAs are done with both CTAs
    if (warp == Cfg::MMA) {
        __syncwarp();
        tc_fence_after();
        if constexpr (PAIR) tmem_dealloc_pair(tmem, 512);
        else tmem_dealloc(tmem, 512);
    }
}

// ------------------------------------------------------- the rows as FP16
struct ExpandArgs {
    I8Product p;
    uint16_t *plane;                  // [rows][ld], in group order
    int64_t ld;
    float *xs;                        // [rows]
    uint4 *clear;                     // sums and tickets
    int64_t clear_n;
    int per, chunks;                  // codes of a row that a warp takes at once (512 or 2048), such parts of a row
    int own_flags;                    // block 0 looks at all rows and sets the flag word
};

// 16 codes a lane.  Bound by HBM and L2: one byte read and two written an element.
template <bool WIDE>
__global__ void __launch_bounds__(256) i8_expand_kernel(const ExpandArgs a)
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
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.clear_n; i += (int64_t)gridDim.x * 256) a.clear[i] = make_uint4(0u, 0u, 0u, 0u);
    const int64_t units = (int64_t)p.rows * a.chunks;
    for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < units; i += (int64_t)gridDim.x * 8) {
        const int64_t r = i / a.chunks;
        const int first = (int)(i - r * a.chunks) * a.per;
        const int64_t t = p.src ? __ldg(p.src + r) : r;
        const bool there = t >= 0 && t < p.xrows;
        if (lane == 0 && first == 0) {
            a.xs[r] = !there ? 0.0f : p.xscales ? __ldg(p.xscales + t) : 1.0f;
            if (!there && !a.own_flags) atomicOr(p.flags, (uint32_t)EMU_FLAG_INDEX);
        }
        const int8_t *x = p.X + (there ? t : 0) * p.ldx;
        uint16_t *out = a.plane + r * a.ld;
        constexpr int B = 4;                          // pieces loaded before the first is stored
        uint4 v[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int k = first + lane * 16 + 512 * b;
            v[b] = make_uint4(0u, 0u, 0u, 0u);
            if (there && 512 * b < a.per && k < p.K) v[b] = load_codes<WIDE>(x + k, p.K - k);
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int k = first + lane * 16 + 512 * b;
            if (512 * b >= a.per || k >= p.K) break;
            uint4 f[2];
            codes_f16(v[b].x, f[0].x, f[0].y);
            codes_f16(v[b].y, f[0].z, f[0].w);
            codes_f16(v[b].z, f[1].x, f[1].y);
            codes_f16(v[b].w, f[1].z, f[1].w);
            *reinterpret_cast<uint4 *>(out + k) = f[0];
            if (k + 8 < a.ld) *reinterpret_cast<uint4 *>(out + k + 8) = f[1];
        }
    }
}

// Rows of weights that TMA cannot read: a copy with rows on 16 bytes (the bytes between are not read).
__global__ void __launch_bounds__(256) i8_copy_kernel(const int8_t *W, int64_t ldw, int64_t stridew, int64_t rows, int64_t N,
                                                      int K, int8_t *out, int64_t ld)
{
    const int lane = (int)lane_id();
    for (int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += (int64_t)gridDim.x * 8) {
        const int8_t *w = W + r / N * stridew + r % N * ldw;
        for (int64_t k = lane * 16; k < K; k += 512) *reinterpret_cast<uint4 *>(out + r * ld + k) = load_codes<false>(w + k, (int)(K - k));
    }
}

bool make_code_map(CUtensorMap *map, const int8_t *W, int64_t K, int64_t N, int64_t G, int64_t ld, int64_t stride)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)K, (cuuint64_t)N, (cuuint64_t)G};
    cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)(G > 1 ? stride : N * ld)};
    cuuint32_t box[3] = {kWK, kLRows, 1}, estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<int8_t *>(W), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Which tiles: 256 columns on a pair of SMs, or 64 on one with K in parts while SMs are free; by
// waves times the nanoseconds of 64 codes (measured, weights from HBM: a pair's 290 up to 128 columns and 410
// up to 256, one SM's 240).  32 experts of 2048 x 4096: 1024 rows 63 us with 64 columns and 66 with pairs, 4096 rows 118
// and 88; 512 rows x 4096 x 4096 30 and 32, 1024 rows 55 and 34.
struct Plan {
    bool pair;
    int parts;
    int64_t tiles;
};
Plan plan(int64_t G, int64_t rows, int64_t N, int64_t K)
{
    auto waves = [](int64_t tiles, int64_t units) { return (tiles + units - 1) / units; };
    const int64_t sms = 152, n = (rows + G - 1) / G, least = G * ((n + 63) / 64) * ((N + 127) / 128);
    const int64_t t256 = waves(G * ((n + 255) / 256) * ((N + 255) / 256), sms / 2) * (n <= 128 ? 290 : 410);
    Plan x;
    x.pair = t256 < waves(least, sms) * 240;
    x.tiles = max_tiles(rows, G, N, x.pair ? 256 : 64, x.pair ? 2 : 1);
    x.parts = 1;
    if (!x.pair) {
        int64_t parts = sms / least;
        if (parts > K / 512) parts = K / 512;
        if (parts > 1) x.parts = (int)(parts > 16 ? 16 : parts);
    }
    return x;
}

struct Layout {
    int64_t plane, xs, clear, clear_bytes, copy, bytes;       // offsets behind the header
    int64_t ld, ldcopy;
};
Layout layout(int64_t G, int64_t rows, int64_t N, int64_t K, bool aligned)
{
    const Plan x = plan(G, rows, N, K);
    Layout y = {};
    y.ld = up(K, 8);
    y.ldcopy = up(K, 16);
    y.plane = 0;
    y.xs = y.plane + up(rows * y.ld * 2, 256);
    y.clear = y.xs + up(rows * 4, 256);
    y.clear_bytes = x.parts > 1 ? up(x.tiles * kDrainWarps * 4, 256) + up(rows * N * 4, 256) : 0;
    y.copy = y.clear + y.clear_bytes;
    y.bytes = y.copy + (aligned ? 0 : G * N * y.ldcopy);
    return y;
}

template <int BC, bool PAIR>
cudaError_t run(const CUtensorMap &tw, const CUtensorMap &tc, const CUtensorMap &ts, const I8TileArgs &a, int64_t tiles, cudaStream_t st)
{
    using Cfg = I8Cfg<BC, PAIR>;
    if constexpr (PAIR) {
        // the warps' shares of the registers have to fit what the launch has, or they would be waited for without end
        static std::atomic<int> fit{0};
        if (fit.load(std::memory_order_relaxed) == 0) {
            cudaFuncAttributes at;
            const cudaError_t e = cudaFuncGetAttributes(&at, i8_tile_kernel<BC, PAIR>);
            if (e != cudaSuccess) return e;
            fit.store(at.numRegs * Cfg::THREADS >= kSplitRegisters ? 1 : -1, std::memory_order_relaxed);
        }
        if (fit.load(std::memory_order_relaxed) < 0) return cudaErrorLaunchOutOfResources;
    }
    return launch_persistent<i8_tile_kernel<BC, PAIR>>(Cfg::SMEM, Cfg::THREADS, Cfg::CTAS, tiles * a.parts, st, tw, tc, ts, a);
}

}  // namespace

size_t i8_tile_scratch_bytes(int64_t G, int64_t rows, int64_t N, int64_t K, bool aligned)
{
    return (size_t)layout(G, rows, N, K, aligned).bytes;
}

// scratch: i8_tile_scratch_bytes, 16-byte aligned.
cudaError_t launch_i8_tile(I8Product p, void *scratch, cudaStream_t st)
{
    const bool aligned = i8_tma_reads(p.W, p.G, p.N, p.ldw, p.stridew);
    const Layout y = layout(p.G, p.rows, p.N, p.K, aligned);
    const Plan x = plan(p.G, p.rows, p.N, p.K);
    char *s = static_cast<char *>(scratch);
    I8TileArgs a = {};
    a.xs = reinterpret_cast<float *>(s + y.xs);
    a.parts = x.parts;
    a.tickets = reinterpret_cast<uint32_t *>(s + y.clear);
    a.sums = reinterpret_cast<int32_t *>(s + y.clear + up(x.tiles * kDrainWarps * 4, 256));
    const int64_t wrows = (int64_t)p.G * p.N;
    if (!aligned) {
        int8_t *copy = reinterpret_cast<int8_t *>(s + y.copy);
        const int64_t blocks = (wrows + 7) / 8;
        i8_copy_kernel<<<(unsigned)(blocks > 152 * 16 ? 152 * 16 : blocks), 256, 0, st>>>(p.W, p.ldw, p.G > 1 ? p.stridew : 0, wrows,
                                                                                        p.N, p.K, copy, y.ldcopy);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        p.W = copy;
        p.ldw = y.ldcopy;
        p.stridew = p.N * y.ldcopy;
    }
    a.p = p;
    uint16_t *plane = reinterpret_cast<uint16_t *>(s + y.plane);
    CUtensorMap tw, tc, ts;
    if (!make_code_map(&tw, p.W, p.K, p.N, p.G, p.ldw, p.stridew) ||
        !make_group_map(&tc, plane, p.K, p.rows, 1, 1, y.ld, 0, 0, 64) || !make_group_map(&ts, plane, p.K, p.rows, 1, 1, y.ld, 0, 0, 16))
        return cudaErrorInvalidValue;
    ExpandArgs e = {};
    e.p = p; e.plane = plane; e.ld = y.ld; e.xs = reinterpret_cast<float *>(s + y.xs);
    e.clear = reinterpret_cast<uint4 *>(s + y.clear); e.clear_n = y.clear_bytes / 16;
    e.own_flags = p.rows <= 4096;
    if (!e.own_flags) {
        const cudaError_t c = cudaMemsetAsync(p.flags, 0, sizeof(uint32_t), st);
        if (c != cudaSuccess) return c;
    }
    // short pieces while there are not warps enough
    e.per = (int64_t)p.rows * ((p.K + 2047) / 2048) < 152 * 32 ? 512 : 2048;
    e.chunks = (p.K + e.per - 1) / e.per;
    int64_t blocks = ((int64_t)p.rows * e.chunks + 7) / 8;
    if (blocks < e.clear_n / 512) blocks = e.clear_n / 512;
    const unsigned grid = (unsigned)(blocks > 152 * 8 ? 152 * 8 : blocks);
    if (aligned_codes(p.X, p.xrows > 1 ? p.ldx : 0, 0)) i8_expand_kernel<true><<<grid, 256, 0, st>>>(e);
    else i8_expand_kernel<false><<<grid, 256, 0, st>>>(e);
    const cudaError_t c = cudaGetLastError();
    if (c != cudaSuccess) return c;
    return x.pair ? run<256, true>(tw, tc, ts, a, x.tiles, st) : run<64, false>(tw, tc, ts, a, x.tiles, st);
}

}  // namespace emu
