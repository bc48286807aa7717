// Pieces shared by the two tensor-core kernels of the 8-bit integer products (i8_tile.cu: many
// rows, i8_batch.cu: some).  Each translation unit gets its own copies (unnamed namespace).
//
// This GPU's integer tensor rate is a small part of its FP16 rate, so the codes are
// multiplied as FP16 numbers: a code has at most 8 significant bits, a product 15, and while
// a sum has at most 1024 terms it stays within 2^24, where FP32 holds every integer.  The
// accumulators are read every 1024 terms and added as 32-bit integers in registers: all sums
// are exact.
//
// Output features lie on the MMA's rows, token rows on its columns (as in grouped.cu).  The
// weights cross HBM and L2 as bytes; eight warps turn them into FP16 and write them to tensor memory, from
// which the MMA takes its first operand: the byte u = code + 128 in the mantissa of
// 1024 + u, less 1152 (five instructions for four codes; a published method, the constants follow from FP16's layout).
#pragma once
#include "grouped_tile.cuh"
#include "i8_common.cuh"

namespace emu {

namespace {

constexpr int kI8Chunk = 1024;                        // terms of a sum that FP32 holds exactly: 2^14 each, 2^24 in all
constexpr int kWK = 128;                              // codes of a row per stage (two K-blocks)
constexpr int kDrainWarps = 8;                        // warps that read accumulators and store
constexpr int kConvertWarps = 8;                      // warps that turn weights into FP16, four for each K-block of a stage

// An output tile: features l0 .. (this CTA's 128), `cols` columns (rows of group g) from c0 on,
// MMA columns of its halves, contraction of nk codes from k0.
struct I8Tile {
    int g, l0, c0, cols, n[2], k0, nk;
};

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


// After a warp has stored its columns: zeros in those rows (bits of `gone`, from `row` on) that have no
// source.  Their sums are 0, but a channel's scale that is not finite makes NaN of them.  (Choosing between
// each product and 0 before the stores, or looking after each 32 columns of the pairs' tiles, cost 1 us of 122 for
// 8192 rows over 32 experts.)
__device__ __forceinline__ void clear_rows(const I8Product &p, int64_t row, uint32_t gone, int n)
{
    if (!gone) return;
    __syncwarp();                                     // (a row's features may have been stored by other lanes)
    for (; gone; gone &= gone - 1)
        if (n < p.N) store_value(p, row + __ffs((int)gone) - 1, n, 0.0f, 0);
}

// A converting warp's part of a stage: 64 codes of its lane's feature in shared memory at `from`
// -> FP16 in tensor memory at `to`.  In between, `wait` waits until the MMAs have used what was there; false
// when it gave up.  was_read gives the stage of bytes back to TMA: after the stores to tensor
// memory, which cannot be issued before all that was loaded has arrived.  (Right after the loads it came too
// early: an arrival does not wait for loads from shared memory, and where a box lies past the end of the rows TMA writes its zeros at
// once.  Last codes of a stage came out as zero in one of a hundred products of 1030 rows x 2064 x 700.)
template <typename Read, typename Wait>
__device__ __forceinline__ bool convert_weights(uint32_t from, int first, int row, uint32_t to, bool there, Read &&was_read, Wait &&wait)
{
    uint4 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = lds_u4(from + (uint32_t)(((first + j) ^ (row & 7)) << 4));
    uint32_t f[16];
    half_block(w[0], w[1], f);
    if (!wait()) return false;
    tc_fence_after();
    if (there) {
        tmem_store16(to, f);
        half_block(w[2], w[3], f);
        tmem_store16(to + 16u, f);
        was_read();
        tmem_st_wait();
    } else {
        was_read();                                   // (what was loaded is not used)
    }
    tc_fence_before();
    __syncwarp();
    return true;
}

// Rows of weights that TMA cannot read, and token rows that cannot be read 16 codes at a time, in
// group order: copies with rows on 16 bytes (the bytes between are not read).
struct CopyArgs {
    int64_t wrows, trows;             // rows of weights (of all groups) and of tokens to copy
    int8_t *w, *t;
    int64_t ld;
};
// Row i of the copies, by a warp.
__device__ __forceinline__ void copy_row(const I8Product &p, const CopyArgs &a, int64_t i, int lane)
{
    const int8_t *from = nullptr;
    int8_t *to = a.w + i * a.ld;
    if (i < a.wrows) {
        const int64_t g = i / p.N;
        from = p.W + g * p.stridew + (i - g * p.N) * p.ldw;
    } else {
        const int64_t r = i - a.wrows, t = p.src ? __ldg(p.src + r) : r;
        if (t >= 0 && t < p.xrows) from = p.X + t * p.ldx;
        to = a.t + r * a.ld;
    }
    for (int k = lane * 16; k < p.K; k += 512)
        *reinterpret_cast<uint4 *>(to + k) = from ? load_codes<false>(from + k, p.K - k) : make_uint4(0u, 0u, 0u, 0u);
}

// Tensor map over G matrices of N rows of K codes, boxes of 128 x 128 bytes.
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

}  // namespace

}  // namespace emu
