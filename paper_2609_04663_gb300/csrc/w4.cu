// Matrix-vector products with 4-bit weights and group scales, for one row or
// a few rows of each expert:
//
//   Y[r, n] = sum_k X[r, k] (q[g, n, k] - z[g, n, k / group]) s[g, n, k / group]
//
// with q the unsigned 4-bit codes, z = 8 without zero points, g the expert
// that owns row r.  Bound by reading the weights once (N K / 2 bytes and the
// scales); the arithmetic has to stay below about 22 issue slots per 1024
// weights and SM to keep up, which plain FP32 multiply-adds per row do not.
//
// So the products run on the warp-level BF16 tensor instruction (m16n8k16,
// FP32 accumulators): the codes q - z are integers of at most 15 and exact in
// BF16, 16 features are its rows, and its 8 columns are BF16 rows of X, or the
// three BF16 slices (Eq. (fp32split)) of FP32 rows, whose products are exact as
// well.  (tcgen05 could take decoded weights as its A operand from tensor memory,
// written there by the decoding warps; that form has not been built.)  A code
// pair becomes BF16 by one or-with-mask (128 + q) and one multiply-add that
// takes 128 + z off; since a dot product may take its k in any order, the pairs are the
// nibbles i and i + 4 of a word, and X is staged in that order.  Sums of one
// scale group are scaled and added in FP32.
//
// A CTA takes 32 features; its 4 or 8 warps take a part of K each, on their own
// until their sums are added through shared memory in a fixed order.  A warp
// streams its codes, scales and zero points with 16-byte asynchronous copies
// into a ring and tables of its own, so no wait is a spin, and reads X's columns
// from L1 and L2: BF16 rows as they are, FP32 rows (or such that allow no 16-byte
// reads) as slices that a small kernel has split and put in pair order before.
// What holds it: shifts, masks and multiply-adds of the decoding take 2 clocks
// per warp instruction, two pipes together about half of the 164 clocks that a
// scheduler spends on 1024 weights; leaving any one part out (decoding, MMAs, X,
// copies) saves 2-22 %, so the rest is latency at the 4 warps per scheduler that
// registers allow (more warps spill and are slower; 16 features per CTA: 29 us
// for the 16 rows; K split over a cluster with X staged for 256 features: 28 us
// and 53 us for 7 FP32 rows).
// Measured (GPU time, weights from HBM): 1 row x 4096 x 4096 5.9 us; 1 row x 16384 x
// 16384 44-47 us (2.8-3.1 TB/s of weights); 16 rows over 12 experts of 2048 x 4096 25 us;
// 7 FP32 rows x 16384 x 8192 42 us with the slices' and the flags' kernels.
#include "grouped_common.cuh"
#include "expert_launchers.cuh"
#include "split_f32_pair.cuh"

namespace emu {

namespace {

constexpr int kRows = 32;                             // features per CTA
constexpr int kStageK = 128;                          // k of one ring stage: 64 bytes of codes per row
constexpr int kStages = 4;
constexpr int kStageBytes = kRows * kStageK / 2;
constexpr int kPassK = 1024;                          // k of a warp for which scales are held at once

struct W4Args {
    const void *X;            // rows of X, or planes: column c (row c / S, slice c % S) at c * K
    int64_t ldx;
    const uint8_t *q;
    const void *scales;
    const uint8_t *zeros;
    const int32_t *ends;      // NULL: one matrix, all rows
    void *Y;
    int64_t ldy;
    int G, rows, N, K, group, slice, tokens;          // slice: k per warp; tokens: rows of X per item at most
    int S;                                            // slices of a row: columns per row
    int sp, zp;                                       // row pitches of the held scales and zero points
    int y_f32, s_f32;
};

// The first n of 16 bytes from src (16-byte aligned), the rest zeros.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, int n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A value at byte `at` of shared memory, by an ordinary load: unlike volatile
// assembly it may move between the products of earlier blocks.
template <typename T>
__device__ __forceinline__ T shared_at(const uint8_t *smem, uint32_t at) { return *reinterpret_cast<const T *>(smem + at); }

// Codes of nibbles s / 4 and s / 4 + 4 of w, minus the zero point (as the pair
// -(128 + z)), as a BF16 pair.  One three-input logic operation with both masks
// in registers (written with operators it becomes two), one multiply-add by one.
__device__ __forceinline__ uint32_t decode(uint32_t w, int s, uint32_t zero)
{
    uint32_t p, d;                                                  // BF16 128 + q: (w & mask) | magic
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(p) : "r"(w >> s), "r"(0x000F000Fu), "r"(0x43004300u));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(p), "r"(0x3F803F80u), "r"(zero));
    return d;
}

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same with a zero accumulator.
__device__ __forceinline__ void mma16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// 8 consecutive BF16 as pairs (0,4) (1,5) (2,6) (3,7).
__device__ __forceinline__ uint4 pair_order(uint32_t w01, uint32_t w23, uint32_t w45, uint32_t w67)
{
    return make_uint4(__byte_perm(w01, w45, 0x5410), __byte_perm(w01, w45, 0x7632), __byte_perm(w23, w67, 0x5410),
                      __byte_perm(w23, w67, 0x7632));
}

// Row pitch of the held scales or zero points of one pass: an odd number of
// 16-byte pieces, so that the 8 rows that a warp reads at once lie in
// different banks.  A pass holds pass / group groups where slices and passes
// start on whole ones, part of one where slices divide groups, and may begin
// and end within groups otherwise.
int meta_pitch(int pass, int group, int slice, int size)
{
    const int n = slice % group == 0 && pass % group == 0 ? pass / group : group % slice == 0 ? 1 : pass / group + 2;
    return ((n * size + 15) / 16 | 1) * 16;
}

// Starts a call's flag word with what its ends say.  A launch of its own: within
// the products it costs registers (7 FP32 rows x 16384 x 8192: 43.7 us against 42.0, without
// flags 41.1), and here it overlaps the rows' split.
__global__ void __launch_bounds__(256) w4_flags_kernel(const int32_t *__restrict__ ends, int G, int rows, uint32_t *flags)
{
    __shared__ int starts[kMaxGroups + 1];
    griddep_launch_dependents();
    const bool bad = ends && load_groups(ends, G, rows, starts);
    if (threadIdx.x == 0) *flags = bad ? (uint32_t)EMU_FLAG_INDEX : 0u;
}

// FP32 rows (or BF16 rows of any alignment) -> planes in pair order, 8 k a thread.
// FP32: values whose slices are not finite are flagged.
template <bool F32X>
__global__ void __launch_bounds__(256) w4_planes_kernel(const void *__restrict__ X, int64_t ldx, int rows, int K,
                                                        uint16_t *__restrict__ planes, uint32_t *flags)
{
    griddep_launch_dependents();
    const int octets = K / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    uint32_t amax = 0;
    if (i < (int64_t)rows * octets) {
        const int64_t r = i / octets, k = (i - r * octets) * 8;
        constexpr int S = F32X ? 3 : 1;
        uint32_t w[3][4];
        if constexpr (F32X) {
            const float *x = static_cast<const float *>(X) + r * ldx + k;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u = __ldg(x + 2 * e), v = __ldg(x + 2 * e + 1);
                amax = abs_bits_max(amax, u, v);
                split_pair(u, v, w[0][e], w[1][e], w[2][e]);
            }
        } else {
            const uint16_t *x = static_cast<const uint16_t *>(X) + r * ldx + k;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[0][e] = (uint32_t)__ldg(x + 2 * e) | (uint32_t)__ldg(x + 2 * e + 1) << 16;
        }
#pragma unroll
        for (int s = 0; s < S; ++s)
            *reinterpret_cast<uint4 *>(planes + (r * S + s) * K + k) = pair_order(w[s][0], w[s][1], w[s][2], w[s][3]);
    }
    griddep_wait();                                       // the flag word has been started
    if constexpr (F32X) publish_f32_flags(amax, flags);
}

// NT: tiles of 8 columns; DIRECT: X as rows, not planes.  GB: 32-k blocks of a
// scale group within a stage of 4: 1 or 2 (groups of 32 or 64), 4 (multiples of
// 128); 0: any other group, with its bounds looked for.
template <int NT, bool DIRECT, int GB, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, 16 / kWarps) w4_kernel(const W4Args a)
{
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t rings = 0, sbase = smem_u32(smem);     // shared addresses are offsets from smem
    const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = (int)lane_id(), lr = lane >> 2, lc = lane & 3;
    const int n0 = (int)blockIdx.x * kRows;

    // ---- the item: rows [row0, row0 + m) of X, all of one expert
    int g = 0, row0 = 0, m = a.rows;
    if (a.ends) {
        int *starts = reinterpret_cast<int *>(smem), *item = starts + a.G + 1;     // the rings' memory, before its use
        (void)load_groups(a.ends, a.G, a.rows, starts);
        if (warp == 0) {
            int want = (int)blockIdx.y, found = -1;
            for (int g0 = 0; g0 < a.G; g0 += 32) {
                const int e = g0 + lane;
                const int c = e < a.G ? (starts[e + 1] - starts[e] + a.tokens - 1) / a.tokens : 0;
                int sum = c;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int u = __shfl_up_sync(0xFFFFFFFFu, sum, d);
                    if (lane >= d) sum += u;
                }
                const uint32_t hit = __ballot_sync(0xFFFFFFFFu, sum > want);
                if (hit) {
                    const int at = __ffs(hit) - 1;
                    found = g0 + at;
                    want -= __shfl_sync(0xFFFFFFFFu, sum - c, at);
                    break;
                }
                want -= __shfl_sync(0xFFFFFFFFu, sum, 31);
            }
            if (lane == 0) { item[0] = found; item[1] = want; }
        }
        __syncthreads();
        g = item[0];
        const int chunk = item[1];
        if (g >= 0) {
            row0 = starts[g] + chunk * a.tokens;
            m = min(a.tokens, starts[g + 1] - row0);
        } else {
            // no item left: the first CTA without one clears the rows of no group
            if (chunk == 0) {
                const int n = n0 + lane;
                for (int64_t r = starts[a.G] + warp; r < a.rows; r += kWarps)
                    if (n < a.N) {
                        if (a.y_f32) static_cast<float *>(a.Y)[r * a.ldy + n] = 0.0f;
                        else static_cast<uint16_t *>(a.Y)[r * a.ldy + n] = 0;
                    }
            }
            if (!DIRECT) griddep_wait();              // this launch may not end before the planes' kernel has
            return;
        }
        __syncthreads();                              // the tables are read, the rings may be filled
    } else {
        row0 = (int)blockIdx.y * a.tokens;
        m = min(a.tokens, a.rows - row0);
    }
    const int cols = m * a.S, gb = a.group / 32, ngroups = a.K / a.group;
    const int ssize = a.s_f32 ? 4 : 2, sp = a.sp, zp = a.zp;
    const uint32_t ring = rings + (uint32_t)(warp * kStages * kStageBytes);
    const uint32_t sc = rings + (uint32_t)(kWarps * kStages * kStageBytes + warp * kRows * (sp + (a.zeros ? zp : 0)));
    const uint32_t zs = sc + (uint32_t)(kRows * sp);
    const int k0 = warp * a.slice, k1 = min(a.K, k0 + a.slice);
    const int nst = k1 > k0 ? (k1 - k0 + kStageK - 1) / kStageK : 0;

    // ---- this warp's ring: rows n0 .. n0 + 31, 16-byte piece j of a row at piece j ^ (row / 2 % 4);
    // a lane copies piece lane % 4 of rows lane / 4 + 8 i.  Rows past the last
    // feature read that one again (their sums go nowhere), pieces past the slice
    // are not copied (nor read).
    const int pitch = a.K / 2, tail = (k1 - k0) % kStageK / 32;       // blocks of a last stage that is not whole
    const uint8_t *qp[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        qp[i] = a.q + ((int64_t)g * a.N + min(n0 + lr + 8 * i, a.N - 1)) * pitch + k0 / 2 + lc * 16;
    uint32_t qdst = sbase + ring + (uint32_t)(lr * 64 + ((lc ^ (lr >> 1 & 3)) << 4));
    int asked = 0;                                    // stages asked for
    auto fetch = [&]() {                              // the next one, if there is one
        if (asked < nst && (tail == 0 || asked < nst - 1 || lc < tail)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(qdst + (uint32_t)(i * 512)), "l"(qp[i]) : "memory");
        }
        cp_async_commit();
#pragma unroll
        for (int i = 0; i < 4; ++i) qp[i] += kStageK / 2;
        qdst = (++asked & (kStages - 1)) == 0 ? qdst - (kStages - 1) * kStageBytes : qdst + kStageBytes;
    };
    static_assert((kStages & (kStages - 1)) == 0, "ring stages");
    // n scales or zero points of each feature from group g0 on -> rows of pitch
    // dpitch at dst, by 16-byte copies where the source rows allow it
    auto meta = [&](uint32_t dst, int dpitch, const void *src, int size, int g0, int n) {
        const uint8_t *from = static_cast<const uint8_t *>(src) + (((int64_t)g * a.N + n0) * ngroups + g0) * size;
        const int64_t rowb = (int64_t)ngroups * size;
        const int pieces = dpitch / 16;               // past the n values: zeros
        const uint32_t inv = 65536u / (uint32_t)pieces + 1u;       // i / pieces for i < 4096, pieces < 16
        // whole pieces only: a row's last piece may not run into what follows the array
        const bool wide = ((reinterpret_cast<uintptr_t>(from) | (uintptr_t)rowb) & 15u) == 0;
        for (int i = lane; i < kRows * pieces; i += 32) {
            const int r = pieces < 16 ? (int)((uint32_t)i * inv >> 16) : i / pieces, o = (i - r * pieces) * 16;
            const bool ok = n0 + r < a.N;
            const uint32_t to = sbase + dst + (uint32_t)(r * dpitch + o);
            if (wide) {
                const int len = ok ? min(max(n * size - o, 0), 16) : 0;
                cp_async16(to, len ? from + r * rowb + o : a.q, len);
            } else {
                const int len = ok ? n * size - o : 0;
                for (int b = 0; b < 16; b += size) {
                    const uint8_t *p = from + r * rowb + o + b;
                    if (size == 4) {
                        const uint32_t v = b < len ? __ldg(reinterpret_cast<const uint32_t *>(p)) : 0u;
                        asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + b), "r"(v) : "memory");
                    } else if (size == 2) {
                        const uint16_t v = b < len ? __ldg(reinterpret_cast<const uint16_t *>(p)) : (uint16_t)0;
                        asm volatile("st.shared.b16 [%0], %1;" ::"r"(to + b), "h"(v) : "memory");
                    } else {
                        const uint16_t v = b < len ? __ldg(p) : (uint16_t)0;
                        asm volatile("st.shared.b8 [%0], %1;" ::"r"(to + b), "h"(v) : "memory");
                    }
                }
            }
        }
    };
    // ---- X's columns of this lane: 8 k of column 8 t + lr per block of 32 (columns
    // that are not there read the first one: no other column sees them)
    const uint8_t *xp[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int c = t * 8 + lr < cols ? t * 8 + lr : 0;
        xp[t] = static_cast<const uint8_t *>(a.X) +
                ((DIRECT ? (row0 + c) * a.ldx : ((int64_t)row0 * a.S + c) * a.K) + k0) * 2 + lc * 16;
    }
    // kAhead blocks of X are on their way: with one tile a whole stage's (16 rows
    // over 12 experts 25 us against 30 with one block); with three tiles two
    // already spill (7 FP32 rows 47 us against 41)
    constexpr int kAhead = GB == 0 || NT == 3 ? 1 : 4;
    int ahead = (k1 - k0) / 32;                       // blocks of X still to be loaded
    uint4 xn[kAhead][NT];
    auto load_x = [&](int slot) {
        if (--ahead >= 0) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                xn[slot][t] = __ldg(reinterpret_cast<const uint4 *>(xp[t]));
                xp[t] += 64;
            }
        }
    };

    float total[2][NT][4], part[2][NT][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) total[i][t][e] = part[i][t][e] = 0.0f;

    for (int st0 = 0; st0 < nst; st0 += kPassK / kStageK) {
        // ---- scales and zero points of this pass
        const int p0 = k0 + st0 * kStageK, p1 = min(k1, p0 + kPassK), g0 = p0 / a.group;
        const int ng = (p1 - 1) / a.group - g0 + 1;
        __syncwarp();                                 // the pass before has been read
        meta(sc, sp, a.scales, ssize, g0, ng);
        if (a.zeros) meta(zs, zp, a.zeros, 1, g0, ng);
        cp_async_commit();
        if (st0 == 0) {
#pragma unroll
            for (int st = 0; st < kStages; ++st) fetch();
            if (!DIRECT) griddep_wait();              // the planes: all else was there before their kernel
#pragma unroll
            for (int i = 0; i < kAhead; ++i) load_x(i);
        } else {
            cp_async_wait<0>();                       // these came last
        }
        for (int st = st0; st < min(nst, st0 + kPassK / kStageK); ++st) {
            cp_async_wait<kStages - 1>();             // this stage, and the first pass's scales before it
            __syncwarp();
            const uint32_t stage = ring + (uint32_t)((st % kStages) * kStageBytes) + (uint32_t)(lr * 64 + ((lr >> 1) << 4) + lc * 4);
            const int blocks = st == nst - 1 && tail ? tail : 4;  // 32-k blocks of this stage
            const uint32_t srow = sc + (uint32_t)(lr * sp), zrow = zs + (uint32_t)(lr * zp);
            // block b of the stage: codes of rows lr + 8 r, X's columns
            auto block = [&](int b, bool first, const uint32_t (&z)[4]) {
                uint32_t w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = shared_at<uint32_t>(smem, (stage ^ (uint32_t)(b << 4)) + (uint32_t)(r * 512));
                uint4 x[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const uint4 v = xn[b % kAhead][t];
                    x[t] = DIRECT ? pair_order(v.x, v.y, v.z, v.w) : v;
                }
                load_x(b % kAhead);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t u = w[2 * i], v = w[2 * i + 1], zu = z[2 * i], zv = z[2 * i + 1];
                    const uint32_t u0 = decode(u, 0, zu), u1 = decode(u, 4, zu), u2 = decode(u, 8, zu), u3 = decode(u, 12, zu);
                    const uint32_t v0 = decode(v, 0, zv), v1 = decode(v, 4, zv), v2 = decode(v, 8, zv), v3 = decode(v, 12, zv);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if (first) mma16816_first(part[i][t], u0, v0, u1, v1, x[t].x, x[t].y);
                        else mma16816(part[i][t], u0, v0, u1, v1, x[t].x, x[t].y);
                        mma16816(part[i][t], u2, v2, u3, v3, x[t].z, x[t].w);
                    }
                }
            };
            auto scale_up = [&](const float (&s)[4]) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            total[i][t][e] = fmaf(part[i][t][e], s[2 * i + (e >> 1)], total[i][t][e]);
            };
            if constexpr (GB > 0) {
                constexpr int NG = 4 / GB;            // scale groups of the stage
                const int go = GB == 4 ? (k0 + st * kStageK) / a.group - g0 : (st - st0) * NG;
                float s[NG][4];
                uint32_t z[NG][4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t at = srow + (uint32_t)(r * 8 * sp + go * ssize);
                    uint32_t f[4];
                    if (a.s_f32) {
                        if constexpr (NG == 4) { const uint4 v = shared_at<uint4>(smem, at); f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
                        else if constexpr (NG == 2) { const uint2 v = shared_at<uint2>(smem, at); f[0] = v.x; f[1] = v.y; }
                        else f[0] = shared_at<uint32_t>(smem, at);
                    } else {
                        uint2 v;
                        if constexpr (NG == 4) v = shared_at<uint2>(smem, at);
                        else if constexpr (NG == 2) v.x = shared_at<uint32_t>(smem, at);
                        else v.x = shared_at<uint16_t>(smem, at);
                        f[0] = v.x << 16;
                        f[1] = v.x & 0xFFFF0000u;
                        f[2] = v.y << 16;
                        f[3] = v.y & 0xFFFF0000u;
                    }
                    uint32_t q = 0x08080808u;
                    if (a.zeros) {
                        const uint32_t az = zrow + (uint32_t)(r * 8 * zp + go);
                        q = (NG == 4 ? shared_at<uint32_t>(smem, az) : NG == 2 ? (uint32_t)shared_at<uint16_t>(smem, az) : (uint32_t)smem[az]) & 0x0F0F0F0Fu;
                    }
#pragma unroll
                    for (int n = 0; n < NG; ++n) {
                        s[n][r] = __uint_as_float(f[n]);
                        z[n][r] = __byte_perm(q, 0xC3C3C3C3u, 0x4040u + 0x0101u * n);      // -(128 + z) as a BF16 pair
                    }
                }
                if (blocks == 4) {
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        block(b, b % GB == 0, z[b / GB]);
                        if (b % GB == GB - 1) scale_up(s[b / GB]);
                    }
                } else {                              // (K may end within a stage, but not within a group)
#pragma unroll
                    for (int b = 0; b < 3; ++b) {
                        if (b >= blocks) break;
                        block(b, b % GB == 0, z[b / GB]);
                        if (b % GB == GB - 1) scale_up(s[b / GB]);
                    }
                }
            } else {
                const int kb0 = (k0 + st * kStageK) / 32, kb1 = kb0 + blocks;
                for (int kb = kb0; kb < kb1;) {
                    // the part of a scale group that this stage holds
                    const int gi = kb / gb, end = min(kb1, (gi + 1) * gb);
                    float s[4];
                    uint32_t z[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t at = srow + (uint32_t)(r * 8 * sp + (gi - g0) * ssize);
                        s[r] = __uint_as_float(a.s_f32 ? shared_at<uint32_t>(smem, at) : (uint32_t)shared_at<uint16_t>(smem, at) << 16);
                        const uint32_t q = a.zeros ? smem[zrow + (uint32_t)(r * 8 * zp + gi - g0)] & 15u : 8u;
                        z[r] = __byte_perm(q, 0xC3C3C3C3u, 0x4040u);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) part[i][t][e] = 0.0f;
                    for (; kb < end; ++kb) block(kb - kb0, false, z);
                    scale_up(s);
                }
            }
            __syncwarp();
            fetch();                                  // into the stage just read
        }
    }
    cp_async_wait<0>();
    __syncthreads();                                  // the rings are free: their memory takes the sums

    // ---- the warps' sums, [warp][column][feature]; added in warp order, slices of a
    // row smallest first
    float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = t * 8 + lc * 2 + (e & 1), r = i * 16 + lr + (e >> 1) * 8;
                if (c < cols) sums[(warp * cols + c) * kRows + r] = total[i][t][e];
            }
    __syncthreads();
    const int n = n0 + lane;
    for (int t = warp; t < m; t += kWarps) {
        float y = 0.0f;
        for (int s = a.S - 1; s >= 0; --s)
#pragma unroll
            for (int w = 0; w < kWarps; ++w) y = __fadd_rn(y, sums[(w * cols + t * a.S + s) * kRows + lane]);
        if (n < a.N) {
            const int64_t o = (int64_t)(row0 + t) * a.ldy + n;
            if (a.y_f32) static_cast<float *>(a.Y)[o] = y;
            else static_cast<uint16_t *>(a.Y)[o] = (uint16_t)bf16x2_rn(y, 0.0f);
        }
    }
}

template <int NT, bool DIRECT, int GB, int kWarps>
cudaError_t run_w4(const W4Args &a, int64_t blocks, int64_t items, cudaStream_t st)
{
    constexpr auto kern = w4_kernel<NT, DIRECT, GB, kWarps>;
    const int sm = kWarps * (kStages * kStageBytes + kRows * (a.sp + (a.zeros ? a.zp : 0)));
    cudaError_t e = sm > 48 * 1024 ? cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, sm) : cudaSuccess;
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks, (unsigned)items);
    cfg.blockDim = dim3(32 * kWarps);
    cfg.dynamicSmemBytes = (size_t)sm;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = DIRECT ? 0 : 1;
    e = cudaLaunchKernelEx(&cfg, kern, a);
    if (e != cudaSuccess) return e;
    return cudaGetLastError();
}

}  // namespace

bool w4_direct(bool x_f32, const void *X, int64_t ldx)
{
    return !x_f32 && (reinterpret_cast<uintptr_t>(X) & 15u) == 0 && ldx % 8 == 0;
}

// planes: rows * K values of S = 3 (FP32) or 1 slices, unless w4_direct; flags:
// the flag word, or NULL (only with w4_direct).
cudaError_t launch_w4_matvec(bool x_f32, int64_t G, int64_t rows, int64_t N, int64_t K, int group, const void *X,
                             int64_t ldx, const uint8_t *q, const void *scales, bool s_f32, const uint8_t *zeros,
                             const int32_t *ends, void *Y, int64_t ldy, uint16_t *planes, uint32_t *flags,
                             cudaStream_t st)
{
    const bool direct = w4_direct(x_f32, X, ldx);
    W4Args a = {};
    a.X = direct ? X : planes; a.ldx = ldx; a.q = q; a.scales = scales; a.zeros = zeros; a.ends = ends; a.Y = Y; a.ldy = ldy;
    a.G = (int)G; a.rows = (int)rows; a.N = (int)N; a.K = (int)K; a.group = group;
    a.S = x_f32 ? 3 : 1; a.y_f32 = x_f32 ? 1 : 0; a.s_f32 = s_f32 ? 1 : 0;
    // rows of X per item: up to 24 columns; an expert is expected to get up to
    // twice its share of the rows (one that gets more is read again)
    const int64_t active = !ends ? 1 : (G < rows ? G : rows);
    int64_t want = ends ? 2 * ((rows + active - 1) / active) : rows;
    if (want > rows) want = rows;
    const int nt = want * a.S <= 8 ? 1 : 3;
    a.tokens = 8 * nt / a.S;
    if (a.tokens > rows) a.tokens = (int)rows;
    // where the CTAs fill the GPU, four small ones per SM overlap one's start with
    // the others' products; few take more warps each (1 row, K = 4096, 4 and 8
    // warps: N 4096 6.9 and 6.4 us, 8192 9.6 and 10.0, 16384 14.6 and 18.0; 7 FP32 rows: N
    // 4096 14.3 and 10.3, 16384 23.0 and 26.6)
    const int64_t blocks = (N + kRows - 1) / kRows;
    const int warps = blocks * active >= 2 * 152 ? 4 : 8;
    a.slice = (int)((K + warps * kStageK - 1) / (warps * kStageK) * kStageK);
    const int pass = a.slice < kPassK ? a.slice : kPassK;
    a.sp = meta_pitch(pass, group, a.slice, s_f32 ? 4 : 2);
    a.zp = meta_pitch(pass, group, a.slice, 1);
    const int64_t items = ends ? active + rows / a.tokens + 1 : (rows + a.tokens - 1) / a.tokens;
    if (items > 65535) return cudaErrorInvalidValue;
    if (flags) {
        w4_flags_kernel<<<1, 256, 0, st>>>(ends, (int)G, (int)rows, flags);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    if (!direct) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((rows * (K / 8) + 255) / 256));
        cfg.blockDim = dim3(256);
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const cudaError_t e = x_f32 ? cudaLaunchKernelEx(&cfg, w4_planes_kernel<true>, X, ldx, (int)rows, (int)K, planes, flags)
                                    : cudaLaunchKernelEx(&cfg, w4_planes_kernel<false>, X, ldx, (int)rows, (int)K, planes, flags);
        if (e != cudaSuccess) return e;
    }
#define EMU_W4W(GB, W)                                                                                                  \
    (direct ? (nt == 1 ? run_w4<1, true, GB, W>(a, blocks, items, st) : run_w4<3, true, GB, W>(a, blocks, items, st))   \
            : (nt == 1 ? run_w4<1, false, GB, W>(a, blocks, items, st) : run_w4<3, false, GB, W>(a, blocks, items, st)))
#define EMU_W4(GB) (warps == 4 ? EMU_W4W(GB, 4) : EMU_W4W(GB, 8))
    return group == 32 ? EMU_W4(1) : group == 64 ? EMU_W4(2) : group % 128 == 0 ? EMU_W4(4) : EMU_W4(0);
#undef EMU_W4
#undef EMU_W4W
}

}  // namespace emu
