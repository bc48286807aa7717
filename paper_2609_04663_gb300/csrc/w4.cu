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
// well.  tcgen05 would need the decoded weights back in shared memory.  A code
// pair becomes BF16 by one or-with-mask (128 + q) and one subtraction of
// 128 + z; since a dot product may take its k in any order, the pairs are the
// nibbles i and i + 4 of a word, and X is staged in that order.  Sums of one
// scale group are scaled and added in FP32.
//
// A CTA takes 128 features and one of KS slices of K; the KS CTAs of a cluster
// add their sums through distributed shared memory in a fixed order.  Each warp
// streams its own 32 rows of codes through a ring in shared memory with
// 16-byte asynchronous copies, so no wait is a spin.
#include "grouped_common.cuh"
#include "launchers.cuh"
#include "split_f32_pair.cuh"

namespace emu {

namespace {

constexpr int kWarps = 8, kRows = 32 * kWarps;        // features per CTA
constexpr int kStageK = 128;                          // k of one ring stage: 64 bytes of codes per row
constexpr int kStageBytes = 32 * kStageK / 2;         // of one warp
// Ring stages, and k for which X and the scales are staged at once, by the
// tiles of 8 columns (two CTAs' shared memory fits an SM).
__host__ __device__ constexpr int ring_stages(int nt) { return nt == 1 ? 4 : 3; }
__host__ __device__ constexpr int pass_k(int nt) { return nt == 1 ? 1024 : 512; }

struct W4Args {
    const void *X;
    int64_t ldx;
    const uint8_t *q;
    const void *scales;
    const uint8_t *zeros;
    const int32_t *ends;      // NULL: one matrix, all rows
    void *Y;
    int64_t ldy;
    int G, rows, N, K, group, slice, tokens;          // slice: k per CTA; tokens: rows of X per item at most
    int sp, zp;                                       // row pitches of the staged scales and zero points
    int x_f32, s_f32, x_vec;                          // x_vec: X's rows can be read 16 bytes at a time
};

// The first n of 16 bytes from src (16-byte aligned), the rest zeros.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, int n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint32_t lds32(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a)
{
    uint16_t v;
    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}

// Codes of nibbles s / 4 and s / 4 + 4 of w, minus the zero point, as a BF16 pair.
__device__ __forceinline__ uint32_t decode(uint32_t w, int s, uint32_t zero)
{
    const uint32_t p = ((w >> s) & 0x000F000Fu) | 0x43004300u;      // BF16 128 + q
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(p), "r"(zero));
    return d;
}

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same with a zero accumulator.
__device__ __forceinline__ void mma16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
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

__device__ __forceinline__ void sts128(uint32_t a, uint4 v) { st_shared_v4(a, v.x, v.y, v.z, v.w); }

// Row pitch of the staged scales or zero points of one pass: an odd number of
// 16-byte pieces, so that the 8 rows that a warp reads at once lie in
// different banks.  A pass holds pass / group groups where slices and passes
// start on whole ones, part of one where slices divide groups, and may begin
// and end within groups otherwise.
int meta_pitch(int pass, int group, int slice, int size)
{
    const int n = slice % group == 0 && pass % group == 0 ? pass / group : group % slice == 0 ? 1 : pass / group + 2;
    return ((n * size + 15) / 16 | 1) * 16;
}

// NT: tiles of 8 columns; F32X: FP32 rows, three columns each.  GB: 32-k blocks
// of a scale group within a stage of 4: 1 or 2 (groups of 32 or 64), 4
// (multiples of 128); 0: any other group, with its bounds looked for.
template <int NT, bool F32X, int GB>
__global__ void __launch_bounds__(32 * kWarps, 2) w4_kernel(const W4Args a)
{
    constexpr int S = F32X ? 3 : 1, kStages = ring_stages(NT), kPassK = pass_k(NT);
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t codes = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = (int)lane_id(), lr = lane >> 2, lc = lane & 3;
    uint32_t ks, rank;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ks));
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int n0 = (int)(blockIdx.x / ks) * kRows;

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
            if (chunk == 0 && rank == 0) {
                const int n = n0 + (int)threadIdx.x;
                for (int64_t r = starts[a.G]; r < a.rows; ++r)
                    if (n < a.N) {
                        if (a.x_f32) static_cast<float *>(a.Y)[r * a.ldy + n] = 0.0f;
                        else static_cast<uint16_t *>(a.Y)[r * a.ldy + n] = 0;
                    }
            }
            return;                                   // all CTAs of the cluster take this way
        }
        __syncthreads();                              // the tables are read, the rings may be filled
    } else {
        row0 = (int)blockIdx.y * a.tokens;
        m = min(a.tokens, a.rows - row0);
    }
    const int cols = m * S, gb = a.group / 32, ngroups = a.K / a.group;
    const int ssize = a.s_f32 ? 4 : 2, sp = a.sp, zp = a.zp;
    const uint32_t xs = codes + kWarps * kStages * kStageBytes;
    const uint32_t sc = xs + (uint32_t)((kPassK / 32) * a.tokens * S * 64), zs = sc + (uint32_t)(kRows * sp);
    const int k0 = (int)rank * a.slice, k1 = min(a.K, k0 + a.slice);
    const int nst = k1 > k0 ? (k1 - k0 + kStageK - 1) / kStageK : 0;

    // ---- this warp's ring: rows n0 + 32 warp .. + 31, 16-byte piece j of a row at piece j ^ (row / 2 % 4)
    const uint32_t ring = codes + (uint32_t)(warp * kStages * kStageBytes);
    const int64_t pitch = a.K / 2;
    const uint8_t *qbase = a.q + ((int64_t)g * a.N + n0 + warp * 32) * pitch;
    auto fetch = [&](int st) {
        if (st < nst) {
            const uint32_t dst = ring + (uint32_t)((st % kStages) * kStageBytes);
            const int piece = lane & 3, byte = (k0 + st * kStageK) / 2 + piece * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = i * 8 + (lane >> 2);
                const bool ok = n0 + warp * 32 + r < a.N && byte < k1 / 2;
                cp_async16(dst + (uint32_t)(r * 64 + ((piece ^ (r >> 1 & 3)) << 4)), ok ? qbase + r * pitch + byte : a.q, ok ? 16 : 0);
            }
        }
        cp_async_commit();
    };
    // n scales or zero points of each feature from group g0 on -> rows of pitch
    // dpitch at dst, by 16-byte copies where the source rows allow it
    auto meta = [&](uint32_t dst, int dpitch, const void *src, int size, int g0, int n) {
        const uint8_t *from = static_cast<const uint8_t *>(src) + (((int64_t)g * a.N + n0) * ngroups + g0) * size;
        const int64_t rowb = (int64_t)ngroups * size;
        const int pieces = dpitch / 16;               // past the n values: zeros
        const uint32_t inv = 65536u / (uint32_t)pieces + 1u;       // i / pieces for i < 4096, pieces < 16
        // whole pieces only: a row's last piece may not run into what follows the array
        const bool wide = ((reinterpret_cast<uintptr_t>(from) | (uintptr_t)rowb) & 15u) == 0;
        for (int i = threadIdx.x; i < kRows * pieces; i += 32 * kWarps) {
            const int r = pieces < 16 ? (int)((uint32_t)i * inv >> 16) : i / pieces, o = (i - r * pieces) * 16;
            const bool ok = n0 + r < a.N;
            const uint32_t to = dst + (uint32_t)(r * dpitch + o);
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

    float total[2][NT][4], part[2][NT][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) total[i][t][e] = part[i][t][e] = 0.0f;

    for (int st0 = 0; st0 < nst; st0 += kPassK / kStageK) {
        // ---- X, scales and zero points of this pass
        const int p0 = k0 + st0 * kStageK, p1 = min(k1, p0 + kPassK), g0 = p0 / a.group;
        const int ng = (p1 - 1) / a.group - g0 + 1;
        __syncthreads();                              // the pass before has been read
        meta(sc, sp, a.scales, ssize, g0, ng);
        if (a.zeros) meta(zs, zp, a.zeros, 1, g0, ng);
        cp_async_commit();
        if (st0 == 0) {
#pragma unroll
            for (int st = 0; st < kStages; ++st) fetch(st);
        }
        // eight k of one row at a time, the loads of several in flight
        constexpr int XB = 4;
        for (int i0 = threadIdx.x; i0 < m * (kPassK / 8); i0 += 32 * kWarps * XB) {
            uint4 v[XB][S == 3 ? 2 : 1];
#pragma unroll
            for (int b = 0; b < XB; ++b) {
                const int i = i0 + b * 32 * kWarps, k = p0 + i % (kPassK / 8) * 8;
                const bool in = i < m * (kPassK / 8) && k < p1;
                const char *x = static_cast<const char *>(a.X) + ((int64_t)(row0 + i / (kPassK / 8)) * a.ldx + k) * (F32X ? 4 : 2);
#pragma unroll
                for (int h = 0; h < (F32X ? 2 : 1); ++h) {
                    v[b][h] = make_uint4(0u, 0u, 0u, 0u);
                    if (in && a.x_vec) {
                        v[b][h] = __ldg(reinterpret_cast<const uint4 *>(x) + h);
                    } else if (in && F32X) {
                        const uint32_t *u = reinterpret_cast<const uint32_t *>(x) + 4 * h;
                        v[b][h] = make_uint4(__ldg(u), __ldg(u + 1), __ldg(u + 2), __ldg(u + 3));
                    } else if (in) {
                        const uint16_t *u = reinterpret_cast<const uint16_t *>(x);
                        auto two = [&](int e) { return (uint32_t)__ldg(u + e) | (uint32_t)__ldg(u + e + 1) << 16; };
                        v[b][h] = make_uint4(two(0), two(2), two(4), two(6));
                    }
                }
            }
#pragma unroll
            for (int b = 0; b < XB; ++b) {
                const int i = i0 + b * 32 * kWarps, o = i % (kPassK / 8);
                if (i >= m * (kPassK / 8)) break;
                const uint32_t dst = xs + (uint32_t)(((o >> 2) * cols + i / (kPassK / 8) * S) * 64 + (o & 3) * 16);
                if constexpr (F32X) {
                    uint32_t w[3][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        split_pair(__uint_as_float(v[b][h].x), __uint_as_float(v[b][h].y), w[0][2 * h], w[1][2 * h], w[2][2 * h]);
                        split_pair(__uint_as_float(v[b][h].z), __uint_as_float(v[b][h].w), w[0][2 * h + 1], w[1][2 * h + 1],
                                   w[2][2 * h + 1]);
                    }
#pragma unroll
                    for (int s = 0; s < 3; ++s) sts128(dst + s * 64, pair_order(w[s][0], w[s][1], w[s][2], w[s][3]));
                } else {
                    sts128(dst, pair_order(v[b][0].x, v[b][0].y, v[b][0].z, v[b][0].w));
                }
            }
        }
        // the scales have arrived: with the first pass the codes' first stages
        // may still be on their way, later ones were asked for before the scales
        if (st0 == 0) cp_async_wait<kStages>();
        else cp_async_wait<0>();
        __syncthreads();

        for (int st = st0; st < min(nst, st0 + kPassK / kStageK); ++st) {
            cp_async_wait<kStages - 1>();
            __syncwarp();
            const uint32_t stage = ring + (uint32_t)((st % kStages) * kStageBytes) + (uint32_t)(lr * 64 + lc * 4);
            const uint32_t xst = xs + (uint32_t)((st - st0) * (kStageK / 32) * cols * 64 + lr * 64 + lc * 16);
            const uint32_t srow = sc + (uint32_t)((warp * 32 + lr) * sp), zrow = zs + (uint32_t)((warp * 32 + lr) * zp);
            // block b of the stage: codes of rows lr + 8 r, X's columns
            auto block = [&](int b, bool first, const uint32_t (&z)[4]) {
                uint32_t w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = lds32(stage + (uint32_t)(((b ^ (lr >> 1)) << 4) + r * 512));
                uint4 x[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    x[t] = t * 8 + lr < cols ? lds128(xst + (uint32_t)((b * cols + t * 8) * 64)) : make_uint4(0, 0, 0, 0);
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
                // what lies past the slice is zero codes, zero X and zero scales
                constexpr int NG = 4 / GB;            // scale groups of the stage
                const int go = GB == 4 ? (k0 + st * kStageK) / a.group - g0 : (st - st0) * NG;
                float s[NG][4];
                uint32_t z[NG][4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t at = srow + (uint32_t)(r * 8 * sp + go * ssize);
                    uint32_t f[4];
                    if (a.s_f32) {
                        if constexpr (NG == 4) { const uint4 v = lds128(at); f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
                        else if constexpr (NG == 2) { const uint2 v = lds64(at); f[0] = v.x; f[1] = v.y; }
                        else f[0] = lds32(at);
                    } else {
                        uint2 v;
                        if constexpr (NG == 4) v = lds64(at);
                        else if constexpr (NG == 2) v.x = lds32(at);
                        else v.x = lds16(at);
                        f[0] = v.x << 16;
                        f[1] = v.x & 0xFFFF0000u;
                        f[2] = v.y << 16;
                        f[3] = v.y & 0xFFFF0000u;
                    }
                    uint32_t q = 0x08080808u;
                    if (a.zeros) {
                        const uint32_t az = zrow + (uint32_t)(r * 8 * zp + go);
                        q = (NG == 4 ? lds32(az) : NG == 2 ? lds16(az) : lds8(az)) & 0x0F0F0F0Fu;
                    }
#pragma unroll
                    for (int n = 0; n < NG; ++n) {
                        s[n][r] = __uint_as_float(f[n]);
                        z[n][r] = __byte_perm(q, 0x43434343u, 0x4040u + 0x0101u * n);      // 128 + z as a BF16 pair
                    }
                }
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    block(b, b % GB == 0, z[b / GB]);
                    if (b % GB == GB - 1) scale_up(s[b / GB]);
                }
            } else {
                const int kb0 = (k0 + st * kStageK) / 32, kb1 = min(kb0 + kStageK / 32, k1 / 32);
                for (int kb = kb0; kb < kb1;) {
                    // the part of a scale group that this stage holds
                    const int gi = kb / gb, end = min(kb1, (gi + 1) * gb);
                    float s[4];
                    uint32_t z[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t at = srow + (uint32_t)(r * 8 * sp + (gi - g0) * ssize);
                        s[r] = __uint_as_float(a.s_f32 ? lds32(at) : lds16(at) << 16);
                        const uint32_t q = a.zeros ? lds8(zrow + (uint32_t)(r * 8 * zp + gi - g0)) & 15u : 8u;
                        z[r] = __byte_perm(q, 0x43434343u, 0x4040u);
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
            fetch(st + kStages);                      // into the stage just read
        }
    }
    cp_async_wait<0>();
    __syncwarp();
    __syncthreads();                                  // the rings are free: their memory takes the sums

    // ---- sums of this CTA: [column][feature]
    float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = t * 8 + lc * 2 + (e & 1), r = warp * 32 + i * 16 + lr + (e >> 1) * 8;
                if (c < cols) sums[c * kRows + r] = total[i][t][e];
            }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    // ---- the cluster's sums in rank order, slices of a row smallest first
    const int per = kRows / (int)ks;
    for (int i = threadIdx.x; i < m * per; i += 32 * kWarps) {
        const int t = i / per, r = (int)rank * per + i % per, n = n0 + r;
        float v[8][S], y = 0.0f;
#pragma unroll
        for (uint32_t c = 0; c < 8; ++c) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                uint32_t at;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                             : "=r"(at) : "r"(codes + (uint32_t)(((t * S + s) * kRows + r) * 4)), "r"(c < ks ? c : 0u));
                v[c][s] = 0.0f;
                if (c < ks) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[c][s]) : "r"(at) : "memory");
            }
        }
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int s = S - 1; s >= 0; --s) y = __fadd_rn(y, v[c][s]);
        if (n < a.N) {
            const int64_t o = (int64_t)(row0 + t) * a.ldy + n;
            if (a.x_f32) static_cast<float *>(a.Y)[o] = y;
            else static_cast<uint16_t *>(a.Y)[o] = (uint16_t)bf16x2_rn(y, 0.0f);
        }
    }
    __syncwarp();                                     // the others may still read this CTA's sums
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int NT, bool F32X, int GB>
cudaError_t run_w4(const W4Args &a, int64_t blocks, int64_t items, int ks, cudaStream_t st)
{
    auto kern = w4_kernel<NT, F32X, GB>;
    // the codes' rings, X's columns for one pass (64 bytes per 32 k and column),
    // the pass's scales and zero points
    const int sm = kWarps * ring_stages(NT) * kStageBytes + pass_k(NT) / 32 * a.tokens * (F32X ? 3 : 1) * 64 +
                   kRows * (a.sp + (a.zeros ? a.zp : 0));
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, sm);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(blocks * ks), (unsigned)items);
    cfg.blockDim = dim3(32 * kWarps);
    cfg.dynamicSmemBytes = (size_t)sm;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ks;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kern, a);
    if (e != cudaSuccess) return e;
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_w4_matvec(bool x_f32, int64_t G, int64_t rows, int64_t N, int64_t K, int group, const void *X,
                             int64_t ldx, const uint8_t *q, const void *scales, bool s_f32, const uint8_t *zeros,
                             const int32_t *ends, void *Y, int64_t ldy, cudaStream_t st)
{
    W4Args a = {};
    a.X = X; a.ldx = ldx; a.q = q; a.scales = scales; a.zeros = zeros; a.ends = ends; a.Y = Y; a.ldy = ldy;
    a.G = (int)G; a.rows = (int)rows; a.N = (int)N; a.K = (int)K; a.group = group;
    a.x_f32 = x_f32 ? 1 : 0; a.s_f32 = s_f32 ? 1 : 0;
    a.x_vec = (reinterpret_cast<uintptr_t>(X) & 15u) == 0 && ldx * (x_f32 ? 4 : 2) % 16 == 0;
    // rows of X per item: up to 24 columns; an expert is expected to get up to
    // twice its share of the rows (one that gets more is read again)
    const int S = x_f32 ? 3 : 1;
    const int64_t active = !ends ? 1 : (G < rows ? G : rows);
    int64_t want = ends ? 2 * ((rows + active - 1) / active) : rows;
    if (want > rows) want = rows;
    int nt = (int)((want * S + 7) / 8);
    nt = nt > 1 ? 3 : 1;
    a.tokens = 8 * nt / S;
    if (a.tokens > rows) a.tokens = (int)rows;
    const int pass = pass_k(nt);
    const int64_t blocks = (N + kRows - 1) / kRows;
    const int64_t items = ends ? active + rows / a.tokens + 1 : (rows + a.tokens - 1) / a.tokens;
    if (items > 65535) return cudaErrorInvalidValue;
    // slices of K: one pass each where 8 of them allow it, and more while there
    // are fewer CTAs than SMs and each has 512 k
    int ks = 1;
    while (ks < 8 && (ks * pass < K || (blocks * active * ks < 152 && ks * 2 * 512 <= K))) ks *= 2;
    const int64_t unit = K < (int64_t)ks * pass ? kStageK : pass;
    a.slice = (int)((K + ks * unit - 1) / (ks * unit) * unit);
    a.sp = meta_pitch(pass, group, a.slice, s_f32 ? 4 : 2);
    a.zp = meta_pitch(pass, group, a.slice, 1);
#define EMU_W4(GB)                                                                                              \
    (x_f32 ? (nt == 1 ? run_w4<1, true, GB>(a, blocks, items, ks, st) : run_w4<3, true, GB>(a, blocks, items, ks, st)) \
           : (nt == 1 ? run_w4<1, false, GB>(a, blocks, items, ks, st) : run_w4<3, false, GB>(a, blocks, items, ks, st)))
    return group == 32 ? EMU_W4(1) : group == 64 ? EMU_W4(2) : group % 128 == 0 ? EMU_W4(4) : EMU_W4(0);
#undef EMU_W4
}

}  // namespace emu
