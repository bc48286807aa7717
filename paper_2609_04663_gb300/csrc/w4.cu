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

constexpr int kWarps = 4, kRows = 32 * kWarps;        // features per CTA
constexpr int kStageK = 256;                          // k of one ring stage: 128 bytes of codes per row
constexpr int kStages = 3;
constexpr int kPassK = 1024;                          // k for which X and the scales are staged at once

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
    int x_f32, s_f32, x_vec;                          // x_vec: X's rows can be read 16 bytes at a time
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool valid)
{
    const int n = valid ? 16 : 0;                     // 0: the 16 bytes are filled with zeros
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

// 8 consecutive BF16 as pairs (0,4) (1,5) (2,6) (3,7).
__device__ __forceinline__ uint4 pair_order(uint32_t w01, uint32_t w23, uint32_t w45, uint32_t w67)
{
    return make_uint4(__byte_perm(w01, w45, 0x5410), __byte_perm(w01, w45, 0x7632), __byte_perm(w23, w67, 0x5410),
                      __byte_perm(w23, w67, 0x7632));
}

__device__ __forceinline__ void sts128(uint32_t a, uint4 v) { st_shared_v4(a, v.x, v.y, v.z, v.w); }

// Row pitch of the staged scales or zero points of one pass: an odd number of
// 16-byte pieces, so that the 8 rows that a warp reads at once lie in
// different banks.
__host__ __device__ __forceinline__ int meta_pitch(int group, int size)
{
    const int pieces = ((kPassK / group + 2) * size + 15) / 16;
    return (pieces | 1) * 16;
}

// Shared memory of a CTA, in bytes: the codes' rings, X's columns for one
// pass (64 bytes per 32 k and column), the pass's scales and zero points.
int w4_smem(int cols, int group, int ssize, bool zeros)
{
    return kWarps * kStages * 32 * 128 + (kPassK / 32) * cols * 64 + kRows * meta_pitch(group, ssize) +
           (zeros ? kRows * meta_pitch(group, 1) : 0);
}

// NT: tiles of 8 columns; F32X: FP32 rows, three columns each.
template <int NT, bool F32X>
__global__ void __launch_bounds__(32 * kWarps, 2) w4_kernel(const W4Args a)
{
    constexpr int S = F32X ? 3 : 1;
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
    const int ssize = a.s_f32 ? 4 : 2, sp = meta_pitch(a.group, ssize), zp = meta_pitch(a.group, 1);
    const uint32_t xs = codes + kWarps * kStages * 32 * 128;
    const uint32_t sc = xs + (uint32_t)((kPassK / 32) * a.tokens * S * 64), zs = sc + (uint32_t)(kRows * sp);
    const int k0 = (int)rank * a.slice, k1 = min(a.K, k0 + a.slice);
    const int nst = k1 > k0 ? (k1 - k0 + kStageK - 1) / kStageK : 0;

    // ---- this warp's ring: rows n0 + 32 warp .. + 31, 16-byte piece j of a row at piece j ^ (row % 8)
    const uint32_t ring = codes + (uint32_t)(warp * kStages * 32 * 128);
    const int64_t pitch = a.K / 2;
    const uint8_t *qbase = a.q + ((int64_t)g * a.N + n0 + warp * 32) * pitch;
    auto fetch = [&](int st) {
        if (st < nst) {
            const uint32_t dst = ring + (uint32_t)((st % kStages) * 32 * 128);
            const int piece = lane & 7, byte = (k0 + st * kStageK) / 2 + piece * 16;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = i * 4 + (lane >> 3);
                const bool ok = n0 + warp * 32 + r < a.N && byte < k1 / 2;
                cp_async16(dst + (uint32_t)(r * 128 + ((piece ^ (r & 7)) << 4)), ok ? qbase + r * pitch + byte : a.q, ok);
            }
        }
        cp_async_commit();
    };
    // n scales or zero points of each feature from group g0 on -> rows of pitch
    // dpitch at dst, by 16-byte copies where the source rows allow it
    auto meta = [&](uint32_t dst, int dpitch, const void *src, int size, int g0, int n) {
        const uint8_t *from = static_cast<const uint8_t *>(src) + (((int64_t)g * a.N + n0) * ngroups + g0) * size;
        const int64_t rowb = (int64_t)ngroups * size;
        const int pieces = (n * size + 15) / 16;
        // whole pieces only: a row's last piece may not run into what follows the array
        const bool wide = ((reinterpret_cast<uintptr_t>(from) | (uintptr_t)rowb) & 15u) == 0;
        for (int i = threadIdx.x; i < kRows * pieces; i += 32 * kWarps) {
            const int r = i / pieces, o = (i % pieces) * 16;
            const bool ok = n0 + r < a.N;
            const uint32_t to = dst + (uint32_t)(r * dpitch + o);
            if (wide) {
                cp_async16(to, ok ? from + r * rowb + o : a.q, ok);
            } else {
                const int len = ok ? min(16, n * size - o) : 0;
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
            for (int st = 0; st < kStages - 1; ++st) fetch(st);
        }
        for (int i = threadIdx.x; i < m * (kPassK / 8); i += 32 * kWarps) {
            const int t = i / (kPassK / 8), o = i % (kPassK / 8), k = p0 + o * 8;
            const uint32_t dst = xs + (uint32_t)(((o >> 2) * cols + t * S) * 64 + (o & 3) * 16);
            if constexpr (F32X) {
                const float *x = static_cast<const float *>(a.X) + (int64_t)(row0 + t) * a.ldx + k;
                uint32_t w[3][4];
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (k < p1 && a.x_vec) v = __ldg(reinterpret_cast<const float4 *>(x) + (e >> 1));
                    else if (k < p1) v = make_float4(__ldg(x + 2 * e), __ldg(x + 2 * e + 1), __ldg(x + 2 * e + 2), __ldg(x + 2 * e + 3));
                    split_pair(v.x, v.y, w[0][e], w[1][e], w[2][e]);
                    split_pair(v.z, v.w, w[0][e + 1], w[1][e + 1], w[2][e + 1]);
                }
#pragma unroll
                for (int s = 0; s < 3; ++s) sts128(dst + s * 64, pair_order(w[s][0], w[s][1], w[s][2], w[s][3]));
            } else {
                const uint16_t *x = static_cast<const uint16_t *>(a.X) + (int64_t)(row0 + t) * a.ldx + k;
                uint4 w = make_uint4(0u, 0u, 0u, 0u);
                auto two = [&](int e) { return (uint32_t)__ldg(x + e) | (uint32_t)__ldg(x + e + 1) << 16; };
                if (k < p1 && a.x_vec) w = __ldg(reinterpret_cast<const uint4 *>(x));
                else if (k < p1) w = make_uint4(two(0), two(2), two(4), two(6));
                sts128(dst, pair_order(w.x, w.y, w.z, w.w));
            }
        }
        // the scales have arrived: with the first pass the codes' first stages
        // may still be on their way, later ones were asked for before the scales
        if (st0 == 0) cp_async_wait<kStages - 1>();
        else cp_async_wait<0>();
        __syncthreads();

        for (int st = st0; st < min(nst, st0 + kPassK / kStageK); ++st) {
            cp_async_wait<kStages - 2>();
            __syncwarp();
            fetch(st + kStages - 1);                  // into the stage read in the step before
            const uint32_t stage = ring + (uint32_t)((st % kStages) * 32 * 128) + (uint32_t)(lr * 128 + lc * 4);
            const int kb0 = (k0 + st * kStageK) / 32, kb1 = min(kb0 + 8, k1 / 32);
            int gi = kb0 / gb, left = gb - kb0 % gb;  // scale group, its 32-k blocks left
            for (int kb = kb0; kb < kb1;) {
                // the part of a scale group that this stage holds
                const int end = min(kb1, kb + left);
                float s[4];
                uint32_t z[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = warp * 32 + r * 8 + lr;
                    const uint32_t at = sc + (uint32_t)(row * sp + (gi - g0) * ssize);
                    if (a.s_f32) {
                        s[r] = __uint_as_float(lds32(at));
                    } else {
                        uint16_t h;
                        asm volatile("ld.shared.b16 %0, [%1];" : "=h"(h) : "r"(at));
                        s[r] = __uint_as_float((uint32_t)h << 16);
                    }
                    z[r] = 0x43084308u;               // 128 + z as a BF16 pair (z <= 15)
                    if (a.zeros) {
                        uint32_t v;
                        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(zs + (uint32_t)(row * zp + gi - g0)));
                        z[r] = (v & 15u) * 0x00010001u + 0x43004300u;
                    }
                }
#pragma unroll 2
                for (; kb < end; ++kb) {
                    const uint32_t at = stage + (uint32_t)((((kb - kb0) ^ lr) & 7) << 4);
                    uint32_t w[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) w[r] = lds32(at + r * 1024);      // rows lr + 8 r
                    uint4 b[NT];
                    const uint32_t xa = xs + (uint32_t)((kb - p0 / 32) * cols * 64 + lc * 16);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int n = t * 8 + lr;
                        b[t] = n < cols ? lds128(xa + (uint32_t)(n * 64)) : make_uint4(0, 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t u = w[2 * i], v = w[2 * i + 1], zu = z[2 * i], zv = z[2 * i + 1];
                        const uint32_t u0 = decode(u, 0, zu), u1 = decode(u, 4, zu), u2 = decode(u, 8, zu),
                                       u3 = decode(u, 12, zu);
                        const uint32_t v0 = decode(v, 0, zv), v1 = decode(v, 4, zv), v2 = decode(v, 8, zv),
                                       v3 = decode(v, 12, zv);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            mma16816(part[i][t], u0, v0, u1, v1, b[t].x, b[t].y);
                            mma16816(part[i][t], u2, v2, u3, v3, b[t].z, b[t].w);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            total[i][t][e] = fmaf(part[i][t][e], s[2 * i + (e >> 1)], total[i][t][e]);
                            part[i][t][e] = 0.0f;
                        }
                ++gi;
                left = gb;
            }
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
        float y = 0.0f;
        for (uint32_t c = 0; c < ks; ++c) {
#pragma unroll
            for (int s = S - 1; s >= 0; --s) {
                uint32_t at;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                             : "=r"(at) : "r"(codes + (uint32_t)(((t * S + s) * kRows + r) * 4)), "r"(c));
                float v;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
                y = __fadd_rn(y, v);
            }
        }
        if (n < a.N) {
            const int64_t o = (int64_t)(row0 + t) * a.ldy + n;
            if (a.x_f32) static_cast<float *>(a.Y)[o] = y;
            else static_cast<uint16_t *>(a.Y)[o] = (uint16_t)bf16x2_rn(y, 0.0f);
        }
    }
    __syncwarp();                                     // the others may still read this CTA's sums
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int NT, bool F32X>
cudaError_t run_w4(const W4Args &a, int64_t blocks, int64_t items, int ks, cudaStream_t st)
{
    auto kern = w4_kernel<NT, F32X>;
    const int sm = w4_smem(a.tokens * (F32X ? 3 : 1), a.group, a.s_f32 ? 4 : 2, a.zeros != nullptr);
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
    if (nt > 3) nt = 3;
    a.tokens = 8 * nt / S;
    const int64_t blocks = (N + kRows - 1) / kRows;
    const int64_t items = ends ? active + rows / a.tokens + 1 : (rows + a.tokens - 1) / a.tokens;
    if (items > 65535) return cudaErrorInvalidValue;
    // slices of K: at most one pass each where 8 of them allow it, and as many
    // CTAs as twice the SMs want while each still has one ring stage
    int ks = 1;
    while (ks < 8 && (ks * kPassK < K || (blocks * active * ks < 2 * 152 && ks * 2 * kStageK <= K))) ks *= 2;
    a.slice = (int)((K + (int64_t)ks * kStageK - 1) / ((int64_t)ks * kStageK) * kStageK);
#define EMU_W4(NT) (x_f32 ? run_w4<NT, true>(a, blocks, items, ks, st) : run_w4<NT, false>(a, blocks, items, ks, st))
    return nt == 1 ? EMU_W4(1) : nt == 2 ? EMU_W4(2) : EMU_W4(3);
#undef EMU_W4
}

}  // namespace emu
