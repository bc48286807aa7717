// Products in 8-bit integers for one row or a few rows (of each group): the weights are
// streamed once for up to R rows, with four-way integer dot products into 32-bit sums, which
// are exact.
//
// The rows of a chunk (up to R of one group) are kept in shared memory.  A warp has four features
// and a part of K; a lane copies 16 consecutive codes of each feature into a ring of its own in shared
// memory, kDepth - 1 steps ahead (also into the next item), and reads them back: 48 KB in flight a CTA.
// WK warps of a CTA split K between them and add their sums in shared memory.  CTAs have a range
// of items (a chunk and a block of features) in a row, so that most of them bring in
// one chunk.
//
// Bound by HBM and by getting there: one row x 16384 x 16384 takes 43 us (6.2 TB/s), one x 4096 x 4096 5.1 (launch and
// the first loads' latency), 16 rows over 12 experts of 2048 x 4096 20.7 (4.9 TB/s).
// 8 rows x 4096 x 4096 take 10.6, 5 more than one: with a fourth of the dot products 9.5, with one of the rows brought
// in 9.8, with an eighth of the additions over lanes 10.2, with a row's reads from shared memory for all 10.7.
#include <atomic>

#include "i8_common.cuh"

namespace emu {

namespace {

constexpr int kF = 4;                 // features per warp
constexpr int kWarps = 8;
constexpr int kRowBytes = 32768;      // of a chunk's rows in shared memory
constexpr int kDepth = 4;             // steps of weights in a warp's ring
constexpr int kRing = kDepth * kF * 512;
constexpr int kCtas = 304;            // two for each SM

// 16 bytes from global to shared memory, the first n of them (0: none are read), zeros behind.
__device__ __forceinline__ void copy16(uint32_t to, const int8_t *from, int n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
}

struct RowsArgs {
    I8Product p;
    int fblocks, wk;                  // feature blocks, warps that split K
};

template <int R, bool WIDEX, bool WIDEW>
__global__ void __launch_bounds__(32 * kWarps, 2) i8_rows_kernel(const RowsArgs a)
{
    constexpr int KS = kRowBytes / R;                 // codes of a row that are kept at once
    extern __shared__ int4 dyn[];
    __shared__ int part[kWarps][kF * R];
    int8_t *rows = reinterpret_cast<int8_t *>(dyn) + kWarps * kRing;       // [R][pitch]
    const I8Product &p = a.p;
    const int pitch = min(KS, (p.K + 511) & ~511);
    int *starts = reinterpret_cast<int *>(rows + R * pitch), *pre = starts + p.G + 1;     // chunks before each group
    const int warp = (int)threadIdx.x >> 5, lane = (int)lane_id();
    bool bad = false;
    if (p.ends) bad = load_groups(p.ends, p.G, p.rows, starts);
    if (blockIdx.x == 0 && p.flags) {                 // the flag word is this kernel's alone: one CTA sets it
        if (p.src)
            for (int r = threadIdx.x; r < p.rows; r += 32 * kWarps) {
                const int t = __ldg(p.src + r);
                bad |= t < 0 || t >= p.xrows;
            }
        bad = __syncthreads_or(bad ? 1 : 0) != 0;
        if (threadIdx.x == 0) *p.flags = bad ? (uint32_t)EMU_FLAG_INDEX : 0u;
    }
    int chunks = (p.rows + R - 1) / R;
    if (p.ends) {
        if (warp == 0) {
            int carry = 0;
            for (int g0 = 0; g0 < p.G; g0 += 32) {
                const int q = g0 + lane;
                int v = q < p.G ? (starts[q + 1] - starts[q] + R - 1) / R : 0;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int u = __shfl_up_sync(0xFFFFFFFFu, v, d);
                    if (lane >= d) v += u;
                }
                if (q < p.G) pre[q + 1] = carry + v;
                carry += __shfl_sync(0xFFFFFFFFu, v, 31);
            }
            if (lane == 0) pre[0] = 0;
        }
        __syncthreads();
        // rows of no group are zero
        for (int64_t r = (int64_t)starts[p.G] + blockIdx.x; r < p.rows; r += gridDim.x)
            for (int n = threadIdx.x; n < p.N; n += 32 * kWarps) store_value(p, r, n, 0.0f, 0);
        chunks = pre[p.G];
    }
    const int64_t items = (int64_t)chunks * a.fblocks;
    const int64_t first = items * blockIdx.x / gridDim.x, last = items * (blockIdx.x + 1) / gridDim.x;
    const int fper = kWarps / a.wk * kF, kpart = warp % a.wk, kstep = 512 * a.wk;
    auto group_of = [&](int chunk) { return p.ends ? find_group(pre, p.G, chunk) : 0; };
    // the weights' way into the ring: next item and place in K
    const uint32_t ring = smem_u32(dyn) + (uint32_t)(warp * kRing + lane * 16);
    int64_t ahead = kpart * 512 < p.K ? first : last;
    int achunk = (int)(first / a.fblocks), afb = (int)(first - (int64_t)achunk * a.fblocks), ak = kpart * 512 + lane * 16;
    const int8_t *agroup = p.W, *aw = nullptr;        // its group's matrix, its first feature's row
    int left = 0;                                     // features from that on
    uint32_t as = 0;
    const int fwarp = warp / a.wk * kF;
    auto open = [&]() {
        const int f0 = afb * fper + fwarp;
        aw = agroup + (int64_t)min(f0, p.N - 1) * p.ldw;
        left = p.N - f0;
    };
    auto fetch = [&]() {
        if (ahead < last) {
            const int n = p.K - ak;
#pragma unroll
            for (int f = 0; f < kF; ++f) {
                const int8_t *from = f < left ? aw + f * p.ldw + ak : p.W;
                const uint32_t to = ring + as * (kF * 512) + f * 512;
                if (WIDEW) {
                    copy16(to, from, f < left ? min(max(n, 0), 16) : 0);
                } else {
                    const uint4 v = load_codes<false>(from, f < left ? n : 0);
                    st_shared_v4(to, v.x, v.y, v.z, v.w);
                }
            }
            ak += kstep;
            if (ak - lane * 16 >= p.K) {
                ak = kpart * 512 + lane * 16;
                if (++ahead < last) {
                    if (++afb == a.fblocks) {
                        afb = 0;
                        agroup = p.W + group_of(++achunk) * p.stridew;
                    }
                    open();
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++as == kDepth) as = 0;
    };
    if (ahead < last) {
        agroup = p.W + group_of(achunk) * p.stridew;
        open();
    }
    int chunk = achunk, fb = afb - 1;
#pragma unroll 1
    for (int d = 0; d < kDepth - 1; ++d) fetch();
    uint32_t cs = 0;                                  // stage that is used next
    int held = -1, g = 0, r0 = 0, nr = 0;             // the chunk in shared memory, its group and rows
    for (int64_t item = first; item < last; ++item) {
        if (++fb == a.fblocks) { fb = 0; ++chunk; }
        const int f0 = fb * fper + fwarp;
        if (chunk != held) {
            g = group_of(chunk);
            r0 = p.ends ? starts[g] + (chunk - pre[g]) * R : chunk * R;
            nr = min(R, (p.ends ? starts[g + 1] : p.rows) - r0);
        }
        int acc[kF][R];
#pragma unroll
        for (int f = 0; f < kF; ++f)
#pragma unroll
            for (int r = 0; r < R; ++r) acc[f][r] = 0;
        int k = kpart * 512;                          // (the same for all lanes)
        for (int k0 = 0; k0 < p.K; k0 += KS) {
            const int to = min(p.K, k0 + KS);
            if (chunk != held || p.K > KS) {
                __syncthreads();                      // the rows before have been used
                const int pieces = (to - k0 + 15) >> 4;
                for (int i = threadIdx.x; i < R * pieces; i += 32 * kWarps) {
                    const int r = i / pieces, c = (i - r * pieces) * 16;
                    int64_t t = -1;
                    if (r < nr) t = p.src ? (int64_t)__ldg(p.src + r0 + r) : r0 + r;
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (t >= 0 && t < p.xrows) v = load_codes<WIDEX>(p.X + t * p.ldx + k0 + c, to - k0 - c);
                    *reinterpret_cast<uint4 *>(rows + r * pitch + c) = v;
                }
                __syncthreads();
                held = chunk;
            }
            for (; k < to; k += kstep) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 2) : "memory");
                uint4 v[kF];
#pragma unroll
                for (int f = 0; f < kF; ++f)
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(v[f].x), "=r"(v[f].y), "=r"(v[f].z), "=r"(v[f].w)
                                 : "r"(ring + cs * (kF * 512) + f * 512) : "memory");
                if (++cs == kDepth) cs = 0;
                fetch();                              // into the stage that was used before this one
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    // (past K the weights are zero, and the rows' places whatever they are)
                    const uint4 x = *reinterpret_cast<const uint4 *>(rows + r * pitch + (k - k0) + lane * 16);
#pragma unroll
                    for (int f = 0; f < kF; ++f) {
                        acc[f][r] = __dp4a((int)v[f].x, (int)x.x, acc[f][r]);
                        acc[f][r] = __dp4a((int)v[f].y, (int)x.y, acc[f][r]);
                        acc[f][r] = __dp4a((int)v[f].z, (int)x.z, acc[f][r]);
                        acc[f][r] = __dp4a((int)v[f].w, (int)x.w, acc[f][r]);
                    }
                }
            }
        }
        int sum = 0;                                  // lane f R + r: that feature's and row's sum
#pragma unroll
        for (int f = 0; f < kF; ++f)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int s = __reduce_add_sync(0xFFFFFFFFu, acc[f][r]);
                if (lane == f * R + r) sum = s;
            }
        if (a.wk > 1) {
            __syncthreads();                          // the item before has been added
            if (lane < kF * R) part[warp][lane] = sum;
            __syncthreads();
            if (kpart != 0) continue;
            if (lane < kF * R)
                for (int w2 = 1; w2 < a.wk; ++w2) sum += part[warp + w2][lane];
        }
        const int n = f0 + lane / R, r = lane % R;
        if (lane >= kF * R || n >= p.N || r >= nr) continue;
        int64_t t = r0 + r;
        if (p.src) t = __ldg(p.src + t);
        const bool there = t >= 0 && t < p.xrows;
        const float xs = !there ? 0.0f : p.xscales ? __ldg(p.xscales + t) : 1.0f;
        const float ws = p.wscales ? __ldg(p.wscales + (int64_t)g * p.N + n) : 1.0f;
        store_value(p, r0 + r, n, there ? scaled_sum(sum, ws, xs) : 0.0f, there ? sum : 0);
    }
}

template <int R, bool WIDEX, bool WIDEW>
cudaError_t run(RowsArgs a, cudaStream_t st)
{
    const int64_t groups = a.p.G < a.p.rows ? a.p.G : a.p.rows;
    const int64_t chunks = a.p.ends ? a.p.rows / R + groups : (a.p.rows + R - 1) / R;     // of groups: at most
    // K is split until there is an item for each CTA that fits, of groups two, as there may be half as many
    // (3 rows x 4096 x 4096 with two: 9.1 us against 7.4)
    a.wk = 1;
    const int64_t enough = a.p.ends ? 2 * kCtas : kCtas;
    auto items = [&]() { const int per = kWarps / a.wk * kF; return chunks * (((int64_t)a.p.N + per - 1) / per); };
    while (a.wk < kWarps && a.p.K > 512 * a.wk && items() < enough) a.wk *= 2;
    const int per = kWarps / a.wk * kF, pitch = a.p.K < kRowBytes / R ? (a.p.K + 511) / 512 * 512 : kRowBytes / R;
    a.fblocks = (a.p.N + per - 1) / per;
    const int64_t grid = items() < kCtas ? items() : kCtas;
    constexpr int most = kWarps * kRing + kRowBytes + 2 * (kMaxGroups + 1) * 4;
    static std::atomic<uint64_t> known{0};            // devices that know how much shared memory the kernel takes
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
    if (!(known.load(std::memory_order_relaxed) & bit)) {
        e = cudaFuncSetAttribute(i8_rows_kernel<R, WIDEX, WIDEW>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e != cudaSuccess) return e;
        known.fetch_or(bit, std::memory_order_relaxed);
    }
    const size_t smem = (size_t)kWarps * kRing + (size_t)R * pitch + (a.p.ends ? 2 * (a.p.G + 1) * sizeof(int) : 0);
    i8_rows_kernel<R, WIDEX, WIDEW><<<(unsigned)grid, 32 * kWarps, smem, st>>>(a);
    return cudaGetLastError();
}

template <int R>
cudaError_t by_alignment(const RowsArgs &a, cudaStream_t st)
{
    const bool x = aligned_codes(a.p.X, a.p.xrows > 1 ? a.p.ldx : 0, 0), w = aligned_codes(a.p.W, a.p.ldw, a.p.G > 1 ? a.p.stridew : 0);
    return x && w ? run<R, true, true>(a, st) : x ? run<R, true, false>(a, st)
           : w ? run<R, false, true>(a, st) : run<R, false, false>(a, st);
}

}  // namespace

// Up to where the tensor cores' kernel is slower: 8 rows x 2048 x 2048 5.7 us here and 8.5 there, x 4096 x 4096 10.5
// and 10.6, x 8192 x 8192 32 and 20; 4 rows x 8192 x 8192 19 and 20, x 16384 x 16384 55 and 50; 2 rows there 46 and 50.
// One row of each of 32 experts of 1024 x 1024 12.6 and 13.1, two 14.7 and 13.3; two of each of 8 of 4096 x 4096 27 and
// 31, four 32 and 31.
bool i8_few_rows(int64_t G, int64_t rows, int64_t N, int64_t K)
{
    const int64_t weights = N * K;
    if (G > 1) return rows <= (G <= 8 ? 2 * G : G);
    return rows <= 2 || (rows <= 4 && weights <= (int64_t)1 << 26) || (rows <= 8 && weights <= (int64_t)1 << 24);
}

cudaError_t launch_i8_rows(const I8Product &p, cudaStream_t st)
{
    RowsArgs a = {};
    a.p = p;
    return p.rows == 1 ? by_alignment<1>(a, st) : p.rows <= 2 ? by_alignment<2>(a, st)
           : p.G > 1 && p.rows <= p.G ? by_alignment<2>(a, st) : p.rows <= 4 || p.G > 1 ? by_alignment<4>(a, st)
           : by_alignment<8>(a, st);
}

}  // namespace emu
