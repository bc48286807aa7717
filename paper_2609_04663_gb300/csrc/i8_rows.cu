// Products in 8-bit integers for one row or a few rows (of each group): the weights are
// streamed once for up to R rows, with four-way integer dot products into 32-bit sums, which
// are exact.
//
// A warp has F features and a part of K; a lane reads 16 consecutive codes of each
// feature and of each row.  WK warps of a CTA split K between them and add their sums in shared
// memory.
#include "i8_common.cuh"

namespace emu {

namespace {

constexpr int kF = 4;                 // features per warp
constexpr int kWarps = 8;

struct RowsArgs {
    I8Product p;
    int fblocks, wk;                  // feature blocks, warps that split K
};

template <int R, bool WIDEX, bool WIDEW>
__global__ void __launch_bounds__(32 * kWarps) i8_rows_kernel(const RowsArgs a)
{
    extern __shared__ int starts[];                   // [G + 1], [G + 1] (chunks before each group)
    __shared__ int part[kWarps][kF * R];
    const I8Product &p = a.p;
    const int warp = (int)threadIdx.x >> 5, lane = (int)lane_id();
    const int chunk = (int)blockIdx.x / a.fblocks, fb = (int)blockIdx.x - chunk * a.fblocks;
    int g = 0, r0 = chunk * R, r1 = p.rows;
    bool bad = false;
    if (p.ends) bad = load_groups(p.ends, p.G, p.rows, starts);
    if (blockIdx.x == 0) {                            // the flag word is this kernel's alone: one CTA sets it
        if (p.src)
            for (int r = threadIdx.x; r < p.rows; r += 32 * kWarps) {
                const int t = __ldg(p.src + r);
                bad |= t < 0 || t >= p.xrows;
            }
        bad = __syncthreads_or(bad ? 1 : 0) != 0;
        if (threadIdx.x == 0) *p.flags = bad ? (uint32_t)EMU_FLAG_INDEX : 0u;
    }
    if (p.ends) {
        int *pre = starts + p.G + 1;
        if (warp == 0) {                              // chunks of R rows before each group
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
        if (chunk >= pre[p.G]) return;
        g = find_group(pre, p.G, chunk);
        r0 = starts[g] + (chunk - pre[g]) * R;
        r1 = starts[g + 1];
    }
    const int nr = min(R, r1 - r0);
    const int fper = kWarps / a.wk * kF, kpart = warp % a.wk;
    const int f0 = fb * fper + warp / a.wk * kF;
    int64_t from[R];                                  // the rows' places in X; negative: none
#pragma unroll
    for (int r = 0; r < R; ++r) {
        from[r] = -1;
        if (r < nr) {
            int64_t t = r0 + r;
            if (p.src) t = __ldg(p.src + t);
            if (t >= 0 && t < p.xrows) from[r] = t;
        }
    }
    const int8_t *w[kF];
#pragma unroll
    for (int f = 0; f < kF; ++f) w[f] = p.W + g * p.stridew + (int64_t)min(f0 + f, p.N - 1) * p.ldw;
    int acc[kF][R];
#pragma unroll
    for (int f = 0; f < kF; ++f)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[f][r] = 0;
    if (f0 < p.N) {
#pragma unroll 2
        for (int k = kpart * 512 + lane * 16; k < p.K; k += 512 * a.wk) {
            uint4 v[kF];
#pragma unroll
            for (int f = 0; f < kF; ++f) v[f] = load_codes<WIDEW>(w[f] + k, p.K - k);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (from[r] < 0) continue;
                const uint4 x = load_codes<WIDEX>(p.X + from[r] * p.ldx + k, p.K - k);
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
    int mine = 0;                                     // lane f R + r: that feature's and row's sum
#pragma unroll
    for (int f = 0; f < kF; ++f)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int s = __reduce_add_sync(0xFFFFFFFFu, acc[f][r]);
            if (lane == f * R + r) mine = s;
        }
    if (a.wk > 1) {
        if (lane < kF * R) part[warp][lane] = mine;
        __syncthreads();
        if (kpart != 0) return;
        if (lane < kF * R)
            for (int w2 = 1; w2 < a.wk; ++w2) mine += part[warp + w2][lane];
    }
    const int n = f0 + lane / R, r = lane % R;
    if (lane >= kF * R || n >= p.N || r >= nr) return;
    int64_t t = r0 + r;
    if (p.src) t = __ldg(p.src + t);
    const bool there = t >= 0 && t < p.xrows;
    const float xs = !there ? 0.0f : p.xscales ? __ldg(p.xscales + t) : 1.0f;
    const float ws = p.wscales ? __ldg(p.wscales + (int64_t)g * p.N + n) : 1.0f;
    store_value(p, r0 + r, n, there ? scaled_sum(mine, ws, xs) : 0.0f, there ? mine : 0);
}

template <int R, bool WIDEX, bool WIDEW>
cudaError_t run(RowsArgs a, cudaStream_t st)
{
    const int64_t groups = a.p.G < a.p.rows ? a.p.G : a.p.rows, chunks = a.p.rows / R + groups;
    // K is split until there are two CTAs for each SM
    a.wk = 1;
    auto blocks = [&]() { const int per = kWarps / a.wk * kF; return chunks * (((int64_t)a.p.N + per - 1) / per); };
    while (a.wk < kWarps && a.p.K > 512 * a.wk && blocks() < 152 * 4) a.wk *= 2;
    const int per = kWarps / a.wk * kF;
    a.fblocks = (a.p.N + per - 1) / per;
    const int64_t grid = blocks();
    if (grid >= ((int64_t)1 << 31)) return cudaErrorInvalidConfiguration;
    i8_rows_kernel<R, WIDEX, WIDEW><<<(unsigned)grid, 32 * kWarps, a.p.ends ? 2 * (a.p.G + 1) * sizeof(int) : 0, st>>>(a);
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

bool i8_few_rows(int64_t G, int64_t rows) { return rows <= (G > 1 ? 4 * G : 8); }

cudaError_t launch_i8_rows(const I8Product &p, cudaStream_t st)
{
    RowsArgs a = {};
    a.p = p;
    return p.rows == 1 ? by_alignment<1>(a, st) : p.rows <= 2 ? by_alignment<2>(a, st)
           : p.rows <= 4 || p.rows <= p.G ? by_alignment<4>(a, st) : by_alignment<8>(a, st);
}

}  // namespace emu
