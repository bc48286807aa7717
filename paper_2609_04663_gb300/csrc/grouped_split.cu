// Component planes of the operands of products grouped by expert: the FP32
// three-slice split of Eq. (fp32split), or for BF16 one plane (the values
// themselves, for operands whose rows the tensor memory accelerator cannot
// read or whose rows are gathered).  Planes keep the operand's own row order
// (no transposition: the product reads either dimension as the contraction).
// Token rows are gathered through `src` and put at padded positions, each
// group starting at a multiple of 16 rows and filled up with zero rows, so
// that the weight gradient's contraction over a group's rows ends on whole
// MMAs.
//
// Bound by HBM: 10 bytes per FP32 element (4 read, 6 written), 4 per BF16
// element.  One warp takes a row, a lane 8 consecutive elements per step
// (two 16-byte loads, one 16-byte store per plane).  16384 x 2048 FP32 rows: 54
// us (6.2 TB/s); 16 matrices of 2048 x 2048: 103 us (6.5 TB/s); 32768 BF16 rows of
// 2048 gathered from 8192: 30 us.
#include "grouped_common.cuh"
#include "expert_launchers.cuh"
#include "split_f32_pair.cuh"

namespace emu {

namespace {

constexpr int kThreads = 256;

struct SplitArgs {
    const void *X;
    int64_t rows, cols, ldx, per, stride;   // weights: row r is X + (r / per) * stride + (r % per) * ldx
    int64_t xrows;                          // tokens: rows of X that src may name
    const int32_t *src, *ends;              // tokens: gathered rows (or NULL), group ends
    int G;
    uint16_t *comps;
    int64_t ldcomp, plane;
    uint32_t *flags;
};

// Eight elements of one row -> S plane words of 16 bytes each.
template <int S>
__device__ __forceinline__ uint32_t split8(const float (&x)[8], uint4 (&w)[S], uint32_t amax)
{
    uint32_t p[3][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        amax = abs_bits_max(amax, x[2 * e], x[2 * e + 1]);
        split_pair(x[2 * e], x[2 * e + 1], p[0][e], p[1][e], p[2][e]);
    }
#pragma unroll
    for (int r = 0; r < S; ++r) w[r] = make_uint4(p[r][0], p[r][1], p[r][2], p[r][3]);
    return amax;
}

// Elements j0 .. j0 + 7 of a row (zeros past the last column, or for a row
// without a source).
template <int S>
__device__ __forceinline__ uint32_t load8(const void *row, int64_t j0, int64_t cols, bool vec, uint4 (&w)[S],
                                          uint32_t amax)
{
    const bool full = j0 + 8 <= cols;
    if constexpr (S == 3) {
        const float *src = static_cast<const float *>(row) + j0;
        float x[8];
        if (row && vec && full) {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(src)), b = __ldg(reinterpret_cast<const float4 *>(src) + 1);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (row && j0 + e < cols) ? __ldg(src + e) : 0.0f;
        }
        return split8<3>(x, w, amax);
    } else {
        const uint16_t *src = static_cast<const uint16_t *>(row) + j0;
        if (row && vec && full) {
            w[0] = __ldg(reinterpret_cast<const uint4 *>(src));
        } else {
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = (row && j0 + e < cols) ? (uint32_t)__ldg(src + e) : 0u;
            w[0] = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        }
        return amax;
    }
}

template <int S, bool TOKENS>
__global__ void __launch_bounds__(kThreads) grouped_split_kernel(const SplitArgs a)
{
    extern __shared__ int starts[];
    griddep_launch_dependents();              // a product launched as this kernel's dependent sets itself up meanwhile
    const int esize = S == 3 ? 4 : 2;
    int64_t nrows = a.rows;
    int total = 0;
    if constexpr (TOKENS) {
        if (load_groups(a.ends, a.G, (int)a.rows, starts) && blockIdx.x == 0 && threadIdx.x == 0)
            atomicOr(a.flags, (uint32_t)EMU_FLAG_INDEX);
        total = starts[a.G];
        nrows = padded_start(total, a.G);         // past the last group's padding
    }
    const bool vec = (reinterpret_cast<uintptr_t>(a.X) & 15u) == 0 && (a.ldx * esize) % 16 == 0 &&
                     (TOKENS || (a.stride * esize) % 16 == 0);
    const int lane = (int)lane_id();
    uint32_t amax = 0, bad = 0;
    for (int64_t p = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); p < nrows;
         p += (int64_t)gridDim.x * (kThreads / 32)) {
        const char *row = nullptr;
        if constexpr (TOKENS) {
            // the last group that starts at or before padded row p
            int lo = 0, hi = a.G - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (padded_start(starts[mid], mid) <= p) lo = mid;
                else hi = mid - 1;
            }
            const int64_t s = starts[lo] + (p - padded_start(starts[lo], lo));
            if (s >= starts[lo] && s < starts[lo + 1]) {
                int64_t r = s;
                if (a.src) {
                    r = a.src[s];
                    if (r < 0 || r >= a.xrows) { bad = 1; r = -1; }
                }
                if (r >= 0) row = static_cast<const char *>(a.X) + r * a.ldx * esize;
            }
        } else {
            row = static_cast<const char *>(a.X) + ((p / a.per) * a.stride + (p % a.per) * a.ldx) * esize;
        }
        uint16_t *dst = a.comps + p * a.ldcomp;
        constexpr int B = 4;                      // pieces loaded before the first is stored
        for (int64_t j0 = lane * 8; j0 < a.ldcomp; j0 += 256 * B) {
            uint4 w[B][S];
#pragma unroll
            for (int b = 0; b < B; ++b)
                if (j0 + 256 * b < a.ldcomp) amax = load8<S>(row, j0 + 256 * b, a.cols, vec, w[b], amax);
#pragma unroll
            for (int b = 0; b < B; ++b)
                if (j0 + 256 * b < a.ldcomp) {
#pragma unroll
                    for (int r = 0; r < S; ++r)
                        *reinterpret_cast<uint4 *>(dst + r * a.plane + j0 + 256 * b) = w[b][r];
                }
        }
    }
    if constexpr (S == 3) publish_f32_flags(amax, a.flags);
    if (bad && lane == 0) atomicOr(a.flags, (uint32_t)EMU_FLAG_INDEX);
}

template <int S, bool TOKENS>
cudaError_t run_split(const SplitArgs &a, int64_t nrows, cudaStream_t st)
{
    if (nrows <= 0 || a.cols <= 0) return cudaSuccess;
    int64_t blocks = (nrows + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 152 * 8) blocks = 152 * 8;
    const size_t sm = TOKENS ? (size_t)(a.G + 1) * sizeof(int) : 0;
    grouped_split_kernel<S, TOKENS><<<(unsigned)blocks, kThreads, sm, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

// Planes of G matrices of rows x cols (row pitch ldx, distance `stride`):
// [S][G * rows][ldcomp], ldcomp a multiple of 8.
cudaError_t launch_grouped_split(bool f32, int64_t G, int64_t rows, int64_t cols, const void *X, int64_t ldx,
                                 int64_t stride, uint16_t *comps, int64_t ldcomp, uint32_t *flags, cudaStream_t st)
{
    SplitArgs a = {};
    a.X = X; a.rows = G * rows; a.cols = cols; a.ldx = ldx; a.per = rows; a.stride = stride;
    a.comps = comps; a.ldcomp = ldcomp; a.plane = G * rows * ldcomp; a.flags = flags;
    return f32 ? run_split<3, false>(a, a.rows, st) : run_split<1, false>(a, a.rows, st);
}

// Planes of `rows` token rows at padded positions: [S][padded_rows(rows, G)][ldcomp].
cudaError_t launch_grouped_split_rows(bool f32, int64_t rows, int64_t cols, const void *X, int64_t xrows,
                                      int64_t ldx, const int32_t *src, const int32_t *ends, int64_t G,
                                      uint16_t *comps, int64_t ldcomp, uint32_t *flags, cudaStream_t st)
{
    SplitArgs a = {};
    a.X = X; a.rows = rows; a.cols = cols; a.ldx = ldx; a.xrows = xrows; a.src = src; a.ends = ends; a.G = (int)G;
    a.comps = comps; a.ldcomp = ldcomp; a.plane = padded_rows(rows, G) * ldcomp; a.flags = flags;
    return f32 ? run_split<3, true>(a, padded_rows(rows, G), st) : run_split<1, true>(a, padded_rows(rows, G), st);
}

}  // namespace emu
