// Rows to 8-bit integers with a scale for each row:
//   s = max_k |x_k| / 127, rounded to FP32; q_k = x_k / s rounded to the nearest
// integer, ties to even, exactly (the quotient is never rounded first), so that the
// codes are a matter of definition and not of the way to them.
//
// A quotient's nearest integer comes from x times the reciprocal (off by less than
// 2e-5), and where that lies within 1e-4 of the border between two integers, from the sign of
// x - (n +- 1/2) s, which one fused multiply-add gives exactly.  That is not rare: half of
// a row's largest value is at 63.5, and of BF16 values every three-hundredth or so is that.
//
// A group of R threads (32 to 512) has a row, four pieces of 16 bytes a thread in
// registers: each element is read once while rows have up to 4 R pieces, longer rows are read
// again from L2.
//
// 16384 x 4096 in BF16 takes 39.6 us (5.1 TB/s; 29.7 at the measured copy rate): integer and logic operations, 4 to
// 5 an element, keep their pipe two thirds busy while HBM is read.  One row of 4096: 2.4 us, a launch.
#include "i8_common.cuh"

namespace emu {

namespace {

constexpr int kPieces = 4;

struct QuantArgs {
    const void *X;
    int64_t rows, per, ldx, stridex;      // row r is X + (r / per) * stridex + (r % per) * ldx
    int8_t *q;
    int64_t ldq, strideq;
    float *scales;
    uint32_t *flags;                      // or NULL
    int cols;
};

// 4 FP32 or 8 BF16 values from column c on, zeros past the last one.
template <bool F32, bool VEC>
__device__ __forceinline__ uint4 load_values16(const char *row, int c, int cols)
{
    constexpr int N = F32 ? 4 : 8;
    if (VEC && c + N <= cols) return __ldg(reinterpret_cast<const uint4 *>(row + (int64_t)c * (F32 ? 4 : 2)));
    uint32_t w[4];
    if constexpr (F32) {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(row) + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = c + i < cols ? __ldg(p + i) : 0u;
    } else {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = c + 2 * i < cols ? (uint32_t)__ldg(p + 2 * i) : 0u;
            if (c + 2 * i + 1 < cols) w[i] |= (uint32_t)__ldg(p + 2 * i + 1) << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The values of a piece as pairs of FP32 numbers.
template <bool F32>
__device__ __forceinline__ void as_pairs(uint4 v, uint64_t (&x)[F32 ? 2 : 4])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (F32) {
        x[0] = (uint64_t)w[1] << 32 | w[0];
        x[1] = (uint64_t)w[3] << 32 | w[2];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (uint64_t)(w[i] & 0xFFFF0000u) << 32 | (w[i] << 16);
    }
}

// The larger magnitude of each, NaN if one is; of FP32 values, or of two BF16 values (halves),
// whose signs are then of no meaning.
template <bool F32>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
{
    if constexpr (F32) asm("{\n\t.reg .f32 x, y;\n\tmov.b32 x, %1;\n\tmov.b32 y, %2;\n\tabs.f32 y, y;\n\tmax.NaN.f32 x, x, y;\n\tmov.b32 %0, x;\n\t}" : "=r"(a) : "r"(a), "r"(b));
    else asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
    return a;
}
template <bool F32>
__device__ __forceinline__ uint32_t largest(uint4 v, uint32_t top)
{
    return larger<F32>(larger<F32>(larger<F32>(larger<F32>(top, v.x), v.y), v.z), v.w);
}

__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t both(float x) { return (uint64_t)__float_as_uint(x) << 32 | __float_as_uint(x); }
__device__ __forceinline__ float first_of(uint64_t x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float second_of(uint64_t x) { return __uint_as_float((uint32_t)(x >> 32)); }

// Codes of a piece from m, whose low bytes are the codes + 128 (so that nothing is carried from
// one to the next).
template <bool F32>
__device__ __forceinline__ uint2 pack(const uint32_t (&m)[F32 ? 4 : 8])
{
    uint2 o = make_uint2(0u, 0u);
    o.x = __byte_perm(m[1] * 256u + m[0], m[3] * 256u + m[2], 0x5410) ^ 0x80808080u;
    if constexpr (!F32) o.y = __byte_perm(m[5] * 256u + m[4], m[7] * 256u + m[6], 0x5410) ^ 0x80808080u;
    return o;
}

// The nearest integers to x lift / s (ties to even), s well inside the normal range: the
// signs of x - (n +- 1/2) s are exact.
template <bool F32>
__device__ __noinline__ uint2 codes_exact(uint4 v, float lift, float s, float inv)
{
    constexpr int N = F32 ? 4 : 8;
    uint64_t x[N / 2];
    as_pairs<F32>(v, x);
    uint32_t m[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float y = (e & 1 ? second_of(x[e / 2]) : first_of(x[e / 2])) * lift;
        float n = rintf(y * inv);
        const float up = fmaf(-(n + 0.5f), s, y), down = fmaf(-(n - 0.5f), s, y);
        const bool odd = ((int)n & 1) != 0;
        if (up > 0.0f || (up == 0.0f && odd)) n += 1.0f;
        else if (down < 0.0f || (down == 0.0f && odd)) n -= 1.0f;
        m[e] = (uint32_t)((int)fminf(fmaxf(n, -127.0f), 127.0f) + 128);
    }
    return pack<F32>(m);
}

// What n, an integer next to x / s with n - x / s about d, is off by: 1 or -1 where
// x / s lies past the border n +- 1/2, or on it and n (of whose bits m has the last) is odd.
// The sign of x - (n +- 1/2) s is exact.
__device__ __forceinline__ uint32_t beyond_border(float x, float s, float n, float d, uint32_t m)
{
    const bool above = __float_as_int(d) < 0;         // x / s is above n (where d is 0, either side will do)
    const float t = fmaf(-(n + (above ? 0.5f : -0.5f)), s, x), past = above ? t : -t;
    const bool off = past > 0.0f || (past == 0.0f && (m & 1u));
    return off ? (above ? 1u : 0xFFFFFFFFu) : 0u;
}

// VEC: rows are read 16 bytes at a time; R threads a row; ONE: one matrix.
template <bool F32, bool VEC, int R, bool ONE>
__global__ void __launch_bounds__(R < 256 ? 256 : R) quantize_kernel(const QuantArgs a)
{
    constexpr int N = F32 ? 4 : 8, NT = R < 256 ? 256 : R, ROWS = NT / R, W = R / 32;
    __shared__ uint32_t part[W > 1 ? NT / 32 : 1];
    const int sub = (int)threadIdx.x / R, tid = (int)threadIdx.x % R;
    const int64_t r = (int64_t)blockIdx.x * ROWS + sub;
    const bool here = r < a.rows;
    const int64_t g = ONE || !here ? 0 : r / a.per, i = here ? r - g * a.per : 0;
    const char *row = static_cast<const char *>(a.X) + (g * a.stridex + i * a.ldx) * (F32 ? 4 : 2);
    const int cols = here ? a.cols : 0;
    uint4 v[kPieces];
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        const int c = (p * R + tid) * N;
        v[p] = make_uint4(0u, 0u, 0u, 0u);
        if (c < cols) v[p] = load_values16<F32, VEC>(row, c, cols);
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p) top = largest<F32>(v[p], top);
    for (int64_t c = (int64_t)(kPieces * R + tid) * N; c < cols; c += R * N)
        top = largest<F32>(load_values16<F32, VEC>(row, (int)c, cols), top);
    if constexpr (!F32) top = max(top & 0x7FFFu, top >> 16 & 0x7FFFu) << 16;
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if constexpr (W > 1) {
        if (lane_id() == 0) part[threadIdx.x >> 5] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) top = max(top, part[sub * W + w]);
    }
    if (!here) return;
    const bool finite = top < 0x7F800000u;
    const float amax = __uint_as_float(top);
    float s = __fdiv_rn(amax, 127.0f);
    if (tid == 0) {
        a.scales[r] = finite ? s : __uint_as_float(0x7FFFFFFFu);
        if (!finite && a.flags) atomicOr(a.flags, (uint32_t)EMU_FLAG_NONFINITE);
    }
    // tiny rows are lifted by a power of two, away from the subnormal range, where differences
    // lose their sign (a scale that is itself rounded there can give codes above 127: codes_exact clamps)
    const bool tiny = amax < 0x1p-60f;
    const float lift = tiny ? 0x1p80f : 1.0f;
    s *= lift;
    const bool none = !finite || !(s > 0.0f);         // such rows have zero codes
    const float inv = none ? 0.0f : __frcp_rn(s);
    const uint64_t inv2 = both(inv), minus_inv2 = both(-inv);
    int8_t *q = a.q + g * a.strideq + i * a.ldq;
    const bool words = ((reinterpret_cast<uintptr_t>(q)) & (N - 1u)) == 0;
    auto piece = [&](uint4 w, int c) {
        uint64_t x[N / 2];
        as_pairs<F32>(w, x);
        uint32_t m[N];
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
            // 1.5 * 2^23 has the units at its last bit: the low byte of the sum is the integer (+ 128)
            const uint64_t b = fma2(x[e], inv2, both(12583040.0f));
            const uint64_t n = add2(b, both(-12583040.0f)), d = fma2(x[e], minus_inv2, n);
            m[2 * e] = (uint32_t)b;
            m[2 * e + 1] = (uint32_t)(b >> 32);
            const float d0 = first_of(d), d1 = second_of(d);
            if (fmaxf(fabsf(d0), fabsf(d1)) > 0.4999f) {
                m[2 * e] += beyond_border(first_of(x[e]), s, first_of(n), d0, m[2 * e]);
                m[2 * e + 1] += beyond_border(second_of(x[e]), s, second_of(n), d1, m[2 * e + 1]);
            }
        }
        uint2 o = tiny ? codes_exact<F32>(w, lift, s, inv) : pack<F32>(m);
        if (none) o = make_uint2(0u, 0u);
        int8_t *to = q + c;
        if (words && c + N <= cols) {
            if constexpr (F32) *reinterpret_cast<uint32_t *>(to) = o.x;
            else *reinterpret_cast<uint2 *>(to) = o;
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (c + e < cols) to[e] = (int8_t)((e < 4 ? o.x : o.y) >> (8 * (e & 3)) & 0xFFu);
        }
    };
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        const int c = (p * R + tid) * N;
        if (c < cols) piece(v[p], c);
    }
    for (int64_t c = (int64_t)(kPieces * R + tid) * N; c < cols; c += R * N) piece(load_values16<F32, VEC>(row, (int)c, cols), (int)c);
}

template <bool F32, bool VEC, int R>
cudaError_t run(const QuantArgs &a, cudaStream_t st)
{
    constexpr int NT = R < 256 ? 256 : R, ROWS = NT / R;
    const unsigned grid = (unsigned)((a.rows + ROWS - 1) / ROWS);
    if (a.per == a.rows) quantize_kernel<F32, VEC, R, true><<<grid, NT, 0, st>>>(a);
    else quantize_kernel<F32, VEC, R, false><<<grid, NT, 0, st>>>(a);
    return cudaGetLastError();
}

// As few threads a row as hold it in registers.  (16 pieces a thread, a fourth of the threads:
// 66 us for 16384 x 4096 in BF16 against 40; twice the threads with half of their pieces unused: 16384 x
// 4096 in FP32 79 us.)
template <bool F32, bool VEC>
cudaError_t by_width(const QuantArgs &a, cudaStream_t st)
{
    const int pieces = (a.cols + (F32 ? 3 : 7)) / (F32 ? 4 : 8), least = (pieces + kPieces - 1) / kPieces;
    return least <= 32 ? run<F32, VEC, 32>(a, st) : least <= 64 ? run<F32, VEC, 64>(a, st) : least <= 128 ? run<F32, VEC, 128>(a, st)
           : least <= 256 ? run<F32, VEC, 256>(a, st) : run<F32, VEC, 512>(a, st);
}

}  // namespace

cudaError_t launch_i8_quantize(bool f32, int64_t G, int64_t rows, int64_t cols, const void *X, int64_t ldx, int64_t stridex,
                               int8_t *q, int64_t ldq, int64_t strideq, float *scales, uint32_t *flags, cudaStream_t st)
{
    if (G * rows == 0) return cudaSuccess;
    QuantArgs a = {};
    a.X = X; a.rows = G * rows; a.per = rows; a.ldx = ldx; a.stridex = G > 1 ? stridex : 0;
    a.q = q; a.ldq = ldq; a.strideq = G > 1 ? strideq : 0; a.scales = scales; a.flags = flags; a.cols = (int)cols;
    const int es = f32 ? 4 : 2;
    const bool vec = (reinterpret_cast<uintptr_t>(X) & 15u) == 0 && ldx * es % 16 == 0 && a.stridex * es % 16 == 0;
    return f32 ? (vec ? by_width<true, true>(a, st) : by_width<true, false>(a, st))
               : (vec ? by_width<false, true>(a, st) : by_width<false, false>(a, st));
}

}  // namespace emu
