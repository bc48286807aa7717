// Rows to 8-bit integers with a scale for each row:
//   s = max_k |x_k| / 127, rounded to FP32; q_k = x_k / s rounded to the nearest
// integer, ties to even, exactly (the quotient is never rounded first), so that the
// codes are a matter of definition and not of the way to them.
//
// A quotient's nearest integer comes from x times the reciprocal (off by less than
// 2e-5), and where that lies within 1e-4 of the border between two integers, from the sign of
// x - (n +- 1/2) s, which one fused multiply-add gives exactly.
//
// A group of R threads (32, 128 or 512) has a row, four pieces of 16 bytes a thread in
// registers: each element is read once while rows have up to 4 R pieces, longer rows are read
// again from L2.
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

template <bool F32>
__device__ __forceinline__ void as_floats(uint4 v, float (&x)[F32 ? 4 : 8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
            x[i] = __uint_as_float(w[i]);
        } else {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

// Bits of the largest magnitude: magnitudes order like their bits, NaN above infinity.
template <bool F32>
__device__ __forceinline__ uint32_t largest(uint4 v, uint32_t top)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
            top = max(top, w[i] & 0x7FFFFFFFu);
        } else {
            top = max(top, w[i] << 16 & 0x7FFFFFFFu);
            top = max(top, w[i] & 0x7FFF0000u);
        }
    }
    return top;
}

// The nearest integer to x / s (ties to even), for s well inside the normal range.
__device__ __noinline__ int nearest_exact(float x, float s, float inv)
{
    float n = rintf(x * inv);
    const float up = fmaf(-(n + 0.5f), s, x), down = fmaf(-(n - 0.5f), s, x);     // signs are exact
    const bool odd = ((int)n & 1) != 0;
    if (up > 0.0f || (up == 0.0f && odd)) n += 1.0f;
    else if (down < 0.0f || (down == 0.0f && odd)) n -= 1.0f;
    return (int)fminf(fmaxf(n, -127.0f), 127.0f);
}

template <bool F32, bool VEC, int R>
__global__ void __launch_bounds__(R < 256 ? 256 : R) quantize_kernel(const QuantArgs a)
{
    constexpr int N = F32 ? 4 : 8, NT = R < 256 ? 256 : R, ROWS = NT / R, W = R / 32;
    __shared__ uint32_t part[W > 1 ? NT / 32 : 1];
    const int sub = (int)threadIdx.x / R, tid = (int)threadIdx.x % R;
    const int64_t r = (int64_t)blockIdx.x * ROWS + sub;
    const bool here = r < a.rows;
    const int64_t g = here ? r / a.per : 0, i = here ? r - g * a.per : 0;
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
    // tiny rows: scaled up by a power of two, away from the subnormal range, where differences
    // lose their sign (a scale that is itself rounded there can give codes above 127: nearest_exact clamps)
    const bool tiny = amax < 0x1p-60f;
    const float lift = tiny ? 0x1p80f : 1.0f;
    s *= lift;
    const bool some = finite && s > 0.0f;
    const float inv = some ? __frcp_rn(s) : 0.0f;
    int8_t *q = a.q + g * a.strideq + i * a.ldq;
    auto piece = [&](uint4 w, int c) {
        float x[N];
        as_floats<F32>(w, x);
        uint32_t m[N];
        bool close = tiny;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float y = some ? x[e] * inv : 0.0f, b = y + 12582912.0f;     // 1.5 * 2^23: the low bits are the integer
            m[e] = __float_as_uint(b);
            close |= fabsf(y - (b - 12582912.0f)) > 0.4999f;
        }
        if (close) {
#pragma unroll
            for (int e = 0; e < N; ++e) m[e] = some ? (uint32_t)nearest_exact(x[e] * lift, s, inv) : 0u;
        }
        uint32_t o[N / 4];
#pragma unroll
        for (int j = 0; j < N / 4; ++j)
            o[j] = __byte_perm(__byte_perm(m[4 * j], m[4 * j + 1], 0x0040), __byte_perm(m[4 * j + 2], m[4 * j + 3], 0x0040), 0x5410);
        int8_t *to = q + c;
        if (c + N <= cols && (reinterpret_cast<uintptr_t>(to) & (N - 1u)) == 0) {
            if constexpr (F32) *reinterpret_cast<uint32_t *>(to) = o[0];
            else *reinterpret_cast<uint2 *>(to) = make_uint2(o[0], o[1]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (c + e < cols) to[e] = (int8_t)(m[e] & 0xFFu);
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
    quantize_kernel<F32, VEC, R><<<(unsigned)((a.rows + ROWS - 1) / ROWS), NT, 0, st>>>(a);
    return cudaGetLastError();
}

// As few threads a row as hold it in registers.
template <bool F32, bool VEC>
cudaError_t by_width(const QuantArgs &a, cudaStream_t st)
{
    const int pieces = (a.cols + (F32 ? 3 : 7)) / (F32 ? 4 : 8);
    return pieces <= 32 * kPieces ? run<F32, VEC, 32>(a, st) : pieces <= 128 * kPieces ? run<F32, VEC, 128>(a, st)
                                                                                        : run<F32, VEC, 512>(a, st);
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
