// Pieces shared by the kernels of the 8-bit integer operators.
#pragma once

#include "grouped_common.cuh"
#include "expert_launchers.cuh"
#include "split_f32_pair.cuh"

namespace emu {

// Up to 16 consecutive codes from p on, as four words, zeros past the n-th.  WIDE: p
// is 16-byte aligned (then n >= 16 is one load).
template <bool WIDE>
__device__ __forceinline__ uint4 load_codes(const int8_t *p, int n)
{
    if (WIDE && n >= 16) return __ldg(reinterpret_cast<const uint4 *>(p));
    uint32_t w[4];
    if (n >= 16 && (reinterpret_cast<uintptr_t>(p) & 3u) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __ldg(reinterpret_cast<const uint32_t *>(p) + i);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b)
                if (4 * i + b < n) w[i] |= (uint32_t)(uint8_t)__ldg(p + 4 * i + b) << (8 * b);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One value of a product: the sum of codes' products times the channel's and the
// token's scale, in FP32 (three roundings of 2^-24), then rounded to the result's type.
__device__ __forceinline__ float scaled_sum(int sum, float wscale, float xscale)
{
    return __int2float_rn(sum) * wscale * xscale;
}

// A result: FP32, BF16 or the sum itself.
__device__ __forceinline__ void store_value(const I8Product &p, int64_t row, int n, float y, int sum)
{
    const int64_t at = row * p.ldy + n;
    if (p.ytype == EMU_F32) static_cast<float *>(p.Y)[at] = y;
    else if (p.ytype == EMU_BF16) static_cast<uint16_t *>(p.Y)[at] = (uint16_t)bf16x2_rn(y, 0.0f);
    else static_cast<int32_t *>(p.Y)[at] = sum;
}

// Whether rows of codes can be read 16 at a time.
inline bool aligned_codes(const void *q, int64_t ld, int64_t stride)
{
    return ((reinterpret_cast<uintptr_t>(q) | (uintptr_t)ld | (uintptr_t)stride) & 15u) == 0;
}

// Whether the tensor memory accelerator can read weights as they stand.
inline bool i8_tma_reads(const void *W, int64_t G, int64_t N, int64_t ldw, int64_t stridew)
{
    return G <= 1 ? aligned_codes(W, ldw, 0) : aligned_codes(W, ldw, stridew) && stridew >= N * ldw;
}

}  // namespace emu
