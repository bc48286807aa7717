// Launches of the expert-layer kernels, called by the C entry points.
#pragma once

#include "../../include/emu_experts.h"
#include "common.cuh"
#include "launchers.cuh"

namespace emu {

// Products grouped by expert (grouped.cu).  One operand as planes: S planes
// `plane` elements apart, row pitch ld; weights: matrices `stride` elements
// apart; token rows: `rows` plane rows, `padded` when each group starts at
// padded_start (grouped_common.cuh) and ends in zero rows.
struct GroupedOperand {
    const uint16_t *planes = nullptr;
    int64_t rows = 0, ld = 0, stride = 0, plane = 0;
    bool padded = false;       // (three planes of a gradient's operands: always)
};
cudaError_t launch_grouped_split(bool f32, int64_t G, int64_t rows, int64_t cols, const void *X, int64_t ldx,
                                 int64_t stride, uint16_t *comps, int64_t ldcomp, uint32_t *flags, cudaStream_t st);
cudaError_t launch_grouped_split_rows(bool f32, int64_t rows, int64_t cols, const void *X, int64_t xrows,
                                      int64_t ldx, const int32_t *src, const int32_t *ends, int64_t G,
                                      uint16_t *comps, int64_t ldcomp, uint32_t *flags, cudaStream_t st);
// own_flags: nothing else sets the flag word (the kernel clears it).
cudaError_t launch_grouped_product(int nslices, bool trans, int64_t G, int64_t rows, int64_t N, int64_t K,
                                   const GroupedOperand &X, const GroupedOperand &W, const int32_t *ends, void *Y,
                                   bool y_f32, int64_t ldy, uint32_t *flags, bool own_flags, cudaStream_t st);
// FP32 weights that meet few rows each, split inside the product
// (grouped_fused.cu); fused_takes: whether their rows can be read by TMA;
// kFusedRows: up to so many rows for each group on average that is the faster
// way (16 groups of 1024 x 2048: 64 rows 44 us against 103 through planes, 256 115
// and 141, 384 170 and 182, 512 216 and 205; 8 of 4096 x 4096: 384 603 and 658, 512
// 778 and 723).
bool fused_takes(const float *W, int64_t G, int64_t ldw, int64_t stridew);
cudaError_t launch_grouped_fused(bool trans, int64_t G, int64_t rows, int64_t N, int64_t K, const GroupedOperand &X,
                                 const float *W, int64_t ldw, int64_t stridew, const int32_t *ends, float *Y,
                                 int64_t ldy, uint32_t *flags, cudaStream_t st);
constexpr int64_t kFusedRows = 448;
cudaError_t launch_grouped_gradient(int nslices, int64_t G, int64_t rows, int64_t M, int64_t N, const GroupedOperand &A,
                                    const GroupedOperand &B, const int32_t *ends, void *D, bool d_f32, int64_t ldd,
                                    int64_t strided, uint32_t *flags, bool own_flags, cudaStream_t st);

// Matrix-vector products with 4-bit weights (w4.cu), routing and the weighted
// sum of answers (route.cu).
cudaError_t launch_w4_matvec(bool x_f32, int64_t G, int64_t rows, int64_t N, int64_t K, int group, const void *X,
                             int64_t ldx, const uint8_t *q, const void *scales, bool s_f32, const uint8_t *zeros,
                             const int32_t *ends, void *Y, int64_t ldy, uint16_t *planes, uint32_t *flags,
                             cudaStream_t st);
bool w4_direct(bool x_f32, const void *X, int64_t ldx);     // X is read as it is, without planes
size_t route_scratch_bytes(int64_t E);
cudaError_t launch_route(int64_t T, int64_t E, int k, bool renorm, const void *logits, bool f32, int64_t ldl,
                         float *weights, int32_t *experts, int32_t *slots, int32_t *rows, int32_t *ends,
                         int32_t *counts, WsHeader *ws, cudaStream_t st, uint32_t missing = 0,
                         unsigned long long limit_ns = kWaitLimitNs);      // missing: arrivals that never come
cudaError_t launch_route_backward(int64_t T, int64_t E, int k, bool renorm, const void *logits, bool f32, int64_t ldl,
                                  const int32_t *experts, const float *dw, void *dl, int64_t lddl, cudaStream_t st);
cudaError_t launch_combine(bool f32, int64_t T, int k, int64_t cols, const void *Y, int64_t yrows, int64_t ldy,
                           const int32_t *slots, const float *weights, void *O, int64_t ldo, cudaStream_t st);
cudaError_t launch_combine_backward(bool f32, int64_t T, int k, int64_t cols, const void *dO, int64_t lddo,
                                    const void *Y, int64_t yrows, int64_t ldy, const int32_t *slots,
                                    const float *weights, void *dY, int64_t lddy, float *dw, int32_t *owner,
                                    cudaStream_t st);       // owner: [yrows], or NULL: unnamed rows of dY are left

// Balance loss of the routing (balance.cu).
size_t balance_scratch_bytes(int64_t T, int64_t E);      // 0: none
cudaError_t launch_balance(int64_t T, int64_t E, int k, const void *logits, bool f32, int64_t ldl, const int32_t *experts,
                           const uint8_t *mask, float coef, float *loss, int32_t *counts, int32_t *tokens, void *scratch,
                           uint32_t *flags, cudaStream_t st);
cudaError_t launch_balance_backward(int64_t T, int64_t E, int k, const void *logits, bool f32, int64_t ldl,
                                    const int32_t *counts, const int32_t *tokens, const uint8_t *mask, float coef, const float *dloss,
                                    const void *add, int64_t lda, void *dlogits, int64_t ldd, cudaStream_t st);

// 8-bit integers (i8_*.cu): rows to codes, and products of codes.
cudaError_t launch_i8_quantize(bool f32, int64_t G, int64_t rows, int64_t cols, const void *X, int64_t ldx, int64_t stridex,
                               int8_t *q, int64_t ldq, int64_t strideq, float *scales, uint32_t *flags, cudaStream_t st);
struct I8Product {
    const int8_t *X, *W;
    const float *xscales, *wscales;        // or NULL: 1
    const int32_t *src, *ends;             // or NULL: row r is X's, one group
    int64_t xrows, ldx, ldw, stridew, ldy;
    void *Y;
    int ytype, G, rows, N, K;
    uint32_t *flags;                       // (NULL for launch_i8_rows: none are reported)
};
cudaError_t launch_i8_rows(const I8Product &p, cudaStream_t st);
bool i8_few_rows(int64_t G, int64_t rows, int64_t N, int64_t K);      // launch_i8_rows is the faster way
// On the tensor cores, many rows (i8_tile.cu), or some in one launch with K in `parts` (i8_batch.cu); scratch: the
// bytes below (aligned: X's and W's rows can be read 16 bytes at a time).
size_t i8_tile_scratch_bytes(int64_t G, int64_t rows, int64_t N, int64_t K, bool aligned);
cudaError_t launch_i8_tile(I8Product p, void *scratch, cudaStream_t st);
size_t i8_batch_scratch_bytes(int64_t G, int64_t rows, int64_t N, int64_t K, bool aligned);
cudaError_t launch_i8_batch(I8Product p, int parts, void *scratch, cudaStream_t st,
                            unsigned long long selftest_ns = 0);      // not 0: no products, a wait that runs out

}  // namespace emu
