// C-ABI of the expert layers (declared in include/emu_experts.h):
// argument checks, workspace layout and launch sequences.
#include "grouped_common.cuh"
#include "expert_launchers.cuh"

using namespace emu;

namespace {

// Kernels index with 32-bit coordinates, which they take up to a tile, a stage or
// a block's share past the last element: sizes that they walk through stay
// below kMaxWalk.
constexpr int64_t kMaxDim = (int64_t)1 << 31, kMaxWalk = kMaxDim - 65536;

int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// Whether p is aligned to its elements.
bool fits(const void *p, int type) { return (reinterpret_cast<uintptr_t>(p) & (type == EMU_F32 ? 3u : 1u)) == 0; }
emu_status cuda_status(cudaError_t e) { return e == cudaSuccess ? EMU_OK : EMU_ERR_CUDA; }
int64_t plane_ld(int64_t cols) { return round_up(cols < 1 ? 1 : cols, 8); }
bool known(int dtype) { return dtype == EMU_F32 || dtype == EMU_BF16; }

emu_status check_ws(void *ws, size_t ws_bytes, size_t need)
{
    if (!ws) return EMU_ERR_INVALID_ARG;
    if (ws_bytes < need) return EMU_ERR_WORKSPACE_TOO_SMALL;
    return aligned16(ws) ? EMU_OK : EMU_ERR_MISALIGNED;
}

cudaError_t clear_flags(void *ws, cudaStream_t st)
{
    return cudaMemsetAsync(&static_cast<WsHeader *>(ws)->flags, 0, sizeof(uint32_t), st);
}

// Takes EMU_KEEP_FLAGS off a type or a number of slices.
bool take_keep(int &arg)
{
    const bool keep = arg >= 0 && (arg & EMU_KEEP_FLAGS) != 0;
    if (keep) arg &= ~EMU_KEEP_FLAGS;
    return keep;
}

// Sizes of a grouped call: G groups over `rows` rows, a and b the two matrix
// dimensions; also keeps the tile counts within 32 bits.
emu_status check_sizes(int64_t G, int64_t rows, int64_t a, int64_t b)
{
    if (G < 1 || rows < 0 || a < 0 || b < 0) return EMU_ERR_INVALID_ARG;
    if (G > kMaxGroups || rows >= kMaxWalk || a >= kMaxWalk || b >= kMaxWalk || G * a >= kMaxDim || G * b >= kMaxDim)
        return EMU_ERR_UNSUPPORTED;
    const int64_t ta = a / 128 + 1, tb = b / 128 + 1;
    if ((rows / 64 + G + 1) * ta >= kMaxDim || (rows / 64 + G + 1) * tb >= kMaxDim || G * ta >= kMaxDim / tb)
        return EMU_ERR_UNSUPPORTED;
    return EMU_OK;
}

// A matrix operand as the tensor memory accelerator reads it.
emu_status check_planes(const void *p, int64_t ld, int64_t cols, int64_t stride)
{
    if (!p || ld < cols) return EMU_ERR_INVALID_ARG;
    if (!aligned16(p) || ld % 8 != 0 || stride % 8 != 0) return EMU_ERR_MISALIGNED;
    return EMU_OK;
}

cudaError_t zero_rows(void *p, int64_t rows, int64_t cols, int64_t ld, int esize, cudaStream_t st)
{
    if (rows <= 0 || cols <= 0) return cudaSuccess;
    return cudaMemset2DAsync(p, (size_t)ld * esize, 0, (size_t)cols * esize, (size_t)rows, st);
}

emu_status product(int S, int opW, int64_t G, int64_t rows, int64_t N, int64_t K, const GroupedOperand &X,
                   const GroupedOperand &W, const int32_t *ends, void *Y, int ytype, int64_t ldy, uint32_t *flags,
                   bool own_flags, cudaStream_t st)
{
    const int esize = ytype == EMU_F32 ? 4 : 2;
    if (rows == 0 || N == 0) return EMU_OK;
    if (K == 0) return cuda_status(zero_rows(Y, rows, N, ldy, esize, st));
    return cuda_status(launch_grouped_product(S, opW == EMU_OP_T, G, rows, N, K, X, W, ends, Y, ytype == EMU_F32, ldy,
                                              flags, own_flags, st));
}

emu_status check_route(int dtype, int64_t T, int64_t E, int64_t k, const void *logits, int64_t ldl, const float *weights,
                       const int32_t *experts, const int32_t *slots, const int32_t *rows, const int32_t *ends, void *ws,
                       size_t ws_bytes)
{
    if (!known(dtype) || T < 0 || E < 1 || k < 1 || k > E || ldl < E || !ends) return EMU_ERR_INVALID_ARG;
    if (E > kMaxGroups || k > 32 || T >= kMaxWalk / k) return EMU_ERR_UNSUPPORTED;
    if (T > 0 && (!logits || !weights || !experts || !slots || !rows)) return EMU_ERR_INVALID_ARG;
    if (!fits(logits, dtype) || !fits(weights, EMU_F32) || !fits(experts, EMU_F32) || !fits(slots, EMU_F32) ||
        !fits(rows, EMU_F32) || !fits(ends, EMU_F32))
        return EMU_ERR_MISALIGNED;
    return check_ws(ws, ws_bytes, kWsHeaderBytes + route_scratch_bytes(E));
}

int32_t *route_counts(void *ws) { return reinterpret_cast<int32_t *>(static_cast<char *>(ws) + kWsHeaderBytes); }

emu_status check_combine_backward(int dtype, int64_t T, int64_t k, int64_t cols, const void *dO, int64_t lddo,
                                  const void *Y, int64_t yrows, int64_t ldy, const int32_t *slots,
                                  const float *weights, const void *dY, int64_t lddy, const float *dweights)
{
    if (!known(dtype) || T < 0 || k < 1 || cols < 0 || yrows < 0 || lddo < cols || lddy < cols ||
        (dweights && ldy < cols))
        return EMU_ERR_INVALID_ARG;
    if (k >= 65536 || T >= kMaxDim / k || cols >= kMaxDim - 8 || yrows >= kMaxDim) return EMU_ERR_UNSUPPORTED;
    if (T > 0 && (!slots || (cols > 0 && (!dO || (yrows > 0 && (!dY || (dweights && !Y))))))) return EMU_ERR_INVALID_ARG;
    if (T > 0 && (!fits(dO, dtype) || !fits(Y, dtype) || !fits(dY, dtype) || !fits(weights, EMU_F32) ||
                  !fits(dweights, EMU_F32) || !fits(slots, EMU_F32)))
        return EMU_ERR_MISALIGNED;
    return EMU_OK;
}

}  // namespace

extern "C" {

int64_t emu_grouped_plane_rows(int64_t rows, int64_t G)
{
    return rows < 0 || G < 1 ? 0 : padded_rows(rows, G);
}

emu_status emu_grouped_split(int dtype, int64_t G, int64_t rows, int64_t cols, const void *X, int64_t ldx,
                             int64_t stridex, uint16_t *comps, int64_t ldcomp, void *ws, size_t ws_bytes,
                             emu_stream_t stream)
{
    const bool keep = take_keep(dtype);
    if (!known(dtype) || ldx < cols || (G > 1 && stridex < 0)) return EMU_ERR_INVALID_ARG;
    emu_status s = check_sizes(G, 0, rows, cols);
    if (s != EMU_OK) return s;
    if (G * rows > 0 && cols > 0) {
        if (!X) return EMU_ERR_INVALID_ARG;
        if (!fits(X, dtype)) return EMU_ERR_MISALIGNED;
        s = check_planes(comps, ldcomp, cols, 0);
        if (s != EMU_OK) return s;
    }
    s = check_ws(ws, ws_bytes, kWsHeaderBytes);
    if (s != EMU_OK) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e = keep ? cudaSuccess : clear_flags(ws, st);
    if (e == cudaSuccess)
        e = launch_grouped_split(dtype == EMU_F32, G, rows, cols, X, ldx, stridex, comps, ldcomp,
                                 &static_cast<WsHeader *>(ws)->flags, st);
    return cuda_status(e);
}

emu_status emu_grouped_split_rows(int dtype, int64_t rows, int64_t cols, const void *X, int64_t xrows, int64_t ldx,
                                  const int32_t *src, const int32_t *ends, int64_t G, uint16_t *comps,
                                  int64_t ldcomp, void *ws, size_t ws_bytes, emu_stream_t stream)
{
    const bool keep = take_keep(dtype);
    if (!known(dtype) || xrows < 0 || ldx < cols || (!src && xrows < rows)) return EMU_ERR_INVALID_ARG;
    emu_status s = check_sizes(G, rows, cols, 0);
    if (s != EMU_OK) return s;
    if (rows > 0 && cols > 0) {
        if (!ends || (xrows > 0 && !X)) return EMU_ERR_INVALID_ARG;
        if (!fits(X, dtype) || !fits(src, EMU_F32) || !fits(ends, EMU_F32)) return EMU_ERR_MISALIGNED;
        s = check_planes(comps, ldcomp, cols, 0);
        if (s != EMU_OK) return s;
    }
    s = check_ws(ws, ws_bytes, kWsHeaderBytes);
    if (s != EMU_OK) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e = keep ? cudaSuccess : clear_flags(ws, st);
    if (e == cudaSuccess && rows > 0 && cols > 0)
        e = launch_grouped_split_rows(dtype == EMU_F32, rows, cols, X, xrows, ldx, src, ends, G, comps, ldcomp,
                                      &static_cast<WsHeader *>(ws)->flags, st);
    return cuda_status(e);
}

emu_status emu_grouped_prodsum(int nslices, int opW, int64_t G, int64_t rows, int64_t N, int64_t K,
                               const uint16_t *Xcomps, int64_t ldx, int padded, const uint16_t *Wcomps, int64_t ldw,
                               int64_t stridew, const int32_t *ends, void *Y, int ytype, int64_t ldy, void *ws,
                               size_t ws_bytes, emu_stream_t stream)
{
    const bool keep = take_keep(nslices);
    if ((nslices != 1 && nslices != 3) || (opW != EMU_OP_N && opW != EMU_OP_T) || !known(ytype) || ldy < N)
        return EMU_ERR_INVALID_ARG;
    emu_status s = check_sizes(G, rows, N, K);
    if (s != EMU_OK) return s;
    const int64_t wrows = opW == EMU_OP_T ? N : K, wcols = opW == EMU_OP_T ? K : N;
    if (rows > 0 && N > 0) {
        if (!ends || !Y) return EMU_ERR_INVALID_ARG;
        if (!fits(ends, EMU_F32) || !fits(Y, ytype)) return EMU_ERR_MISALIGNED;
        if (K > 0) {
            // slices of the weights are planes of G dense matrices
            if (nslices == 3 && G > 1 && stridew != wrows * ldw) return EMU_ERR_INVALID_ARG;
            if (G > 1 && stridew < (wrows - 1) * ldw + wcols) return EMU_ERR_INVALID_ARG;      // matrices overlap
            s = check_planes(Xcomps, ldx, K, 0);
            if (s == EMU_OK) s = check_planes(Wcomps, ldw, wcols, G > 1 ? stridew : 0);
            if (s != EMU_OK) return s;
        }
    }
    s = check_ws(ws, ws_bytes, kWsHeaderBytes);
    if (s != EMU_OK) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool runs = rows > 0 && N > 0 && K > 0;     // the kernel then sets the flag word itself
    if (!runs && !keep && clear_flags(ws, st) != cudaSuccess) return EMU_ERR_CUDA;
    GroupedOperand X, W;
    X.planes = Xcomps; X.rows = padded ? padded_rows(rows, G) : rows; X.ld = ldx; X.plane = X.rows * ldx;
    X.padded = padded != 0;
    W.planes = Wcomps; W.ld = ldw; W.stride = stridew; W.plane = G * wrows * ldw;
    return product(nslices, opW, G, rows, N, K, X, W, ends, Y, ytype, ldy, &static_cast<WsHeader *>(ws)->flags, !keep, st);
}

size_t emu_grouped_gemm_workspace_bytes(int dtype, int64_t G, int64_t rows, int64_t N, int64_t K)
{
    if (G < 1 || rows < 0 || N < 0 || K < 0) return 0;
    if (dtype != EMU_F32) return kWsHeaderBytes;
    // planes of the weights in the larger of their two orientations
    const int64_t w = N * plane_ld(K) > K * plane_ld(N) ? N * plane_ld(K) : K * plane_ld(N);
    return kWsHeaderBytes + (size_t)round_up(3 * padded_rows(rows, G) * plane_ld(K) * 2, 256) +
           (size_t)round_up(3 * G * w * 2, 256);
}

emu_status emu_grouped_gemm_f32(int opW, int64_t G, int64_t rows, int64_t N, int64_t K, const float *X, int64_t xrows,
                                int64_t ldx, const int32_t *src, const float *W, int64_t ldw, int64_t stridew,
                                const int32_t *ends, float *Y, int64_t ldy, void *ws, size_t ws_bytes,
                                emu_stream_t stream)
{
    if ((opW != EMU_OP_N && opW != EMU_OP_T) || ldy < N || ldx < K || xrows < 0 || (!src && xrows < rows))
        return EMU_ERR_INVALID_ARG;
    emu_status s = check_sizes(G, rows, N, K);
    if (s != EMU_OK) return s;
    const int64_t wrows = opW == EMU_OP_T ? N : K, wcols = opW == EMU_OP_T ? K : N;
    if (ldw < wcols || (G > 1 && stridew < 0)) return EMU_ERR_INVALID_ARG;
    if (rows > 0 && N > 0 && (!ends || !Y || (K > 0 && (!W || (xrows > 0 && !X))))) return EMU_ERR_INVALID_ARG;
    if (!fits(X, EMU_F32) || !fits(W, EMU_F32) || !fits(Y, EMU_F32) || !fits(src, EMU_F32) || !fits(ends, EMU_F32))
        return EMU_ERR_MISALIGNED;
    s = check_ws(ws, ws_bytes, emu_grouped_gemm_workspace_bytes(EMU_F32, G, rows, N, K));
    if (s != EMU_OK) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    uint32_t *flags = &static_cast<WsHeader *>(ws)->flags;
    if (clear_flags(ws, st) != cudaSuccess) return EMU_ERR_CUDA;
    GroupedOperand xo, wo;
    if (rows > 0 && N > 0 && K > 0) {
        uint16_t *xp = reinterpret_cast<uint16_t *>(static_cast<char *>(ws) + kWsHeaderBytes);
        xo.rows = padded_rows(rows, G); xo.ld = plane_ld(K); xo.plane = xo.rows * xo.ld; xo.padded = true; xo.planes = xp;
        uint16_t *wp = reinterpret_cast<uint16_t *>(reinterpret_cast<char *>(xp) + round_up(3 * xo.plane * 2, 256));
        wo.ld = plane_ld(wcols); wo.stride = wrows * wo.ld; wo.plane = G * wo.stride; wo.planes = wp;
        cudaError_t e = launch_grouped_split_rows(true, rows, K, X, xrows, ldx, src, ends, G, xp, xo.ld, flags, st);
        if (e == cudaSuccess && rows <= kFusedRows * G && fused_takes(W, G, ldw, stridew))
            return cuda_status(launch_grouped_fused(opW == EMU_OP_T, G, rows, N, K, xo, W, ldw, stridew, ends, Y, ldy, flags, st));
        if (e == cudaSuccess) e = launch_grouped_split(true, G, wrows, wcols, W, ldw, stridew, wp, wo.ld, flags, st);
        if (e != cudaSuccess) return EMU_ERR_CUDA;
    }
    return product(3, opW, G, rows, N, K, xo, wo, ends, Y, EMU_F32, ldy, flags, false, st);
}

emu_status emu_grouped_prodsum_wgrad(int nslices, int64_t G, int64_t rows, int64_t M, int64_t N,
                                     const uint16_t *Acomps, int64_t lda, int apadded, const uint16_t *Bcomps,
                                     int64_t ldb, int bpadded, const int32_t *ends, void *D, int dtype, int64_t ldd,
                                     int64_t strided, void *ws, size_t ws_bytes, emu_stream_t stream)
{
    const bool keep = take_keep(nslices);
    if ((nslices != 1 && nslices != 3) || (nslices == 3 && (!apadded || !bpadded)) || !known(dtype) || ldd < N || (G > 1 && strided < M * ldd))
        return EMU_ERR_INVALID_ARG;
    emu_status s = check_sizes(G, rows, M, N);
    if (s != EMU_OK) return s;
    if (M > 0 && N > 0) {
        if (!D) return EMU_ERR_INVALID_ARG;
        if (!fits(D, dtype) || !fits(ends, EMU_F32)) return EMU_ERR_MISALIGNED;
        if (rows > 0) {
            if (!ends) return EMU_ERR_INVALID_ARG;
            s = check_planes(Acomps, lda, M, 0);
            if (s == EMU_OK) s = check_planes(Bcomps, ldb, N, 0);
            if (s != EMU_OK) return s;
        }
    }
    s = check_ws(ws, ws_bytes, kWsHeaderBytes);
    if (s != EMU_OK) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if ((M == 0 || N == 0 || rows == 0) && !keep && clear_flags(ws, st) != cudaSuccess) return EMU_ERR_CUDA;
    if (M == 0 || N == 0) return EMU_OK;
    if (rows == 0) {
        for (int64_t g = 0; g < G; ++g) {
            const int esize = dtype == EMU_F32 ? 4 : 2;
            if (zero_rows(static_cast<char *>(D) + g * strided * esize, M, N, ldd, esize, st) != cudaSuccess)
                return EMU_ERR_CUDA;
        }
        return EMU_OK;
    }
    GroupedOperand A, B;
    A.planes = Acomps; A.padded = apadded != 0; A.rows = apadded ? padded_rows(rows, G) : rows; A.ld = lda;
    A.plane = A.rows * lda;
    B.planes = Bcomps; B.padded = bpadded != 0; B.rows = bpadded ? padded_rows(rows, G) : rows; B.ld = ldb;
    B.plane = B.rows * ldb;
    return cuda_status(launch_grouped_gradient(nslices, G, rows, M, N, A, B, ends, D, dtype == EMU_F32, ldd, strided,
                                               &static_cast<WsHeader *>(ws)->flags, !keep, st));
}

// The flag word and the slices.
size_t emu_w4_workspace_bytes(int dtype, int64_t rows, int64_t K)
{
    return rows < 0 || K < 0 ? 0 : kWsHeaderBytes + (size_t)rows * (size_t)K * (dtype == EMU_F32 ? 6 : 2);
}

emu_status emu_w4_matvec(int dtype, int64_t G, int64_t rows, int64_t N, int64_t K, int64_t group, const void *X,
                         int64_t ldx, const uint8_t *q, const void *scales, int stype, const uint8_t *zeros,
                         const int32_t *ends, void *Y, int64_t ldy, void *ws, size_t ws_bytes, emu_stream_t stream)
{
    if (!known(dtype) || !known(stype) || ldx < K || ldy < N || group < 32 || group % 32 != 0 || K < 0 || K % group != 0 ||
        (!ends && G != 1))
        return EMU_ERR_INVALID_ARG;
    emu_status s = check_sizes(G, rows, N, K);
    if (s != EMU_OK) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int esize = dtype == EMU_F32 ? 4 : 2;
    if (rows == 0 || N == 0 || K == 0) {                        // nothing to multiply
        if (rows > 0 && N > 0 && !Y) return EMU_ERR_INVALID_ARG;
        if (ws) {
            s = check_ws(ws, ws_bytes, kWsHeaderBytes);
            if (s != EMU_OK) return s;
            if (clear_flags(ws, st) != cudaSuccess) return EMU_ERR_CUDA;
        }
        return cuda_status(zero_rows(Y, rows, N, ldy, esize, st));
    }
    if (!Y || !X || !q || !scales) return EMU_ERR_INVALID_ARG;
    if (!aligned16(q) || !fits(X, dtype) || !fits(Y, dtype) || !fits(scales, stype) || !fits(ends, EMU_F32))
        return EMU_ERR_MISALIGNED;
    if (rows > 65535 * 2) return EMU_ERR_UNSUPPORTED;           // items of two rows and more on the grid's y dimension
    const bool direct = w4_direct(dtype == EMU_F32, X, ldx);
    if (!direct || ws) {
        s = check_ws(ws, ws_bytes, direct ? kWsHeaderBytes : emu_w4_workspace_bytes(dtype, rows, K));
        if (s != EMU_OK) return s;
    }
    return cuda_status(launch_w4_matvec(dtype == EMU_F32, G, rows, N, K, (int)group, X, ldx, q, scales,
                                        stype == EMU_F32, zeros, ends, Y, ldy,
                                        direct ? nullptr : reinterpret_cast<uint16_t *>(static_cast<char *>(ws) + kWsHeaderBytes),
                                        ws ? &static_cast<WsHeader *>(ws)->flags : nullptr, st));
}

size_t emu_route_workspace_bytes(int64_t T, int64_t E, int64_t k)
{
    (void)T;
    (void)k;
    return E < 1 ? 0 : kWsHeaderBytes + route_scratch_bytes(E);
}

emu_status emu_route(int dtype, int64_t T, int64_t E, int64_t k, int renorm, const void *logits, int64_t ldl,
                     float *weights, int32_t *experts, int32_t *slots, int32_t *rows, int32_t *ends, void *ws,
                     size_t ws_bytes, emu_stream_t stream)
{
    const emu_status s = check_route(dtype, T, E, k, logits, ldl, weights, experts, slots, rows, ends, ws, ws_bytes);
    if (s != EMU_OK) return s;
    return cuda_status(launch_route(T, E, (int)k, renorm != 0, logits, dtype == EMU_F32, ldl, weights, experts, slots,
                                    rows, ends, route_counts(ws), static_cast<WsHeader *>(ws),
                                    reinterpret_cast<cudaStream_t>(stream)));
}

emu_status emu_selftest_route_timeout(uint32_t timeout_us, int64_t T, int64_t E, int64_t k, const float *logits,
                                      int64_t ldl, float *weights, int32_t *experts, int32_t *slots, int32_t *rows,
                                      int32_t *ends, void *ws, size_t ws_bytes, emu_stream_t stream)
{
    if (timeout_us < 1 || timeout_us > 1000000 || T <= 32) return EMU_ERR_INVALID_ARG;      // (32 tokens: one block)
    const emu_status s = check_route(EMU_F32, T, E, k, logits, ldl, weights, experts, slots, rows, ends, ws, ws_bytes);
    if (s != EMU_OK) return s;
    return cuda_status(launch_route(T, E, (int)k, true, logits, true, ldl, weights, experts, slots, rows, ends,
                                    route_counts(ws), static_cast<WsHeader *>(ws),
                                    reinterpret_cast<cudaStream_t>(stream), 1u, 1000ull * timeout_us));
}

emu_status emu_route_backward(int dtype, int64_t T, int64_t E, int64_t k, int renorm, const void *logits, int64_t ldl,
                              const int32_t *experts, const float *dweights, void *dlogits, int64_t lddl,
                              emu_stream_t stream)
{
    if (!known(dtype) || T < 0 || E < 1 || k < 1 || k > E || ldl < E || lddl < E) return EMU_ERR_INVALID_ARG;
    if (E > kMaxGroups || k > 32 || T >= kMaxDim / k) return EMU_ERR_UNSUPPORTED;
    if (T == 0) return EMU_OK;
    if (!logits || !experts || !dweights || !dlogits) return EMU_ERR_INVALID_ARG;
    if (!fits(logits, dtype) || !fits(dlogits, dtype) || !fits(experts, EMU_F32) || !fits(dweights, EMU_F32))
        return EMU_ERR_MISALIGNED;
    return cuda_status(launch_route_backward(T, E, (int)k, renorm != 0, logits, dtype == EMU_F32, ldl, experts,
                                             dweights, dlogits, lddl, reinterpret_cast<cudaStream_t>(stream)));
}

emu_status emu_rows_combine(int dtype, int64_t T, int64_t k, int64_t cols, const void *Y, int64_t yrows, int64_t ldy,
                            const int32_t *slots, const float *weights, void *O, int64_t ldo, emu_stream_t stream)
{
    if (!known(dtype) || T < 0 || k < 1 || cols < 0 || yrows < 0 || ldy < cols || ldo < cols) return EMU_ERR_INVALID_ARG;
    if (k >= 65536 || T >= kMaxDim / k || cols >= kMaxDim - 8 || yrows >= kMaxDim) return EMU_ERR_UNSUPPORTED;
    if (T == 0 || cols == 0) return EMU_OK;
    if (!slots || !O || (yrows > 0 && !Y)) return EMU_ERR_INVALID_ARG;
    if (!fits(Y, dtype) || !fits(O, dtype) || !fits(weights, EMU_F32) || !fits(slots, EMU_F32)) return EMU_ERR_MISALIGNED;
    return cuda_status(launch_combine(dtype == EMU_F32, T, (int)k, cols, Y, yrows, ldy, slots, weights, O, ldo,
                                      reinterpret_cast<cudaStream_t>(stream)));
}

emu_status emu_rows_combine_backward(int dtype, int64_t T, int64_t k, int64_t cols, const void *dO, int64_t lddo,
                                     const void *Y, int64_t yrows, int64_t ldy, const int32_t *slots,
                                     const float *weights, void *dY, int64_t lddy, float *dweights,
                                     emu_stream_t stream)
{
    const emu_status s = check_combine_backward(dtype, T, k, cols, dO, lddo, Y, yrows, ldy, slots, weights, dY, lddy, dweights);
    if (s != EMU_OK || T == 0) return s;
    return cuda_status(launch_combine_backward(dtype == EMU_F32, T, (int)k, cols, dO, lddo, Y, yrows, ldy, slots,
                                               weights, dY, lddy, dweights, nullptr,
                                               reinterpret_cast<cudaStream_t>(stream)));
}

size_t emu_rows_combine_workspace_bytes(int64_t yrows)
{
    return yrows < 0 ? 0 : (size_t)yrows * sizeof(int32_t);
}

emu_status emu_rows_combine_backward_full(int dtype, int64_t T, int64_t k, int64_t cols, const void *dO, int64_t lddo,
                                          const void *Y, int64_t yrows, int64_t ldy, const int32_t *slots,
                                          const float *weights, void *dY, int64_t lddy, float *dweights, void *ws,
                                          size_t ws_bytes, emu_stream_t stream)
{
    emu_status s = check_combine_backward(dtype, T, k, cols, dO, lddo, Y, yrows, ldy, slots, weights, dY, lddy, dweights);
    if (s != EMU_OK) return s;
    if (yrows > 0 && cols > 0) {
        if (!dY) return EMU_ERR_INVALID_ARG;              // (every row is written, also without tokens)
        if (!fits(dY, dtype)) return EMU_ERR_MISALIGNED;
        s = check_ws(ws, ws_bytes, emu_rows_combine_workspace_bytes(yrows));
        if (s != EMU_OK) return s;
    }
    return cuda_status(launch_combine_backward(dtype == EMU_F32, T, (int)k, cols, dO, lddo, Y, yrows, ldy, slots,
                                               weights, dY, lddy, dweights,
                                               yrows > 0 && cols > 0 ? static_cast<int32_t *>(ws) : nullptr,
                                               reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
