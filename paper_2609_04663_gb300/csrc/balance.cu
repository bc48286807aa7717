// Balance loss of the routing, its counts and its gradient.
//
// With n tokens that count, p_t the softmax of token t's logits over all E experts,
// counts_e the assignments to expert e and f_e = coef E counts_e / (n k):
//   loss = sum_e f_e P_e, P_e = 1/n sum_t p_te;
//   dl_te = dloss / n p_te (f_e - sum_e' f_e' p_te')
// (counts are constants in the gradient).  A group of L lanes (8, 16 or 32: as few as hold a
// row with V values each) has a token; lanes keep their experts' sums of p in FP32 over
// all their tokens, a block adds its warps' in a fixed order, and one block of a second
// launch adds the blocks' in a fixed order: no floating-point atomics, the same bits every
// time.  With few tokens the first launch is one block and does both.
#include "grouped_common.cuh"
#include "expert_launchers.cuh"
#include "split_f32_pair.cuh"

namespace emu {

namespace {

constexpr int kBalanceBlocks = 152;

struct BalanceArgs {
    const void *logits, *add;
    int64_t ldl, lda, ldd;
    const int32_t *experts;
    const uint8_t *mask;
    const float *dloss;
    void *dlogits;
    float *loss;
    int32_t *counts;              // [E + 1]: assignments of each expert, tokens that count
    float *sums;                  // [blocks][E] sums of p
    int32_t *parts;               // [blocks][E + 2]: counts, tokens, flags
    uint32_t *flags;
    float coef;
    int T, E, k, blocks;
};

// V values of a row for one of L lanes: consecutive ones (VEC: rows start on whole
// lanes, and E is a multiple of 4), or every L-th.  NaN and places past the end as minus
// infinity.
template <int V, int L, bool VEC>
__device__ __forceinline__ int expert_of(int lane, int i) { return VEC ? lane * V + i : i * L + lane; }

template <int V, int L, bool F32, bool VEC, bool KEPT = true>     // KEPT: nothing writes there during the launch
__device__ __forceinline__ void load_values(const void *base, int64_t at, int lane, int E, float (&x)[V], float none)
{
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const int e = lane * V + i;
            if (e < E) {
                if constexpr (F32) {
                    const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(base) + at + e);
                    const float4 v = KEPT ? __ldg(p) : *p;
                    x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
                } else {
                    const uint2 *p = reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(base) + at + e);
                    const uint2 v = KEPT ? __ldg(p) : *p;
                    x[i] = __uint_as_float(v.x << 16); x[i + 1] = __uint_as_float(v.x & 0xFFFF0000u);
                    x[i + 2] = __uint_as_float(v.y << 16); x[i + 3] = __uint_as_float(v.y & 0xFFFF0000u);
                }
            } else {
                x[i] = x[i + 1] = x[i + 2] = x[i + 3] = none;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = i * L + lane;
            x[i] = none;
            if (e >= E) continue;
            if constexpr (F32) {
                const float *p = static_cast<const float *>(base) + at + e;
                x[i] = KEPT ? __ldg(p) : *p;
            } else {
                const uint16_t *p = static_cast<const uint16_t *>(base) + at + e;
                x[i] = __uint_as_float((uint32_t)(KEPT ? __ldg(p) : *p) << 16);
            }
        }
    }
}

template <int L>
__device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}

// x: logits -> exp(x - max); returns 1 / their sum, or 0 where all are minus infinity.
template <int V, int L>
__device__ __forceinline__ float softmax_parts(float (&x)[V])
{
    float top = x[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, x[i]);
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    const bool some = top > -INFINITY;
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        x[i] = some ? expf(x[i] - top) : 0.0f;
        total += x[i];
    }
    total = lanes_sum<L>(total);
    return some ? 1.0f / total : 0.0f;
}

// coef E / (n k): what a count is multiplied by in f.
__device__ __forceinline__ float count_scale(const BalanceArgs &a, int n)
{
    return n > 0 ? a.coef * (float)a.E / ((float)n * (float)a.k) : 0.0f;
}

// One block: counts and the loss from the sums of `blocks` blocks.  sm: NT floats and
// NT ints at least.
template <int NT>
__device__ void finish(const BalanceArgs &a, const float *sums, const int32_t *parts, int blocks, float *sm)
{
    __shared__ float warp_part[NT / 32];
    __shared__ int n_all, bits;
    const int tid = threadIdx.x;
    if (tid == 0) { n_all = 0; bits = 0; }
    __syncthreads();
    for (int b = tid; b < blocks; b += NT) {
        const int32_t *p = parts + (int64_t)b * (a.E + 2) + a.E;
        atomicAdd(&n_all, p[0]);
        if (p[1]) atomicOr(&bits, p[1]);
    }
    __syncthreads();
    const int n = n_all;
    const float cs = count_scale(a, n), inv_n = n > 0 ? 1.0f / (float)n : 0.0f;
    // W columns at a time, `split` threads a column, each every split-th block
    int W = 32;
    while (W < a.E && W < NT) W *= 2;
    const int split = NT / W, col = tid % W, part = tid / W;
    int *si = reinterpret_cast<int *>(sm + NT);
    float loss = 0.0f;
    for (int e0 = 0; e0 < a.E; e0 += W) {
        const int e = e0 + col;
        float s = 0.0f;
        int c = 0;
        if (e < a.E) {
#pragma unroll 4
            for (int b = part; b < blocks; b += split) {
                s += sums[(int64_t)b * a.E + e];
                c += parts[(int64_t)b * (a.E + 2) + e];
            }
        }
        sm[tid] = s;
        si[tid] = c;
        __syncthreads();
        if (part == 0 && e < a.E) {
            for (int q = 1; q < split; ++q) { s += sm[q * W + col]; c += si[q * W + col]; }
            a.counts[e] = c;
            loss = fmaf((float)c * cs, s * inv_n, loss);
        }
        __syncthreads();
    }
    loss = lanes_sum<32>(loss);
    if (lane_id() == 0) warp_part[tid >> 5] = loss;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < NT / 32; ++w) loss += warp_part[w];
        *a.loss = loss;
        a.counts[a.E] = n;
        if (a.flags) *a.flags = (uint32_t)bits;
    }
}

template <int V, int L, bool F32, bool VEC, int NT>
__global__ void __launch_bounds__(NT) balance_kernel(const BalanceArgs a)
{
    extern __shared__ float sm[];                 // [warps][E] sums, then [E] counts
    constexpr int WARPS = NT / 32, PER = 32 / L;
    int *hist = reinterpret_cast<int *>(sm + (size_t)WARPS * a.E);
    __shared__ int tokens, bits;
    const int warp = threadIdx.x >> 5, lane = (int)lane_id() % L, sub = (int)lane_id() / L;
    if (threadIdx.x == 0) { tokens = 0; bits = 0; }
    for (int e = threadIdx.x; e < a.E; e += NT) hist[e] = 0;
    __syncthreads();
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    int n = 0, odd = 0;
    for (int64_t t0 = ((int64_t)blockIdx.x * WARPS + warp) * PER; t0 < a.T; t0 += (int64_t)gridDim.x * WARPS * PER) {
        const int64_t t = t0 + sub;
        const bool here = t < a.T;
        const bool on = here && (!a.mask || __ldg(a.mask + t) != 0);
        float x[V];
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = -INFINITY;
        if (on) load_values<V, L, F32, VEC>(a.logits, t * a.ldl, lane, a.E, x, -INFINITY);
        if (on) {
            for (int j = lane; j < a.k; j += L) {
                const int e = __ldg(a.experts + t * a.k + j);
                if (e >= 0 && e < a.E) atomicAdd(hist + e, 1);
                else odd |= EMU_FLAG_INDEX;
            }
            n += lane == 0;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!(x[i] < INFINITY)) odd |= EMU_FLAG_NONFINITE;
            x[i] = fmaxf(x[i], -INFINITY);                // NaN counts as minus infinity
        }
        const float inv = softmax_parts<V, L>(x);
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = fmaf(x[i], inv, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int d = 16; d >= L; d >>= 1) acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], d);
    if (sub == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = expert_of<V, L, VEC>(lane, i);
            if (e < a.E) sm[(size_t)warp * a.E + e] = acc[i];
        }
    }
    if (n) atomicAdd(&tokens, n);
    if (odd) atomicOr(&bits, odd);
    __syncthreads();
    float *sums = a.sums + (int64_t)blockIdx.x * a.E;
    int32_t *parts = a.parts + (int64_t)blockIdx.x * (a.E + 2);
    for (int e = threadIdx.x; e < a.E; e += NT) {
        float s = sm[e];
        for (int w = 1; w < WARPS; ++w) s += sm[(size_t)w * a.E + e];
        sums[e] = s;
        parts[e] = hist[e];
    }
    if (threadIdx.x == 0) { parts[a.E] = tokens; parts[a.E + 1] = bits; }
    if (gridDim.x == 1) {
        __syncthreads();                              // (global writes too: of this block alone)
        finish<NT>(a, a.sums, a.parts, 1, sm);
    }
}

__global__ void __launch_bounds__(1024) balance_finish_kernel(const BalanceArgs a)
{
    __shared__ float sm[2048];
    griddep_wait();
    finish<1024>(a, a.sums, a.parts, a.blocks, sm);
}

template <int V, int L, bool F32, bool VEC>
__global__ void __launch_bounds__(256) balance_backward_kernel(const BalanceArgs a)
{
    constexpr int PER = 32 / L;
    const int lane = (int)lane_id() % L, sub = (int)lane_id() / L;
    const int n = __ldg(a.counts + a.E);
    const float cs = count_scale(a, n);
    const float scale = n > 0 ? (a.dloss ? __ldg(a.dloss) : 1.0f) / (float)n : 0.0f;
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = expert_of<V, L, VEC>(lane, i);
        f[i] = e < a.E ? (float)__ldg(a.counts + e) * cs : 0.0f;
    }
    for (int64_t t0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * PER; t0 < a.T; t0 += (int64_t)gridDim.x * 8 * PER) {
        const int64_t t = t0 + sub;
        const bool here = t < a.T, on = here && (!a.mask || __ldg(a.mask + t) != 0);
        float x[V], d[V];
#pragma unroll
        for (int i = 0; i < V; ++i) { x[i] = -INFINITY; d[i] = 0.0f; }
        if (on) load_values<V, L, F32, VEC>(a.logits, t * a.ldl, lane, a.E, x, -INFINITY);
        // (dlogits may be `add`: each entry is read before the same lane writes it)
        if (here && a.add) load_values<V, L, F32, VEC, false>(a.add, t * a.lda, lane, a.E, d, 0.0f);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = fmaxf(x[i], -INFINITY);
        const float inv = softmax_parts<V, L>(x);
        float inner = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] *= inv;
            inner = fmaf(x[i], f[i], inner);
        }
        inner = lanes_sum<L>(inner);
        if (!here) continue;
        if (on) {
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] = fmaf(scale * x[i], f[i] - inner, d[i]);
        }
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const int e = lane * V + i;
                if (e >= a.E) continue;
                if constexpr (F32)
                    *reinterpret_cast<float4 *>(static_cast<float *>(a.dlogits) + t * a.ldd + e) = make_float4(d[i], d[i + 1], d[i + 2], d[i + 3]);
                else
                    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.dlogits) + t * a.ldd + e) =
                        make_uint2(bf16x2_rn(d[i], d[i + 1]), bf16x2_rn(d[i + 2], d[i + 3]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int e = i * L + lane;
                if (e >= a.E) continue;
                if constexpr (F32) static_cast<float *>(a.dlogits)[t * a.ldd + e] = d[i];
                else static_cast<uint16_t *>(a.dlogits)[t * a.ldd + e] = (uint16_t)bf16x2_rn(d[i], 0.0f);
            }
        }
    }
}

// Rows that lanes can read 4 values at a time.
bool whole_lanes(const void *p, int64_t ld, bool f32)
{
    return !p || ((reinterpret_cast<uintptr_t>(p) & (f32 ? 15u : 7u)) == 0 && ld % 4 == 0);
}

template <int V, int L, bool F32, bool VEC>
cudaError_t run_balance(BalanceArgs a, bool backward, cudaStream_t st)
{
    if (backward) {
        const int64_t blocks = ((int64_t)a.T + 8 * (32 / L) - 1) / (8 * (32 / L));
        balance_backward_kernel<V, L, F32, VEC><<<(unsigned)(blocks > 152 * 8 ? 152 * 8 : blocks), 256, 0, st>>>(a);
        return cudaGetLastError();
    }
    constexpr int NT = V >= 16 ? 512 : 1024, PASS = NT / L;
    const size_t need = ((size_t)(NT / 32) * a.E + a.E) * 4, least = (size_t)NT * 8;
    const size_t sm = need > least ? need : least;
    auto kern = balance_kernel<V, L, F32, VEC, NT>;
    if (sm > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sm);
        if (e != cudaSuccess) return e;
    }
    int64_t blocks = ((int64_t)a.T + PASS - 1) / PASS;
    if (blocks <= 4) blocks = 1;
    if (blocks > kBalanceBlocks) blocks = kBalanceBlocks;
    a.blocks = (int)blocks;
    kern<<<(unsigned)blocks, NT, sm, st>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || blocks == 1) return e;
    balance_finish_kernel<<<1, 1024, 0, st>>>(a);
    return cudaGetLastError();
}

template <bool F32, bool VEC>
cudaError_t by_experts(const BalanceArgs &a, bool backward, cudaStream_t st)
{
    if (a.E <= 32) return run_balance<4, 8, F32, VEC>(a, backward, st);
    if (a.E <= 64) return run_balance<4, 16, F32, VEC>(a, backward, st);
    if (a.E <= 128) return run_balance<4, 32, F32, VEC>(a, backward, st);
    if (a.E <= 256) return run_balance<8, 32, F32, VEC>(a, backward, st);
    if (a.E <= 512) return run_balance<16, 32, F32, VEC>(a, backward, st);
    return run_balance<32, 32, F32, VEC>(a, backward, st);
}

cudaError_t by_type(const BalanceArgs &a, bool f32, bool backward, cudaStream_t st)
{
    const bool vec = a.E % 4 == 0 && whole_lanes(a.logits, a.ldl, f32) &&
                     (!backward || (whole_lanes(a.add, a.lda, f32) && whole_lanes(a.dlogits, a.ldd, f32)));
    return f32 ? (vec ? by_experts<true, true>(a, backward, st) : by_experts<true, false>(a, backward, st))
               : (vec ? by_experts<false, true>(a, backward, st) : by_experts<false, false>(a, backward, st));
}

}  // namespace

size_t balance_scratch_bytes(int64_t E) { return (size_t)kBalanceBlocks * (size_t)(2 * E + 2) * 4; }

cudaError_t launch_balance(int64_t T, int64_t E, int k, const void *logits, bool f32, int64_t ldl, const int32_t *experts,
                           const uint8_t *mask, float coef, float *loss, int32_t *counts, void *scratch, uint32_t *flags,
                           cudaStream_t st)
{
    BalanceArgs a = {};
    a.logits = logits; a.ldl = ldl; a.experts = experts; a.mask = mask; a.coef = coef; a.loss = loss; a.counts = counts;
    a.T = (int)T; a.E = (int)E; a.k = k; a.flags = flags;
    a.sums = static_cast<float *>(scratch);
    a.parts = reinterpret_cast<int32_t *>(a.sums + (size_t)kBalanceBlocks * E);
    if (T == 0) a.experts = nullptr;
    return by_type(a, f32, false, st);
}

cudaError_t launch_balance_backward(int64_t T, int64_t E, int k, const void *logits, bool f32, int64_t ldl,
                                    const int32_t *counts, const uint8_t *mask, float coef, const float *dloss,
                                    const void *add, int64_t lda, void *dlogits, int64_t ldd, cudaStream_t st)
{
    BalanceArgs a = {};
    a.logits = logits; a.ldl = ldl; a.counts = const_cast<int32_t *>(counts); a.mask = mask; a.coef = coef;
    a.dloss = dloss; a.add = add; a.lda = lda; a.dlogits = dlogits; a.ldd = ldd; a.T = (int)T; a.E = (int)E; a.k = k;
    return by_type(a, f32, true, st);
}

}  // namespace emu
