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
// time.  With few tokens the first launch is one cluster, whose first block does that through shared
// memory.
//
// 32768 tokens of 128 experts in BF16, with gradient, take 18.3 us on the GPU (bytes: 3.9, what is read again comes from
// L2): three launches whose own latency and ends are most of their 4 to 8 us each.  64 tokens: 6.6.
#include "grouped_common.cuh"
#include "expert_launchers.cuh"
#include "pair_common.cuh"
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
    int32_t *counts;              // [E] assignments of each expert
    int32_t *tokens;              // tokens that count
    float *sums;                  // [blocks][E] sums of p
    int32_t *parts;               // [blocks][E + 2]: counts, tokens, flags
    uint32_t *flags;
    float coef;
    int T, E, k, blocks;
    int cluster;                  // the blocks are one cluster
};

// The expert of value i of a lane, of L lanes with V values each: C neighbouring ones at a
// time (one load: E and the row pitch are multiples of C then), the lanes side by side.
template <int L, int C>
__device__ __forceinline__ int expert_of(int lane, int i) { return i / C * (C * L) + lane * C + i % C; }

// A lane's values of a row, `none` past the last expert.  KEPT: nothing writes there during the launch.
template <int V, int L, bool F32, int C, bool KEPT = true>
__device__ __forceinline__ void load_values(const void *base, int64_t at, int lane, int E, float (&x)[V], float none)
{
#pragma unroll
    for (int i = 0; i < V; i += C) {
        const int e = expert_of<L, C>(lane, i);
#pragma unroll
        for (int j = 0; j < C; ++j) x[i + j] = none;
        if (e >= E) continue;
        if constexpr (F32) {
            const float *p = static_cast<const float *>(base) + at + e;
            if constexpr (C == 4) {
                const float4 *q = reinterpret_cast<const float4 *>(p);
                const float4 v = KEPT ? __ldg(q) : *q;
                x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
            } else {
                x[i] = KEPT ? __ldg(p) : *p;
            }
        } else {
            const uint16_t *p = static_cast<const uint16_t *>(base) + at + e;
            uint32_t w[4] = {};
            if constexpr (C == 8) {
                const uint4 *q = reinterpret_cast<const uint4 *>(p);
                const uint4 v = KEPT ? __ldg(q) : *q;
                w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            } else if constexpr (C == 4) {
                const uint2 *q = reinterpret_cast<const uint2 *>(p);
                const uint2 v = KEPT ? __ldg(q) : *q;
                w[0] = v.x; w[1] = v.y;
            } else {
                w[0] = KEPT ? __ldg(p) : *p;
            }
#pragma unroll
            for (int j = 0; j < C; ++j) x[i + j] = __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
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

// The larger one, NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}

// x: logits -> exp(x - max); returns 1 / their sum, or 0 where all are minus infinity.  NaN
// counts as minus infinity.  odd: set where a lane's value is NaN or plus infinity.
// As powers of two: x log2 e - c with one rounding, c = max log2 e rounded.  What c is off by is a
// factor that the whole row has and the sum takes out again, while it is
// small: below 2^(1/16) for |max| <= 2^20, 2^128 at worst from 2^31 on.  Larger ones are subtracted first, which is
// exact for values whose exponentials are not 0 (within 104 of the largest; always subtracting would put a
// second rounding into ordinary rows).  A power of two is off by 2^-22 at most.
template <int V, int L>
__device__ __forceinline__ float softmax_parts(float (&x)[V], bool &odd)
{
    float top = x[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = max_nan(top, x[i]);
    odd = !(top < INFINITY);
    if (odd) {
        top = -INFINITY;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] = fmaxf(x[i], -INFINITY);
            top = fmaxf(top, x[i]);
        }
    }
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    const bool some = top > -INFINITY;
    if (some && fabsf(top) > 0x1p20f) {               // (a row of a mask's -1e9, or of the type's lowest value)
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] -= top;
        top = 0.0f;
    }
    constexpr float log2e = 1.4426950408889634f;
    const float c = some ? top * log2e : 0.0f;
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(x[i]) : "f"(fmaf(x[i], log2e, -c)));
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

// Adds `rows` rows of E sums, all threads of a block: W columns at a time with NT / W threads
// a column, in an order that depends on the sizes alone.  at(row, e): a sum; done(e, sum): column e's, in
// one thread.
template <int NT, typename At, typename Done>
__device__ __forceinline__ void add_columns(int rows, int E, float *red, At at, Done done)
{
    int W = 32;
    while (W < E && W < NT) W *= 2;
    const int tid = (int)threadIdx.x, split = NT / W, col = tid % W, part = tid / W;
    for (int e0 = 0; e0 < E; e0 += W) {
        const int e = e0 + col;
        float s = 0.0f;
        if (e < E) {
#pragma unroll 8
            for (int r = part; r < rows; r += split) s += at(r, e);
        }
        if (split > 1) {
            red[tid] = s;
            __syncthreads();
            if (part == 0)
                for (int q = 1; q < split; ++q) s += red[q * W + col];
        }
        if (part == 0 && e < E) done(e, s);
        if (split > 1) __syncthreads();
    }
}

// The loss from every thread's share of it, and what else there is to say; a whole block.
template <int NT>
__device__ __forceinline__ void publish(const BalanceArgs &a, float share, int n, uint32_t bits, float *red)
{
    share = lanes_sum<32>(share);
    __syncthreads();
    if (lane_id() == 0) red[threadIdx.x >> 5] = share;
    __syncthreads();
    if (threadIdx.x < 32) {
        share = lanes_sum<32>(threadIdx.x < NT / 32 ? red[threadIdx.x] : 0.0f);
        if (threadIdx.x == 0) {
            *a.loss = share;
            *a.tokens = n;
            if (a.flags) *a.flags = bits;
        }
    }
}

template <int V, int L, bool F32, int C, int NT>
__global__ void __launch_bounds__(NT) balance_kernel(const BalanceArgs a)
{
    extern __shared__ float sm[];                 // [warps][E] sums, [E] counts
    constexpr int WARPS = NT / 32, PER = 32 / L;
    int *hist = reinterpret_cast<int *>(sm + (size_t)WARPS * a.E);
    __shared__ float red[NT];
    __shared__ int tokens, bits;
    griddep_launch_dependents();
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
        if (on) load_values<V, L, F32, C>(a.logits, t * a.ldl, lane, a.E, x, -INFINITY);
        if (on) {
            for (int j = lane; j < a.k; j += L) {
                const int e = __ldg(a.experts + t * a.k + j);
                if (e >= 0 && e < a.E) atomicAdd(hist + e, 1);
                else odd |= EMU_FLAG_INDEX;
            }
            n += lane == 0;
        }
        bool bad;
        const float inv = softmax_parts<V, L>(x, bad);
        if (bad) odd |= EMU_FLAG_NONFINITE;
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
            const int e = expert_of<L, C>(lane, i);
            if (e < a.E) sm[(size_t)warp * a.E + e] = acc[i];
        }
    }
    n = __reduce_add_sync(0xFFFFFFFFu, n);
    odd = (int)__reduce_or_sync(0xFFFFFFFFu, (unsigned)odd);
    if (lane_id() == 0) {
        if (n) atomicAdd(&tokens, n);
        if (odd) atomicOr(&bits, odd);
    }
    __syncthreads();
    const int all = tokens;
    auto at = [&](int w, int e) { return sm[(size_t)w * a.E + e]; };
    if (a.cluster) {
        // the block's sums end up in its first warp's row
        add_columns<NT>(WARPS, a.E, red, at, [&](int e, float s) { sm[e] = s; });
        if (a.blocks > 1) cluster_sync();
        else __syncthreads();
        if (blockIdx.x == 0) {
            auto other = [&](const void *p, int r) {
                uint32_t v;
                asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(peer_addr(smem_u32(p), (uint32_t)r)) : "memory");
                return v;
            };
            int n_all = 0;
            uint32_t some = 0;
            for (int r = 0; r < a.blocks; ++r) { n_all += (int)other(&tokens, r); some |= other(&bits, r); }
            const float cs = count_scale(a, n_all), inv_n = n_all > 0 ? 1.0f / (float)n_all : 0.0f;
            float loss = 0.0f;
            for (int e = threadIdx.x; e < a.E; e += NT) {
                float s = 0.0f;
                int c = 0;
                for (int r = 0; r < a.blocks; ++r) {
                    s += __uint_as_float(other(sm + e, r));
                    c += (int)other(hist + e, r);
                }
                a.counts[e] = c;
                loss = fmaf((float)c * cs, s * inv_n, loss);
            }
            publish<NT>(a, loss, n_all, some, red);
        }
        if (a.blocks > 1) cluster_sync();             // shared memory stays until it has been read
    } else {
        float *sums = a.sums + (int64_t)blockIdx.x * a.E;
        int32_t *parts = a.parts + (int64_t)blockIdx.x * (a.E + 2);
        add_columns<NT>(WARPS, a.E, red, at, [&](int e, float s) {
            sums[e] = s;
            parts[e] = hist[e];
        });
        if (threadIdx.x == 0) { parts[a.E] = all; parts[a.E + 1] = bits; }
    }
}

// The second launch: a cluster of 8 CTAs, each with an eighth of the experts; the first one adds
// their shares of the loss, through shared memory, in order.
constexpr int kFinishCtas = 8;
__global__ void __cluster_dims__(kFinishCtas, 1, 1) __launch_bounds__(512) balance_finish_kernel(const BalanceArgs a)
{
    constexpr int NT = 512;
    __shared__ float red[NT], share;
    __shared__ int redc[NT], tokens, bits;
    const int tid = (int)threadIdx.x, rank = (int)cluster_rank();
    if (tid == 0) { tokens = 0; bits = 0; }
    __syncthreads();
    griddep_wait();
    if (tid < a.blocks) {
        const int32_t *p = a.parts + (int64_t)tid * (a.E + 2) + a.E;
        if (p[0]) atomicAdd(&tokens, p[0]);
        if (p[1]) atomicOr(&bits, p[1]);
    }
    static_assert(kBalanceBlocks <= NT, "a thread a block");
    const int each = (a.E + kFinishCtas - 1) / kFinishCtas, e0 = rank * each;      // at most 128
    int W = 16;
    while (W < each) W *= 2;
    const int split = NT / W, col = tid % W, part = tid / W, e = e0 + col;
    const bool mine = col < each && e < a.E;
    float s = 0.0f;
    int c = 0;
    if (mine) {
#pragma unroll 8
        for (int b = part; b < a.blocks; b += split) {
            s += a.sums[(int64_t)b * a.E + e];
            c += a.parts[(int64_t)b * (a.E + 2) + e];
        }
    }
    red[tid] = s;
    redc[tid] = c;
    __syncthreads();
    const int n = tokens;
    const float cs = count_scale(a, n), inv_n = n > 0 ? 1.0f / (float)n : 0.0f;
    float loss = 0.0f;
    if (part == 0 && mine) {
        for (int q = 1; q < split; ++q) { s += red[q * W + col]; c += redc[q * W + col]; }
        a.counts[e] = c;
        loss = (float)c * cs * (s * inv_n);
    }
    loss = lanes_sum<32>(loss);
    __syncthreads();
    if (lane_id() == 0) red[tid >> 5] = loss;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < NT / 32; ++w) loss += red[w];
        share = loss;
    }
    cluster_sync();
    if (rank == 0 && tid == 0) {
        float v[kFinishCtas];
#pragma unroll
        for (int r = 0; r < kFinishCtas; ++r)
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[r]) : "r"(peer_addr(smem_u32(&share), (uint32_t)r)) : "memory");
        loss = v[0];
#pragma unroll
        for (int r = 1; r < kFinishCtas; ++r) loss += v[r];
        *a.loss = loss;
        *a.tokens = n;
        if (a.flags) *a.flags = (uint32_t)bits;
    }
    cluster_sync();                                   // shared memory stays until it has been read
}

template <int V, int L, bool F32, int C>
__global__ void __launch_bounds__(256) balance_backward_kernel(const BalanceArgs a)
{
    constexpr int PER = 32 / L;
    const int lane = (int)lane_id() % L, sub = (int)lane_id() / L;
    const int n = __ldg(a.tokens);
    const float cs = count_scale(a, n);
    const float scale = n > 0 ? (a.dloss ? __ldg(a.dloss) : 1.0f) / (float)n : 0.0f;
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = expert_of<L, C>(lane, i);
        f[i] = e < a.E ? (float)__ldg(a.counts + e) * cs : 0.0f;
    }
    for (int64_t t0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * PER; t0 < a.T; t0 += (int64_t)gridDim.x * 8 * PER) {
        const int64_t t = t0 + sub;
        const bool here = t < a.T, on = here && (!a.mask || __ldg(a.mask + t) != 0);
        float x[V], d[V];
#pragma unroll
        for (int i = 0; i < V; ++i) { x[i] = -INFINITY; d[i] = 0.0f; }
        if (on) load_values<V, L, F32, C>(a.logits, t * a.ldl, lane, a.E, x, -INFINITY);
        // (dlogits may be `add`: each entry is read before the same lane writes it)
        if (here && a.add) load_values<V, L, F32, C, false>(a.add, t * a.lda, lane, a.E, d, 0.0f);
        bool bad;
        const float inv = softmax_parts<V, L>(x, bad);
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
#pragma unroll
        for (int i = 0; i < V; i += C) {
            const int e = expert_of<L, C>(lane, i);
            if (e >= a.E) continue;
            if constexpr (F32) {
                float *o = static_cast<float *>(a.dlogits) + t * a.ldd + e;
                if constexpr (C == 4) *reinterpret_cast<float4 *>(o) = make_float4(d[i], d[i + 1], d[i + 2], d[i + 3]);
                else *o = d[i];
            } else {
                uint16_t *o = static_cast<uint16_t *>(a.dlogits) + t * a.ldd + e;
                if constexpr (C == 8)
                    *reinterpret_cast<uint4 *>(o) = make_uint4(bf16x2_rn(d[i], d[i + 1]), bf16x2_rn(d[i + 2], d[i + 3]),
                                                               bf16x2_rn(d[i + 4], d[i + 5]), bf16x2_rn(d[i + 6], d[i + 7]));
                else if constexpr (C == 4)
                    *reinterpret_cast<uint2 *>(o) = make_uint2(bf16x2_rn(d[i], d[i + 1]), bf16x2_rn(d[i + 2], d[i + 3]));
                else
                    *o = (uint16_t)bf16x2_rn(d[i], 0.0f);
            }
        }
    }
}

// Lanes a token.
int lanes_of(int E) { return E <= 128 ? 8 : E <= 256 ? 16 : 32; }

// Few tokens: at most four passes over them by a cluster of 8.
bool one_cluster(int64_t T, int64_t E) { return T * lanes_of((int)E) <= 4 * 8 * (E > 512 ? 512 : 1024); }

// Whether rows can be read C values at a time.
bool whole_lanes(const void *p, int64_t ld, int bytes, int C)
{
    return !p || ((reinterpret_cast<uintptr_t>(p) & (unsigned)(bytes * C - 1)) == 0 && ld % C == 0);
}

template <int V, int L, bool F32, int C>
cudaError_t run_balance(BalanceArgs a, bool backward, cudaStream_t st)
{
    if (backward) {
        const int64_t blocks = ((int64_t)a.T + 8 * (32 / L) - 1) / (8 * (32 / L));
        balance_backward_kernel<V, L, F32, C><<<(unsigned)(blocks > 152 * 8 ? 152 * 8 : blocks), 256, 0, st>>>(a);
        return cudaGetLastError();
    }
    constexpr int NT = V >= 32 ? 512 : 1024, PASS = NT / L;      // (as one_cluster has it)
    const size_t sm = ((size_t)(NT / 32) * a.E + a.E) * 4;
    auto kern = balance_kernel<V, L, F32, C, NT>;
    if (sm > 44 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sm);
        if (e != cudaSuccess) return e;
    }
    const int64_t passes = ((int64_t)a.T + PASS - 1) / PASS;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = sm;
    cfg.stream = st;
    cfg.attrs = &attr;
    a.cluster = one_cluster(a.T, a.E) ? 1 : 0;
    a.blocks = passes > kBalanceBlocks ? kBalanceBlocks : (int)passes;
    if (a.cluster) a.blocks = passes <= 1 ? 1 : passes <= 2 ? 2 : passes <= 4 ? 4 : 8;
    cfg.gridDim = dim3((unsigned)a.blocks);
    if (a.cluster && a.blocks > 1) {
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)a.blocks;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.numAttrs = 1;
    }
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, a);
    if (e != cudaSuccess || a.cluster) return e != cudaSuccess ? e : cudaGetLastError();
    cfg.gridDim = dim3(kFinishCtas);
    cfg.blockDim = dim3(512);
    cfg.dynamicSmemBytes = 0;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, balance_finish_kernel, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

// Rows read in pieces of 16 bytes (8 for the fewest experts in BF16), or value by value.
template <int V, int L, bool F32>
cudaError_t by_pieces(const BalanceArgs &a, bool backward, cudaStream_t st)
{
    constexpr int C = F32 || V < 8 ? 4 : 8, bytes = F32 ? 4 : 2;
    const bool whole = a.E % C == 0 && whole_lanes(a.logits, a.ldl, bytes, C) &&
                       (!backward || (whole_lanes(a.add, a.lda, bytes, C) && whole_lanes(a.dlogits, a.ldd, bytes, C)));
    return whole ? run_balance<V, L, F32, C>(a, backward, st) : run_balance<V, L, F32, 1>(a, backward, st);
}

template <bool F32>
cudaError_t by_experts(const BalanceArgs &a, bool backward, cudaStream_t st)
{
    return a.E <= 32 ? by_pieces<4, 8, F32>(a, backward, st) : a.E <= 64 ? by_pieces<8, 8, F32>(a, backward, st)
           : a.E <= 128 ? by_pieces<16, 8, F32>(a, backward, st) : a.E <= 256 ? by_pieces<16, 16, F32>(a, backward, st)
           : a.E <= 512 ? by_pieces<16, 32, F32>(a, backward, st) : by_pieces<32, 32, F32>(a, backward, st);
}

cudaError_t by_type(const BalanceArgs &a, bool f32, bool backward, cudaStream_t st)
{
    return f32 ? by_experts<true>(a, backward, st) : by_experts<false>(a, backward, st);
}

}  // namespace

size_t balance_scratch_bytes(int64_t T, int64_t E)
{
    return one_cluster(T, E) ? 0 : (size_t)kBalanceBlocks * (size_t)(2 * E + 2) * 4;
}

cudaError_t launch_balance(int64_t T, int64_t E, int k, const void *logits, bool f32, int64_t ldl, const int32_t *experts,
                           const uint8_t *mask, float coef, float *loss, int32_t *counts, int32_t *tokens, void *scratch, uint32_t *flags,
                           cudaStream_t st)
{
    BalanceArgs a = {};
    a.logits = logits; a.ldl = ldl; a.experts = experts; a.mask = mask; a.coef = coef; a.loss = loss; a.counts = counts; a.tokens = tokens;
    a.T = (int)T; a.E = (int)E; a.k = k; a.flags = flags;
    a.sums = static_cast<float *>(scratch);
    a.parts = reinterpret_cast<int32_t *>(a.sums + (size_t)kBalanceBlocks * E);
    if (T == 0) a.experts = nullptr;
    return by_type(a, f32, false, st);
}

cudaError_t launch_balance_backward(int64_t T, int64_t E, int k, const void *logits, bool f32, int64_t ldl,
                                    const int32_t *counts, const int32_t *tokens, const uint8_t *mask, float coef, const float *dloss,
                                    const void *add, int64_t lda, void *dlogits, int64_t ldd, cudaStream_t st)
{
    BalanceArgs a = {};
    a.logits = logits; a.ldl = ldl; a.counts = const_cast<int32_t *>(counts);
    a.tokens = const_cast<int32_t *>(tokens); a.mask = mask; a.coef = coef;
    a.dloss = dloss; a.add = add; a.lda = lda; a.dlogits = dlogits; a.ldd = ldd; a.T = (int)T; a.E = (int)E; a.k = k;
    return by_type(a, f32, true, st);
}

}  // namespace emu
