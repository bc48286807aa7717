// Routing of tokens to experts, its gradient, and the weighted sum of the
// experts' answers with its gradients.
//
// route: for each token the k largest logits (ties: the lower index), their
// softmax weights, and the stable order of all T k assignments by expert: a
// counting sort.  One launch: every block ranks a contiguous range of tokens and
// every warp one within it (a token at a time: the largest key by a warp maximum,
// its lowest index, k times), each warp counts its own choices per expert, and
// after one grid barrier it places them behind those of the blocks and warps
// before it.  A single block needs no barrier.  Bound by instructions (sorting a
// lane's keys, k warp maxima) and by the barrier's and counts' latency:
// 32768 x 128 BF16, k = 8: 21 us, of which ranking 11, barrier and counts 4
// (the logits' bytes alone: 1.2); 8 x 64: 3.7 us; the gradient at 32768 x 128:
// 11 us.
//
// combine: bound by HBM; every answer row is read once, rows in 16-byte pieces.
// 16384 tokens, k = 4, 2048 BF16 columns: 54 us (6.2 TB/s), gradients 86 us (7.0
// TB/s with what L2 keeps), looking for rows without a slot 3 us.
#include "grouped_common.cuh"
#include "expert_launchers.cuh"
#include "split_f32_pair.cuh"

namespace emu {

namespace {

constexpr int kRouteThreads = 1024, kRouteWarps = kRouteThreads / 32, kRouteBlocks = 152;

__device__ __forceinline__ float bf16_f32(uint32_t b) { return __uint_as_float(b << 16); }
__device__ __forceinline__ uint16_t f32_bf16(float x) { return (uint16_t)bf16x2_rn(x, 0.0f); }

__device__ __forceinline__ float load_logit(const void *row, int e, bool f32)
{
    return f32 ? __ldg(static_cast<const float *>(row) + e) : bf16_f32(__ldg(static_cast<const uint16_t *>(row) + e));
}

// Order-preserving key of a logit that is not NaN, never 0; negative zero like
// zero.
__device__ __forceinline__ uint32_t logit_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k)
{
    return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}

struct RouteArgs {
    const void *logits;
    int64_t ldl;
    int T, E, k, f32, renorm;
    float *weights;
    int32_t *experts, *slots, *rows, *ends;
    int32_t *counts;                      // [blocks][count_pitch(E)]
    uint32_t *flags, *bar;
    uint32_t arrivals;                    // blocks that the barrier waits for
    unsigned long long limit_ns;          // and how long at most
};

// Row pitch of the blocks' counts: whole 16-byte pieces.
__host__ __device__ __forceinline__ int count_pitch(int E) { return (E + 3) & ~3; }

// Bounded barrier over the blocks of a cooperative launch (one use per launch;
// *bar starts at zero).  False, in every thread of the block, when the wait was
// given up: other blocks' counts may be missing then, and the block has to end.
__device__ __forceinline__ bool route_barrier(const RouteArgs &a)
{
    __syncthreads();
    bool late = false;
    if (threadIdx.x == 0) {
        __threadfence();
        atomicAdd(a.bar, 1u);
        volatile uint32_t *seen = a.bar;
        const unsigned long long t0 = globaltimer_ns();
        for (uint32_t it = 0; *seen < a.arrivals; ++it) {
            if (it >= (1u << 30) || ((it & 63u) == 63u && globaltimer_ns() - t0 > a.limit_ns)) {
                atomicOr(a.flags, (uint32_t)EMU_FLAG_TIMEOUT);
                late = true;
                break;
            }
        }
        __threadfence();
    }
    return __syncthreads_or(late ? 1 : 0) == 0;
}

// V: logits per lane (E <= 32 V).
template <int V, bool F32>
__global__ void __launch_bounds__(kRouteThreads) route_kernel(const RouteArgs a)
{
    extern __shared__ int32_t sm[];
    int32_t *hist = sm;                                   // [kRouteWarps][E]
    int32_t *base = sm + kRouteWarps * a.E;               // [E] first slot of this block's assignments
    int32_t *all = base + a.E;                            // [E] assignments of all blocks
    const int warp = threadIdx.x >> 5, lane = (int)lane_id();
    const int per = (a.T + (int)gridDim.x - 1) / (int)gridDim.x;
    const int t0 = min(a.T, (int)blockIdx.x * per), n = min(a.T, t0 + per) - t0;
    // this warp's tokens: a contiguous range, so that it can count and place its
    // own choices, in order (a token's experts are distinct: lanes never collide)
    const int wper = (n + kRouteWarps - 1) / kRouteWarps;
    const int w0 = t0 + min(n, warp * wper), w1 = t0 + min(n, (warp + 1) * wper);
    int32_t *h = hist + warp * a.E;
    for (int e = lane; e < a.E; e += 32) h[e] = 0;
    __syncwarp();

    // ---- the k largest of each token
    bool odd = false;
    const int64_t pitch = a.ldl * (F32 ? 4 : 2);
    const char *row = static_cast<const char *>(a.logits) + w0 * pitch;
    int64_t out = (int64_t)w0 * a.k + lane;
    for (int t = w0; t < w1; ++t, row += pitch, out += a.k) {
        uint32_t key[V];
        float x[V];
        int at[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = i * 32 + lane;
            x[i] = e < a.E ? load_logit(row, e, F32) : -INFINITY;
        }
        // lanes past the last expert hold minus infinity under higher indexes than
        // every expert's: with k <= E they are never taken
#pragma unroll
        for (int i = 0; i < V; ++i) {
            at[i] = i * 32 + lane;
            odd |= !(x[i] < INFINITY);                    // NaN or plus infinity
            x[i] = fmaxf(x[i], -INFINITY);                // NaN counts as minus infinity
            key[i] = logit_key(x[i]);
            // a BF16 logit's key fills the upper half: with the inverted index below
            // it the largest word is the largest logit of the lowest index
            if (!F32) key[i] = (key[i] & 0xFFFF0000u) | (0xFFFFu - (uint32_t)at[i]);
        }
        // up to 8 logits a lane: its candidates by falling key (equal keys: rising
        // index), the best of all lanes' firsts taken off k times; more: each lane
        // looks for its best again every time
        constexpr bool SORT = V <= 8;
        if constexpr (SORT) {
#pragma unroll
            for (int i = 1; i < V; ++i)
#pragma unroll
                for (int q = V - 1; q >= i; --q) {
                    const bool swap = key[q] > key[q - 1];
                    const uint32_t hi = max(key[q], key[q - 1]), lo = min(key[q], key[q - 1]);
                    const int u = at[q], v = at[q - 1];
                    key[q - 1] = hi; key[q] = lo;
                    if (F32) { at[q - 1] = swap ? u : v; at[q] = swap ? v : u; }
                }
        }
        // the padding below a BF16 key is its logit's lower half: zeros, or ones where negative
        auto logit = [&](uint32_t k) { return key_logit(F32 ? k : (k & 0x80000000u) ? k & 0xFFFF0000u : k | 0xFFFFu); };
        float total = 0.0f;
        if (!a.renorm) {                                  // the softmax over all, while the logits are at hand
            uint32_t best = key[0];
            if constexpr (!SORT) {
#pragma unroll
                for (int i = 1; i < V; ++i) best = max(best, key[i]);
            }
            const float top = logit(__reduce_max_sync(0xFFFFFFFFu, best));
            if (top > -INFINITY) {
#pragma unroll
                for (int i = 0; i < V; ++i) total += expf(x[i] - top);
            }
        }
        uint32_t mine = 0u;                               // lane j: the j-th key
        int chosen = 0;
#pragma unroll (SORT ? 4 : 1)                         // (E = 1024: 31 us against 33 unrolled)
        for (int j = 0; j < a.k; ++j) {
            uint32_t best = key[0];
            int first = at[0];
            if constexpr (!SORT) {
#pragma unroll
                for (int i = 1; i < V; ++i)
                    if (key[i] > best) { best = key[i]; first = i * 32 + lane; }
            }
            const uint32_t most = __reduce_max_sync(0xFFFFFFFFu, best);
            bool own = best == most;
            int e = 0;
            if constexpr (F32) {
                const uint32_t hit = __ballot_sync(0xFFFFFFFFu, own);
                if ((hit & (hit - 1)) == 0) e = __shfl_sync(0xFFFFFFFFu, first, __ffs(hit) - 1);
                else e = (int)__reduce_min_sync(0xFFFFFFFFu, own ? (uint32_t)first : 0x7FFFFFFFu);
                own = own && first == e;
                chosen = lane == j ? e : chosen;
            }
            if constexpr (SORT) {
#pragma unroll
                for (int i = 1; i < V; ++i) {
                    key[i - 1] = own ? key[i] : key[i - 1];
                    if (F32) at[i - 1] = own ? at[i] : at[i - 1];
                }
                key[V - 1] = own ? 0u : key[V - 1];
            } else {
                if (!F32) e = 0xFFFF - (int)(most & 0xFFFFu);
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i * 32 + lane == e) key[i] = 0u;
            }
            mine = lane == j ? most : mine;
        }
        if (!F32) chosen = 0xFFFF - (int)(mine & 0xFFFFu);
        const float own_logit = logit(mine), top = __shfl_sync(0xFFFFFFFFu, own_logit, 0);
        const bool some = top > -INFINITY;                // else no expert is allowed: weights 0
        const float p = some && lane < a.k ? expf(own_logit - top) : 0.0f;
        total = warp_sum(a.renorm ? p : total);
        if (lane < a.k) {
            a.weights[out] = some ? p / total : 0.0f;
            a.experts[out] = chosen;
            ++h[chosen];
        }
        __syncwarp();
    }
    if (gridDim.x == 1) {                                 // the only block: it sets the flag word
        if (__syncthreads_or(odd ? 1 : 0)) {
            if (threadIdx.x == 0) *a.flags = (uint32_t)EMU_FLAG_NONFINITE;
        } else if (threadIdx.x == 0) {
            *a.flags = 0u;
        }
    } else {
        if (__any_sync(0xFFFFFFFFu, odd) && lane == 0) atomicOr(a.flags, (uint32_t)EMU_FLAG_NONFINITE);
        __syncthreads();
    }

    // ---- each warp's count per expert -> the counts of the warps before it
    for (int e = threadIdx.x; e < a.E; e += kRouteThreads) {
        int sum = 0;
#pragma unroll 8
        for (int w = 0; w < kRouteWarps; ++w) {
            const int c = hist[w * a.E + e];
            hist[w * a.E + e] = sum;
            sum += c;
        }
        all[e] = gridDim.x > 1 ? 0 : sum;
        base[e] = 0;
        if (gridDim.x > 1) a.counts[(int64_t)blockIdx.x * count_pitch(a.E) + e] = sum;
    }
    if (gridDim.x > 1) {
        if (!route_barrier(a)) return;                    // slots, rows and ends stay as they were
        // parts of the threads sum up every parts-th block's counts, four experts a thread
        const int quads = (a.E + 3) / 4, parts = max(1, kRouteThreads / quads);
        const int part = (int)threadIdx.x / quads, q = (int)threadIdx.x - part * quads;
        if (part < parts) {
            int4 before = make_int4(0, 0, 0, 0), sum = before;
            const int4 *from = reinterpret_cast<const int4 *>(a.counts) + q;
#pragma unroll 8
            for (int b = part; b < (int)gridDim.x; b += parts) {
                const int4 c = __ldcg(from + (int64_t)b * quads);
                sum.x += c.x; sum.y += c.y; sum.z += c.z; sum.w += c.w;
                if (b < (int)blockIdx.x) { before.x += c.x; before.y += c.y; before.z += c.z; before.w += c.w; }
            }
            const int s[4] = {sum.x, sum.y, sum.z, sum.w}, f[4] = {before.x, before.y, before.z, before.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)                   // (integers: the order does not matter)
                if (q * 4 + i < a.E) {
                    atomicAdd(all + q * 4 + i, s[i]);
                    atomicAdd(base + q * 4 + i, f[i]);
                }
        }
    }
    __syncthreads();
    // ---- experts' first slots: thread e has expert e
    {
        __shared__ int32_t warps[kRouteWarps];
        const int e = (int)threadIdx.x, c = e < a.E ? all[e] : 0;
        int v = c;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(0xFFFFFFFFu, v, d);
            if (lane >= d) v += u;
        }
        if (lane == 31) warps[warp] = v;
        __syncthreads();
        const int earlier = (int)__reduce_add_sync(0xFFFFFFFFu, lane < warp ? warps[lane] : 0);
        if (e < a.E) {
            base[e] += earlier + v - c;
            if (blockIdx.x == 0) a.ends[e] = earlier + v;
        }
    }
    __syncthreads();

    // ---- slots: behind the same expert's assignments of earlier blocks, warps and
    // tokens.  Every lane reads back what it wrote.
    out = (int64_t)w0 * a.k + lane;
    const uint32_t total = (uint32_t)a.T * (uint32_t)a.k;
    for (int t = w0; t < w1; t += 4) {
        int e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = lane < a.k && t + i < w1 ? a.experts[out + i * a.k] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (e[i] >= 0) {
                const int before = h[e[i]], slot = base[e[i]] + before;
                h[e[i]] = before + 1;
                a.slots[out + i * a.k] = slot;
                // (a workspace that another call overwrites meanwhile must not lead out of rows)
                if ((uint32_t)slot < total) a.rows[slot] = t + i;
            }
            __syncwarp();
        }
        out += 4 * a.k;
    }
}

struct RouteBackArgs {
    const void *logits;
    int64_t ldl;
    const int32_t *experts;
    const float *dw;
    void *dl;
    int64_t lddl;
    int T, E, k, f32, renorm;
};

// V consecutive values of a row from V * lane on, as floats; NaN as minus
// infinity, past the end too.  VEC: rows allow one load per lane.
template <int V, bool VEC>
__device__ __forceinline__ void load_row(const char *row, int lane, int E, bool f32, float (&x)[V])
{
    if (VEC && lane * V < E) {
        if (f32) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const float4 v = __ldg(reinterpret_cast<const float4 *>(row) + (lane * V + i) / 4);
                x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const uint2 v = __ldg(reinterpret_cast<const uint2 *>(row) + (lane * V + i) / 4);
                x[i] = __uint_as_float(v.x << 16); x[i + 1] = __uint_as_float(v.x & 0xFFFF0000u);
                x[i + 2] = __uint_as_float(v.y << 16); x[i + 3] = __uint_as_float(v.y & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = !VEC && lane * V + i < E ? load_logit(row, lane * V + i, f32) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = x[i] == x[i] ? x[i] : -INFINITY;
}

// One warp per token.  With p the probabilities that the weights came from
// (over the chosen experts, or over all) and g the weights' gradients:
// dl_e = p_e ([e chosen] g_e - sum over the chosen of p g).  Lane j has the
// j-th chosen expert and writes its entry over the row's other formula, which
// the lanes have stored before.
template <int V, bool VEC>
__global__ void __launch_bounds__(256) route_backward_kernel(const RouteBackArgs a)
{
    const int lane = (int)lane_id();
    const int es = a.f32 ? 4 : 2;
    for (int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); t < a.T; t += (int64_t)gridDim.x * 8) {
        const char *row = static_cast<const char *>(a.logits) + t * a.ldl * es;
        char *out = static_cast<char *>(a.dl) + t * a.lddl * es;
        int e = lane < a.k ? __ldg(a.experts + t * a.k + lane) : -1;
        const float gw = lane < a.k ? __ldg(a.dw + t * a.k + lane) : 0.0f;
        float x[V];
        if (!a.renorm) load_row<V, VEC>(row, lane, a.E, a.f32 != 0, x);
        if (e >= a.E) e = -1;
        const float g = e >= 0 ? gw : 0.0f;
        float mine = e >= 0 ? load_logit(row, e, a.f32 != 0) : -INFINITY;
        mine = mine == mine ? mine : -INFINITY;
        float top = mine;
        if (!a.renorm) {
#pragma unroll
            for (int i = 0; i < V; ++i) top = fmaxf(top, x[i]);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        const bool some = top > -INFINITY;            // else no expert is allowed: gradients 0
        float p = some ? expf(mine - top) : 0.0f, total = p;
        if (!a.renorm) {
            total = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[i] = some ? expf(x[i] - top) : 0.0f;
                total += x[i];
            }
        }
        total = warp_sum(total);
        const float inv = some ? 1.0f / total : 0.0f;
        p *= inv;
        const float inner = warp_sum(p * g), scale = a.renorm ? 0.0f : -inner * inv;
        float d[V];
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] = a.renorm ? 0.0f : x[i] * scale;
        if (VEC) {
            if (lane * V < a.E) {
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    if (a.f32)
                        reinterpret_cast<float4 *>(out)[(lane * V + i) / 4] = make_float4(d[i], d[i + 1], d[i + 2], d[i + 3]);
                    else
                        reinterpret_cast<uint2 *>(out)[(lane * V + i) / 4] = make_uint2(bf16x2_rn(d[i], d[i + 1]), bf16x2_rn(d[i + 2], d[i + 3]));
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (lane * V + i < a.E) {
                    if (a.f32) reinterpret_cast<float *>(out)[lane * V + i] = d[i];
                    else reinterpret_cast<uint16_t *>(out)[lane * V + i] = f32_bf16(d[i]);
                }
        }
        __syncwarp();
        if (e >= 0) {
            const float s = p * (g - inner);
            if (a.f32) reinterpret_cast<float *>(out)[e] = s;
            else reinterpret_cast<uint16_t *>(out)[e] = f32_bf16(s);
        }
    }
}

// ------------------------------------------------------------------ combine
struct CombineArgs {
    const void *Y, *dO;
    int64_t yrows, ldy, ldo, lddy;
    const int32_t *slots;
    const float *weights;
    void *O, *dY;
    float *dw;
    int32_t *owner;           // [yrows], or NULL: the assignment t k + j whose slot names the row
    int64_t T;
    int k, cols;
};

// 16 bytes of a row: 4 FP32 or 8 BF16.  VEC (rows are 16-byte aligned and whole
// pieces): from column c on at once.  Else one by one, columns c, c + STEP, ..;
// columns past the last read as zero and are not stored (c is in the row).
template <bool F32, bool VEC, int STEP>
__device__ __forceinline__ uint4 load_piece(const char *row, int64_t c, int cols)
{
    if constexpr (VEC) {
        return __ldg(reinterpret_cast<const uint4 *>(row + c * (F32 ? 4 : 2)));
    } else if constexpr (F32) {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(row) + c;
        return make_uint4(__ldg(p), c + STEP < cols ? __ldg(p + STEP) : 0u, c + 2 * STEP < cols ? __ldg(p + 2 * STEP) : 0u,
                          c + 3 * STEP < cols ? __ldg(p + 3 * STEP) : 0u);
    } else {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + c;
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = i == 0 || c + STEP * i < cols ? (uint32_t)__ldg(p + STEP * i) : 0u;
        return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    }
}

template <bool F32>
__device__ __forceinline__ void to_floats(uint4 v, float (&x)[F32 ? 4 : 8])
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

template <bool F32, bool VEC, int STEP>
__device__ __forceinline__ void store_piece(char *row, int64_t c, int cols, const float (&x)[F32 ? 4 : 8])
{
    if constexpr (VEC) {
        uint4 v;
        if constexpr (F32) v = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
        else v = make_uint4(bf16x2_rn(x[0], x[1]), bf16x2_rn(x[2], x[3]), bf16x2_rn(x[4], x[5]), bf16x2_rn(x[6], x[7]));
        *reinterpret_cast<uint4 *>(row + c * (F32 ? 4 : 2)) = v;
    } else {
#pragma unroll
        for (int i = 0; i < (F32 ? 4 : 8); ++i)
            if (c + STEP * i < cols) {
                if constexpr (F32) reinterpret_cast<float *>(row)[c + STEP * i] = x[i];
                else reinterpret_cast<uint16_t *>(row)[c + STEP * i] = f32_bf16(x[i]);
            }
    }
}

constexpr int kBatch = 4;             // rows or pieces that a thread loads before it uses the first

// O[t] = sum_j w[t, j] Y[slots[t, j]], j ascending, in FP32; a thread has one
// piece of one token.
template <bool F32, bool VEC>
__global__ void __launch_bounds__(256) combine_kernel(const CombineArgs a)
{
    constexpr int N = F32 ? 4 : 8, ES = F32 ? 4 : 2;
    const int pieces = (a.cols + N - 1) / N;
    const int64_t total = a.T * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = total < 0x7FFFFFFF ? (int64_t)((uint32_t)i / (uint32_t)pieces) : i / pieces;
        const int64_t c = (i - t * pieces) * N;
        float acc[N] = {};
        for (int j0 = 0; j0 < a.k; j0 += kBatch) {
            uint4 v[kBatch];
            float w[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int64_t s = j0 + j < a.k ? __ldg(a.slots + t * a.k + j0 + j) : -1;
                w[j] = j0 + j < a.k && a.weights ? __ldg(a.weights + t * a.k + j0 + j) : 1.0f;
                v[j] = make_uint4(0u, 0u, 0u, 0u);
                const bool ok = s >= 0 && s < a.yrows;
                if (!ok) w[j] = 0.0f;
                else v[j] = load_piece<F32, VEC, 1>(static_cast<const char *>(a.Y) + s * a.ldy * ES, c, a.cols);
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                float x[N];
                to_floats<F32>(v[j], x);
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] = fmaf(w[j], x[e], acc[e]);
            }
        }
        store_piece<F32, VEC, 1>(static_cast<char *>(a.O) + t * a.ldo * ES, c, a.cols, acc);
    }
}

// dY[slots[t, j]] = w[t, j] dO[t], dw[t, j] = Y[slots[t, j]] . dO[t]; W lanes
// for each (t, j), those of a token next to each other, so that they share its dO
// row in the caches.  Fewer than a warp for short rows (32768 tokens, k = 2, 64 BF16
// columns: 8 us with 8 lanes, 24 with 32).  Rows that allow no 16-byte pieces: lanes
// have neighbouring columns, so that a load or store touches one line or two
// (16384 tokens, k = 4, 2047 BF16 columns: 200 us, 304 with consecutive columns per
// lane; the weighted sum itself keeps these: 113 us there against 108, but 23 against
// 42 for 30000 tokens, k = 8, 97 columns, whose lanes would be idle).
template <bool F32, bool VEC, int W>
__global__ void __launch_bounds__(256) combine_backward_kernel(const CombineArgs a)
{
    constexpr int N = F32 ? 4 : 8, ES = F32 ? 4 : 2, PER = 32 / W;
    static_assert(VEC || W == 32, "lanes with neighbouring columns are a warp");
    const int lane = (int)lane_id() % W;
    const int64_t total = a.T * a.k;
    for (int64_t i0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * PER; i0 < total; i0 += (int64_t)gridDim.x * 8 * PER) {
        const int64_t i = i0 + (int64_t)lane_id() / W;
        const bool here = i < total;
        const int64_t t = (int64_t)((uint32_t)i / (uint32_t)a.k), s = here ? __ldg(a.slots + i) : -1;
        const bool ok = s >= 0 && s < a.yrows;
        const float w = here && a.weights ? __ldg(a.weights + i) : 1.0f;
        const char *dO = static_cast<const char *>(a.dO) + (ok ? t : 0) * a.ldo * ES;
        const char *y = static_cast<const char *>(a.Y) + (ok ? s : 0) * a.ldy * ES;
        char *dY = static_cast<char *>(a.dY) + (ok ? s : 0) * a.lddy * ES;
        const int cols = ok ? a.cols : 0;
        if (a.owner && ok && lane == 0) a.owner[s] = (int32_t)i;
        float dot = 0.0f;
        for (int64_t c0 = VEC ? lane * N : lane; c0 < cols; c0 += W * N * kBatch) {
            uint4 d[kBatch], v[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int64_t c = c0 + W * N * b;
                d[b] = v[b] = make_uint4(0u, 0u, 0u, 0u);
                if (c < cols) {
                    d[b] = load_piece<F32, VEC, 32>(dO, c, cols);
                    if (a.dw) v[b] = load_piece<F32, VEC, 32>(y, c, cols);
                }
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const int64_t c = c0 + W * N * b;
                float x[N], u[N];
                to_floats<F32>(d[b], x);
                to_floats<F32>(v[b], u);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    dot = fmaf(u[e], x[e], dot);
                    x[e] *= w;
                }
                if (c < cols) store_piece<F32, VEC, 32>(dY, c, cols, x);
            }
        }
        if (a.dw) {
            __syncwarp();
#pragma unroll
            for (int d = W / 2; d > 0; d >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, d);
            if (here && lane == 0) a.dw[i] = ok ? dot : 0.0f;
        }
    }
}

// Rows of dY that no slot names are zero: row r is named where the assignment
// that is written down for it has r for its slot, so that whatever `owner` held
// before the gradients' kernel wrote it names no row.  A warp looks at 32 rows, and
// then clears those that it found, as bytes or in pieces of 16.  With every row
// named it reads 8 bytes a row (16384 tokens, k = 4, 2048 BF16 columns with the weighted
// sum: 154 us a call, 150 without).
__global__ void __launch_bounds__(256) clear_unnamed_kernel(const CombineArgs a, int64_t row_bytes, int64_t pitch)
{
    const int lane = (int)lane_id();
    const uint32_t total = (uint32_t)(a.T * a.k);
    const bool wide = ((reinterpret_cast<uintptr_t>(a.dY) | (uintptr_t)pitch | (uintptr_t)row_bytes) & 15u) == 0;
    for (int64_t r0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * 32; r0 < a.yrows; r0 += (int64_t)gridDim.x * 256) {
        const int64_t r = r0 + lane;
        bool named = true;
        if (r < a.yrows) {
            const uint32_t i = (uint32_t)__ldcg(a.owner + r);
            named = i < total && __ldg(a.slots + i) == r;
        }
        for (uint32_t left = __ballot_sync(0xFFFFFFFFu, !named); left; left &= left - 1) {
            char *row = static_cast<char *>(a.dY) + (r0 + __ffs(left) - 1) * pitch;
            if (wide) {
                for (int64_t b = lane * 16; b < row_bytes; b += 512) *reinterpret_cast<uint4 *>(row + b) = make_uint4(0u, 0u, 0u, 0u);
            } else {
                for (int64_t b = lane * 2; b < row_bytes; b += 64) *reinterpret_cast<uint16_t *>(row + b) = 0;
            }
        }
    }
}

template <bool F32, bool VEC, int W>
cudaError_t run_combine_back(const CombineArgs &a, cudaStream_t st)
{
    const int64_t per = 8 * (32 / W), blocks = (a.T * a.k + per - 1) / per;
    combine_backward_kernel<F32, VEC, W><<<(unsigned)(blocks > 152 * 64 ? 152 * 64 : blocks), 256, 0, st>>>(a);
    return cudaGetLastError();
}

template <bool F32>
cudaError_t combine_back(const CombineArgs &a, bool vec, cudaStream_t st)
{
    const int pieces = a.cols / (F32 ? 4 : 8);
    if (!vec) return run_combine_back<F32, false, 32>(a, st);
    return pieces <= 8 ? run_combine_back<F32, true, 8>(a, st) : pieces <= 16 ? run_combine_back<F32, true, 16>(a, st)
                                                                             : run_combine_back<F32, true, 32>(a, st);
}

bool can_vec(const void *p, int64_t ld, int esize)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * esize % 16 == 0;
}

template <int V>
cudaError_t run_route(const RouteArgs &a, int blocks, cudaStream_t st)
{
    const size_t sm = (size_t)(kRouteWarps + 2) * a.E * sizeof(int32_t);
    auto kern = a.f32 ? route_kernel<V, true> : route_kernel<V, false>;
    cudaError_t e = cudaSuccess;
    if (sm > 48 * 1024) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sm);
    if (e != cudaSuccess) return e;
    if (blocks == 1) {
        kern<<<1, kRouteThreads, sm, st>>>(a);
        return cudaGetLastError();
    }
    void *args[] = {(void *)&a};
    return cudaLaunchCooperativeKernel((const void *)kern, dim3((unsigned)blocks), dim3(kRouteThreads), args, sm, st);
}

template <int V>
cudaError_t run_route_back(const RouteBackArgs &a, cudaStream_t st)
{
    const int64_t blocks = ((int64_t)a.T + 7) / 8;
    const unsigned grid = (unsigned)(blocks > 152 * 16 ? 152 * 16 : blocks);
    // whole lanes of 4 values, rows that start on them
    const int es = a.f32 ? 4 : 2;
    bool vec = false;
    if constexpr (V >= 4)
        vec = a.E % V == 0 && can_vec(a.logits, a.ldl, es) && can_vec(a.dl, a.lddl, es);
    if constexpr (V >= 4) {
        if (vec) {
            route_backward_kernel<V, true><<<grid, 256, 0, st>>>(a);
            return cudaGetLastError();
        }
    }
    route_backward_kernel<V, false><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

size_t route_scratch_bytes(int64_t E) { return (size_t)kRouteBlocks * (size_t)count_pitch((int)E) * sizeof(int32_t); }

cudaError_t launch_route(int64_t T, int64_t E, int k, bool renorm, const void *logits, bool f32, int64_t ldl,
                         float *weights, int32_t *experts, int32_t *slots, int32_t *rows, int32_t *ends,
                         int32_t *counts, WsHeader *ws, cudaStream_t st, uint32_t missing, unsigned long long limit_ns)
{
    RouteArgs a = {};
    a.logits = logits; a.ldl = ldl; a.T = (int)T; a.E = (int)E; a.k = k; a.f32 = f32; a.renorm = renorm;
    a.weights = weights; a.experts = experts; a.slots = slots; a.rows = rows; a.ends = ends; a.counts = counts;
    a.flags = &ws->flags; a.bar = &ws->fix_any;
    // a warp per token while there are SMs left
    int64_t blocks = (T + kRouteWarps - 1) / kRouteWarps;
    if (blocks > 1) {
        int dev = 0, sms = 0;
        if (cudaGetDevice(&dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1)
            return cudaErrorInvalidDevice;
        const int64_t most = sms < kRouteBlocks ? sms : kRouteBlocks;     // one block per SM: all of them run at once
        if (blocks > most) blocks = most;
        // the flag word and the barrier's count (a single block sets the one and needs no other)
        const cudaError_t e = cudaMemsetAsync(ws, 0, 2 * sizeof(uint32_t), st);
        if (e != cudaSuccess) return e;
    }
    if (blocks < 1) blocks = 1;
    a.arrivals = (uint32_t)blocks + missing; a.limit_ns = limit_ns;
    const int v = (int)((E + 31) / 32);
    return v <= 1 ? run_route<1>(a, (int)blocks, st) : v <= 2 ? run_route<2>(a, (int)blocks, st)
           : v <= 4 ? run_route<4>(a, (int)blocks, st) : v <= 8 ? run_route<8>(a, (int)blocks, st)
           : v <= 16 ? run_route<16>(a, (int)blocks, st) : run_route<32>(a, (int)blocks, st);
}

cudaError_t launch_route_backward(int64_t T, int64_t E, int k, bool renorm, const void *logits, bool f32, int64_t ldl,
                                  const int32_t *experts, const float *dw, void *dl, int64_t lddl, cudaStream_t st)
{
    RouteBackArgs a = {};
    a.logits = logits; a.ldl = ldl; a.experts = experts; a.dw = dw; a.dl = dl; a.lddl = lddl;
    a.T = (int)T; a.E = (int)E; a.k = k; a.f32 = f32; a.renorm = renorm;
    const int v = (int)((E + 31) / 32);
    return v <= 1 ? run_route_back<1>(a, st) : v <= 2 ? run_route_back<2>(a, st) : v <= 4 ? run_route_back<4>(a, st)
           : v <= 8 ? run_route_back<8>(a, st) : v <= 16 ? run_route_back<16>(a, st) : run_route_back<32>(a, st);
}

cudaError_t launch_combine(bool f32, int64_t T, int k, int64_t cols, const void *Y, int64_t yrows, int64_t ldy,
                           const int32_t *slots, const float *weights, void *O, int64_t ldo, cudaStream_t st)
{
    CombineArgs a = {};
    a.Y = Y; a.yrows = yrows; a.ldy = ldy; a.slots = slots; a.weights = weights; a.O = O; a.ldo = ldo;
    a.T = T; a.k = k; a.cols = (int)cols;
    const int es = f32 ? 4 : 2;
    const bool vec = can_vec(Y, ldy, es) && can_vec(O, ldo, es) && cols * es % 16 == 0;
    const int64_t blocks = (T * ((cols + (f32 ? 3 : 7)) / (f32 ? 4 : 8)) + 255) / 256;
    const unsigned grid = (unsigned)(blocks > 152 * 64 ? 152 * 64 : blocks);
    if (f32 && vec) combine_kernel<true, true><<<grid, 256, 0, st>>>(a);
    else if (f32) combine_kernel<true, false><<<grid, 256, 0, st>>>(a);
    else if (vec) combine_kernel<false, true><<<grid, 256, 0, st>>>(a);
    else combine_kernel<false, false><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_combine_backward(bool f32, int64_t T, int k, int64_t cols, const void *dO, int64_t lddo,
                                    const void *Y, int64_t yrows, int64_t ldy, const int32_t *slots,
                                    const float *weights, void *dY, int64_t lddy, float *dw, int32_t *owner,
                                    cudaStream_t st)
{
    CombineArgs a = {};
    a.Y = Y; a.dO = dO; a.yrows = yrows; a.ldy = ldy; a.ldo = lddo; a.lddy = lddy; a.slots = slots;
    a.weights = weights; a.dY = dY; a.dw = dw; a.owner = owner; a.T = T; a.k = k; a.cols = (int)cols;
    const int es = f32 ? 4 : 2;
    const bool vec = (!dw || can_vec(Y, ldy, es)) && can_vec(dO, lddo, es) && can_vec(dY, lddy, es) && cols * es % 16 == 0;
    cudaError_t e = T == 0 ? cudaSuccess : f32 ? combine_back<true>(a, vec, st) : combine_back<false>(a, vec, st);
    if (e != cudaSuccess || !owner || yrows == 0 || cols == 0) return e;
    const int64_t blocks = (yrows + 255) / 256;
    clear_unnamed_kernel<<<(unsigned)(blocks > 152 * 8 ? 152 * 8 : blocks), 256, 0, st>>>(a, cols * es, lddy * es);
    return cudaGetLastError();
}

}  // namespace emu
