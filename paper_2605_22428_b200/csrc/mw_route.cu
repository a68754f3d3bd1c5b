// The router's choice: logits -> the K experts of every token and their weights.  Declared in include/mw.h.
//
// One warp per token.  key[e] = logit[e] + bias[e], or score[e] + bias[e], in float32; lane l holds experts l, l + 32, ... (coalesced loads).  For the warp's
// integer reductions a key is mapped to an unsigned integer of the same order (sign bit flipped for positive keys, all bits for negative ones; 0:
// never chosen).
//
// The K-th largest of the lanes' own maxima is at most the K-th largest key, so the keys from it on are all that can be chosen:
// for random scores a dozen.  They are brought together in shared memory, one per lane, in the order of their experts, and each
// counts the keys before it: that is its place.  Where they are more than 32 (many ties, large K) the choice is made in K rounds
// over all keys instead, the largest of the lanes' largest by one integer reduction.  Exact either way, ties to the lowest expert.
// Bound by instruction issue where there are many tokens (65536 of 256 experts, top-8: 49 us, an instruction issued in 80 % of cycles, floor 10.2; rounds alone 62), by
// the latency of a warp's own chain up to a wave of them (4096 tokens 5.9 us, rounds alone 8.1; 50 % of cycles), by the launch for a few (3.1 us on the device).
#include "mw_internal.cuh"

namespace {

constexpr int kWarpsPerBlock = 4;
constexpr unsigned kAll = 0xffffffffu;

struct RouteArgs {
    const uint8_t *logits;
    int64_t stride;             // bytes between rows
    const float *bias;
    int32_t *ids;
    float *weights;
    int T, E, K;
    uint32_t flags;
    float scale;
};

template <bool BF16>
__device__ __forceinline__ float load_logit(const uint8_t *row, int e)
{
    if (BF16) return __uint_as_float((uint32_t)((const uint16_t *)row)[e] << 16);
    return ((const float *)row)[e];
}

// Order-preserving image of a key; 0 = never chosen.  (-0 is first made +0: they compare equal.)
__device__ __forceinline__ uint32_t ordered(float key)
{
    if (!(key > -INFINITY)) return 0u;                   // -inf and NaN
    const uint32_t u = __float_as_uint(key + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
    return v;
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, d));
    return v;
}

// Sum over all experts of the exponentials of logits relative to `top`, the largest of them.
template <int V>
__device__ __forceinline__ float exponentials(const float (&logit)[V], float &top)
{
    float m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) m = fmaxf(m, logit[i]);                 // (passes over NaN)
    top = warp_max(m);
#pragma unroll
    for (int i = 0; i < V; ++i) s += logit[i] > -INFINITY ? expf(logit[i] - top) : 0.0f;
    return warp_sum(s);
}

// SCORE: the bias is added to the score, so every expert's is computed first (4096 tokens, 256 experts, top-8: sigmoid 7.9 us, softmax 8.3, against 5.9).
// (A kernel of its own: as a branch its registers cost the other form 4% at 65536 tokens.)
template <int V, bool BF16, bool SCORE>
__global__ void __launch_bounds__(32 * kWarpsPerBlock) k_route(const __grid_constant__ RouteArgs a)
{
    __shared__ uint4 held_s[kWarpsPerBlock][32];
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int t = blockIdx.x * kWarpsPerBlock + (threadIdx.x >> 5);
    if (t >= a.T) return;
    const uint8_t *row = a.logits + (int64_t)t * a.stride;
    uint4 *held = held_s[threadIdx.x >> 5];
    float logit[V], key[V];                 // NaN counts as -inf; a key of -inf is never chosen
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = i * 32 + lane;
        logit[i] = e < a.E ? load_logit<BF16>(row, e) : -INFINITY;
    }
    if (SCORE) {
        const bool sigmoid = a.flags & MW_ROUTE_SIGMOID;
        float top = 0.0f, sum = 1.0f;
        if (!sigmoid) sum = exponentials(logit, top);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            key[i] = -INFINITY;
            if (logit[i] > -INFINITY)
                key[i] = fmaxf((sigmoid ? 1.0f / (1.0f + expf(-logit[i])) : expf(logit[i] - top) / sum) + a.bias[i * 32 + lane], -INFINITY);
        }
    } else if (a.bias) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = i * 32 + lane;
            key[i] = fmaxf(e < a.E ? logit[i] + a.bias[e] : -INFINITY, -INFINITY);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = fmaxf(logit[i], -INFINITY);
    }
    // the lane's candidates for the result: experts, their places and logits; two of them only after rounds
    int chosen[2] = {-1, -1}, place[2] = {0, 0}, found = 0;
    float chosen_logit[2] = {-INFINITY, -INFINITY};

    float most = key[0], bound = -INFINITY;
#pragma unroll
    for (int i = 1; i < V; ++i) most = fmaxf(most, key[i]);
    for (uint32_t mine = ordered(most), n = 0; n < (uint32_t)a.K;) {
        const uint32_t top = __reduce_max_sync(kAll, mine);
        if (top == 0u) { bound = -INFINITY; break; }        // fewer lanes than K have any
        const unsigned b = __ballot_sync(kAll, mine == top);
        bound = __shfl_sync(kAll, most, __ffs(b) - 1);
        n += __popc(b);
        if (mine == top) mine = 0u;
    }
    int count = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool in = key[i] >= bound && key[i] > -INFINITY;
        const unsigned b = __ballot_sync(kAll, in);
        if (b) {
            const int at = count + __popc(b & ((1u << lane) - 1));
            if (in && at < 32) held[at] = make_uint4(ordered(key[i]), i * 32 + lane, __float_as_uint(logit[i]), 0u);
            count += __popc(b);
        }
    }
    __syncwarp();
    if (count <= 32) {
        const uint4 c = held[lane < count ? lane : 0];
        int before = 0;
        for (int j = 0; j < count; ++j) {
            const uint32_t other = __shfl_sync(kAll, c.x, j);
            before += other > c.x || (other == c.x && j < lane);
        }
        if (lane < count && before < a.K) { chosen[0] = (int)c.y; place[0] = before; chosen_logit[0] = __uint_as_float(c.z); }
        found = count < a.K ? count : a.K;
    } else {
        for (int k = 0; k < a.K; ++k) {
            float first = -INFINITY;
            int at = 0;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (key[i] > first) { first = key[i]; at = i; }             // the first of equals: lowest expert of the lane
            const uint32_t best = ordered(first), top = __reduce_max_sync(kAll, best);
            if (top == 0u) break;
            const int e = (int)__reduce_min_sync(kAll, best == top ? (unsigned)(at * 32 + lane) : kAll);
            if (lane == (e & 31)) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i == (e >> 5)) key[i] = -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)                     // (not indexed by k: that would put the arrays into local memory)
                if (k == j * 32 + lane) { chosen[j] = e; place[j] = k; }
            found = k + 1;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (chosen[j] >= 0) {
                const float l = load_logit<BF16>(row, chosen[j]);
                chosen_logit[j] = l == l ? l : -INFINITY;
            }
    }
    // weights, from the logits alone
    const bool renorm = a.flags & MW_ROUTE_RENORMALISE, sigmoid = a.flags & MW_ROUTE_SIGMOID;
    float w[2];
    const float top_chosen = warp_max(fmaxf(chosen_logit[0], chosen_logit[1]));
    if (sigmoid) {
        // sigmoid(l) = e^l (1 + o(1)) for very negative l: the ratio of two such is that of the exponentials, which does not underflow
        const bool tiny = renorm && top_chosen < -60.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            w[j] = chosen[j] < 0 ? 0.0f : tiny ? expf(chosen_logit[j] - top_chosen) : 1.0f / (1.0f + expf(-chosen_logit[j]));
    } else {
        float top = top_chosen, sum = 1.0f;
        if (!renorm) sum = exponentials(logit, top);
        // renormalised, the sum over all experts cancels: exponentials relative to the largest chosen logit, so that the sum is at least 1
#pragma unroll
        for (int j = 0; j < 2; ++j) w[j] = chosen[j] < 0 ? 0.0f : expf(chosen_logit[j] - top) / sum;
    }
    if (renorm) {
        const float sum = warp_sum(w[0] + w[1]);
#pragma unroll
        for (int j = 0; j < 2; ++j) w[j] = chosen[j] < 0 ? 0.0f : w[j] / sum;
    }
    int32_t *ids = a.ids + (int64_t)t * a.K;
    float *weights = a.weights + (int64_t)t * a.K;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (chosen[j] >= 0) { ids[place[j]] = chosen[j]; weights[place[j]] = w[j] * a.scale; }
        const int k = j * 32 + lane;
        if (k >= found && k < a.K) { ids[k] = -1; weights[k] = 0.0f; }      // nothing left to choose
    }
}

template <int V, bool SCORE>
cudaError_t launch(const RouteArgs &a, bool bf16, cudaStream_t st)
{
    const dim3 grid((unsigned)((a.T + kWarpsPerBlock - 1) / kWarpsPerBlock)), block(32 * kWarpsPerBlock);
    return bf16 ? mw_launch(k_route<V, true, SCORE>, grid, block, 0, st, true, a) : mw_launch(k_route<V, false, SCORE>, grid, block, 0, st, true, a);
}

template <bool SCORE>
cudaError_t launch(const RouteArgs &a, bool bf16, cudaStream_t st)
{
    const int v = (a.E + 31) / 32;
    return v <= 1 ? launch<1, SCORE>(a, bf16, st) : v <= 2 ? launch<2, SCORE>(a, bf16, st) : v <= 4 ? launch<4, SCORE>(a, bf16, st)
         : v <= 8 ? launch<8, SCORE>(a, bf16, st) : v <= 16 ? launch<16, SCORE>(a, bf16, st) : launch<32, SCORE>(a, bf16, st);
}

}  // namespace

extern "C" int mw_route(const void *logits, int32_t logits_dtype, int64_t logits_stride_bytes, const float *bias, int32_t T, int32_t E,
                        int32_t K, uint32_t flags, float scale, int32_t *topk_ids, float *topk_weights, void *stream)
{
    if (T < 0 || E < 1 || E > MW_MAX_ROUTE_EXPERTS || K < 1 || K > E || K > MW_MAX_TOPK || logits_stride_bytes < 0) return MW_ERR_INVALID_ARG;
    if (logits_dtype != MW_DTYPE_F32 && logits_dtype != MW_DTYPE_BF16) return MW_ERR_INVALID_ARG;
    if (flags & ~(uint32_t)(MW_ROUTE_SIGMOID | MW_ROUTE_RENORMALISE | MW_ROUTE_SCORE_BIAS)) return MW_ERR_INVALID_ARG;
    if (T == 0) return MW_OK;
    if (!logits || !topk_ids || !topk_weights) return MW_ERR_INVALID_ARG;
    const int es = logits_dtype == MW_DTYPE_BF16 ? 2 : 4;
    if (logits_stride_bytes && logits_stride_bytes < (int64_t)E * es) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)logits | (uint64_t)logits_stride_bytes) % es || (uintptr_t)bias % 4 || (uintptr_t)topk_ids % 4 || (uintptr_t)topk_weights % 4)
        return MW_ERR_ALIGNMENT;
    RouteArgs a;
    a.logits = (const uint8_t *)logits; a.stride = logits_stride_bytes ? logits_stride_bytes : (int64_t)E * es;
    a.bias = bias; a.ids = topk_ids; a.weights = topk_weights;
    a.T = T; a.E = E; a.K = K; a.flags = flags; a.scale = scale;
    const bool bf16 = es == 2;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = bias && (flags & MW_ROUTE_SCORE_BIAS) ? launch<true>(a, bf16, st) : launch<false>(a, bf16, st);
    if (e != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
    return MW_OK;
}
