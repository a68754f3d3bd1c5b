// The router's choice: logits -> the K experts of every token and their weights.  Declared in include/mw.h.
//
// One warp per token.  key[e] = logit[e] + bias[e] is mapped to an unsigned integer of the same order (sign bit flipped for
// positive keys, all bits for negative ones; 0 stands for "never chosen": -inf, NaN and experts already taken), so the
// largest key of the warp is one integer reduction and the lowest expert that has it another: K rounds, exact, ties to the
// lowest expert.  Lane l holds experts l, l + 32, ... (coalesced loads, and within a lane ascending expert = ascending register).
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

template <int V, bool BF16>
__global__ void __launch_bounds__(32 * kWarpsPerBlock) k_route(const __grid_constant__ RouteArgs a)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const int t = blockIdx.x * kWarpsPerBlock + (threadIdx.x >> 5);
    if (t >= a.T) return;
    const uint8_t *row = a.logits + (int64_t)t * a.stride;
    float logit[V];
    uint32_t key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = i * 32 + lane;
        logit[i] = e < a.E ? load_logit<BF16>(row, e) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = i * 32 + lane;
        key[i] = e < a.E ? ordered(a.bias ? logit[i] + a.bias[e] : logit[i]) : 0u;
        if (logit[i] != logit[i]) logit[i] = -INFINITY;
    }
    // K rounds; lane k keeps choice k and choice k + 32
    int chosen[2] = {-1, -1};
    float chosen_logit[2] = {-INFINITY, -INFINITY};
    for (int k = 0; k < a.K; ++k) {
        uint32_t best = 0u;
        int at = 0;
        float best_logit = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (key[i] > best) { best = key[i]; at = i; best_logit = logit[i]; }        // the first of equals: lowest expert of the lane
        const uint32_t top = __reduce_max_sync(kAll, best);
        if (top == 0u) break;
        const int e = (int)__reduce_min_sync(kAll, best == top ? (unsigned)(at * 32 + lane) : kAll);
        const float l = __shfl_sync(kAll, best_logit, e & 31);
        if (lane == (e & 31)) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i == (e >> 5)) key[i] = 0u;
        }
        if (lane == (k & 31)) { chosen[k >> 5] = e; chosen_logit[k >> 5] = l; }
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
        if (!renorm) {
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < V; ++i) m = fmaxf(m, logit[i]);
            top = warp_max(m);
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) s += logit[i] > -INFINITY ? expf(logit[i] - top) : 0.0f;
            sum = warp_sum(s);
        }
        // renormalised, the sum over all experts cancels: exponentials relative to the largest chosen logit, so that the sum is at least 1
#pragma unroll
        for (int j = 0; j < 2; ++j) w[j] = chosen[j] < 0 ? 0.0f : expf(chosen_logit[j] - top) / sum;
    }
    if (renorm) {
        const float sum = warp_sum(w[0] + w[1]);
#pragma unroll
        for (int j = 0; j < 2; ++j) w[j] = chosen[j] < 0 ? 0.0f : w[j] / sum;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int k = j * 32 + lane;
        if (k < a.K) {
            a.ids[(int64_t)t * a.K + k] = chosen[j];
            a.weights[(int64_t)t * a.K + k] = w[j] * a.scale;
        }
    }
}

template <int V>
cudaError_t launch(const RouteArgs &a, bool bf16, cudaStream_t st)
{
    const dim3 grid((unsigned)((a.T + kWarpsPerBlock - 1) / kWarpsPerBlock)), block(32 * kWarpsPerBlock);
    return bf16 ? mw_launch(k_route<V, true>, grid, block, 0, st, true, a) : mw_launch(k_route<V, false>, grid, block, 0, st, true, a);
}

}  // namespace

extern "C" int mw_route(const void *logits, int32_t logits_dtype, int64_t logits_stride_bytes, const float *bias, int32_t T, int32_t E,
                        int32_t K, uint32_t flags, float scale, int32_t *topk_ids, float *topk_weights, void *stream)
{
    if (T < 0 || E < 1 || E > MW_MAX_ROUTE_EXPERTS || K < 1 || K > E || K > MW_MAX_TOPK || logits_stride_bytes < 0) return MW_ERR_INVALID_ARG;
    if (logits_dtype != MW_DTYPE_F32 && logits_dtype != MW_DTYPE_BF16) return MW_ERR_INVALID_ARG;
    if (flags & ~(uint32_t)(MW_ROUTE_SIGMOID | MW_ROUTE_RENORMALISE)) return MW_ERR_INVALID_ARG;
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
    const int v = (E + 31) / 32;
    const cudaError_t e = v <= 1 ? launch<1>(a, bf16, st) : v <= 2 ? launch<2>(a, bf16, st) : v <= 4 ? launch<4>(a, bf16, st)
                        : v <= 8 ? launch<8>(a, bf16, st) : v <= 16 ? launch<16>(a, bf16, st) : launch<32>(a, bf16, st);
    if (e != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
    return MW_OK;
}
