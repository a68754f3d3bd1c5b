// The experts of one rank for few tokens.  Declared in include/mw.h.
// Plain form: one warp per activation and one warp per output value.
#include <new>
#include <string.h>

#include "mw_internal.cuh"

struct mw_experts {
    mw_experts_config cfg;
    const uint16_t *w_gate_up, *w_down;
    void *slab;
    int32_t *status;
    uint16_t *act;              // [max_tokens * K, I] bf16
    int64_t launches;
};

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float bf16_to_f32(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

__device__ __forceinline__ uint16_t f32_to_bf16(float f)
{
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7fc0u;
    u += 0x7fffu + ((u >> 16) & 1u);
    return (uint16_t)(u >> 16);
}

__device__ __forceinline__ float warp_dot(const uint16_t *a, const uint16_t *b, int n, int lane)
{
    float s = 0.0f;
    for (int i = lane; i < n; i += 32) s = fmaf(bf16_to_f32(a[i]), bf16_to_f32(b[i]), s);
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    return s;
}

// The expert of a pick as an index into this rank's weights, -1 = none here.
__device__ __forceinline__ int local_expert(int id, const mw_experts_config &c, int32_t *status)
{
    if (id < -1 || id >= c.E) atomicCAS(status, MW_OK, MW_ERR_BAD_INDEX);
    const int e = id - c.expert_first;
    return id >= 0 && id < c.E && e >= 0 && e < c.expert_count ? e : -1;
}

__global__ void __launch_bounds__(kThreads) k_experts_up(mw_experts_config c, const uint8_t *x, int64_t xs, const int32_t *ids,
                                                         const uint16_t *w, uint16_t *act, int32_t *status)
{
    const int lane = threadIdx.x & 31, i = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), pick = blockIdx.y;
    if (i >= c.I) return;
    const int e = local_expert(ids[pick], c, status);
    if (e < 0) return;
    const uint16_t *row = (const uint16_t *)(x + (int64_t)(pick / c.K) * xs);
    const float g = warp_dot(w + ((int64_t)e * 2 * c.I + i) * c.H, row, c.H, lane);
    const float u = warp_dot(w + ((int64_t)e * 2 * c.I + c.I + i) * c.H, row, c.H, lane);
    if (lane == 0) act[(int64_t)pick * c.I + i] = f32_to_bf16(g / (1.0f + expf(-g)) * u);
}

__global__ void __launch_bounds__(kThreads) k_experts_down(mw_experts_config c, const int32_t *ids, const float *weights, const uint16_t *w,
                                                           const uint16_t *act, uint8_t *y, int64_t ys, int32_t *status)
{
    const int lane = threadIdx.x & 31, h = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), t = blockIdx.y;
    if (h >= c.H) return;
    float s = 0.0f;
    for (int k = 0; k < c.K; ++k) {
        const int e = local_expert(ids[t * c.K + k], c, status);
        if (e < 0) continue;
        s = fmaf(weights ? weights[t * c.K + k] : 1.0f,
                 warp_dot(w + ((int64_t)e * c.H + h) * c.I, act + (int64_t)(t * c.K + k) * c.I, c.I, lane), s);
    }
    if (lane == 0) ((uint16_t *)(y + (int64_t)t * ys))[h] = f32_to_bf16(s);
}

}  // namespace

extern "C" {

int mw_experts_create(mw_experts **out, const mw_experts_config *cfg, const void *w_gate_up, const void *w_down)
{
    if (!out) return MW_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || !w_gate_up || !w_down) return MW_ERR_INVALID_ARG;
    if (cfg->E < 1 || cfg->K < 1 || cfg->K > MW_MAX_TOPK || cfg->max_tokens < 1 || cfg->max_tokens > MW_EXPERTS_MAX_TOKENS ||
        (int64_t)cfg->max_tokens * cfg->K > MW_EXPERTS_MAX_PICKS || cfg->H < 8 || cfg->H % 8 || cfg->I < 16 || cfg->I % 16 ||
        cfg->expert_first < 0 || cfg->expert_count < 1 || cfg->expert_count > MW_EXPERTS_MAX_LOCAL ||
        cfg->expert_first > cfg->E - cfg->expert_count || cfg->device < 0 ||
        (cfg->flags & ~(uint32_t)(MW_FLAG_NO_OVERLAP | MW_FLAG_SHORT_WAITS)))
        return MW_ERR_INVALID_ARG;
    if (((uintptr_t)w_gate_up | (uintptr_t)w_down) & 15u) return MW_ERR_ALIGNMENT;
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || cfg->device >= ndev) return MW_ERR_CUDA;
    if (cudaSetDevice(cfg->device) != cudaSuccess) return MW_ERR_CUDA;
    mw_experts *m = new (std::nothrow) mw_experts();
    if (!m) return MW_ERR_INVALID_ARG;
    memset(m, 0, sizeof(*m));
    m->cfg = *cfg;
    m->w_gate_up = (const uint16_t *)w_gate_up; m->w_down = (const uint16_t *)w_down;
    const size_t bytes = 256 + (size_t)cfg->max_tokens * cfg->K * cfg->I * 2;
    if (cudaMalloc(&m->slab, bytes) != cudaSuccess) { cudaGetLastError(); delete m; return MW_ERR_CUDA; }
    m->status = (int32_t *)m->slab;
    m->act = (uint16_t *)((uint8_t *)m->slab + 256);
    if (cudaMemset(m->slab, 0, bytes) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) { mw_experts_destroy(m); return MW_ERR_CUDA; }
    *out = m;
    return MW_OK;
}

int mw_experts_destroy(mw_experts *m)
{
    if (!m) return MW_OK;
    cudaSetDevice(m->cfg.device);
    cudaDeviceSynchronize();
    const int rc = cudaFree(m->slab) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
    delete m;
    return rc;
}

int mw_experts_forward(mw_experts *m, const void *x, int64_t x_stride_bytes, const int32_t *topk_ids, const float *weights, int32_t T,
                       void *y, int64_t y_stride_bytes, void *stream)
{
    if (!m || T < 0 || T > m->cfg.max_tokens || x_stride_bytes < 0 || y_stride_bytes < 0) return MW_ERR_INVALID_ARG;
    if (T == 0) return MW_OK;
    if (!x || !topk_ids || !y) return MW_ERR_INVALID_ARG;
    const int64_t row = (int64_t)m->cfg.H * 2;
    if ((x_stride_bytes && x_stride_bytes < row) || (y_stride_bytes && y_stride_bytes < row)) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)y | (uint64_t)x_stride_bytes | (uint64_t)y_stride_bytes) & 15u) return MW_ERR_ALIGNMENT;
    if (((uintptr_t)topk_ids | (uintptr_t)weights) & 3u) return MW_ERR_ALIGNMENT;
    cudaStream_t st = (cudaStream_t)stream;
    const int64_t xs = x_stride_bytes ? x_stride_bytes : row, ys = y_stride_bytes ? y_stride_bytes : row;
    constexpr int W = kThreads / 32;
    k_experts_up<<<dim3((m->cfg.I + W - 1) / W, T * m->cfg.K), kThreads, 0, st>>>(m->cfg, (const uint8_t *)x, xs, topk_ids, m->w_gate_up, m->act, m->status);
    k_experts_down<<<dim3((m->cfg.H + W - 1) / W, T), kThreads, 0, st>>>(m->cfg, topk_ids, weights, m->w_down, m->act, (uint8_t *)y, ys, m->status);
    m->launches += 2;
    return cudaGetLastError() == cudaSuccess ? MW_OK : MW_ERR_CUDA;
}

int mw_experts_get_status(mw_experts *m, int32_t *status, void *stream)
{
    if (!m || !status) return MW_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemcpyAsync(status, m->status, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(m->status, 0, 4, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return MW_ERR_CUDA;
    return MW_OK;
}

int64_t mw_experts_kernel_launches(const mw_experts *m) { return m ? m->launches : 0; }

}  // extern "C"
