// The shared projection with low-rank adapters.  Declared in include/mw.h.
// Plain form: one warp per low-rank value and one warp per output value.
#include <new>
#include <string.h>

#include "mw_internal.cuh"

struct mw_project {
    mw_project_config cfg;
    const uint16_t *w, *a, *b;
    const float *scale;
    void *slab;
    int32_t *status;
    uint16_t *v;                // [max_tokens, rank] bf16
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

__global__ void __launch_bounds__(kThreads) k_project_shrink(mw_project_config c, const uint8_t *x, int64_t xs, const int32_t *ids,
                                                             const uint16_t *a, const float *scale, uint16_t *v, int32_t *status)
{
    const int lane = threadIdx.x & 31, t = blockIdx.x, id = ids[t];
    if (id < -1 || id >= c.adapters) atomicCAS(status, MW_OK, MW_ERR_BAD_INDEX);
    if (id < 0 || id >= c.adapters) return;
    for (int j = threadIdx.x >> 5; j < c.rank; j += kThreads / 32) {
        const float d = warp_dot(a + ((int64_t)id * c.rank + j) * c.H, (const uint16_t *)(x + (int64_t)t * xs), c.H, lane);
        if (lane == 0) v[(int64_t)t * c.rank + j] = f32_to_bf16(scale ? scale[id] * d : d);
    }
}

__global__ void __launch_bounds__(kThreads) k_project(mw_project_config c, int T, const uint8_t *x, int64_t xs, const int32_t *ids, const uint16_t *w,
                                                      const uint16_t *b, const uint16_t *v, uint8_t *y, int64_t ys, int f32)
{
    const int lane = threadIdx.x & 31, o = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (o >= c.O) return;
    for (int t = blockIdx.y; t < T; t += gridDim.y) {
        float s = warp_dot(w + (int64_t)o * c.H, (const uint16_t *)(x + (int64_t)t * xs), c.H, lane);
        const int id = ids ? ids[t] : -1;
        if (id >= 0 && id < c.adapters) s += warp_dot(b + ((int64_t)id * c.O + o) * c.rank, v + (int64_t)t * c.rank, c.rank, lane);
        if (lane == 0) {
            if (f32) ((float *)(y + (int64_t)t * ys))[o] = s;
            else ((uint16_t *)(y + (int64_t)t * ys))[o] = f32_to_bf16(s);
        }
    }
}

}  // namespace

extern "C" {

int mw_project_create(mw_project **out, const mw_project_config *cfg, const void *w, const void *a, const void *b, const float *scale)
{
    if (!out) return MW_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || !w) return MW_ERR_INVALID_ARG;
    if (cfg->H < 8 || cfg->H % 8 || cfg->O < 1 || cfg->max_tokens < 1 || cfg->max_tokens > (1 << 24) || cfg->adapters < 0 || cfg->device < 0 ||
        (cfg->flags & ~(uint32_t)(MW_FLAG_NO_OVERLAP | MW_FLAG_SHORT_WAITS)))
        return MW_ERR_INVALID_ARG;
    if (cfg->adapters ? (cfg->rank < 8 || cfg->rank % 8 || cfg->rank > MW_MAX_ADAPTER_RANK || !a || !b) : cfg->rank != 0) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)w & 15u) || (cfg->adapters && ((((uintptr_t)a | (uintptr_t)b) & 15u) || ((uintptr_t)scale & 3u)))) return MW_ERR_ALIGNMENT;
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || cfg->device >= ndev) return MW_ERR_CUDA;
    if (cudaSetDevice(cfg->device) != cudaSuccess) return MW_ERR_CUDA;
    mw_project *m = new (std::nothrow) mw_project();
    if (!m) return MW_ERR_INVALID_ARG;
    memset(m, 0, sizeof(*m));
    m->cfg = *cfg;
    m->w = (const uint16_t *)w; m->a = (const uint16_t *)a; m->b = (const uint16_t *)b; m->scale = scale;
    const size_t bytes = 256 + (size_t)cfg->max_tokens * cfg->rank * 2;
    if (cudaMalloc(&m->slab, bytes) != cudaSuccess) { cudaGetLastError(); delete m; return MW_ERR_CUDA; }
    m->status = (int32_t *)m->slab;
    m->v = (uint16_t *)((uint8_t *)m->slab + 256);
    if (cudaMemset(m->slab, 0, bytes) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) { mw_project_destroy(m); return MW_ERR_CUDA; }
    *out = m;
    return MW_OK;
}

int mw_project_destroy(mw_project *m)
{
    if (!m) return MW_OK;
    cudaSetDevice(m->cfg.device);
    cudaDeviceSynchronize();
    const int rc = cudaFree(m->slab) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
    delete m;
    return rc;
}

int mw_project_forward(mw_project *m, const void *x, int64_t x_stride_bytes, const int32_t *adapter_ids, int32_t T, void *y, int32_t y_dtype,
                       int64_t y_stride_bytes, void *stream)
{
    if (!m || T < 0 || T > m->cfg.max_tokens || x_stride_bytes < 0 || y_stride_bytes < 0) return MW_ERR_INVALID_ARG;
    if (y_dtype != MW_DTYPE_F32 && y_dtype != MW_DTYPE_BF16) return MW_ERR_INVALID_ARG;
    if (T == 0) return MW_OK;
    if (!x || !y) return MW_ERR_INVALID_ARG;
    const int ye = y_dtype == MW_DTYPE_F32 ? 4 : 2;
    const int64_t xrow = (int64_t)m->cfg.H * 2, yrow = (int64_t)m->cfg.O * ye;
    if ((x_stride_bytes && x_stride_bytes < xrow) || (y_stride_bytes && y_stride_bytes < yrow)) return MW_ERR_INVALID_ARG;
    if ((((uintptr_t)x | (uint64_t)x_stride_bytes) & 15u) || ((uintptr_t)y | (uint64_t)y_stride_bytes) % ye || ((uintptr_t)adapter_ids & 3u))
        return MW_ERR_ALIGNMENT;
    cudaStream_t st = (cudaStream_t)stream;
    const int64_t xs = x_stride_bytes ? x_stride_bytes : xrow, ys = y_stride_bytes ? y_stride_bytes : yrow;
    if (adapter_ids && m->cfg.adapters) {
        k_project_shrink<<<T, kThreads, 0, st>>>(m->cfg, (const uint8_t *)x, xs, adapter_ids, m->a, m->scale, m->v, m->status);
        m->launches += 1;
    }
    k_project<<<dim3((m->cfg.O + kThreads / 32 - 1) / (kThreads / 32), T < 1024 ? T : 1024), kThreads, 0, st>>>(
        m->cfg, T, (const uint8_t *)x, xs, adapter_ids, m->w, m->b, m->v, (uint8_t *)y, ys, ye == 4);
    m->launches += 1;
    return cudaGetLastError() == cudaSuccess ? MW_OK : MW_ERR_CUDA;
}

int mw_project_get_status(mw_project *m, int32_t *status, void *stream)
{
    if (!m || !status) return MW_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemcpyAsync(status, m->status, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(m->status, 0, 4, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return MW_ERR_CUDA;
    return MW_OK;
}

int64_t mw_project_kernel_launches(const mw_project *m) { return m ? m->launches : 0; }

}  // extern "C"
