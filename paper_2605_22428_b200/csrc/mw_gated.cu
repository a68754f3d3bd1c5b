// The gated feed-forward block, y = W_down (act(W_gate x) * (W_up x)), and its gradients.  Declared in include/mw.h.
//
//   forward:   g = W_gate x, u = W_up x, h = act(g) u      one launch: a thread of the epilogue has both sums
//              y = W_down h                                the second
//   backward:  dh = W_down^T dy, dg = dh u act'(g), du = dh act(g), h once more        one launch
//              dx = W_gate^T dg + W_up^T du (one sum over 2 I), dW_gate and dW_up from (dg, du) and x, dW_down from dy and h      one to three launches
//
// g and u are kept in float32, or in the rows' type where the caller has them so: half the bytes between the two calls, but their rounding is as large as that of dg (gradients off by
// 0.0030 to 0.0035 in the 2-norm instead of 0.0024).
// 7168 wide, 2048 deep, bf16, call after call: 19.5 us for one token (weights 88 MB, 13.6 us at the rate of a copy), 23.8 for 64; 4096 tokens (361 GFLOP) 288 us under the power cap (1.25 PFLOP/s;
// 245 in runs too short for it), forward and backward 868 (734).
#include <new>
#include <string.h>

#include "mw_dense.cuh"

using namespace mw_dense;

struct mw_gated {
    mw_gated_config cfg;
    const uint16_t *w_gate_up, *w_down;
    void *slab;
    int32_t *status;
    uint16_t *h;                // [max_tokens, I]
    uint16_t *d_gate_up;        // [max_tokens, 2 I], with MW_FLAG_TRAIN
    Room room;
    int skew;                   // bytes added to the announced sizes of the next call's loads (test hook)
    int64_t launches;
    Ways ways;
};

namespace {

inline size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// Rows of `row` bytes at a distance of `stride` (0: compact).
int check_rows(const void *p, int64_t stride, int64_t row)
{
    if (stride < 0 || (stride && stride < row)) return MW_ERR_INVALID_ARG;
    return (((uintptr_t)p | (uint64_t)stride) & 15u) ? MW_ERR_ALIGNMENT : MW_OK;
}

// What a call's launches share.
Call begin(mw_gated *m, void *stream)
{
    const bool quick = (m->cfg.flags & MW_FLAG_SHORT_WAITS) != 0;
    Call call = {(cudaStream_t)stream, !(m->cfg.flags & MW_FLAG_NO_OVERLAP), m->cfg.dtype, &m->room, {quick ? 1 << 10 : 1 << 20, m->skew, m->status}, false, &m->launches, &m->ways};
    m->skew = 0;
    m->ways.count = 0;
    return call;
}

}  // namespace

extern "C" {

int mw_gated_create(mw_gated **out, const mw_gated_config *cfg, const void *w_gate_up, const void *w_down)
{
    if (!out) return MW_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || !w_gate_up || !w_down) return MW_ERR_INVALID_ARG;
    if (cfg->H < 8 || cfg->H % 8 || cfg->H > MW_GATED_MAX_WIDTH || cfg->I < 8 || cfg->I % 8 || cfg->I > MW_GATED_MAX_WIDTH || cfg->max_tokens < 1 ||
        cfg->max_tokens > MW_GATED_MAX_TOKENS || (cfg->dtype != MW_DTYPE_BF16 && cfg->dtype != MW_DTYPE_F16) ||
        (cfg->activation != MW_ACT_SILU && cfg->activation != MW_ACT_GELU) || cfg->device < 0 ||
        (cfg->flags & ~(uint32_t)(MW_FLAG_TRAIN | MW_FLAG_NO_OVERLAP | MW_FLAG_SHORT_WAITS)))
        return MW_ERR_INVALID_ARG;
    if (((uintptr_t)w_gate_up | (uintptr_t)w_down) & 15u) return MW_ERR_ALIGNMENT;
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || cfg->device >= ndev) { cudaGetLastError(); return MW_ERR_CUDA; }
    OnDevice here(cfg->device);
    if (!here.ok) { cudaGetLastError(); return MW_ERR_CUDA; }
    mw_gated *m = new (std::nothrow) mw_gated();
    if (!m) return MW_ERR_INVALID_ARG;
    m->cfg = *cfg;
    m->w_gate_up = (const uint16_t *)w_gate_up; m->w_down = (const uint16_t *)w_down;
    const size_t b_h = round256((size_t)cfg->max_tokens * cfg->I * 2), bytes = 256 + b_h + ((cfg->flags & MW_FLAG_TRAIN) ? 2 * b_h : 0);
    if (cudaMalloc(&m->slab, bytes) != cudaSuccess) { cudaGetLastError(); delete m; return MW_ERR_CUDA; }
    uint8_t *p = (uint8_t *)m->slab;
    m->status = (int32_t *)p; p += 256;
    m->h = (uint16_t *)p; p += b_h;
    m->d_gate_up = (cfg->flags & MW_FLAG_TRAIN) ? (uint16_t *)p : nullptr;
    if (find_room(&m->room, cfg->device) != cudaSuccess || load_kernels<Gate>() != cudaSuccess || load_kernels<Store>() != cudaSuccess ||
        load_kernels<GateBack<false>>() != cudaSuccess || load_kernels<GateBack<true>>() != cudaSuccess || cudaMemset(m->slab, 0, 256) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
        cudaGetLastError();
        mw_gated_destroy(m);
        return MW_ERR_CUDA;
    }
    *out = m;
    return MW_OK;
}

int mw_gated_destroy(mw_gated *m)
{
    if (!m) return MW_OK;
    OnDevice here(m->cfg.device);
    cudaDeviceSynchronize();
    const int rc = cudaFree(m->slab) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
    delete m;
    return rc;
}

int mw_gated_forward(mw_gated *m, const void *x, int64_t x_stride_bytes, int32_t T, void *y, int64_t y_stride_bytes, void *gate_up, void *stream)
{
    return mw_gated_forward_keep(m, x, x_stride_bytes, T, y, y_stride_bytes, gate_up, MW_DTYPE_F32, stream);
}

int mw_gated_forward_keep(mw_gated *m, const void *x, int64_t x_stride_bytes, int32_t T, void *y, int64_t y_stride_bytes, void *gate_up,
                          int32_t gate_up_dtype, void *stream)
{
    if (!m || T < 0 || T > m->cfg.max_tokens) return MW_ERR_INVALID_ARG;
    const mw_gated_config &c = m->cfg;
    if (gate_up_dtype != MW_DTYPE_F32 && gate_up_dtype != c.dtype) return MW_ERR_INVALID_ARG;
    const int H = c.H, I = c.I;
    const int64_t row = (int64_t)H * 2;
    if (T && (!x || !y)) return MW_ERR_INVALID_ARG;
    int rc = check_rows(x, x_stride_bytes, row);
    if (rc == MW_OK) rc = check_rows(y, y_stride_bytes, row);
    if (rc == MW_OK) rc = check_rows(gate_up, 0, 0);
    if (rc != MW_OK) return rc;
    if (T == 0) return MW_OK;
    OnDevice here(c.device);
    if (!here.ok) { cudaGetLastError(); return MW_ERR_CUDA; }
    Call call = begin(m, stream);
    Gate gate;
    gate.h = m->h; gate.gate_up = gate_up; gate.width = I; gate.activation = c.activation; gate.half = c.dtype == MW_DTYPE_F16; gate.rounded = gate_up_dtype != MW_DTYPE_F32;
    cudaError_t e = product(call, Job<Gate>{{x, x_stride_bytes ? x_stride_bytes : row, T, true}, {m->w_gate_up, row, 2 * I, true}, I, H, gate});
    call.early = true;
    const Store store = {(uint8_t *)y, y_stride_bytes ? y_stride_bytes : row, c.dtype, 0};
    if (e == cudaSuccess) e = product(call, Job<Store>{{m->h, (int64_t)I * 2, T, true}, {m->w_down, (int64_t)I * 2, H, true}, H, I, store});
    if (e != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
    return MW_OK;
}

int mw_gated_backward(mw_gated *m, const void *x, int64_t x_stride_bytes, const void *gate_up, const void *dy, int64_t dy_stride_bytes, int32_t T,
                      void *dx, int64_t dx_stride_bytes, void *dw_gate_up, void *dw_down, int32_t dw_dtype, int32_t accumulate, void *stream)
{
    return mw_gated_backward_kept(m, x, x_stride_bytes, gate_up, MW_DTYPE_F32, dy, dy_stride_bytes, T, dx, dx_stride_bytes, dw_gate_up, dw_down, dw_dtype, accumulate, stream);
}

int mw_gated_backward_kept(mw_gated *m, const void *x, int64_t x_stride_bytes, const void *gate_up, int32_t gate_up_dtype, const void *dy, int64_t dy_stride_bytes,
                           int32_t T, void *dx, int64_t dx_stride_bytes, void *dw_gate_up, void *dw_down, int32_t dw_dtype, int32_t accumulate, void *stream)
{
    if (!m || !m->d_gate_up || T < 0 || T > m->cfg.max_tokens) return MW_ERR_INVALID_ARG;
    const mw_gated_config &c = m->cfg;
    if (gate_up_dtype != MW_DTYPE_F32 && gate_up_dtype != c.dtype) return MW_ERR_INVALID_ARG;
    if (T && (!x || !gate_up || !dy)) return MW_ERR_INVALID_ARG;
    const int H = c.H, I = c.I;
    const int64_t row = (int64_t)H * 2, wide = (int64_t)I * 2;
    int rc = check_rows(x, x_stride_bytes, row);
    if (rc == MW_OK) rc = check_rows(dy, dy_stride_bytes, row);
    if (rc == MW_OK) rc = check_rows(dx, dx_stride_bytes, row);
    if (rc == MW_OK) rc = check_rows((const void *)((uintptr_t)gate_up | (uintptr_t)dw_gate_up | (uintptr_t)dw_down), 0, 0);
    if (rc != MW_OK) return rc;
    if (dw_dtype != MW_DTYPE_F32 && dw_dtype != c.dtype) return MW_ERR_INVALID_ARG;
    if (!dx && !dw_gate_up && !dw_down) return MW_OK;
    OnDevice here(c.device);
    if (!here.ok) { cudaGetLastError(); return MW_ERR_CUDA; }
    const int64_t size = element_bytes(dw_dtype);
    cudaError_t e = cudaSuccess;
    if (T == 0) {
        if (dw_gate_up && !accumulate) e = cudaMemsetAsync(dw_gate_up, 0, 2 * (size_t)I * H * size, (cudaStream_t)stream);
        if (e == cudaSuccess && dw_down && !accumulate) e = cudaMemsetAsync(dw_down, 0, (size_t)H * I * size, (cudaStream_t)stream);
        if (e != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
        return MW_OK;
    }
    Call call = begin(m, stream);
    const int64_t xs = x_stride_bytes ? x_stride_bytes : row, dys = dy_stride_bytes ? dy_stride_bytes : row;
    const auto through_the_gate = [&](auto back) {
        back.gate_up = (const uint8_t *)gate_up; back.d_gate_up = m->d_gate_up; back.h = m->h;
        back.width = I; back.activation = c.activation; back.half = c.dtype == MW_DTYPE_F16;
        return product(call, Job<decltype(back)>{{dy, dys, T, true}, {m->w_down, wide, I, false}, I, H, back});
    };
    e = gate_up_dtype == MW_DTYPE_F32 ? through_the_gate(GateBack<false>()) : through_the_gate(GateBack<true>());
    // The three products that follow need the first one's results and nothing of one another: one launch where that is faster (777 tokens, 1024 wide, 688 deep: the three 26 us one
    // after the other, 15 together).
    Job<Store> jobs[3];
    int count = 0;
    if (dx)
        jobs[count++] = {{m->d_gate_up, 2 * wide, T, true}, {m->w_gate_up, row, H, false}, H, 2 * I,
                         {(uint8_t *)dx, dx_stride_bytes ? dx_stride_bytes : row, c.dtype, 0}};
    if (dw_gate_up) jobs[count++] = {{m->d_gate_up, 2 * wide, 2 * I, false}, {x, xs, H, false}, H, T, {(uint8_t *)dw_gate_up, H * size, dw_dtype, accumulate != 0}};
    if (dw_down) jobs[count++] = {{dy, dys, H, false}, {m->h, wide, I, false}, I, T, {(uint8_t *)dw_down, I * size, dw_dtype, accumulate != 0}};
    // (long sums first, so that the last tiles are short ones)
    if (dx && 2 * I < T)
        for (int i = 0; i + 1 < count; ++i) { const Job<Store> j = jobs[i]; jobs[i] = jobs[i + 1]; jobs[i + 1] = j; }
    call.early = dx && count == 1;
    if (e == cudaSuccess) e = product(call, jobs, count);
    if (e != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
    return MW_OK;
}

int mw_gated_get_status(mw_gated *m, int32_t *status, void *stream)
{
    if (!m || !status) return MW_ERR_INVALID_ARG;
    OnDevice here(m->cfg.device);
    cudaStream_t st = (cudaStream_t)stream;
    if (!here.ok || cudaMemcpyAsync(status, m->status, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(m->status, 0, 4, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) {
        cudaGetLastError();
        return MW_ERR_CUDA;
    }
    return MW_OK;
}

int mw_gated_test_skew_waits(mw_gated *m)
{
    if (!m) return MW_ERR_INVALID_ARG;
    m->skew = 16;
    return MW_OK;
}

int mw_gated_test_ways(const mw_gated *m, mw_dense_way *ways, int32_t *count)
{
    if (!m || !ways || !count) return MW_ERR_INVALID_ARG;
    memcpy(ways, m->ways.list, sizeof m->ways.list);
    *count = m->ways.count;
    return MW_OK;
}

int64_t mw_gated_kernel_launches(const mw_gated *m) { return m ? m->launches : 0; }

}  // extern "C"
