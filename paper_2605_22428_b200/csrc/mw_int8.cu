// Rows in 8-bit integers with a scale each, and products held in them.  Declared in include/mw.h.
//
//   scale = max |x| / 127, q = nearest even integer to x / scale;      y = x_scale w_scale (sum of q w, exact in 32 bits)
//
// The weights lie in 8 bits and are read so: half the bytes of 16 bits where they are the bound (one token, 7168 to 7168: 12.2 us in two launches, 8.0 at the rate of a copy), twice the
// rate where the tensor cores are (4096 tokens: 173 us under the power cap, 149 in runs too short for it, 18.6 of them to quantise).  The row is quantised by a launch of its own: by every block of the product one token took 16.1 us.
#include <new>
#include <string.h>

#include <type_traits>

#include "mw_dense.cuh"

using namespace mw_dense;

struct mw_int8 {
    mw_int8_config cfg;
    const int8_t *w;
    const float *w_scale;
    void *slab;
    int32_t *status;
    int8_t *q;                  // [max_tokens, H]
    float *scale;               // [max_tokens]
    Room room;
    int skew;                   // bytes added to the announced sizes of the next call's loads (test hook)
    int64_t launches;
    Ways ways;
};

namespace {

struct RowArgs {
    const uint8_t *x;
    int64_t x_stride;
    int H, dtype, activation;
    int8_t *q;
    float *scale;
};

// Eight neighbouring entries as they lie: of float32 or 16 bits, with an activation those of gate and up.  (All of a thread's are loaded before any is looked at: each
// by itself, 4096 rows of 7168 took 32 us.)
template <bool WIDE, bool GATED>
struct Piece { uint4 q[(WIDE ? 2 : 1) * (GATED ? 2 : 1)]; };

template <bool WIDE, bool GATED>
__device__ __forceinline__ void load_piece(const uint8_t *row, int H, int i, Piece<WIDE, GATED> &p)
{
    constexpr int kSize = WIDE ? 4 : 2, kVecs = WIDE ? 2 : 1;
#pragma unroll
    for (int g = 0; g < (GATED ? 2 : 1); ++g)
#pragma unroll
        for (int j = 0; j < kVecs; ++j) p.q[g * kVecs + j] = ((const uint4 *)(row + ((int64_t)g * H + i) * kSize))[j];
}
template <bool WIDE>
__device__ __forceinline__ void values_of(const uint4 *q, bool half, float (&v)[8])
{
    const uint32_t w[8] = {q[0].x, q[0].y, q[0].z, q[0].w, q[WIDE].x, q[WIDE].y, q[WIDE].z, q[WIDE].w};
    if (WIDE)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
    else if (half)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = from16((uint16_t)(w[j >> 1] >> (16 * (j & 1))), true);
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = from16((uint16_t)(w[j >> 1] >> (16 * (j & 1))), false);
}
template <bool WIDE, bool GATED>
__device__ __forceinline__ void entries_of(const Piece<WIDE, GATED> &p, const RowArgs &a, float (&v)[8])
{
    values_of<WIDE>(p.q, a.dtype == MW_DTYPE_F16, v);
    if (GATED) {
        float u[8];
        values_of<WIDE>(p.q + (GATED ? (WIDE ? 2 : 1) : 0), a.dtype == MW_DTYPE_F16, u);
        if (a.activation == MW_ACT_GELU)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = activate(v[j], MW_ACT_GELU) * u[j];
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = activate(v[j], MW_ACT_SILU) * u[j];
    }
}

// The integer nearest to x / s, the even one of two.  From an approximate quotient it is the right one or its neighbour; what it leaves, x - q s, is
// exact in float32 (a multiple of half the last place of s that is hardly more than s / 2), so comparing it with s / 2 decides.
__device__ __forceinline__ int nearest(float x, float s, float inverse)
{
    float q = rintf(x * inverse);
    const float rest = fmaf(-q, s, x), twice = 2.0f * fabsf(rest);
    if (twice > s || (twice == s && ((int)q & 1))) q += rest > 0.0f ? 1.0f : -1.0f;
    return (int)fminf(fmaxf(q, -127.0f), 127.0f);
}

// The largest of eight values, as bits: NaN above infinity above numbers.
__device__ __forceinline__ uint32_t largest_of(const float (&v)[8], uint32_t most)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[j]) & 0x7fffffffu);
    return most;
}
// The same of entries as they lie, where they are what is taken to 8 bits: two of 16 bits at a time.
template <bool WIDE>
__device__ __forceinline__ uint32_t largest_of(const Piece<WIDE, false> &p, uint32_t most)
{
#pragma unroll
    for (int j = 0; j < (WIDE ? 2 : 1); ++j) {
        const uint32_t w[4] = {p.q[j].x, p.q[j].y, p.q[j].z, p.q[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) most = WIDE ? max(most, w[i] & 0x7fffffffu) : __vmaxu2(most, w[i] & 0x7fff7fffu);
    }
    return most;
}
struct RowScale {
    float scale;                                // what the caller gets
    float lift, s, inverse;                     // tiny rows times 2^64, which is exact, so that 1 / s is finite and the rests are not denormal
    bool any;
    __device__ __forceinline__ explicit RowScale(uint32_t most)
    {
        const bool finite = most < 0x7f800000u;
        scale = finite ? __fdiv_rn(__uint_as_float(most), 127.0f) : __uint_as_float(0x7fffffffu);
        any = finite && scale > 0.0f;
        lift = scale < 0x1p-60f ? 0x1p64f : 1.0f;
        s = any ? scale * lift : 1.0f;
        inverse = 1.0f / s;
    }
};

// Eight values as integers.  Rounding by adding 1.5 * 2^23 (the integer is then in the last bits) costs two plain operations, where a conversion runs at an eighth of their
// rate; where what is left of one of the eight is not below s / 2, `nearest` decides.  Without `lift` no quotient is above 127 by more than roundings.
__device__ __forceinline__ void store_nearest(int8_t *q, const float (&v)[8], const RowScale &r)
{
    constexpr float kShift = 12582912.0f;
    uint32_t w[8] = {};
    float worst = 0.0f;
    if (r.any && r.lift == 1.0f) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float shifted = fmaf(v[j], r.inverse, kShift);
            worst = fmaxf(worst, fabsf(fmaf(kShift - shifted, r.s, v[j])));
            w[j] = __float_as_uint(shifted);
        }
    }
    if (r.any && (r.lift != 1.0f || worst >= 0.5f * r.s))
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = (uint32_t)nearest(v[j] * r.lift, r.s, r.inverse);
    uint2 out;
    out.x = __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
    out.y = __byte_perm(__byte_perm(w[4], w[5], 0x0040), __byte_perm(w[6], w[7], 0x0040), 0x5410);
    *(uint2 *)q = out;
}

// A block has a row and reads it once: each thread keeps V pieces of eight values while the largest is found (V = 0, rows of more than 16384 values: it reads them a
// second time, from L2).  Bound by HBM for many rows (4096 of 7168 in bf16: 88 MB, 13.6 us at the rate of a copy; 18.6 us,
// 20.6 call after call on other rows; 4096 of 2 x 7168 with an activation 147 MB, 22.7 and 31.4), by latency for few (64: 2.2 us replayed).
template <int V, bool WIDE, bool GATED>
__global__ void __launch_bounds__(V <= 1 ? 1024 : V == 2 ? 1024 : 512) k_quantise(const __grid_constant__ RowArgs a)
{
    __shared__ uint32_t part[32];
    grid_dependency_wait();
    grid_launch_dependents();
    const uint8_t *row = a.x + blockIdx.x * a.x_stride;
    int8_t *q = a.q + blockIdx.x * (int64_t)a.H;
    float v[V ? V : 1][8];
    uint32_t most = 0;
    if (V) {
        Piece<WIDE, GATED> p[V ? V : 1];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int at = (i * blockDim.x + threadIdx.x) * 8;
            load_piece(row, a.H, at < a.H ? at : 0, p[i]);      // (what lies beyond the row is counted as its begin, and not stored)
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            entries_of(p[i], a, v[i]);
            if constexpr (GATED) most = largest_of(v[i], most);
            else most = largest_of(p[i], most);
        }
    } else
        for (int at = threadIdx.x * 8; at < a.H; at += blockDim.x * 8) {
            Piece<WIDE, GATED> p;
            load_piece(row, a.H, at, p);
            if constexpr (GATED) {
                entries_of(p, a, v[0]);
                most = largest_of(v[0], most);
            } else most = largest_of(p, most);
        }
    if (!GATED && !WIDE) most = __float_as_uint(from16((uint16_t)max(most & 0xffffu, most >> 16), a.dtype == MW_DTYPE_F16));
    most = __reduce_max_sync(0xffffffffu, most);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = most;
    __syncthreads();
    most = __reduce_max_sync(0xffffffffu, threadIdx.x % 32 < blockDim.x / 32 ? part[threadIdx.x % 32] : 0);
    const RowScale s(most);
    if (threadIdx.x == 0) a.scale[blockIdx.x] = s.scale;
    if (V)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int at = (i * blockDim.x + threadIdx.x) * 8;
            if (at < a.H) store_nearest(q + at, v[i], s);
        }
    else
        for (int at = threadIdx.x * 8; at < a.H; at += blockDim.x * 8) {
            Piece<WIDE, GATED> p;
            load_piece(row, a.H, at, p);
            entries_of(p, a, v[0]);
            store_nearest(q + at, v[0], s);
        }
}

int check_quantise(const void *x, int dtype, int64_t stride, int H, int activation)
{
    if (dtype != MW_DTYPE_F32 && dtype != MW_DTYPE_BF16 && dtype != MW_DTYPE_F16) return MW_ERR_INVALID_ARG;
    if (activation != MW_ACT_NONE && activation != MW_ACT_SILU && activation != MW_ACT_GELU) return MW_ERR_INVALID_ARG;
    const int64_t row = (int64_t)H * (activation ? 2 : 1) * element_bytes(dtype);
    if (stride < 0 || (stride && stride < row)) return MW_ERR_INVALID_ARG;
    return (((uintptr_t)x | (uint64_t)stride) & 15u) ? MW_ERR_ALIGNMENT : MW_OK;
}

RowArgs row_args(const void *x, int dtype, int64_t stride, int H, int activation, int8_t *q, float *scale)
{
    RowArgs a;
    a.x = (const uint8_t *)x; a.x_stride = stride ? stride : (int64_t)H * (activation ? 2 : 1) * element_bytes(dtype);
    a.H = H; a.dtype = dtype; a.activation = activation; a.q = q; a.scale = scale;
    return a;
}

cudaError_t quantise(const RowArgs &a, int T, cudaStream_t st, bool overlap)
{
    const int H = a.H, dtype = a.dtype, activation = a.activation;
    // Pieces of eight values per thread: one or two where rows are few and their latency counts, four where blocks share SMs.
    const int pieces = H / 8, v = pieces > 2048 ? 0 : T >= 256 && pieces > 256 ? 4 : ceil_div(pieces, 1024);
    const dim3 threads(v ? (ceil_div(pieces, v) + 31) & ~31 : 1024);
    const auto launch = [&](auto wide, auto gated) {
        if (v == 0) return mw_launch(k_quantise<0, wide, gated>, dim3(T), threads, 0, st, overlap, a);
        if (v == 1) return mw_launch(k_quantise<1, wide, gated>, dim3(T), threads, 0, st, overlap, a);
        if (v == 2) return mw_launch(k_quantise<2, wide, gated>, dim3(T), threads, 0, st, overlap, a);
        return mw_launch(k_quantise<4, wide, gated>, dim3(T), threads, 0, st, overlap, a);
    };
    if (dtype == MW_DTYPE_F32) return activation ? launch(std::true_type(), std::true_type()) : launch(std::true_type(), std::false_type());
    return activation ? launch(std::false_type(), std::true_type()) : launch(std::false_type(), std::false_type());
}

template <bool WIDE, bool GATED>
cudaError_t load_quantise_of()
{
    cudaError_t e = load_kernel(k_quantise<0, WIDE, GATED>);
    if (e == cudaSuccess) e = load_kernel(k_quantise<1, WIDE, GATED>);
    if (e == cudaSuccess) e = load_kernel(k_quantise<2, WIDE, GATED>);
    return e == cudaSuccess ? load_kernel(k_quantise<4, WIDE, GATED>) : e;
}
cudaError_t load_quantise()
{
    cudaError_t e = load_quantise_of<false, false>();
    if (e == cudaSuccess) e = load_quantise_of<false, true>();
    if (e == cudaSuccess) e = load_quantise_of<true, false>();
    return e == cudaSuccess ? load_quantise_of<true, true>() : e;
}

inline size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// Whether a kernel on `device` may have this address: the device's own memory, or host memory that is mapped.  (Anything else would be a fault there.)
bool reaches(int device, const void *p)
{
    cudaPointerAttributes a;
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) { cudaGetLastError(); return false; }
    return a.type == cudaMemoryTypeDevice ? a.device == device : a.type != cudaMemoryTypeUnregistered;
}

}  // namespace

extern "C" {

int mw_quantise_rows(const void *x, int32_t x_dtype, int64_t x_stride_bytes, int32_t T, int32_t H, int32_t activation, int8_t *q, float *scale, void *stream)
{
    if (T < 0 || H < 16 || H % 16 || H > MW_INT8_MAX_H) return MW_ERR_INVALID_ARG;
    const int rc = check_quantise(x, x_dtype, x_stride_bytes, H, activation);
    if (rc != MW_OK) return rc;
    if (T == 0) return MW_OK;
    if (!x || !q || !scale) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)q & 15u) || ((uintptr_t)scale & 3u)) return MW_ERR_ALIGNMENT;
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
    if (!reaches(device, x) || !reaches(device, q) || !reaches(device, scale)) return MW_ERR_INVALID_ARG;
    if (quantise(row_args(x, x_dtype, x_stride_bytes, H, activation, q, scale), T, (cudaStream_t)stream, true) != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
    return MW_OK;
}

int mw_int8_create(mw_int8 **out, const mw_int8_config *cfg, const int8_t *w, const float *w_scale)
{
    if (!out) return MW_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || !w || !w_scale) return MW_ERR_INVALID_ARG;
    if (cfg->H < 16 || cfg->H % 16 || cfg->H > MW_INT8_MAX_H || cfg->O < 1 || cfg->O > MW_INT8_MAX_O || cfg->max_tokens < 1 ||
        cfg->max_tokens > MW_INT8_MAX_TOKENS || cfg->device < 0 || (cfg->flags & ~(uint32_t)(MW_FLAG_NO_OVERLAP | MW_FLAG_SHORT_WAITS)))
        return MW_ERR_INVALID_ARG;
    if (((uintptr_t)w & 15u) || ((uintptr_t)w_scale & 3u)) return MW_ERR_ALIGNMENT;
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || cfg->device >= ndev) { cudaGetLastError(); return MW_ERR_CUDA; }
    OnDevice here(cfg->device);
    if (!here.ok) { cudaGetLastError(); return MW_ERR_CUDA; }
    mw_int8 *m = new (std::nothrow) mw_int8();
    if (!m) return MW_ERR_INVALID_ARG;
    m->cfg = *cfg;
    m->w = w; m->w_scale = w_scale;
    const size_t b_q = round256((size_t)cfg->max_tokens * cfg->H), b_scale = round256((size_t)cfg->max_tokens * 4);
    if (cudaMalloc(&m->slab, 256 + b_q + b_scale) != cudaSuccess) { cudaGetLastError(); delete m; return MW_ERR_CUDA; }
    uint8_t *p = (uint8_t *)m->slab;
    m->status = (int32_t *)p; p += 256;
    m->q = (int8_t *)p; p += b_q;
    m->scale = (float *)p;
    if (find_room(&m->room, cfg->device) != cudaSuccess || load_kernels<Scaled>() != cudaSuccess || load_quantise() != cudaSuccess || cudaMemset(m->slab, 0, 256) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
        cudaGetLastError();
        mw_int8_destroy(m);
        return MW_ERR_CUDA;
    }
    *out = m;
    return MW_OK;
}

int mw_int8_destroy(mw_int8 *m)
{
    if (!m) return MW_OK;
    OnDevice here(m->cfg.device);
    cudaDeviceSynchronize();
    const int rc = cudaFree(m->slab) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
    delete m;
    return rc;
}

int mw_int8_forward(mw_int8 *m, const void *x, int32_t x_dtype, int64_t x_stride_bytes, const float *x_scale, int32_t activation, int32_t T, void *y,
                    int32_t y_dtype, int64_t y_stride_bytes, void *stream)
{
    if (!m || T < 0 || T > m->cfg.max_tokens) return MW_ERR_INVALID_ARG;
    const mw_int8_config &c = m->cfg;
    if (y_dtype != MW_DTYPE_F32 && y_dtype != MW_DTYPE_BF16 && y_dtype != MW_DTYPE_F16) return MW_ERR_INVALID_ARG;
    const bool ready = x_dtype == MW_DTYPE_I8;
    if (ready) {
        if (activation != MW_ACT_NONE || x_stride_bytes < 0 || (x_stride_bytes && x_stride_bytes < c.H) || (T && !x_scale)) return MW_ERR_INVALID_ARG;
        if ((((uintptr_t)x | (uint64_t)x_stride_bytes) & 15u) || ((uintptr_t)x_scale & 3u)) return MW_ERR_ALIGNMENT;
    } else {
        if (x_scale) return MW_ERR_INVALID_ARG;
        const int rc = check_quantise(x, x_dtype, x_stride_bytes, c.H, activation);
        if (rc != MW_OK) return rc;
    }
    const int ye = element_bytes(y_dtype);
    const int64_t yrow = (int64_t)c.O * ye;
    if (y_stride_bytes < 0 || (y_stride_bytes && y_stride_bytes < yrow) || (T && (!x || !y))) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)y | (uint64_t)y_stride_bytes) % ye) return MW_ERR_ALIGNMENT;
    if (T == 0) return MW_OK;
    OnDevice here(c.device);
    if (!here.ok) { cudaGetLastError(); return MW_ERR_CUDA; }
    cudaStream_t st = (cudaStream_t)stream;
    const bool overlap = !(c.flags & MW_FLAG_NO_OVERLAP);
    const bool quick = (c.flags & MW_FLAG_SHORT_WAITS) != 0;
    const Call call = {st, overlap, MW_DTYPE_I8, &m->room, {quick ? 1 << 10 : 1 << 20, m->skew, m->status}, !ready, &m->launches, &m->ways};
    m->skew = 0;
    m->ways.count = 0;
    Scaled s;
    s.row_scale = ready ? x_scale : m->scale; s.col_scale = m->w_scale;
    s.out = (uint8_t *)y; s.stride = y_stride_bytes ? y_stride_bytes : yrow; s.dtype = y_dtype;
    s.aligned = !(((uintptr_t)y | (uint64_t)s.stride) & 15u);
    s.eights = s.aligned && y_dtype != MW_DTYPE_F32 && !(m->cfg.O & 7) && !((uintptr_t)m->w_scale & 15u);
    cudaError_t e = cudaSuccess;
    if (!ready) {
        e = quantise(row_args(x, x_dtype, x_stride_bytes, c.H, activation, m->q, m->scale), T, st, overlap);
        m->launches += 1;
    }
    const Operand rows = {ready ? x : m->q, ready && x_stride_bytes ? x_stride_bytes : c.H, T, true}, cols = {m->w, c.H, c.O, true};
    if (e == cudaSuccess) e = product(call, Job<Scaled>{rows, cols, c.O, c.H, s});
    if (e != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
    return MW_OK;
}

int mw_int8_get_status(mw_int8 *m, int32_t *status, void *stream)
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

int mw_int8_test_skew_waits(mw_int8 *m)
{
    if (!m) return MW_ERR_INVALID_ARG;
    m->skew = 16;
    return MW_OK;
}

int mw_int8_test_ways(const mw_int8 *m, mw_dense_way *ways, int32_t *count)
{
    if (!m || !ways || !count) return MW_ERR_INVALID_ARG;
    memcpy(ways, m->ways.list, sizeof m->ways.list);
    *count = m->ways.count;
    return MW_OK;
}

int64_t mw_int8_kernel_launches(const mw_int8 *m) { return m ? m->launches : 0; }

}  // extern "C"
