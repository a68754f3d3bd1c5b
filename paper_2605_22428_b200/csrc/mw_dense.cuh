// The products behind mw_gated and mw_int8: out[r][c] = sum over k of R(r, k) C(c, k) for dense operands, and what becomes of the sums.
#pragma once

#include <math.h>

#include <atomic>

#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mw_stream.cuh"

namespace mw_dense {

using mw_stream::encode_map;

// An operand: `count` indices times `depth` along the sum.  Either a row of memory holds one index (k_major) or one step of the sum.
struct Operand {
    const void *base;
    int64_t stride_bytes;                       // between rows of memory
    int count;
    bool k_major;
};

// The current device for as long as this lives; the one before when it ends.
struct OnDevice {
    int before = -1;
    bool ok;
    explicit OnDevice(int device)
    {
        ok = cudaGetDevice(&before) == cudaSuccess && (before == device || cudaSetDevice(device) == cudaSuccess);
        if (before == device) before = -1;
    }
    ~OnDevice() { if (before >= 0) cudaSetDevice(before); }
    OnDevice(const OnDevice &) = delete;
};

inline int element_bytes(int dtype) { return dtype == MW_DTYPE_F32 ? 4 : dtype == MW_DTYPE_I8 ? 1 : 2; }

#ifdef __CUDACC__

using mw_stream::bar_expect;
using mw_stream::bar_init;
using mw_stream::bar_try;
using mw_stream::elect_one;
using mw_stream::fence_after;
using mw_stream::fence_before;
using mw_stream::prefetch_map;
using mw_stream::read16;
using mw_stream::smem_addr;

// ---- elements ----
__device__ __forceinline__ uint16_t to16(float f, bool half)        // to nearest even
{
    return half ? __half_as_ushort(__float2half_rn(f)) : __bfloat16_as_ushort(__float2bfloat16_rn(f));
}
__device__ __forceinline__ float from16(uint16_t v, bool half)
{
    return half ? __half2float(__ushort_as_half(v)) : __uint_as_float((uint32_t)v << 16);
}

// V neighbouring elements; eight are aligned to 16 bytes, four to four elements.
template <int V>
__device__ __forceinline__ void store32(float *p, const float (&v)[V])
{
    if constexpr (V >= 4)
#pragma unroll
        for (int i = 0; i < V; i += 4) *(float4 *)(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    else
        for (int i = 0; i < V; ++i) p[i] = v[i];
}
template <int V>
__device__ __forceinline__ void load32(const float *p, float (&v)[V])
{
    if constexpr (V >= 4)
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 q = *(const float4 *)(p + i);
            v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
        }
    else
        for (int i = 0; i < V; ++i) v[i] = p[i];
}

// Float32 to 16 bits, two at a time (a conversion at a time, chosen for each, took as long as the activation).
template <bool HALF>
__device__ __forceinline__ uint32_t round_two(float low, float high)
{
    uint32_t w;
    if (HALF) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(high), "f"(low));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(high), "f"(low));
    return w;
}
template <int V>
__device__ __forceinline__ void round_all(const float (&f)[V], uint32_t *w, bool half)
{
    if (half)
#pragma unroll
        for (int i = 0; i < V / 2; ++i) w[i] = round_two<true>(f[2 * i], f[2 * i + 1]);
    else
#pragma unroll
        for (int i = 0; i < V / 2; ++i) w[i] = round_two<false>(f[2 * i], f[2 * i + 1]);
}
template <int V>
__device__ __forceinline__ void store_rounded(uint16_t *p, const float (&f)[V], bool half)
{
    if constexpr (V == 8) {
        uint32_t w[4];
        round_all<8>(f, w, half);
        *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
    } else if constexpr (V == 4) {
        uint32_t w[2];
        round_all<4>(f, w, half);
        *(uint2 *)p = make_uint2(w[0], w[1]);
    } else
        for (int i = 0; i < V; ++i) p[i] = to16(f[i], half);
}

// The activations are g s(k(g)), s the logistic function: k = g (silu), or k = 2 sqrt(2 / pi) (g + 0.044715 g^3) (gelu's tanh form).  s and 1 - s from
// e = exp(-|k|), which neither overflows nor cancels.
constexpr float kGelu = 1.5957691216057308f, kGeluCube = 0.044715f;     // 2 sqrt(2 / pi)
__device__ __forceinline__ float inner(float g, int activation) { return activation == MW_ACT_GELU ? kGelu * (g + kGeluCube * g * g * g) : g; }
__device__ __forceinline__ float activate(float g, int activation)
{
    const float k = inner(g, activation), e = __expf(-fabsf(k)), big = __fdividef(1.0f, 1.0f + e);
    return g * (k < 0.0f ? e * big : big);
}
// act(g), and act'(g) = s + g s (1 - s) k'(g).  k' is kept finite: where s (1 - s) has vanished so has its term.
__device__ __forceinline__ void activate_back(float g, int activation, float &act, float &slope)
{
    const float k = inner(g, activation), e = __expf(-fabsf(k)), big = __fdividef(1.0f, 1.0f + e), small = e * big, s = k < 0.0f ? small : big;
    act = g * s;
    const float t = g * (big * small);
    slope = activation == MW_ACT_GELU ? fmaf(t, fminf(kGelu * fmaf(3.0f * kGeluCube * g, g, 1.0f), 1e30f), s) : s + t;
}

// ---- what becomes of the sums: emit(row, col, valid, a, b, x) takes V neighbouring columns of a row, V = 8, 4 or 1 (eight and four are aligned), of which the first `valid` are
// wanted (all of them, unless kRagged); `b` is the second product's where kPairs; `x` is what fetch(row, col, valid, x) has read for them ahead. ----
struct Nothing {};

// To memory, rounded once, or added to what is there.
struct Store {
    using Acc = float;
    static constexpr int kBytes = 2;            // of an operand's element
    static constexpr float kFinish = 0.0065f, kBusy = 0.0102f;    // us per column of a pair's sums (256 rows): after the last product; where tiles come one after the other
    __host__ __device__ __forceinline__ float busy(int n) const { return rounds() && n >= 128 ? 0.0048f : kBusy; }
    static constexpr bool kDots = true;
    static constexpr bool kPairs = false, kRagged = false;
    static constexpr bool kFours = true, kEights = true;        // of 32 bits four columns of a row are a lane's, else eight: 16 bytes, and neighbouring lanes' side by side
    __device__ __forceinline__ bool fours() const { return dtype == MW_DTYPE_F32; }
    static constexpr int kProblems = 3;
    static constexpr bool kRounds = true;       // nothing but a rounding to 16 bits, where rounds()
    uint8_t *out;
    int64_t stride;                             // bytes
    int dtype, accumulate;
    __host__ __device__ __forceinline__ bool rounds() const { return !accumulate && dtype != MW_DTYPE_F32; }
    __device__ __forceinline__ int64_t row_bytes() const { return stride; }
    using OfRow = Nothing; using OfColumns = Nothing;
    __device__ __forceinline__ void of_row(int, OfRow &) const {}
    __device__ __forceinline__ void of_columns(int, int, OfColumns &) const {}
    __device__ __forceinline__ void round16(const uint32_t (&r)[16], uint32_t *w, const Nothing &, const Nothing &, int) const
    {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
        round_all<16>(v, w, dtype == MW_DTYPE_F16);
    }
    template <int V> struct Extra { uint32_t raw[V]; };     // as it lies, so that nothing waits for it in fetch
    __device__ __forceinline__ uint8_t *at(int64_t row, int col) const { return out + row * stride + (int64_t)col * (dtype == MW_DTYPE_F32 ? 4 : 2); }
    template <int V>
    __device__ __forceinline__ void fetch(int64_t row, int col, int valid, Extra<V> &x) const
    {
        if (!accumulate) return;
        if (V == 4 || dtype == MW_DTYPE_F32) {
            float f[V];
            load32((const float *)at(row, col), f);
#pragma unroll
            for (int i = 0; i < V; ++i) x.raw[i] = __float_as_uint(f[i]);
        }
        else if constexpr (V == 8) {
            const uint4 q = *(const uint4 *)at(row, col);
            x.raw[0] = q.x; x.raw[1] = q.y; x.raw[2] = q.z; x.raw[3] = q.w;
        } else x.raw[0] = *(const uint16_t *)at(row, col);
    }
    template <int V>
    __device__ __forceinline__ void emit(int64_t row, int col, int valid, const float (&a)[V], const float (&)[V], const Extra<V> &x) const
    {
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = a[i];
        if (accumulate)
#pragma unroll
            for (int i = 0; i < V; ++i)
                f[i] += V == 4 || dtype == MW_DTYPE_F32 ? __uint_as_float(x.raw[i]) : from16((uint16_t)(x.raw[i >> 1] >> (16 * (i & 1))), dtype == MW_DTYPE_F16);
        if (V == 4 || dtype == MW_DTYPE_F32) store32((float *)at(row, col), f);
        else store_rounded((uint16_t *)at(row, col), f, dtype == MW_DTYPE_F16);
    }
};

// h = act(g) u, and g and u themselves where they are kept.
struct Gate {
    using Acc = float;
    static constexpr int kBytes = 2;            // of an operand's element
    static constexpr float kFinish = 0.020f, kBusy = 0.0165f;    // us per column of a pair's sums (256 rows): after the last product; where tiles come one after the other
    static constexpr bool kDots = true;
    static constexpr bool kPairs = true, kRagged = false;
    static constexpr bool kFours = true, kEights = false;
    static __device__ __forceinline__ bool fours() { return kFours; }
    static constexpr int kProblems = 1;
    static constexpr bool kRounds = true;       // nothing but h, where rounds()
    static float busy(int) { return kBusy; }    // (0.0085 where g and u are not kept; but y is to have the same bits then, so the choice is the same)
    uint16_t *h;                                // [T, I]
    void *gate_up;                              // [T, 2 I] or null
    int width, activation, half;
    int rounded;                                // gate_up is of the operands' type, else float32
    __device__ __forceinline__ bool rounds() const { return !gate_up; }
    __device__ __forceinline__ uint8_t *at(int64_t row, int col) const { return (uint8_t *)(h + row * width + col); }
    __device__ __forceinline__ int64_t row_bytes() const { return 2 * (int64_t)width; }
    // Sixteen columns' g, then their u.
    using OfRow = Nothing; using OfColumns = Nothing;
    __device__ __forceinline__ void of_row(int, OfRow &) const {}
    __device__ __forceinline__ void of_columns(int, int, OfColumns &) const {}
    __device__ __forceinline__ void round16(const uint32_t (&r)[32], uint32_t *w, const Nothing &, const Nothing &, int) const
    {
        float v[16];
        if (activation == MW_ACT_GELU)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = activate(__uint_as_float(r[i]), MW_ACT_GELU) * __uint_as_float(r[16 + i]);
        else
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = activate(__uint_as_float(r[i]), MW_ACT_SILU) * __uint_as_float(r[16 + i]);
        round_all<16>(v, w, half);
    }
    template <int V> using Extra = Nothing;
    template <int V>
    __device__ __forceinline__ void fetch(int64_t, int, int, Nothing &) const {}
    template <int V>
    __device__ __forceinline__ void emit(int64_t row, int col, int valid, const float (&g)[V], const float (&u)[V], const Nothing &) const
    {
        float v[V];
        if (activation == MW_ACT_GELU)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = activate(g[i], MW_ACT_GELU) * u[i];
        else
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = activate(g[i], MW_ACT_SILU) * u[i];
        store_rounded(h + row * width + col, v, half);
        const int64_t kept = row * 2 * width + col;
        if (gate_up && rounded) {
            store_rounded((uint16_t *)gate_up + kept, g, half);
            store_rounded((uint16_t *)gate_up + kept + width, u, half);
        } else if (gate_up) {
            store32((float *)gate_up + kept, g);
            store32((float *)gate_up + kept + width, u);
        }
    }
};

// From dh: dg, du and, once more, h.  ROUNDED: g and u were kept in the operands' type, else in float32.  (By a run-time branch the pairs' kernel has no room for its registers.)
template <bool ROUNDED>
struct GateBack {
    using Acc = float;
    static constexpr int kBytes = 2;            // of an operand's element
    static constexpr float kFinish = 0.031f, kBusy = 0.055f;    // us per column of a pair's sums (256 rows): after the last product; where tiles come one after the other
    static constexpr bool kDots = false;        // (the weights' rows lie across the sum: no dot products)
    static constexpr bool kPairs = false, kRagged = false;
    static constexpr bool kFours = false, kEights = true;
    static __device__ __forceinline__ bool fours() { return kFours; }
    static constexpr int kProblems = 1;
    static constexpr bool kRounds = false;
    static float busy(int) { return kBusy; }
    const uint8_t *gate_up;                     // [T, 2 I]
    uint16_t *d_gate_up, *h;                    // [T, 2 I], [T, I]
    int width, activation, half;
    template <int V> struct Extra { uint32_t g[ROUNDED ? V / 2 : V], u[ROUNDED ? V / 2 : V]; };     // as they lie, so that nothing waits for them in fetch
    template <int N>
    static __device__ __forceinline__ void load_raw(const uint8_t *p, uint32_t (&raw)[N])
    {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 q = *(const uint4 *)(p + 4 * i);
            raw[i] = q.x; raw[i + 1] = q.y; raw[i + 2] = q.z; raw[i + 3] = q.w;
        }
    }
    template <int V>
    __device__ __forceinline__ void fetch(int64_t row, int col, int valid, Extra<V> &x) const
    {
        constexpr int kSize = ROUNDED ? 2 : 4;
        const uint8_t *kept = gate_up + (row * 2 * width + col) * kSize;
        load_raw(kept, x.g);
        load_raw(kept + (int64_t)width * kSize, x.u);
    }
    template <int V, int N>
    __device__ __forceinline__ void values(const uint32_t (&raw)[N], float (&v)[V]) const
    {
        if (!ROUNDED)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = __uint_as_float(raw[i % N]);
        else if (half)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = from16((uint16_t)(raw[i >> 1] >> (16 * (i & 1))), true);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = from16((uint16_t)(raw[i >> 1] >> (16 * (i & 1))), false);
    }
    template <int V>
    __device__ __forceinline__ void emit(int64_t row, int col, int valid, const float (&dh)[V], const float (&)[V], const Extra<V> &x) const
    {
        const int64_t at = row * 2 * width + col;
        float g[V], u[V], act[V], slope[V];
        values(x.g, g);
        values(x.u, u);
        if (activation == MW_ACT_GELU)
#pragma unroll
            for (int i = 0; i < V; ++i) activate_back(g[i], MW_ACT_GELU, act[i], slope[i]);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) activate_back(g[i], MW_ACT_SILU, act[i], slope[i]);
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act[i] * u[i];
        store_rounded(h + row * width + col, v, half);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = dh[i] * u[i] * slope[i];
        store_rounded(d_gate_up + at, v, half);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = dh[i] * act[i];
        store_rounded(d_gate_up + at + width, v, half);
    }
};

// Integers with a scale per row and per column.
struct Scaled {
    using Acc = int32_t;
    static constexpr int kBytes = 1;
    static constexpr float kFinish = 0.017f, kBusy = 0.0165f;    // us per column of a pair's sums (256 rows): after the last product; where tiles come one after the other
    static constexpr bool kDots = true;
    static constexpr bool kPairs = false, kRagged = true;
    static constexpr bool kFours = true, kEights = false;
    static __device__ __forceinline__ bool fours() { return kFours; }
    static constexpr int kProblems = 1;
    static constexpr bool kRounds = true;       // where rounds()
    float busy(int n) const { return eights && n >= 128 ? 0.007f : aligned ? kBusy : 0.028f; }
    const float *row_scale, *col_scale;
    uint8_t *out;
    int64_t stride;                             // bytes
    int dtype, aligned;                         // rows begin on 16 bytes
    int eights;                                 // besides, the type has 16 bits, columns come in eights and their scales begin on 16 bytes
    __device__ __forceinline__ bool rounds() const { return eights; }
    __device__ __forceinline__ uint8_t *at(int64_t row, int col) const { return out + row * stride + (int64_t)col * 2; }
    __device__ __forceinline__ int64_t row_bytes() const { return stride; }
    struct OfRow { float r; };
    struct OfColumns { float c[32]; };
    __device__ __forceinline__ void of_row(int row, OfRow &x) const { x.r = row_scale[row]; }
    __device__ __forceinline__ void of_columns(int col, int end, OfColumns &x) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 q = col + 4 * i < end ? *(const float4 *)(col_scale + col + 4 * i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            x.c[4 * i] = q.x; x.c[4 * i + 1] = q.y; x.c[4 * i + 2] = q.z; x.c[4 * i + 3] = q.w;
        }
    }
    __device__ __forceinline__ void round16(const uint32_t (&a)[16], uint32_t *w, const OfRow &row, const OfColumns &x, int from) const
    {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = (float)(int32_t)a[i] * row.r * x.c[from + i];
        round_all<16>(v, w, dtype == MW_DTYPE_F16);
    }
    template <int V> struct Extra { float r, c[V]; };
    template <int V>
    __device__ __forceinline__ void fetch(int64_t row, int col, int valid, Extra<V> &x) const
    {
        x.r = row_scale[row];
#pragma unroll
        for (int i = 0; i < V; ++i) x.c[i] = col_scale[col + (i < valid ? i : 0)];
    }
    template <int V>
    __device__ __forceinline__ void emit(int64_t row, int col, int valid, const int32_t (&a)[V], const int32_t (&)[V], const Extra<V> &x) const
    {
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)a[i] * x.r * x.c[i];
        uint8_t *p = out + row * stride + (int64_t)col * (dtype == MW_DTYPE_F32 ? 4 : 2);
        if ((aligned || V == 1) && valid == V) {
            if (dtype == MW_DTYPE_F32) store32((float *)p, f);
            else store_rounded((uint16_t *)p, f, dtype == MW_DTYPE_F16);
        } else
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < valid) {
                    if (dtype == MW_DTYPE_F32) ((float *)p)[i] = f[i];
                    else ((uint16_t *)p)[i] = to16(f[i], dtype == MW_DTYPE_F16);
                }
    }
};

// ---- shared memory, barriers, products ----
constexpr int kLine = 128;                      // bytes of the sum's axis per step: 64 elements of 16 bits, 128 of 8
constexpr int kLanes = 128;                     // rows of an operand per CTA
constexpr uint32_t kTileBytes = kLanes * kLine;
constexpr int kMaxStages = 8;
constexpr int kMaxCols = 256;                   // columns of an accumulator

struct Waits {
    int limit, skew;
    int32_t *status;
};

struct Bars {
    uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], drained;
    uint32_t tmem, issued;
    volatile uint32_t peer_issued, peer_abort;  // pairs: the other CTA's, at the end
    volatile uint32_t abort;
};

// Waits for the phase of the given parity; false when the wait gave up, here or elsewhere in the CTA.
__device__ __forceinline__ bool wait_for(uint64_t *bar, uint32_t parity, Bars *s, const Waits &w)
{
#pragma unroll 1
    for (int i = 0; i < w.limit; ++i) {
        if (bar_try(bar, parity)) return true;
        if (s->abort) return false;
    }
    s->abort = 1;
    atomicExch(w.status, MW_ERR_TIMEOUT);
    return false;
}
// A place in the ring of stages, and whether its barrier was found ready.  It is asked for a step ahead: an answer takes 200 clocks, which with that of the step itself is
// more than a step of products takes.
struct Place {
    uint32_t slot = 0, round = 0, ready = 0;
    __device__ __forceinline__ void step(uint32_t stages) { if (++slot == stages) { slot = 0; round ^= 1; } }
    __device__ __forceinline__ void ask(uint64_t *bars, uint32_t flip) { ready = bar_try(&bars[slot], round ^ flip); }
    __device__ __forceinline__ bool wait(uint64_t *bars, uint32_t flip, Bars *s, const Waits &w) const { return ready || wait_for(&bars[slot], round ^ flip, s, w); }
};
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, Bars *s, const Waits &w) { return __all_sync(0xffffffffu, wait_for(bar, parity, s, w)); }

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// The address of a place in shared memory in another CTA of the cluster.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
// (without order for memory, which costs a microsecond: after barriers were made and fenced, or where only time counts)
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void arrive_at(uint32_t addr) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory"); }
__device__ __forceinline__ void expect_at(uint32_t addr, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(addr), "r"(bytes) : "memory");
}

__device__ __forceinline__ void put_at(uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }

// A box of a tensor to this CTA's memory, reported to a barrier of the pair (GROUP 2) or of this CTA.
template <int GROUP, int RANK>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2 = 0)
{
    if constexpr (GROUP == 2 && RANK == 2)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
    else if constexpr (GROUP == 2)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
    else if constexpr (RANK == 2)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}

// Descriptor of an operand in shared memory, 128-byte lines swizzled in groups of eight as TMA stores them: address / 16, leading distance / 16 in bits
// 16..29, stride distance / 16 in bits 32..45, version 1 in bit 46, 128-byte swizzle in bits 61..63.  K-major: a line is one index, groups of eight indices are 1024
// bytes apart.  Else a line is 64 indices of one k, groups of eight k are 1024 bytes apart, the next 64 indices kBlock.
constexpr uint32_t kBlock = 64 * kLine;
// (An address of a CTA of a cluster has the CTA's number in its upper bits, which do not belong here.)
__device__ __forceinline__ uint64_t place_of(uint32_t addr) { return (addr & 0x3ffffu) >> 4; }
__device__ __forceinline__ uint64_t describe(int k_major)
{
    return ((uint64_t)(k_major ? 1 : kBlock >> 4) << 16) | ((1024ull >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// 32 bytes of a line along the sum, or 16 lines of it, / 16.
__device__ __forceinline__ uint32_t advance(int k_major) { return k_major ? 2 : 16 * kLine >> 4; }

// A product as the kernels take it.  A launch has up to E::kProblems of them, one's tiles after the other's: products that wait for the same results and for nothing of one
// another then have one start, and one last round of tiles.
template <class E>
struct Problem {
    CUtensorMap map_r, map_c;
    int rows, cols, steps;
    int row_tiles, col_tiles, first;            // `first`: its first tile among those of the launch
    int tile_rows, n;                           // clusters: rows of the output per tile; the same rounded up to 16
    int r_k, c_k;                               // operands are K-major
    uint32_t idesc, bytes;                      // bytes that a step's loads of a CTA bring
    uint32_t idesc_cut, bytes_cut;              // pairs: of a tile that is cut in two
    E e;
};
template <class E>
__device__ __forceinline__ const Problem<E> &problem_of(const Problem<E> (&p)[E::kProblems], int count, int tile)
{
    if constexpr (E::kProblems == 1) return p[0];
    int i = 0;
    while (i + 1 < count && tile >= p[i + 1].first) ++i;
    return p[i];
}

template <int GROUP, int BYTES>
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    if constexpr (GROUP == 2 && BYTES == 2)
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
    else if constexpr (GROUP == 2)
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
    else if constexpr (BYTES == 2)
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// Products so far done: an arrival at `bar`, with BOTH at that of both CTAs.
template <int GROUP, bool BOTH = GROUP == 2>
__device__ __forceinline__ void commit(uint64_t *bar)
{
    if constexpr (GROUP == 2 && !BOTH)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
    else if constexpr (GROUP == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// Instruction: float32 sums of bf16 or fp16, or 32-bit sums of signed 8-bit integers; operands that are not K-major; M and N.
inline uint32_t instruction(int dtype, bool a_k, bool b_k, int m, int n)
{
    const uint32_t sum = dtype == MW_DTYPE_I8 ? 2 : 1, type = dtype == MW_DTYPE_F16 ? 0 : 1;
    return sum << 4 | type << 7 | type << 10 | (a_k ? 0u : 1u << 15) | (b_k ? 0u : 1u << 16) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

// 16 columns of the thread's TMEM lane, or 16 and 16 (without the wait).
__device__ __forceinline__ void read16_16(uint32_t a, uint32_t b, uint32_t (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(a));
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(b));
}
__device__ __forceinline__ void read16_raw(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
// (The values go through it, so that nothing uses them before.)
template <int N>
__device__ __forceinline__ void read_done(uint32_t (&r)[N])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                   "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
    if constexpr (N == 32)
        asm volatile("" : "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                          "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void as_sum(uint32_t r, float &v) { v = __uint_as_float(r); }
__device__ __forceinline__ void as_sum(uint32_t r, int32_t &v) { v = (int32_t)r; }

// Eight columns from `col` on, of which those below `end` count: how many.
template <class E, int V>
__device__ __forceinline__ int valid_of(int col, int end)
{
    if (!E::kRagged) return col < end ? V : 0;
    const int left = end - col;
    return left < 0 ? 0 : left < V ? left : V;
}

// After a wait gave up, when all roles have ended, one thread of the CTA that owns the barriers: waits (bounded) for the loads in flight, before the memory goes to another
// kernel.  Each of `parties` (1 or 2) has arrived at the barriers of its first issued[i] stages; what one of them has not asked for is arrived at in its place.
__device__ __forceinline__ void let_loads_land(Bars *s, int stages, const uint32_t *issued, int parties, const Waits &w)
{
    uint32_t end = 0;
    for (int i = 0; i < parties; ++i) end = max(end, issued[i]);
    int polls = 0;
#pragma unroll 1
    for (uint32_t n = end > (uint32_t)stages ? end - stages : 0; n < end; ++n) {
        uint64_t *full = &s->full[n % stages];
        for (int i = 0; i < parties; ++i)
            if (n >= issued[i]) arrive_at(smem_addr(full));
        while (polls < w.limit && !bar_try(full, (n / stages) & 1)) ++polls;
    }
}

// A warp's sums of 32 rows pass through shared memory, from a row per lane to four (or, rounded, eight) neighbouring columns per lane, so that a row's columns leave the SM together (from a row per
// lane, 16 bytes each, an epilogue took twice as long and slowed the loads under it).  Lines of N x 16 bytes, a row's pieces swapped by its number: no two lanes
// meet in a bank.
template <int N>
__device__ __forceinline__ int piece_at(int row, int piece) { return N == 8 ? row * 8 + (piece ^ ((row & 1) << 2 | (row >> 1 & 3))) : row * 4 + (piece ^ (row >> 1 & 3)); }
template <int N>
__device__ __forceinline__ void put_row(float4 *buf, int lane, const uint32_t (&r)[4 * N])
{
#pragma unroll
    for (int j = 0; j < N; ++j)
        buf[piece_at<N>(lane, j)] = make_float4(__uint_as_float(r[4 * j]), __uint_as_float(r[4 * j + 1]), __uint_as_float(r[4 * j + 2]), __uint_as_float(r[4 * j + 3]));
}
template <int N, int V, class Acc>
__device__ __forceinline__ void get_columns(const float4 *buf, int row, int piece, Acc (&v)[V])
{
#pragma unroll
    for (int h = 0; h < V / 4; ++h) {
        const float4 q = buf[piece_at<N>(row, piece + h)];
        as_sum(__float_as_uint(q.x), v[4 * h]); as_sum(__float_as_uint(q.y), v[4 * h + 1]);
        as_sum(__float_as_uint(q.z), v[4 * h + 2]); as_sum(__float_as_uint(q.w), v[4 * h + 3]);
    }
}

// ---- many rows: pairs of CTAs on one tile ----
// A tile is 256 rows times up to 256 columns: each CTA of a pair loads its 128 rows and half of the columns, one thread of the first issues
// tcgen05.mma for both (cta_group::2), each CTA's TMEM holds its 128 rows of the sums, in two buffers, so that one tile's epilogue runs under the next one's
// products.  Pairs are persistent and take tiles in turn, in blocks of kBand row tiles so that what runs at a time shares operands in L2.
// Bound by the tensor cores: 256 x 256 is the largest tile whose sums fit TMEM twice, and at 64 bytes per clock and SM about what L2 feeds.  4096 rows, caches cold: 7168 to 2 x 2048
// with the activation 159 us (1.51 PFLOP/s), 2048 to 7168 82 us (1.46), the gradients of x and all weights together 388 us (1.55), 8 bits 7168 to 7168 124 us (3.4 POP/s).
// Where at most half of the pairs would have a tile in the last round, these tiles are cut in two (half the columns each; 4096 rows, 7168 to 2 x 2048: 256 tiles for 74 pairs,
// 168 us whole, 158 us so).
// With two products (E::kPairs) the first CTA loads the first one's columns, the second the second's: a thread then holds both sums of an output.
// Warps 0 ... kWarps - 1 finish tiles, the next loads, the one after issues products.  Finishing a tile is a chain of latencies, so sixteen warps take it where one has a single
// product's 16 columns at a time (eight of 32 columns took 30.6 us against 25.2 for 4086 rows of 8 bits, 560 to 1462, and 99 against 89 for the training step of 64 tokens, 7168
// and 2048; where the products take longer than the finishing it is the same).  Sums that are only rounded (E::kRounds) are rounded before they are turned: half the shared memory,
// 64 bytes of a row at a time instead of 32 (both gradients of the weights from 64 tokens 24.7 us instead of 37; gate and up of 2000 rows, 512 to 2 x 8192, 27.8 instead of 36.4).  What
// leaves in 32 bits does so with four columns in a lane, so that a store's 16 bytes lie beside the next lane's (eight columns, two stores: half of every 32 bytes at a time; gate and up of 1000 rows,
// 512 to 2 x 8000, g and u kept, 34.9 us against 27.9).
template <class E>
constexpr int kWarps = E::kPairs ? 8 : 16;
template <class E>
constexpr int kPairThreads = (kWarps<E> + 2) * 32;
template <class E>
constexpr int kWholeTurn = kWarps<E> / 4 * 32;   // columns that the warps finish at a time where a row's are rounded before they leave its lane
constexpr int kBand = 8;
constexpr uint32_t kTurnBytes = 32 * 1024;      // of all warps' sums on their way from a row per lane to four or eight columns per lane
constexpr uint32_t kPairRing = 6 * 2 * kTileBytes;                  // of the stages: six of 256 columns, eight of 128
constexpr size_t kPairSmem = 1024 + kPairRing + kTurnBytes + sizeof(Bars);

template <class E>
struct PairArgs {
    Problem<E> p[E::kProblems];
    int count, tiles, whole;                    // tiles, of which the first `whole` are, and the others halves
    int tile_cols, n;                           // columns of the output per tile; of the accumulator
    int box;                                    // K-major columns per load
    uint32_t stages, stage_bytes;
    Waits w;
};

// Tile t of the launch: its product, first row and first column, and by how many bits it is narrower than `tile_cols`.
template <class E>
__device__ __forceinline__ const Problem<E> &tile_at(const PairArgs<E> &a, int t, int &row, int &col, int &cut)
{
    cut = t >= a.whole;
    const int part = cut ? (t - a.whole) & 1 : 0;
    if (cut) t = a.whole + ((t - a.whole) >> 1);
    const Problem<E> &p = problem_of<E>(a.p, a.count, t);
    const int row_tiles = p.row_tiles, col_tiles = p.col_tiles;
    t -= p.first;
    const int band = t / (kBand * col_tiles), first = band * kBand, height = min(row_tiles - first, kBand), in = t - first * col_tiles;
    row = (first + in % height) * 2 * kLanes;
    col = in / height * a.tile_cols + part * (a.tile_cols >> 1);
    return p;
}

template <class E>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads<E>, 1) k_pair(const __grid_constant__ PairArgs<E> a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Bars *s = (Bars *)(smem + kPairRing + kTurnBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    constexpr int kLoads = kWarps<E>, kProducts = kWarps<E> + 1;
    if (warp == kLoads && elect_one())
        for (int i = 0; i < a.count; ++i) { prefetch_map(&a.p[i].map_r); prefetch_map(&a.p[i].map_c); }
    if (threadIdx.x == 0) {
        for (int i = 0; i < kMaxStages; ++i) { bar_init(&s->full[i], 2); bar_init(&s->empty[i], 1); }
        for (int i = 0; i < 2; ++i) { bar_init(&s->acc_full[i], 1); bar_init(&s->acc_empty[i], 2 * kWarps<E>); }
        bar_init(&s->drained, 1);
        s->abort = 0;
        s->peer_abort = 0;
        s->issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kProducts) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s->tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        fence_before();
    }
    __syncthreads();
    cluster_arrive_relaxed();
    cluster_wait();
    fence_after();
    grid_dependency_wait();
    grid_launch_dependents();
    const uint32_t tmem = s->tmem;
    const int tiles = a.tiles, pairs = gridDim.x >> 1, first = blockIdx.x >> 1;

    if (warp == kLoads) {
        // ---- loads ----
        constexpr int kStep = kLine / E::kBytes;
        // (one thread goes through all of it: with a warp that waits and elects anew, a step took 600 clocks)
        if (elect_one()) {
            Place at;
            uint32_t issued = 0;
            bool ok = true;
            at.ask(s->empty, 1);
#pragma unroll 1
            for (int t = first; ok && t < tiles; t += pairs) {
                int row, col, cut;
                const Problem<E> &p = tile_at(a, t, row, col, cut);
                const int half = a.n >> (1 + cut);
                row += (int)rank * kLanes;
                col += E::kPairs ? 0 : (int)rank * half;
                const uint32_t bytes = cut ? p.bytes_cut : p.bytes;
#pragma unroll 1
                for (int k = 0; k < p.steps; ++k) {
                    ok = at.wait(s->empty, 1, s, a.w);
                    if (!ok) break;
                    const uint32_t bar = in_cta(smem_addr(&s->full[at.slot]), 0), dst = smem_addr(smem) + at.slot * a.stage_bytes;
                    at.step(a.stages);
                    at.ask(s->empty, 1);
                    expect_at(bar, bytes + (rank == 0 ? a.w.skew : 0));
                    if (p.r_k) load_box<2, 2>(dst, &p.map_r, bar, k * kStep, row);
                    else {
                        load_box<2, 2>(dst, &p.map_r, bar, row, k * kStep);
                        load_box<2, 2>(dst + kBlock, &p.map_r, bar, row + 64, k * kStep);
                    }
                    const uint32_t cols = dst + kTileBytes;
                    if (E::kPairs) {
                        load_box<2, 3>(cols, &p.map_c, bar, k * kStep, col, (int)rank);
                        if (half > a.box) load_box<2, 3>(cols + kBlock, &p.map_c, bar, k * kStep, col + 64, (int)rank);
                    } else if (p.c_k) {
                        load_box<2, 2>(cols, &p.map_c, bar, k * kStep, col);
                        if (half > a.box) load_box<2, 2>(cols + kBlock, &p.map_c, bar, k * kStep, col + 64);
                    } else {
                        load_box<2, 2>(cols, &p.map_c, bar, col, k * kStep);
                        if (half > 64) load_box<2, 2>(cols + kBlock, &p.map_c, bar, col + 64, k * kStep);
                    }
                    ++issued;
                }
            }
            s->issued = issued;
            // the products' last arrivals come before this CTA may end
            for (uint32_t i = 0; ok && i < a.stages; ++i) {
                ok = at.wait(s->empty, 1, s, a.w);
                at.step(a.stages);
                at.ready = 0;
            }
        }
        __syncwarp();
    } else if (warp == kProducts) {
        // ---- products ----
        if (rank == 0 && elect_one()) {
            Place at;
            int seq = 0;
            bool ok = true;
            at.ask(s->full, 0);
#pragma unroll 1
            for (int t = first; ok && t < tiles; t += pairs, ++seq) {
                int row, col, cut;
                const Problem<E> &p = tile_at(a, t, row, col, cut);
                const int buf = seq & 1, steps = p.steps;
                const uint32_t idesc = cut ? p.idesc_cut : p.idesc, by_r = advance(p.r_k), by_c = advance(p.c_k);
                const uint64_t of_r = describe(p.r_k), of_c = describe(p.c_k);
                if (seq >= 2) ok = wait_for(&s->acc_empty[buf], ((seq >> 1) - 1) & 1, s, a.w);
                if (!ok) break;
                fence_after();
                const uint32_t d = tmem + buf * kMaxCols;
#pragma unroll 1
                for (int k = 0; k < steps; ++k) {
                    ok = at.wait(s->full, 0, s, a.w);
                    if (!ok) break;
                    const uint32_t src = smem_addr(smem) + at.slot * a.stage_bytes;
                    const uint64_t dr = of_r | place_of(src), dc = of_c | place_of(src + kTileBytes);
                    uint64_t *const empty = &s->empty[at.slot];
                    at.step(a.stages);
                    at.ask(s->full, 0);
                    fence_after();
#pragma unroll
                    for (int i = 0; i < 4; ++i) multiply<2, E::kBytes>(d, dr + i * by_r, dc + i * by_c, idesc, k > 0 || i > 0);
                    commit<2>(empty);
                }
                if (ok) commit<2>(&s->acc_full[buf]);
            }
            if (!ok) {                          // products in flight end before their operands go away (bounded)
                commit<2, false>(&s->drained);
                for (int n = 0; n < a.w.limit && !bar_try(&s->drained, 0); ++n) {}
            }
        }
        __syncwarp();
    } else {
        // ---- epilogue ----
        // groups of four warps take turns at the columns
        using Acc = typename E::Acc;
        constexpr int kPieces = E::kPairs ? 8 : 4;
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
        float4 *turned = (float4 *)(smem + kPairRing + warp * (kTurnBytes / kWarps<E>));
        int seq = 0;
#pragma unroll 1
        for (int t = first; t < tiles; t += pairs, ++seq) {
            const int buf = seq & 1;
            int top, col, cut;
            const Problem<E> &p = tile_at(a, t, top, col, cut);
            top += (int)rank * kLanes + (warp & 3) * 32;        // the warp's 32 rows
            const int tile_cols = a.tile_cols >> cut, end = min(p.cols, col + tile_cols);
            const auto sums_there = [&] {
                if (!warp_wait(&s->acc_full[buf], (seq >> 1) & 1, s, a.w)) return false;
                fence_after();
                return true;
            };
            const auto sums_read = [&] {
                fence_before();
                __syncwarp();
                if (lane == 0) arrive_at(in_cta(smem_addr(&s->acc_empty[buf]), 0));
            };
            // 16 columns (with two products 16 of each) at a time: a lane then has V columns of every 2 V-th row
            const auto finish = [&](auto width) {
                constexpr int V = decltype(width)::value, kStep = 2 * V, kTurn = kWarps<E> / 4 * 16;
                const int in = lane / (16 / V), piece = lane % (16 / V) * (V / 4), row = top + in;
                int at = col + (warp >> 2) * 16 + piece * 4, valid = valid_of<E, V>(at, end);
                typename E::template Extra<V> x[32 / kStep];        // read a turn ahead
#pragma unroll
                for (int j = 0; j < 32 / kStep; ++j)
                    if (row + kStep * j < p.rows && valid > 0) p.e.template fetch<V>(row + kStep * j, at, valid, x[j]);
                if (!sums_there()) return false;
#pragma unroll 1
                for (int c = (warp >> 2) * 16; c < tile_cols; c += kTurn) {
                    uint32_t r[4 * kPieces];
                    const uint32_t from = lanes + buf * kMaxCols + c;
                    if constexpr (E::kPairs) read16_16(from, from + tile_cols, r);
                    else read16_raw(from, r);
                    read_done(r);
                    put_row<kPieces>(turned, lane, r);
                    if (c + kTurn >= tile_cols) sums_read();
                    __syncwarp();
                    if constexpr (E::kRagged)
                        if (!p.e.aligned) {         // a column per lane, two rows at a time: a row's 16 leave together, whatever they are aligned to
                            const int mine = col + c + (lane & 15), odd = lane >> 4;
                            typename E::template Extra<1> one;
                            if (mine < end) one.c[0] = p.e.col_scale[mine];
                            const float scale_of_lane = top + lane < p.rows ? p.e.row_scale[top + lane] : 0.0f;
#pragma unroll 4
                            for (int j = 0; j < 32; j += 2) {
                                one.r = __shfl_sync(0xffffffffu, scale_of_lane, j + odd);
                                const Acc v[1] = {((const Acc *)turned)[piece_at<kPieces>(j + odd, (lane & 15) >> 2) * 4 + (lane & 3)]};
                                if (mine < end && top + j + odd < p.rows) p.e.template emit<1>(top + j + odd, mine, 1, v, v, one);
                            }
                            __syncwarp();
                            continue;
                        }
                    const int to = at + kTurn, there = valid_of<E, V>(to, end);
#pragma unroll
                    for (int j = 0; j < 32 / kStep; ++j) {
                        Acc v[V], u[V];
                        get_columns<kPieces>(turned, in + kStep * j, piece, v);
                        if (E::kPairs) get_columns<kPieces>(turned, in + kStep * j, piece + 4, u);
                        if constexpr (E::kFours && E::kEights) __builtin_assume(p.e.fours() == (V == 4));
                        if (row + kStep * j < p.rows && valid > 0) p.e.template emit<V>(row + kStep * j, at, valid, v, u, x[j]);
                        if (row + kStep * j < p.rows && there > 0) p.e.template fetch<V>(row + kStep * j, to, there, x[j]);
                    }
                    at = to;
                    valid = there;
                    __syncwarp();
                }
                return true;
            };
            bool rounds = false, done = true;
            if constexpr (E::kRounds) {
                rounds = p.e.rounds() && tile_cols >= kWholeTurn<E>;
                if (rounds) {
                    // 32 columns at a time, rounded before they are turned: a lane then has eight columns of every eighth row
                    const int row = top + (lane >> 2), mine = top + lane;
                    int c = (warp >> 2) * 32, left = end - (col + c + (lane & 3) * 8);
                    done = sums_there();
                    uint8_t *to = p.e.at(row, col + c + (lane & 3) * 8);
                    const int64_t pitch = p.e.row_bytes();
                    typename E::OfRow of_row;
                    if (mine < p.rows) p.e.of_row(mine, of_row);
#pragma unroll 1
                    for (; done && c < tile_cols; c += kWholeTurn<E>) {
                        uint32_t r[2][4 * kPieces], w[16];
                        typename E::OfColumns of_columns;
                        p.e.of_columns(col + c, end, of_columns);
                        const uint32_t from = lanes + buf * kMaxCols + c;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            if constexpr (E::kPairs) read16_16(from + 16 * i, from + 16 * i + tile_cols, r[i]);
                            else read16_raw(from + 16 * i, r[i]);
                        }
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            read_done(r[i]);
                            p.e.round16(r[i], w + 8 * i, of_row, of_columns, 16 * i);
                        }
                        put_row<4>(turned, lane, w);
                        if (c + kWholeTurn<E> >= tile_cols) sums_read();
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 32; j += 8)
                            if (left > 0 && row + j < p.rows) *(float4 *)(to + j * pitch) = turned[piece_at<4>((lane >> 2) + j, lane & 3)];
                        to += kWholeTurn<E> * 2;
                        left -= kWholeTurn<E>;
                        __syncwarp();
                    }
                }
            }
            if constexpr (E::kFours)
                if (!rounds && p.e.fours()) done = finish(std::integral_constant<int, 4>());
            if constexpr (E::kEights)
                if (!rounds && !p.e.fours()) done = finish(std::integral_constant<int, 8>());
            if (!done) break;
        }
    }
    fence_before();
    __syncthreads();
    // (the other CTA is told of a wait that gave up, if one did: an arrival that orders memory, which waits for all stores, is kept for that)
    if (s->abort && threadIdx.x == 0) {
        put_at(in_cta(smem_addr((void *)&s->peer_abort), rank ^ 1), 1);
        asm volatile("fence.acq_rel.cluster;" ::: "memory");
    }
    __syncwarp();
    cluster_arrive_relaxed();
    cluster_wait();
    if (s->abort || s->peer_abort) {            // (both CTAs see the same; else all that was loaded has been used)
        if (threadIdx.x == 0) put_at(in_cta(smem_addr((void *)&s->peer_issued), rank ^ 1), s->issued);
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (rank == 0 && threadIdx.x == 0) {
            const uint32_t issued[2] = {s->issued, s->peer_issued};
            let_loads_land(s, a.stages, issued, 2, a.w);
        }
        __syncthreads();
        cluster_arrive();
        cluster_wait();
    }
    if (warp == kProducts) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// ---- few rows: clusters of CTAs along the sum ----
// A CTA has 128 columns of the output (weights, the M operand) and up to 256 rows (tokens, the N operand), and a piece of the sum; the CTAs of a cluster have the
// same tile.  Each CTA finishes some of the tile's rows: the others copy their parts of these into its shared memory, and it adds them up in the order of the pieces.  So
// the cluster is the only thing that waits, and the bits do not depend on timing.  With two products a CTA has 64 columns of each.
// Bound by HBM while it streams (6.9 TB/s), else by its start and end: 64 rows, 7168 to 2 x 2048 15.5 us (58.7 MB of weights, 9.1 us), 2048 to 7168 11 us (29.4 MB, 4.5 us).
constexpr int kSplitThreads = 256;              // warp 4: loads, 5: products; all: accumulators and the parts' sum
constexpr uint32_t kRowBytes = kLanes * 4;      // of a row of sums
constexpr int kMaxSplit = 8;

template <class E>
struct SplitArgs {
    Problem<E> p[E::kProblems];
    int count, stages;
    uint32_t stage_bytes, tmem_cols;
    uint32_t parts_at;                          // where in shared memory the others' parts go (a CTA's own are at its begin, over its stages)
    int apart;                                  // that is behind the stages; else over them too, and nobody copies before all CTAs' products are done
    int early;                                  // the columns' operand of the first product is not written by the kernel before: its first loads go ahead of the wait for it
    Waits w;
};

template <class E>
__global__ void __launch_bounds__(kSplitThreads) k_split(const __grid_constant__ SplitArgs<E> a)
{
    using Acc = typename E::Acc;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ Bars bars;
    Bars *s = &bars;
    const int warp = threadIdx.x >> 5;
    const int pieces = gridDim.x, piece = blockIdx.x;                      // (a cluster is a row of the grid)
    const Problem<E> &p = problem_of<E>(a.p, a.count, blockIdx.y);
    constexpr int kTileCols = E::kPairs ? kLanes / 2 : kLanes;
    const int tile = blockIdx.y - p.first, col = tile % p.col_tiles * kTileCols, row = tile / p.col_tiles * p.tile_rows;
    const int k0 = (int)((int64_t)p.steps * piece / pieces), k1 = (int)((int64_t)p.steps * (piece + 1) / pieces);
    const int n = min(p.rows - row, p.tile_rows), share = (n + pieces - 1) / pieces;      // rows; of each CTA
    const int mine = max(min(n - piece * share, share), 0);
    uint64_t *const parts_full = &s->acc_full[1];
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s->tmem)), "r"(a.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    constexpr int kStep = kLine / E::kBytes;

    if (warp == 4) {
        if (elect_one()) {
            prefetch_map(&p.map_c);
            prefetch_map(&p.map_r);
            for (int i = 0; i < kMaxStages; ++i) { bar_init(&s->full[i], 1); bar_init(&s->empty[i], 1); }
            bar_init(&s->acc_full[0], 1);
            bar_init(parts_full, 1);
            s->abort = 0;
            s->issued = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            bar_expect(parts_full, (pieces - 1) * mine * kRowBytes);
        }
        __syncwarp();
        const uint32_t bytes = p.bytes + a.w.skew;
        const auto load_cols = [&](int k, uint32_t at, uint32_t bar) {
            if (E::kPairs) {
                load_box<1, 3>(at, &p.map_c, bar, k * kStep, col, 0);
                load_box<1, 3>(at + kTileBytes / 2, &p.map_c, bar, k * kStep, col, 1);
            } else if (p.c_k) load_box<1, 2>(at, &p.map_c, bar, k * kStep, col);
            else {
                load_box<1, 2>(at, &p.map_c, bar, col, k * kStep);
                load_box<1, 2>(at + kBlock, &p.map_c, bar, col + 64, k * kStep);
            }
        };
        const auto load_rows = [&](int k, uint32_t at, uint32_t bar) {
            if (p.r_k) load_box<1, 2>(at, &p.map_r, bar, k * kStep, row);
            else
                for (int i = 0; i < p.n; i += 64) load_box<1, 2>(at + i / 64 * kBlock, &p.map_r, bar, row + i, k * kStep);
        };
        const uint32_t base = smem_addr(smem);
        const int ahead = a.early && p.first == 0 ? min(a.stages, k1 - k0) : 0;
        if (elect_one())
            for (int i = 0; i < ahead; ++i) {
                const uint32_t bar = smem_addr(&s->full[i]);
                bar_expect(&s->full[i], bytes);
                load_cols(k0 + i, base + i * a.stage_bytes, bar);
            }
        __syncwarp();
        __syncthreads();
        cluster_arrive_relaxed();               // (this CTA's barriers are there)
        grid_dependency_wait();
        if (elect_one()) {
            Place at;
            uint32_t issued = ahead;
            at.ask(s->empty, 1);
#pragma unroll 1
            for (int k = k0; k < k1; ++k) {
                if (!at.wait(s->empty, 1, s, a.w)) break;
                uint64_t *const full = &s->full[at.slot];
                const uint32_t dst = base + at.slot * a.stage_bytes;
                at.step(a.stages);
                at.ask(s->empty, 1);
                if (k - k0 >= ahead) {
                    bar_expect(full, bytes);
                    load_cols(k, dst, smem_addr(full));
                    ++issued;
                }
                load_rows(k, dst + kTileBytes, smem_addr(full));
            }
            s->issued = issued;
        }
        __syncwarp();
    } else {
        __syncthreads();
        cluster_arrive_relaxed();
        grid_dependency_wait();
    }
    fence_after();
    const uint32_t tmem = s->tmem;
    grid_launch_dependents();
    if (warp == 5) {
        if (elect_one()) {
            Place at;
            const uint32_t idesc = p.idesc, by_r = advance(p.r_k), by_c = advance(p.c_k);
            const uint64_t of_r = describe(p.r_k), of_c = describe(p.c_k);
            at.ask(s->full, 0);
#pragma unroll 1
            for (int k = k0; k < k1; ++k) {
                if (!at.wait(s->full, 0, s, a.w)) break;
                const uint32_t src = smem_addr(smem) + at.slot * a.stage_bytes;
                const uint64_t dc = of_c | place_of(src), dr = of_r | place_of(src + kTileBytes);
                uint64_t *const empty = &s->empty[at.slot];
                at.step(a.stages);
                at.ask(s->full, 0);
                fence_after();
#pragma unroll
                for (int i = 0; i < 4; ++i) multiply<1, E::kBytes>(tmem, dc + i * by_c, dr + i * by_r, idesc, k > k0 || i > 0);
                commit<1>(empty);
            }
            commit<1>(&s->acc_full[0]);         // (also after a wait that gave up: products in flight end before their operands go away)
        }
        __syncwarp();
    }
    // ---- parts to the CTAs that finish them ----
    float *const own = (float *)smem;           // [n][128]
    constexpr int kVecs = E::kPairs ? 8 : 16;   // of eight columns, in a row of the tile
    const int end = min(p.cols, col + kTileCols), at = col + threadIdx.x % kVecs * 8, valid = valid_of<E, 8>(at, end), first = row + piece * share;
    typename E::template Extra<8> x, next;
    if (threadIdx.x / kVecs < mine && valid > 0) p.e.template fetch<8>(first + threadIdx.x / kVecs, at, valid, x);
    bool ok = warp_wait(&s->acc_full[0], 0, s, a.w);
    fence_after();
    ok = __syncthreads_and(ok && !s->abort);
    if (!ok && threadIdx.x == 0) let_loads_land(s, a.stages, &s->issued, 1, a.w);
    if (ok) {
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
#pragma unroll 1
        for (int c = (warp >> 2) * 16; c < n; c += 32) {
            float v[16];
            read16(lanes + c, v);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (c + i < n) own[(c + i) * kLanes + (threadIdx.x & 127)] = v[i];
        }
        fence_before();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    cluster_wait();
    if (!a.apart) {
        cluster_arrive();
        cluster_wait();
    }
    if (ok && warp < pieces && warp != piece) { // (a warp for each other CTA)
        const int theirs = min(n - warp * share, share);
        if (theirs > 0 && elect_one())
            asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(in_cta(smem_addr(smem) + a.parts_at + (piece - (piece > warp)) * share * kRowBytes, warp)), "r"(smem_addr(own) + warp * share * kRowBytes),
                           "r"(theirs * kRowBytes), "r"(in_cta(smem_addr(parts_full), warp)) : "memory");
        __syncwarp();
    }
    if (warp == 5) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(a.tmem_cols) : "memory");
    // ---- their sum ----
    ok = warp_wait(parts_full, 0, s, a.w) && ok;
    // (no CTA ends before the others have its parts)
    cluster_arrive_relaxed();
    bool by_rows = true;
    if constexpr (E::kRagged) by_rows = p.e.aligned;
    if constexpr (E::kRagged)
        if (ok && !by_rows) {                   // a column per lane, as for pairs
            const int one_col = threadIdx.x & 127;
#pragma unroll 2
            for (int r = threadIdx.x >> 7; r < mine && col + one_col < end; r += 2) {
                typename E::template Extra<1> one;
                p.e.template fetch<1>(first + r, col + one_col, 1, one);
                Acc sum[1] = {};
                for (int i = 0; i < pieces; ++i)
                    sum[0] += *(const Acc *)(smem + (i == piece ? (piece * share + r) * kRowBytes : a.parts_at + ((i - (i > piece)) * share + r) * kRowBytes) + one_col * 4);
                p.e.template emit<1>(first + r, col + one_col, 1, sum, sum, one);
            }
        }
    if (ok && by_rows) {
        const uint8_t *from = smem + threadIdx.x % kVecs * 32;
#pragma unroll 1
        for (int r = threadIdx.x / kVecs; r < mine && valid > 0; r += kSplitThreads / kVecs) {
            const int then = r + kSplitThreads / kVecs;
            if (then < mine) p.e.template fetch<8>(first + then, at, valid, next);
            Acc sum[2][8] = {};
#pragma unroll 2
            for (int i = 0; i < pieces; ++i) {
                const uint8_t *part = from + (i == piece ? (piece * share + r) * kRowBytes : a.parts_at + ((i - (i > piece)) * share + r) * kRowBytes);
#pragma unroll
                for (int h = 0; h < (E::kPairs ? 2 : 1); ++h) {
                    const uint4 *q = (const uint4 *)(part + h * 256);
                    const uint4 lo = q[0], hi = q[1];
                    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        Acc one;
                        as_sum(w[j], one);
                        sum[h][j] += one;
                    }
                }
            }
            p.e.template emit<8>(first + r, at, valid, sum[0], sum[1], x);
            x = next;
        }
    }
    __syncwarp();
    cluster_wait();
}

// ---- a few rows: plain dot products ----
// A warp has R neighbouring columns of the output (with two products a column of each) and all rows, lanes lie along the sum, 16 bytes each; S warps share the columns and
// halve, quarter ... the sum.  Weights are read once, straight into registers; nothing has to be set up, and blocks of the next product find room beside these and
// ask for their weights before these have ended.  Bound by HBM: one row, 7168 to 2 x 2048 13.2 us (58.7 MB, 9.1 us), 2048 to 7168 7.6 us (29.4 MB, 4.5 us), the two chained 19.4 us.
constexpr int kRowThreads = 256;
// Rows up to which that is the faster way, against clusters, us: one token everywhere; two of bf16 22.6 / 26.1 (7168, 2 x 2048), of integers 20.0 / 16.9 (7168 to 7168); three of bf16 38 / 27.5.
constexpr int kFewRows16 = 2, kFewRows8 = 1;

template <class E>
struct RowsArgs {
    const uint8_t *r, *c;
    int64_t r_stride, c_stride, pair;           // bytes; from a column of the first product to the second's
    int cols, steps, tail;                      // steps of 512 bytes along the sum; bytes of the last one
    int split, half, early;
    E e;
};

__device__ __forceinline__ uint4 load_once(const uint8_t *p)
{
    uint4 q;
    asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p));
    return q;
}
__device__ __forceinline__ void pair_of(uint32_t w, int half, float &lo, float &hi)
{
    if (half) {
        const float2 f = __half22float2(*(const __half2 *)&w);
        lo = f.x; hi = f.y;
    } else {
        lo = __uint_as_float(w << 16);
        hi = __uint_as_float(w & 0xffff0000u);
    }
}
__device__ __forceinline__ void dot16(const uint4 &w, const uint4 &x, int half, float &sum)
{
    const uint32_t a[4] = {w.x, w.y, w.z, w.w}, b[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float wl, wh, xl, xh;
        pair_of(a[i], half, wl, wh);
        pair_of(b[i], half, xl, xh);
        sum = fmaf(wl, xl, sum);
        sum = fmaf(wh, xh, sum);
    }
}
__device__ __forceinline__ void dot16(const uint4 &w, const uint4 &x, int, int32_t &sum)
{
    sum = __dp4a((int)w.x, (int)x.x, sum); sum = __dp4a((int)w.y, (int)x.y, sum);
    sum = __dp4a((int)w.z, (int)x.z, sum); sum = __dp4a((int)w.w, (int)x.w, sum);
}

template <class E, int T, int R>
__global__ void __launch_bounds__(kRowThreads) k_rows(const __grid_constant__ RowsArgs<E> a)
{
    using Acc = typename E::Acc;
    constexpr int kSums = E::kPairs ? 2 : 1, kLoads = E::kBytes == 1 ? 4 : 8, kAhead = kLoads / R / kSums < 1 ? 1 : kLoads / R / kSums;    // steps asked for at a time
    __shared__ Acc parts[kRowThreads / 32][kSums][R][T];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int groups = kRowThreads / 32 / a.split, col = (blockIdx.x * groups + warp / a.split) * R, part = warp % a.split;
    const int k0 = a.steps * part / a.split, k1 = a.steps * (part + 1) / a.split;
    const uint8_t *c[kSums][R];
#pragma unroll
    for (int h = 0; h < kSums; ++h)
#pragma unroll
        for (int i = 0; i < R; ++i) c[h][i] = a.c + (int64_t)min(col + i, a.cols - 1) * a.c_stride + h * a.pair + lane * 16;
    Acc sum[kSums][R][T] = {};
    uint4 w[kAhead][kSums][R];
    const auto ask = [&](int k) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < kSums; ++h)
#pragma unroll
                for (int i = 0; i < R; ++i)
                    w[u][h][i] = k + u < k1 && (k + u + 1 < a.steps || lane * 16 < a.tail) ? load_once(c[h][i] + (int64_t)(k + u) * 512) : make_uint4(0, 0, 0, 0);
    };
    if (a.early) ask(k0);
    grid_dependency_wait();
    grid_launch_dependents();
    if (!a.early) ask(k0);
#pragma unroll 1
    for (int k = k0; k < k1; k += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (k + u < k1) {
                const bool in = k + u + 1 < a.steps || lane * 16 < a.tail;
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const uint4 x = in ? *(const uint4 *)(a.r + t * a.r_stride + (int64_t)(k + u) * 512 + lane * 16) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int h = 0; h < kSums; ++h)
#pragma unroll
                        for (int i = 0; i < R; ++i) dot16(w[u][h][i], x, a.half, sum[h][i][t]);
                }
            }
        if (k + kAhead < k1) ask(k + kAhead);
    }
#pragma unroll
    for (int h = 0; h < kSums; ++h)
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int d = 16; d; d >>= 1) sum[h][i][t] += __shfl_xor_sync(0xffffffffu, sum[h][i][t], d);
    if (lane == 0)
#pragma unroll
        for (int h = 0; h < kSums; ++h)
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int t = 0; t < T; ++t) parts[warp][h][i][t] = sum[h][i][t];
    __syncthreads();
    const int g = threadIdx.x / (R * T), i = threadIdx.x / T % R, t = threadIdx.x % T, out = (blockIdx.x * groups + g) * R + i;
    if (g >= groups || out >= a.cols) return;
    Acc x[1] = {}, y[1] = {};
    for (int p = 0; p < a.split; ++p) {
        x[0] += parts[g * a.split + p][0][i][t];
        if (kSums == 2) y[0] += parts[g * a.split + p][kSums - 1][i][t];
    }
    typename E::template Extra<1> extra;
    a.e.template fetch<1>(t, out, 1, extra);
    a.e.template emit<1>(t, out, 1, x, y, extra);
}

// ---- host side ----
// What a device can run at once: SMs, and clusters of each size whose blocks have an SM each (an SM is in one of several groups, which a cluster does not leave: of clusters of eight
// there are fewer than an eighth of the SMs, and one more than there is room for runs after the others).
struct Room {
    int sms, clusters[kMaxSplit + 1];
};

// How the launches of a handle's last call made their products (test hook).
constexpr int kMaxWays = 4;
struct Ways {
    int32_t count;
    mw_dense_way list[kMaxWays];
};

struct Call {
    cudaStream_t st;
    bool overlap;                               // kernels may start while the one before drains
    int dtype;
    const Room *room;
    Waits w;
    bool early;                                 // the columns' operand was there before the kernel that this one follows
    int64_t *launches;                          // counted
    Ways *ways;                                 // noted
};
inline void note(const Call &call, int columns, int tiles, int halves, int pieces)
{
    ++*call.launches;
    if (call.ways->count < kMaxWays) call.ways->list[call.ways->count++] = {columns, tiles, halves, pieces};
}

// A map of boxes `box` indices high (K-major), or 64 indices wide and 64 steps high.  `pairs`: the operand is two of `count` / 2 indices.
inline bool map_operand(CUtensorMap *map, const Operand &o, int depth, int bytes, int box, bool pairs)
{
    const uint64_t stride = (uint64_t)o.stride_bytes;
    if (!o.k_major) {
        const uint64_t d[2] = {(uint64_t)o.count, (uint64_t)depth}, st[1] = {stride};
        const uint32_t b[2] = {64, 64};
        return encode_map(map, o.base, 2, d, st, b, bytes);
    }
    const uint64_t count = pairs ? o.count / 2 : o.count;
    const uint64_t d[3] = {(uint64_t)depth, count, 2}, st[2] = {stride, stride * count};
    const uint32_t b[3] = {(uint32_t)(kLine / bytes), (uint32_t)box, 1};
    return encode_map(map, o.base, pairs ? 3 : 2, d, st, b, bytes);
}

inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Lets a kernel have that much shared memory on the current device, asked for once (`done`: a bit per device).
template <class K>
cudaError_t allow_memory(std::atomic<uint64_t> &done, K *kernel, int bytes)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const uint64_t bit = device < 64 ? 1ull << device : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// A product to be made: out = R C^T for `cols` columns and sums of `depth` products.
template <class E>
struct Job {
    Operand r, c;
    int cols, depth;
    E e;
};

template <class E>
int steps_of(const Job<E> &j) { return ceil_div(j.depth, kLine / E::kBytes); }
// Bytes of the columns' operand per step and CTA (pairs of n columns), of the rows' (clusters of n rows).
inline uint32_t pair_bytes(bool c_k, int n) { return kTileBytes + (c_k ? n / 2 * kLine : ceil_div(n / 2, 64) * kBlock); }
inline uint32_t split_bytes(bool r_k, int n) { return kTileBytes + (r_k ? n * kLine : ceil_div(n, 64) * kBlock); }

template <class E>
bool describe_problem(Problem<E> *p, const Job<E> &j, int box_r, int box_c)
{
    p->rows = j.r.count; p->cols = j.cols; p->steps = steps_of(j);
    p->r_k = j.r.k_major; p->c_k = j.c.k_major;
    p->e = j.e;
    return map_operand(&p->map_r, j.r, j.depth, E::kBytes, box_r, false) && map_operand(&p->map_c, j.c, j.depth, E::kBytes, box_c, E::kPairs);
}

// Tiles at the end that are cut in two.
inline int cut_tiles(int64_t tiles, int slots, int n)
{
    const int64_t rest = tiles % slots;
    return n == kMaxCols && tiles > slots && 2 * rest <= slots ? (int)rest : 0;
}

template <class E>
cudaError_t launch_pair(const Call &call, const Job<E> *jobs, int count, int n)
{
    PairArgs<E> a;
    a.n = n; a.tile_cols = E::kPairs ? n / 2 : n;
    a.count = count; a.tiles = 0; a.stage_bytes = 0;
    for (int i = 0; i < count; ++i) a.tiles += ceil_div(jobs[i].r.count, 2 * kLanes) * ceil_div(jobs[i].cols, a.tile_cols);
    const int slots = call.room->sms / 2, rest = cut_tiles(a.tiles, slots, n);
    a.whole = a.tiles - rest;
    a.box = rest ? 64 : n / 2;                  // (two loads of 64 where one of 128 would do cost 4 %)
    a.tiles = 0;
    for (int i = 0; i < count; ++i) {
        Problem<E> &p = a.p[i];
        if (!describe_problem(&p, jobs[i], kLanes, a.box)) return cudaErrorInvalidValue;
        p.row_tiles = ceil_div(p.rows, 2 * kLanes); p.col_tiles = ceil_div(p.cols, a.tile_cols); p.first = a.tiles;
        p.tile_rows = 2 * kLanes; p.n = 2 * kLanes;
        p.idesc = instruction(call.dtype, p.r_k, p.c_k, 2 * kLanes, n);
        p.idesc_cut = instruction(call.dtype, p.r_k, p.c_k, 2 * kLanes, n / 2);
        p.bytes = pair_bytes(p.c_k, n);
        p.bytes_cut = pair_bytes(p.c_k, n / 2);
        a.tiles += p.row_tiles * p.col_tiles;
        a.stage_bytes = a.stage_bytes > p.bytes ? a.stage_bytes : p.bytes;
    }
    a.stages = kPairRing / a.stage_bytes < kMaxStages ? kPairRing / a.stage_bytes : kMaxStages;
    a.w = call.w;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t set = allow_memory(allowed, k_pair<E>, (int)kPairSmem);
    if (set != cudaSuccess) return set;
    a.tiles += rest;
    const int pairs = a.tiles < slots ? a.tiles : slots;
    note(call, n, a.tiles, 2 * rest, 0);
    return mw_launch(k_pair<E>, dim3(2 * pairs), dim3(kPairThreads<E>), kPairSmem, call.st, call.overlap, a);
}

// The launch of clusters of `pieces` blocks; attr: room for two.
inline cudaLaunchConfig_t cluster_launch(cudaLaunchAttribute *attr, int pieces, int tiles, size_t smem, cudaStream_t st, bool overlap)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(pieces, tiles);
    cfg.blockDim = dim3(kSplitThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = pieces; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = overlap ? 2 : 1;
    return cfg;
}
constexpr size_t kSplitSmem = 225 * 1024;

// Of the current device; found once (a device does not change while a process runs).
inline cudaError_t find_room(Room *room, int device)
{
    static std::atomic<int> state[64];          // 0: nobody has looked, 1: somebody writes `known`, 2: it is there
    static Room known[64];
    if (device < 64 && state[device].load(std::memory_order_acquire) == 2) { *room = known[device]; return cudaSuccess; }
    const auto kernel = k_split<Store>;
    cudaError_t e = cudaDeviceGetAttribute(&room->sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSplitSmem);
    room->clusters[0] = 0;
    for (int p = 1; p <= kMaxSplit && e == cudaSuccess; ++p) {
        cudaLaunchAttribute attr[2];
        const cudaLaunchConfig_t cfg = cluster_launch(attr, p, 1, kSplitSmem, nullptr, false);
        e = cudaOccupancyMaxActiveClusters(&room->clusters[p], kernel, &cfg);
    }
    int nobody = 0;
    if (e == cudaSuccess && device < 64 && state[device].compare_exchange_strong(nobody, 1)) {
        known[device] = *room;
        state[device].store(2, std::memory_order_release);
    }
    return e;
}

// Loads kernels now, so that a first call may be one that is captured.
template <class K>
cudaError_t load_kernel(K *kernel)
{
    cudaFuncAttributes attributes;
    return cudaFuncGetAttributes(&attributes, kernel);
}
template <class E>
cudaError_t load_dots()
{
    cudaError_t e = load_kernel(k_rows<E, 1, 1>);
    if (e == cudaSuccess) e = load_kernel(k_rows<E, 1, 2>);
    if constexpr (!E::kPairs)
        if (e == cudaSuccess) e = load_kernel(k_rows<E, 1, 4>);
    if constexpr (E::kBytes == 2) {
        if (e == cudaSuccess) e = load_kernel(k_rows<E, 2, 1>);
        if (e == cudaSuccess) e = load_kernel(k_rows<E, 2, 2>);
        if constexpr (!E::kPairs)
            if (e == cudaSuccess) e = load_kernel(k_rows<E, 2, 4>);
    }
    return e;
}
template <class E>
cudaError_t load_kernels()
{
    cudaError_t e = load_kernel(k_pair<E>);
    if (e == cudaSuccess) e = load_kernel(k_split<E>);
    if constexpr (E::kDots)
        if (e == cudaSuccess) e = load_dots<E>();
    return e;
}

// Rows per tile where at most `most` are wanted: tiles about equally full, multiples of 16 (loads of 64 neighbouring indices begin on 16 bytes).
inline int cluster_rows(int rows, int most) { return (ceil_div(rows, ceil_div(rows, most)) + 15) & ~15; }

template <class E>
cudaError_t launch_split(const Call &call, const Job<E> *jobs, int count, int most, int pieces)
{
    constexpr int kTileCols = E::kPairs ? kLanes / 2 : kLanes;
    SplitArgs<E> a;
    a.count = count; a.stage_bytes = 0;
    int tiles = 0, n = 0;
    for (int i = 0; i < count; ++i) {
        Problem<E> &p = a.p[i];
        const int rows = cluster_rows(jobs[i].r.count, most);
        if (!describe_problem(&p, jobs[i], rows, kTileCols)) return cudaErrorInvalidValue;
        p.tile_rows = p.n = rows;
        p.row_tiles = ceil_div(p.rows, rows); p.col_tiles = ceil_div(p.cols, kTileCols); p.first = tiles;
        p.idesc = instruction(call.dtype, p.c_k, p.r_k, kLanes, rows);
        p.bytes = split_bytes(p.r_k, rows);
        tiles += p.row_tiles * p.col_tiles;
        a.stage_bytes = a.stage_bytes > p.bytes ? a.stage_bytes : p.bytes;
        n = n > rows ? n : rows;
    }
    a.tmem_cols = 32;
    while ((int)a.tmem_cols < n) a.tmem_cols *= 2;
    // One block per SM: what counts is how much is asked for ahead (half the memory for each, so that the next kernel's blocks find room beside: 64 tokens through 7168,
    // 2 x 2048 30.0 us instead of 27.8).  The others' parts have room of their own where four stages are left (one wait for the cluster less).  A block's share of shared
    // memory is never smaller than its share of TMEM, so that blocks that share an SM find their columns.
    const size_t room = kSplitSmem - 1024, own = (size_t)n * kRowBytes;
    // (Tiles of 256 rows have room for four pieces, of 240 for six.  `choose` does not know: what it expects of more pieces of such a tile is of a launch that is not made.)
    while (pieces > 1 && own + (size_t)(pieces - 1) * ceil_div(n, pieces) * kRowBytes > room) --pieces;
    const size_t parts = (size_t)(pieces - 1) * ceil_div(n, pieces) * kRowBytes, beside = (room - parts) / a.stage_bytes;
    a.apart = beside >= 4;
    a.stages = (int)(a.apart ? beside : room / a.stage_bytes);
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    const size_t held = (size_t)a.stages * a.stage_bytes;
    a.parts_at = (uint32_t)(a.apart && held > own ? held : own);
    const size_t used = a.parts_at + parts > held ? a.parts_at + parts : held, least = (size_t)a.tmem_cols * 456;
    const size_t smem = 1024 + (used > least ? used : least);
    a.early = call.early; a.w = call.w;
    const auto kernel = k_split<E>;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t set = allow_memory(allowed, kernel, (int)kSplitSmem);
    if (set != cudaSuccess) return set;
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = cluster_launch(attr, pieces, tiles, smem, call.st, call.overlap);
    note(call, 0, tiles, 0, pieces);
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <class E, int T>
cudaError_t launch_rows(const Call &call, const Job<E> &j, int per_warp, int split)
{
    constexpr int BYTES = E::kBytes;
    const Operand &r = j.r, &c = j.c;
    const int cols = j.cols, depth = j.depth;
    RowsArgs<E> a;
    a.r = (const uint8_t *)r.base; a.c = (const uint8_t *)c.base;
    a.r_stride = r.stride_bytes; a.c_stride = c.stride_bytes; a.pair = c.stride_bytes * cols;
    a.cols = cols; a.steps = ceil_div(depth * BYTES, 512); a.tail = depth * BYTES - (a.steps - 1) * 512;
    a.split = split; a.half = call.dtype == MW_DTYPE_F16; a.early = call.early; a.e = j.e;
    const dim3 grid(ceil_div(cols, kRowThreads / 32 / split * per_warp));
    note(call, 0, (int)grid.x, 0, 0);
    if (per_warp == 1) return mw_launch(k_rows<E, T, 1>, grid, dim3(kRowThreads), 0, call.st, call.overlap, a);
    if constexpr (!E::kPairs)
        if (per_warp == 4) return mw_launch(k_rows<E, T, 4>, grid, dim3(kRowThreads), 0, call.st, call.overlap, a);
    return mw_launch(k_rows<E, T, 2>, grid, dim3(kRowThreads), 0, call.st, call.overlap, a);
}
template <class E>
cudaError_t choose_rows(const Call &call, const Job<E> &j)
{
    constexpr int BYTES = E::kBytes;
    const int cols = j.cols, depth = j.depth;
    // Warps per SM: fewer columns per warp, then pieces of the sum, until there are as many.  16 / 32 per SM, one token: bf16 7168 to 2 x 2048 13.2 / 15.0 us, 2048 to 7168
    // 7.6 / 8.3; integers 7168 to 7168 11.0 / 10.6, 7168 to 4096 9.5 / 7.3.
    // (Loads of 16 bytes under way per lane, kLoads: eight of 16-bit operands, four of integers.  The other way round, replayed: the gated block (7168, 2048) of one token 21.3 us instead of 19.2, of two
    // 24.2 instead of 22.6, 4096 wide and deep 25.9 instead of 23.7; integers 7168 to 7168 14.5 instead of 11.8, 2048 to 7168 6.1 instead of 5.1; only 4096 to 28672 gains, 21.2 instead of 22.7.)
    const int want = call.room->sms * (BYTES == 1 ? 32 : 16), steps = ceil_div(depth * BYTES, 512);
    int per_warp = E::kPairs ? 2 : 4, split = 1;
    while (per_warp > 1 && cols / per_warp < want) per_warp /= 2;
    while (split < 8 && (int64_t)ceil_div(cols, per_warp) * split < want && steps / split >= 4) split *= 2;
    if constexpr (BYTES == 2)
        if (j.r.count == 2) return launch_rows<E, 2>(call, j, per_warp, split);
    return launch_rows<E, 1>(call, j, per_warp, split);
}

// Which of the two ways, and its tiles: the least of what they are expected to take, in us (caches cold, a launch by itself).  A step takes what its products take, or what the running
// CTAs draw from L2 together at 16 TB/s; beyond the steps of the longest chain there is the start, and what comes after the last product.  Measured against expected, us: gate and up of 777 rows
// (1024 to 2 x 688) clusters of 64 rows 9.4 / 11.2, of 128 11.0 / 11.7, pairs of 128 columns 11.4 / 11.5, of 256 16.6 / 16.8; of 512 rows (7168 to 2 x 2048) pairs of 128 30.4 / 31,
// of 256 45.9 / 46, clusters of 256 rows by two 33 / 34; down of 512 rows (2048 to 7168) pairs of 224 17.7 / 15.8, of 128 19.4 / 21.5, clusters of 256 22.8 / 21; both gradients of the
// weights from 64 tokens (7168, 2048) pairs of 64 55 / 52, of 128 30 / 29, of 224 27 / 25, of 256 25 / 24.
// (Pairs of 160 and 192 columns are slower than of 224: 132 us against 112, 4096 rows, 2048 to 7168.)
constexpr float kL2Rate = 16e6f;                // bytes per us

struct Way {
    float us;
    int n;                                      // pairs: columns of the accumulator; 0: clusters
    int most, pieces;                           // clusters: rows per tile at most, pieces of the sum
};
inline void better(Way &best, const Way &w) { if (w.us < best.us) best = w; }

// Rows along the sum that do not begin on 128 bytes: a step's 128 bytes of one lie in two lines of L2, and a step of a cluster takes longer, twice as long where both operands do so (201 rows, 2808 to 1024, us: clusters of 64
// rows by one 17.7, by two 11.8, by four 9.5; of 256 29.9, 19.6, 16.0).  Pairs, of which one loads at most 32 KB a step, are left as they are: with a factor the others were chosen where they are slower.
template <class E>
float lines_apart(const Job<E> &j)
{
    const bool r = j.r.k_major && j.r.stride_bytes % 128, c = j.c.k_major && j.c.stride_bytes % 128;
    return r && c ? 2.2f : r || c ? 1.3f : 1.0f;
}

template <class E>
Way choose(const Room &room, const Job<E> *jobs, int count)
{
    const int slots = room.sms / 2;
    Way best = {1e30f, 0, 0, 0};
    for (const int n : {256, 224, 128, 64}) {
        // (the first pair takes the first tile of every round)
        int64_t tiles = 0;
        for (int i = 0; i < count; ++i) tiles += (int64_t)ceil_div(jobs[i].r.count, 2 * kLanes) * ceil_div(jobs[i].cols, E::kPairs ? n / 2 : n);
        const float finish = n * E::kFinish, running = 2.0f * (tiles < slots ? tiles : slots);
        const bool cut = cut_tiles(tiles, slots, n) > 0;
        float us = 6.5f + finish;
        int64_t first = 0;
        for (int i = 0; i < count; ++i) {
            const int64_t end = first + (int64_t)ceil_div(jobs[i].r.count, 2 * kLanes) * ceil_div(jobs[i].cols, E::kPairs ? n / 2 : n);
            const float step = fmaxf(fmaxf(0.14f, n * 0.00105f), running * pair_bytes(jobs[i].c.k_major, n) / kL2Rate);
            const float products = steps_of(jobs[i]) * step, tile = fmaxf(products, 0.6f + n * jobs[i].e.busy(n));
            if (i == 0) us += products - tile;  // (nothing goes before the first)
            us += ((end + slots - 1) / slots - (first + slots - 1) / slots) * tile;
            if (cut && i == count - 1) us -= 0.35f * tile;
            first = end;
        }
        better(best, {us, n, 0, 0});
    }
    for (const int most : {256, 128, 64}) {
        int64_t tiles = 0;
        float bytes = 0.0f;
        for (int i = 0; i < count; ++i) {
            const int n = cluster_rows(jobs[i].r.count, most);
            const int64_t of = (int64_t)ceil_div(jobs[i].r.count, n) * ceil_div(jobs[i].cols, E::kPairs ? kLanes / 2 : kLanes);
            tiles += of;
            bytes += (float)of * split_bytes(jobs[i].r.k_major, n);
        }
        for (int p = 1; p <= kMaxSplit; ++p) {
            if (tiles > room.clusters[p]) continue;
            float us = 0.0f;
            for (int i = 0; i < count; ++i) {
                const int n = cluster_rows(jobs[i].r.count, most), steps = steps_of(jobs[i]);
                const float step = fmaxf(fmaxf(0.11f, n * 0.00103f) * lines_apart(jobs[i]), p * bytes / kL2Rate);
                us = fmaxf(us, p > steps ? 1e30f : 5.95f + 0.016f * n + fmaxf(0.012f, E::kFinish * 0.85f) * n / p + ceil_div(steps, p) * step);
            }
            better(best, {us, 0, most, p});
        }
    }
    return best;
}

// Makes the jobs, up to three, which need nothing of one another: in one launch, one by itself and the others together, or each by itself, whichever is expected to take least.  (One launch saves
// starts and last rounds of tiles; but all its products have one kind of tile, and the gradient of few tokens is a few long sums beside large outer products: 15 tokens, 568 wide, 5056 deep,
// forward and backward 73 us together, 36 apart.)
template <class E>
cudaError_t product(const Call &call, const Job<E> *jobs, int count)
{
    if constexpr (E::kDots)
        if (count == 1 && jobs->r.k_major && jobs->c.k_major && jobs->r.count <= (E::kBytes == 1 ? kFewRows8 : kFewRows16)) return choose_rows(call, *jobs);
    const Way w = choose(*call.room, jobs, count);
    if constexpr (E::kProblems > 1)
        if (count > 1) {
            float least = w.us;
            int alone = -1;
            Job<E> others[E::kProblems];
            for (int i = 0; i < count; ++i) {
                int n = 0;
                for (int j = 0; j < count; ++j)
                    if (j != i) others[n++] = jobs[j];
                const float rest = n == 1 ? choose(*call.room, others, 1).us : fminf(choose(*call.room, others, 2).us, choose(*call.room, others, 1).us + choose(*call.room, others + 1, 1).us);
                const float us = choose(*call.room, jobs + i, 1).us + rest;
                if (us < least) { least = us; alone = i; }
            }
            if (alone >= 0) {
                int n = 0;
                for (int j = 0; j < count; ++j)
                    if (j != alone) others[n++] = jobs[j];
                const cudaError_t e = product(call, jobs + alone, 1);
                Call after = call;
                after.early = false;
                return e == cudaSuccess ? product(after, others, n) : e;
            }
        }
    return w.n ? launch_pair(call, jobs, count, w.n) : launch_split(call, jobs, count, w.most, w.pieces);
}
template <class E>
cudaError_t product(const Call &call, const Job<E> &job) { return product(call, &job, 1); }

#endif  // __CUDACC__

}  // namespace mw_dense
