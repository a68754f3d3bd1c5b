// The shared projection with low-rank adapters: y[t] = W x[t] + scale[a] B[a] (A[a] x[t]), a = adapter of token t.
// Declared in include/mw.h.
//
// W x runs on the tensor cores, tokens in tiles of up to 256; the epilogue adds B[a] v[t], v[t] = scale[a] A[a] x[t], an
// adapter at a time, and each token takes its own adapter's product only.  (As steps of the tensor-core product, with zeros in the other tokens'
// columns, it let a NaN or infinity in one adapter's B reach the other requests: 0 * NaN.)
// v is made by launches of their own, before; the projection begins while they run, and its epilogue waits for them:
//   low     few values (T * rank up to kDirect): a block per (token, four ranks), plain dot products;
//   lists, shrink   more: per tile of 64 tokens its distinct adapters, in order of first use; then the A rows of all adapters of a
//           tile, stacked to tiles of 128 rows, times all tokens of the tile on the tensor cores: most of these products are not
//           wanted, but an adapter's A is read once for 64 tokens; a token keeps the rows of its own adapter.
//
// Bound: HBM for few tokens (7168 x 7168, rank 16: one token 23.5 us, 4.4 TB/s, floor 15.7; 64 tokens 30.9 us, floor 17.8), the tensor cores for prompts
// (4096 tokens at rank 64: 505 us in calls back to back, 0.85 PFLOP/s under the power cap; without adapters 469 us, 0.9 PFLOP/s).  What the prompts lose: one CTA's
// 128 x 256 tile keeps its shared memory busier than the tensor core (weights and tokens both written and read for each step; the tensor pipe is active
// 57 % of the time), and 35 us of shrink and 22 of the last tile's additions lie outside the products.  The router's logits (float32, 256 columns, 7168 deep)
// are two tiles of rows: 1 token 10.1 us, 64 tokens 15.0, 4096 tokens 38.9 (floors 0.6, 0.7, 10.2), the latency of ten CTAs' long sums.
#include <new>
#include <string.h>

#include "mw_stream.cuh"

using namespace mw_stream;

struct mw_project {
    mw_project_config cfg;
    const void *w, *a, *b;
    const float *scale;
    CUtensorMap map_w, map_a;
    void *slab;
    int32_t *status;
    unsigned int *counts, *done;
    float *parts;
    int32_t *found;             // [tiles]            distinct adapters of a tile of shrink
    int32_t *entries;           // [tiles * 64]       the adapters
    int32_t *at;                // [tiles + 1]        exclusive prefix sums of the adapter groups of a tile
    uint4 *v;                   // [max_tokens, rank / 4], see split_low
    int sm_count;
    int skew;                   // bytes added to the announced size of the next call's loads of weights (test hook)
    int64_t launches;
};

namespace {

constexpr size_t kSmem = 227 * 1024 - 512;      // dynamic shared memory of a block (a few bytes are static)
constexpr int kListThreads = 64;                 // tokens per tile of shrink
constexpr int kLowThreads = 256;
// Low-rank values, T * rank, up to which they are plain dot products: with all that fits the SMs at once, a launch less and no second start of the
// pipeline count for more than reading an adapter's A again for each of its tokens.  Measured, dot products / lists and shrink, us per call at rank 16: 64 tokens
// 31 / 58, 256 tokens 65 / 76 (7168 x 7168), 512 tokens 58.7 / 57.8 (4096 x 4096), 1024 tokens 162 / 150 (7168 x 7168).
constexpr int kDirect = 4096;
constexpr int kAddPitch = 17;                    // floats between two rows of a warp's 32 x 16 additions in shared memory

// The low-rank values are kept as sums of two bf16, sixteen bits that count, in the layout of the products' operands: of four neighbouring ranks
// the first terms, then the second, which are what the first leave (nothing, where the first is not finite).  A finite value that would round to
// infinity has the largest finite first term.
// (Kept as float32 and split in `add`, again for each row of tiles: 467 us instead of 450 for 4096 tokens of rank 64, 7168 x 7168.)
__device__ __forceinline__ void split_low(float f, uint16_t &hi, uint16_t &lo)
{
    hi = f32_to_bf16(f);
    if ((hi & 0x7fffu) == 0x7f80u && fabsf(f) < INFINITY) --hi;
    const float p = __uint_as_float((uint32_t)hi << 16);
    lo = f32_to_bf16(fabsf(p) < INFINITY ? f - p : 0.0f);
}
__device__ __forceinline__ uint4 split_low(const float4 &f)
{
    uint16_t hi[4], lo[4];
    split_low(f.x, hi[0], lo[0]);
    split_low(f.y, hi[1], lo[1]);
    split_low(f.z, hi[2], lo[2]);
    split_low(f.w, hi[3], lo[3]);
    return make_uint4(hi[0] | (uint32_t)hi[1] << 16, hi[2] | (uint32_t)hi[3] << 16, lo[0] | (uint32_t)lo[1] << 16, lo[2] | (uint32_t)lo[3] << 16);
}

struct ListArgs {
    const int32_t *ids;
    int T, tiles, adapters;
    int per_group;              // adapters whose A rows fit one tile of weight rows
    int32_t *found, *at, *entries;
    unsigned int *done;
    int32_t *status;
};

// One block per token tile, one thread per token; the last block to finish adds up the tiles.
__global__ void __launch_bounds__(kListThreads) k_adapter_lists(const __grid_constant__ ListArgs a)
{
    constexpr int kWarps = kListThreads / 32;
    __shared__ int id_s[kListThreads], count_s[kWarps], last_s;
    grid_dependency_wait();
    grid_launch_dependents();
    const int c = threadIdx.x, lane = c & 31, warp = c >> 5;
    const int64_t t = (int64_t)blockIdx.x * kListThreads + c;
    int id = t < a.T ? a.ids[t] : -1;
    if (id < -1 || id >= a.adapters) { atomicCAS(a.status, MW_OK, MW_ERR_BAD_INDEX); id = -1; }
    id_s[c] = id;
    __syncthreads();
    int first = 0;                                          // the first token of the tile with this adapter
    if (id >= 0) while (id_s[first] != id) ++first;
    const bool leads = id >= 0 && first == c;
    const unsigned b = __ballot_sync(0xffffffffu, leads);
    if (lane == 0) count_s[warp] = __popc(b);
    __syncthreads();
    int at = __popc(b & ((1u << lane) - 1)), n = 0;
    for (int w = 0; w < kWarps; ++w) { if (w < warp) at += count_s[w]; n += count_s[w]; }
    if (leads) a.entries[(int64_t)blockIdx.x * kListThreads + at] = id;
    if (c == 0) {
        a.found[blockIdx.x] = n;
        __threadfence();
        last_s = atomicAdd(a.done, 1u) == gridDim.x - 1;
        if (last_s) *a.done = 0;
        __threadfence();
    }
    __syncthreads();
    if (!last_s) return;
    int base = 0;
    for (int from = 0; from < a.tiles; from += kListThreads) {
        const int i = from + c, k = i < a.tiles ? (__ldcg(a.found + i) + a.per_group - 1) / a.per_group : 0;
        int incl = k;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += v;
        }
        __syncthreads();
        if (lane == 31) count_s[warp] = incl;
        __syncthreads();
        int before = base, all = 0;
        for (int w = 0; w < kWarps; ++w) { if (w < warp) before += count_s[w]; all += count_s[w]; }
        if (i < a.tiles) a.at[i] = before + incl - k;
        base += all;
    }
    if (c == 0) a.at[a.tiles] = base;
}

__device__ __forceinline__ void unpack(const uint4 &q, float (&f)[8])
{
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(u[i] << 16); f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}

struct LowArgs {
    const int32_t *ids;
    const uint8_t *x;
    int64_t x_stride;
    const uint16_t *a;
    const float *scale;
    uint4 *v;
    int adapters, rank, H;
    int32_t *status;
};

// v[t, 4 j ... 4 j + 3]: block (j, t).  Bound by latency (one wave of blocks; runs beside the first products).  The five rows are read once each, kBatch * 5 16-byte loads in flight per thread.
__global__ void __launch_bounds__(kLowThreads) k_project_low(const __grid_constant__ LowArgs a)
{
    constexpr int kBatch = 4;
    __shared__ float4 sums[kLowThreads / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    const int t = blockIdx.y, j = blockIdx.x * 4, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int id = a.ids[t];
    if (id < 0 || id >= a.adapters) {
        if (id != -1 && j == 0 && threadIdx.x == 0) atomicCAS(a.status, MW_OK, MW_ERR_BAD_INDEX);
        return;
    }
    const int n = a.H / 8;
    const uint4 *x = (const uint4 *)(a.x + (int64_t)t * a.x_stride), *p = (const uint4 *)(a.a + ((int64_t)id * a.rank + j) * a.H);
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int h0 = threadIdx.x; h0 < n; h0 += kLowThreads * kBatch) {
        uint4 xv[kBatch], pv[kBatch][4];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int h = h0 + b * kLowThreads;
            if (h < n) {
                xv[b] = __ldg(x + h);
#pragma unroll
                for (int r = 0; r < 4; ++r) pv[b][r] = __ldg(p + (int64_t)r * n + h);
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
            if (h0 + b * kLowThreads < n) {
                float f[8], g[8];
                unpack(xv[b], f);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    unpack(pv[b][r], g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[r] = fmaf(f[i], g[i], s[r]);
                }
            }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] += __shfl_xor_sync(0xffffffffu, s[r], d);
    if (lane == 0) sums[warp] = make_float4(s[0], s[1], s[2], s[3]);
    __syncthreads();
    if (threadIdx.x == 0) {
        float4 v = sums[0];
        for (int w = 1; w < kLowThreads / 32; ++w) { v.x += sums[w].x; v.y += sums[w].y; v.z += sums[w].z; v.w += sums[w].w; }
        const float scale = a.scale ? a.scale[id] : 1.0f;
        a.v[((int64_t)t * a.rank + j) >> 2] = split_low(make_float4(scale * v.x, scale * v.y, scale * v.z, scale * v.w));
    }
}

enum { SHRINK, PROJECT };

template <int KIND>
struct Product {
    struct Args {
        CUtensorMap weights, tokens;            // SHRINK: A and x; PROJECT: W and x
        Common c;
        const int32_t *ids;                     // null: no adapters in this call
        int T, cols, tiles, adapters, rank;
        int row_tiles, units_per_tile, per_group, H, O;
        const int32_t *found, *at, *entries;    // SHRINK
        const float *scale;
        const uint16_t *b;                      // PROJECT
        uint4 *v;
        uint8_t *y;
        int64_t y_stride;
        int values_at;                          // SHRINK: bytes from the lists to the values on their way to v
        int y_f32, y_wide;                      // PROJECT: float32 rows; bf16 rows on 16-byte boundaries
    };
    static constexpr int kProducts = 1;
    static constexpr bool kEarly = false, kLate = false, kAdds = KIND == PROJECT, kClaims = false;
    static __device__ __forceinline__ bool tells(int) { return false; }

    static __host__ __device__ size_t lists_bytes(int tiles) { return (KIND == SHRINK ? (size_t)(tiles + 1) * 4 : 0) + (size_t)4 * 32 * kAddPitch * 4; }

    static __device__ __forceinline__ void prologue(const Args &a)
    {
        if (threadIdx.x == 0) { prefetch_map(&a.weights); prefetch_map(&a.tokens); }
        // Project begins while the kernel before it runs, and reads x and W before it has waited: that kernel, and the one before it,
        // let the next start only after their own wait, so whatever wrote x has completed.  Its epilogue waits for v.
        if (KIND == SHRINK || !a.ids) grid_dependency_wait();
        grid_launch_dependents();
    }
    static __device__ __forceinline__ void setup(const Args &a, uint8_t *p)
    {
        if (KIND == SHRINK)
            for (int i = threadIdx.x; i <= a.tiles; i += kThreads) ((int32_t *)p)[i] = __ldcg(a.at + i);
    }
    static __device__ __forceinline__ int tiles(const Args &a, uint8_t *p, int) { return KIND == SHRINK ? ((const int32_t *)p)[a.tiles] : a.row_tiles * a.tiles; }

    // Weight rows outermost, so that neighbouring tiles read the same weights.
    static __device__ __forceinline__ Tile tile(const Args &a, uint8_t *p, int q, int)
    {
        Tile t;
        if (KIND == SHRINK) {
            const int32_t *at = (const int32_t *)p;
            int lo = 0, hi = a.tiles - 1;       // the last token tile that begins at or before group q
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (at[mid] <= q) lo = mid;
                else hi = mid - 1;
            }
            t.which = lo;
            t.row = q - at[lo];                 // group of adapters
        } else {
            t.row = q / a.tiles;
            t.which = q % a.tiles;
        }
        t.parts = 1;
        t.off = t.which * a.cols;
        t.n = a.T - t.off < a.cols ? a.T - t.off : a.cols;
        t.n16 = (t.n + 15) & ~15;
        return t;
    }

    // SHRINK: the adapters of the group.
    static __device__ __forceinline__ int note_weights(const Args &a, uint8_t *, const Tile &t, int lane, int *rows)
    {
        if (KIND != SHRINK) return 0;
        const int left = __ldcg(a.found + t.which) - t.row * a.per_group, n = left < a.per_group ? left : a.per_group;
        if (lane < n) rows[lane] = __ldcg(&a.entries[(int64_t)t.which * kListThreads + t.row * a.per_group + lane]);
        return n;
    }

    static __device__ __forceinline__ void note_tokens(const Args &, uint8_t *, const Tile &, int, int *, int) {}
    static __device__ __forceinline__ uint32_t weight_bytes(const Args &a, int n) { return KIND == SHRINK ? (uint32_t)(n * a.rank) * (kChunk * 2) : kWeightBytes; }
    static __device__ __forceinline__ uint32_t token_bytes(const Args &a, const Tile &, int) { return a.cols * kChunk * 2; }
    static __device__ __forceinline__ uint32_t room(const Args &a, const Tile &) { return a.cols * kChunk * 2; }
    static __device__ __forceinline__ int depth(const Args &a, int) { return a.H; }
    static __device__ __forceinline__ int units_per_tile(const Args &a, int) { return a.units_per_tile; }
    static __device__ __forceinline__ void leave(const Args &, uint8_t *) {}
    static __device__ __forceinline__ bool wait_tokens(const Args &, uint8_t *, Shared *, const Tile &, int) { return true; }
    static __device__ __forceinline__ void early(const Args &, uint8_t *, int, int) {}
    static __device__ __forceinline__ uint16_t *claims(const Args &, uint8_t *) { return nullptr; }
    static __device__ __forceinline__ int claim(const Args &) { return 0; }
    static __device__ __forceinline__ void tell(const Args &, uint8_t *, const Tile &) {}

    static __device__ __forceinline__ void load_weights(const Args &a, const Tile &t, const int *rows, int n, int k, uint32_t addr, uint64_t *bar, int)
    {
        if (KIND == SHRINK) {
            for (int i = 0; i < n; ++i) load_tile<3>(addr + i * a.rank * (kChunk * 2), &a.weights, bar, k * kChunk, 0, rows[i]);
        } else load_tile<2>(addr, &a.weights, bar, k * kChunk, t.row * kRows);
    }
    static __device__ __forceinline__ void load_tokens(const Args &a, const Tile &t, const int *, int k, uint32_t addr, uint64_t *bar, int)
    {
        load_tile<2>(addr, &a.tokens, bar, k * kChunk, t.off);
    }

    struct Cols { int adapter, rank; float scale; };     // SHRINK: the adapter this thread's row belongs to (-1: none), the rank it is
    static __device__ __forceinline__ Cols cols(const Args &a, uint8_t *, const Tile &t, int w, int lane)
    {
        Cols c;
        c.adapter = -1;
        c.rank = 0;
        c.scale = 1.0f;
        if (KIND == SHRINK) {
            const int i = (w * 32 + lane) / a.rank, at = t.row * a.per_group + i;
            c.rank = w * 32 + lane - i * a.rank;
            if (i < a.per_group && at < __ldcg(a.found + t.which)) {
                c.adapter = __ldcg(&a.entries[(int64_t)t.which * kListThreads + at]);
                if (a.scale) c.scale = __ldcg(a.scale + c.adapter);
            }
        }
        return c;
    }

    // PROJECT: the rows of B that `add` reads for these columns.
    static __device__ __forceinline__ void prefetch(const Args &a, const Tile &t, int lane, int c)
    {
        if (KIND != PROJECT || !a.ids || lane >= 16 || c + lane >= t.n) return;
        const int id = __ldg(a.ids + t.off + c + lane), rows = a.O - t.row * kRows < kRows ? a.O - t.row * kRows : kRows;
        if (id >= 0 && id < a.adapters)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;"
                         ::"l"(a.b + ((int64_t)id * a.O + t.row * kRows) * a.rank), "r"(rows * a.rank * 2) : "memory");
    }

    // PROJECT: values += B[adapter of token][row] . v[token], by warp products of 16 rows x 8 tokens x 16 ranks, two for the two terms of v.
    // One adapter at a time, and every token takes the column of its own only.  The 16 ranks of a step are dealt out so that a thread's
    // four are neighbours in memory, in both operands alike.  What costs is the latency of the loads: the next 16 tokens' ids and values
    // are asked for a turn ahead (values of more ranks than fit the registers by a load per cache line, to be found in L1), an adapter's rows
    // of B stay in registers while the 16 tokens have no other (prompts), and where they have several, four adapters' rows are asked
    // for at once.
    // Measured: 16 columns of a tile take 2900 cycles at rank 64 (32 products of about 80 cycles each: these instructions run at the rate of plain
    // multiply-adds here, dependent or not), 1100 to 1300 at rank 16 with a change of adapter in every third.
    static constexpr int kSteps = 4;            // sixteens of ranks held in registers: larger ranks read the rest as they go
    static __device__ __forceinline__ uint4 low_at(const Args &a, const Tile &t, int c, int n, int k, int lane)
    {
        const int token = c + 8 * n + (lane >> 2), r = k + (lane & 3) * 4;     // beyond the rank or the tokens: zeros
        return r < a.rank && token < t.n ? a.v[((int64_t)(t.off + token) * a.rank + r) >> 2] : make_uint4(0, 0, 0, 0);
    }
    static __device__ __forceinline__ void ask_low(const Args &a, const Tile &t, int c, int lane, uint4 (&x)[kSteps][2])
    {
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int n = 0; n < 2; ++n) x[j][n] = low_at(a, t, c, n, 16 * j, lane);
    }
    // Lane l: the adapter of token c + l mod 16; and, where `ask_low` does not get all, a touch of every cache line of the 16 tokens' values.
    static __device__ __forceinline__ int ask(const Args &a, const Tile &t, int c, int lane)
    {
        const int id = c + (lane & 15) < t.n ? __ldg(a.ids + t.off + c + (lane & 15)) : -1;
        const int tokens = t.n - c < 16 ? t.n - c : 16;
        const float *low = (const float *)a.v + (int64_t)(t.off + c) * a.rank;
        float unused;
        if (a.rank > 16 * kSteps)
            for (int i = lane * 32; i < tokens * a.rank; i += 32 * 32) asm volatile("ld.global.ca.f32 %0, [%1];" : "=f"(unused) : "l"(low + i));
        return id >= 0 && id < a.adapters ? id : -1;
    }
    static __device__ __forceinline__ bool adds(const Args &a) { return KIND == PROJECT && a.ids; }
    static __device__ __forceinline__ void add(const Args &a, uint8_t *p, const Tile &t, int w, int lane, int c, int step_cols, uint32_t dst, bool more)
    {
        constexpr int kAdapters = 4;
        const int group = lane >> 2, quad = lane & 3, row0 = t.row * kRows + w * 32 + group;
        const uint16_t *rows[4];                // this thread's rows of B of adapter 0, at its first rank
#pragma unroll
        for (int i = 0; i < 4; ++i) rows[i] = a.b + (int64_t)(row0 + 8 * i < a.O ? row0 + 8 * i : a.O - 1) * a.rank + quad * 4;
        const int64_t next = (int64_t)a.O * a.rank;
        int held = -1;                          // the adapter whose rows are in `b`
        uint2 b[kSteps][4];
        int ahead = c < t.n16 ? ask(a, t, c, lane) : -1;
        uint4 low[kSteps][2];                   // the next 16 tokens' values
        ask_low(a, t, c, lane, low);
#pragma unroll 1
        for (; c < t.n16; c += step_cols) {
            const int id = ahead;
            const bool here = c + (lane & 15) < t.n;
            if (c + step_cols < t.n16) ahead = ask(a, t, c + step_cols, lane);
            float sum[2][2][4];                 // [16 rows][8 tokens][row group: tokens 2 quad, 2 quad + 1; row group + 8: likewise]
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i >> 3][(i >> 2) & 1][i & 3] = 0.0f;
            unsigned todo = __ballot_sync(0xffffffffu, id >= 0) & 0xffffu;
            const int first = __shfl_sync(0xffffffffu, id, 0);
            if (todo && __all_sync(0xffffffffu, !here || id == first)) {
                if (held != first) {
                    held = first;
#pragma unroll
                    for (int j = 0; j < kSteps; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            b[j][i] = 16 * j + quad * 4 < a.rank ? __ldg((const uint2 *)(rows[i] + first * next + 16 * j)) : make_uint2(0, 0);
                }
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
                    if (16 * j < a.rank) {
#pragma unroll
                        for (int n = 0; n < 2; ++n) step(sum, n, b[j], low[j][n]);
                    }
#pragma unroll 1
                for (int k = 16 * kSteps; k < a.rank; k += 16) {
                    uint2 q[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) q[i] = k + quad * 4 < a.rank ? __ldg((const uint2 *)(rows[i] + first * next + k)) : make_uint2(0, 0);
#pragma unroll
                    for (int n = 0; n < 2; ++n) step(sum, n, q, low_at(a, t, c, n, k, lane));
                }
            } else if (todo) {
                held = -1;
                do {
                    int adapter[kAdapters];
                    unsigned own[kAdapters];
#pragma unroll
                    for (int q = 0; q < kAdapters; ++q) {
                        adapter[q] = __shfl_sync(0xffffffffu, id, todo ? __ffs(todo) - 1 : 0);
                        own[q] = todo ? __ballot_sync(0xffffffffu, id == adapter[q]) & 0xffffu : 0u;
                        todo &= ~own[q];
                    }
#pragma unroll 1
                    for (int k = 0; k < a.rank; k += 16) {
                        uint2 q[kAdapters][4];
#pragma unroll
                        for (int i = 0; i < kAdapters; ++i)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                q[i][r] = k + quad * 4 < a.rank && own[i] ? __ldg((const uint2 *)(rows[r] + adapter[i] * next + k)) : make_uint2(0, 0);
                        uint4 some[2];
#pragma unroll
                        for (int n = 0; n < 2; ++n) some[n] = low_at(a, t, c, n, k, lane);
#pragma unroll
                        for (int i = 0; i < kAdapters; ++i)
#pragma unroll
                            for (int n = 0; n < 2; ++n)
                                if (own[i] >> (8 * n) & 0xffu) {
                                    float part[2][2][4];
#pragma unroll
                                    for (int r = 0; r < 4; ++r) part[0][n][r] = part[1][n][r] = 0.0f;
                                    step(part, n, q[i], some[n]);
#pragma unroll
                                    for (int r = 0; r < 4; ++r)
                                        if (own[i] >> (8 * n + 2 * quad + (r & 1)) & 1u) { sum[0][n][r] += part[0][n][r]; sum[1][n][r] += part[1][n][r]; }
                                }
                    }
                } while (todo);
            }
            ask_low(a, t, c + step_cols, lane, low);
            // from the products' layout to one row per lane
            float *s = (float *)p + w * 32 * kAddPitch, v[16];
            __syncwarp();
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[(16 * m + 8 * (i >> 1) + group) * kAddPitch + 8 * n + 2 * quad + (i & 1)] = sum[m][n][i];
            if (more) read16(dst + c, v);
            else {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = 0.0f;
            }
            __syncwarp();
            float *mine = s + lane * kAddPitch, d[16], odd = 0.0f;         // odd: NaN if one of them is (or infinities of both signs are among them)
#pragma unroll
            for (int i = 0; i < 16; ++i) d[i] = mine[i];
#pragma unroll
            for (int i = 0; i < 16; i += 4) odd += (d[i] + d[i + 1]) + (d[i + 2] + d[i + 3]);
            if (__any_sync(0xffffffffu, odd != odd)) {
                infinite(a, t, t.row * kRows + w * 32 + lane, id, c, mine);
#pragma unroll
                for (int i = 0; i < 16; ++i) d[i] = mine[i];
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] += d[i];
            write16(dst + c, v);
        }
    }
    // The products take v's two terms one after the other: an infinity of B becomes NaN where the second term is 0 or has the other
    // sign.  A row's values that are NaN are made again from the terms' sum; `id` as in `add`.
    static __device__ __forceinline__ void infinite(const Args &a, const Tile &t, int row, int id, int c, float *values)
    {
        const uint16_t *rows = a.b + (int64_t)(row < a.O ? row : a.O - 1) * a.rank;
#pragma unroll 1
        for (int i = 0; i < 16; ++i) {
            const int adapter = __shfl_sync(0xffffffffu, id, i);
            if (adapter < 0 || values[i] == values[i]) continue;
            const uint16_t *b = rows + (int64_t)adapter * a.O * a.rank, *v = (const uint16_t *)(a.v + ((int64_t)(t.off + c + i) * a.rank >> 2));
            float f = 0.0f;
#pragma unroll 1
            for (int k = 0; k < a.rank; ++k) {
                const uint16_t *p = v + (k >> 2) * 8 + (k & 3);
                f = fmaf(__uint_as_float((uint32_t)__ldg(b + k) << 16), __uint_as_float((uint32_t)p[0] << 16) + __uint_as_float((uint32_t)p[4] << 16), f);
            }
            values[i] = f;
        }
    }
    static __device__ __forceinline__ void step(float (&d)[2][2][4], int n, const uint2 (&b)[4], const uint4 &low)
    {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            product(d[m][n], b[2 * m], b[2 * m + 1], low.x, low.y);
            product(d[m][n], b[2 * m], b[2 * m + 1], low.z, low.w);
        }
    }
    // d += the 16 x 16 left operand (rows `group` and `group` + 8, four ranks each) times the 16 x 8 right one.
    static __device__ __forceinline__ void product(float (&d)[4], const uint2 &r0, const uint2 &r8, uint32_t x0, uint32_t x1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(r0.x), "r"(r8.x), "r"(r0.y), "r"(r8.y), "r"(x0), "r"(x1));
    }

    static __device__ __forceinline__ void store(const Args &a, uint8_t *p, const Tile &t, const Cols &cols, int w, int lane, int c, const float (&v)[16], int)
    {
        const int row = w * 32 + lane;
        if (KIND == SHRINK) {
            // a short loop over values in shared memory: its instructions are run once or twice, and fetching them all unrolled took longer
            float *mine = (float *)(p + a.values_at) + row * kAddPitch;
#pragma unroll
            for (int i = 0; i < 16; ++i) mine[i] = v[i];
            const int ids = c + (lane & 15) < t.n ? __ldg(a.ids + t.off + c + (lane & 15)) : -1;
            uint16_t *to = (uint16_t *)(a.v + (((int64_t)(t.off + c) * a.rank + (cols.rank & ~3)) >> 2)) + (cols.rank & 3);
#pragma unroll 1
            for (int i = 0; i < 16; ++i, to += a.rank * 2) {
                const int id = __shfl_sync(0xffffffffu, ids, i);
                if (id == cols.adapter && id >= 0) split_low(cols.scale * mine[i], to[0], to[4]);
            }
        } else {
            const int o = t.row * kRows + row;
            if (a.y_wide && t.row * kRows + w * 32 + 32 <= a.O) {
                // bf16 rows on 16-byte boundaries: turned over in shared memory, so that two lanes have a token's 32 values
                float *turn = (float *)p + w * 32 * kAddPitch;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 16; ++i) turn[lane * kAddPitch + i] = v[i];
                __syncwarp();
                const int token = lane >> 1, half = lane & 1;
                uint32_t q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float *r = turn + (half * 16 + 2 * i) * kAddPitch + token;
                    q[i] = (uint32_t)f32_to_bf16(r[0]) | (uint32_t)f32_to_bf16(r[kAddPitch]) << 16;
                }
                if (c + token < t.n) {
                    uint4 *dst = (uint4 *)(a.y + (int64_t)(t.off + c + token) * a.y_stride + (t.row * kRows + w * 32 + half * 16) * 2);
                    dst[0] = make_uint4(q[0], q[1], q[2], q[3]);
                    dst[1] = make_uint4(q[4], q[5], q[6], q[7]);
                }
            } else if (o < a.O) {
                uint8_t *dst = a.y + (int64_t)(t.off + c) * a.y_stride + (int64_t)o * (a.y_f32 ? 4 : 2);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (c + i < t.n) {
                        if (a.y_f32) *(float *)dst = v[i];
                        else *(uint16_t *)dst = f32_to_bf16(v[i]);
                    }
                    dst += a.y_stride;
                }
            }
        }
    }
};

inline size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }
inline int round16(int n) { return (n + 15) & ~15; }
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// The tokens' ring holds as many stages as the weights have slots.
inline size_t ring_for(int cols, int steps)
{
    const size_t stage = (size_t)(kRows + cols) * kChunk * 2 * steps, n = (kSmem - 16 * 1024) / stage;
    return (n < (size_t)kSlots ? n : (size_t)kSlots) * cols * kChunk * 2 * steps;
}

// Tokens per tile: as even as can be, so that the last tile is about as full as the others.
inline int tile_cols(int T) { return round16(ceil_div(T, ceil_div(T, kMaxCols))); }

bool make_maps(mw_project *m)
{
    const mw_project_config &c = m->cfg;
    const uint64_t H = c.H, O = c.O, r = c.rank, n = c.adapters;
    const uint64_t wd[2] = {H, O}, ws[1] = {H * 2};
    const uint32_t wb[2] = {kChunk, kRows};
    if (!encode_map(&m->map_w, m->w, 2, wd, ws, wb)) return false;
    if (!n) return true;
    const uint64_t ad[3] = {H, r, n}, as[2] = {H * 2, r * H * 2};
    const uint32_t ab[3] = {kChunk, (uint32_t)r, 1};
    return encode_map(&m->map_a, m->a, 3, ad, as, ab);
}

}  // namespace

extern "C" {

int mw_project_create(mw_project **out, const mw_project_config *cfg, const void *w, const void *a, const void *b, const float *scale)
{
    if (!out) return MW_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || !w) return MW_ERR_INVALID_ARG;
    if (cfg->H < 8 || cfg->H % 8 || cfg->H > MW_PROJECT_MAX_WIDTH || cfg->O < 1 || cfg->O > MW_PROJECT_MAX_WIDTH || cfg->max_tokens < 1 ||
        cfg->max_tokens > MW_PROJECT_MAX_TOKENS || cfg->adapters < 0 || cfg->device < 0 ||
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
    m->w = w; m->a = a; m->b = b; m->scale = scale;
    cudaDeviceGetAttribute(&m->sm_count, cudaDevAttrMultiProcessorCount, cfg->device);
    const size_t tiles = (size_t)ceil_div(cfg->max_tokens, kListThreads);
    // parts: of a tile of project, and of shrink where max_tokens allows it
    const int cols = cfg->max_tokens < kMaxCols ? round16(cfg->max_tokens < kListThreads ? kListThreads : cfg->max_tokens) : kMaxCols;
    const size_t b_counts = round256((size_t)m->sm_count * 4), b_tiles = round256((tiles + 1) * 4);
    const size_t b_v = round256((size_t)cfg->max_tokens * cfg->rank * 4), b_entries = cfg->adapters ? tiles * kListThreads * 4 : 0;
    const size_t zeroed = 512 + b_counts, bytes = zeroed + b_v + 2 * b_tiles + b_entries + 2 * (size_t)m->sm_count * cols * kRows * 4;
    if (cudaMalloc(&m->slab, bytes) != cudaSuccess) { cudaGetLastError(); delete m; return MW_ERR_CUDA; }
    uint8_t *p = (uint8_t *)m->slab;
    m->status = (int32_t *)p; p += 256;
    m->done = (unsigned int *)p; p += 256;
    m->counts = (unsigned int *)p; p += b_counts;
    m->v = (uint4 *)p; p += b_v;
    m->found = (int32_t *)p; p += b_tiles;
    m->at = (int32_t *)p; p += b_tiles;
    m->entries = (int32_t *)p; p += b_entries;
    m->parts = (float *)p;
    int rc = MW_OK;
    if (cudaMemset(m->slab, 0, zeroed) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) rc = MW_ERR_CUDA;
    if (rc == MW_OK && (cudaFuncSetAttribute(k_stream<Product<SHRINK>>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) != cudaSuccess ||
                        cudaFuncSetAttribute(k_stream<Product<PROJECT>>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) != cudaSuccess))
        rc = MW_ERR_CUDA;
    if (rc == MW_OK && !make_maps(m)) rc = MW_ERR_CUDA;
    if (rc != MW_OK) { cudaGetLastError(); mw_project_destroy(m); return rc; }
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
    const mw_project_config &c = m->cfg;
    const int ye = y_dtype == MW_DTYPE_F32 ? 4 : 2;
    const int64_t xrow = (int64_t)c.H * 2, yrow = (int64_t)c.O * ye;
    if ((x_stride_bytes && x_stride_bytes < xrow) || (y_stride_bytes && y_stride_bytes < yrow)) return MW_ERR_INVALID_ARG;
    if ((((uintptr_t)x | (uint64_t)x_stride_bytes) & 15u) || ((uintptr_t)y | (uint64_t)y_stride_bytes) % ye || ((uintptr_t)adapter_ids & 3u))
        return MW_ERR_ALIGNMENT;
    cudaStream_t st = (cudaStream_t)stream;
    const bool overlap = !(c.flags & MW_FLAG_NO_OVERLAP);
    // Steps per unit, 4 / 2 / 1: one token 24.0 / 24.8 / 29.9 us, 16 tokens 25.3 / 26.8 / 33, 64 tokens - / 31 / 42, 96 tokens (4096 x 4096) - / 28.4 / 27.3,
    // 256 tokens - / 67.7 / 65.1, at rank 16 in 7168 x 7168.  A unit's fixed cost asks for more, the shared memory left for others in flight for fewer.
    const int cols = tile_cols(T), tiles = ceil_div(T, cols), steps = cols <= 32 ? 4 : cols <= 64 ? 2 : 1;
    const int units_per_tile = ceil_div(c.H, kChunk * steps);
    cudaError_t e = cudaSuccess;

    Product<PROJECT>::Args g = {};
    const uint64_t xd[2] = {(uint64_t)c.H, (uint64_t)T}, xs[1] = {(uint64_t)(x_stride_bytes ? x_stride_bytes : xrow)};
    const uint32_t xb[2] = {kChunk, (uint32_t)cols};
    if (!encode_map(&g.tokens, x, 2, xd, xs, xb)) return MW_ERR_INVALID_ARG;
    g.weights = m->map_w;
    g.ids = c.adapters ? adapter_ids : nullptr;
    g.c.steps = steps;
    split_memory(&g.c, kSmem - Product<PROJECT>::lists_bytes(tiles), ring_for(cols, steps));
    // up to 128 tokens TMEM has room for the additions, and they are made while the products run (made after them: one token 25.4 us instead of 24.0,
    // 64 tokens 42 instead of 31, 128 tokens 61 instead of 44, at rank 16 in 7168 x 7168)
    g.c.acc_cols = cols;
    g.c.add_col = g.ids && cols <= kMaxCols / 2 ? 2 * cols : 0;
    g.c.tmem_cols = 32;
    while ((int)g.c.tmem_cols < (g.c.add_col ? 3 : 2) * cols) g.c.tmem_cols *= 2;
    g.c.wait_limit = (c.flags & MW_FLAG_SHORT_WAITS) ? (1 << 10) : (1 << 20);
    g.c.skew = m->skew;
    m->skew = 0;
    g.c.wait_first = (c.flags & MW_FLAG_SHORT_WAITS) != 0;
    g.c.min_units = 2;
    g.c.shares = m->sm_count;
    g.c.part_cols = cols;
    g.c.parts = m->parts; g.c.counts = m->counts; g.c.status = m->status;
    g.T = T; g.cols = cols; g.tiles = tiles; g.adapters = c.adapters; g.rank = c.rank;
    g.row_tiles = ceil_div(c.O, kRows); g.units_per_tile = units_per_tile; g.per_group = c.adapters ? kRows / c.rank : 1; g.H = c.H; g.O = c.O;
    g.b = (const uint16_t *)m->b; g.v = m->v;
    g.y = (uint8_t *)y; g.y_stride = y_stride_bytes ? y_stride_bytes : yrow; g.y_f32 = ye == 4;
    g.y_wide = ye == 2 && !(((uintptr_t)y | (uint64_t)g.y_stride) & 15u);
    if (g.ids && (int64_t)T * c.rank <= kDirect) {
        LowArgs l;
        l.ids = adapter_ids; l.x = (const uint8_t *)x; l.x_stride = (int64_t)xs[0]; l.a = (const uint16_t *)m->a; l.scale = m->scale; l.v = m->v;
        l.adapters = c.adapters; l.rank = c.rank; l.H = c.H; l.status = m->status;
        e = mw_launch(k_project_low, dim3(c.rank / 4, T), dim3(kLowThreads), 0, st, overlap, l);
        m->launches += 1;
    }
    else if (adapter_ids) {
        const int list_tiles = ceil_div(T, kListThreads), per_group = c.adapters ? kRows / c.rank : 1;
        ListArgs l;
        l.ids = adapter_ids; l.T = T; l.tiles = list_tiles; l.adapters = c.adapters; l.per_group = per_group;
        l.found = m->found; l.at = m->at; l.entries = m->entries; l.done = m->done; l.status = m->status;
        e = mw_launch(k_adapter_lists, dim3(list_tiles), dim3(kListThreads), 0, st, overlap, l);
        m->launches += 1;
        if (g.ids) {
            Product<SHRINK>::Args s = {};
            const uint32_t sb[2] = {kChunk, kListThreads};
            if (!encode_map(&s.tokens, x, 2, xd, xs, sb)) return MW_ERR_INVALID_ARG;
            s.weights = m->map_a; s.c = g.c;
            s.c.steps = 2;
            s.c.min_units = 4;
            s.values_at = (list_tiles + 1) * 4;
            s.c.acc_cols = kListThreads; s.c.add_col = 0; s.c.tmem_cols = 2 * kListThreads;
            split_memory(&s.c, kSmem - Product<SHRINK>::lists_bytes(list_tiles), ring_for(kListThreads, 2));
            s.ids = adapter_ids; s.T = T; s.cols = kListThreads; s.tiles = list_tiles; s.adapters = c.adapters; s.rank = c.rank;
            s.units_per_tile = ceil_div(c.H, kChunk * 2); s.per_group = per_group; s.H = c.H; s.O = c.O;
            s.found = m->found; s.at = m->at; s.entries = m->entries; s.scale = m->scale; s.v = m->v;
            if (e == cudaSuccess) e = mw_launch(k_stream<Product<SHRINK>>, dim3(m->sm_count), dim3(kThreads), kSmem, st, overlap, s);
            m->launches += 1;
        }
    }
    if (e == cudaSuccess) e = mw_launch(k_stream<Product<PROJECT>>, dim3(m->sm_count), dim3(kThreads), kSmem, st, overlap, g);
    if (e != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
    m->launches += 1;
    return MW_OK;
}

int mw_project_get_status(mw_project *m, int32_t *status, void *stream)
{
    if (!m || !status) return MW_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemcpyAsync(status, m->status, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(m->status, 0, 4, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return MW_ERR_CUDA;
    // a wait that gave up may have left tiles half counted
    if (*status == MW_ERR_TIMEOUT && (cudaMemsetAsync(m->done, 0, 256 + (size_t)m->sm_count * 4, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess))
        return MW_ERR_CUDA;
    return MW_OK;
}

int mw_project_test_skew_waits(mw_project *m)
{
    if (!m) return MW_ERR_INVALID_ARG;
    m->skew = 16;
    return MW_OK;
}

int64_t mw_project_kernel_launches(const mw_project *m) { return m ? m->launches : 0; }

}  // extern "C"
