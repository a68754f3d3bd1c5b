// The experts of one rank for few tokens: y[t] = sum_k w[t,k] W_down[e] (silu(W_gate[e] x[t]) * (W_up[e] x[t])).
// Declared in include/mw.h.
//
// Two launches: the products of both layers, and the weighted sum over a token's picks.  A pick is a (token, slot) pair.  Every block lists
// the picks by expert for itself in shared memory (a microsecond or two; a kernel of its own would cost a launch before the first weight can be
// asked for), in the same order everywhere.  Activations are stored in that order, and rows of x copied into it, so that an expert's
// tokens are neighbours (up to sixteen tokens of x are gathered where they lie, as the copy would be waited for: one token on 8 experts 120.8 us instead of 122.1); output rows by pick, so that the sum runs in slot order.
// Inside the first launch the products' tokens wait, expert by expert, for a count of copied pieces and of finished tiles; the weights do not
// wait, and HBM stays busy from one product to the other.  The counts are kept twice, and the launch clears the next one's.
// Blocks take their shares of the products, and their parts of the copies, by tickets, in an order in which nothing waits for
// what comes later: a call ends also when only some of its blocks get an SM at a time (a partition of the device, calls on other streams).
//
// Bound: HBM, the weights of every chosen expert once.  Measured (H 7168, I 2048): one token on 8 experts 121 us (705 MB, 5.8 TB/s), 64 tokens on about 222 of 256
// experts 2.9 ms (19.6 GB, 6.7 to 7.0 TB/s, what a kernel that only reads reaches), 201 tokens on 4 experts 83 us (358 MB, 4.3 TB/s): of these 35 us stream the first
// product's weights at 6.7 TB/s, 9 us go before the first product (lists, copies of x), about 12 pass from the last tiles of gate and up to the first
// of down, 5 for the sum; the rest is down at 5 TB/s, half of it on the 76 CTAs that have a second tile.
#include <new>
#include <string.h>

#include "mw_stream.cuh"

using namespace mw_stream;

struct mw_experts {
    mw_experts_config cfg;
    const void *w_gate_up, *w_down;
    CUtensorMap map_gate_up, map_down, map_rows, map_rows_few, map_act, map_act_few;
    void *slab;
    int32_t *status;
    uint16_t *rows;             // [max_tokens * K, H] bf16: x in the order of the list
    uint16_t *act;              // [max_tokens * K, I] bf16, likewise
    float *out;                 // [max_tokens * K, H], by pick
    float *parts;
    unsigned int *counts;
    unsigned int *state;        // [kHead]: launches so far, blocks that have left, tickets of shares and of copies; then [2][2][expert_count]: copied pieces, finished tiles of gate and up
    int sm_count;
    int skew;                   // bytes added to the announced size of the next call's loads of weights (test hook)
    int blocks;                 // blocks of the next call's first launch, 0: one per SM (test hook)
    int64_t launches;
};

namespace {

enum { kLaunch, kLeft, kShareTicket, kCopyTicket, kHead };     // mw_experts::state

constexpr size_t kSmem = 227 * 1024 - 512;      // dynamic shared memory of a block (a few bytes are static)
constexpr int kSumThreads = 128;
constexpr size_t kMinRing = 64 * 1024;          // of the tokens' ring: a stage of 256 tokens

// Shared-memory lists: per expert the exclusive prefix sums of (token tiles << 16 | picks), then the picks grouped by expert,
// ascending (a tile may be cut between blocks, so every block has to list them in the same order); the rest is scratch of setup.
struct Lists {
    uint32_t *launch;           // the launch's number
    uint32_t *copies;           // the copies' ticket of this block's first worker; no worker's number where all tokens are gathered
    uint32_t *prefix;           // [count + 1]
    uint16_t *picks;            // [picks]
    uint16_t *local;            // [picks]         expert of each pick, 0xffff = none here
    uint16_t *seen;             // [warps][count]  picks of the expert in the warp's part, then where the warp's next one goes
    uint16_t *claims;           // [2 * shares + 1]  shares this block has taken, as numbers (share_of); 2 * shares and more: none was left
};
__host__ __device__ inline size_t lists_bytes(int count, int picks, int shares)
{
    return ((size_t)(count + 3) * 4 + (size_t)picks * 4 + (size_t)count * (kThreads / 32) * 2 + (size_t)(2 * shares + 1) * 2 + 15) & ~(size_t)15;
}

struct ExpertArgs {
    CUtensorMap gate_up, down;
    CUtensorMap rows, rows_few, act_box, act_few;   // tokens in boxes of 64 and of 16 rows
    CUtensorMap x_row;                              // x itself, one row at a time
    Common c;
    const int32_t *ids;
    const uint8_t *x;
    int64_t x_stride;
    int picks, K, E, first, count;
    int max_cols;               // tokens per tile
    int H, I;
    uint16_t *sorted;           // x in the order of the list
    uint16_t *act;
    float *out;
    unsigned int *state;
};

// Product 0: gate and up, 1: down.
struct Product {
    using Args = ExpertArgs;
    static constexpr int kProducts = 2;
    static constexpr bool kEarly = true, kLate = true, kAdds = false, kClaims = true;
    static constexpr int kWorkers = 5;          // warps that copy rows of x
    static __device__ __forceinline__ bool tells(int product) { return product == 0; }

    static __device__ __forceinline__ int row_tiles(const Args &a, int product) { return product ? (a.H + kRows - 1) / kRows : (a.I + kRows / 2 - 1) / (kRows / 2); }
    static __device__ __forceinline__ int depth(const Args &a, int product) { return product ? a.I : a.H; }
    static __device__ __forceinline__ int units_per_tile(const Args &a, int product) { return (depth(a, product) + kChunk * a.c.steps - 1) / (kChunk * a.c.steps); }

    static __device__ __forceinline__ Lists lists_at(const Args &a, uint8_t *p)
    {
        uint32_t *u = (uint32_t *)p;
        uint16_t *q = (uint16_t *)(u + a.count + 3), *seen = q + 2 * a.picks;
        return {u, u + 1, u + 2, q, q + a.picks, seen, seen + (kThreads / 32) * a.count};
    }
    static __device__ __forceinline__ uint16_t *claims(const Args &a, uint8_t *p) { return lists_at(a, p).claims; }
    static __device__ __forceinline__ int claim(const Args &a) { return (int)atomicAdd(a.state + kShareTicket, 1u); }
    static __device__ __forceinline__ int expert_of(const Args &a, int id)
    {
        const int e = id - a.first;
        return id >= 0 && id < a.E && e >= 0 && e < a.count ? e : -1;
    }

    static __device__ __forceinline__ void prologue(const Args &a)
    {
        if (threadIdx.x < 7) prefetch_map(&a.gate_up + threadIdx.x);
        grid_dependency_wait();
        grid_launch_dependents();
    }
    static __device__ __forceinline__ void leave(const Args &a, uint8_t *p)
    {
        if (threadIdx.x == 0 && atomicInc(a.state + kLeft, gridDim.x - 1) == gridDim.x - 1) {
            a.state[kLaunch] = *lists_at(a, p).launch + 1;
            a.state[kShareTicket] = a.state[kCopyTicket] = 0;
        }
    }

    // Counting sort of the picks by expert, stable: warp w takes the w-th part of the picks, counts each expert in it, and after a
    // scan over (expert, warp) places them; lanes with the same expert order themselves by lane.
    static __device__ __forceinline__ void setup(const Args &a, uint8_t *p)
    {
        constexpr int kWarps = kThreads / 32;
        __shared__ uint32_t warp_sums[kWarps];
        const Lists l = lists_at(a, p);
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        const int steps = (a.picks + kThreads - 1) / kThreads, part = warp * steps * 32;
        uint16_t *seen = l.seen + warp * a.count;
        uint32_t launch = 0, share = 0, copies = 0;
        if (threadIdx.x == 0) {
            launch = __ldcg(a.state + kLaunch);
            share = claim(a);
            copies = atomicAdd(a.state + kCopyTicket, (unsigned)kWorkers);
        }
        for (int i = threadIdx.x; i < 2 * a.c.shares; i += kThreads) l.claims[i + 1] = kNoShare;
        constexpr int kBatch = 8;               // ids asked for at once
        for (int i0 = 0; i0 < steps; i0 += kBatch) {
            int id[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int at = part + (i0 + i) * 32 + lane;
                id[i] = i0 + i < steps && at < a.picks ? __ldcg(a.ids + at) : -1;
            }
            if (i0 == 0) {
                for (int e = threadIdx.x; e < a.count * kWarps; e += kThreads) l.seen[e] = 0;
                __syncthreads();
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                if (i0 + i >= steps) break;
                const int at = part + (i0 + i) * 32 + lane, e = expert_of(a, id[i]);
                if (at < a.picks) l.local[at] = (uint16_t)e;
                if (blockIdx.x == 0 && (id[i] < -1 || id[i] >= a.E)) atomicCAS(a.c.status, MW_OK, MW_ERR_BAD_INDEX);
                const unsigned same = __match_any_sync(0xffffffffu, e);
                if (e >= 0 && lane == __ffs(same) - 1) seen[e] += (uint16_t)__popc(same);
                __syncwarp();
            }
        }
        if (threadIdx.x == 0) *l.launch = launch;
        __syncthreads();
        const int per = (a.count + kThreads - 1) / kThreads, begin = threadIdx.x * per;
        uint32_t sum = 0, most = 0;             // (of an expert: its picks)
        for (int e = begin; e < begin + per && e < a.count; ++e) {
            uint32_t n = 0;
            for (int w = 0; w < kWarps; ++w) {
                const uint32_t k = l.seen[w * a.count + e];
                l.seen[w * a.count + e] = (uint16_t)n;
                n += k;
            }
            l.prefix[e] = ((n + a.max_cols - 1) / a.max_cols) << 16 | n;
            most = n > most ? n : most;
            sum += l.prefix[e];
        }
        uint32_t incl = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += v;
        }
        if (lane == 31) warp_sums[warp] = incl;
        const bool copying = __syncthreads_or(most > kFew);
        uint32_t run = incl - sum;
        for (int w = 0; w < warp; ++w) run += warp_sums[w];
        for (int e = begin; e < begin + per && e < a.count; ++e) {
            const uint32_t n = l.prefix[e];
            l.prefix[e] = run;
            run += n;
            if (e == a.count - 1) l.prefix[a.count] = run;
        }
        __syncthreads();
        for (int i = 0; i < steps; ++i) {
            const int at = part + i * 32 + lane;
            const int e = at < a.picks ? (int)(int16_t)l.local[at] : -1;
            const unsigned same = __match_any_sync(0xffffffffu, e);
            if (e >= 0) l.picks[(l.prefix[e] & 0xffffu) + seen[e] + __popc(same & ((1u << lane) - 1))] = (uint16_t)at;
            __syncwarp();
            if (e >= 0 && lane == __ffs(same) - 1) seen[e] += (uint16_t)__popc(same);
            __syncwarp();
        }
        // (*launch is visible: there were barriers since)
        unsigned int *next = a.state + kHead + ((*l.launch + 1) & 1) * 2 * a.count;
        for (int e = blockIdx.x * kThreads + threadIdx.x; e < 2 * a.count; e += gridDim.x * kThreads) next[e] = 0;
        if (threadIdx.x == 0) { l.claims[0] = (uint16_t)share; *l.copies = copying ? copies : kWorkers * a.c.shares; }
    }

    static __device__ __forceinline__ int tiles(const Args &a, uint8_t *p, int product) { return (int)(lists_at(a, p).prefix[a.count] >> 16) * row_tiles(a, product); }

    // Experts in order; inside one, the row tiles in order with its token tiles (nearly always one) innermost.
    static __device__ __forceinline__ Tile tile(const Args &a, uint8_t *p, int q, int product)
    {
        const Lists l = lists_at(a, p);
        const int rows = row_tiles(a, product);
        int lo = 0, hi = a.count - 1;           // the last expert that begins at or before tile q
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((int)(l.prefix[mid] >> 16) * rows <= q) lo = mid;
            else hi = mid - 1;
        }
        const uint32_t from = l.prefix[lo], to = l.prefix[lo + 1];
        const int parts = (int)((to >> 16) - (from >> 16)), in = q - (int)(from >> 16) * rows;
        const int n = (int)((to & 0xffffu) - (from & 0xffffu)), j = parts == 1 ? 0 : in % parts;
        Tile t;
        t.row = parts == 1 ? in : in / parts;
        t.which = lo;
        t.parts = parts;
        t.off = (int)(from & 0xffffu) + j * a.max_cols;
        t.n = n - j * a.max_cols < a.max_cols ? n - j * a.max_cols : a.max_cols;
        t.n16 = (t.n + 15) & ~15;
        return t;
    }
    static __device__ __forceinline__ int note_weights(const Args &, uint8_t *, const Tile &, int, int *) { return 0; }
    static __device__ __forceinline__ uint32_t weight_bytes(const Args &, int) { return kWeightBytes; }
    // Gate and up with few tokens: their rows of x; a last group of four that is not full repeats the last token.
    static __device__ __forceinline__ bool gathers(const Tile &t, int product) { return product == 0 && t.parts == 1 && t.n <= kFew; }
    static __device__ __forceinline__ void note_tokens(const Args &a, uint8_t *p, const Tile &t, int lane, int *rows, int product)
    {
        if (gathers(t, product) && lane < kFew) rows[lane] = lists_at(a, p).picks[t.off + (lane < t.n ? lane : t.n - 1)] / a.K;
    }
    static __device__ __forceinline__ uint32_t token_bytes(const Args &, const Tile &t, int product) { return (gathers(t, product) ? (t.n + 3) & ~3 : t.n16) * kChunk * 2; }
    static __device__ __forceinline__ uint32_t room(const Args &, const Tile &t) { return t.n16 * kChunk * 2; }

    static __device__ __forceinline__ void load_weights(const Args &a, const Tile &t, const int *, int, int k, uint32_t addr, uint64_t *bar, int product)
    {
        // gate and up rows interleaved in sixteens: rows 32 g ... 32 g + 15 of the tile are gate rows, the next 16 the up rows of the same values
        if (product) load_tile<3>(addr, &a.down, bar, k * kChunk, t.row * kRows, t.which);
        else load_tile<5>(addr, &a.gate_up, bar, k * kChunk, 0, 0, t.row * (kRows / 32), t.which);
    }
    // (The last box may reach into the next expert's rows or past the end: columns that nobody reads.)
    static __device__ __forceinline__ void load_tokens(const Args &a, const Tile &t, const int *rows, int k, uint32_t addr, uint64_t *bar, int product)
    {
        int c = 0;
        if (gathers(t, product)) {
            for (; c < t.n; c += 4) {
                const int4 r = *(const int4 *)(rows + c);
                gather4(addr + c * (kChunk * 2), &a.x_row, bar, k * kChunk, r.x, r.y, r.z, r.w);
            }
            return;
        }
        for (; c + 64 <= t.n16; c += 64) load_tile<2>(addr + c * (kChunk * 2), product ? &a.act_box : &a.rows, bar, k * kChunk, t.off + c);
        for (; c < t.n16; c += 16) load_tile<2>(addr + c * (kChunk * 2), product ? &a.act_few : &a.rows_few, bar, k * kChunk, t.off + c);
    }

    // This launch's counts of copied pieces (0) and of finished tiles (1).
    static __device__ __forceinline__ unsigned int *counts(const Args &a, uint8_t *p, int which)
    {
        return a.state + kHead + ((*lists_at(a, p).launch & 1) * 2 + which) * a.count;
    }
    // Rows of x to the order of the list, in pieces of 2 KB, the first expert's first.  They are dealt out to kWorkers times as many workers as
    // there are shares; the warps of a block are the workers that its ticket names, then any that nobody has been yet.
    static constexpr int kPiece = 4 * 32;       // 16-byte values
    static __device__ __forceinline__ int pieces(const Args &a) { return (a.H / 8 + kPiece - 1) / kPiece; }
    static __device__ __forceinline__ void early(const Args &a, uint8_t *p, int w, int lane)
    {
        const Lists l = lists_at(a, p);
        unsigned int *done = counts(a, p, 0);
        const int workers = kWorkers * a.c.shares, per_row = pieces(a), all = (int)(l.prefix[a.count] & 0xffffu) * per_row, n = a.H / 8;
        for (int worker = (int)*l.copies + w; worker < workers;) {
            for (int i = worker; i < all; i += workers) {
                const int at = i / per_row, first = (i - at * per_row) * kPiece + lane, pick = l.picks[at], e = l.local[pick];
                if (((l.prefix[e + 1] - l.prefix[e]) & 0xffffu) <= kFew) continue;
                const uint4 *src = (const uint4 *)(a.x + (int64_t)(pick / a.K) * a.x_stride);
                uint4 *dst = (uint4 *)(a.sorted + (int64_t)at * a.H);
                uint4 q[kPiece / 32];
#pragma unroll
                for (int j = 0; j < kPiece / 32; ++j) if (first + 32 * j < n) q[j] = __ldg(src + first + 32 * j);
#pragma unroll
                for (int j = 0; j < kPiece / 32; ++j) if (first + 32 * j < n) dst[first + 32 * j] = q[j];
                __threadfence();
                __syncwarp();
                if (lane == 0) atomicAdd(done + e, 1u);
            }
            if (lane == 0) worker = (int)atomicAdd(a.state + kCopyTicket, 1u);
            worker = __shfl_sync(0xffffffffu, worker, 0);
        }
    }
    // Waits until the expert's rows of x are copied / all tiles of its gate and up products are stored.
    static __device__ __forceinline__ bool wait_tokens(const Args &a, uint8_t *p, Shared *s, const Tile &t, int product)
    {
        if (gathers(t, product)) return true;
        const Lists l = lists_at(a, p);
        const unsigned int *done = counts(a, p, product) + t.which;
        const unsigned int all = product ? (unsigned int)(row_tiles(a, 0) * t.parts)
                                      : ((l.prefix[t.which + 1] - l.prefix[t.which]) & 0xffffu) * (unsigned int)pieces(a);
        bool ok = false;
        for (int i = 0; i < a.c.wait_limit && !ok && !s->abort; ++i) {
            unsigned int n;
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(n) : "l"(done) : "memory");
            ok = n == all;
        }
        if (!ok && !s->abort) { s->abort = 1; atomicExch(a.c.status, MW_ERR_TIMEOUT); }
        ok = __all_sync(0xffffffffu, ok);
        asm volatile("fence.proxy.async;" ::: "memory");
        return ok;
    }
    static __device__ __forceinline__ void tell(const Args &a, uint8_t *p, const Tile &t) { atomicAdd(counts(a, p, 1) + t.which, 1u); }

    struct Cols {};
    static __device__ __forceinline__ Cols cols(const Args &, uint8_t *, const Tile &, int, int) { return {}; }

    static __device__ __forceinline__ void prefetch(const Args &, const Tile &, int, int) {}
    static __device__ __forceinline__ bool adds(const Args &) { return false; }
    static __device__ __forceinline__ void add(const Args &, uint8_t *, const Tile &, int, int, int, int, uint32_t, bool) {}
    static __device__ __forceinline__ void store(const Args &a, uint8_t *p, const Tile &t, const Cols &, int w, int lane, int c, const float (&v)[16], int product)
    {
        if (product) {
            const uint16_t *pick = lists_at(a, p).picks + t.off;
            const int h = t.row * kRows + w * 32 + lane;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (h < a.H && c + i < t.n) a.out[(int64_t)pick[c + i] * a.H + h] = v[i];
        } else {
            // lanes 0..15 hold gate values, lanes 16..31 the up values of the same rows: each half finishes eight of the columns
            const int i0 = t.row * (kRows / 2) + w * 16 + (lane & 15);
            const bool low = lane < 16;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float other = __shfl_xor_sync(0xffffffffu, low ? v[8 + i] : v[i], 16);
                const float gate = low ? v[i] : other, up = low ? other : v[8 + i];
                const int col = c + i + (low ? 0 : 8);
                // silu(g) = g e^g / (1 + e^g) below zero (e^-g would be infinite from -88.7 on, and a quotient by 2^126 or more is 0 here).  The fast
                // forms: 2 + 1.2 |g| units in the last place and 2 more, far below the rounding to bf16 (expf and / : 256 tokens on 32 experts 44 -> 48 us).
                const float e = __expf(-fabsf(gate)), silu = __fdividef(gate * (gate < 0.0f ? e : 1.0f), 1.0f + e);
                if (col < t.n && i0 < a.I) a.act[(int64_t)(t.off + col) * a.I + i0] = f32_to_bf16(silu * up);
            }
        }
    }
};

// y[t] = sum over its picks on this rank, in slot order.  Reads what the launch before left in L2; a launch's latency (5 us) bounds it.
struct SumArgs {
    const int32_t *ids;
    const float *weights, *out;
    uint8_t *y;
    int64_t y_stride;
    int K, E, first, count, H;
};

// y[t] = sum over the token's picks here, in slot order, of weight * output row.  One thread per 8 values, four rows in flight; ids and
// weights are read before the wait for the rows.  Bound by L2 and launch latency.
__global__ void __launch_bounds__(kSumThreads) k_experts_sum(const __grid_constant__ SumArgs a)
{
    constexpr int kBatch = 4;
    __shared__ float w_s[MW_MAX_TOPK];
    __shared__ int pick_s[MW_MAX_TOPK];
    __shared__ int n_s;
    const int t = blockIdx.y, h = (blockIdx.x * kSumThreads + threadIdx.x) * 8;
    if (threadIdx.x < 32) {                     // the picks here, closed up
        int n = 0;
        for (int k0 = 0; k0 < a.K; k0 += 32) {
            const int k = k0 + threadIdx.x, id = k < a.K ? __ldcg(a.ids + t * a.K + k) : -1, e = id - a.first;
            const float w = k < a.K && a.weights ? __ldcg(a.weights + t * a.K + k) : 1.0f;
            const bool here = id >= 0 && id < a.E && e >= 0 && e < a.count;
            const unsigned b = __ballot_sync(0xffffffffu, here);
            if (here) {
                const int at = n + __popc(b & ((1u << threadIdx.x) - 1));
                pick_s[at] = t * a.K + k;
                w_s[at] = w;
            }
            n += __popc(b);
        }
        if (threadIdx.x == 0) n_s = n;
    }
    __syncthreads();
    grid_dependency_wait();
    grid_launch_dependents();
    if (h >= a.H) return;
    float acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
    const int n = n_s;
    for (int k0 = 0; k0 < n; k0 += kBatch) {
        float4 q[kBatch][2];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (k0 + k < n) {
                const float4 *p = (const float4 *)(a.out + (int64_t)pick_s[k0 + k] * a.H + h);
                q[k][0] = __ldcg(p);
                q[k][1] = __ldcg(p + 1);
            }
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (k0 + k < n) {
                const float w = w_s[k0 + k];
                acc[0] = fmaf(w, q[k][0].x, acc[0]); acc[1] = fmaf(w, q[k][0].y, acc[1]); acc[2] = fmaf(w, q[k][0].z, acc[2]);
                acc[3] = fmaf(w, q[k][0].w, acc[3]); acc[4] = fmaf(w, q[k][1].x, acc[4]); acc[5] = fmaf(w, q[k][1].y, acc[5]);
                acc[6] = fmaf(w, q[k][1].z, acc[6]); acc[7] = fmaf(w, q[k][1].w, acc[7]);
            }
    }
    uint4 o;
    o.x = f32_to_bf16(acc[0]) | (uint32_t)f32_to_bf16(acc[1]) << 16;
    o.y = f32_to_bf16(acc[2]) | (uint32_t)f32_to_bf16(acc[3]) << 16;
    o.z = f32_to_bf16(acc[4]) | (uint32_t)f32_to_bf16(acc[5]) << 16;
    o.w = f32_to_bf16(acc[6]) | (uint32_t)f32_to_bf16(acc[7]) << 16;
    *(uint4 *)(a.y + (int64_t)t * a.y_stride + (int64_t)h * 2) = o;
}

inline size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }
inline int round16(int n) { return (n + 15) & ~15; }

bool make_maps(mw_experts *m)
{
    const mw_experts_config &c = m->cfg;
    const uint64_t H = c.H, I = c.I, n = c.expert_count;
    const uint64_t gd[5] = {H, 16, 2, I / 16, n}, gs[4] = {H * 2, I * H * 2, 16 * H * 2, 2 * I * H * 2};
    const uint32_t gb[5] = {kChunk, 16, 2, kRows / 32, 1};
    const uint64_t dd[3] = {I, H, n}, ds[2] = {I * 2, H * I * 2};
    const uint32_t db[3] = {kChunk, kRows, 1};
    const uint64_t picks = (uint64_t)c.max_tokens * c.K, rd[2] = {H, picks}, rs[1] = {H * 2}, ad[2] = {I, picks}, as[1] = {I * 2};
    const uint32_t ab[2] = {kChunk, 64}, fb[2] = {kChunk, 16};
    return encode_map(&m->map_gate_up, m->w_gate_up, 5, gd, gs, gb) && encode_map(&m->map_down, m->w_down, 3, dd, ds, db) &&
           encode_map(&m->map_rows, m->rows, 2, rd, rs, ab) && encode_map(&m->map_rows_few, m->rows, 2, rd, rs, fb) &&
           encode_map(&m->map_act, m->act, 2, ad, as, ab) && encode_map(&m->map_act_few, m->act, 2, ad, as, fb);
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
        cfg->H > MW_EXPERTS_MAX_WIDTH || cfg->I > MW_EXPERTS_MAX_WIDTH ||
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
    m->w_gate_up = w_gate_up; m->w_down = w_down;
    cudaDeviceGetAttribute(&m->sm_count, cudaDevAttrMultiProcessorCount, cfg->device);
    const size_t picks = (size_t)cfg->max_tokens * cfg->K;
    const int cols = round16(cfg->max_tokens) < kMaxCols ? round16(cfg->max_tokens) : kMaxCols;
    const size_t b_rows = round256(picks * cfg->H * 2), b_act = round256(picks * cfg->I * 2), b_out = round256(picks * cfg->H * 4);
    const size_t b_parts = 4 * (size_t)m->sm_count * cols * kRows * 4, b_counts = round256(2 * (size_t)m->sm_count * 4);
    const size_t b_state = round256((kHead + 4 * (size_t)cfg->expert_count) * 4);
    if (cudaMalloc(&m->slab, 256 + b_counts + b_state + b_rows + b_act + b_out + b_parts) != cudaSuccess) { cudaGetLastError(); delete m; return MW_ERR_CUDA; }
    uint8_t *p = (uint8_t *)m->slab;
    m->status = (int32_t *)p; p += 256;
    m->counts = (unsigned int *)p; p += b_counts;
    m->state = (unsigned int *)p; p += b_state;
    m->rows = (uint16_t *)p; p += b_rows;
    m->act = (uint16_t *)p; p += b_act;
    m->out = (float *)p; p += b_out;
    m->parts = (float *)p;
    int rc = MW_OK;
    if (cudaMemset(m->slab, 0, 256 + b_counts + b_state) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) rc = MW_ERR_CUDA;
    if (rc == MW_OK && cudaFuncSetAttribute(k_stream<Product>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) != cudaSuccess)
        rc = MW_ERR_CUDA;
    if (rc == MW_OK && !make_maps(m)) rc = MW_ERR_CUDA;
    if (rc != MW_OK) { cudaGetLastError(); mw_experts_destroy(m); return rc; }
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
    const mw_experts_config &c = m->cfg;
    const int64_t row = (int64_t)c.H * 2;
    if ((x_stride_bytes && x_stride_bytes < row) || (y_stride_bytes && y_stride_bytes < row)) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)y | (uint64_t)x_stride_bytes | (uint64_t)y_stride_bytes) & 15u) return MW_ERR_ALIGNMENT;
    if (((uintptr_t)topk_ids | (uintptr_t)weights) & 3u) return MW_ERR_ALIGNMENT;
    cudaStream_t st = (cudaStream_t)stream;
    const bool overlap = !(c.flags & MW_FLAG_NO_OVERLAP);
    // Up to 48 picks for each expert of the domain (what a rank's experts have of them is on the device; rows that were delivered to a rank are more):
    // four steps per unit and tiles of up to 128 tokens, else two and 256 (a stage has to fit the tokens' ring).  More tokens of one expert are
    // several tiles that run side by side.  Four / two steps, us: 32 experts, top-4, 1024 x 688, 256 tokens 44.0 / 46.1, 512 tokens (64 picks each) 51.9 / 52.7; 8 experts,
    // top-4, 4096 x 2048, 200 tokens (100 picks each) 132.8 / 105.5; rows delivered to 4 of 256 experts, top-8, 7168 x 2048: 64 tokens (18 picks each of these four) 71.5 / 75.6,
    // 201 tokens (56) 83.1 / 83.5, 256 tokens (70) 87.5 / 88.8.
    const int picks = T * c.K;
    const bool few = picks <= 48 * (int64_t)c.E && picks <= 2048;           // (beyond, the lists leave too little for stages of that size)
    const int most = few ? kMaxCols / 2 : kMaxCols, cols = round16(T) < most ? round16(T) : most;

    ExpertArgs g;
    const uint64_t xd[2] = {(uint64_t)c.H, (uint64_t)T}, xs[1] = {(uint64_t)(x_stride_bytes ? x_stride_bytes : row)};
    const uint32_t xb[2] = {kChunk, 1};
    if (!encode_map(&g.x_row, x, 2, xd, xs, xb)) return MW_ERR_INVALID_ARG;
    g.gate_up = m->map_gate_up; g.down = m->map_down; g.rows = m->map_rows; g.rows_few = m->map_rows_few; g.act_box = m->map_act; g.act_few = m->map_act_few;
    const size_t lists = lists_bytes(c.expert_count, picks, m->sm_count);
    g.c.steps = few ? 4 : 2;
    split_memory(&g.c, kSmem - lists, kMinRing);
    g.c.tmem_cols = 32;
    while ((int)g.c.tmem_cols < 2 * cols) g.c.tmem_cols *= 2;
    g.c.acc_cols = g.c.tmem_cols / 2; g.c.add_col = 0;
    g.c.wait_limit = (c.flags & MW_FLAG_SHORT_WAITS) ? (1 << 10) : (1 << 20);
    g.c.wait_first = (c.flags & MW_FLAG_SHORT_WAITS) != 0;
    g.c.skew = m->skew;
    m->skew = 0;
    g.c.min_units = few ? 4 : 8;
    g.c.shares = m->sm_count;
    g.c.part_cols = cols;
    g.c.parts = m->parts; g.c.counts = m->counts; g.c.status = m->status;
    g.ids = topk_ids; g.x = (const uint8_t *)x; g.x_stride = x_stride_bytes ? x_stride_bytes : row;
    g.picks = picks; g.K = c.K; g.E = c.E; g.first = c.expert_first; g.count = c.expert_count; g.max_cols = cols;
    g.H = c.H; g.I = c.I; g.sorted = m->rows; g.act = m->act; g.out = m->out; g.state = m->state;
    const int blocks = m->blocks && m->blocks < m->sm_count ? m->blocks : m->sm_count;
    m->blocks = 0;
    cudaError_t e = mw_launch(k_stream<Product>, dim3(blocks), dim3(kThreads), kSmem, st, overlap, g);

    SumArgs s;
    s.ids = topk_ids; s.weights = weights; s.out = m->out; s.y = (uint8_t *)y; s.y_stride = y_stride_bytes ? y_stride_bytes : row;
    s.K = c.K; s.E = c.E; s.first = c.expert_first; s.count = c.expert_count; s.H = c.H;
    if (e == cudaSuccess) e = mw_launch(k_experts_sum, dim3((c.H + 8 * kSumThreads - 1) / (8 * kSumThreads), T), dim3(kSumThreads), 0, st, overlap, s);
    if (e != cudaSuccess) { cudaGetLastError(); return MW_ERR_CUDA; }
    m->launches += 2;
    return MW_OK;
}

int mw_experts_get_status(mw_experts *m, int32_t *status, void *stream)
{
    if (!m || !status) return MW_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemcpyAsync(status, m->status, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(m->status, 0, 4, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return MW_ERR_CUDA;
    // a wait that gave up may have left tiles half counted
    if (*status == MW_ERR_TIMEOUT && (cudaMemsetAsync(m->counts, 0, (size_t)((uint8_t *)m->rows - (uint8_t *)m->counts), st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess))
        return MW_ERR_CUDA;
    return MW_OK;
}

int mw_experts_test_skew_waits(mw_experts *m)
{
    if (!m) return MW_ERR_INVALID_ARG;
    m->skew = 16;
    return MW_OK;
}

int mw_experts_test_few_blocks(mw_experts *m, int32_t blocks)
{
    if (!m || blocks < 1) return MW_ERR_INVALID_ARG;
    m->blocks = blocks;
    return MW_OK;
}

int64_t mw_experts_kernel_launches(const mw_experts *m) { return m ? m->launches : 0; }

}  // extern "C"
