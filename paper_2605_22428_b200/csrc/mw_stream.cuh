// The engine behind the products of mw_experts and mw_project: out = W B^T for many (W, B) pairs at once, W streamed from HBM.
//
// Every product here has few right-hand columns (tokens) for its left-hand rows (weights), so the weights are the M
// operand: a tile is 128 weight rows x up to 256 tokens, one tcgen05.mma of M = 128 per 16 elements of K, accumulators in
// TMEM (two buffers, so that a tile's epilogue runs under the next tile's products).  A step is 64 elements along K: 16 KB of
// weights by one TMA load, and the tokens' 128-byte pieces by TMA, in boxes where they are neighbours; a gather of four rows takes
// about as long as a box of 128 (16-byte copies by threads are no faster), so it serves a few tokens only.  A unit of work is `steps` of them, loaded and multiplied together: one stage of the pipeline.
// Weights have slots of fixed size; tokens go through a ring in which each stage takes exactly the bytes it needs.
//
// A product's tiles are dealt out in shares, one per SM: rounds of whole tiles, as many as all can have, then a piece of the tiles
// left over, which may end one tile and begin the next (share_of).  A tile that is cut between shares is joined in float32: each contributor
// writes its part to scratch and counts itself in; the last to arrive adds the parts in the order of the shares and finishes the tile.
// So nobody waits for another part, and the sum does not depend on who came last.
// A kernel of one product has as many CTAs as shares, and CTA c takes share c.  Where a second product waits for the first one's
// results, CTAs take shares by tickets, the first product's before the second's: whatever a CTA waits for was taken by one that
// runs already and itself waits for earlier work only, so a call ends however few of its CTAs get an SM, and however late.
//
// Warp 0 loads weights, warp 2 tokens, one thread of warp 1 issues the products, warps 4-7 read the accumulators (warp w reads TMEM
// lanes 32 (w - 4) ...); these and warp 3 are free for a product's own work at the start.  Every wait is bounded; one that runs out
// ends the kernel with MW_ERR_TIMEOUT in the handle's status.
//
// A kernel runs one product, or two of which the second takes the first one's results as its tokens; the pipeline goes on
// from one to the other, so the second product's first weights arrive while the first one's last tiles are finished.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>

#include "mw_internal.cuh"

namespace mw_stream {

constexpr int kThreads = 256;
constexpr int kSlots = 16;                      // stages at most
constexpr int kChunk = 64;                      // elements of K per step
constexpr int kRows = 128;                      // weight rows per tile
constexpr int kMaxCols = 256;                   // tokens per tile at most
constexpr int kFew = 16;                        // tokens that are gathered
constexpr int kLong = 64;                       // steps of a tile that is worth equal pieces
constexpr int kPieces = 5;                       // pieces a tile is cut into at most
constexpr uint32_t kWeightBytes = kRows * kChunk * 2;

// What the tokens' warp tells the issuing thread about a stage.
struct Stage {
    uint32_t tokens;                            // shared-memory address of the first step's tokens
    uint32_t room;                              // bytes between the tokens of two steps
    uint32_t what;                              // bits 0..2: first / last unit of a segment, end; 4..15: products of 16 along K; 16..: tokens, rounded up to 16
};
constexpr uint32_t kFirst = 1, kLast = 2, kEnd = 4;

struct Shared {
    uint64_t full[kSlots], empty[kSlots];
    uint64_t acc_full[2], acc_empty[2], drained;
    uint32_t tmem;
    uint32_t before[2], after;                  // contributors that had put their part down: when this part was ready (by accumulator), when it was down too
    volatile uint32_t abort;
    Stage stage[kSlots];
    int weight_rows[kRows / 8];                 // notes of the weights' warp about its tile
    alignas(16) int token_rows[kFew];           // notes of the tokens' warp about its tile
    uint32_t held[kSlots];                      // bytes of the ring each stage holds
    uint32_t issued[2];                         // stages whose weights, whose tokens were asked for (set at the end)
};

// A tile, as every role sees it.
struct Tile {
    int n, n16;                                 // tokens; the same rounded up to 16
    int row;                                    // weight-row tile
    int which;                                  // expert / token tile (the product's own meaning)
    int parts;                                  // token tiles of the expert (experts)
    int off;                                    // first token of the tile, or first entry of a list (likewise)
};

// Arguments common to all products.
struct Common {
    int slots;                                  // stages, at most kSlots
    uint32_t ring_bytes;                        // of the tokens' ring
    uint32_t tmem_cols;                         // power of two >= 32
    uint32_t acc_cols;                          // columns of an accumulator
    uint32_t add_col;                           // column of the additions that are made before the products are done; 0: made after them
    int wait_limit, skew;
    int wait_first;                             // every warp waits for the kernel before at once (else only those that need its results)
    int steps;                                  // steps per unit
    int min_units;                              // smallest piece of a tile
    int shares;                                 // of a product: CTAs that a launch would have with the device to itself
    int part_cols;                              // columns of a scratch part
    float *parts;                               // [products][2 * shares][part_cols / 4][kRows][4]
    unsigned int *counts;                       // [products][shares], zero between launches
    int32_t *status;
};

// ---- host side (mw_stream.cu) ----
// Tensor map of a row-major array of bf16 elements, boxes 128 bytes wide and stored swizzled: dims innermost first, strides[i] = bytes between neighbours along dim i + 1.
bool encode_map(CUtensorMap *map, const void *base, int rank, const uint64_t *dims, const uint64_t *strides, const uint32_t *box);

// Divides a block's shared memory: at least `ring` bytes for the tokens' ring, weight slots of c->steps steps as many as fit, the rest to the ring.
void split_memory(Common *c, size_t bytes, size_t ring);

#ifdef __CUDACC__

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// One thread of a converged warp.  (The instructions of TMA and the tensor cores take their operands from uniform registers; under
// `if (lane == 0)` the compiler cannot know that one thread is left and guards each of them with a loop.)
__device__ __forceinline__ bool elect_one()
{
    uint32_t one;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0;
}

__device__ __forceinline__ void bar_init(uint64_t *bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory"); }
__device__ __forceinline__ void bar_expect(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
    return ok != 0;
}

// Waits for the phase of the given parity to complete; false when the wait gave up here or elsewhere in the CTA.
__device__ __forceinline__ bool bar_wait(uint64_t *bar, uint32_t parity, Shared *s, const Common &c)
{
#pragma unroll 1
    for (int i = 0; i < c.wait_limit; ++i) {
        if (bar_try(bar, parity)) return true;
        if (s->abort) return false;
    }
    s->abort = 1;
    atomicExch(c.status, MW_ERR_TIMEOUT);
    return false;
}

template <int RANK>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int c0, int c1, int c2 = 0, int c3 = 0, int c4 = 0)
{
    const uint32_t b = smem_addr(bar);
    if constexpr (RANK == 2)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(b) : "memory");
    else if constexpr (RANK == 3)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(b) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(b) : "memory");
}

// Four rows of a 2-D map whose boxes are one row high, to consecutive rows in shared memory.
__device__ __forceinline__ void gather4(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int x, int r0, int r1, int r2, int r3)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(smem_addr(bar)) : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// Descriptor of a K-major operand in shared memory, rows of 128 bytes in groups of eight, swizzled within the group as TMA stores
// them: address / 16, distance of the groups / 16 in bits 32..45, version 1 in bit 46, layout 2 (128-byte swizzle) in bits 61..63.
__device__ __forceinline__ uint64_t operand(uint32_t addr)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | ((1024ull >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// bf16 x bf16 -> f32, both operands K-major, M = 128.
__device__ __forceinline__ uint32_t instruction(int n16) { return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n16 >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24); }

__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 16 columns of the thread's TMEM lane.
__device__ __forceinline__ void read16(uint32_t addr, float (&v)[16])
{
    uint32_t r[16];
    __syncwarp();
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// The same without the wait (read_wait), so that several can be under way.
__device__ __forceinline__ void read16_begin(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
// (The values go through it, so that nothing uses them before.)
__device__ __forceinline__ void read_wait(uint32_t (&r)[2][16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0][0]), "+r"(r[0][1]), "+r"(r[0][2]), "+r"(r[0][3]), "+r"(r[0][4]), "+r"(r[0][5]), "+r"(r[0][6]), "+r"(r[0][7]),
                   "+r"(r[0][8]), "+r"(r[0][9]), "+r"(r[0][10]), "+r"(r[0][11]), "+r"(r[0][12]), "+r"(r[0][13]), "+r"(r[0][14]), "+r"(r[0][15]),
                   "+r"(r[1][0]), "+r"(r[1][1]), "+r"(r[1][2]), "+r"(r[1][3]), "+r"(r[1][4]), "+r"(r[1][5]), "+r"(r[1][6]), "+r"(r[1][7])
                 :: "memory");
    asm volatile("" : "+r"(r[1][8]), "+r"(r[1][9]), "+r"(r[1][10]), "+r"(r[1][11]), "+r"(r[1][12]), "+r"(r[1][13]), "+r"(r[1][14]), "+r"(r[1][15]));
}
__device__ __forceinline__ void write16(uint32_t addr, const float (&v)[16])
{
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[i]);
    __syncwarp();
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                   "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// All 128 threads of the epilogue warps: barrier, and the logical and of `ok`.
__device__ __forceinline__ bool epilogue_all(bool ok)
{
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.and.pred q, 1, 128, p;\n selp.u32 %0, 1, 0, q;\n}"
                 : "=r"(r) : "r"((uint32_t)ok) : "memory");
    return r != 0;
}

__device__ __forceinline__ uint16_t f32_to_bf16(float f)     // to nearest even
{
    uint16_t r;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(f));
    return r;
}

// First unit of piece c when `units` are cut into `pieces`, and the piece that has unit u.  (Divisions here and below are of 32
// bits: the rest of a call is fewer tiles than there are shares, a tile at most 2^14 units; 64-bit ones cost hundreds of instructions,
// which at the start of a kernel have to be fetched first.)
__device__ __forceinline__ uint32_t first_unit(uint32_t units, uint32_t pieces, uint32_t c) { return units * c / pieces; }
__device__ __forceinline__ int piece_of(uint32_t units, uint32_t pieces, uint32_t u) { return (int)(((u + 1) * pieces - 1) / units); }

// P describes a kernel's products: their arguments, lists in shared memory and tiles (see mw_experts.cu and mw_project.cu).  `product` is 0, or 1
// for the second of two: a run-time argument, because code of its own for the second would have to be fetched when it begins.
//   P::kProducts                         1 or 2
//   P::Args                              kernel arguments, with a member `c` of type Common
//   P::prologue(a)                       waits for earlier kernels as far as setup needs it, lets the next kernel start
//   P::setup(a, lists)                   all threads: builds the lists
//   P::leave(a, lists)                   all threads, at the end
//   P::tiles(a, lists, product)          tiles of the whole call;  P::units_per_tile(a, product)
//   P::tile(a, lists, q, product)        the q-th of them
//   P::depth(a, product)                 length of the sums (elements of K)
//   P::room(a, tile)                     bytes of the ring a step's tokens take, a multiple of 1024
//   P::note_weights(a, lists, tile, lane, rows)       all lanes of the loading warp: what the tile's loads need; returns a count
//   P::note_tokens(a, lists, tile, lane, rows, product)     likewise, at most kFew values
//   P::weight_bytes(a, n), P::token_bytes(a, tile, product) bytes that a step's loads deliver, n from the notes
//   P::load_weights(a, tile, rows, n, step, addr, bar, product), P::load_tokens(a, tile, rows, step, addr, bar, product)    one thread: issue the loads of a step
//   P::kClaims                           CTAs take shares by tickets: P::claim(a) takes one, P::claims(a, lists) keeps those of this CTA in order, the
//                                        first from setup on, the others kNoShare until they are taken; product 0's shares come first, then product 1's
//   P::kEarly, P::early(a, lists, w, lane)            work of warps 3-7 (w = 0..4) at the start
//   P::kLate, P::wait_tokens(a, lists, s, tile, product)    tokens are made in this kernel: waits for those of a tile, false if it gave up
//   P::Cols, P::cols(a, lists, tile, warp, lane)      per-thread state of the epilogue for a tile
//   P::kAdds, P::adds(a)                              something that is no product is added to the values (by one contributor for each):
//   P::prefetch(a, tile, lane, c)                     asks L2 for what P::add will read for columns c ... c + 15
//   P::add(a, lists, tile, warp, lane, c, step, dst, more)     adds it to (`more`), or writes it to, columns c ... c + 15, then c + step ... of TMEM at dst
//   P::store(a, lists, tile, cols, warp, lane, c, v, product)  takes row 32 warp + lane, columns c ... c + 15 of the finished tile
//   P::tells(product), P::tell(a, lists, tile)        one thread, when all of a tile is stored and visible

// The last contributor of a cut tile adds the OTHERS' parts to its own, which is still in the accumulators, in the order of the
// shares (`place` is its own).  Eight to sixteen 16-byte loads per thread are in flight.
// parts: the thread's row of the first contributor's first part; pair: distance of two shares' parts in float4.
template <int OTHERS>
__device__ __forceinline__ void join(int n16, uint32_t acc, const float4 *parts, int64_t pair, int place)
{
    constexpr int kGroup = OTHERS == 1 ? 2 : 1;                             // batches of 16 columns at a time
#pragma unroll 1
    for (int c0 = 0; c0 < n16; c0 += 16 * kGroup) {
        float4 q[kGroup][OTHERS][4];
#pragma unroll
        for (int g = 0; g < kGroup; ++g)
#pragma unroll
            for (int p = 0; p < OTHERS; ++p)
                if (c0 + 16 * g < n16) {
                    const int from = p + (p >= place);                      // counted from the first contributor, whose part is its second
                    const float4 *src = parts + from * pair + (from == 0 ? pair / 2 : 0) + ((c0 >> 2) + 4 * g) * kRows;
#pragma unroll
                    for (int i = 0; i < 4; ++i) q[g][p][i] = __ldcg(src + i * kRows);
                }
#pragma unroll
        for (int g = 0; g < kGroup; ++g)
            if (c0 + 16 * g < n16) {
                float v[16], sum[16];
                read16(acc + c0 + 16 * g, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] = 0.0f;
#pragma unroll
                for (int p = 0; p <= OTHERS; ++p) {
                    if (p == place) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[i] += v[i];
                    }
                    if (p < OTHERS) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            sum[4 * i] += q[g][p][i].x; sum[4 * i + 1] += q[g][p][i].y; sum[4 * i + 2] += q[g][p][i].z; sum[4 * i + 3] += q[g][p][i].w;
                        }
                    }
                }
                write16(acc + c0 + 16 * g, sum);
            }
    }
}

// Hands a finished tile's values on.
template <class P>
__device__ __forceinline__ void store_tile(const typename P::Args &a, uint8_t *lists, const Tile &tile, const typename P::Cols &cols, int w, int lane, uint32_t acc, int product)
{
#pragma unroll 1
    for (int c = 0; c < tile.n16; c += 32) {
        uint32_t r[2][16];
        __syncwarp();
        read16_begin(acc + c, r[0]);
        if (c + 16 < tile.n16) read16_begin(acc + c + 16, r[1]);
        read_wait(r);
#pragma unroll
        for (int g = 0; g < 2; ++g)
            if (c + 16 * g < tile.n16) {
                float v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[g][i]);
                P::store(a, lists, tile, cols, w, lane, c + 16 * g, v, product);
            }
    }
}

// A share of a product: as many whole tiles as every share can have, in rounds (tile c of a round to share c, so that the
// first tiles are finished first), then a piece of the tiles left over.
struct Share {
    int whole;                                  // whole tiles of this share
    int first;                                  // the first tile left over
    uint32_t len, units;                        // units of a tile; of all tiles left over
    uint32_t u0, u1;                            // this share's piece of these
    int pieces, me;                             // shares that have pieces; which this is
    int product;
};
constexpr uint16_t kNoShare = 0xffffu;

// The rest: each tile is cut into the same number of pieces, as many as there are shares for, at most kPieces, of min_units or more: a hundred SMs
// can already draw all that HBM gives, and each piece costs a join.  Where a tile is long (kLong steps or more) and a round has gone before, all shares
// get equal pieces as long as the rest is a quarter as many tiles (a tile is cut between five shares at most).
// Measured, same pieces / equal pieces: one token on 8 experts, 112 steps a tile after a round, 131.5 / 127.9 us; 256 tokens on 32 experts, 16 and 11
// steps, 55.6 / 64.0; 201 tokens on 4 experts, 112 steps and no round, 82 / 94, and 32 steps after a round as well, 82 / 92; a projection of
// 512 tokens, 4096 x 4096, 64 steps and no round, 58 / 72, of 64 tokens, 7168 x 7168, 31 / 37 to 39.
// `number`: the product times the number of shares, plus which of them.
template <class P>
__device__ __forceinline__ Share share_of(const typename P::Args &a, uint8_t *lists, int number)
{
    Share sh;
    const int all = a.c.shares;
    sh.product = P::kProducts > 1 && number >= all;
    sh.me = sh.product ? number - all : number;
    const int tiles = P::tiles(a, lists, sh.product);
    sh.len = P::units_per_tile(a, sh.product);
    sh.whole = tiles / all;
    sh.first = sh.whole * all;
    const int left = tiles - sh.first;
    sh.units = left * sh.len;
    sh.pieces = all;
    const bool equal = sh.whole > 0 && (int)sh.len * a.c.steps >= kLong;
    if (!equal || left * 4 < all || (uint32_t)(all * a.c.min_units) > sh.units) {
        int pieces = left ? all / left : 1;
        const int most = (int)sh.len / a.c.min_units;
        pieces = pieces < kPieces ? pieces : kPieces;
        pieces = pieces < most ? pieces : most;
        sh.pieces = pieces > 1 ? left * pieces : left ? left : 1;
    }
    sh.u0 = sh.me < sh.pieces ? first_unit(sh.units, sh.pieces, sh.me) : sh.units;
    sh.u1 = sh.me < sh.pieces ? first_unit(sh.units, sh.pieces, sh.me + 1) : sh.units;
    return sh;
}

// The n-th share this CTA takes, for a whole warp; -1: none is left, or the wait gave up (`ok` false).  Tickets are taken by the warp that
// loads weights, before its last load of the share before, so the others hardly ever wait here.
template <class P>
__device__ __forceinline__ int share_at(const typename P::Args &a, uint8_t *lists, Shared *s, int n, bool &ok)
{
    if (!P::kClaims) return n < P::kProducts ? n * a.c.shares + (int)blockIdx.x : -1;
    const volatile uint16_t *claim = P::claims(a, lists) + n;
    int number = kNoShare;
    for (int i = 0; i < a.c.wait_limit && !s->abort; ++i) {
        number = *claim;
        if (number != kNoShare) break;
        __nanosleep(20);
    }
    number = __shfl_sync(0xffffffffu, number, 0);
    if (number == kNoShare) {
        if (!s->abort) { s->abort = 1; atomicExch(a.c.status, MW_ERR_TIMEOUT); }
        ok = false;
        return -1;
    }
    return number < P::kProducts * a.c.shares ? number : -1;
}

// The tiles and pieces of tiles in a share, in order:  for (Walk<P> w(...); w.more(); w.next())  units [k0, k1) of `tile`.
template <class P>
struct Walk {
    const typename P::Args &a;
    uint8_t *lists;
    const Share &sh;
    int round;
    uint32_t u, start;                          // in the rest, once the rounds are done: the next unit, the tile's first
    Tile tile;
    int k0, k1;
    __device__ __forceinline__ Walk(const typename P::Args &a_, uint8_t *lists_, const Share &sh_) : a(a_), lists(lists_), sh(sh_), round(0), u(sh_.u0), start(0) { piece(); }
    __device__ __forceinline__ bool whole() const { return round < sh.whole; }
    __device__ __forceinline__ bool more() const { return whole() || u < sh.u1; }
    __device__ __forceinline__ void piece()
    {
        if (!more()) return;
        const uint32_t q = u / sh.len;
        start = q * sh.len;
        tile = P::tile(a, lists, whole() ? round * a.c.shares + sh.me : sh.first + (int)q, sh.product);
        k0 = whole() ? 0 : (int)(u - start);
        k1 = whole() || sh.u1 - start > sh.len ? (int)sh.len : (int)(sh.u1 - start);
    }
    __device__ __forceinline__ void next()
    {
        if (whole()) ++round;
        else u = start + k1;
        piece();
    }
    // Nothing comes after this piece.
    __device__ __forceinline__ bool last() const { return whole() ? round + 1 == sh.whole && u >= sh.u1 : start + k1 >= sh.u1; }
    // The shares that have the tile's first and last unit.
    __device__ __forceinline__ bool alone() const { return k0 == 0 && k1 == (int)sh.len; }
    __device__ __forceinline__ int from() const { return alone() ? sh.me : piece_of(sh.units, sh.pieces, start); }
    __device__ __forceinline__ int to() const { return alone() ? sh.me : piece_of(sh.units, sh.pieces, start + sh.len - 1); }
};

// A place in a circle of slots, the parity of the round, and the steps so far.
struct Place {
    uint32_t slot, round, passed;
    __device__ __forceinline__ void step(uint32_t slots) { ++passed; if (++slot == slots) { slot = 0; round ^= 1; } }
};

// ---- weights ----
// `n`: the share is the n-th of this CTA.
template <class P>
__device__ __forceinline__ bool load_all_weights(const typename P::Args &a, uint8_t *lists, Shared *s, const Share &sh, int n, int lane, uint32_t base, Place &at)
{
    const int all_steps = (P::depth(a, sh.product) + kChunk - 1) / kChunk;
    Walk<P> w(a, lists, sh);
    if (P::kClaims && !w.more() && lane == 0) ((volatile uint16_t *)P::claims(a, lists))[n + 1] = (uint16_t)P::claim(a);
#pragma unroll 1
    for (; w.more(); w.next()) {
        __syncwarp();
        const int rows = P::note_weights(a, lists, w.tile, lane, s->weight_rows);
        __syncwarp();
        const uint32_t bytes = P::weight_bytes(a, rows);
        const int claim_at = P::kClaims && w.last() ? w.k1 - 1 : -1;       // (asked for before the wait, needed after the load)
#pragma unroll 1
        for (int k = w.k0; k < w.k1; ++k) {
            int next = 0;
            if (P::kClaims && k == claim_at && lane == 0) next = P::claim(a);
            if (!__all_sync(0xffffffffu, bar_wait(&s->empty[at.slot], at.round ^ 1, s, a.c))) return false;
            if (elect_one()) {
                const int first = k * a.c.steps, left = all_steps - first, steps = left < a.c.steps ? left : a.c.steps;
                const uint32_t addr = base + at.slot * (kWeightBytes * a.c.steps);
                bar_expect(&s->full[at.slot], bytes * steps + a.c.skew);
                for (int i = 0; i < steps; ++i)
                    P::load_weights(a, w.tile, s->weight_rows, rows, first + i, addr + i * kWeightBytes, &s->full[at.slot], sh.product);
            }
            __syncwarp();
            at.step(a.c.slots);
            if (P::kClaims && k == claim_at && lane == 0) ((volatile uint16_t *)P::claims(a, lists))[n + 1] = (uint16_t)next;
        }
    }
    return true;
}

// ---- tokens ----
struct Ring {
    Place head, tail;                           // the next stage; the oldest that still holds bytes
    uint32_t live, pos, used;                   // stages and bytes held (gaps at the end included), next free byte
};

__device__ __forceinline__ bool free_one(const Common &c, Shared *s, Ring &r)
{
    if (!__all_sync(0xffffffffu, bar_wait(&s->empty[r.tail.slot], r.tail.round, s, c))) return false;
    r.used -= s->held[r.tail.slot];
    --r.live;
    r.tail.step(c.slots);
    return true;
}

template <class P>
__device__ __forceinline__ bool load_all_tokens(const typename P::Args &a, uint8_t *lists, Shared *s, const Share &sh, int lane, uint32_t base, Ring &r)
{
    const int depth = P::depth(a, sh.product), all_steps = (depth + kChunk - 1) / kChunk;
    int known = -1;                             // kLate: the tokens that have been waited for
#pragma unroll 1
    for (Walk<P> w(a, lists, sh); w.more(); w.next()) {
        if (P::kLate && known != w.tile.which) {
            if (!P::wait_tokens(a, lists, s, w.tile, sh.product)) return false;
            known = w.tile.which;
        }
        __syncwarp();
        P::note_tokens(a, lists, w.tile, lane, s->token_rows, sh.product);
        __syncwarp();
        const uint32_t bytes = P::token_bytes(a, w.tile, sh.product), room = P::room(a, w.tile), size = room * a.c.steps;
#pragma unroll 1
        for (int k = w.k0; k < w.k1; ++k) {
            uint32_t gap;                       // bytes left unused at the end of the ring when the stage has to start over at its begin
            for (;;) {
                if (r.live == 0) r.pos = 0;
                gap = r.pos + size > a.c.ring_bytes ? a.c.ring_bytes - r.pos : 0;
                if (r.used + gap + size <= a.c.ring_bytes && r.live < (uint32_t)a.c.slots) break;
                if (!free_one(a.c, s, r)) return false;
            }
            if (r.pos + size > a.c.ring_bytes) r.pos = 0;
            if (elect_one()) {
                const int first = k * a.c.steps, left = all_steps - first, steps = left < a.c.steps ? left : a.c.steps;
                const int elements = depth - first * kChunk < steps * kChunk ? depth - first * kChunk : steps * kChunk;
                const uint32_t addr = base + r.pos, slot = r.head.slot;
                s->held[slot] = gap + size;
                s->stage[slot] = {addr, room, (k == w.k0 ? kFirst : 0) | (k == w.k1 - 1 ? kLast : 0) | (uint32_t)((elements + 15) / 16) << 4 | (uint32_t)w.tile.n16 << 16};
                bar_expect(&s->full[slot], bytes * steps);
                for (int i = 0; i < steps; ++i) P::load_tokens(a, w.tile, s->token_rows, first + i, addr + i * room, &s->full[slot], sh.product);
            }
            __syncwarp();
            r.pos += size;
            r.used += gap + size;
            ++r.live;
            r.head.step(a.c.slots);
        }
    }
    return true;
}

// ---- accumulators ----
template <class P>
__device__ __forceinline__ bool finish_all(const typename P::Args &a, uint8_t *lists, Shared *s, const Share &sh, int w, int lane, uint32_t tmem, uint32_t &seg)
{
    const int64_t part = (int64_t)a.c.part_cols * kRows;
    const int row = w * 32 + lane;
    // (of its own for each product: one CTA may be at the second while another still joins a tile of the first)
    float *const all_parts = a.c.parts + sh.product * 2 * (int64_t)a.c.shares * part;
    unsigned int *const counts = a.c.counts + sh.product * a.c.shares;
#pragma unroll 1
    for (Walk<P> walk(a, lists, sh); walk.more(); walk.next()) {
        const Tile &tile = walk.tile;
        const int buf = seg & 1;
        typename P::Cols cols = P::cols(a, lists, tile, w, lane);
        // the tile's contributors besides this one, and its place among them
        const int from = walk.from(), to = walk.to();
        const int others = to - from, place = sh.me - from;
        const uint32_t lanes = tmem + ((uint32_t)w << 21), acc = lanes + buf * a.c.acc_cols;
        float v[16];
        // the contributors take turns at the additions, 16 columns each
        const bool adds = P::kAdds && P::adds(a);
        // before the products are ready (to columns of their own), or after: a loop, so that their code is there once
#pragma unroll 1
        for (int turn = 0; turn < 2; ++turn) {
            if (adds && (a.c.add_col != 0) == (turn == 0))
                P::add(a, lists, tile, w, lane, place * 16, (others + 1) * 16, turn == 0 ? lanes + a.c.add_col : acc, turn != 0);
            if (turn == 0) {
                const bool ok = bar_wait(&s->acc_full[buf], (seg >> 1) & 1, s, a.c);
                if (threadIdx.x == 128 && others) s->before[buf] = *(volatile unsigned int *)&counts[to];
                if (!epilogue_all(ok)) return false;
                fence_after();
            }
        }
        if (adds && a.c.add_col) {
#pragma unroll 1
            for (int c = place * 16; c < tile.n16; c += (others + 1) * 16) {
                float d[16];
                read16(lanes + a.c.add_col + c, d);
                read16(acc + c, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] += d[i];
                write16(acc + c, v);
            }
        }
        bool last = others == 0 || s->before[buf] == (unsigned)others;      // the other parts are all down
        if (!last) {
            // shares that begin inside a tile have it as the first piece of their rest, the one that begins it as its last
            float4 *mine = (float4 *)(all_parts + (2 * (int64_t)sh.me + (walk.k0 > 0 ? 0 : 1)) * part) + row;
#pragma unroll 1
            for (int c = 0; c < tile.n16; c += 16) {
                read16(acc + c, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) mine[((c >> 2) + i) * kRows] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
            __threadfence();
            epilogue_all(true);
            if (threadIdx.x == 128) s->after = atomicAdd(&counts[to], 1u);
            epilogue_all(true);
            last = s->after == (unsigned)others;
        }
        if (last) {
            if (others) __threadfence();
            const float4 *parts = (const float4 *)(all_parts + (2 * (int64_t)from) * part) + row;
            switch (others) {
            case 0: break;
            case 1: join<1>(tile.n16, acc, parts, part / 2, place); break;
            case 2: join<2>(tile.n16, acc, parts, part / 2, place); break;
            case 3: join<3>(tile.n16, acc, parts, part / 2, place); break;
            default: join<4>(tile.n16, acc, parts, part / 2, place); break;
            }
            store_tile<P>(a, lists, tile, cols, w, lane, acc, sh.product);
            if (others && threadIdx.x == 128) counts[to] = 0;
        }
        fence_before();
        bar_arrive(&s->acc_empty[buf]);
        if (P::tells(sh.product) && last) {
            __threadfence();
            epilogue_all(true);
            if (threadIdx.x == 128) P::tell(a, lists, tile);
        }
        ++seg;
    }
    return true;
}

// After a wait gave up, one thread, when all roles have ended: waits (bounded) until the loads in flight have landed, before the CTA's memory goes
// to another one.  A stage of which only the weights or only the tokens were asked for lacks the other's arrival.
__device__ __forceinline__ void let_loads_land(Shared *s, const Common &c)
{
    const uint32_t slots = c.slots, w = s->issued[0], t = s->issued[1], end = w > t ? w : t;
    int polls = 0;
#pragma unroll 1
    for (uint32_t n = end > slots ? end - slots : 0; n < end; ++n) {
        uint64_t *full = &s->full[n % slots];
        if (n >= w || n >= t) bar_arrive(full);
        while (polls < c.wait_limit && !bar_try(full, (n / slots) & 1)) ++polls;
    }
}

template <class P>
__global__ void __launch_bounds__(kThreads, 1) k_stream(const __grid_constant__ typename P::Args a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *weights = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t slot_bytes = kWeightBytes * a.c.steps;
    uint8_t *ring = weights + slot_bytes * a.c.slots;
    Shared *s = (Shared *)(ring + a.c.ring_bytes);
    uint8_t *lists = (uint8_t *)(s + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kSlots; ++i) { bar_init(&s->full[i], 2); bar_init(&s->empty[i], 1); }
        for (int i = 0; i < 2; ++i) { bar_init(&s->acc_full[i], 1); bar_init(&s->acc_empty[i], 128); }
        bar_init(&s->drained, 1);
        s->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s->tmem)), "r"(a.c.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        fence_before();
    }
    P::prologue(a);
    P::setup(a, lists);
    __syncthreads();
    fence_after();
    const uint32_t tmem = s->tmem;

    if (warp == 0) {
        if (a.c.wait_first) grid_dependency_wait();
        Place at = {0, 0, 0};
        bool ok = true;
#pragma unroll 1
        for (int n = 0; ok; ++n) {
            const int share = share_at<P>(a, lists, s, n, ok);
            if (share < 0) break;
            ok = load_all_weights<P>(a, lists, s, share_of<P>(a, lists, share), n, lane, smem_addr(weights), at);
        }
        if (lane == 0) s->issued[0] = at.passed;
        // the end marker: nothing to load
        if (ok) ok = __all_sync(0xffffffffu, bar_wait(&s->empty[at.slot], at.round ^ 1, s, a.c));
        if (ok && elect_one()) bar_arrive(&s->full[at.slot]);
    } else if (warp == 2) {
        Ring r = {{0, 0, 0}, {0, 0, 0}, 0, 0, 0};
        bool ok = true;
#pragma unroll 1
        for (int n = 0; ok; ++n) {
            const int share = share_at<P>(a, lists, s, n, ok);
            if (share < 0) break;
            ok = load_all_tokens<P>(a, lists, s, share_of<P>(a, lists, share), lane, smem_addr(ring), r);
        }
        if (lane == 0) s->issued[1] = r.head.passed;
        while (ok && r.live == (uint32_t)a.c.slots) ok = free_one(a.c, s, r);
        if (ok && elect_one()) {
            s->stage[r.head.slot].what = kEnd;
            bar_arrive(&s->full[r.head.slot]);
        }
    } else if (warp == 3) {
        if (P::kEarly) P::early(a, lists, 0, lane);
        // ---- what the additions will read ----
        if (P::kAdds && P::adds(a) && a.c.add_col) {
            const Share sh = share_of<P>(a, lists, blockIdx.x);
#pragma unroll 1
            for (Walk<P> w(a, lists, sh); w.more(); w.next()) {
                const int from = w.from(), to = w.to();
                for (int c = (sh.me - from) * 16; c < w.tile.n16; c += (to - from + 1) * 16) P::prefetch(a, w.tile, lane, c);
            }
        }
    } else if (warp == 1) {
        // ---- products ----
        if (a.c.wait_first) grid_dependency_wait();
        const uint32_t base = smem_addr(weights);
        uint32_t seg = 0;                       // pieces of tiles begun
        for (Place at = {0, 0, 0};; at.step(a.c.slots)) {
            if (!__all_sync(0xffffffffu, bar_wait(&s->full[at.slot], at.round, s, a.c))) break;
            const Stage st = s->stage[at.slot];
            if (st.what & kEnd) break;
            if (st.what & kFirst) {
                ++seg;
                if (seg > 2 && !__all_sync(0xffffffffu, bar_wait(&s->acc_empty[(seg - 1) & 1], ((seg - 3) >> 1) & 1, s, a.c))) break;
            }
            fence_after();
            if (elect_one()) {
                const uint32_t d = tmem + ((seg - 1) & 1) * a.c.acc_cols;
                const uint32_t idesc = instruction(st.what >> 16);
                const int products = (int)(st.what >> 4) & 0xfff;
                uint64_t da = operand(base + at.slot * slot_bytes), db = operand(st.tokens);
                bool add = !(st.what & kFirst);
                int j = 0;
                for (; j + 4 <= products; j += 4) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) mma(d, da + 2 * q, db + 2 * q, idesc, q > 0 || add);
                    add = true;
                    da += kWeightBytes >> 4;
                    db += st.room >> 4;
                }
                for (; j < products; ++j, da += 2, db += 2) { mma(d, da, db, idesc, add); add = true; }
                mma_commit(&s->empty[at.slot]);
                if (st.what & kLast) mma_commit(&s->acc_full[(seg - 1) & 1]);
            }
            __syncwarp();
        }
        if (s->abort) {                         // gave up: products in flight end before their operands go away (bounded)
            if (elect_one()) mma_commit(&s->drained);
            for (int n = 0; n < a.c.wait_limit && !bar_try(&s->drained, 0); ++n) {}
        }
        __syncwarp();
    } else {
        grid_dependency_wait();                 // scratch and outputs may still be in use by the kernel before
        if (P::kEarly) P::early(a, lists, warp - 3, lane);
        uint32_t seg = 0;
        bool ok = true;
#pragma unroll 1
        for (int n = 0; ok; ++n) {
            const int share = share_at<P>(a, lists, s, n, ok);
            if (P::kClaims) ok = epilogue_all(ok);          // (the warps agree, as they meet at barriers)
            if (share < 0 || !ok) break;
            ok = finish_all<P>(a, lists, s, share_of<P>(a, lists, share), warp - 4, lane, tmem, seg);
        }
    }
    fence_before();
    __syncthreads();
    if (s->abort && threadIdx.x == 0) let_loads_land(s, a.c);
    P::leave(a, lists);
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(a.c.tmem_cols) : "memory");
}

#endif  // __CUDACC__

}  // namespace mw_stream
