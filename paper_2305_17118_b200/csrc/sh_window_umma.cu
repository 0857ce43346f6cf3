// sh_window_prefill on the 5th-generation tensor cores: 16-bit types, head_dim 64 or 128.
//
// out = softmax(scale Q.K^T + mask) V with the running maximum and sum of an online softmax.  A work item is one key head and
// two query tiles; a tile is 128 rows = TPT tokens x GB query heads of the group (heads innermost), so the heads that share keys
// share a tile and the tile spans few tokens.  The keys come in tiles of 64: first the slots of the cache, then the chunk's own
// rows; tiles that none of the item's rows can see are never loaded, tiles that a query tile does not see are not multiplied for it.
//
//   warps 0-3, 4-7   softmax of query tile 0 and 1: thread = row.  S from tensor memory, mask, exponentials, P (16 bits) back into
//                    the columns of S, the rare rescaling of O, and the division and store at the end
//   warps 8, 9       issue the MMAs of query tile 0 and 1: S = Q.K^T (both operands in shared memory, K-major), O += P.V (P in
//                    tensor memory, V MN-major)
//   warp 10          works out the steps (key tiles of an item) and who sees what in them, publishes them in a ring, and requests
//                    the tiles (tiled TMA copies, 128-byte swizzle; rows outside a tensor are zeros)
//
// A query tile has two buffers of S: S(n+1) is made while the softmax of step n runs, and goes into the buffer whose P the product
// P.V(n-1), issued before it, has read (the tensor pipe keeps the order of one warp's MMAs).  Tensor memory is full with that: two
// query tiles x (2 x 64 columns of S + 128 of O).  With one buffer of 128 columns each step waited for softmax and both products in
// turn: 2.3 instead of 2.0 ms for the 32768-token prompt below.
//
// A running CTA takes over the items of CTAs that have not started (cluster launch control), so it sets up once and long and short
// items even out: 153 -> 139 us for prompts of 1 to 4001 tokens, 150 -> 118 us for continued chunks, whose contexts differ most (97
// with the sequences in order of what they have cached).
// The next item's queries have a place of their own, so its first S follows the last one of the present item at once.  What finished
// leaves by a copy from shared memory (8192 tokens, window 256: 77 -> 71 us against stores by the threads).
//
// P is rounded once, to the storage type; its row sum is taken before the rounding, in fp32.  That is a price paid for speed: the
// single-token kernels hold P in two 16-bit parts, and here too the low part would have a place (the columns of S that P leaves free), but
// P.V would be issued twice and every weight split.  Measured with one part and with two: 132 and 151 us for prompts of 1 to 4001 tokens,
// 1.88 and 2.53 ms for the 32768 tokens below, 97 and 113 us for continued chunks.  With one the error against 64 bits is 1.2 to 1.4 times
// that of the output's rounding alone.
// The subtracted maximum is only renewed when it has grown by more than 8 (log2), so weights stay below 2^8; fp16 weights carry a
// factor 2^7 (at most 2^15), which cancels in O / l: weights down to 2^-21 of the row's largest keep 11 bits, below that they are multiples
// of 2^-31 of it.  (Renewing at 4, with a factor of 2^11, would reach 2^-25 and cost fp16 prompts 2 to 3 %.)
//
// Weights of unseen keys are zero, but 0 * NaN is NaN: a value row that is not finite poisons rows that do not see it (a slot
// that holds no token, a later token, another sequence's row).  That shows as an O that is not finite; such rows are computed
// again after the CTA's last item, one warp per row over the visible keys only.  Rows whose result is rightly not finite take that way
// too.  As that is slow (0.1 to 0.6 us a row and key), and slots that hold no token may hold anything, the load warp zeroes the rows of a value tile behind the sequence's last
// slot or token before it hands the tile on (512 tokens over 1000 in a cache with NaN behind them: 3655 -> 34 us).
//
// 32768 tokens, window 4096, 16 sinks, 32 query and 8 key heads of 128, fp16: 1.84 to 1.90 ms replayed from a graph, 1100 TFLOP/s, 0.68 to
// 0.70 of the measured bf16 peak (2.14 ms a call when calls follow for seconds, under the power cap); 8192 tokens, full causal
// attention, bf16: 0.48 ms, 1150 TFLOP/s.  Bound by the operands' reads from shared memory and the chain around them: a step takes about
// 1950 cycles, of which the operands (48 KB per S of 64 keys, 16 KB per P.V, 32 KB written) need 1250 and the exponentials 1024 on each
// quarter of the SM; with the exponentials left out it took 1600.  A part of the exponentials on the FMA
// pipe (a quarter of them by a polynomial) gained nothing at this register split: 473 against 482 us for the 8192 tokens.
// Items of few steps pay for their ends: 8192 tokens with window 1024 (18 steps an item) run at 850 TFLOP/s, with window 256 at 485.
#include <cuda.h>
#include <math_constants.h>

#include <algorithm>

#include "sh_elem.cuh"
#include "sh_pairs.cuh"
#include "sh_umma.cuh"
#include "sh_window.cuh"

namespace {

using namespace shasync;
using namespace shpair;
using namespace shumma;
using namespace shwin;

constexpr int TM = 128, TN = 64;           // rows of a query tile, keys of a key tile
constexpr int QHALF = TM * 128, HALF = TN * 128;      // bytes of a tile's rows x 64 elements
constexpr int SOFTMAX_WARPS = 8, NTH = 384;      // 8 softmax warps, 2 that issue MMAs, 1 that loads; the last one only makes a whole warpgroup
constexpr int REGS_SOFTMAX = 184, REGS_OTHER = 136;    // 256 * 184 + 128 * 136 = 384 * 168, what the CTA is launched with
constexpr float RENEW = 8.f;               // log2 growth of the maximum at which O is rescaled

__device__ int g_window_error;             // code of the first bounded wait that gave up
#ifdef SH_DEBUG_BOUNDS
__device__ int g_window_selftest = -1;     // self-test: the work item whose load warp gives up before it has listed the item
#endif

constexpr int STEPS = 8, BAR_BYTES = 2048; // steps in flight between the load warp and the others; barriers, step ring, rows to do again
constexpr int AGAIN = 16;                  // items of a warp with such rows, at most: see Bars

template <int D> struct Cfg {
    static constexpr int QTILE = D / 64 * QHALF, TILE = D / 64 * HALF;      // bytes of a query tile, of a key or value tile
    static constexpr int STAGES = D == 128 ? 3 : 6;    // steps in flight: a stage holds a key and a value tile
    static constexpr int OFF_KV = 4 * QTILE;           // query tiles of two items; a finished item's tiles serve to lay out its output
    static constexpr int OFF_BAR = OFF_KV + STAGES * 2 * TILE;
    static constexpr int SMEM = OFF_BAR + BAR_BYTES;
    static constexpr int O_COL = 4 * TN;               // tensor memory: per query tile two buffers of S (P inside), then O0, O1
    static_assert(SMEM <= 232448 && O_COL + 2 * D <= 512, "");
};

// A step is one key tile of one item.  The warp that requests the loads works out what it asks for and who sees what, and hands
// that to the MMA warp and the softmax warps through a ring.
enum {
    STEP_NEED0 = 1, STEP_NEED1 = 2,        // the query tile sees keys of this step
    STEP_WHOLE0 = 4, STEP_WHOLE1 = 8,      // every row of the query tile sees every key
    STEP_CACHE = 16, STEP_FIRST = 32, STEP_LAST = 64, STEP_END = 128,
    STEP_PART = 256,                       // other CTAs have key tiles of this item too
    STEP_DEAD = 512                        // the tile ends in rows that are not the sequence's
};
struct __align__(16) Step {
    int flags, x;                          // first slot of the tile, or its first row in the chunk
    int first, count;                      // the sequence's rows of the chunk tensors
    int cached, a, kvh, hb;                // as in Item
    int head, ring2;                       // end of the slots [sinks, head), end of the slots [head, ring2)
    int id, pad;                           // of the item
};
struct Bars {
    uint64_t q_full[2][2], q_free[2][2];   // [query tile][item mod 2]: landed / its place may be filled again
    uint64_t full[6], empty[6];            // stages: landed / read by the MMAs
    uint64_t s_full[2][2], p_ready[2][2];  // [query tile][buffer of S]
    uint64_t pv_done[2][2];                // (by buffer too: when a softmax warp waits for P.V(n), only P.V(n-2) is sure to be over)
    uint64_t step_full[STEPS], step_empty[STEPS];
    uint4 claim;                           // answer to the last request for work
    uint64_t claimed;
    uint64_t landed;                       // a tile whose dead rows are zeroed before anybody reads it
    Step steps[STEPS];
    // Rows to be computed again wait for the end of the CTA's items, when nobody waits for their warps any more: 32 of them over a million
    // keys take up to 19 s.  An item that begins after the first of them was noted asks for no further one (CTAs that have not started
    // take the rest).  So a softmax warp may still come to the item of the step it has read ahead, those of STEPS published steps
    // behind that, the item being published and the one asked for already.
    int2 again[SOFTMAX_WARPS][AGAIN];      // (item, rows of the warp)
    int again_count[SOFTMAX_WARPS], no_more;
    uint32_t tmem;
    int abort_flag;
};
static_assert(AGAIN >= STEPS + 4, "see Bars");
static_assert(sizeof(Bars) <= BAR_BYTES, "barrier block");

// Wait for a phase, bounded by time, in few instructions: the code of a wait that gave up goes to the CTA's abort word, and from
// there to g_window_error at the end.
#ifdef SH_DEBUG_BOUNDS
constexpr unsigned long long LIMIT_NS = 200000000ull;      // (its self-test waits for it)
#else
constexpr unsigned long long LIMIT_NS = 8000000000ull;
#endif
__device__ __forceinline__ bool wait_for(Bars *bars, uint64_t *bar, uint32_t parity, int code) {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < LIMIT_NS)
        if (mbar_try_wait(bar, parity)) return true;
    if (code) *(volatile int *)&bars->abort_flag = code;
    return false;
}

struct UmmaParams {
    WindowParams w;
    int tpt, gb, hblocks;                  // tokens and heads of a tile, head blocks per key head
    bool copy_out;                         // a warp's 32 rows are whole tokens
    int share;                             // CTAs of the device per item
    int parts;                             // the most CTAs that an item's key tiles are dealt out to (1: results go straight to the output)
};

// Few items over many keys: the key tiles of an item are dealt out to several CTAs, 4 tiles each at least, whose results a second
// launch merges.  It pays when the tiles that no CTA has to walk over any more, at about 1.1 us each, outweigh that launch (2 us where
// nothing was dealt out, 4 to 7 us else).  An item's count depends on the tiles it needs and on the number of items, not on whether
// there is a cache.  Measured with 32 query heads over 8, 128 wide, one CTA an item against several: 64 tokens over 32768 538 -> 56 us
// (18 parts), over 8000 147 -> 28 us; 16 over 2000 34 -> 16 us (7 parts), over 832 18.3 -> 14.5 us (3 parts); 400 over none in a cache
// of 4100 14.7 -> 17.3 us (the second launch finds nothing to do).
__host__ __device__ __forceinline__ int parts_of(long long tiles, int share) {
    const int parts = tiles / 4 < share ? (int)(tiles / 4) : share;
    return parts >= 2 && tiles - tiles / parts > 8 ? parts : 1;
}

// What a part leaves for the merge, rows next to each other: O as [item's part][query tile][D / 4][row] of 4 floats, then what its
// exponents are counted from and its sum (below zero: nothing else was written), then for each item: its parts, its first row, the
// rows from there to the sequence's end.
constexpr int MAX_SHARE = 160;             // items times parts
template <int D> __device__ __forceinline__ float4 *part_o(const UmmaParams &p, int id, int t) { return reinterpret_cast<float4 *>(p.w.part) + (id * 2 + t) * (D / 4) * TM; }
template <int D> __device__ __forceinline__ float2 *part_sum(const UmmaParams &p, int id, int t) { return reinterpret_cast<float2 *>(p.w.part + MAX_SHARE * 2 * TM * D) + (id * 2 + t) * TM; }
template <int D> __device__ __forceinline__ int4 *part_item(const UmmaParams &p) { return reinterpret_cast<int4 *>(p.w.part + MAX_SHARE * 2 * TM * (D + 2)); }

__device__ __forceinline__ uint64_t desc_sw128(uint32_t saddr, uint32_t lbo, uint32_t sbo) { return smem_desc(saddr, lbo, sbo) | (2ull << 61); }

__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_ld32_nowait(uint32_t taddr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
// Wait for this thread's tensor-memory loads; the values pass through the asm, so that no use of them moves before the wait.
template <int N>
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tmem_ld16_nowait(uint32_t taddr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tma_3d(void *dst, const CUtensorMap *map, int c0, int c1, int c2, uint64_t *bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                     smem_u32(dst)),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
                 : "memory");
}
// Key and value tiles: the halves of a row are the outermost dimension of the map, so one copy brings both.
__device__ __forceinline__ void tma_4d(void *dst, const CUtensorMap *map, int head, int token, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(head), "r"(token), "r"(0), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tma_5d(void *dst, const CUtensorMap *map, int slot, int head, int sequence, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(slot), "r"(head), "r"(sequence), "r"(0), "r"(smem_u32(bar))
        : "memory");
}
// Cluster launch control: the grid has a CTA for every item, and a running CTA takes over the item of one that has not started yet.
// Ask for one (the 16-byte answer lands in shared memory, counted on `bar`) ...
__device__ __forceinline__ void claim_request(uint4 *answer, uint64_t *bar) {
    mbar_arrive_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(answer)), "r"(smem_u32(bar))
                 : "memory");
}
// ... and read the answer: the index of the CTA taken over, or -1: there is none left (then nobody may ask again).
__device__ __forceinline__ int claim_read(const uint4 *answer) {
    int x, got;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        ".reg .b128 r;\n\t"
        "ld.shared.b128 r, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "selp.s32 %1, 1, 0, p;\n\t"
        "mov.s32 %0, -1;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, r;\n\t}"
        : "=r"(x), "=r"(got)
        : "r"(smem_u32(answer))
        : "memory");
    return got ? x : -1;
}
// A tile of output rows, laid out like a query tile, to global memory; tracked by the thread's bulk group.
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, const void *src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(reinterpret_cast<uint64_t>(map)),
                 "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(src))
                 : "memory");
}
// One lane of the warp, which must be converged.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(p));
    return p != 0;
}

// One work item and the key tiles it has to walk over.  Tiles 0 .. ctiles - 1 are blocks of TN cache slots, tile ctiles + j holds the
// chunk's rows TN * j ...
struct Item : Ring {
    int seq, first, count;                 // seq < 0: there is no such item
    int kvh, hb, part;
    int a;                                 // first token of query tile 0, counted in the chunk; tile t starts at a + t * tpt
    int ctiles, jlo, jhi, tpt;

    __device__ __forceinline__ int ring2() const { return wrapped ? sinks + window : 0; }
    __device__ __forceinline__ int from(int t) const { return a + t * tpt; }
    __device__ __forceinline__ bool has(int t) const { return from(t) < count; }
    __device__ __forceinline__ int last(int t) const { return min(from(t) + tpt, count) - 1; }
    // does query tile t see a key of tile i?
    __device__ __forceinline__ bool need(int t, int i) const {
        if (!has(t)) return false;
        const int oldest = cached + from(t) - window + 1;      // position
        if (i < ctiles) return any(i * TN, i * TN + TN, oldest);
        const int j = (i - ctiles) * TN;
        return j <= last(t) && (cached + j + TN - 1 >= oldest || cached + j < sinks);
    }
    // does every row of query tile t see every key of tile i?  (a tile over several runs of slots counts as no)
    __device__ __forceinline__ bool whole(int t, int i) const {
        const int newest = cached + last(t) - window + 1;      // the last row's window starts here
        if (i < ctiles) {
            const int x = i * TN, y = x + TN;
            if (y <= min(sinks, cached)) return true;
            if (x >= sinks && y <= head) return cached - head + x >= newest;
            return wrapped && x >= head && y <= sinks + window && cached - window + x - head >= newest;
        }
        const int j = (i - ctiles) * TN;
        return j + TN - 1 <= from(t) && (cached + j >= newest || cached + j + TN <= sinks);
    }
    __device__ __forceinline__ int next(int i) const {         // -1: no further tile
        for (++i; i < ctiles; ++i)
            if (need(0, i) || need(1, i)) return i;
        if (i - ctiles < jlo && cached + (i - ctiles) * TN >= sinks) i = ctiles + jlo;      // what lies between the sinks and the window
        return i <= ctiles + jhi ? i : -1;
    }
};

// Where the search for an item left off: a CTA's items mostly come in rising order, and the sequences before are not counted again.
struct Found {
    int base = 0;
    long long before = 0;
};
__device__ __forceinline__ Item find_item(const UmmaParams &p, int id, Found &from) {
    const int per = p.w.hk * p.hblocks * p.parts, in = id % per;
    const int lane = threadIdx.x & 31, span = 2 * p.tpt;
    const int tile = id / per;
    if (tile < from.before) from = Found();
    Item r;
    r.seq = -1;
    r.a = r.tpt = r.count = 0;
    long long before = from.before;
    for (int base = from.base; base < p.w.sequences; base += 32) {
        int first = 0, count = 0, cached = 0;
        if (base + lane < p.w.sequences) sequence_rows(p.w, base + lane, first, count, cached);
        const int mine = (count + span - 1) / span;
        // of 32 sequences those with most cached keys to walk over come first (103 -> 96 us for chunks of 17 to 256 tokens over 1 to
        // 2052 rows; ordered by the tokens of the chunk too, prompts of 1 to 4001 tokens took 132 instead of 130 us)
        const unsigned key = (unsigned)(p.w.kc ? min(cached, p.w.sinks + p.w.window) / TN : 0) << 5 | (31 - lane);
        long long upto = 0, all = 0;
#pragma unroll 4
        for (int o = 0; o < min(32, p.w.sequences - base); ++o) {
            const unsigned other = __shfl_sync(0xffffffffu, key, o);
            const int x = __shfl_sync(0xffffffffu, mine, o);
            all += x;
            if (other >= key) upto += x;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, before + upto > tile && before + upto - mine <= tile);
        if (hit) {
            const int l = __ffs(hit) - 1;
            from.base = base;
            from.before = before;
            r.seq = base + l;
            r.first = __shfl_sync(0xffffffffu, first, l);
            r.count = __shfl_sync(0xffffffffu, count, l);
            r.cached = __shfl_sync(0xffffffffu, cached, l);
            // a sequence's items go from its end to its start, where causality leaves fewer keys: the short ones come last
            r.a = (int)(before + __shfl_sync(0xffffffffu, upto, l) - 1 - tile) * span;
            break;
        }
        before += all;
    }
    if (r.seq < 0) return r;
    r.part = in % p.parts;
    r.kvh = in / p.parts / p.hblocks; r.hb = in / p.parts % p.hblocks;
    r.tpt = p.tpt;
    static_cast<Ring &>(r) = Ring(p.w.kc ? r.cached : 0, p.w.sinks, p.w.window);
    r.ctiles = (r.live + TN - 1) / TN;
    r.jlo = max(0, r.a - r.window + 1) / TN;
    r.jhi = r.last(r.has(1) ? 1 : 0) / TN;
    return r;
}

// Keys of a tile that the query at chunk index qi sees: up to three runs [lo, hi) counted from the tile's first key.
struct Runs {
    int lo[3], hi[3];
};
__device__ __forceinline__ Runs visible_runs(bool in_cache, int x, int cached, int head, int ring2, int sinks, int window, int qi) {
    Runs r;
    if (in_cache) {
        r.lo[0] = 0; r.hi[0] = min(sinks, cached) - x;
        r.lo[1] = max(sinks, head + qi - window + 1) - x; r.hi[1] = head - x;
        r.lo[2] = head + qi + 1 - x; r.hi[2] = ring2 - x;
    } else {
        r.lo[0] = 0; r.hi[0] = min(sinks - cached, qi + 1) - x;
        r.lo[1] = max(0, qi - window + 1) - x; r.hi[1] = qi + 1 - x;
        r.lo[2] = 0; r.hi[2] = 0;
    }
    return r;
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : (n <= 0 ? 0u : (1u << n) - 1u); }
__device__ __forceinline__ uint32_t run_bits(const Runs &r, int base) {
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) m |= low_bits(r.hi[k] - base) & ~low_bits(r.lo[k] - base);
    return m;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// One row by one warp, over its visible keys only, in fp32 on CUDA cores: for rows next to values that are not finite.
template <typename T, int D>
__device__ __noinline__ void slow_row(const UmmaParams &u, int id, int qi, int h) {
    constexpr int E = D / 32;
    const WindowParams &p = u.w;
    Found from;
    const Item w = find_item(u, id, from);
    if (w.seq < 0 || qi < 0 || qi >= w.count) return;      // (only where a CTA gave up a wait)
    const int lane = threadIdx.x & 31;
    float q[E], o[E], m = -CUDART_INF_F, l = 0.f;
    const T *qr = reinterpret_cast<const T *>(p.q.p + (long long)(w.first + qi) * p.q.ts + h * p.q.hs) + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) { q[e] = (float)qr[e] * p.scale_log2e; o[e] = 0.f; }
    for (int i = w.next(-1); i >= 0; i = w.next(i)) {
        const bool in_cache = i < w.ctiles;
        const int base = (in_cache ? i : i - w.ctiles) * TN;
        const Runs runs = visible_runs(in_cache, base, w.cached, w.head, w.ring2(), w.sinks, w.window, qi);
        for (int c = 0; c < TN; ++c) {
            if (!((run_bits(runs, c & ~31) >> (c & 31)) & 1u)) continue;
            const long long ko = in_cache ? w.seq * p.css + w.kvh * p.chs + (long long)(base + c) * p.cls : (long long)(w.first + base + c) * p.k.ts + w.kvh * p.k.hs;
            const long long vo = in_cache ? ko : (long long)(w.first + base + c) * p.v.ts + w.kvh * p.v.hs;
            const T *kr = reinterpret_cast<const T *>((in_cache ? p.kc : p.k.p) + ko) + lane * E;
            const T *vr = reinterpret_cast<const T *>((in_cache ? p.vc : p.v.p) + vo) + lane * E;
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) s = fmaf(q[e], (float)kr[e], s);
#pragma unroll
            for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
            const float mn = fmaxf(m, s), b = mn == -CUDART_INF_F ? 0.f : mn, keep = ex2_approx(m - b), e1 = ex2_approx(s - b);
            m = mn;
            l = l * keep + e1;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(e1, (float)vr[e], o[e] * keep);
        }
    }
    T *dst = reinterpret_cast<T *>(p.out.p + (long long)(w.first + qi) * p.out.ts + h * p.out.hs) + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) dst[e] = (T)(o[e] / l);
}

// Note rows of a softmax warp that have to be computed again, and do them.  (Calls, as inlined they cost the loop over the steps
// 3 %: 534 against 518 us for 8192 tokens, full causal attention, with their append.)
__device__ __noinline__ void note_again(Bars *bars, int warp, int id, unsigned rows) {
    if ((threadIdx.x & 31) == 0) {
        const int n = bars->again_count[warp];
        if (n < AGAIN) {
            bars->again[warp][n] = make_int2(id, (int)rows);
            bars->again_count[warp] = n + 1;
            *(volatile int *)&bars->no_more = 1;
        } else {
            *(volatile int *)&bars->abort_flag = 0x626;
        }
    }
    __syncwarp();
}

template <typename T, int D>
__device__ __noinline__ void do_again(const UmmaParams &p, const int2 *list, int count, int t, int quarter) {
    for (int i = 0; i < count; ++i) {
        const int2 e = list[i];
        Found from;
        const Item w = find_item(p, e.x, from);
        for (unsigned rows = (unsigned)e.y; rows; rows &= rows - 1) {
            const int r = quarter * 32 + __ffs(rows) - 1;
            slow_row<T, D>(p, e.x, w.from(t) + r / p.gb, w.kvh * p.w.g + w.hb * p.gb + r % p.gb);
        }
    }
}

template <typename T> struct Fmt;
template <> struct Fmt<__half> { static constexpr int CODE = 0; static constexpr float LIFT = 7.f; };
template <> struct Fmt<__nv_bfloat16> { static constexpr int CODE = 1; static constexpr float LIFT = 0.f; };

template <typename T, int D>
__global__ void __launch_bounds__(NTH, 1)
sh_window_prefill_umma_kernel(const __grid_constant__ UmmaParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                              const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_kc,
                              const __grid_constant__ CUtensorMap map_vc, const __grid_constant__ CUtensorMap map_o) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) unsigned char sm[];
    unsigned char *kv = sm + C::OFF_KV;
    Bars *bars = reinterpret_cast<Bars *>(sm + C::OFF_BAR);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto aborted = [&]() { return *(volatile int *)&bars->abort_flag != 0; };

    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) {
        for (int t = 0; t < 2; ++t) {
            for (int b = 0; b < 2; ++b) {
                mbar_init(&bars->q_full[t][b], 1); mbar_init(&bars->q_free[t][b], 4);
                mbar_init(&bars->pv_done[t][b], 1); mbar_init(&bars->s_full[t][b], 1); mbar_init(&bars->p_ready[t][b], 4);
            }
        }
        for (int s = 0; s < C::STAGES; ++s) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], 2); }
        mbar_init(&bars->claimed, 1); mbar_init(&bars->landed, 1);
        for (int s = 0; s < STEPS; ++s) { mbar_init(&bars->step_full[s], 1); mbar_init(&bars->step_empty[s], SOFTMAX_WARPS); }
        for (int w = 0; w < SOFTMAX_WARPS; ++w) bars->again_count[w] = 0;
        bars->abort_flag = bars->no_more = 0;
        if ((smem_u32(sm) & 1023u) != 0) bars->abort_flag = 0x620;      // the swizzled tiles need the alignment the declaration asks for
        fence_barrier_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = bars->tmem;             // 0: all 512 columns are this CTA's
    bool ok = __all_sync(0xffffffffu, !aborted() && tbase == 0);
    if (tbase != 0) *(volatile int *)&bars->abort_flag = 0x621;

    if (warp >= SOFTMAX_WARPS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_OTHER));
    // What these warps issue takes its operands from uniform registers.  So their control flow and values are kept uniform in a
    // way the compiler can see: outcomes of waits go through a vote, values from memory through a shuffle.
    if (warp < SOFTMAX_WARPS + 2) {
        // ------------------------------------------------------------------------------------------------ MMAs
        // One warp per query tile.  A step's entry in the ring is published with its loads and not written again before this warp
        // has released the stage of a later step.
        const int t = __shfl_sync(0xffffffffu, warp, 0) - SOFTMAX_WARPS;
        constexpr uint32_t idesc_s = instr_desc(Fmt<T>::CODE, 0, TM, TN), idesc_pv = instr_desc(Fmt<T>::CODE, 0, TM, D) | (1u << 16);
        // descriptors: the high word is the same for all operands of a kind, the low word holds address / 16 in its low bits
        const uint64_t q_desc = desc_sw128(smem_u32(sm) + t * C::QTILE, 16, 1024), k_desc = desc_sw128(smem_u32(kv), 16, 1024),
                       v_desc = desc_sw128(smem_u32(kv) + C::TILE, HALF, 1024);
        auto plus = [](uint64_t d, uint32_t bytes) { return (d & 0xffffffff00000000ull) | (uint32_t)((uint32_t)d + (bytes >> 4)); };
        uint32_t st = 0, par = 0;                     // stage and parity of the next step
        uint32_t items = 0, steps = 0, done_s = 0, done_pv = 0;      // products S and P.V issued
        uint32_t due = C::STAGES;                     // stage of the step whose P.V is due (STAGES: none)
        bool due_adds = false, begun = false;         // that P.V adds to O (its item's first overwrites it); S of this item was issued
        auto issue_pv = [&]() {
            const uint32_t b = done_pv & 1;
            ok = __all_sync(0xffffffffu, wait_for(bars, &bars->p_ready[t][b], (done_pv >> 1) & 1, 0x604));
            tc_fence_after();
            if (ok && elect_one()) {
                const uint64_t vd = plus(v_desc, due * 2 * C::TILE);
#pragma unroll
                for (int x = 0; x < TN / 16; ++x) umma_ts(C::O_COL + t * D, (2 * t + b) * TN + x * 8, plus(vd, x * 2048), idesc_pv, due_adds || x > 0);
                umma_commit(&bars->pv_done[t][b]);
                umma_commit(&bars->empty[due]);
            }
            __syncwarp();
            ++done_pv;
            due = C::STAGES;
        };
        while (ok) {
            // (if the next step is not there yet - the first of an item may be late - the P.V that is due does not wait for it)
            if (due < C::STAGES && !__all_sync(0xffffffffu, mbar_test(&bars->full[st], par))) issue_pv();
            if (!ok) break;
            ok = __all_sync(0xffffffffu, wait_for(bars, &bars->full[st], par, 0x603));
            if (!ok) break;
            const int now = __shfl_sync(0xffffffffu, *(volatile int *)&bars->steps[steps++ % STEPS].flags, 0);
            if (now & STEP_END) {
                if (due < C::STAGES) issue_pv();
                break;
            }
            if (now & STEP_FIRST) {
                ok = __all_sync(0xffffffffu, wait_for(bars, &bars->q_full[t][items & 1], (items >> 1) & 1, 0x601) && !aborted());
                if (!ok) break;
                ++items;
                begun = false;
            }
            const bool need = now & (STEP_NEED0 << t);
            tc_fence_after();
            if (elect_one()) {
                if (need) {
                    // S of this step goes into the buffer whose P the last but one P.V has read: the pipe keeps that order
                    const uint64_t kd = plus(k_desc, st * 2 * C::TILE), qd = plus(q_desc, ((items - 1) & 1) * 2 * C::QTILE);
                    const uint32_t b = done_s & 1;
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)
                        umma_f16((2 * t + b) * TN, plus(qd, (x >> 2) * QHALF + (x & 3) * 32), plus(kd, (x >> 2) * HALF + (x & 3) * 32), idesc_s, x > 0);
                    umma_commit(&bars->s_full[t][b]);
                } else {
                    mbar_arrive(&bars->empty[st]);
                }
            }
            __syncwarp();
            if (due < C::STAGES) issue_pv();          // of the step before: its softmax ran while this S was made
            if (need) {
                ++done_s;
                due = st;
                due_adds = begun;
                begun = true;
            }
            if (++st == C::STAGES) { st = 0; par ^= 1; }
        }
    } else if (warp == SOFTMAX_WARPS + 2) {
        // ------------------------------------------------------------------------------------------------ loads
        uint32_t items = 0, steps = 0;                // items begun, steps published
        uint32_t st = 0, par = 1;                     // the next stage, and the parity of its last release (the first pass: none)
        const int q_bytes = D / 64 * p.tpt * p.gb * 128;
        // publish a step and take the stage for its tiles
        auto publish = [&](const Item &w, int id, int flags, int x) {
            const uint32_t e = steps % STEPS;
            bool go = steps < STEPS || wait_for(bars, &bars->step_empty[e], (steps / STEPS - 1) & 1, 0x613);
            go = go && (steps < C::STAGES || wait_for(bars, &bars->empty[st], par, 0x612));
            ok = __all_sync(0xffffffffu, go);
            if (ok && elect_one()) {
                Step &d = bars->steps[e];
                *reinterpret_cast<int4 *>(&d) = make_int4(flags, x, w.first, w.count);
                *reinterpret_cast<int4 *>(&d.cached) = make_int4(w.cached, w.a, w.kvh, w.hb);
                *reinterpret_cast<int4 *>(&d.head) = make_int4(w.head, w.ring2(), id, 0);
                mbar_arrive(&bars->step_full[e]);
            }
            __syncwarp();
            ++steps;
        };
        auto queries = [&](const Item &w, int t) {
            const uint32_t b = items & 1;
            ok = __all_sync(0xffffffffu, (items < 2 || wait_for(bars, &bars->q_free[t][b], ((items >> 1) - 1) & 1, 0x611)) && !aborted());
            if (ok && elect_one()) {
                if (w.has(t)) {
                    mbar_arrive_expect_tx(&bars->q_full[t][b], q_bytes);
#pragma unroll
                    for (int h = 0; h < D / 64; ++h)
                        tma_3d(sm + (2 * b + t) * C::QTILE + h * QHALF, &map_q, h * 64, w.kvh * p.w.g + w.hb * p.gb, w.first + w.from(t), &bars->q_full[t][b]);
                } else {
                    mbar_arrive(&bars->q_full[t][b]);
                }
            }
            __syncwarp();
        };
        Found from;
        // an item that nobody works on any more: the merge finds nothing to do
        auto drop = [&](int i) {
            if (p.parts > 1 && i >= 0 && i % p.parts == 0) part_item<D>(p)[i / p.parts] = make_int4(0, 0, 0, 0);
        };
        if (!ok && lane == 0) drop(blockIdx.x);
        uint32_t asked = 0, answered = 0;             // requests for work, answers read
        uint32_t cleaned = 0;                         // tiles with dead rows
        for (int id = blockIdx.x; ok && id >= 0;) {
            const Item w = find_item(p, id, from);
            if (w.seq < 0) {                          // (the grid is an upper bound: behind the last item nothing follows)
                if (elect_one()) drop(id);
                __syncwarp();
                break;
            }
#ifdef SH_DEBUG_BOUNDS
            if (id == g_window_selftest) {
                *(volatile int *)&bars->abort_flag = 0x6ff;
                ok = false;
                break;
            }
#endif
            bool first = true, ask = __shfl_sync(0xffffffffu, *(volatile int *)&bars->no_more, 0) == 0;
            const int last_tile = w.ctiles + w.jhi;   // (the tile of the last row itself: always needed)
            int flags = 0, x = 0;                     // a step that waits to learn whether it is the last
            // 32 tiles at a time, a lane each; what lies between the sinks and the window is passed over
            auto skip = [&](int base) {
                return base >= w.ctiles && base - w.ctiles < w.jlo && w.cached + (base - w.ctiles) * TN >= w.sinks ? w.ctiles + w.jlo : base;
            };
            // (what lies outside the tensors is zeros already)
            auto dead = [&](int i) {
                return i < w.ctiles ? i * TN + TN > w.live && w.live < w.sinks + w.window : (i - w.ctiles) * TN + TN > w.count && w.first + w.count < p.w.tokens;
            };
            auto needed = [&](int i) { return i <= last_tile && (w.need(0, i) || w.need(1, i)); };
            int seen = 0, parts = 1;                  // needed tiles so far, CTAs that share them
            if (p.parts > 1) {
                int all = 0;
                for (int base = 0; base <= last_tile; base += 32) {
                    base = skip(base);
                    all += __popc(__ballot_sync(0xffffffffu, needed(base + lane)));
                }
                parts = min(parts_of(all, p.share), p.parts);
                if (w.part == 0 && elect_one()) part_item<D>(p)[id / p.parts] = make_int4(parts, w.first + w.a, w.count - w.a, 0);
                __syncwarp();
            }
            const int shared = parts > 1 ? STEP_PART : 0;
            auto step = [&]() {
                flags |= (first ? STEP_FIRST : 0) | shared;
                publish(w, id, flags, x);
                if (ok && first) queries(w, 0);
                if (ok && elect_one()) {
                    unsigned char *dst = kv + st * 2 * C::TILE;
                    uint64_t *full = flags & STEP_DEAD ? &bars->landed : &bars->full[st];
                    mbar_arrive_expect_tx(full, 2 * C::TILE);
                    if (flags & STEP_CACHE) {
                        tma_5d(dst, &map_kc, x, w.kvh, w.seq, full);
                        tma_5d(dst + C::TILE, &map_vc, x, w.kvh, w.seq, full);
                    } else {
                        tma_4d(dst, &map_k, w.kvh, w.first + x, full);
                        tma_4d(dst + C::TILE, &map_v, w.kvh, w.first + x, full);
                    }
                }
                __syncwarp();
                if (ok && first) queries(w, 1);
                if (ok && (flags & STEP_DEAD)) {
                    ok = __all_sync(0xffffffffu, wait_for(bars, &bars->landed, cleaned++ & 1, 0x615));
                    const int keep = (flags & STEP_CACHE ? w.live : w.count) - x;
                    unsigned char *v = kv + st * 2 * C::TILE + C::TILE;
                    for (int i = keep * 8 + lane; i < TN * 8 && ok; i += 32)
#pragma unroll
                        for (int h = 0; h < D / 64; ++h) *reinterpret_cast<uint4 *>(v + h * HALF + i * 16) = make_uint4(0, 0, 0, 0);
                    fence_async_shared();
                    __syncwarp();
                    if (ok && elect_one()) mbar_arrive(&bars->full[st]);
                    __syncwarp();
                }
                if (++st == C::STAGES) { st = 0; par ^= 1; }
                items += first;
                first = false;
                flags = 0;
            };
            for (int base = w.part < parts ? 0 : last_tile + 1; base <= last_tile && ok; base += 32) {
                base = skip(base);
                const int i = base + lane;
                const bool need0 = i <= last_tile && w.need(0, i), need1 = i <= last_tile && w.need(1, i);
                const int mine = (need0 ? STEP_NEED0 : 0) | (need1 ? STEP_NEED1 : 0) | (need0 && w.whole(0, i) ? STEP_WHOLE0 : 0) |
                                 (need1 && w.whole(1, i) ? STEP_WHOLE1 : 0) | (i < w.ctiles ? STEP_CACHE : 0) | (dead(i) ? STEP_DEAD : 0);
                unsigned todo = __ballot_sync(0xffffffffu, need0 || need1);
                if (parts > 1) {                      // every parts-th of them is this CTA's
                    const unsigned all = todo;
                    todo = __ballot_sync(0xffffffffu, (need0 || need1) && (seen + __popc(all & ((1u << lane) - 1u))) % parts == w.part);
                    seen += __popc(all);
                }
                while (todo && ok) {
                    // the next item is asked for a few steps before the end of this one: soon enough to cover the answer's latency, late
                    // enough for the next item to go to whoever is done first
                    if (ask && base + 32 > last_tile && __popc(todo) <= 3) {
                        if (elect_one()) claim_request(&bars->claim, &bars->claimed);
                        __syncwarp();
                        ask = false;
                        ++asked;
                    }
                    if (flags) step();
                    if (!ok) break;
                    const int bit = __ffs(todo) - 1;
                    todo &= todo - 1;
                    flags = __shfl_sync(0xffffffffu, mine, bit);
                    x = (base + bit - (flags & STEP_CACHE ? 0 : w.ctiles)) * TN;
                }
            }
            if (!ok) break;
            if (w.part < parts) {                     // (a part has 4 tiles at least)
                flags |= STEP_LAST;
                step();
            }
            if (ok && ask) {
                if (elect_one()) claim_request(&bars->claim, &bars->claimed);
                __syncwarp();
                ++asked;
            }
            if (!ok || asked == answered) break;
            ok = __all_sync(0xffffffffu, wait_for(bars, &bars->claimed, answered & 1, 0x614));
            if (!ok) break;
            ++answered;
            id = __shfl_sync(0xffffffffu, claim_read(&bars->claim), 0);
            fence_async_shared();                     // (read before the next answer is written)
            __syncwarp();
        }
        const uint32_t loads = steps;                 // (a step that was published without a load only makes the drain below wait in vain)
        if (ok) {                                     // the end: a step without a load
            Item none;
            none.first = none.count = none.cached = none.a = none.kvh = none.hb = none.head = 0;
            none.wrapped = false;
            publish(none, 0, STEP_END, 0);
            if (ok && elect_one()) mbar_arrive(&bars->full[st]);
            __syncwarp();
        }
        // let the copies (and the answer) requested last land before the CTA goes away (a phase that is past reads as complete; with the last step
        // published, its stage's earlier load has been waited for)
        if (lane == 0) {
            if (answered != asked && wait_for(bars, &bars->claimed, answered & 1, 0)) drop(claim_read(&bars->claim));
            if (items > 0)
                for (int t = 0; t < 2; ++t) wait_for(bars, &bars->q_full[t][(items - 1) & 1], ((items - 1) >> 1) & 1, 0);
            for (uint32_t k = 0; k < C::STAGES - (ok ? 1u : 0u) && k < loads; ++k)
                wait_for(bars, &bars->full[(loads - 1 - k) % C::STAGES], ((loads - 1 - k) / C::STAGES) & 1, 0);
        }
        __syncwarp();
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX));
        // ------------------------------------------------------------------------------------------------ softmax
        const int t = warp >> 2, row = tid & 127;
        const uint32_t lanes = tbase + ((uint32_t)((warp & 3) * 32) << 16), s_addr = lanes + 2 * t * TN, o_addr = lanes + C::O_COL + t * D;
        const int tok = row / p.gb, hrow = row % p.gb;
        const float c = p.w.scale_log2e;
        uint32_t cnt = 0, steps = 0, items = 0;
        int id = 0;                                   // present item
        int qi = 0, h = 0, kvh = 0, row0 = 0;
        bool live = false, begun = false;
        float m = -CUDART_INF_F, l = 0.f;
        // The entry of the next step is read while the present one is worked on.
        int4 e0, e1, e2;
        // The place of an item's queries is given back when its outputs, which were laid out there, have been read: a step later.
        int owed = -1;                                // (of the lane that stores) the place still to be given back
        auto give_back = [&]() {
            if (owed < 0) return;
            bulk_wait_read_all();
            mbar_arrive(&bars->q_free[t][owed]);
            owed = -1;
        };
        auto fetch = [&]() {
            give_back();
            const uint32_t e = steps % STEPS;
            ok = wait_for(bars, &bars->step_full[e], (steps / STEPS) & 1, 0x624) && ok;
            ++steps;
            const Step &d = bars->steps[e];
            e0 = *reinterpret_cast<const int4 *>(&d);
            e1 = *reinterpret_cast<const int4 *>(&d.cached);
            e2 = *reinterpret_cast<const int4 *>(&d.head);
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->step_empty[e]);
        };
        fetch();
        while (true) {
            if (__any_sync(0xffffffffu, !ok)) break;
            const int flags = e0.x;
            if (flags & STEP_END) break;
            if (flags & STEP_FIRST) {
                id = e2.z;
                qi = e1.y + t * p.tpt + tok;
                h = e1.w * p.gb + hrow;
                kvh = e1.z;
                row0 = e0.z;
                live = tok < p.tpt && qi < e0.w && h < p.w.g;
                begun = false;
                m = -CUDART_INF_F;
                l = 0.f;
                ok = !aborted();
                ++items;
            }
            if (flags & (STEP_NEED0 << t)) {
                const bool whole = flags & (STEP_WHOLE0 << t);
                Runs runs;
                if (!whole) runs = visible_runs(flags & STEP_CACHE, e0.y, e1.x, e2.x, e2.y, p.w.sinks, p.w.window, qi);
                const uint32_t buf = cnt & 1;
                ok = wait_for(bars, &bars->s_full[t][buf], (cnt >> 1) & 1, 0x621) && ok;
                if (__any_sync(0xffffffffu, !ok)) break;
                tc_fence_after();
                uint32_t s[TN];
#pragma unroll
                for (int x = 0; x < TN / 32; ++x) tmem_ld32_nowait(s_addr + buf * TN + x * 32, s + x * 32);
                tmem_wait_ld(s);
                if (!whole) {
#pragma unroll
                    for (int b = 0; b < TN / 32; ++b) {
                        const uint32_t bits = run_bits(runs, b * 32);
#pragma unroll
                        for (int k = 0; k < 32; ++k) s[b * 32 + k] = (bits >> k) & 1u ? s[b * 32 + k] : 0xff800000u;      // -inf
                    }
                }
                float mx[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) mx[k] = fmaxf(__uint_as_float(s[k]), __uint_as_float(s[k + 8]));
#pragma unroll
                for (int k = 16; k < TN; k += 16)
#pragma unroll
                    for (int c8 = 0; c8 < 8; ++c8) mx[c8] = max3(mx[c8], __uint_as_float(s[k + c8]), __uint_as_float(s[k + 8 + c8]));
                const float mn = fmaxf(fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7]))), m);
                // renew the subtracted maximum when it has grown enough (or is the first): rescale O and l.
                const bool grown = live && (mn - m) * c > RENEW;      // (-inf - -inf: no)
                if (__any_sync(0xffffffffu, grown)) {
                    const float f = m == -CUDART_INF_F ? 0.f : ex2_approx((m - mn) * c);
                    if (begun) {
                        ok = wait_for(bars, &bars->pv_done[t][buf ^ 1], ((cnt - 1) >> 1) & 1, 0x622);      // the product before this one is in O
                        if (__any_sync(0xffffffffu, !ok)) break;
                        tc_fence_after();
#pragma unroll
                        for (int b = 0; b < D / 16; ++b) {      // (16 columns at a time: S is held meanwhile)
                            uint32_t o[16];
                            tmem_ld16_nowait(o_addr + b * 16, o);
                            tmem_wait_ld(o);
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            tmem_st16(o_addr + b * 16, o);
                        }
                    }
                    l *= f;
                    m = mn;
                }
                fetch();
                const float base = m == -CUDART_INF_F ? 0.f : m * c - Fmt<T>::LIFT;
                const uint64_t c2 = f2(c, c), b2 = f2(-base, -base);
                uint64_t sum0 = f2(0.f, 0.f), sum1 = sum0;
#pragma unroll
                for (int b = 0; b < TN / 32; ++b) {
                    uint32_t pk[16];
#pragma unroll
                    for (int k = 0; k < 32; k += 2) {
                        float x, y;
                        un2(fma2(f2(__uint_as_float(s[b * 32 + k]), __uint_as_float(s[b * 32 + k + 1])), c2, b2), x, y);
                        x = ex2_approx(x);
                        y = ex2_approx(y);
                        if (k & 2) sum1 = add2(sum1, f2(x, y)); else sum0 = add2(sum0, f2(x, y));
                        pk[k / 2] = shelem::Vec<T>::pack2(x, y);
                    }
                    tmem_st16(s_addr + buf * TN + b * 16, pk);
                }
                float x, y;
                un2(add2(sum0, sum1), x, y);
                l += x + y;
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();                  // (one arrival per warp: those of 32 lanes on one barrier are taken one by one)
                if (lane == 0) mbar_arrive(&bars->p_ready[t][buf]);
                ++cnt;
                begun = true;
            } else {
                fetch();
            }
            if (!(flags & STEP_LAST)) continue;
            const uint32_t qbuf = (items - 1) & 1;
            if (flags & STEP_PART) {
                if (begun) {
                    ok = wait_for(bars, &bars->pv_done[t][(cnt - 1) & 1], ((cnt - 1) >> 1) & 1, 0x625);
                    if (__any_sync(0xffffffffu, !ok)) break;
                    tc_fence_after();
                    float4 *to = part_o<D>(p, id, t) + row;
#pragma unroll
                    for (int b = 0; b < D / 32; ++b) {
                        uint32_t o[32];
                        tmem_ld32_nowait(o_addr + b * 32, o);
                        tmem_wait_ld(o);
                        if (live) {
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                to[(b * 8 + k) * TM] = make_float4(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1]), __uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3]));
                        }
                    }
                    tc_fence_before();
                }
                if (live) part_sum<D>(p, id, t)[row] = make_float2(m == -CUDART_INF_F ? m : m * c - Fmt<T>::LIFT, begun ? l : -1.f);
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->q_free[t][qbuf]);
                continue;
            }
            if (!begun) {                             // (a query tile without rows)
                if (lane == 0) mbar_arrive(&bars->q_free[t][qbuf]);
                continue;
            }
            ok = wait_for(bars, &bars->pv_done[t][(cnt - 1) & 1], ((cnt - 1) >> 1) & 1, 0x623);
            if (__any_sync(0xffffffffu, !ok)) break;
            tc_fence_after();
            const float inv = 1.f / l;
            // the rows of O, one per thread, are laid out in the place of the item's queries (every S of the item is over), like a
            // query tile, and a warp's 32 rows leave from there as one copy if they are whole tokens; rows next to somebody else's,
            // or that have to be done again, go by the threads, in whole lines
            unsigned char *place = sm + (2 * qbuf + t) * C::QTILE;
            const long long at = (long long)(row0 + qi) * p.w.out.ts + (long long)(kvh * p.w.g + h) * p.w.out.hs;
            const uint64_t inv2 = f2(inv, inv);
            uint64_t zero = 0;                        // stays zero unless a value is not finite
#pragma unroll
            for (int b = 0; b < D / 32; ++b) {
                uint32_t o[32];
                tmem_ld32_nowait(o_addr + b * 32, o);
                tmem_wait_ld(o);
#pragma unroll
                for (int k = 0; k < 32; k += 8) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const uint64_t y = mul2(f2(__uint_as_float(o[k + e]), __uint_as_float(o[k + e + 1])), inv2);
                        zero = fma2(y, 0, zero);
                        un2(y, x[e], x[e + 1]);
                    }
                    *reinterpret_cast<uint4 *>(place + b / 2 * QHALF + row * 128 + (((b % 2 * 4 + k / 8) ^ (row & 7)) << 4)) = shelem::Vec<T>::pack(x);
                }
            }
            float z0, z1;
            un2(zero, z0, z1);
            const bool odd = !(z0 + z1 == 0.f);
            tc_fence_before();      // O has been read before the arrivals that let the next item overwrite it
            fence_async_shared();   // (for the copy, and for the queries that arrive here next)
            __syncwarp();
            if (!__any_sync(0xffffffffu, !live || odd) && p.copy_out) {
                if (lane == 0) {
#pragma unroll
                    for (int x = 0; x < D / 64; ++x) tma_store_3d(&map_o, place + x * QHALF + (warp & 3) * 32 * 128, x * 64, kvh * p.w.g + h, row0 + qi);
                    bulk_commit();
                    owed = qbuf;
                }
                continue;
            }
            constexpr int CH = D / 8;
#pragma unroll 4
            for (int r = 0; r < 32; r += 32 / CH) {
                const int mine = r + lane / CH, c = lane % CH, of = (warp & 3) * 32 + mine;
                const long long to = __shfl_sync(0xffffffffu, at, mine);
                const uint4 x = *reinterpret_cast<const uint4 *>(place + c / 8 * QHALF + of * 128 + ((c % 8 ^ (of & 7)) << 4));
                if (__shfl_sync(0xffffffffu, (int)live, mine)) *reinterpret_cast<uint4 *>(p.w.out.p + to + c * 16) = x;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->q_free[t][qbuf]);
            const unsigned again = __ballot_sync(0xffffffffu, live && odd);
            if (again) note_again(bars, warp, id, again);
        }
        __syncwarp();
        do_again<T, D>(p, bars->again[warp], bars->again_count[warp], t, warp & 3);
        bulk_wait_all();            // outputs on their way from shared memory
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && bars->abort_flag) atomicCAS(&g_window_error, 0, bars->abort_flag);
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(512) : "memory");
    }
}

// Merge the parts of each item: 8 rows of a query tile a CTA, 4 columns a thread (so a part's floats come as runs of 128 bytes).
template <typename T, int D>
__global__ void __launch_bounds__(2 * D) sh_window_prefill_merge_kernel(const __grid_constant__ UmmaParams p) {
    constexpr int ROWS = 8;
    __shared__ float2 sums[MAX_SHARE][ROWS];
    __shared__ int odd[ROWS];
    const int tid = threadIdx.x, r = tid % ROWS, c4 = tid / ROWS;
    const int t = blockIdx.x / (TM / ROWS) % 2, row0 = blockIdx.x % (TM / ROWS) * ROWS, row = row0 + r;
    const int item = blockIdx.x / (2 * TM / ROWS), id = item * p.parts;      // id: of its first part
    const int in = item % (p.w.hk * p.hblocks), kvh = in / p.hblocks, hb = in % p.hblocks;
    const int tok = t * p.tpt + row / p.gb, h = hb * p.gb + row % p.gb;      // of the item
    sh_pdl_wait();
    const int4 w = part_item<D>(p)[item];
    const int parts = min(w.x, p.parts);
    // (the entry of an item that was lost with a CTA that gave up a wait holds anything)
    if (w.y < 0 || w.y > p.w.tokens || w.z > p.w.tokens - w.y) return;
    if (parts <= 1 || row0 / p.gb >= p.tpt || t * p.tpt + row0 / p.gb >= w.z) return;
    const bool live = row / p.gb < p.tpt && tok < w.z && h < p.w.g;
    for (int i = c4; i < parts; i += D / 4) sums[i][r] = live ? part_sum<D>(p, id + i, t)[row] : make_float2(0.f, -1.f);
    if (tid < ROWS) odd[tid] = 0;
    __syncthreads();
    float M = -CUDART_INF_F;
    for (int i = 0; i < parts; ++i) M = fmaxf(M, sums[i][r].x);
    float L = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    const float4 *at = part_o<D>(p, id, t) + c4 * TM + row;
#pragma unroll 8
    for (int i = 0; i < parts; ++i) {
        const float2 s = sums[i][r];
        if (s.y < 0.f) continue;                     // (nothing was written)
        const float4 x = at[(long long)i * 2 * (D / 4) * TM];
        const float f = s.x == -CUDART_INF_F ? 0.f : ex2_approx(s.x - M);      // (0 times NaN stays one)
        L += s.y * f;
        o.x = fmaf(x.x, f, o.x); o.y = fmaf(x.y, f, o.y); o.z = fmaf(x.z, f, o.z); o.w = fmaf(x.w, f, o.w);
    }
    const float inv = 1.f / L;                       // (as where there is nothing to merge)
    o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
    if (live && !(isfinite(o.x) && isfinite(o.y) && isfinite(o.z) && isfinite(o.w))) odd[r] = 1;
    __syncthreads();
    if (live && !odd[r]) {
        T *dst = reinterpret_cast<T *>(p.w.out.p + (long long)(w.y + tok) * p.w.out.ts + (kvh * p.w.g + h) * p.w.out.hs) + c4 * 4;
        *reinterpret_cast<uint2 *>(dst) = make_uint2(shelem::Vec<T>::pack2(o.x, o.y), shelem::Vec<T>::pack2(o.z, o.w));
    }
    for (int i = tid >> 5; i < ROWS; i += D / 16) {  // rows next to values that are not finite
        if (!odd[i]) continue;
        Found from;
        slow_row<T, D>(p, id, find_item(p, id, from).from(t) + (row0 + i) / p.gb, kvh * p.w.g + hb * p.gb + (row0 + i) % p.gb);
    }
}

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor-map encoder, looked up through the runtime (the library does not link against the driver).
EncodeTiled encoder() {
    static EncodeTiled fn = [] {
        void *sym = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
            sym = nullptr;
        return reinterpret_cast<EncodeTiled>(sym);
    }();
    return fn;
}

// Map over rows of 16-bit elements, 64 of them innermost: dims and byte strides of what lies outside of them, the box's extents
// there; 128-byte swizzle, zeros outside the tensor.
bool make_map(CUtensorMap *m, const void *base, int outer, const uint64_t *dim, const uint64_t *stride, const uint32_t *extent, uint64_t inner = 64) {
    EncodeTiled enc = encoder();
    if (!enc) return false;
    cuuint64_t gdim[5] = {inner}, gstride[4];
    cuuint32_t box[5] = {64u}, one[5] = {1u, 1u, 1u, 1u, 1u};
    for (int i = 0; i < outer; ++i) {
        gdim[i + 1] = dim[i];
        gstride[i] = stride[i];
        box[i + 1] = extent[i];
    }
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, outer + 1, const_cast<void *>(base), gdim, gstride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// [half][token][head][64]: all halves of TN tokens of one head are one copy
bool keys_map(CUtensorMap *m, const WinRows &r, int heads, int tokens, uint64_t halves) {
    const uint64_t dim[3] = {(uint64_t)heads, (uint64_t)tokens, halves}, st[3] = {(uint64_t)r.hs, (uint64_t)r.ts, 128};
    const uint32_t box[3] = {1, TN, (uint32_t)halves};
    return make_map(m, r.p, 3, dim, st, box);
}

// The most items a call can have: c tokens of a sequence make (c - 1) / span + 1.
long long most_items(int tokens, int sequences, int hk, int g) {
    const int gb = g < TM ? g : TM;
    const long long n = std::min(sequences, tokens);
    return ((tokens - n) / (2 * (TM / gb)) + n) * hk * ((g + gb - 1) / gb);
}
// The device's CTAs per item, and the most parts of an item: how many keys there are is known on the device only, but the rows of an
// item see no more than the window and the sinks hold, and without a cache no more than the call's tokens.
void share_out(long long items, int tokens, int window, int sinks, int g, bool with_cache, int sms, int &share, int &parts) {
    const int gb = g < TM ? g : TM;
    const long long sees = ((long long)window + sinks + 2 * (TM / gb)) / TN + 3, own = ((long long)tokens + TN - 1) / TN;
    share = (int)(std::min(sms, MAX_SHARE) / items);
    parts = parts_of(with_cache ? sees : std::min(sees, own), share);
}

template <typename T, int D>
cudaError_t launch(const WindowParams &w, cudaStream_t s) {
    UmmaParams p;
    p.w = w;
    p.gb = w.g < TM ? w.g : TM;
    p.tpt = TM / p.gb;
    p.hblocks = (w.g + p.gb - 1) / p.gb;
    CUtensorMap mq, mk, mv, mkc, mvc, mo;
    const uint64_t qdim[2] = {(uint64_t)w.hq, (uint64_t)w.tokens}, qst[2] = {(uint64_t)w.q.hs, (uint64_t)w.q.ts};
    const uint32_t qbox[2] = {(uint32_t)p.gb, (uint32_t)p.tpt};
    p.copy_out = 32 % p.gb == 0;
    const uint64_t ost[2] = {(uint64_t)w.out.hs, (uint64_t)w.out.ts};
    const uint32_t obox[2] = {(uint32_t)p.gb, p.copy_out ? 32u / p.gb : 1u};
    if (!make_map(&mq, w.q.p, 2, qdim, qst, qbox, D) || !make_map(&mo, w.out.p, 2, qdim, ost, obox, D) || !keys_map(&mk, w.k, w.hk, w.tokens, D / 64) || !keys_map(&mv, w.v, w.hk, w.tokens, D / 64))
        return cudaErrorNotSupported;
    mkc = mk; mvc = mv;
    if (w.kc) {
        const uint64_t dim[4] = {(uint64_t)w.sinks + w.window, (uint64_t)w.hk, (uint64_t)w.sequences, D / 64};
        const uint64_t st[4] = {(uint64_t)w.cls, (uint64_t)w.chs, (uint64_t)w.css, 128};
        const uint32_t box[4] = {TN, 1, 1, D / 64};
        if (!make_map(&mkc, w.kc, 4, dim, st, box) || !make_map(&mvc, w.vc, 4, dim, st, box)) return cudaErrorNotSupported;
    }
    auto kern = sh_window_prefill_umma_kernel<T, D>;
    static ShKernelSetup setup;
    int sms = 0;
    const cudaError_t e = sh_setup_kernel(setup, kern, Cfg<D>::SMEM, &sms);
    if (e != cudaSuccess) return e;
    const long long items = most_items(w.tokens, w.sequences, w.hk, w.g);
    share_out(items, w.tokens, w.window, w.sinks, w.g, w.kc != nullptr, sms, p.share, p.parts);
    if (!w.part) p.parts = 1;
    if (items > 0x7fffffffll) return cudaErrorInvalidValue;
    kern<<<(unsigned)(items * p.parts), NTH, Cfg<D>::SMEM, s>>>(p, mq, mk, mv, mkc, mvc, mo);
    if (p.parts == 1) return cudaGetLastError();
    const cudaError_t e2 = cudaGetLastError();
    if (e2 != cudaSuccess) return e2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(items * (2 * TM / 8)));
    cfg.blockDim = dim3(2 * D);
    cfg.stream = s;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sh_window_prefill_merge_kernel<T, D>, p);
}

}  // namespace

cudaError_t sh_launch_window_prefill_umma(const WindowParams &p, int dtype, int D, cudaStream_t s) {
    if (dtype == SH_F16) return D == 128 ? launch<__half, 128>(p, s) : launch<__half, 64>(p, s);
    return D == 128 ? launch<__nv_bfloat16, 128>(p, s) : launch<__nv_bfloat16, 64>(p, s);
}

size_t sh_window_prefill_scratch(int tokens, int sequences, int hk, int g, int window, int sinks, bool with_cache, int dtype, int D) {
    if (dtype == SH_F32 || tokens < 1 || sequences < 1) return 0;
    int share, parts;
    share_out(most_items(tokens, sequences, hk, g), tokens, window, sinks, g, with_cache, MAX_SHARE, share, parts);
    return parts > 1 ? sizeof(float) * MAX_SHARE * (2 * TM * (size_t)(D + 2) + 4) : 0;
}

#ifdef SH_DEBUG_BOUNDS
// Self-test of the give-up path of the waits (bounds-checked build only): the next launches' CTA that takes work item `item` gives up;
// -1: none.
extern "C" int sh_window_selftest(int item) {
    return cudaMemcpyToSymbol(g_window_selftest, &item, sizeof(int)) == cudaSuccess ? SH_OK : SH_ECUDA;
}
#endif

cudaError_t sh_window_error_take(int *code, cudaStream_t s) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(code, g_window_error, sizeof(int), 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess || *code == 0) return e;
    static const int zero = 0;
    e = cudaMemcpyToSymbolAsync(g_window_error, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, s);
    return e == cudaSuccess ? cudaStreamSynchronize(s) : e;
}
