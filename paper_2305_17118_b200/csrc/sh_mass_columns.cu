// Prompts, 16-bit types: mass[j] += sum over the chunk's tokens and the group's heads of exp(s_j - log sum of the row), on the 5th-generation
// tensor cores.
//
// The scores are made transposed, S^T = K.Q^T with 128 keys as M and 128 rows (token x head of the group, heads innermost) as N: a thread
// then owns a key, one lane of tensor memory, and its sum never leaves a register.  Nothing of size keys x rows leaves the SM.  The chunk is
// in the cache already, so all keys come from there.
//
//   warps 0-15       sums: thread = key; the four groups of four warps take the row tiles in turn.  S from tensor memory, exponentials, addition
//   warp 16          issues the MMAs (both operands in shared memory, K-major)
//   warp 17          finds the items (128 keys of a key head), publishes them in a ring and requests the tiles (TMA, 128-byte swizzle)
//
// Four buffers of S fill tensor memory.  The rows' logs are read from global memory two tiles ahead by the group that needs them, a thread
// a row, and handed around in shared memory.  A CTA takes the next item when it has requested the last tile of the one before (the first
// key blocks of a sequence are seen by all its rows, the last by few: long ones come first).  Where an item would be long against what an SM has to do in all, its
// row tiles are dealt out to several items, whose sums a second launch adds up in their order: whoever takes them, the result is the same.
//
// Bound by the exponentials: a tile has 16384, at 16 a cycle on an SM, while its MMAs take 512 cycles (D = 128).  8192 tokens, 32 query
// heads over 8 of 128, fp16: 0.35 ms with the unit 81 % busy (the attention itself: 0.54 ms); 16384 tokens 1.28 ms.  With two groups of warps
// instead of four the unit was idle 40 % of the time (1.75 ms).  A quarter of the exponentials by a polynomial on the FMA pipe brought 5 % here
// and 2 % of the whole prompt.
#include <math_constants.h>

#include <algorithm>
#include <cmath>

#include "sh_mass.h"
#include "sh_pairs.cuh"
#include "sh_tiles.cuh"
#include "sh_window.cuh"

namespace {

using namespace shasync;
using namespace shpair;
using namespace shtile;
using namespace shumma;
using namespace shwin;

constexpr int KEYS = 128, ROWS = 128;              // of a tile of S
constexpr int HALF = 128 * 128;                    // bytes of a tile's rows x 64 elements
constexpr int GROUPS = 4, SUM_WARPS = 4 * GROUPS, NTH = 32 * (SUM_WARPS + 2);
constexpr int STAGES = 4, BUFS = 4, RING = 4;      // row tiles in flight, buffers of S, items in flight
constexpr float LOG2E = 1.4426950408889634f;

__device__ int g_mass_error;                       // code of the first bounded wait that gave up

struct __align__(16) ColItem {
    int seq, first, count, cached;                 // seq < 0: the end
    int slot0, kvh, tok0, tiles;                   // first key, key head, first token that sees it, row tiles
    int part, pad[3];
};
struct ColBars {
    uint64_t k_full[2], k_free[2], q_full[STAGES], q_free[STAGES], s_full[BUFS], s_free[BUFS], item_full[RING], item_free[RING];
    uint64_t logs_full[GROUPS], part_full;              // a group's logs, an item's sums are there
    ColItem items[RING];
    float logs[GROUPS][2][ROWS];                   // [group][its tile mod 2]: minus the rows' logs, base 2
    float part[2][GROUPS][KEYS];                        // [item mod 2][group]: sums
    uint32_t tmem;
    int abort_flag;
};
template <int D> struct ColCfg {
    static constexpr int TILE = D / 64 * HALF, OFF_Q = 2 * TILE, OFF_BAR = OFF_Q + STAGES * TILE, SMEM = OFF_BAR + (int)sizeof(ColBars);
    static_assert(SMEM <= 232448, "");
};

struct ColParams {
    WindowParams w;
    int tpt, gb, hblocks;                          // tokens and heads of a row tile, head blocks per key head
    int parts;                                     // items that share the row tiles of 128 keys; more than one: they leave their sums in
};                                                 // w.part, [part][sequence][key head][slot]

constexpr unsigned long long LIMIT_NS = 8000000000ull;
__device__ __forceinline__ bool wait_for(ColBars *bars, uint64_t *bar, uint32_t parity, int code) {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < LIMIT_NS)
        if (mbar_try_wait(bar, parity)) return true;
    *(volatile int *)&bars->abort_flag = code;
    return false;
}
__device__ __forceinline__ ColItem find_item(const ColParams &p, long long id) {
    ColItem r = {};
    const int lane = threadIdx.x & 31;
    const long long tile = id / p.parts / p.w.hk;
    r.seq = -1;
    long long before = 0;
    for (int base = 0; base < p.w.sequences; base += 32) {
        int first = 0, count = 0, cached = 0;
        if (base + lane < p.w.sequences) sequence_rows<ATTEND_MASS>(p.w, base + lane, first, count, cached);
        const int mine = count > 0 ? (cached + count + KEYS - 1) / KEYS : 0;
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, before + upto > tile);
        if (hit) {
            const int l = __ffs(hit) - 1;
            r.seq = base + l;
            r.first = __shfl_sync(0xffffffffu, first, l);
            r.count = __shfl_sync(0xffffffffu, count, l);
            r.cached = __shfl_sync(0xffffffffu, cached, l);
            r.slot0 = (int)(tile - before - __shfl_sync(0xffffffffu, upto - mine, l)) * KEYS;
            r.kvh = (int)(id / p.parts % p.w.hk);
            r.part = (int)(id % p.parts);
            r.tok0 = max(0, r.slot0 - r.cached);
            const int all = (r.count - r.tok0 + p.tpt - 1) / p.tpt * p.hblocks;
            r.tiles = (all - r.part + p.parts - 1) / p.parts;
            return r;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    return r;
}

// Row tile n of an item: its first token (in the chunk), its first head, and how many of its rows there are.
__device__ __forceinline__ void tile_of(const ColParams &p, const ColItem &w, int n, int &tok, int &h, int &rows) {
    n = n * p.parts + w.part;
    if (p.hblocks > 1) {                           // a tile is one token
        tok = w.tok0 + n / p.hblocks;
        h = n % p.hblocks * p.gb;
        rows = min(p.gb, p.w.g - h);
    } else {
        tok = w.tok0 + n * p.tpt;
        h = 0;
        rows = min(p.tpt, w.count - tok) * p.gb;
    }
}

template <int FMT, int D>
__global__ void __launch_bounds__(NTH, 1)
sh_mass_columns_umma_kernel(const __grid_constant__ ColParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k) {
    using C = ColCfg<D>;
    extern __shared__ __align__(1024) unsigned char sm[];
    ColBars *bars = reinterpret_cast<ColBars *>(sm + C::OFF_BAR);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto aborted = [&]() { return *(volatile int *)&bars->abort_flag != 0; };
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) { mbar_init(&bars->k_full[i], 1); mbar_init(&bars->k_free[i], 1); }
        for (int i = 0; i < STAGES; ++i) { mbar_init(&bars->q_full[i], 1); mbar_init(&bars->q_free[i], 1); }
        for (int i = 0; i < BUFS; ++i) { mbar_init(&bars->s_full[i], 1); mbar_init(&bars->s_free[i], 4); }
        for (int i = 0; i < RING; ++i) { mbar_init(&bars->item_full[i], 1); mbar_init(&bars->item_free[i], SUM_WARPS + 1); }
        for (int i = 0; i < GROUPS; ++i) mbar_init(&bars->logs_full[i], 4);
        mbar_init(&bars->part_full, SUM_WARPS);
        bars->abort_flag = (smem_u32(sm) & 1023u) != 0 ? 0x630 : 0;      // the swizzled tiles need the alignment the declaration asks for
        fence_barrier_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    sh_pdl_launch_dependents();
    sh_pdl_wait();                                 // (the rows' logs, the chunk in the cache)
    const uint32_t tbase = bars->tmem;
    if (tbase != 0) *(volatile int *)&bars->abort_flag = 0x631;          // (all 512 columns are this CTA's)
    bool ok = __all_sync(0xffffffffu, !aborted() && tbase == 0);

    if (warp == SUM_WARPS) {
        // ------------------------------------------------------------------------------------------------ MMAs
        constexpr uint32_t idesc = instr_desc(FMT, 0, KEYS, ROWS);
        uint32_t it = 0, tiles = 0, loads = 0;                           // items, row tiles, items with tiles so far
        while (ok) {
            ok = __all_sync(0xffffffffu, wait_for(bars, &bars->item_full[it % RING], it / RING & 1, 0x632));
            if (!ok) break;
            const int seq = __shfl_sync(0xffffffffu, *(volatile int *)&bars->items[it % RING].seq, 0);
            const int count = __shfl_sync(0xffffffffu, *(volatile int *)&bars->items[it % RING].tiles, 0);
            __syncwarp();
            if (elect_one()) mbar_arrive(&bars->item_free[it % RING]);
            __syncwarp();
            ++it;
            if (seq < 0) break;
            if (count == 0) continue;
            const uint32_t kb = loads & 1;
            ok = __all_sync(0xffffffffu, wait_for(bars, &bars->k_full[kb], loads >> 1 & 1, 0x633));
            const uint64_t kd = desc_sw128(smem_u32(sm) + kb * C::TILE, 16, 1024), qd0 = desc_sw128(smem_u32(sm) + C::OFF_Q, 16, 1024);
            for (int n = 0; n < count && ok; ++n, ++tiles) {
                const uint32_t st = tiles % STAGES, b = tiles % BUFS;
                ok = __all_sync(0xffffffffu, wait_for(bars, &bars->q_full[st], tiles / STAGES & 1, 0x634) &&
                                                 (tiles < BUFS || wait_for(bars, &bars->s_free[b], (tiles / BUFS - 1) & 1, 0x635)));
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t qd = qd0 + (st * C::TILE >> 4);
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) umma_f16(b * ROWS, kd + (((x >> 2) * HALF + (x & 3) * 32) >> 4), qd + (((x >> 2) * HALF + (x & 3) * 32) >> 4), idesc, x > 0);
                    umma_commit(&bars->s_full[b]);
                    umma_commit(&bars->q_free[st]);
                    if (n == count - 1) umma_commit(&bars->k_free[kb]);
                }
                __syncwarp();
            }
            ++loads;
        }
    } else if (warp == SUM_WARPS + 1) {
        // ------------------------------------------------------------------------------------------------ loads
        const int q_bytes = D / 64 * p.tpt * p.gb * 128;
        uint32_t it = 0, tiles = 0, loads = 0;
        bool more = true;
        while (ok && more) {
            int id = 0;
            if (lane == 0) id = atomicAdd(p.w.taken, 1);
            const ColItem w = find_item(p, __shfl_sync(0xffffffffu, id, 0));
            more = w.seq >= 0;
            ok = __all_sync(0xffffffffu, it < RING || wait_for(bars, &bars->item_free[it % RING], (it / RING - 1) & 1, 0x636));
            if (!ok) break;
            if (elect_one()) {
                bars->items[it % RING] = w;
                mbar_arrive(&bars->item_full[it % RING]);
            }
            __syncwarp();
            ++it;
            if (!more || w.tiles == 0) continue;
            const uint32_t kb = loads & 1;
            ok = __all_sync(0xffffffffu, loads < 2 || wait_for(bars, &bars->k_free[kb], ((loads >> 1) - 1) & 1, 0x637));
            if (!ok) break;
            if (elect_one()) {
                mbar_arrive_expect_tx(&bars->k_full[kb], C::TILE);
                tma_5d(sm + kb * C::TILE, &map_k, w.slot0, w.kvh, w.seq, &bars->k_full[kb]);
            }
            __syncwarp();
            ++loads;
            for (int n = 0; n < w.tiles; ++n, ++tiles) {
                const uint32_t st = tiles % STAGES;
                ok = __all_sync(0xffffffffu, (tiles < STAGES || wait_for(bars, &bars->q_free[st], (tiles / STAGES - 1) & 1, 0x638)) && !aborted());
                if (!ok) break;
                int tok, h, rows;
                tile_of(p, w, n, tok, h, rows);
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bars->q_full[st], q_bytes);
#pragma unroll
                    for (int x = 0; x < D / 64; ++x)
                        tma_3d(sm + C::OFF_Q + st * C::TILE + x * HALF, &map_q, x * 64, w.kvh * p.w.g + h, w.first + tok, &bars->q_full[st]);
                }
                __syncwarp();
            }
        }
        // let the copies requested last land before the CTA goes away (a phase that is past reads as complete)
        if (lane == 0) {
            for (uint32_t k = 0; k < 2 && k < loads; ++k) wait_for(bars, &bars->k_full[(loads - 1 - k) & 1], (loads - 1 - k) >> 1 & 1, 0x639);
            for (uint32_t k = 0; k < STAGES && k < tiles; ++k) wait_for(bars, &bars->q_full[(tiles - 1 - k) % STAGES], (tiles - 1 - k) / STAGES & 1, 0x63a);
        }
        __syncwarp();
    } else if (warp < SUM_WARPS) {
        // ------------------------------------------------------------------------------------------------ sums
        const int grp = warp >> 2, key = tid & 127, key_tok = key / p.gb, key_head = key % p.gb;      // (and of the row whose log it fetches)
        const uint32_t s_addr = tbase + ((uint32_t)((warp & 3) * 32) << 16);
        const float c = p.w.scale_log2e;
        const uint64_t c2 = f2(c, c);
        uint32_t it = 0, tiles = 0;                                      // items, row tiles of the CTA before the present item
        while (true) {
            ok = wait_for(bars, &bars->item_full[it % RING], it / RING & 1, 0x63b) && ok;
            if (__any_sync(0xffffffffu, !ok)) break;
            const ColItem w = bars->items[it % RING];
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->item_free[it % RING]);
            const uint32_t turn = it & 1;
            ++it;
            if (w.seq < 0) break;
            const int slot = w.slot0 + key, n_keys = w.cached + w.count;
            // minus the log of this thread's row of the item's n-th tile
            auto log_of = [&](int n) {
                int tok, h, rows;
                if (n >= w.tiles) return 0.f;
                tile_of(p, w, n, tok, h, rows);
                if (key >= rows) return 0.f;
                return -LOG2E * p.w.lse[(long long)(w.first + tok + key_tok) * p.w.hq + w.kvh * p.w.g + h + key_head];
            };
            uint64_t sum0 = 0, sum1 = 0;
            int n = (grp - (int)(tiles % GROUPS) + GROUPS) % GROUPS;     // this group takes every fourth tile, counted over the CTA
            float mine = log_of(n), next = log_of(n + GROUPS);
            for (; n < w.tiles; n += GROUPS) {
                const uint32_t t = tiles + n, b = t % BUFS;
                float *logs = bars->logs[grp][t / GROUPS & 1];
                logs[key] = mine;
                mine = next;
                next = log_of(n + 2 * GROUPS);
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->logs_full[grp]);
                int tok, h, rows;
                tile_of(p, w, n, tok, h, rows);
                const bool whole = rows == ROWS && w.slot0 + KEYS - 1 <= w.cached + tok;
                // rows that see this key: from the token at its slot on
                const int lo = p.hblocks > 1 ? (slot <= w.cached + tok ? 0 : ROWS) : max(0, slot - w.cached - tok) * p.gb;
                // (whoever has passed the wait for its logs knows that the group is done with those of the tile before, whose place comes next)
                ok = wait_for(bars, &bars->logs_full[grp], t / GROUPS & 1, 0x63d) && wait_for(bars, &bars->s_full[b], t / BUFS & 1, 0x63c) && ok;
                if (__any_sync(0xffffffffu, !ok)) break;
                tc_fence_after();
#pragma unroll
                for (int x = 0; x < ROWS / 32; ++x) {
                    uint32_t s[32];
                    tmem_ld32_nowait(s_addr + b * ROWS + x * 32, s);
                    tmem_wait_ld(s);
                    if (x == ROWS / 32 - 1) {                            // all of S is in registers
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars->s_free[b]);
                    }
                    const float4 *l4 = reinterpret_cast<const float4 *>(logs + x * 32);
                    if (whole) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float4 l = l4[k / 4];
                            float e0, e1, e2, e3;
                            un2(fma2(f2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, f2(l.x, l.y)), e0, e1);
                            un2(fma2(f2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])), c2, f2(l.z, l.w)), e2, e3);
                            sum0 = add2(sum0, f2(ex2_approx(e0), ex2_approx(e1)));
                            sum1 = add2(sum1, f2(ex2_approx(e2), ex2_approx(e3)));
                        }
                    } else {
                        const int from = lo - x * 32, to = rows - x * 32;
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float4 l = l4[k / 4];
                            float e[4] = {fmaf(__uint_as_float(s[k]), c, l.x), fmaf(__uint_as_float(s[k + 1]), c, l.y), fmaf(__uint_as_float(s[k + 2]), c, l.z),
                                          fmaf(__uint_as_float(s[k + 3]), c, l.w)};
#pragma unroll
                            for (int i = 0; i < 4; ++i) e[i] = k + i >= from && k + i < to ? ex2_approx(e[i]) : 0.f;
                            sum0 = add2(sum0, f2(e[0], e[1]));
                            sum1 = add2(sum1, f2(e[2], e[3]));
                        }
                    }
                }
            }
            if (__any_sync(0xffffffffu, !ok)) break;
            const uint32_t lead = tiles % GROUPS;                        // the group that has taken the item's first tile
            tiles += w.tiles;
            float a, b;
            un2(add2(sum0, sum1), a, b);
            bars->part[turn][grp][key] = a + b;
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->part_full);
            ok = wait_for(bars, &bars->part_full, turn, 0x63e);
            if (__any_sync(0xffffffffu, !ok)) break;
            if (grp == (int)(it % GROUPS) && slot < n_keys) {
                // in the order of the tiles, whatever the CTA has done before
                auto part = [&](uint32_t i) { return bars->part[turn][(lead + i) % GROUPS][key]; };
                const float x = (part(0) + part(1)) + (part(2) + part(3));
                if (p.parts == 1) p.w.mass[w.seq * p.w.rss + w.kvh * p.w.rhs + slot] += x;
                else p.w.part[(((long long)w.part * p.w.sequences + w.seq) * p.w.hk + w.kvh) * p.w.slots + slot] = x;
            }
        }
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && bars->abort_flag) atomicCAS(&g_mass_error, 0, bars->abort_flag);
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(512) : "memory");
    }
}

// The parts' sums, in their order.
constexpr int ADD = 256;
__global__ void __launch_bounds__(ADD) sh_mass_columns_add_kernel(const __grid_constant__ WindowParams p, int blocks, int parts) {
    const int kvh = blockIdx.x / blocks % p.hk, seq = blockIdx.x / blocks / p.hk, slot = blockIdx.x % blocks * ADD + threadIdx.x;
    int first, count, cached;
    sequence_rows<ATTEND_MASS>(p, seq, first, count, cached);
    sh_pdl_wait();
    if (count == 0 || slot >= cached + count) return;
    float x = 0.f;
    for (int i = 0; i < parts; ++i) x += p.part[(((long long)i * p.sequences + seq) * p.hk + kvh) * p.slots + slot];
    p.mass[seq * p.rss + kvh * p.rhs + slot] += x;
}

// How many items share the row tiles of a key block.  The longest sequence is taken to have twice the average's tokens: its first key blocks see
// `tiles` row tiles, an SM has about `load` in all (half of them lie behind the diagonal), and an item should be half of that.  Four tiles an
// item at least.  2048 tokens in one part 97 us, five 83, eight 86 (with the attention); 4096 tokens of one key head 173 in two, 112 in eight;
// 1 to 2048 tokens of six sequences 130 in two and three, 140 in eight.  (148: the SMs of a B200.  The size of the workspace follows from this too,
// and is asked for where there is no device to look at.)
int parts_of(int tokens, int sequences, int hk, int g, int slots) {
    const double longest = std::min((double)tokens, 2.0 * tokens / sequences), tiles = longest * g / ROWS;
    const double load = hk * std::ceil((double)tokens / KEYS) * tiles / 2 / 148;
    const double most = std::min(std::min(8.0, tiles / 4), (double)(64 << 20) / (4.0 * sequences * hk * slots));      // (64 MB of sums)
    return (int)std::max(1.0, std::min(most, std::ceil(2 * tiles / std::max(load, 1.0))));
}

template <int FMT, int D>
cudaError_t launch(const WindowParams &w, cudaStream_t s) {
    ColParams p;
    p.w = w;
    p.gb = std::min(w.g, ROWS);
    p.tpt = ROWS / p.gb;
    p.hblocks = (w.g + p.gb - 1) / p.gb;
    if (p.hblocks > 1) p.tpt = 1;
    CUtensorMap mq, mk;
    const uint64_t qdim[2] = {(uint64_t)w.hq, (uint64_t)w.tokens}, qst[2] = {(uint64_t)w.q.hs, (uint64_t)w.q.ts};
    const uint32_t qbox[2] = {(uint32_t)p.gb, (uint32_t)p.tpt};
    const uint64_t kdim[4] = {(uint64_t)w.slots, (uint64_t)w.hk, (uint64_t)w.sequences, D / 64}, kst[4] = {(uint64_t)w.cls, (uint64_t)w.chs, (uint64_t)w.css, 128};
    const uint32_t kbox[4] = {KEYS, 1, 1, D / 64};
    if (!make_map(&mq, w.q.p, 2, qdim, qst, qbox, D) || !make_map(&mk, w.kc, 4, kdim, kst, kbox)) return cudaErrorNotSupported;
    auto kern = sh_mass_columns_umma_kernel<FMT, D>;
    static ShKernelSetup setup;
    int sms = 0;
    const cudaError_t e = sh_setup_kernel(setup, kern, ColCfg<D>::SMEM, &sms);
    if (e != cudaSuccess) return e;
    p.parts = parts_of(w.tokens, w.sequences, w.hk, w.g, w.slots);
    const long long items = (long long)std::min(w.sequences, w.tokens) * ((w.slots + KEYS - 1) / KEYS) * w.hk * p.parts;      // at most
    const long long blocks = (w.slots + ADD - 1) / ADD;
    if (blocks * w.sequences * w.hk > 0x7fffffffll) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min<long long>(items, sms));
    cfg.blockDim = dim3(NTH);
    cfg.dynamicSmemBytes = ColCfg<D>::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e2 = cudaLaunchKernelEx(&cfg, kern, p, mq, mk);
    if (e2 != cudaSuccess || p.parts == 1) return e2;
    cfg.gridDim = dim3((unsigned)(blocks * w.sequences * w.hk));
    cfg.blockDim = dim3(ADD);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, sh_mass_columns_add_kernel, w, (int)blocks, p.parts);
}

}  // namespace

cudaError_t sh_launch_mass_columns_umma(const WindowParams &p, int dtype, int D, cudaStream_t s) {
    if (dtype == SH_F16) return D == 128 ? launch<0, 128>(p, s) : launch<0, 64>(p, s);
    return D == 128 ? launch<1, 128>(p, s) : launch<1, 64>(p, s);
}

cudaError_t sh_mass_error_take(int *code, cudaStream_t s) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(code, g_mass_error, sizeof(int), 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess || *code == 0) return e;
    static const int zero = 0;
    e = cudaMemcpyToSymbolAsync(g_mass_error, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, s);
    return e == cudaSuccess ? cudaStreamSynchronize(s) : e;
}

size_t sh_mass_columns_scratch(int tokens, int sequences, int hk, int g, int slots) {
    const int parts = parts_of(tokens, sequences, hk, g, slots);
    return parts > 1 ? sizeof(float) * parts * (size_t)sequences * hk * slots : 0;
}
