// sh_mass_evict: of every (sequence, key head) keep the `recent` newest rows and those with the largest mass, `keep` in all.
//
// Rows are ordered by one 32-bit key: the newest come first, then masses from large to small (fp32 as an unsigned number of the same
// order; NaN before everything else), among equal keys the lower slot.  The keep-th largest key is found by radix selection, 8 bits a pass
// from the top; a last pass over the slots in order gives every row its place.  In place a survivor from behind slot keep - 1 moves into
// the hole of a row that goes, the lowest hole taking the lowest of them, so no more rows move than go; into another cache survivors are
// written in the order of their slots.  A second launch moves the rows.  Bound by HBM: the records are read once, moved rows read and written.
#include <algorithm>

#include "sh_mass.h"

namespace {

constexpr int NT = 512, WARPS = NT / 32;
constexpr unsigned NEWEST = 0xffffffffu, NOT_A_NUMBER = 0xfffffffeu;
constexpr int MAX_KEYS = 48 * 1024;      // keys that are kept in shared memory; longer caches read the records again in every pass

__device__ __forceinline__ unsigned order_of(float x) {
    if (x != x) return NOT_A_NUMBER;
    const unsigned b = __float_as_uint(x + 0.f);      // (-0 counts as 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Sums over the CTA, for every thread; `sh` holds a word per warp.
__device__ __forceinline__ int block_max(int x, int *sh) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    x = sh[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i) x = max(x, sh[i]);
    return x;
}

__global__ void __launch_bounds__(NT) sh_mass_select_kernel(const __grid_constant__ EvictParams p, int cached_keys) {
    extern __shared__ unsigned keys[];
    __shared__ int hist[256], warp_sums[3][WARPS], found[3];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int unit = blockIdx.x, kvh = unit % p.heads, seq = unit / p.heads;
    sh_pdl_launch_dependents();
    const int n = min(p.lengths[seq], p.slots);
    if (n <= p.keep) {                         // nothing goes
        if (tid == 0) p.count[unit] = p.in_place ? 0 : max(n, 0);
        if (!p.in_place)
            for (int i = tid; i < n; i += NT) p.moves[(long long)unit * p.most + i] = make_int2(i, i);
        return;
    }
    const float *mass = p.rec.mass + seq * p.rec.ss + kvh * p.rec.hs;
    const int32_t *positions = p.rec.positions + seq * p.rec.ss + kvh * p.rec.hs;
    int newest = 0x80000000;
    if (p.recent > 0) {
        for (int j = tid; j < n; j += NT) newest = max(newest, positions[j]);
        newest = block_max(newest, warp_sums[0]);
    }
    auto read_key = [&](int j) {
        if (p.recent > 0 && (long long)positions[j] > (long long)newest - p.recent) return NEWEST;
        return order_of(mass[j]);
    };
    if (cached_keys)
        for (int j = tid; j < n; j += NT) keys[j] = read_key(j);
    auto key = [&](int j) { return cached_keys ? keys[j] : read_key(j); };
    // the keep-th largest key: its top bits pass by pass
    unsigned prefix = 0, known = 0;
    int want = p.keep;                         // place of the key among those that share the known bits
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += NT) hist[i] = 0;
        __syncthreads();
        for (int j0 = warp * 32; j0 < n; j0 += NT) {
            const int j = j0 + lane;
            const unsigned k = j < n ? key(j) : 0u;
            const bool in = j < n && (k & known) == prefix;
            const unsigned who = __ballot_sync(0xffffffffu, in);
            if (in) {                          // one count for all lanes of the warp with the same digit
                const unsigned same = __match_any_sync(who, (k >> shift) & 255u);
                if (lane == __ffs(same) - 1) atomicAdd(&hist[(k >> shift) & 255u], __popc(same));
            }
        }
        __syncthreads();
        if (warp == 0) {                       // from the largest digit down: lane l has 8 of them
            int mine[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) { mine[i] = hist[255 - (lane * 8 + i)]; sum += mine[i]; }
            int upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += x;
            }
            int before = upto - sum;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (before < want && want <= before + mine[i]) { found[0] = 255 - (lane * 8 + i); found[1] = want - before; }
                before += mine[i];
            }
        }
        __syncthreads();
        prefix |= (unsigned)found[0] << shift;
        known |= 255u << shift;
        want = found[1];
    }
    // Slots in order: rows above the threshold stay, and the first `want` of those equal to it.
    int equal = 0, holes = 0, movers = 0;      // so far; movers: rows that stay (another cache), or those of them behind the last kept slot
    int2 *moves = p.moves + (long long)unit * p.most;
    for (int j0 = 0; j0 < n; j0 += NT) {
        const int j = j0 + tid;
        const unsigned k = j < n ? key(j) : 0u;
        const bool tie = j < n && k == prefix;
        const unsigned ties = __ballot_sync(0xffffffffu, tie);
        __syncthreads();
        if (lane == 0) warp_sums[0][warp] = __popc(ties);
        __syncthreads();
        int before = equal, all = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) before += warp_sums[0][w];
            all += warp_sums[0][w];
        }
        equal += all;
        const bool stays = j < n && (k > prefix || (tie && before + __popc(ties & ((1u << lane) - 1u)) < want));
        const bool hole = p.in_place && j < p.keep && !stays, mover = stays && (!p.in_place || j >= p.keep);
        const unsigned hole_bits = __ballot_sync(0xffffffffu, hole), mover_bits = __ballot_sync(0xffffffffu, mover);
        if (lane == 0) { warp_sums[1][warp] = __popc(hole_bits); warp_sums[2][warp] = __popc(mover_bits); }
        __syncthreads();
        int h = holes, m = movers;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) { h += warp_sums[1][w]; m += warp_sums[2][w]; }
            holes += warp_sums[1][w];
            movers += warp_sums[2][w];
        }
        const unsigned below = (1u << lane) - 1u;
        if (hole) moves[h + __popc(hole_bits & below)].x = j;
        if (mover) {
            const int at = m + __popc(mover_bits & below);
            moves[at].y = j;
            if (!p.in_place) moves[at].x = at;
        }
    }
    if (tid == 0) p.count[unit] = movers;      // (as many holes as movers: keep rows stay)
}

// Lanes of 16 bytes move the rows: MOVE_WARPS * 32 threads take ROWS moves of a unit.
constexpr int MOVE_NT = 256, ROWS = 64;
__global__ void __launch_bounds__(MOVE_NT) sh_mass_move_kernel(const __grid_constant__ EvictParams p, int blocks) {
    const int unit = blockIdx.x / blocks, block = blockIdx.x % blocks, kvh = unit % p.heads, seq = unit / p.heads;
    const int pieces = p.row_bytes / 16, tid = threadIdx.x;
    sh_pdl_wait();                             // (the moves)
    if (block == 0 && kvh == 0 && tid == 0) p.left[seq] = min(p.lengths[seq], p.keep);      // (may be the place of the lengths: nobody reads them any more)
    const int count = min(p.count[unit] - block * ROWS, ROWS);
    const int2 *moves = p.moves + (long long)unit * p.most + block * ROWS;
    const long long from = seq * p.ss + kvh * p.hs, to = seq * p.oss + kvh * p.ohs;
    for (int i = tid; i < count * pieces; i += MOVE_NT) {
        const int2 m = moves[i / pieces];
        const int c = i % pieces * 16;
        const uint4 a = *reinterpret_cast<const uint4 *>(p.k + from + m.y * p.ls + c), b = *reinterpret_cast<const uint4 *>(p.v + from + m.y * p.ls + c);
        *reinterpret_cast<uint4 *>(p.ko + to + m.x * p.ols + c) = a;
        *reinterpret_cast<uint4 *>(p.vo + to + m.x * p.ols + c) = b;
    }
    for (int i = tid; i < count; i += MOVE_NT) {
        const int2 m = moves[i];
        const long long x = seq * p.rec.ss + kvh * p.rec.hs + m.y, y = seq * p.out.ss + kvh * p.out.hs + m.x;
        p.out.mass[y] = p.rec.mass[x];
        p.out.positions[y] = p.rec.positions[x];
    }
}

}  // namespace

size_t sh_mass_evict_scratch(long long units, int most) { return (size_t)units * ((size_t)most * sizeof(int2) + sizeof(int)) + 16; }

cudaError_t sh_launch_mass_evict(const EvictParams &p, cudaStream_t s) {
    const long long units = (long long)p.sequences * p.heads, blocks = (p.most + ROWS - 1) / ROWS;
    if (units * std::max(blocks, 1ll) > 0x7fffffffll) return cudaErrorInvalidValue;
    static ShKernelSetup setup;
    int sms = 0;
    cudaError_t e = sh_setup_kernel(setup, sh_mass_select_kernel, MAX_KEYS * sizeof(unsigned), &sms);
    if (e != cudaSuccess) return e;
    const bool cached = p.slots <= MAX_KEYS;
    sh_mass_select_kernel<<<(unsigned)units, NT, cached ? p.slots * sizeof(unsigned) : 0, s>>>(p, cached);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * std::max(blocks, 1ll)));
    cfg.blockDim = dim3(MOVE_NT);
    cfg.stream = s;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sh_mass_move_kernel, p, (int)std::max(blocks, 1ll));
}
