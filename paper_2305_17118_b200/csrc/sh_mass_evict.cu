// sh_mass_evict: of every (sequence, key head) keep the `recent` newest rows and those with the largest mass, `keep` in all.
//
// Rows are ordered by one 32-bit key: the newest come first, then masses from large to small (fp32 as an unsigned number of the same
// order; NaN before everything else), among equal keys the lower slot.  The keep-th largest key is searched for, then a pass over the slots in
// order gives every row its place.  In place a survivor from behind slot keep - 1 moves into the hole of a row that goes, the lowest hole
// taking the lowest of them, so no more rows move than go; into another cache survivors are written in the order of their slots.
//
// Short caches (1024 slots): a small CTA takes a unit, its keys in registers, and settles one bit of the key after the other by counting.
// Long ones: a cluster takes a unit and settles 11 bits at a time by histograms in shared memory, added up through
// distributed shared memory.  Rows are moved by a second launch, with a CTA for 64 moves; many short units move their own.
// Bound by HBM where many rows move: 9216 units of 474 rows, 64 moved each in rows of 256 bytes: 123 us, 4.9 TB/s (a warp a unit: 146, its
// select alone is four thousand instructions; moves by a second launch: 150 and more).  64 units of up to 32768 rows brought down to 2048 in
// another cache: selection 27 us, moves 22 us (6.3 TB/s); a selection of 8 bits a pass, whose remote loads came one after the other, took 47.
#include <cooperative_groups.h>

#include <algorithm>

#include "sh_mass.h"

namespace cg = cooperative_groups;

namespace {

constexpr unsigned NEWEST = 0xffffffffu, NOT_A_NUMBER = 0xfffffffeu;

// Never 0: that stands for no row at all.
__device__ __forceinline__ unsigned order_of(float x) {
    if (x != x) return NOT_A_NUMBER;
    const unsigned b = __float_as_uint(x + 0.f);      // (-0 counts as 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned key_of(const EvictParams &p, const float *mass, const int32_t *positions, int j, int newest) {
    if (p.recent > 0 && (long long)positions[j] > (long long)newest - p.recent) return NEWEST;
    return order_of(mass[j]);
}

// The rows of a unit (16-byte pieces) and their records, from slot m.y to slot m.x; `lanes` threads take them in turn, AHEAD of a thread's in flight.
template <int AHEAD, typename Moves>
__device__ __forceinline__ void move_rows(const EvictParams &p, int seq, int kvh, int count, int lane, int lanes, Moves move) {
    const long long from = seq * p.ss + kvh * p.hs, to = seq * p.oss + kvh * p.ohs;
    const int shift = p.row_bytes == 512 ? 5 : (p.row_bytes == 256 ? 4 : 3);      // log2 of a row's pieces
    for (int i0 = lane; i0 < count << shift; i0 += lanes * AHEAD) {
        uint4 a[AHEAD], b[AHEAD];
        long long at[AHEAD];
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) {
            const int i = i0 + x * lanes;
            if (i >= count << shift) break;
            const int2 m = move(i >> shift);
            const int c = (i & ((1 << shift) - 1)) * 16;
            a[x] = *reinterpret_cast<const uint4 *>(p.k + from + m.y * p.ls + c);
            b[x] = *reinterpret_cast<const uint4 *>(p.v + from + m.y * p.ls + c);
            at[x] = to + m.x * p.ols + c;
        }
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) {
            if (i0 + x * lanes >= count << shift) break;
            *reinterpret_cast<uint4 *>(p.ko + at[x]) = a[x];
            *reinterpret_cast<uint4 *>(p.vo + at[x]) = b[x];
        }
    }
    for (int i = lane; i < count; i += lanes) {
        const int2 m = move(i);
        const long long x = seq * p.rec.ss + kvh * p.rec.hs + m.y, y = seq * p.out.ss + kvh * p.out.hs + m.x;
        p.out.mass[y] = p.rec.mass[x];
        p.out.positions[y] = p.rec.positions[x];
    }
}

// ---------------------------------------------------------------------------------------------------------------- short caches
constexpr int SHORT = 1024, SHORT_WARPS = 4, SHORT_NT = 32 * SHORT_WARPS;

template <int EACH>      // keys of a thread; a warp has EACH * 32 neighbouring slots
__global__ void __launch_bounds__(SHORT_NT) sh_mass_select_short_kernel(const __grid_constant__ EvictParams p, bool fused) {
    __shared__ unsigned short holes[EACH * SHORT_NT], movers[EACH * SHORT_NT];
    __shared__ int counts[2][SHORT_WARPS], ties_of[SHORT_WARPS], holes_of[SHORT_WARPS], movers_of[SHORT_WARPS];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int unit = blockIdx.x, kvh = unit % p.heads, seq = unit / p.heads;
    if (!fused) sh_pdl_launch_dependents();
    const int n = min(p.lengths[seq], p.slots);
    int count = 0;                             // rows that move
    const bool whole = n <= p.keep;            // nothing goes
    if (whole) {
        count = p.in_place ? 0 : max(n, 0);
    } else {
        const float *mass = p.rec.mass + seq * p.rec.ss + kvh * p.rec.hs;
        const int32_t *positions = p.rec.positions + seq * p.rec.ss + kvh * p.rec.hs;
        const int j0 = warp * EACH * 32 + lane;
        unsigned key[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) key[i] = j0 + i * 32 < n ? order_of(mass[j0 + i * 32]) : 0u;
        if (p.recent > 0) {
            int pos[EACH], newest = 0x80000000;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                pos[i] = j0 + i * 32 < n ? positions[j0 + i * 32] : 0x80000000;
                newest = max(newest, pos[i]);
            }
            newest = __reduce_max_sync(0xffffffffu, newest);
            if (lane == 0) ties_of[warp] = newest;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < SHORT_WARPS; ++w) newest = max(newest, ties_of[w]);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (j0 + i * 32 < n && (long long)pos[i] > (long long)newest - p.recent) key[i] = NEWEST;
        }
        // the keep-th largest key, from its top bit down; done early where a bit parts the rows as wanted
        unsigned at = 0;
        bool parted = false;
        int turn = 0;
        auto sum = [&](int c) {                // over the CTA
            c = __reduce_add_sync(0xffffffffu, c);
            if (lane == 0) counts[turn][warp] = c;
            __syncthreads();
            c = 0;
#pragma unroll
            for (int w = 0; w < SHORT_WARPS; ++w) c += counts[turn][w];
            turn ^= 1;
            return c;
        };
#pragma unroll 1
        for (unsigned bit = 0x80000000u; bit && !parted; bit >>= 1) {
            int c = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) c += key[i] >= (at | bit);
            c = sum(c);
            if (c >= p.keep) at |= bit;
            parted = c == p.keep;
        }
        int c = 0, t = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            c += key[i] > at;
            t += __popc(__ballot_sync(0xffffffffu, key[i] == at));
        }
        if (lane == 0) ties_of[warp] = t;
        const int want = p.keep - sum(c);      // rows equal to that key that stay, the lowest slots
        int ties = 0;
#pragma unroll
        for (int w = 0; w < SHORT_WARPS; ++w)
            if (w < warp) ties += ties_of[w];
        unsigned hole_bits[EACH], mover_bits[EACH];
        int h = 0, m = 0;
        const unsigned below = (1u << lane) - 1u;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int j = j0 + i * 32;
            const bool tie = key[i] == at;
            const unsigned tie_bits = __ballot_sync(0xffffffffu, tie);
            const bool stays = key[i] > at || (tie && ties + __popc(tie_bits & below) < want);
            ties += __popc(tie_bits);
            hole_bits[i] = __ballot_sync(0xffffffffu, p.in_place && j < p.keep && !stays);      // (keep < n)
            mover_bits[i] = __ballot_sync(0xffffffffu, stays && (!p.in_place || j >= p.keep));
            h += __popc(hole_bits[i]);
            m += __popc(mover_bits[i]);
        }
        if (lane == 0) { holes_of[warp] = h; movers_of[warp] = m; }
        __syncthreads();
        h = m = 0;
#pragma unroll
        for (int w = 0; w < SHORT_WARPS; ++w) {
            if (w < warp) { h += holes_of[w]; m += movers_of[w]; }
            count += movers_of[w];             // (as many holes in place: keep rows stay)
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (hole_bits[i] >> lane & 1u) holes[h + __popc(hole_bits[i] & below)] = (unsigned short)(j0 + i * 32);
            if (mover_bits[i] >> lane & 1u) movers[m + __popc(mover_bits[i] & below)] = (unsigned short)(j0 + i * 32);
            h += __popc(hole_bits[i]);
            m += __popc(mover_bits[i]);
        }
        __syncthreads();
    }
    if (fused && kvh == 0 && tid == 0 && p.left != p.lengths) p.left[seq] = min(p.lengths[seq], p.keep);
    auto move = [&](int i) { return whole ? make_int2(i, i) : make_int2(p.in_place ? holes[i] : i, movers[i]); };
    if (fused) {
        move_rows<2>(p, seq, kvh, count, tid, SHORT_NT, move);
        return;
    }
    if (tid == 0) p.count[unit] = count;
    for (int i = tid; i < count; i += SHORT_NT) p.moves[(long long)unit * p.most + i] = move(i);
}

// ---------------------------------------------------------------------------------------------------------------- long caches
constexpr int NT = 1024, WARPS = NT / 32, MAX_CLUSTER = 8, PASSES = 3, BINS = 2 * NT;
constexpr int MAX_KEYS = 45 * 1024;      // keys that a CTA keeps in shared memory; beyond it the records are read again in every pass

// What all CTAs of the cluster have at the place of `mine`, added up.  (The loads are in flight together: one remote latency, not S.)
template <typename T, typename F>
__device__ __forceinline__ void over_cluster(cg::cluster_group &cluster, T *mine, int S, F f) {
    T x[MAX_CLUSTER];
#pragma unroll
    for (int r = 0; r < MAX_CLUSTER; ++r)
        if (r < S) x[r] = *cluster.map_shared_rank(mine, r);
#pragma unroll
    for (int r = 0; r < MAX_CLUSTER; ++r)
        if (r < S) f(r, x[r]);
}
// Sum of x over the threads before this one.
__device__ __forceinline__ int before_me(int x, int *sums) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int upto = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
    }
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    const int all = sums[lane];
    const int ahead = __reduce_add_sync(0xffffffffu, lane < warp ? all : 0);
    return ahead + upto - x;
}

__global__ void __launch_bounds__(NT) sh_mass_select_kernel(const __grid_constant__ EvictParams p, int cached_keys) {
    extern __shared__ unsigned keys[];
    __shared__ int hist[PASSES][BINS], sums[PASSES][WARPS], found[PASSES][2], newest_sh;
    __shared__ int4 tally[WARPS];              // of a warp's rows: above the key below and from slot keep on, equal to it likewise
    __shared__ int4 bases[WARPS * MAX_CLUSTER];
    cg::cluster_group cluster = cg::this_cluster();
    const int S = cluster.num_blocks(), rank = cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int unit = blockIdx.x / S, kvh = unit % p.heads, seq = unit / p.heads;
    sh_pdl_launch_dependents();
    const int n = min(p.lengths[seq], p.slots);
    int2 *moves = p.moves + (long long)unit * p.most;
    if (n <= p.keep) {                         // nothing goes (the same for the whole cluster)
        if (tid == 0 && rank == 0) p.count[unit] = p.in_place ? 0 : max(n, 0);
        if (!p.in_place)
            for (int i = rank * NT + tid; i < n; i += S * NT) moves[i] = make_int2(i, i);
        return;
    }
    const float *mass = p.rec.mass + seq * p.rec.ss + kvh * p.rec.hs;
    const int32_t *positions = p.rec.positions + seq * p.rec.ss + kvh * p.rec.hs;
    const int each = (n + S * NT - 1) / (S * NT) * 32, per = each * WARPS;      // rows of a warp, of a CTA, in the order of their slots
    const int lo = min(n, rank * per), hi = min(n, lo + per);
    for (int i = tid; i < PASSES * BINS; i += NT) (&hist[0][0])[i] = 0;
    int newest = 0x80000000;
    if (p.recent > 0) {
#pragma unroll 8
        for (int j = lo + tid; j < hi; j += NT) {
            newest = max(newest, positions[j]);
            if (cached_keys) keys[j - lo] = order_of(mass[j]);
        }
        newest = __reduce_max_sync(0xffffffffu, newest);
        if (lane == 0) sums[0][warp] = newest;
        __syncthreads();
        if (warp == 0) {
            newest = __reduce_max_sync(0xffffffffu, sums[0][lane]);
            if (lane == 0) newest_sh = newest;
        }
        cluster.sync();
        over_cluster(cluster, &newest_sh, S, [&](int, int x) { newest = max(newest, x); });
    }
    if (cached_keys) {
#pragma unroll 8
        for (int j = lo + tid; j < hi; j += NT) {
            if (p.recent == 0) keys[j - lo] = order_of(mass[j]);
            else if ((long long)positions[j] > (long long)newest - p.recent) keys[j - lo] = NEWEST;
        }
    }
    auto key = [&](int j) { return cached_keys ? keys[j - lo] : key_of(p, mass, positions, j, newest); };
    __syncthreads();
    // the keep-th largest key: 11, 11 and 10 bits a pass.  (The first has sign, exponent and two bits more: with fewer, most rows would meet
    // in a few places of the histogram.)
    unsigned prefix = 0, known = 0;
    int want = p.keep;                         // place of the key among those that share the known bits
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        constexpr int SHIFT[PASSES] = {21, 10, 0};
        const int shift = SHIFT[pass];
        const unsigned mask = pass == 2 ? BINS / 2 - 1 : BINS - 1;
#pragma unroll 4
        for (int j = lo + tid; j < hi; j += NT) {
            const unsigned k = key(j);
            if ((k & known) == prefix) atomicAdd(&hist[pass][k >> shift & mask], 1);
        }
        cluster.sync();
        int mine[2] = {};                      // from the largest digit down, a thread has two
#pragma unroll
        for (int i = 0; i < 2; ++i) over_cluster(cluster, &hist[pass][BINS - 1 - (2 * tid + i)], S, [&](int, int x) { mine[i] += x; });
        const int before = before_me(mine[0] + mine[1], sums[pass]);
        if (before < want && want <= before + mine[0] + mine[1]) {
            const int second = want > before + mine[0];
            found[pass][0] = BINS - 1 - (2 * tid + second);
            found[pass][1] = want - before - (second ? mine[0] : 0);
        }
        __syncthreads();
        prefix |= (unsigned)found[pass][0] << shift;
        known |= mask << shift;
        want = found[pass][1];
    }
    // Rows above that key stay, and the first `want` of those equal to it.  Every warp counts its own ...
    const int from = lo + warp * each, to = min(hi, from + each);
    int4 t = make_int4(0, 0, 0, 0);
    for (int j = from + lane; j < to; j += 32) {
        const unsigned k = key(j);
        if (j < p.keep) { t.x += k > prefix; t.z += k == prefix; }
        else { t.y += k > prefix; t.w += k == prefix; }
    }
    t = make_int4(__reduce_add_sync(0xffffffffu, t.x), __reduce_add_sync(0xffffffffu, t.y), __reduce_add_sync(0xffffffffu, t.z), __reduce_add_sync(0xffffffffu, t.w));
    if (lane == 0) tally[warp] = t;
    cluster.sync();
    // ... and a warp of each CTA works out what comes before whom: rows equal to the key, holes, rows that move.  Warp w of CTA r is the
    // (32 r + w)-th; lane l takes the l-th of each CTA, one CTA after the other.
    if (warp == 0) {
        int ties = 0, h = 0, m = 0;            // before the CTA
        over_cluster(cluster, &tally[lane], S, [&](int r, int4 x) {
            auto scan = [&](int v) {
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, v, o);
                    if (lane >= o) v += y;
                }
                return v;
            };
            const int w = r * WARPS + lane, both = x.z + x.w, t1 = scan(both), mine = ties + t1 - both;
            const int low = min(max(want - mine, 0), x.z), high = min(max(want - mine - x.z, 0), x.w);      // equal ones that stay
            const int hh = min(max(p.keep - w * each, 0), each) - (x.x + low);      // (slots below keep that this warp has; keep < n)
            const int mm = x.y + high + (p.in_place ? 0 : x.x + low);
            const int h1 = scan(hh), m1 = scan(mm);
            bases[w] = make_int4(mine, h + h1 - hh, m + m1 - mm, 0);
            ties += __shfl_sync(0xffffffffu, t1, 31);
            h += __shfl_sync(0xffffffffu, h1, 31);
            m += __shfl_sync(0xffffffffu, m1, 31);
        });
        if (lane == 0 && rank == 0) p.count[unit] = m;
    }
    __syncthreads();
    int ties = bases[rank * WARPS + warp].x, h = bases[rank * WARPS + warp].y, m = bases[rank * WARPS + warp].z;
    const unsigned below = (1u << lane) - 1u;
    for (int j0 = from; j0 < to; j0 += 32) {
        const int j = j0 + lane;
        const unsigned k = j < to ? key(j) : 0u;
        const bool tie = j < to && k == prefix;
        const unsigned tie_bits = __ballot_sync(0xffffffffu, tie);
        const bool stays = j < to && (k > prefix || (tie && ties + __popc(tie_bits & below) < want));
        const bool hole = p.in_place && j < to && j < p.keep && !stays, mover = stays && (!p.in_place || j >= p.keep);
        const unsigned hole_bits = __ballot_sync(0xffffffffu, hole), mover_bits = __ballot_sync(0xffffffffu, mover);
        if (hole) moves[h + __popc(hole_bits & below)].x = j;
        if (mover) {
            const int at = m + __popc(mover_bits & below);
            moves[at].y = j;
            if (!p.in_place) moves[at].x = at;
        }
        ties += __popc(tie_bits);
        h += __popc(hole_bits);
        m += __popc(mover_bits);
    }
    cluster.sync();                            // nobody's shared memory goes away while it is read
}

// ---------------------------------------------------------------------------------------------------------------- moves
constexpr int MOVE_NT = 256, ROWS = 64;
__global__ void __launch_bounds__(MOVE_NT) sh_mass_move_kernel(const __grid_constant__ EvictParams p, int blocks) {
    const int unit = blockIdx.x / blocks, block = blockIdx.x % blocks, kvh = unit % p.heads, seq = unit / p.heads;
    sh_pdl_wait();                             // (the moves)
    if (block == 0 && kvh == 0 && threadIdx.x == 0) p.left[seq] = min(p.lengths[seq], p.keep);      // (may be the place of the lengths: nobody else reads them any more)
    const int count = min(p.count[unit] - block * ROWS, ROWS);
    const int2 *moves = p.moves + (long long)unit * p.most + block * ROWS;
    move_rows<1>(p, seq, kvh, count, threadIdx.x, MOVE_NT, [&](int i) { return moves[i]; });
}
// Where the units have moved their rows themselves, and the new lengths take the place of the old ones.
__global__ void sh_mass_left_kernel(const __grid_constant__ EvictParams p) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    sh_pdl_wait();
    if (i < p.sequences) p.left[i] = min(p.lengths[i], p.keep);
}

template <typename... A>
cudaError_t launch(void (*kern)(A...), unsigned ctas, int threads, size_t smem, cudaLaunchAttributeID id, int cluster, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr = {};
    attr.id = id;
    if (id == cudaLaunchAttributeClusterDimension) { attr.val.clusterDim.x = cluster; attr.val.clusterDim.y = attr.val.clusterDim.z = 1; }
    else attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}
constexpr auto AFTER = cudaLaunchAttributeProgrammaticStreamSerialization;

template <int EACH>
cudaError_t select_short(const EvictParams &p, int units, bool fused, cudaStream_t s) {
    sh_mass_select_short_kernel<EACH><<<units, SHORT_NT, 0, s>>>(p, fused);
    return cudaGetLastError();
}

}  // namespace

size_t sh_mass_evict_scratch(long long units, int most) { return (size_t)units * ((size_t)most * sizeof(int2) + sizeof(int)) + 16; }

cudaError_t sh_launch_mass_evict(const EvictParams &p, cudaStream_t s) {
    const long long units = (long long)p.sequences * p.heads, blocks = std::max((p.most + ROWS - 1) / ROWS, 1);
    if (units * blocks > 0x7fffffffll || units * MAX_CLUSTER > 0x7fffffffll) return cudaErrorInvalidValue;
    int dev = 0, sms = 0;
    cudaError_t e = sh_device_sms(&dev, &sms);
    if (e != cudaSuccess) return e;
    if (p.slots <= SHORT) {
        // units move their own rows when there are several for each place of the device, or few to move
        const bool fused = units >= 8ll * sms || p.most <= 16;
        const int n = (int)units;
        e = p.slots <= SHORT_NT ? select_short<1>(p, n, fused, s) : p.slots <= 2 * SHORT_NT ? select_short<2>(p, n, fused, s) : p.slots <= 4 * SHORT_NT ? select_short<4>(p, n, fused, s) : select_short<8>(p, n, fused, s);
        if (e != cudaSuccess) return e;
        if (fused) return p.left != p.lengths ? cudaSuccess : launch(sh_mass_left_kernel, (unsigned)((p.sequences + 127) / 128), 128, 0, AFTER, 0, s, p);
    } else {
        int S = 1;
        while (S < MAX_CLUSTER && units * S * 2 <= sms && p.slots >= 2 * S * NT) S *= 2;
        const int most = (p.slots + S * NT - 1) / (S * NT) * NT;      // rows of a CTA
        const bool cached = most <= MAX_KEYS;
        static ShKernelSetup setup;
        e = sh_setup_kernel(setup, sh_mass_select_kernel, MAX_KEYS * sizeof(unsigned), &sms);
        if (e != cudaSuccess) return e;
        e = launch(sh_mass_select_kernel, (unsigned)(units * S), NT, cached ? most * sizeof(unsigned) : 0, cudaLaunchAttributeClusterDimension, S, s, p, (int)cached);
        if (e != cudaSuccess) return e;
    }
    return launch(sh_mass_move_kernel, (unsigned)(units * blocks), MOVE_NT, 0, AFTER, 0, s, p, (int)blocks);
}
