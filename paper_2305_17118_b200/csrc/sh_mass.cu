// The records of the cache with accumulated weights: mass[j] += sum over queries and heads of p_j, p_j = exp(s_j - log sum of the row).
// Weights are only known when the row's sum is, so they are worked out after the attention has left those logs: single tokens from
// the scores that it stored on its way (sh_mass_fold_kernel), prompts from queries and keys once more (the columns kernels; the one for 16-bit types is in sh_mass_columns.cu).
#include <cooperative_groups.h>
#include <math_constants.h>

#include <algorithm>

#include "sh_mass.h"
#include "sh_pairs.cuh"
#include "sh_umma.cuh"
#include "sh_window.cuh"

namespace cg = cooperative_groups;

namespace {

using shumma::ex2_approx;
using namespace shpair;
using namespace shwin;

constexpr float LOG2E = 1.4426950408889634f;

// ---------------------------------------------------------------------------------------------------------------- single tokens
constexpr int FOLD = 128, EACH = 4;      // threads, slots of a thread
// 64 sequences of up to 4090 slots, 32 query heads over 8: 8 us, 33 MB of scores out of L2.

// A thread per slot: the weights of the group's heads are added up in their order, so the result does not depend on the launch.
__global__ void __launch_bounds__(FOLD) sh_mass_fold_kernel(const __grid_constant__ WindowParams p, int blocks) {
    const int block = blockIdx.x % blocks, kvh = blockIdx.x / blocks % p.hk, seq = blockIdx.x / blocks / p.hk;
    const int t = p.lengths[seq];
    const bool part = t >= 0 && t < p.slots && block * (FOLD * EACH) <= t;
    sh_pdl_wait();                       // (what the attention before this launch has left)
    if (!part) return;
    const float *score = p.scores + ((long long)seq * p.hq + kvh * p.g) * p.score_stride, *total = p.total + (long long)seq * p.hq + kvh * p.g;
    const long long at = seq * p.rss + kvh * p.rhs;
    const int j0 = block * (FOLD * EACH) + threadIdx.x;
    float sum[EACH] = {}, old[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) old[i] = j0 + i * FOLD < t ? p.mass[at + j0 + i * FOLD] : 0.f;
    for (int h = 0; h < p.g; ++h) {
        const float l = total[h];
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (j0 + i * FOLD <= t) sum[i] += ex2_approx(score[h * p.score_stride + j0 + i * FOLD] - l);
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int j = j0 + i * FOLD;
        if (j <= t) p.mass[at + j] = old[i] + sum[i];
        if (j == t) p.held[at + j] = p.seen[seq];
    }
}

// ---------------------------------------------------------------------------------------------------------------- prompts
constexpr int CNT = 256, BK = 64, BQ = 64;      // threads, keys and rows of a tile

// Blocks of BK slots of a sequence that takes part, over all key heads; one warp, all lanes.  The first blocks of a sequence see most
// queries and come first.
struct Keys {
    int seq, first, count, cached, slot0;      // seq < 0: no such block
};
__device__ __forceinline__ Keys find_keys(const WindowParams &p, long long tile) {
    const int lane = threadIdx.x & 31;
    Keys r = {-1, 0, 0, 0, 0};
    long long before = 0;
    for (int base = 0; base < p.sequences; base += 32) {
        int first = 0, count = 0, cached = 0;
        if (base + lane < p.sequences) sequence_rows<ATTEND_MASS>(p, base + lane, first, count, cached);
        const long long mine = count > 0 ? (cached + count + BK - 1) / BK : 0;
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
            r.slot0 = (int)(tile - before - __shfl_sync(0xffffffffu, upto - mine, l)) * BK;
            return r;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    return r;
}

// fp32, on CUDA cores: a cluster of S CTAs takes 64 keys, its CTAs take the row tiles (64 rows of token x head of the group) in turn; a thread
// works on 4 keys x 4 rows and keeps its keys' sums; threads, then CTAs, are added up in a fixed order.
template <int D> struct Cols {
    static constexpr int LD = D + 4, BYTES = (BK + BQ) * LD * 4;
};
template <int D>
__global__ void __launch_bounds__(CNT) sh_mass_columns_f32_kernel(const __grid_constant__ WindowParams p) {
    constexpr int LD = Cols<D>::LD, CH = D / 4;
    extern __shared__ __align__(16) float sm[];
    float *Ks = sm, *Qs = sm + BK * LD;
    __shared__ float log_of[BQ], red[16][BK], part[BK];
    __shared__ int last_of[BQ];                // last slot that a row sees (-1: no such row)
    __shared__ Keys keys_sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int S = cluster.num_blocks(), rank = cluster.block_rank();
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    for (long long item = blockIdx.x / S;; item += gridDim.x / S) {
        const int kvh = (int)(item % p.hk);
        if (tid < 32) {
            const Keys k = find_keys(p, item / p.hk);
            if (tid == 0) keys_sh = k;
        }
        __syncthreads();
        const Keys w = keys_sh;
        if (w.seq < 0) break;                  // (the same for every CTA of the cluster)
        const int n = w.cached + w.count, rows = w.count * p.g;
        for (int i = tid; i < BK * CH; i += CNT) {
            const int r = i / CH, c = i % CH;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (w.slot0 + r < n) x = *reinterpret_cast<const uint4 *>(p.kc + w.seq * p.css + kvh * p.chs + (long long)(w.slot0 + r) * p.cls + c * 16);
            *reinterpret_cast<uint4 *>(Ks + r * LD + c * 4) = x;
        }
        float acc[4] = {};
        // a row tile's queries and logs are asked for while the tile before is worked on
        constexpr int EACH_Q = BQ * CH / CNT;
        uint4 ahead[EACH_Q];
        float log_ahead = 0.f;
        int last_ahead = -1;
        auto ask = [&](int base) {
#pragma unroll
            for (int k = 0; k < EACH_Q; ++k) {
                const int i = tid + k * CNT, row = base + i / CH;
                ahead[k] = make_uint4(0, 0, 0, 0);
                if (row < rows) ahead[k] = *reinterpret_cast<const uint4 *>(p.q.p + (long long)(w.first + row / p.g) * p.q.ts + (kvh * p.g + row % p.g) * p.q.hs + i % CH * 16);
            }
            const int row = base + tid;
            last_ahead = -1;
            if (tid < BQ && row < rows) {
                last_ahead = w.cached + row / p.g;
                log_ahead = p.lse[(long long)(w.first + row / p.g) * p.hq + kvh * p.g + row % p.g] * LOG2E;
            }
        };
        int base = max(0, w.slot0 - w.cached) * p.g + rank * BQ;
        if (base < rows) ask(base);
        for (; base < rows; base += S * BQ) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < EACH_Q; ++k) {
                const int i = tid + k * CNT;
                *reinterpret_cast<uint4 *>(Qs + i / CH * LD + i % CH * 4) = ahead[k];
            }
            if (tid < BQ) {
                last_of[tid] = last_ahead;
                log_of[tid] = log_ahead;
            }
            __syncthreads();
            if (base + S * BQ < rows) ask(base + S * BQ);
            uint64_t s2[4][4] = {};
#pragma unroll 4
            for (int d = 0; d < D; d += 4) {
                ulonglong2 k[4], q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) k[i] = *reinterpret_cast<const ulonglong2 *>(Ks + (tx + 16 * i) * LD + d);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const ulonglong2 *>(Qs + (ty + 16 * i) * LD + d);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s2[i][j] = fma2(k[i].y, q[j].y, fma2(k[i].x, q[j].x, s2[i][j]));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int last = last_of[ty + 16 * j];
                const float l = log_of[ty + 16 * j];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x, y;
                    un2(s2[i][j], x, y);
                    if (w.slot0 + tx + 16 * i <= last) acc[i] += ex2_approx(fmaf(x + y, p.scale_log2e, -l));
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) red[ty][tx + 16 * i] = acc[i];
        __syncthreads();
        if (tid < BK) {
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) x += red[i][tid];
            part[tid] = x;
        }
        cluster.sync();
        if (rank == 0 && tid < BK && w.slot0 + tid < n) {
            float x = 0.f;
            for (int r = 0; r < S; ++r) x += *cluster.map_shared_rank(&part[tid], r);
            p.mass[w.seq * p.rss + kvh * p.rhs + w.slot0 + tid] += x;
        }
        cluster.sync();
    }
}

template <int D>
cudaError_t launch_columns(const WindowParams &p, cudaStream_t s) {
    auto kern = sh_mass_columns_f32_kernel<D>;
    static ShKernelSetup setup;
    int sms = 0;
    const cudaError_t e = sh_setup_kernel(setup, kern, Cols<D>::BYTES, &sms);
    if (e != cudaSuccess) return e;
    // As many key blocks as there can be; CTAs of a cluster share a block's row tiles.  A tile takes about 3 us, a block 6 to begin and end, 4
    // more in a cluster; the longest block has the rows of all tokens.  (690 tokens of one key head: 72 us alone, 34 by 8; 592 short blocks of 8
    // heads: 119 alone, 188 by 2.)
    const long long blocks = std::min((long long)std::min(p.sequences, p.tokens) * ((p.slots + BK - 1) / BK), (1ll << 31) / p.hk) * p.hk, places = 2ll * sms;
    const double tiles = (double)p.tokens * p.g / BQ;
    auto us = [&](int n) { return (double)((blocks * n + places - 1) / places) * (n > 1 ? 10 : 6) + tiles / n * 3; };
    int S = 1;
    for (int n = 2; n <= 8; n *= 2)
        if (us(n) < us(S)) S = n;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(std::min(blocks, std::max(1ll, places / S)) * S));
    cfg.blockDim = dim3(CNT);
    cfg.dynamicSmemBytes = Cols<D>::BYTES;
    cfg.stream = s;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = S; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

}  // namespace

cudaError_t sh_launch_mass_fold(const WindowParams &p, cudaStream_t s) {
    const long long blocks = (p.slots + FOLD * EACH - 1) / (FOLD * EACH), all = blocks * p.sequences * p.hk;
    if (all > 0x7fffffffll) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)all);
    cfg.blockDim = dim3(FOLD);
    cfg.stream = s;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sh_mass_fold_kernel, p, (int)blocks);
}

cudaError_t sh_launch_mass_columns_f32(const WindowParams &p, int D, cudaStream_t s) { return D == 128 ? launch_columns<128>(p, s) : launch_columns<64>(p, s); }
