// sh_window_prefill for fp32 rows, on CUDA cores, and sh_window_append.
//
// One CTA per 32 rows (token, head of the group) and key head.  It walks over the blocks of keys that one of its rows can see, first
// those of the cache, then the chunk's, with the running maximum and sum of an online softmax; everything is fp32.  A thread
// works on 4 rows: S for every 16th key, O for 4 neighbouring columns of each 64.  Two elements of d share a register pair (packed
// multiply-adds), so the operands of S come as they lie in the rows.  Keys and values arrive by cp.async: a block's values while its
// S is worked out, the next block's keys during P.V; rows in nobody's sight are filled with zeros, whatever they hold.
// 700 + 511 tokens, 16 heads of 64, window 346, 64 sinks: 81 us, 17 TFLOP/s of a possible 74 (the first version, 64-row tiles with
// transposed operands: 127 us).  Bound by the latency of shared-memory reads at 16 warps an SM (8 of 16 bytes for 32 packed
// multiply-adds), and by the tiles' masked parts, half again of the work.
#include <cooperative_groups.h>
#include <math_constants.h>

#include <algorithm>

#include "sh_pairs.cuh"
#include "sh_umma.cuh"
#include "sh_window.cuh"

namespace cg = cooperative_groups;

namespace {

using namespace shpair;
using namespace shwin;

constexpr int NT = 128, R = 4, BM = 8 * R;      // threads, rows of a thread, rows of a CTA

template <int D> struct Simt {
    static constexpr int BN = D == 64 ? 64 : 32, NC = BN / 16;      // keys of a block, of a thread
    static constexpr int LDK = D + 4, LDP = BN + 4;            // padded rows: lanes on neighbouring rows meet different banks
    static constexpr int OFF_K = BM * LDK, OFF_V = OFF_K + BN * LDK, OFF_P = OFF_V + BN * D, OFF_POS = OFF_P + BM * LDP, FLOATS = OFF_POS + 2 * BN;
    static constexpr int EACH = BN * D / 4 / NT;               // 16-byte pieces of a block's keys per thread
    static_assert(NT % (D / 4) == 0, "a thread's pieces share a column");
};

__device__ __forceinline__ void cp16_or_zero(void *dst, const void *src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(shasync::smem_u32(dst)), "l"(src), "r"(take ? 16 : 0) : "memory");
}

template <int D, int MODE>
__global__ void __launch_bounds__(NT, 4) sh_window_prefill_f32_kernel(const WindowParams p) {
    using C = Simt<D>;
    constexpr int BN = C::BN, NC = C::NC, LDK = C::LDK, LDP = C::LDP;
    extern __shared__ __align__(16) float sm[];
    float *Qs = sm, *Ks = sm + C::OFF_K, *Vs = sm + C::OFF_V, *Ps = sm + C::OFF_P;
    int *kpos = reinterpret_cast<int *>(sm + C::OFF_POS);            // positions of a block's keys (-1: in nobody's sight), two blocks in turn
    __shared__ Tile tile_sh;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int kvh = blockIdx.y;
    // (contexts and caches with masses) the CTAs of a cluster take the blocks of keys in turn
    cg::cluster_group cluster = cg::this_cluster();
    const int S = MODE == ATTEND_WINDOW ? 1 : cluster.num_blocks(), rank = MODE == ATTEND_WINDOW ? 0 : cluster.block_rank();
    if (tid < 32) {
        const Tile t = find_tile<MODE>(p, MODE == ATTEND_WINDOW ? blockIdx.x : blockIdx.x / S, BM);
        if (tid == 0) tile_sh = t;
    }
    __syncthreads();
    const Tile t = tile_sh;
    if (t.seq < 0) {                                                 // (the whole cluster)
        if (MODE != ATTEND_WINDOW) sh_pdl_wait();
        return;
    }
    const long long rows = (long long)t.count * p.g;
    const int qlo = (int)(t.row0 / p.g), qhi = (int)((min(t.row0 + BM, rows) - 1) / p.g);      // the tile's first and last token in the chunk
    const int oldest = t.cached + qlo - p.window + 1;                // the first row's window starts here
    const Ring ring(p.kc ? t.cached : 0, p.sinks, p.window);
    const int cblocks = (ring.live + BN - 1) / BN, blocks = cblocks + (MODE == ATTEND_CONTEXT ? 0 : qhi / BN + 1);
    // the first block from b on with a key in sight
    auto seek = [&](int b) {
        for (; b < cblocks; ++b)
            if (ring.any(b * BN, b * BN + BN, oldest)) return b;
        const int lo = max(0, qlo - p.window + 1) / BN;              // (what lies between the sinks and the window is passed over)
        return MODE != ATTEND_CONTEXT && b - cblocks < lo && t.cached + (b - cblocks) * BN >= p.sinks ? cblocks + lo : b;
    };
    auto position = [&](int b, int j) {
        int pos;
        if (b < cblocks) pos = position_in(b * BN + j, t.cached, p.sinks, p.window);
        else pos = (b - cblocks) * BN + j <= qhi ? t.cached + (b - cblocks) * BN + j : -1;
        return pos >= p.sinks && pos < oldest ? -1 : pos;
    };
    // keys or values of block b; kpos of the block is there
    auto request = [&](int b, int turn, bool value) {
        constexpr int PIECES = D / 4, STEP = NT / PIECES;
        const int c = tid % PIECES;
        const char *src;
        long long stride;
        if (b < cblocks) {
            src = (value ? p.vc : p.kc) + t.seq * p.css + kvh * p.chs + (long long)b * BN * p.cls;
            stride = p.cls;
        } else {
            const WinRows &x = value ? p.v : p.k;
            src = x.p + ((long long)t.first + (b - cblocks) * BN) * x.ts + kvh * x.hs;
            stride = x.ts;
        }
#pragma unroll
        for (int i = 0; i < C::EACH; ++i) {
            const int j = tid / PIECES + i * STEP;
            const bool take = kpos[turn * BN + j] >= 0;
            cp16_or_zero(value ? Vs + j * D + c * 4 : Ks + j * LDK + c * 4, take ? src + j * stride + c * 16 : p.q.p, take);
        }
        shumma::cp_async_commit();
    };
    auto next_of = [&](int b) {
        b = seek(b + 1);
        for (int i = 1; i < S && b < blocks; ++i) b = seek(b + 1);
        return b;
    };
    int b = seek(0), turn = 0;
    for (int i = 0; i < rank && b < blocks; ++i) b = seek(b + 1);
    if (tid < BN) kpos[tid] = position(b, tid);
    for (int i = tid; i < BM * (D / 4); i += NT) {
        const int r = i / (D / 4), c = i % (D / 4);
        const long long row = t.row0 + r, tok = t.first + row / p.g;
        const bool take = row < rows;
        cp16_or_zero(Qs + r * LDK + c * 4, take ? p.q.p + tok * p.q.ts + (kvh * p.g + (int)(row % p.g)) * p.q.hs + c * 16 : p.q.p, take);
    }
    __syncthreads();
    if (MODE == ATTEND_WINDOW || b < blocks) request(b, 0, false);      // (a context may have no rows, a CTA no blocks)
    int qp[R];
    float m[R], l[R];
    uint64_t o[R][D / 32];                                           // pairs of columns
#pragma unroll
    for (int a = 0; a < R; ++a) {
        const long long row = t.row0 + ty * R + a;
        qp[a] = row < rows ? t.cached + (int)(row / p.g) : -1;
        m[a] = -CUDART_INF_F; l[a] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) o[a][c] = 0;
    }
    if (MODE != ATTEND_WINDOW && b >= blocks) shumma::cp_async_wait_all();
    while (b < blocks) {
        shumma::cp_async_wait_all();
        __syncthreads();                                             // the keys are there; the last block's P.V is done
        request(b, turn, true);
        const int next = MODE == ATTEND_WINDOW ? seek(b + 1) : next_of(b);
        if (next < blocks && tid < BN) kpos[(turn ^ 1) * BN + tid] = position(next, tid);
        uint64_t s2[R][NC] = {};                                     // even and odd elements of d
#pragma unroll 2
        for (int d = 0; d < D; d += 4) {
            ulonglong2 q[R], k[NC];
#pragma unroll
            for (int a = 0; a < R; ++a) q[a] = *reinterpret_cast<const ulonglong2 *>(Qs + (ty * R + a) * LDK + d);
#pragma unroll
            for (int c = 0; c < NC; ++c) k[c] = *reinterpret_cast<const ulonglong2 *>(Ks + (tx + 16 * c) * LDK + d);
#pragma unroll
            for (int a = 0; a < R; ++a)
#pragma unroll
                for (int c = 0; c < NC; ++c) s2[a][c] = fma2(q[a].y, k[c].y, fma2(q[a].x, k[c].x, s2[a][c]));
        }
        int kp[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) kp[c] = kpos[turn * BN + tx + 16 * c];
#pragma unroll
        for (int a = 0; a < R; ++a) {
            float s[NC], mx = -CUDART_INF_F;
            bool vis[NC];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                float x, y;
                un2(s2[a][c], x, y);
                s[c] = (x + y) * p.scale_log2e;
                vis[c] = kp[c] >= 0 && kp[c] <= qp[a] && (kp[c] < p.sinks || kp[c] > qp[a] - p.window);
                if (vis[c]) mx = fmaxf(mx, s[c]);
            }
#pragma unroll
            for (int off = 8; off; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            const float mn = fmaxf(m[a], mx), base = mn == -CUDART_INF_F ? 0.f : mn;      // nothing seen yet: all weights are 0
            const float keep = shumma::ex2_approx(m[a] - base);
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const float e = vis[c] ? shumma::ex2_approx(s[c] - base) : 0.f;
                sum += e;
                Ps[(ty * R + a) * LDP + tx + 16 * c] = e;
            }
            m[a] = mn;
            l[a] = l[a] * keep + sum;
            const uint64_t keep2 = f2(keep, keep);
#pragma unroll
            for (int c = 0; c < D / 32; ++c) o[a][c] = mul2(o[a][c], keep2);
        }
        shumma::cp_async_wait_all();
        bool odd = false;                                            // a value that is not finite: weights of zero must not meet it
#pragma unroll
        for (int i = 0; i < C::EACH; ++i) {
            const float4 v = *reinterpret_cast<const float4 *>(Vs + (tid / (D / 4) + i * (NT / (D / 4))) * D + tid % (D / 4) * 4);      // (its own pieces)
            odd |= !(isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w));
        }
        odd = __syncthreads_or(odd);                                 // values and weights are there; S is done with the keys
        if (next < blocks) request(next, turn ^ 1, false);
        if (!odd) {
#pragma unroll 2
            for (int j = 0; j < BN; j += 4) {
                float w[R][4];
#pragma unroll
                for (int a = 0; a < R; ++a) {
                    const float4 x = *reinterpret_cast<const float4 *>(Ps + (ty * R + a) * LDP + j);
                    w[a][0] = x.x; w[a][1] = x.y; w[a][2] = x.z; w[a][3] = x.w;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) {
                        const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(Vs + (j + e) * D + c * 64 + tx * 4);
#pragma unroll
                        for (int a = 0; a < R; ++a) {
                            const uint64_t ww = f2(w[a][e], w[a][e]);
                            o[a][2 * c] = fma2(ww, v.x, o[a][2 * c]);
                            o[a][2 * c + 1] = fma2(ww, v.y, o[a][2 * c + 1]);
                        }
                    }
            }
        } else {
            for (int j = 0; j < BN; ++j) {
                const int kpj = kpos[turn * BN + j];
#pragma unroll
                for (int a = 0; a < R; ++a) {
                    if (!(kpj >= 0 && kpj <= qp[a] && (kpj < p.sinks || kpj > qp[a] - p.window))) continue;
                    const float w = Ps[(ty * R + a) * LDP + j];
                    const uint64_t ww = f2(w, w);
#pragma unroll
                    for (int c = 0; c < D / 32; ++c)
                        o[a][c] = fma2(ww, *reinterpret_cast<const uint64_t *>(Vs + j * D + (c / 2) * 64 + tx * 4 + (c % 2) * 2), o[a][c]);
                }
            }
        }
        b = next;
        turn ^= 1;
    }
#pragma unroll
    for (int a = 0; a < R; ++a) {
#pragma unroll
        for (int off = 8; off; off >>= 1) l[a] += __shfl_xor_sync(0xffffffffu, l[a], off);
    }
    // a cluster's CTAs merge: each finishes every S-th row from what the others have left in their shared memory
    constexpr int LDO = D + 4;
    if (MODE != ATTEND_WINDOW && S > 1) {
        __syncthreads();                                             // (nobody reads tiles any more)
#pragma unroll
        for (int a = 0; a < R; ++a) {
            float *row = sm + (ty * R + a) * LDO;
#pragma unroll
            for (int c = 0; c < D / 64; ++c) *reinterpret_cast<ulonglong2 *>(row + c * 64 + tx * 4) = make_ulonglong2(o[a][2 * c], o[a][2 * c + 1]);
            if (tx == 0) { row[D] = m[a]; row[D + 1] = l[a]; }
        }
        cluster.sync();
#pragma unroll
        for (int a = 0; a < R; ++a) {
            if ((ty * R + a) % S != rank) continue;
            float M = -CUDART_INF_F;
            for (int r = 0; r < S; ++r) M = fmaxf(M, cluster.map_shared_rank(sm + (ty * R + a) * LDO, r)[D]);
            const float base = M == -CUDART_INF_F ? 0.f : M;
            float L = 0.f;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) o[a][c] = 0;
            for (int r = 0; r < S; ++r) {
                const float *row = cluster.map_shared_rank(sm + (ty * R + a) * LDO, r);
                const float f = shumma::ex2_approx(row[D] - base);
                L += row[D + 1] * f;
#pragma unroll
                for (int c = 0; c < D / 64; ++c) {
                    const ulonglong2 x = *reinterpret_cast<const ulonglong2 *>(row + c * 64 + tx * 4);
                    o[a][2 * c] = fma2(x.x, f2(f, f), o[a][2 * c]);
                    o[a][2 * c + 1] = fma2(x.y, f2(f, f), o[a][2 * c + 1]);
                }
            }
            m[a] = M; l[a] = L;
        }
        cluster.sync();                                              // nobody's shared memory goes away while it is read
    }
#pragma unroll
    for (int a = 0; a < R; ++a) {
        const float sum = l[a];
        if (qp[a] < 0 || (MODE != ATTEND_WINDOW && (ty * R + a) % S != rank)) continue;
        const long long row = t.row0 + ty * R + a, tok = t.first + row / p.g;
        const int h = kvh * p.g + (int)(row % p.g);
        Close end = {};
        if constexpr (MODE != ATTEND_WINDOW) {
            end = close_row<MODE>(p, tok, h, m[a], sum);
            if (tx == 0) p.lse[tok * p.hq + h] = 0.69314718055994531f * end.total;
            if (MODE == ATTEND_CONTEXT && blocks == 0) end.own = 1.f;      // no rows: zeros
        }
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            float x[4];
            un2(o[a][2 * c], x[0], x[1]);
            un2(o[a][2 * c + 1], x[2], x[3]);
            if constexpr (MODE == ATTEND_WINDOW) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] /= sum;
            } else {
                float y[4] = {};
                if (end.other != 0.f) prior_row<float>(p, tok, h, c * 64 + tx * 4, y);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = fmaf(y[e], end.other, x[e] * end.own);
            }
            store_row<float, MODE>(p, tok, h, c * 64 + tx * 4, x);
        }
    }
    if (MODE != ATTEND_WINDOW) sh_pdl_wait();                        // who comes after this launch also comes after the one beside it
}

// Copy the rows that a later token can see into their slots: PIECES lanes move one token's key and value row of one head.
// A warp's rows are neighbouring heads of the same token.
template <int MODE>
__global__ void __launch_bounds__(256) sh_window_append_kernel(const WindowParams p, int pieces) {
    if (MODE == ATTEND_MASS) {
        sh_pdl_launch_dependents();      // (the attention needs nothing of this)
        if (blockIdx.x == 0 && threadIdx.x == 0 && p.taken) *p.taken = 0;
    }
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(id % pieces);
    const long long rh = id / pieces;
    const int h = (int)(rh % p.hk);
    const long long tok = rh / p.hk;
    if (tok >= p.tokens) return;
    int lo, first, count, cached;
    if (!sequence_of<MODE>(p, tok, lo, first, count, cached)) return;
    const int pos = cached + (int)(tok - first), end = cached + count;
    if (pos >= p.sinks && pos < end - p.window) return;      // pushed out of the window by the chunk itself
    const long long slot = slot_of(pos, p.sinks, p.window);
    const long long at = lo * p.css + h * p.chs + slot * p.cls + c * 16;
    const uint4 kk = *reinterpret_cast<const uint4 *>(p.k.p + tok * p.k.ts + h * p.k.hs + c * 16);
    const uint4 vv = *reinterpret_cast<const uint4 *>(p.v.p + tok * p.v.ts + h * p.v.hs + c * 16);
    *reinterpret_cast<uint4 *>(p.kc + at) = kk;
    *reinterpret_cast<uint4 *>(p.vc + at) = vv;
    if (MODE == ATTEND_MASS && c == 0) {
        const long long r = lo * p.rss + h * p.rhs + slot;
        p.mass[r] = 0.f;
        p.held[r] = p.seen[lo] + (int)(tok - first);
    }
}

// Zeros, and -infinity, in the rows before the first context's and behind the last one's.
__global__ void __launch_bounds__(256) sh_clear_rest_kernel(const WindowParams p, int pieces) {
    sh_pdl_launch_dependents();      // (the attention writes other rows)
    const int first = min(max(p.starts[0], 0), p.tokens), end = min(max(p.starts[p.sequences], first), p.tokens);
    const long long rows = (long long)(p.tokens - (end - first)) * p.hq;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += gridDim.x * 256ll) {
        const int c = (int)(i % pieces), h = (int)(i / pieces % p.hq);
        long long tok = i / pieces / p.hq;
        if (tok >= first) tok += end - first;
        *reinterpret_cast<uint4 *>(p.out.p + tok * p.out.ts + h * p.out.hs + c * 16) = make_uint4(0, 0, 0, 0);
        if (c == 0) p.lse[tok * p.hq + h] = -CUDART_INF_F;
    }
}

template <int D, int MODE>
cudaError_t launch(const WindowParams &p, cudaStream_t s) {
    auto kern = sh_window_prefill_f32_kernel<D, MODE>;
    constexpr int bytes = Simt<D>::FLOATS * 4;
    static ShKernelSetup setup;
    static_assert(BM * (D + 4) <= Simt<D>::FLOATS, "a CTA's result takes the place of its tiles");
    int sms = 0;
    const cudaError_t e = sh_setup_kernel(setup, kern, bytes, &sms);
    if (e != cudaSuccess) return e;
    const long long tiles = (long long)p.tokens * p.g / BM + p.sequences;      // each sequence adds at most one partial tile
    if (tiles > 0x7fffffffll) return cudaErrorInvalidValue;
    if constexpr (MODE == ATTEND_WINDOW) {
        kern<<<dim3((unsigned)tiles, p.hk), NT, bytes, s>>>(p);
        return cudaGetLastError();
    } else {
        // few row tiles: clusters share the keys of one, up to 16 CTAs an SM (4 run at once, so in up to four waves) with two blocks each.
        // Chunks of 64, 17 and 200 tokens over 500, 0 and 31 rows, 12 heads of 64: 47 -> 32 us.  Up to 16 an SM against up to 4, us of attention
        // to contexts: 128 tokens over 3000 rows, 40 heads of 64: 173, 198; 256 tokens: 313, 373; chunks
        // of 64, 17 and 200 over 7900, 4000 and 7000, 12 heads: 288, 310; 512 over 3000, 8 heads: 138, 130; 4 x 64 over 3900, 16 heads over 2
        // of 128: 327, 315.  Where the caches hold little of what they have room for (4 x 64 over 390 of 4000), it costs more: 58, 50.
        int S = 1;
        while (S < 8 && tiles * p.hk * S * 2 <= 16ll * sms && p.slots >= 2 * S * 2 * Simt<D>::BN) S *= 2;
        if (tiles * S > 0x7fffffffll) return cudaErrorInvalidValue;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(tiles * S), p.hk);
        cfg.blockDim = dim3(NT);
        cfg.dynamicSmemBytes = bytes;
        cfg.stream = s;
        cudaLaunchAttribute attr[2] = {};
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = S; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = MODE == ATTEND_MASS || p.clear_rest ? 2 : 1;  // (beside the launch that stores the chunk, or clears what belongs to no context)
        return cudaLaunchKernelEx(&cfg, kern, p);
    }
}

}  // namespace

cudaError_t sh_launch_window_prefill_f32(const WindowParams &p, int D, int mode, cudaStream_t s) {
    if (mode == ATTEND_CONTEXT) return D == 128 ? launch<128, ATTEND_CONTEXT>(p, s) : launch<64, ATTEND_CONTEXT>(p, s);
    if (mode == ATTEND_MASS) return D == 128 ? launch<128, ATTEND_MASS>(p, s) : launch<64, ATTEND_MASS>(p, s);
    return D == 128 ? launch<128, ATTEND_WINDOW>(p, s) : launch<64, ATTEND_WINDOW>(p, s);
}

cudaError_t sh_launch_window_append(const WindowParams &p, int es, int D, int mode, cudaStream_t s) {
    const int pieces = D * es / 16;
    const long long blocks = ((long long)p.tokens * p.hk * pieces + 255) / 256;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    if (mode == ATTEND_MASS) sh_window_append_kernel<ATTEND_MASS><<<(unsigned)blocks, 256, 0, s>>>(p, pieces);
    else sh_window_append_kernel<ATTEND_WINDOW><<<(unsigned)blocks, 256, 0, s>>>(p, pieces);
    return cudaGetLastError();
}

cudaError_t sh_launch_clear_rest(const WindowParams &p, int row_bytes, cudaStream_t s) {
    sh_clear_rest_kernel<<<32, 256, 0, s>>>(p, row_bytes / 16);
    return cudaGetLastError();
}
