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
#include <math_constants.h>

#include "sh_pairs.cuh"
#include "sh_umma.cuh"
#include "sh_window.cuh"

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

template <int D>
__global__ void __launch_bounds__(NT, 4) sh_window_prefill_f32_kernel(const WindowParams p) {
    using C = Simt<D>;
    constexpr int BN = C::BN, NC = C::NC, LDK = C::LDK, LDP = C::LDP;
    extern __shared__ __align__(16) float sm[];
    float *Qs = sm, *Ks = sm + C::OFF_K, *Vs = sm + C::OFF_V, *Ps = sm + C::OFF_P;
    int *kpos = reinterpret_cast<int *>(sm + C::OFF_POS);            // positions of a block's keys (-1: in nobody's sight), two blocks in turn
    __shared__ Tile tile_sh;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int kvh = blockIdx.y;
    if (tid < 32) {
        const Tile t = find_tile(p, blockIdx.x, BM);
        if (tid == 0) tile_sh = t;
    }
    __syncthreads();
    const Tile t = tile_sh;
    if (t.seq < 0) return;
    const long long rows = (long long)t.count * p.g;
    const int qlo = (int)(t.row0 / p.g), qhi = (int)((min(t.row0 + BM, rows) - 1) / p.g);      // the tile's first and last token in the chunk
    const int oldest = t.cached + qlo - p.window + 1;                // the first row's window starts here
    const Ring ring(p.kc ? t.cached : 0, p.sinks, p.window);
    const int cblocks = (ring.live + BN - 1) / BN, blocks = cblocks + qhi / BN + 1;
    // the first block from b on with a key in sight
    auto seek = [&](int b) {
        for (; b < cblocks; ++b)
            if (ring.any(b * BN, b * BN + BN, oldest)) return b;
        const int lo = max(0, qlo - p.window + 1) / BN;              // (what lies between the sinks and the window is passed over)
        return b - cblocks < lo && t.cached + (b - cblocks) * BN >= p.sinks ? cblocks + lo : b;
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
            cp16_or_zero(value ? Vs + j * D + c * 4 : Ks + j * LDK + c * 4, take ? src + j * stride + c * 16 : (value ? p.v.p : p.k.p), take);
        }
        shumma::cp_async_commit();
    };
    int b = seek(0), turn = 0;
    if (tid < BN) kpos[tid] = position(b, tid);
    for (int i = tid; i < BM * (D / 4); i += NT) {
        const int r = i / (D / 4), c = i % (D / 4);
        const long long row = t.row0 + r, tok = t.first + row / p.g;
        const bool take = row < rows;
        cp16_or_zero(Qs + r * LDK + c * 4, take ? p.q.p + tok * p.q.ts + (kvh * p.g + (int)(row % p.g)) * p.q.hs + c * 16 : p.q.p, take);
    }
    __syncthreads();
    request(b, 0, false);
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
    while (b < blocks) {
        shumma::cp_async_wait_all();
        __syncthreads();                                             // the keys are there; the last block's P.V is done
        request(b, turn, true);
        const int next = seek(b + 1);
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
        float sum = l[a];
#pragma unroll
        for (int off = 8; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (qp[a] < 0) continue;
        const long long row = t.row0 + ty * R + a, tok = t.first + row / p.g;
        float *dst = reinterpret_cast<float *>(p.out.p + tok * p.out.ts + (kvh * p.g + (int)(row % p.g)) * p.out.hs);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            float x[4];
            un2(o[a][2 * c], x[0], x[1]);
            un2(o[a][2 * c + 1], x[2], x[3]);
            *reinterpret_cast<float4 *>(dst + c * 64 + tx * 4) = make_float4(x[0] / sum, x[1] / sum, x[2] / sum, x[3] / sum);
        }
    }
}

// Copy the rows that a later token can see into their slots: PIECES lanes move one token's key and value row of one head.
// Rows are found by bisection of `starts`; a warp's rows are neighbouring heads of the same token.
__global__ void __launch_bounds__(256) sh_window_append_kernel(const WindowParams p, int pieces) {
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(id % pieces);
    const long long rh = id / pieces;
    const int h = (int)(rh % p.hk);
    const long long tok = rh / p.hk;
    if (tok >= p.tokens) return;
    int lo = 0, hi = p.sequences;      // the last sequence that starts at or before tok (empty ones before it are passed over)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.starts[mid] <= tok) lo = mid; else hi = mid;
    }
    int first, count, cached;
    sequence_rows(p, lo, first, count, cached);
    if (tok < first || tok >= (long long)first + count) return;
    const int pos = cached + (int)(tok - first), end = cached + count;
    if (pos >= p.sinks && pos < end - p.window) return;      // pushed out of the window by the chunk itself
    const long long slot = slot_of(pos, p.sinks, p.window);
    const long long at = lo * p.css + h * p.chs + slot * p.cls + c * 16;
    const uint4 kk = *reinterpret_cast<const uint4 *>(p.k.p + tok * p.k.ts + h * p.k.hs + c * 16);
    const uint4 vv = *reinterpret_cast<const uint4 *>(p.v.p + tok * p.v.ts + h * p.v.hs + c * 16);
    *reinterpret_cast<uint4 *>(p.kc + at) = kk;
    *reinterpret_cast<uint4 *>(p.vc + at) = vv;
}

template <int D>
cudaError_t launch(const WindowParams &p, cudaStream_t s) {
    auto kern = sh_window_prefill_f32_kernel<D>;
    constexpr int bytes = Simt<D>::FLOATS * 4;
    static ShKernelSetup setup;
    int sms = 0;
    const cudaError_t e = sh_setup_kernel(setup, kern, bytes, &sms);
    if (e != cudaSuccess) return e;
    const long long tiles = (long long)p.tokens * p.g / BM + p.sequences;      // each sequence adds at most one partial tile
    if (tiles > 0x7fffffffll) return cudaErrorInvalidValue;
    kern<<<dim3((unsigned)tiles, p.hk), NT, bytes, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t sh_launch_window_prefill_f32(const WindowParams &p, int D, cudaStream_t s) { return D == 128 ? launch<128>(p, s) : launch<64>(p, s); }

cudaError_t sh_launch_window_append(const WindowParams &p, int es, int D, cudaStream_t s) {
    const int pieces = D * es / 16;
    const long long blocks = ((long long)p.tokens * p.hk * pieces + 255) / 256;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    sh_window_append_kernel<<<(unsigned)blocks, 256, 0, s>>>(p, pieces);
    return cudaGetLastError();
}
