// sh_window_prefill on CUDA cores, and sh_window_append.
//
// One CTA per 64 rows (token, head of the group) and key head.  It walks over the blocks of 64 keys that one of its rows can
// see, first those of the cache, then the chunk's, with the running maximum and sum of an online softmax; everything is fp32.
// The products are 4 x 4 (S) and 4 x D/16 (P.V) register tiles over operands in shared memory, so the kernel is bound by
// FMA issue and shared-memory reads.
#include <math_constants.h>

#include "sh_elem.cuh"
#include "sh_umma.cuh"
#include "sh_window.cuh"

namespace {

using shelem::Vec;
using namespace shwin;

constexpr int BM = 64, BN = 64, NT = 256, LD = BM + 4;

template <int D> constexpr int smem_floats() { return 2 * D * LD + BN * D + BN * LD + BN; }

template <typename T, int D>
__global__ void __launch_bounds__(NT) sh_window_prefill_simt_kernel(const WindowParams p) {
    extern __shared__ __align__(16) float sm[];
    float *Qs = sm, *Ks = Qs + D * LD, *Vs = Ks + D * LD, *Ps = Vs + BN * D;      // Qs[d][row], Ks[d][key], Vs[key][d], Ps[key][row]
    int *kpos = reinterpret_cast<int *>(Ps + BN * LD);
    __shared__ Tile tile_sh;
    constexpr int N = Vec<T>::N, PIECES = D / N;
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
    for (int i = tid; i < BM * PIECES; i += NT) {
        const int r = i / PIECES, c = i % PIECES;
        float x[N] = {};
        if (t.row0 + r < rows) {
            const long long row = t.row0 + r, tok = t.first + row / p.g;
            const int h = kvh * p.g + (int)(row % p.g);
            Vec<T>::unpack(*reinterpret_cast<const uint4 *>(p.q.p + tok * p.q.ts + h * p.q.hs + c * 16), x);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) Qs[(c * N + e) * LD + r] = x[e] * p.scale_log2e;
    }
    const int qlo = (int)(t.row0 / p.g), qhi = (int)((min(t.row0 + BM, rows) - 1) / p.g);      // the tile's first and last token in the chunk
    int qp[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) qp[a] = t.row0 + ty * 4 + a < rows ? t.cached + (int)((t.row0 + ty * 4 + a) / p.g) : -1;
    const int oldest = t.cached + qlo - p.window + 1;      // the first row's window starts here
    float m[4], l[4], o[4][D / 16];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        m[a] = -CUDART_INF_F; l[a] = 0.f;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) o[a][b] = 0.f;
    }
    const int slots = min(t.cached, p.sinks + p.window);      // live slots are the first ones
    const int cblocks = p.kc ? (slots + BN - 1) / BN : 0, blocks = cblocks + (qhi + BN) / BN;
    for (int b = 0; b < blocks; ++b) {
        const bool in_cache = b < cblocks;
        const int j0 = (in_cache ? b : b - cblocks) * BN;
        if (!in_cache && t.cached + j0 >= p.sinks && t.cached + j0 + BN <= oldest) continue;      // behind every row's window
        __syncthreads();      // the previous block's operands have been read
        int mine = -1;
        if (tid < BN) {
            mine = in_cache ? (j0 + tid < slots ? position_in(j0 + tid, t.cached, p.sinks, p.window) : -1)
                            : (j0 + tid <= qhi ? t.cached + j0 + tid : -1);
            if (mine >= p.sinks && mine < oldest) mine = -1;      // seen by no row of the tile
            kpos[tid] = mine;
        }
        if (!__syncthreads_or(mine >= 0)) continue;
        bool odd = false;      // a value that is not finite: weights of zero must not meet it
        for (int i = tid; i < BN * PIECES; i += NT) {
            const int r = i / PIECES, c = i % PIECES;
            float x[N] = {}, y[N] = {};
            if (kpos[r] >= 0) {
                const char *kr = in_cache ? p.kc + t.seq * p.css + kvh * p.chs + (j0 + r) * p.cls : p.k.p + (long long)(t.first + j0 + r) * p.k.ts + kvh * p.k.hs;
                const char *vr = in_cache ? p.vc + t.seq * p.css + kvh * p.chs + (j0 + r) * p.cls : p.v.p + (long long)(t.first + j0 + r) * p.v.ts + kvh * p.v.hs;
                Vec<T>::unpack(*reinterpret_cast<const uint4 *>(kr + c * 16), x);
                Vec<T>::unpack(*reinterpret_cast<const uint4 *>(vr + c * 16), y);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                Ks[(c * N + e) * LD + r] = x[e];
                Vs[r * D + c * N + e] = y[e];
                odd |= !isfinite(y[e]);
            }
        }
        odd = __syncthreads_or(odd);
        float s[4][4] = {};
#pragma unroll 8
        for (int d = 0; d < D; ++d) {
            const float4 qv = *reinterpret_cast<const float4 *>(Qs + d * LD + ty * 4), kv = *reinterpret_cast<const float4 *>(Ks + d * LD + tx * 4);
            const float qa[4] = {qv.x, qv.y, qv.z, qv.w}, ka[4] = {kv.x, kv.y, kv.z, kv.w};
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[a][c] = fmaf(qa[a], ka[c], s[a][c]);
        }
        const int4 kp4 = *reinterpret_cast<const int4 *>(kpos + tx * 4);
        const int kp[4] = {kp4.x, kp4.y, kp4.z, kp4.w};
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            float mx = -CUDART_INF_F;
            bool vis[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                vis[c] = kp[c] >= 0 && kp[c] <= qp[a] && (kp[c] < p.sinks || kp[c] > qp[a] - p.window);
                if (vis[c]) mx = fmaxf(mx, s[a][c]);
            }
#pragma unroll
            for (int off = 8; off; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            const float mn = fmaxf(m[a], mx), base = mn == -CUDART_INF_F ? 0.f : mn;      // nothing seen yet: all weights are 0
            const float keep = shumma::ex2_approx(m[a] - base);
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float e = vis[c] ? shumma::ex2_approx(s[a][c] - base) : 0.f;
                sum += e;
                Ps[(tx * 4 + c) * LD + ty * 4 + a] = e;
            }
            m[a] = mn;
            l[a] = l[a] * keep + sum;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) o[a][c] *= keep;
        }
        __syncthreads();
        if (!odd) {
#pragma unroll 4
            for (int j = 0; j < BN; ++j) {
                const float4 pv = *reinterpret_cast<const float4 *>(Ps + j * LD + ty * 4);
                const float pa[4] = {pv.x, pv.y, pv.z, pv.w};
#pragma unroll
                for (int c = 0; c < D / 64; ++c) {
                    const float4 vv = *reinterpret_cast<const float4 *>(Vs + j * D + c * 64 + tx * 4);
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        o[a][4 * c] = fmaf(pa[a], vv.x, o[a][4 * c]);
                        o[a][4 * c + 1] = fmaf(pa[a], vv.y, o[a][4 * c + 1]);
                        o[a][4 * c + 2] = fmaf(pa[a], vv.z, o[a][4 * c + 2]);
                        o[a][4 * c + 3] = fmaf(pa[a], vv.w, o[a][4 * c + 3]);
                    }
                }
            }
        } else {
            for (int j = 0; j < BN; ++j)
                for (int a = 0; a < 4; ++a) {
                    const int kpj = kpos[j];
                    if (!(kpj >= 0 && kpj <= qp[a] && (kpj < p.sinks || kpj > qp[a] - p.window))) continue;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) o[a][c] = fmaf(Ps[j * LD + ty * 4 + a], Vs[j * D + (c / 4) * 64 + tx * 4 + c % 4], o[a][c]);
                }
        }
    }
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        float sum = l[a];
#pragma unroll
        for (int off = 8; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (qp[a] < 0) continue;
        const long long row = t.row0 + ty * 4 + a, tok = t.first + row / p.g;
        const int h = kvh * p.g + (int)(row % p.g);
        T *dst = reinterpret_cast<T *>(p.out.p + tok * p.out.ts + h * p.out.hs);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = o[a][4 * c + e] / sum;
            if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4 *>(dst + c * 64 + tx * 4) = Vec<T>::pack(x);
            else *reinterpret_cast<uint2 *>(dst + c * 64 + tx * 4) = make_uint2(Vec<T>::pack2(x[0], x[1]), Vec<T>::pack2(x[2], x[3]));
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

template <typename T, int D>
cudaError_t launch(const WindowParams &p, cudaStream_t s) {
    auto kern = sh_window_prefill_simt_kernel<T, D>;
    constexpr int bytes = smem_floats<D>() * 4;
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

cudaError_t sh_launch_window_prefill_f32(const WindowParams &p, int D, cudaStream_t s) { return D == 128 ? launch<float, 128>(p, s) : launch<float, 64>(p, s); }

cudaError_t sh_launch_window_append(const WindowParams &p, int es, int D, cudaStream_t s) {
    const int pieces = D * es / 16;
    const long long blocks = ((long long)p.tokens * p.hk * pieces + 255) / 256;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    sh_window_append_kernel<<<(unsigned)blocks, 256, 0, s>>>(p, pieces);
    return cudaGetLastError();
}
