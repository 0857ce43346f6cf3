// sh_window_decode on CUDA cores: one token per sequence over the window cache.
//
// Let t be the sequence's length before the step and s the slot of position t.  After the append the live slots are
// 0 .. min(t + 1, sinks + window) - 1, and every one of them holds a token that the query sees (the one that left the window
// lived in slot s).  So no position is ever needed: the kernel attends over the slots below min(t, sinks + window) except s,
// and over the new token, which it takes from the call's arguments.
//
// A cluster of S CTAs takes one (sequence, key head) and up to GQ of its query heads; rows are dealt out to the warps in
// blocks.  Eight lanes hold a row; each group of eight keeps its own running maximum, sum and output, merged through
// shuffles, shared memory and distributed shared memory at the end.  Bound by HBM: every live row is read once.
#include <cooperative_groups.h>
#include <math_constants.h>

#include "sh_rope.cuh"
#include "sh_umma.cuh"
#include "sh_window.cuh"

namespace cg = cooperative_groups;

namespace {

using shelem::Vec;
using shumma::ex2_approx;
using namespace shwin;

constexpr int WARPS = 8, NT = WARPS * 32;
constexpr int R = 2;                 // rows in flight per group of eight lanes
constexpr int BLOCK = 4 * R;         // rows of a warp per pass

// q rows (fp32) and the new token's key and value (as the cache holds them) into shared memory, prepared by `rope` if there is one.
template <typename T, int D, int GQ>
__device__ __forceinline__ void stage_token(const WindowParams &p, int seq, int kvh, int h0, int nq, float *qs, float *ks, float *vs) {
    constexpr int LPR = D / 16, ROWS = 32 / LPR;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pl = lane % LPR, sub = lane / LPR;
    // rows: the nq queries, the key, the value
    if (warp * ROWS >= nq + 2) return;
    float c[8], s[8];
    int e0 = 16 * pl, e1 = 16 * pl + 8;
    if (p.with_rope) {
        shrope::runs<D>(p.rope, pl, e0, e1);
        shrope::turns_of_lane<D>(p.rope, seq, lane, c, s);
    }
    for (int base = warp * ROWS; base < nq + 2; base += WARPS * ROWS) {
        const int row = base + sub;
        const bool is_q = row < nq, is_k = row == nq, live = row < nq + 2;
        const char *src = is_q ? p.q.p + seq * p.q.ts + (h0 + row) * p.q.hs
                               : (is_k ? p.k.p + seq * p.k.ts + kvh * p.k.hs : p.v.p + seq * p.v.ts + kvh * p.v.hs);
        float x[16] = {};
        if (live) shrope::load16<T>(src, e0, e1, x);
        if (p.with_rope) {
            const void *weight = is_q ? p.rope.qw : p.rope.kw;
            float w[16] = {}, y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = x[i];
            if (weight) shrope::load16<T>(static_cast<const char *>(weight), e0, e1, w);
            shrope::apply<D>(p.rope, pl, p.rope.qw || p.rope.kw, weight != nullptr, w, c, s, y);
            if (is_q || is_k) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = y[i];
            }
        }
        if (live) {
            float *dst = is_q ? qs + row * D : (is_k ? ks : vs);
            if (is_k) {      // the row as it will be read back
#pragma unroll
                for (int i = 0; i < 16; i += Vec<T>::N) Vec<T>::unpack(Vec<T>::pack(x + i), x + i);
            }
            const float f = is_q ? p.scale_log2e : 1.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) { dst[e0 + i] = x[i] * f; dst[e1 + i] = x[8 + i] * f; }
        }
    }
}

template <typename T, int D, int GQ>
__global__ void __launch_bounds__(NT) sh_window_decode_simt_kernel(const WindowParams p, int qblocks) {
    constexpr int N = Vec<T>::N, CH = D / N / 8, EL = CH * N;      // 16-byte pieces and elements of a row per lane
    __shared__ __align__(16) float qs[GQ * D], ks[D], vs[D];
    __shared__ float part[WARPS][GQ][D + 2];
    __shared__ float cta[GQ][D + 2];                                // this CTA's maximum, sum, output
    cg::cluster_group cluster = cg::this_cluster();
    const int S = cluster.num_blocks(), rank = cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, l8 = lane & 7, grp = lane >> 3;
    const long long unit = blockIdx.x / S;
    const int qb = (int)(unit % qblocks), kvh = (int)(unit / qblocks % p.hk), seq = (int)(unit / qblocks / p.hk);
    const int t = min(p.lengths[seq], MAX_POS);
    if (t < 0) return;                                              // idle: the whole cluster leaves
    const int h0 = kvh * p.g + qb * GQ, nq = min(GQ, p.g - qb * GQ);
    const int live = min(t, p.sinks + p.window), snew = slot_of(t, p.sinks, p.window);
    for (int i = tid; i < GQ * D; i += NT) qs[i] = 0.f;
    __syncthreads();
    stage_token<T, D, GQ>(p, seq, kvh, h0, nq, qs, ks, vs);
    __syncthreads();

    float m[GQ], l[GQ], o[GQ][EL];
#pragma unroll
    for (int q = 0; q < GQ; ++q) {
        m[q] = -CUDART_INF_F; l[q] = 0.f;
#pragma unroll
        for (int e = 0; e < EL; ++e) o[q][e] = 0.f;
    }
    // fold R rows (k, v: this lane's elements; valid: the group's row is to be used) into the running state
    auto fold = [&](const float (&k)[R][EL], const float (&v)[R][EL], const bool (&valid)[R]) {
#pragma unroll
        for (int q = 0; q < GQ; ++q) {
            float s[R];
#pragma unroll
            for (int r = 0; r < R; ++r) s[r] = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float qv = qs[q * D + (c * 8 + l8) * N + e];
#pragma unroll
                    for (int r = 0; r < R; ++r) s[r] = fmaf(qv, k[r][c * N + e], s[r]);
                }
            float mn = m[q];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
                s[r] += __shfl_xor_sync(0xffffffffu, s[r], 2);
                s[r] += __shfl_xor_sync(0xffffffffu, s[r], 4);
                if (valid[r]) mn = fmaxf(mn, s[r]);
            }
            const float base = mn == -CUDART_INF_F ? 0.f : mn, keep = ex2_approx(m[q] - base);
            m[q] = mn;
            float w[R], sum = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                w[r] = valid[r] ? ex2_approx(s[r] - base) : 0.f;
                sum += w[r];
            }
            l[q] = l[q] * keep + sum;
#pragma unroll
            for (int e = 0; e < EL; ++e) {
                float x = o[q][e] * keep;
#pragma unroll
                for (int r = 0; r < R; ++r) x = fmaf(w[r], v[r][e], x);
                o[q][e] = x;
            }
        }
    };
    const char *kc = p.kc + seq * p.css + kvh * p.chs, *vc = p.vc + seq * p.css + kvh * p.chs;
    for (int base = (rank * WARPS + warp) * BLOCK; base < live; base += S * WARPS * BLOCK) {
        float k[R][EL], v[R][EL];
        bool valid[R];
        uint4 kr[R][CH], vr[R][CH];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int j = base + r * 4 + grp;
            valid[r] = j < live && j != snew;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                kr[r][c] = vr[r][c] = make_uint4(0, 0, 0, 0);       // rows that are not used count as zeros, whatever they hold
                if (valid[r]) {
                    kr[r][c] = *reinterpret_cast<const uint4 *>(kc + j * p.cls + (c * 8 + l8) * 16);
                    vr[r][c] = *reinterpret_cast<const uint4 *>(vc + j * p.cls + (c * 8 + l8) * 16);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                Vec<T>::unpack(kr[r][c], k[r] + c * N);
                Vec<T>::unpack(vr[r][c], v[r] + c * N);
            }
        fold(k, v, valid);
    }
    if (rank == 0 && warp == 0) {      // the new token: one group counts it, and the first query block stores it
        float k[R][EL] = {}, v[R][EL] = {};
        bool valid[R] = {};
        valid[0] = grp == 0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                k[0][c * N + e] = ks[(c * 8 + l8) * N + e];
                v[0][c * N + e] = valid[0] ? vs[(c * 8 + l8) * N + e] : 0.f;
            }
        fold(k, v, valid);
        if (qb == 0 && grp == 0) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                *reinterpret_cast<uint4 *>(p.kc + seq * p.css + kvh * p.chs + snew * p.cls + (c * 8 + l8) * 16) = Vec<T>::pack(k[0] + c * N);
                *reinterpret_cast<uint4 *>(p.vc + seq * p.css + kvh * p.chs + snew * p.cls + (c * 8 + l8) * 16) = Vec<T>::pack(v[0] + c * N);
            }
        }
    }
    // the four groups of the warp
#pragma unroll
    for (int q = 0; q < GQ; ++q) {
        float M = m[q];
        M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 8));
        M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 16));
        const float f = ex2_approx(m[q] - (M == -CUDART_INF_F ? 0.f : M));
        float L = l[q] * f;
        L += __shfl_xor_sync(0xffffffffu, L, 8);
        L += __shfl_xor_sync(0xffffffffu, L, 16);
#pragma unroll
        for (int e = 0; e < EL; ++e) {
            float x = o[q][e] * f;
            x += __shfl_xor_sync(0xffffffffu, x, 8);
            x += __shfl_xor_sync(0xffffffffu, x, 16);
            if (grp == 0) part[warp][q][2 + ((e / N) * 8 + l8) * N + e % N] = x;
        }
        if (lane == 0) { part[warp][q][0] = M; part[warp][q][1] = L; }
    }
    __syncthreads();
    for (int i = tid; i < GQ * D; i += NT) {      // the warps
        const int q = i / D, d = i % D;
        float M = -CUDART_INF_F, L = 0.f, x = 0.f;
        for (int w = 0; w < WARPS; ++w) M = fmaxf(M, part[w][q][0]);
        const float base = M == -CUDART_INF_F ? 0.f : M;
        for (int w = 0; w < WARPS; ++w) {
            const float f = ex2_approx(part[w][q][0] - base);
            L += part[w][q][1] * f;
            x += part[w][q][2 + d] * f;
        }
        cta[q][2 + d] = x;
        if (d == 0) { cta[q][0] = M; cta[q][1] = L; }
    }
    cluster.sync();
    for (int i = rank * NT + tid; i < nq * (D / N); i += S * NT) {      // the CTAs of the cluster: each finishes some pieces
        const int q = i / (D / N), d = i % (D / N) * N;
        float M = -CUDART_INF_F, L = 0.f, x[N] = {};
        for (int r = 0; r < S; ++r) M = fmaxf(M, cluster.map_shared_rank(&cta[q][0], r)[0]);
        const float base = M == -CUDART_INF_F ? 0.f : M;
        for (int r = 0; r < S; ++r) {
            const float *c = cluster.map_shared_rank(&cta[q][0], r);
            const float f = ex2_approx(c[0] - base);
            L += c[1] * f;
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = fmaf(c[2 + d + e], f, x[e]);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] /= L;
        *reinterpret_cast<uint4 *>(p.out.p + seq * p.out.ts + (h0 + q) * p.out.hs + d * (int)sizeof(T)) = Vec<T>::pack(x);
    }
    cluster.sync();      // nobody's shared memory goes away while it is read
}

template <typename T, int D, int GQ>
cudaError_t launch(const WindowParams &p, cudaStream_t s) {
    const int qblocks = (p.g + GQ - 1) / GQ;
    const long long units = (long long)p.sequences * p.hk * qblocks;
    int sms = 0, dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    // few units: split the axis of keys while that fills SMs and leaves each CTA two passes of its warps at least
    int S = 1;
    while (S < 8 && units * S * 2 <= 2 * sms && (p.window + p.sinks) >= 2 * S * 2 * WARPS * BLOCK) S *= 2;
    if (units * S > 0x7fffffffll) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * S));
    cfg.blockDim = dim3(NT);
    cfg.stream = s;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = S; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sh_window_decode_simt_kernel<T, D, GQ>, p, qblocks);
}

template <typename T, int D>
cudaError_t launch_g(const WindowParams &p, cudaStream_t s) {
    return p.g == 1 ? launch<T, D, 1>(p, s) : (p.g == 2 ? launch<T, D, 2>(p, s) : launch<T, D, 4>(p, s));
}
template <typename T>
cudaError_t launch_d(const WindowParams &p, int D, cudaStream_t s) {
    return D == 128 ? launch_g<T, 128>(p, s) : launch_g<T, 64>(p, s);
}

}  // namespace

cudaError_t sh_launch_window_decode(const WindowParams &p, int dtype, int D, cudaStream_t s) {
    if (dtype == SH_F32) return launch_d<float>(p, D, s);
    return dtype == SH_F16 ? launch_d<__half>(p, D, s) : launch_d<__nv_bfloat16>(p, D, s);
}
