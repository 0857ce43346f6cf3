// sh_qk_norm_rope: norm and rotation of query and key rows in one pass.
//
// A warp takes one token and walks over groups of its heads (4 heads of 128 elements or 8 of 64 at a time, D / 16 lanes a
// row), query heads first, then key heads; sines and cosines are made once per token and warp.  Bound by HBM: each row is
// read and written once.
#include "sh_rope.cuh"

namespace {

using namespace shrope;

constexpr int WARPS = 8;

template <typename T, int D>
__global__ void __launch_bounds__(WARPS * 32) sh_qk_norm_rope_kernel(const RopeParams r) {
    constexpr int LPR = D / 16, ROWS = 32 / LPR;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, p = lane % LPR;
    const int qg = (r.q_heads + ROWS - 1) / ROWS, kg = (r.k_heads + ROWS - 1) / ROWS;      // groups never mix queries and keys
    const int slices = (qg + kg + r.hpw - 1) / r.hpw;
    const long long item = (long long)blockIdx.x * WARPS + warp;
    const long long t = item / slices;
    if (t >= r.tokens) return;
    const int g0 = (int)(item % slices) * r.hpw, g1 = min(g0 + r.hpw, qg + kg);
    int e0, e1;
    runs<D>(r, p, e0, e1);
    float c[8], s[8];
    turns_of_lane<D>(r, t, lane, c, s);
    float w[16];
    const void *loaded = nullptr;
    for (int g = g0; g < g1; ++g) {
        const bool is_q = g < qg;
        const int h = (is_q ? g : g - qg) * ROWS + lane / LPR;
        const bool live = h < (is_q ? r.q_heads : r.k_heads);
        const WinRows &src = is_q ? r.q : r.k, &dst = is_q ? r.qo : r.ko;
        const void *weight = is_q ? r.qw : r.kw;
        if (weight && weight != loaded) {
            load16<T>(static_cast<const char *>(weight), e0, e1, w);
            loaded = weight;
        }
        float x[16] = {};
        if (live) load16<T>(src.p + t * src.ts + h * src.hs, e0, e1, x);
        apply<D>(r, p, weight != nullptr, weight != nullptr, w, c, s, x);
        if (live) store16<T>(dst.p + t * dst.ts + h * dst.hs, e0, e1, x);
    }
}

template <typename T, int D>
cudaError_t launch(RopeParams p, cudaStream_t s) {
    constexpr int ROWS = 32 / (D / 16);
    const int groups = (p.q_heads + ROWS - 1) / ROWS + (p.k_heads + ROWS - 1) / ROWS;
    p.hpw = groups;
    const int slices = (groups + p.hpw - 1) / p.hpw;
    const long long blocks = ((long long)p.tokens * slices + WARPS - 1) / WARPS;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    sh_qk_norm_rope_kernel<T, D><<<(unsigned)blocks, WARPS * 32, 0, s>>>(p);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_d(const RopeParams &p, int D, cudaStream_t s) {
    return D == 128 ? launch<T, 128>(p, s) : launch<T, 64>(p, s);
}

}  // namespace

cudaError_t sh_launch_qk_norm_rope(RopeParams p, int dtype, int D, cudaStream_t s) {
    if (dtype == SH_F32) return launch_d<float>(p, D, s);
    return dtype == SH_F16 ? launch_d<__half>(p, D, s) : launch_d<__nv_bfloat16>(p, D, s);
}
