// sh_qk_norm_rope: norm and rotation of query and key rows in one pass.
//
// A warp takes one token and walks over groups of its heads (4 heads of 128 elements or 8 of 64 at a time, D / 16 lanes a
// row), query heads first, then key heads; sines and cosines are made once per token and warp.  The rows of UNROLL groups are
// requested before the first is worked on.  Bound by HBM: each row is read and written once.
// 16384 tokens of 40 + 8 heads of 128 (bf16, views of a packed projection): 73 us, 5.5 TB/s, 0.84 of the measured copy
// rate.  Instructions come next (two thirds of the issue slots before the arithmetic went to packed pairs: 85 us).  UNROLL 3 / 4 / 6
// at 5 or 6 blocks an SM: 73.1 / 73.5 / 97 us there, 17.2 / 15.9 / 20.2 us for 5003 tokens of 28 + 4 heads (fp16, three axes).
#include "sh_rope.cuh"

namespace {

using namespace shrope;

constexpr int WARPS = 4;

template <typename T, int D, bool ADJ>
__global__ void __launch_bounds__(WARPS * 32, 5) sh_qk_norm_rope_kernel(const RopeParams r) {
    constexpr int LPR = D / 16, ROWS = 32 / LPR, UNROLL = sizeof(T) == 4 ? 2 : 4;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, p = lane % LPR, sub = lane / LPR;
    const int qg = (r.q_heads + ROWS - 1) / ROWS, kg = (r.k_heads + ROWS - 1) / ROWS;      // groups never mix queries and keys
    const int slices = (qg + kg + r.hpw - 1) / r.hpw;
    const long long item = (long long)blockIdx.x * WARPS + warp;
    const long long t = item / slices;
    if (t >= r.tokens) return;
    const int g0 = (int)(item - t * slices) * r.hpw, g1 = min(g0 + r.hpw, qg + kg);
    int e0, e1;
    runs<D>(r, p, e0, e1);
    const char *q = r.q.p + t * r.q.ts, *k = r.k.p + t * r.k.ts;
    char *qo = r.qo.p + t * r.qo.ts, *ko = r.ko.p + t * r.ko.ts;
    Turns<ADJ> turn;
    uint64_t w[8] = {};                   // the weights of the present kind of rows
    const void *loaded = nullptr;
    bool turned = false;
    for (int g = g0; g < g1; g += UNROLL) {
        Raw<T> raw[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const bool is_q = g + u < qg;
            const int h = (is_q ? g + u : g + u - qg) * ROWS + sub;
#pragma unroll
            for (int i = 0; i < 2 * Raw<T>::PIECES; ++i) raw[u].a[i] = make_uint4(0, 0, 0, 0);
            if (g + u < g1 && h < (is_q ? r.q_heads : r.k_heads)) load_raw<T>(is_q ? q + h * r.q.hs : k + h * r.k.hs, e0, e1, raw[u]);
        }
        if (!turned) {                    // (behind the first loads)
            float c[8], s[8];
            turns_of_lane<D>(r, t, lane, c, s);
            turn.set(c, s);
            turned = true;
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (g + u >= g1) break;
            const bool is_q = g + u < qg;
            const int h = (is_q ? g + u : g + u - qg) * ROWS + sub;
            const void *weight = is_q ? r.qw : r.kw;
            if (weight && weight != loaded) {
                Raw<T> wr;
                load_raw<T>(static_cast<const char *>(weight), e0, e1, wr);
                unpack_raw<T>(wr, w);
                loaded = weight;
            }
            uint64_t x[8];
            unpack_raw<T>(raw[u], x);
            apply<D, ADJ>(r, p, weight != nullptr, true, w, turn, x);
            if (h < (is_q ? r.q_heads : r.k_heads)) store16<T>(is_q ? qo + h * r.qo.hs : ko + h * r.ko.hs, e0, e1, x);
        }
    }
}

template <typename T, int D>
cudaError_t launch(RopeParams p, cudaStream_t s) {
    constexpr int ROWS = 32 / (D / 16);
    const int groups = (p.q_heads + ROWS - 1) / ROWS + (p.k_heads + ROWS - 1) / ROWS;
    int dev = 0, sms = 0;
    const cudaError_t e = sh_device_sms(&dev, &sms);
    if (e != cudaSuccess) return e;
    // a warp walks through all of a token's groups once there are tokens for 16 warps on every SM; with fewer, the groups are
    // dealt out to more warps, each of which makes the sines and cosines again
    const long long share = (long long)p.tokens * groups / (16 * sms);
    p.hpw = share < 1 ? 1 : (share < groups ? (int)share : groups);
    const int slices = (groups + p.hpw - 1) / p.hpw;
    const long long blocks = ((long long)p.tokens * slices + WARPS - 1) / WARPS;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    if (p.adjacent) sh_qk_norm_rope_kernel<T, D, true><<<(unsigned)blocks, WARPS * 32, 0, s>>>(p);
    else sh_qk_norm_rope_kernel<T, D, false><<<(unsigned)blocks, WARPS * 32, 0, s>>>(p);
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
