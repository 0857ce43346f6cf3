// Norm and rotation of one row of head_dim elements, shared by D / 16 lanes: the device side of sh_rope.
//
// Lane p of a row's D / 16 lanes holds 16 elements.  While p < rot / 16 they are pairs 8p .. 8p + 7: both members of a
// pair are in one lane, in either pairing ((i, i + rot/2): the pieces at 8p and rot/2 + 8p; (2i, 2i + 1): the 16 elements
// from 16p on), so the rotation needs no exchange.  The lanes behind hold 16 consecutive elements that only get normalised.
// The angle is position * inv_freq in 64 bits, reduced to a fraction of a turn there (the product of a position below
// 2^31 and a frequency of 1 is off by 2^-52 of itself, below 1e-7 turns, where fp32 would be off by whole turns) and handed to sincospif in fp32.
#pragma once
#include "sh_elem.cuh"
#include "sh_window.h"

namespace shrope {

using shelem::Vec;

// Element offsets of this lane's two runs of 8 elements.
template <int D>
__device__ __forceinline__ void runs(const RopeParams &r, int p, int &e0, int &e1) {
    const bool rotates = p < r.rot / 16;
    if (rotates && !r.adjacent) {
        e0 = 8 * p;
        e1 = r.rot / 2 + 8 * p;
    } else {
        e0 = 16 * p;
        e1 = 16 * p + 8;
    }
}

__device__ __forceinline__ int axis_of(const RopeParams &r, int pair) {
    if (r.spread) {
        const int a = pair % 3;
        return (a == 1 && pair < r.spread_h) || (a == 2 && pair < r.spread_w) ? a : 0;
    }
    return pair < r.sec0 ? 0 : (pair < r.sec01 ? 1 : 2);
}

// cos and sin of `pair` for token `t`.
__device__ __forceinline__ void turn(const RopeParams &r, long long t, int pair, float &c, float &s) {
    const int pos = r.positions[axis_of(r, pair) * r.axis_stride + t];
    const double turns = (double)pos * (double)r.inv_freq[pair] * 0.15915494309189533577;      // 1 / (2 pi)
    const float frac = (float)(turns - rint(turns));                                           // in [-1/2, 1/2]
    sincospif(2.f * frac, &s, &c);
}

// This lane's 8 pairs of token t; the warp's other rows need the same values, so every lane works out 8 / ROWS of them
// and the rest comes by shuffle (all 32 lanes call this).
template <int D>
__device__ __forceinline__ void turns_of_lane(const RopeParams &r, long long t, int lane, float (&c)[8], float (&s)[8]) {
    constexpr int LPR = D / 16, ROWS = 32 / LPR, EACH = 8 / ROWS;      // lanes per row, rows of a warp, pairs per lane
    const int p = lane % LPR, g = lane / LPR;
    float mc[EACH], ms[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        mc[i] = 1.f; ms[i] = 0.f;
        if (p < r.rot / 16) turn(r, t, 8 * p + g * EACH + i, mc[i], ms[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        c[i] = __shfl_sync(0xffffffffu, mc[i % EACH], p + (i / EACH) * LPR);
        s[i] = __shfl_sync(0xffffffffu, ms[i % EACH], p + (i / EACH) * LPR);
    }
}

// x[0..7], x[8..15]: the lane's two runs.  Normalise this row if `norm` (w: the weights of the same elements) and rotate.
// `any` is the same for the whole warp: some row of it is normalised (all lanes then take part in the sums).
template <int D>
__device__ __forceinline__ void apply(const RopeParams &r, int p, bool any, bool norm, const float (&w)[16], const float (&c)[8],
                                      const float (&s)[8], float (&x)[16]) {
    if (any) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int o = D / 32; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float inv = 1.f / sqrtf(ss * (1.f / D) + r.eps);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = norm ? x[i] * inv * w[i] : x[i];
    }
    if (p >= r.rot / 16) return;
    if (r.adjacent) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = a * c[i] - b * s[i];
            x[2 * i + 1] = a * s[i] + b * c[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = x[i], b = x[8 + i];
            x[i] = a * c[i] - b * s[i];
            x[8 + i] = a * s[i] + b * c[i];
        }
    }
}

// The lane's 16 elements of the row at `row` (a row of the element type T), and back.
template <typename T>
__device__ __forceinline__ void load16(const char *row, int e0, int e1, float (&x)[16]) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int i = 0; i < 8; i += N) {
        Vec<T>::unpack(*reinterpret_cast<const uint4 *>(row + (e0 + i) * (int)sizeof(T)), x + i);
        Vec<T>::unpack(*reinterpret_cast<const uint4 *>(row + (e1 + i) * (int)sizeof(T)), x + 8 + i);
    }
}
template <typename T>
__device__ __forceinline__ void store16(char *row, int e0, int e1, const float (&x)[16]) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int i = 0; i < 8; i += N) {
        *reinterpret_cast<uint4 *>(row + (e0 + i) * (int)sizeof(T)) = Vec<T>::pack(x + i);
        *reinterpret_cast<uint4 *>(row + (e1 + i) * (int)sizeof(T)) = Vec<T>::pack(x + 8 + i);
    }
}

}  // namespace shrope
