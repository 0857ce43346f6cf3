// Norm and rotation of one row of head_dim elements, shared by D / 16 lanes: the device side of sh_rope.
//
// Lane p of a row's D / 16 lanes holds 16 elements.  While p < rot / 16 they are pairs 8p .. 8p + 7: both members of a
// pair are in one lane, in either pairing ((i, i + rot/2): the pieces at 8p and rot/2 + 8p; (2i, 2i + 1): the 16 elements
// from 16p on), so the rotation needs no exchange.  The lanes behind hold 16 consecutive elements that only get normalised.
// The angle is position * inv_freq in 64 bits, reduced to a fraction of a turn there (the product of a position below
// 2^31 and a frequency of 1 is off by 2^-52 of itself, below 1e-7 turns, where fp32 would be off by whole turns) and handed to sincospif in fp32.
#pragma once
#include "sh_elem.cuh"
#include "sh_pairs.cuh"
#include "sh_window.h"

namespace shrope {

using shelem::Vec;
using namespace shpair;

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

// Sines and cosines arranged for packed pairs of fp32 (Blackwell's two-wide multiply-add): for pairs (i, i + rot/2) two
// neighbouring i share a register pair, for (2i, 2i + 1) the two members of a pair do.
template <bool ADJ> struct Turns {
    static constexpr int N = ADJ ? 8 : 4;
    uint64_t c[N], s[N], n[N];            // adjacent: n = (-sin, sin), s unused; else n = -s
    __device__ __forceinline__ void set(const float (&cc)[8], const float (&ss)[8]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (ADJ) {
                c[i] = f2(cc[i], cc[i]);
                n[i] = f2(-ss[i], ss[i]);
            } else {
                c[i] = f2(cc[2 * i], cc[2 * i + 1]);
                s[i] = f2(ss[2 * i], ss[2 * i + 1]);
                n[i] = f2(-ss[2 * i], -ss[2 * i + 1]);
            }
        }
    }
};

// x: the lane's 16 elements as 8 pairs (4 of each run).  With `any` (the same for the whole warp) the row is normalised: every element
// times its weight w and the row's 1 / sqrt(mean + eps); a row of such a warp that is not (`norm` false, w = 1) keeps its values.
template <int D, bool ADJ>
__device__ __forceinline__ void apply(const RopeParams &r, int p, bool any, bool norm, const uint64_t (&w)[8], const Turns<ADJ> &turn, uint64_t (&x)[8]) {
    if (any) {
        uint64_t ss = mul2(x[0], x[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) ss = fma2(x[i], x[i], ss);
        float lo, hi;
        un2(ss, lo, hi);
        lo += hi;
#pragma unroll
        for (int o = D / 32; o; o >>= 1) lo += __shfl_xor_sync(0xffffffffu, lo, o);
        const float inv = norm ? 1.f / sqrtf(lo * (1.f / D) + r.eps) : 1.f;
        const uint64_t inv2 = f2(inv, inv);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = mul2(mul2(x[i], inv2), w[i]);
    }
    if (p >= r.rot / 16) return;
    if constexpr (ADJ) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float a, b;
            un2(x[i], a, b);
            x[i] = fma2(f2(b, a), turn.n[i], mul2(x[i], turn.c[i]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t a = x[i], b = x[4 + i];
            x[i] = fma2(b, turn.n[i], mul2(a, turn.c[i]));
            x[4 + i] = fma2(b, turn.c[i], mul2(a, turn.s[i]));
        }
    }
}

// The lane's 16 elements of a row: as 16-byte pieces, and as fp32.
template <typename T> struct Raw {
    static constexpr int PIECES = 8 / Vec<T>::N;      // of a run
    uint4 a[2 * PIECES];
};
template <typename T>
__device__ __forceinline__ void load_raw(const char *row, int e0, int e1, Raw<T> &x) {
#pragma unroll
    for (int i = 0; i < Raw<T>::PIECES; ++i) {
        x.a[i] = *reinterpret_cast<const uint4 *>(row + (e0 + i * Vec<T>::N) * (int)sizeof(T));
        x.a[Raw<T>::PIECES + i] = *reinterpret_cast<const uint4 *>(row + (e1 + i * Vec<T>::N) * (int)sizeof(T));
    }
}
template <typename T>
__device__ __forceinline__ void unpack_raw(const Raw<T> &r, uint64_t (&x)[8]) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int i = 0; i < 2 * Raw<T>::PIECES; ++i) {
        float f[N];
        Vec<T>::unpack(r.a[i], f);
#pragma unroll
        for (int e = 0; e < N; e += 2) x[(i * N + e) / 2] = f2(f[e], f[e + 1]);
    }
}
template <typename T>
__device__ __forceinline__ void store16(char *row, int e0, int e1, const uint64_t (&x)[8]) {
    constexpr int N = Vec<T>::N;
    float f[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) un2(x[i], f[2 * i], f[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 8; i += N) {
        *reinterpret_cast<uint4 *>(row + (e0 + i) * (int)sizeof(T)) = Vec<T>::pack(f + i);
        *reinterpret_cast<uint4 *>(row + (e1 + i) * (int)sizeof(T)) = Vec<T>::pack(f + 8 + i);
    }
}

}  // namespace shrope
