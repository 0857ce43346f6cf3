// Device helpers of the window cache kernels: which rows a tile holds and which positions a block of keys has.
#pragma once
#include <math_constants.h>

#include "sh_elem.cuh"
#include "sh_umma.cuh"
#include "sh_window.h"

namespace shwin {

constexpr int MAX_POS = 1 << 30;

// The rows [first, first + count) of the chunk tensors that belong to sequence i (starts that decrease or leave the tensor are
// clamped), and the tokens its cache holds.  An idle sequence (negative length) has no rows.
// MODE: what is attended to (sh_window.h).  Contexts without starts: all tokens share the one there is, or each has its own.
template <int MODE = ATTEND_WINDOW>
__device__ __forceinline__ void sequence_rows(const WindowParams &p, int i, int &first, int &count, int &cached) {
    const int a = MODE == ATTEND_CONTEXT && !p.starts ? (p.sequences == 1 ? 0 : i) : min(max(p.starts[i], 0), p.tokens);
    const int b = MODE == ATTEND_CONTEXT && !p.starts ? (p.sequences == 1 ? p.tokens : i + 1) : min(max(p.starts[i + 1], a), p.tokens);
    cached = p.lengths ? p.lengths[i] : (MODE == ATTEND_CONTEXT ? p.slots : 0);
    first = a;
    count = MODE != ATTEND_CONTEXT && cached < 0 ? 0 : b - a;
    cached = min(max(cached, 0), MODE == ATTEND_CONTEXT ? p.slots : MAX_POS);
    if (MODE == ATTEND_MASS && count > p.fit - cached) count = 0;
}

struct Tile {
    int seq;            // -1: there is no such tile
    int first, count;   // the sequence's rows of the chunk tensors
    int cached;         // tokens in its cache
    long long row0;     // first row of the tile among the sequence's count * g (token, head of the group) rows
};

// The tile-th block of `bm` rows over all sequences.  A row is (token, query head of the group), heads innermost: the heads that
// share a key head sit in one tile and a tile spans few tokens, so few keys.  One warp, all lanes.
template <int MODE = ATTEND_WINDOW>
__device__ __forceinline__ Tile find_tile(const WindowParams &p, long long tile, int bm) {
    const int lane = threadIdx.x & 31;
    Tile r = {-1, 0, 0, 0, 0};
    long long before = 0;
    for (int base = 0; base < p.sequences; base += 32) {
        int first = 0, count = 0, cached = 0;
        if (base + lane < p.sequences) sequence_rows<MODE>(p, base + lane, first, count, cached);
        const long long mine = ((long long)count * p.g + bm - 1) / bm;
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
            r.row0 = (tile - before - __shfl_sync(0xffffffffu, upto - mine, l)) * bm;
            return r;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    return r;
}

// Does token `tok` belong to a sequence?  Found by bisection of `starts`; its number and rows come back.
template <int MODE = ATTEND_WINDOW>
__device__ __forceinline__ bool sequence_of(const WindowParams &p, long long tok, int &seq, int &first, int &count, int &cached) {
    int lo = 0, hi = p.sequences;      // the last sequence that starts at or before tok (empty ones before it are passed over)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.starts[mid] <= tok) lo = mid; else hi = mid;
    }
    seq = lo;
    sequence_rows<MODE>(p, lo, first, count, cached);
    return tok >= first && tok < (long long)first + count;
}

// Slot of position p.
__device__ __forceinline__ int slot_of(int pos, int sinks, int window) { return pos < sinks ? pos : sinks + (pos - sinks) % window; }

// Position held by slot s of a cache with `cached` tokens (-1: none).
__device__ __forceinline__ int position_in(int s, int cached, int sinks, int window) {
    if (s < sinks) return s < cached ? s : -1;
    const int c = cached - sinks, j = s - sinks;      // tokens in the ring so far, ring slot
    if (c <= j || j >= window) return -1;
    return s + (c - 1 - j) / window * window;
}

// The slots of one cache: [0, min(sinks, cached)) hold the sinks, [sinks, head) the positions cached - (head - slot), and, once the ring
// has wrapped, [head, sinks + window) the positions cached - window + (slot - head).  Slots from `live` on hold nothing.
struct Ring {
    int cached, sinks, window, live, head;
    bool wrapped;
    __device__ __forceinline__ Ring() {}
    __device__ __forceinline__ Ring(int cached_, int sinks_, int window_) : cached(cached_), sinks(sinks_), window(window_) {
        live = min(cached, sinks + window);
        wrapped = cached > sinks + window;
        head = wrapped ? sinks + (cached - sinks) % window : cached;
    }
    // do the slots [x, y) hold a sink, or a position from `oldest` on?
    __device__ __forceinline__ bool any(int x, int y, int oldest) const {
        y = min(y, live);
        if (x < min(sinks, cached)) return true;
        if (wrapped && y > head && cached - window + (y - 1 - head) >= oldest) return true;
        return x < head && y > sinks && cached - head + min(y, head) - 1 >= oldest;
    }
};

// The end of a row: its unnormalised output times `own`, plus the prior's row times `other` (0: there is none, or it has seen nothing, and
// its row does not matter).  `total`: the log (base 2) of the sum of exponentials that this is divided by.  `lost`: the prior's log is NaN or
// infinite, and with it the whole row NaN.
struct Close {
    float own, other, total;
    bool lost;
};
// `base` + log2(L) is the log of the row's own sum.
template <int MODE>
__device__ __forceinline__ Close close_row(const WindowParams &p, long long token, int h, float base, float L) {
    Close r = {1.f / L, 0.f, 0.f, false};
    if (MODE == ATTEND_MASS && p.prior_lse) {
        const float pl = p.prior_lse[token * p.hq + h] * 1.4426950408889634f;
        if (pl != -CUDART_INF_F) {
            const float top = fmaxf(base, pl), f = shumma::ex2_approx(base - top), g = shumma::ex2_approx(pl - top);
            L = fmaf(L, f, g);
            r.own = f / L;
            r.other = g / L;
            r.lost = !(pl < CUDART_INF_F);
            base = top;
        }
    }
    if (MODE != ATTEND_WINDOW) r.total = base + log2f(L);
    return r;
}
// N elements of the prior's row, from d on.
template <typename T, int N>
__device__ __forceinline__ void prior_row(const WindowParams &p, long long token, int h, int d, float (&y)[N]) {
    const char *row = p.prior.p + token * p.prior.ts + h * p.prior.hs;
    if (p.prior_f32) {
#pragma unroll
        for (int i = 0; i < N; i += 4) shelem::Vec<float>::unpack(*reinterpret_cast<const uint4 *>(row + (d + i) * 4), y + i);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += shelem::Vec<T>::N) shelem::Vec<T>::unpack(*reinterpret_cast<const uint4 *>(row + (d + i) * (int)sizeof(T)), y + i);
    }
}
// N elements of a row of `out`, from d on.
template <typename T, int MODE, int N>
__device__ __forceinline__ void store_row(const WindowParams &p, long long token, int h, int d, const float (&x)[N]) {
    char *row = p.out.p + token * p.out.ts + h * p.out.hs;
    if (MODE == ATTEND_CONTEXT && p.out_f32) {
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<uint4 *>(row + (d + i) * 4) = shelem::Vec<float>::pack(x + i);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += shelem::Vec<T>::N) *reinterpret_cast<uint4 *>(row + (d + i) * (int)sizeof(T)) = shelem::Vec<T>::pack(x + i);
    }
}

}  // namespace shwin
