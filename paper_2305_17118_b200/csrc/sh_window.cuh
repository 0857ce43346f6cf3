// Device helpers of the window cache kernels: which rows a tile holds and which positions a block of keys has.
#pragma once
#include "sh_window.h"

namespace shwin {

constexpr int MAX_POS = 1 << 30;

// The rows [first, first + count) of the chunk tensors that belong to sequence i (starts that decrease or leave the tensor are
// clamped), and the tokens its cache holds.  An idle sequence (negative length) has no rows.
__device__ __forceinline__ void sequence_rows(const WindowParams &p, int i, int &first, int &count, int &cached) {
    const int a = min(max(p.starts[i], 0), p.tokens);
    const int b = min(max(p.starts[i + 1], a), p.tokens);
    cached = p.lengths ? p.lengths[i] : 0;
    first = a;
    count = cached < 0 ? 0 : b - a;
    cached = min(max(cached, 0), MAX_POS);
}

struct Tile {
    int seq;            // -1: there is no such tile
    int first, count;   // the sequence's rows of the chunk tensors
    int cached;         // tokens in its cache
    long long row0;     // first row of the tile among the sequence's count * g (token, head of the group) rows
};

// The tile-th block of `bm` rows over all sequences.  A row is (token, query head of the group), heads innermost: the heads that
// share a key head sit in one tile and a tile spans few tokens, so few keys.  One warp, all lanes.
__device__ __forceinline__ Tile find_tile(const WindowParams &p, long long tile, int bm) {
    const int lane = threadIdx.x & 31;
    Tile r = {-1, 0, 0, 0, 0};
    long long before = 0;
    for (int base = 0; base < p.sequences; base += 32) {
        int first = 0, count = 0, cached = 0;
        if (base + lane < p.sequences) sequence_rows(p, base + lane, first, count, cached);
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

}  // namespace shwin
