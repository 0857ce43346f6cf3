// Checks of arguments and parameter blocks that the interface files share (host only).
#pragma once
#include <algorithm>
#include <cmath>
#include <utility>

#include "sh_window.h"

namespace shargs {

constexpr long long MAX_STRIDE = 1ll << 38;      // elements; a tensor map holds byte strides below 2^40
constexpr int MAX_POS = 1 << 30;                 // positions, and window + sinks

inline bool aligned16(const void *p) { return p && ((uintptr_t)p & 15) == 0; }
inline int elem_size(int dtype) { return dtype == SH_F32 ? 4 : 2; }
inline bool good_type(int dtype, int D) { return (dtype == SH_F32 || dtype == SH_F16 || dtype == SH_BF16) && (D == 64 || D == 128); }
inline bool good_stride(long long s, int D, int es) { return s >= D && s < MAX_STRIDE && (s * es) % 16 == 0; }

// Rows of a tensor that is read: positive strides along every dimension that is walked.
inline bool rows_in(const sh_rows *r, int tokens, int heads, int D, int es) {
    return r && aligned16(r->data) && (tokens <= 1 || good_stride(r->token_stride, D, es)) &&
           (heads <= 1 || good_stride(r->head_stride, D, es));
}
// Dimensions of a tensor that is written may not share elements: each one steps over all that the smaller ones span.
// (Sorted by stride; dimensions of length one span nothing.)
inline bool disjoint(long long stride0, long long n0, long long stride1, long long n1, long long stride2, long long n2, int D) {
    std::pair<long long, long long> d[3] = {{stride0, n0}, {stride1, n1}, {stride2, n2}};
    std::sort(d, d + 3);
    long long span = D;
    for (const auto &x : d) {
        if (x.second <= 1) continue;
        if (x.first < span) return false;
        if (x.second - 1 > (1ll << 60) / x.first) return false;
        span += (x.second - 1) * x.first;
    }
    return true;
}
inline bool rows_out(const sh_rows *r, int tokens, int heads, int D, int es) {
    return rows_in(r, tokens, heads, D, es) && disjoint(r->token_stride, tokens, r->head_stride, heads, 0, 1, D);
}
// A dimension of length one is never stepped over: its stride is replaced, so that no kernel or tensor map sees a stray value.
inline WinRows rows(const sh_rows *r, int tokens, int heads, int D, int es) {
    return WinRows{static_cast<char *>(r->data), (tokens > 1 ? r->token_stride : D) * es, (heads > 1 ? r->head_stride : D) * es};
}

inline bool good_window(const sh_window *w) {
    if (!w || !good_type(w->dtype, w->head_dim) || w->kv_heads < 1 || w->q_heads < 1 || w->q_heads % w->kv_heads) return false;
    if (w->kv_heads > 65535) return false;
    if (w->window < 1 || w->sinks < 0 || (long long)w->window + w->sinks >= MAX_POS) return false;
    return w->scale == 0.0 || (w->scale > 1e-30 && w->scale < 1e30);      // (NaN: no; fp32 has to hold it)
}
inline bool good_cache(const sh_window_cache *c, const sh_window *w, int sequences) {
    const int D = w->head_dim, es = elem_size(w->dtype);
    const long long slots = (long long)w->window + w->sinks;
    return c && aligned16(c->k) && aligned16(c->v) && (slots <= 1 || good_stride(c->slot_stride, D, es)) &&
           (w->kv_heads <= 1 || good_stride(c->head_stride, D, es)) && (sequences <= 1 || good_stride(c->sequence_stride, D, es)) &&
           disjoint(c->slot_stride, slots, c->head_stride, w->kv_heads, c->sequence_stride, sequences, D);
}
inline bool good_ints(const int32_t *p) { return p && ((uintptr_t)p & 3) == 0; }

inline void fill_window(WindowParams &p, const sh_window *w, const sh_window_cache *c, int sequences) {
    const int D = w->head_dim, es = elem_size(w->dtype);
    p.hq = w->q_heads; p.hk = w->kv_heads; p.g = w->q_heads / w->kv_heads;
    p.window = w->window; p.sinks = w->sinks;
    p.slots = w->window + w->sinks;
    const double scale = w->scale > 0.0 ? w->scale : 1.0 / std::sqrt((double)D);
    p.scale_log2e = (float)(scale * 1.4426950408889634074);
    p.sequences = sequences;
    if (c) {
        p.kc = static_cast<char *>(c->k); p.vc = static_cast<char *>(c->v);
        p.css = (sequences > 1 ? c->sequence_stride : D) * es;
        p.chs = (w->kv_heads > 1 ? c->head_stride : D) * es;
        p.cls = (w->window + w->sinks > 1 ? c->slot_stride : D) * es;
    }
}
inline int done(cudaError_t e) { return e == cudaSuccess ? SH_OK : SH_ECUDA; }


}  // namespace shargs
