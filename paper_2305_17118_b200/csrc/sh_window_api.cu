// Entry points of the query/key preparation and of the window cache: argument checks and parameter blocks.
#include <algorithm>
#include <cmath>
#include <utility>

#include "sh_window.h"

namespace {

constexpr long long MAX_STRIDE = 1ll << 38;      // elements; a tensor map holds byte strides below 2^40
constexpr int MAX_POS = 1 << 30;                 // positions, and window + sinks

bool aligned16(const void *p) { return p && ((uintptr_t)p & 15) == 0; }
int elem_size(int dtype) { return dtype == SH_F32 ? 4 : 2; }
bool good_type(int dtype, int D) { return (dtype == SH_F32 || dtype == SH_F16 || dtype == SH_BF16) && (D == 64 || D == 128); }
bool good_stride(long long s, int D, int es) { return s >= D && s < MAX_STRIDE && (s * es) % 16 == 0; }

// Rows of a tensor that is read: positive strides along every dimension that is walked.
bool rows_in(const sh_rows *r, int tokens, int heads, int D, int es) {
    return r && aligned16(r->data) && (tokens <= 1 || good_stride(r->token_stride, D, es)) &&
           (heads <= 1 || good_stride(r->head_stride, D, es));
}
// Dimensions of a tensor that is written may not share elements: each one steps over all that the smaller ones span.
// (Sorted by stride; dimensions of length one span nothing.)
bool disjoint(long long stride0, long long n0, long long stride1, long long n1, long long stride2, long long n2, int D) {
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
bool rows_out(const sh_rows *r, int tokens, int heads, int D, int es) {
    return rows_in(r, tokens, heads, D, es) && disjoint(r->token_stride, tokens, r->head_stride, heads, 0, 1, D);
}
// A dimension of length one is never stepped over: its stride is replaced, so that no kernel or tensor map sees a stray value.
WinRows rows(const sh_rows *r, int tokens, int heads, int D, int es) {
    return WinRows{static_cast<char *>(r->data), (tokens > 1 ? r->token_stride : D) * es, (heads > 1 ? r->head_stride : D) * es};
}

bool good_rope(const sh_rope *r) {
    if (!r || !good_type(r->dtype, r->head_dim)) return false;
    if (r->rot_dim < 0 || r->rot_dim > r->head_dim || r->rot_dim % 16 || r->axes < 1 || r->axes > 3) return false;
    if ((r->spread | r->adjacent_pairs) & ~1) return false;
    if (r->spread && r->axes != 3) return false;
    long long sum = 0;
    for (int a = 0; a < r->axes; ++a) {
        if (r->sections[a] < 0) return false;
        sum += r->sections[a];
    }
    if (sum != r->rot_dim / 2) return false;
    if (!(r->eps >= 0.f) || !std::isfinite(r->eps)) return false;
    if (r->rot_dim && (!r->inv_freq_dev || ((uintptr_t)r->inv_freq_dev & 3))) return false;
    if ((r->q_weight_dev && !aligned16(r->q_weight_dev)) || (r->k_weight_dev && !aligned16(r->k_weight_dev))) return false;
    return true;
}
void fill_rope(RopeParams &p, const sh_rope *r, const int32_t *positions, long long axis_stride) {
    p.positions = positions; p.axis_stride = axis_stride;
    p.inv_freq = r->inv_freq_dev; p.qw = r->q_weight_dev; p.kw = r->k_weight_dev;
    p.rot = r->rot_dim; p.axes = r->axes;
    p.sec0 = r->sections[0]; p.sec01 = r->axes > 1 ? r->sections[0] + r->sections[1] : r->sections[0];
    p.spread = r->spread; p.adjacent = r->adjacent_pairs;
    p.spread_h = r->spread ? 3 * r->sections[1] : 0;
    p.spread_w = r->spread ? 3 * r->sections[2] : 0;
    p.eps = r->eps;
}
bool good_positions(const int32_t *pos, long long axis_stride, int axes) {
    return pos && ((uintptr_t)pos & 3) == 0 && (axes == 1 || (axis_stride >= 0 && axis_stride < MAX_STRIDE));
}

bool good_window(const sh_window *w) {
    if (!w || !good_type(w->dtype, w->head_dim) || w->kv_heads < 1 || w->q_heads < 1 || w->q_heads % w->kv_heads) return false;
    if (w->kv_heads > 65535) return false;
    if (w->window < 1 || w->sinks < 0 || (long long)w->window + w->sinks >= MAX_POS) return false;
    return w->scale == 0.0 || (w->scale > 1e-30 && w->scale < 1e30);      // (NaN: no; fp32 has to hold it)
}
bool good_cache(const sh_window_cache *c, const sh_window *w, int sequences) {
    const int D = w->head_dim, es = elem_size(w->dtype);
    const long long slots = (long long)w->window + w->sinks;
    return c && aligned16(c->k) && aligned16(c->v) && (slots <= 1 || good_stride(c->slot_stride, D, es)) &&
           (w->kv_heads <= 1 || good_stride(c->head_stride, D, es)) && (sequences <= 1 || good_stride(c->sequence_stride, D, es)) &&
           disjoint(c->slot_stride, slots, c->head_stride, w->kv_heads, c->sequence_stride, sequences, D);
}
bool good_ints(const int32_t *p) { return p && ((uintptr_t)p & 3) == 0; }

void fill_window(WindowParams &p, const sh_window *w, const sh_window_cache *c, int sequences) {
    const int D = w->head_dim, es = elem_size(w->dtype);
    p.hq = w->q_heads; p.hk = w->kv_heads; p.g = w->q_heads / w->kv_heads;
    p.window = w->window; p.sinks = w->sinks;
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
int done(cudaError_t e) { return e == cudaSuccess ? SH_OK : SH_ECUDA; }

}  // namespace

cudaError_t sh_device_sms(int *dev, int *sms) {
    static std::atomic<int> known[ShKernelSetup::DEVICES];
    cudaError_t e = cudaGetDevice(dev);
    if (e != cudaSuccess) return e;
    const bool kept = *dev < ShKernelSetup::DEVICES;
    *sms = kept ? known[*dev].load(std::memory_order_relaxed) : 0;
    if (*sms == 0) {
        e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev);
        if (e == cudaSuccess && kept) known[*dev].store(*sms, std::memory_order_relaxed);
    }
    return e;
}

extern "C" {

int sh_qk_norm_rope(const sh_rope *rope, int tokens, int q_heads, int k_heads, const sh_rows *q, const sh_rows *k, const int32_t *positions_dev,
                    long long axis_stride, const sh_rows *q_out, const sh_rows *k_out, void *stream) {
    if (!good_rope(rope) || tokens < 0 || q_heads < 1 || k_heads < 0) return SH_EINVAL;
    if ((k == nullptr) != (k_out == nullptr) || (k == nullptr) != (k_heads == 0)) return SH_EINVAL;
    if (tokens == 0) return SH_OK;
    const int D = rope->head_dim, es = elem_size(rope->dtype);
    if (!rows_in(q, tokens, q_heads, D, es) || !rows_out(q_out, tokens, q_heads, D, es)) return SH_EINVAL;
    if (k && (!rows_in(k, tokens, k_heads, D, es) || !rows_out(k_out, tokens, k_heads, D, es))) return SH_EINVAL;
    if (rope->rot_dim && !good_positions(positions_dev, axis_stride, rope->axes)) return SH_EINVAL;
    RopeParams p = {};
    fill_rope(p, rope, positions_dev, axis_stride);
    p.tokens = tokens; p.q_heads = q_heads; p.k_heads = k_heads;
    p.q = rows(q, tokens, q_heads, D, es);
    p.qo = rows(q_out, tokens, q_heads, D, es);
    if (k) {
        p.k = rows(k, tokens, k_heads, D, es);
        p.ko = rows(k_out, tokens, k_heads, D, es);
    }
    return done(sh_launch_qk_norm_rope(p, rope->dtype, D, (cudaStream_t)stream));
}

size_t sh_window_prefill_workspace_bytes(const sh_window *w, int tokens, int sequences, int with_cache) {
    if (!good_window(w) || tokens < 1 || tokens >= MAX_POS || sequences < 1) return 0;
    return sh_window_prefill_scratch(tokens, sequences, w->kv_heads, w->q_heads / w->kv_heads, w->window, w->sinks, with_cache != 0, w->dtype, w->head_dim);
}

int sh_window_prefill(const sh_window *w, int tokens, int sequences, const sh_rows *q, const sh_rows *k, const sh_rows *v,
                      const int32_t *starts_dev, const int32_t *lengths_dev, const sh_window_cache *cache, const sh_rows *out, void *workspace_dev,
                      size_t workspace_bytes, void *stream) {
    if (!good_window(w) || tokens < 0 || tokens >= MAX_POS || sequences < 0 || (cache == nullptr) != (lengths_dev == nullptr)) return SH_EINVAL;
    if (tokens == 0 || sequences == 0) return SH_OK;
    const int D = w->head_dim, es = elem_size(w->dtype);
    if (!rows_in(q, tokens, w->q_heads, D, es) || !rows_in(k, tokens, w->kv_heads, D, es) || !rows_in(v, tokens, w->kv_heads, D, es) ||
        !rows_out(out, tokens, w->q_heads, D, es) || !good_ints(starts_dev))
        return SH_EINVAL;
    if (cache && (!good_cache(cache, w, sequences) || !good_ints(lengths_dev))) return SH_EINVAL;
    WindowParams p = {};
    fill_window(p, w, cache, sequences);
    p.tokens = tokens;
    p.q = rows(q, tokens, w->q_heads, D, es);
    p.k = rows(k, tokens, w->kv_heads, D, es);
    p.v = rows(v, tokens, w->kv_heads, D, es);
    p.out = rows(out, tokens, w->q_heads, D, es);
    p.starts = starts_dev; p.lengths = lengths_dev;
    if (workspace_dev) {
        if (!aligned16(workspace_dev)) return SH_EINVAL;
        const size_t need = sh_window_prefill_workspace_bytes(w, tokens, sequences, cache != nullptr);
        if (workspace_bytes < need) return SH_ENOMEM;
        if (need) p.part = static_cast<float *>(workspace_dev);
    }
    return done(w->dtype == SH_F32 ? sh_launch_window_prefill_f32(p, D, (cudaStream_t)stream)
                                   : sh_launch_window_prefill_umma(p, w->dtype, D, (cudaStream_t)stream));
}

int sh_window_append(const sh_window *w, int tokens, int sequences, const sh_rows *k, const sh_rows *v, const int32_t *starts_dev,
                     const int32_t *lengths_dev, const sh_window_cache *cache, void *stream) {
    if (!good_window(w) || tokens < 0 || tokens >= MAX_POS || sequences < 0) return SH_EINVAL;
    if (tokens == 0 || sequences == 0) return SH_OK;
    const int D = w->head_dim, es = elem_size(w->dtype);
    if (!rows_in(k, tokens, w->kv_heads, D, es) || !rows_in(v, tokens, w->kv_heads, D, es) || !good_cache(cache, w, sequences) ||
        !good_ints(starts_dev) || !good_ints(lengths_dev))
        return SH_EINVAL;
    WindowParams p = {};
    fill_window(p, w, cache, sequences);
    p.tokens = tokens;
    p.k = rows(k, tokens, w->kv_heads, D, es);
    p.v = rows(v, tokens, w->kv_heads, D, es);
    p.starts = starts_dev; p.lengths = lengths_dev;
    return done(sh_launch_window_append(p, es, D, (cudaStream_t)stream));
}

size_t sh_window_decode_workspace_bytes(const sh_window *w, int sequences) {
    return good_window(w) && sequences > 0 ? sh_window_decode_scratch(sequences, w->kv_heads, w->q_heads / w->kv_heads, w->dtype, w->head_dim) : 0;
}

int sh_window_decode(const sh_window *w, int sequences, const sh_rows *q, const sh_rows *k, const sh_rows *v, const int32_t *lengths_dev,
                     const sh_window_cache *cache, const sh_rope *rope, const int32_t *positions_dev, long long axis_stride,
                     const sh_rows *out, void *workspace_dev, size_t workspace_bytes, void *stream) {
    if (!good_window(w) || sequences < 0) return SH_EINVAL;
    if (rope && (!good_rope(rope) || rope->dtype != w->dtype || rope->head_dim != w->head_dim)) return SH_EINVAL;
    if (rope && (positions_dev ? !good_positions(positions_dev, axis_stride, rope->axes) : rope->axes != 1)) return SH_EINVAL;
    if (!rope && positions_dev) return SH_EINVAL;
    if (sequences == 0) return SH_OK;
    const int D = w->head_dim, es = elem_size(w->dtype);
    if (!rows_in(q, sequences, w->q_heads, D, es) || !rows_in(k, sequences, w->kv_heads, D, es) || !rows_in(v, sequences, w->kv_heads, D, es) ||
        !rows_out(out, sequences, w->q_heads, D, es) || !good_cache(cache, w, sequences) || !good_ints(lengths_dev))
        return SH_EINVAL;
    WindowParams p = {};
    fill_window(p, w, cache, sequences);
    p.tokens = sequences;
    p.q = rows(q, sequences, w->q_heads, D, es);
    p.k = rows(k, sequences, w->kv_heads, D, es);
    p.v = rows(v, sequences, w->kv_heads, D, es);
    p.out = rows(out, sequences, w->q_heads, D, es);
    p.lengths = lengths_dev;
    p.with_rope = rope != nullptr;
    if (workspace_dev) {
        if (!aligned16(workspace_dev)) return SH_EINVAL;
        const size_t need = sh_window_decode_scratch(sequences, p.hk, p.g, w->dtype, D);
        if (workspace_bytes < need) return SH_ENOMEM;
        if (need) p.part = static_cast<float *>(workspace_dev);
    }
    if (rope) fill_rope(p.rope, rope, positions_dev ? positions_dev : lengths_dev, axis_stride);
    return done(sh_launch_window_decode(p, w->dtype, D, (cudaStream_t)stream));
}

int sh_window_status(void *stream) {
    int code = 0;
    if (sh_window_error_take(&code, (cudaStream_t)stream) != cudaSuccess) return SH_ECUDA;
    return code ? SH_EDEVICE : SH_OK;
}

}  // extern "C"
