// Entry points of shared contexts and of the cache with accumulated weights: argument checks and parameter blocks.
#include "sh_args.h"
#include "sh_mass.h"

namespace {

using namespace shargs;

// The window whose calls take the same arguments: as long as the cache, without sinks.
sh_window as_window(const sh_attention *a) { return sh_window{a->dtype, a->head_dim, a->q_heads, a->kv_heads, a->slots, 0, a->scale}; }
bool good_attention(const sh_attention *a) {
    if (!a) return false;
    const sh_window w = as_window(a);
    return good_window(&w) && (long long)a->q_heads < MAX_POS;
}
// K and V that are only read: rows may be visited twice.
bool cache_in(const sh_window_cache *c, int kv_heads, int D, int es, int slots, int sequences) {
    return c && aligned16(c->k) && aligned16(c->v) && (slots <= 1 || good_stride(c->slot_stride, D, es)) &&
           (kv_heads <= 1 || good_stride(c->head_stride, D, es)) && (sequences <= 1 || good_stride(c->sequence_stride, D, es));
}
bool good_records(const sh_records *r, int slots, int heads, int sequences) {
    const auto fine = [](long long s) { return s >= 1 && s < MAX_STRIDE; };
    return r && good_ints(r->positions) && r->mass && ((uintptr_t)r->mass & 3) == 0 && (heads <= 1 || fine(r->head_stride)) &&
           (sequences <= 1 || fine(r->sequence_stride)) && disjoint(r->head_stride, heads, r->sequence_stride, sequences, 0, 1, slots);
}
MassRecords records(const sh_records *r, int heads, int sequences) {
    return MassRecords{r->mass, r->positions, sequences > 1 ? r->sequence_stride : 0, heads > 1 ? r->head_stride : 0};
}
void fill_records(WindowParams &p, const sh_records *r, int sequences) {
    const MassRecords m = records(r, p.hk, sequences);
    p.mass = m.mass; p.held = m.positions; p.rss = m.ss; p.rhs = m.hs;
}
// A prior: rows like the queries, or in fp32, and the logs of their sums, both or neither.
bool good_prior(const sh_rows *r, int dtype, const float *lse, const sh_attention *a, int tokens) {
    if (!r) return lse == nullptr;
    return (dtype == SH_F32 || dtype == a->dtype) && rows_in(r, tokens, a->q_heads, a->head_dim, elem_size(dtype)) && lse && ((uintptr_t)lse & 3) == 0;
}
void fill_prior(WindowParams &p, const sh_rows *r, int dtype, const float *lse, const sh_attention *a, int tokens) {
    if (!r) return;
    p.prior = rows(r, tokens, a->q_heads, a->head_dim, elem_size(dtype));
    p.prior_lse = lse;
    p.prior_f32 = dtype == SH_F32;
}
size_t up(size_t x, size_t to) { return (x + to - 1) / to * to; }
// Scratch of the single-token kernels' parts.  They cost a second launch and are never chosen for units of less than 432 KB: a cluster of 8 is
// done with those first (best_split).  So nothing is asked for there.
size_t step_scratch(const sh_attention *a, int sequences) {
    return (long long)a->slots * 4 * a->head_dim < 432000 ? 0 : sh_window_decode_scratch(sequences, a->kv_heads, a->q_heads / a->kv_heads, a->dtype, a->head_dim);
}
long long score_stride(const sh_attention *a) { return ((long long)a->slots + 15) / 16 * 16; }

}  // namespace

extern "C" {

size_t sh_context_attention_workspace_bytes(const sh_attention *a, int tokens, int contexts, int with_starts) {
    if (!good_attention(a) || tokens < 1 || tokens >= MAX_POS || contexts < 1) return 0;
    const int g = a->q_heads / a->kv_heads;
    if (!with_starts && tokens == contexts) return step_scratch(a, contexts);
    return sh_window_prefill_scratch(tokens, contexts, a->kv_heads, g, a->slots, 0, true, a->dtype, a->head_dim);
}

int sh_context_attention(const sh_attention *a, int tokens, int contexts, const sh_rows *q, const sh_window_cache *context, const int32_t *starts_dev,
                         const int32_t *lengths_dev, const sh_rows *out, int out_dtype, float *lse_dev, int clear_rest, void *workspace_dev, size_t workspace_bytes,
                         void *stream) {
    if (!good_attention(a) || (out_dtype != SH_F32 && out_dtype != a->dtype) || (clear_rest & ~1) || tokens < 0 || tokens >= MAX_POS || contexts < 0) return SH_EINVAL;
    if (!starts_dev && contexts != 1 && contexts != tokens) return SH_EINVAL;
    if (tokens == 0 || (contexts == 0 && !clear_rest)) return SH_OK;      // (without contexts every row belongs to none)
    const int D = a->head_dim, es = elem_size(a->dtype);
    if (!rows_in(q, tokens, a->q_heads, D, es) || !rows_out(out, tokens, a->q_heads, D, elem_size(out_dtype)) ||
        (contexts > 0 && !cache_in(context, a->kv_heads, D, es, a->slots, contexts)) || (starts_dev && !good_ints(starts_dev)) ||
        (lengths_dev && !good_ints(lengths_dev)) || !lse_dev || ((uintptr_t)lse_dev & 3))
        return SH_EINVAL;
    const sh_window w = as_window(a);
    WindowParams p = {};
    fill_window(p, &w, context, contexts);
    p.tokens = tokens;
    p.q = rows(q, tokens, a->q_heads, D, es);
    p.out = rows(out, tokens, a->q_heads, D, elem_size(out_dtype));
    p.out_f32 = out_dtype == SH_F32;
    p.starts = starts_dev; p.lengths = lengths_dev;
    p.lse = lse_dev;
    if (workspace_dev) {
        if (!aligned16(workspace_dev)) return SH_EINVAL;
        const size_t need = sh_context_attention_workspace_bytes(a, tokens, contexts, starts_dev != nullptr);
        if (workspace_bytes < need) return SH_ENOMEM;
        if (need) p.part = static_cast<float *>(workspace_dev);
    }
    if (!starts_dev && tokens == contexts) return done(sh_launch_window_decode(p, a->dtype, D, ATTEND_CONTEXT, (cudaStream_t)stream));
    p.window = MAX_POS;                          // every row of the context is in sight of every token
    if (clear_rest && starts_dev) {
        p.clear_rest = true;
        const cudaError_t e = sh_launch_clear_rest(p, D * elem_size(out_dtype), (cudaStream_t)stream);
        if (e != cudaSuccess || contexts == 0) return done(e);
    }
    return done(a->dtype == SH_F32 ? sh_launch_window_prefill_f32(p, D, ATTEND_CONTEXT, (cudaStream_t)stream)
                                   : sh_launch_window_prefill_umma(p, a->dtype, D, ATTEND_CONTEXT, (cudaStream_t)stream));
}

// The workspaces of the calls below: what their attention needs, then the logs and scores.
size_t sh_mass_prefill_workspace_bytes(const sh_attention *a, int tokens, int sequences) {
    if (!good_attention(a) || tokens < 1 || tokens >= MAX_POS || sequences < 1) return 0;
    const int g = a->q_heads / a->kv_heads;
    // (the columns kernel comes after the attention: they share a place)
    return up(std::max(sh_window_prefill_scratch(tokens, sequences, a->kv_heads, g, a->slots, 0, true, a->dtype, a->head_dim),
                       a->dtype == SH_F32 ? 0 : sh_mass_columns_scratch(tokens, sequences, a->kv_heads, g, a->slots)), 256) +
           up(sizeof(float) * (size_t)tokens * a->q_heads + sizeof(int), 256);
}

int sh_mass_prefill(const sh_attention *a, int tokens, int sequences, const sh_rows *q, const sh_rows *k, const sh_rows *v, const int32_t *starts_dev,
                    const int32_t *lengths_dev, const int32_t *seen_dev, const sh_window_cache *cache, const sh_records *rec, const sh_rows *prior, int prior_dtype,
                    const float *prior_lse_dev, const sh_rows *out, void *workspace_dev, size_t workspace_bytes, void *stream) {
    if (!good_attention(a) || tokens < 0 || tokens >= MAX_POS || sequences < 0) return SH_EINVAL;
    if (tokens == 0 || sequences == 0) return SH_OK;
    const int D = a->head_dim, es = elem_size(a->dtype);
    const sh_window w = as_window(a);
    if (!rows_in(q, tokens, a->q_heads, D, es) || !rows_in(k, tokens, a->kv_heads, D, es) || !rows_in(v, tokens, a->kv_heads, D, es) ||
        !rows_out(out, tokens, a->q_heads, D, es) || !good_prior(prior, prior_dtype, prior_lse_dev, a, tokens) || !good_cache(cache, &w, sequences) ||
        !good_records(rec, a->slots, a->kv_heads, sequences) || !good_ints(starts_dev) || !good_ints(lengths_dev) || !good_ints(seen_dev) ||
        !aligned16(workspace_dev))
        return SH_EINVAL;
    const size_t need = sh_mass_prefill_workspace_bytes(a, tokens, sequences);
    if (workspace_bytes < need) return SH_ENOMEM;
    WindowParams p = {};
    fill_window(p, &w, cache, sequences);
    fill_records(p, rec, sequences);
    p.tokens = tokens;
    p.q = rows(q, tokens, a->q_heads, D, es);
    p.k = rows(k, tokens, a->kv_heads, D, es);
    p.v = rows(v, tokens, a->kv_heads, D, es);
    p.out = rows(out, tokens, a->q_heads, D, es);
    p.starts = starts_dev; p.lengths = lengths_dev; p.seen = seen_dev;
    p.fit = a->slots;
    const size_t lse_bytes = up(sizeof(float) * (size_t)tokens * a->q_heads + sizeof(int), 256);
    if (need > lse_bytes) p.part = static_cast<float *>(workspace_dev);
    p.lse = reinterpret_cast<float *>(static_cast<char *>(workspace_dev) + need - lse_bytes);
    p.taken = reinterpret_cast<int *>(p.lse + (size_t)tokens * a->q_heads);
    fill_prior(p, prior, prior_dtype, prior_lse_dev, a, tokens);
    const cudaStream_t s = (cudaStream_t)stream;
    // the chunk goes into slots that the attention does not look at: the two run side by side
    cudaError_t e = sh_launch_window_append(p, es, D, ATTEND_MASS, s);
    if (e == cudaSuccess) e = a->dtype == SH_F32 ? sh_launch_window_prefill_f32(p, D, ATTEND_MASS, s) : sh_launch_window_prefill_umma(p, a->dtype, D, ATTEND_MASS, s);
    if (e == cudaSuccess) e = a->dtype == SH_F32 ? sh_launch_mass_columns_f32(p, D, s) : sh_launch_mass_columns_umma(p, a->dtype, D, s);
    return done(e);
}

size_t sh_mass_decode_workspace_bytes(const sh_attention *a, int sequences) {
    if (!good_attention(a) || sequences < 1) return 0;
    return up(step_scratch(a, sequences), 256) +
           sizeof(float) * (size_t)sequences * a->q_heads * (score_stride(a) + 1);
}

int sh_mass_decode(const sh_attention *a, int sequences, const sh_rows *q, const sh_rows *k, const sh_rows *v, const int32_t *lengths_dev,
                   const int32_t *seen_dev, const sh_window_cache *cache, const sh_records *rec, const sh_rows *prior, int prior_dtype,
                   const float *prior_lse_dev, const sh_rows *out, void *workspace_dev, size_t workspace_bytes, void *stream) {
    if (!good_attention(a) || sequences < 0) return SH_EINVAL;
    if (sequences == 0) return SH_OK;
    const int D = a->head_dim, es = elem_size(a->dtype);
    const sh_window w = as_window(a);
    if (!rows_in(q, sequences, a->q_heads, D, es) || !rows_in(k, sequences, a->kv_heads, D, es) || !rows_in(v, sequences, a->kv_heads, D, es) ||
        !rows_out(out, sequences, a->q_heads, D, es) || !good_prior(prior, prior_dtype, prior_lse_dev, a, sequences) || !good_cache(cache, &w, sequences) ||
        !good_records(rec, a->slots, a->kv_heads, sequences) || !good_ints(lengths_dev) || !good_ints(seen_dev) || !aligned16(workspace_dev))
        return SH_EINVAL;
    const size_t need = sh_mass_decode_workspace_bytes(a, sequences);
    if (workspace_bytes < need) return SH_ENOMEM;
    WindowParams p = {};
    fill_window(p, &w, cache, sequences);
    fill_records(p, rec, sequences);
    p.tokens = sequences;
    p.q = rows(q, sequences, a->q_heads, D, es);
    p.k = rows(k, sequences, a->kv_heads, D, es);
    p.v = rows(v, sequences, a->kv_heads, D, es);
    p.out = rows(out, sequences, a->q_heads, D, es);
    p.lengths = lengths_dev; p.seen = seen_dev;
    const size_t part = up(step_scratch(a, sequences), 256);
    if (part) p.part = static_cast<float *>(workspace_dev);
    p.score_stride = score_stride(a);
    p.scores = reinterpret_cast<float *>(static_cast<char *>(workspace_dev) + part);
    p.total = p.scores + (size_t)sequences * p.hq * p.score_stride;
    fill_prior(p, prior, prior_dtype, prior_lse_dev, a, sequences);
    return done(sh_launch_window_decode(p, a->dtype, D, ATTEND_MASS, (cudaStream_t)stream));
}

size_t sh_mass_evict_workspace_bytes(const sh_attention *a, int sequences, int keep, int in_place) {
    if (!good_attention(a) || sequences < 1 || keep < 1 || (in_place && keep > a->slots)) return 0;
    return sh_mass_evict_scratch((long long)sequences * a->kv_heads, in_place ? std::min(keep, a->slots - keep) : std::min(keep, a->slots));
}

int sh_mass_evict(const sh_attention *a, int sequences, const int32_t *lengths_dev, const sh_window_cache *cache, const sh_records *rec, int keep, int recent,
                  const sh_window_cache *into, const sh_records *into_rec, int into_slots, int32_t *left_dev, void *workspace_dev, size_t workspace_bytes,
                  void *stream) {
    if (!good_attention(a) || sequences < 0 || keep < 1 || recent < 0 || recent > keep) return SH_EINVAL;
    if ((into == nullptr) != (into_rec == nullptr) || keep > (into ? into_slots : a->slots) || (into && into_slots >= MAX_POS)) return SH_EINVAL;
    if (sequences == 0) return SH_OK;
    const int D = a->head_dim, es = elem_size(a->dtype);
    const sh_window w = as_window(a);
    if (!(into ? cache_in(cache, a->kv_heads, D, es, a->slots, sequences) : good_cache(cache, &w, sequences)) ||
        !good_records(rec, a->slots, a->kv_heads, sequences) || !good_ints(lengths_dev) || !good_ints(left_dev) || !aligned16(workspace_dev))
        return SH_EINVAL;
    if (left_dev != lengths_dev && left_dev < lengths_dev + sequences && lengths_dev < left_dev + sequences) return SH_EINVAL;
    EvictParams p = {};
    WindowParams from = {}, to = {};
    fill_window(from, &w, cache, sequences);
    p.rec = p.out = records(rec, a->kv_heads, sequences);
    to = from;
    if (into) {
        sh_window w2 = w;
        w2.window = into_slots;
        if (!good_cache(into, &w2, sequences) || !good_records(into_rec, into_slots, a->kv_heads, sequences) || into->k == cache->k || into->v == cache->v ||
            into_rec->mass == rec->mass || into_rec->positions == rec->positions)
            return SH_EINVAL;
        fill_window(to, &w2, into, sequences);
        p.out = records(into_rec, a->kv_heads, sequences);
    }
    const size_t need = sh_mass_evict_workspace_bytes(a, sequences, keep, into == nullptr);
    if (workspace_bytes < need) return SH_ENOMEM;
    p.k = from.kc; p.v = from.vc; p.ss = from.css; p.hs = from.chs; p.ls = from.cls;
    p.ko = to.kc; p.vo = to.vc; p.oss = to.css; p.ohs = to.chs; p.ols = to.cls;
    p.lengths = lengths_dev; p.left = left_dev;
    p.sequences = sequences; p.heads = a->kv_heads; p.slots = a->slots;
    p.keep = keep; p.recent = recent;
    p.row_bytes = D * es;
    p.in_place = into == nullptr;
    p.most = p.in_place ? std::min(keep, a->slots - keep) : std::min(keep, a->slots);
    p.moves = static_cast<int2 *>(workspace_dev);
    p.count = reinterpret_cast<int *>(p.moves + (size_t)sequences * a->kv_heads * p.most);
    return done(sh_launch_mass_evict(p, (cudaStream_t)stream));
}

}  // extern "C"
