// sh_window_decode: one token per sequence over the window cache.  First the kernel for fp32 rows, on CUDA cores; the one for 16-bit
// rows follows below, and what they have in common is said here.
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

#include <algorithm>
#include <type_traits>

#include "sh_mass.h"
#include "sh_rope.cuh"
#include "sh_umma.cuh"
#include "sh_window.cuh"
#include "sh_window_split.h"

namespace cg = cooperative_groups;

namespace {

using shelem::Vec;
using shumma::ex2_approx;
using namespace shwin;

constexpr int WARPS = 8, NT = WARPS * 32;
constexpr int R = 2;                 // rows in flight per group of eight lanes
constexpr int BLOCK = 4 * R;         // rows of a warp per pass

// q rows (fp32) and (KV) the new token's key and value (as the cache holds them) into shared memory, prepared by `rope` if there is one.
template <typename T, int D, int WARPS, bool KV, bool ADJ>
__device__ __forceinline__ void stage_rows(const WindowParams &p, int seq, int kvh, int h0, int nq, float qscale, float *qs, float *ks, float *vs) {
    constexpr int LPR = D / 16, ROWS = 32 / LPR;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pl = lane % LPR, sub = lane / LPR;
    // rows: the nq queries, the key, the value
    const int rows = KV ? nq + 2 : nq;
    if (warp * ROWS >= rows) return;
    shrope::Turns<ADJ> turn;
    int e0 = 16 * pl, e1 = 16 * pl + 8;
    if (p.with_rope) {
        float c[8], s[8];
        shrope::runs<D>(p.rope, pl, e0, e1);
        shrope::turns_of_lane<D>(p.rope, seq, lane, c, s);
        turn.set(c, s);
    }
    for (int base = warp * ROWS; base < rows; base += WARPS * ROWS) {
        const int row = base + sub;
        const bool is_q = row < nq, is_k = row == nq, live = row < rows;
        const char *src = is_q ? p.q.p + seq * p.q.ts + (h0 + row) * p.q.hs
                               : (is_k ? p.k.p + seq * p.k.ts + kvh * p.k.hs : p.v.p + seq * p.v.ts + kvh * p.v.hs);
        shrope::Raw<T> raw = {};
        if (live) shrope::load_raw<T>(src, e0, e1, raw);
        uint64_t x[8];
        shrope::unpack_raw<T>(raw, x);
        if (p.with_rope) {
            const void *weight = is_q ? p.rope.qw : (is_k ? p.rope.kw : nullptr);
            uint64_t w[8], y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) { w[i] = shpair::f2(1.f, 1.f); y[i] = x[i]; }
            if (weight) {
                shrope::Raw<T> wr;
                shrope::load_raw<T>(static_cast<const char *>(weight), e0, e1, wr);
                shrope::unpack_raw<T>(wr, w);
            }
            shrope::apply<D, ADJ>(p.rope, pl, p.rope.qw || p.rope.kw, weight != nullptr, w, turn, y);
            if (is_q || is_k) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = y[i];
            }
        }
        if (live) {
            float f[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) shpair::un2(x[i], f[2 * i], f[2 * i + 1]);
            if (is_k) {      // the row as it will be read back
#pragma unroll
                for (int i = 0; i < 16; i += Vec<T>::N) Vec<T>::unpack(Vec<T>::pack(f + i), f + i);
            }
            float *dst = is_q ? qs + row * D : (is_k ? ks : vs);
            const float m = is_q ? qscale : 1.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) { dst[e0 + i] = f[i] * m; dst[e1 + i] = f[8 + i] * m; }
        }
    }
}
template <typename T, int D, int WARPS, int MODE>
__device__ __forceinline__ void stage_token(const WindowParams &p, int seq, int kvh, int h0, int nq, float qscale, float *qs, float *ks, float *vs) {
    if (MODE == ATTEND_WINDOW && p.with_rope && p.rope.adjacent) stage_rows<T, D, WARPS, true, true>(p, seq, kvh, h0, nq, qscale, qs, ks, vs);
    else stage_rows<T, D, WARPS, MODE != ATTEND_CONTEXT, false>(p, seq, kvh, h0, nq, qscale, qs, ks, vs);
}

// Rows that a sequence holds before the step (below zero: it takes no part).
template <int MODE>
__device__ __forceinline__ int rows_before(const WindowParams &p, int seq) {
    if (MODE == ATTEND_CONTEXT) return p.lengths ? min(max(p.lengths[seq], 0), p.slots) : p.slots;
    const int t = min(p.lengths[seq], MAX_POS);
    return MODE == ATTEND_MASS && t >= p.slots ? -1 : t;      // (a full cache has no place for the token)
}

// The last step for N elements of a row, from d on: `base` + log2(L) is the log of its sum, x its unnormalised output.  Over a cache with
// accumulated weights the row continues from the prior's, if there is one, and leaves that log for the masses in `total`; a context's goes to
// the caller.  Is what the row itself brings not finite?  (Whatever the prior holds, it asks for no second look at the keys.)
template <typename T, int MODE, int N>
__device__ __forceinline__ bool finish(const WindowParams &p, int seq, int h, int d, float base, float L, bool empty, float *total, float (&x)[N]) {
    bool odd = false;
    if constexpr (MODE == ATTEND_WINDOW) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            x[e] /= L;
            odd |= !isfinite(x[e]);
        }
    } else {
        const Close c = close_row<MODE>(p, seq, h, base, L);
        if (MODE == ATTEND_MASS && d == 0) *total = c.total;
        if (MODE == ATTEND_CONTEXT && d == 0) p.lse[(long long)seq * p.hq + h] = empty ? -CUDART_INF_F : 0.69314718055994531f * c.total;
        float y[N] = {};
        if (c.other != 0.f) prior_row<T>(p, seq, h, d, y);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float own = MODE == ATTEND_CONTEXT && empty ? 0.f : x[e] * c.own;
            odd |= !isfinite(own) && !c.lost;
            x[e] = fmaf(y[e], c.other, own);
        }
    }
    return odd;
}

__device__ __forceinline__ float *scores_of(const WindowParams &p, int seq, int h) { return p.scores + ((long long)seq * p.hq + h) * p.score_stride; }
__device__ __forceinline__ float *total_of(const WindowParams &p, int seq, int h) { return p.total + (long long)seq * p.hq + h; }

// The step's weights into the masses, once the unit's scores and totals are there for the whole cluster: a CTA takes the chunks of ROWS slots that
// it attended to, a thread a slot, the heads in their order (as sh_mass_fold_kernel, which does it where a key head has several units or
// its rows were dealt out).
template <int ROWS>
__device__ __forceinline__ void add_weights(const WindowParams &p, int seq, int kvh, int t, int rank, int S) {
    const float *score = scores_of(p, seq, kvh * p.g), *total = total_of(p, seq, kvh * p.g);
    const long long at = seq * p.rss + kvh * p.rhs;
    for (int i = threadIdx.x; ; i += blockDim.x) {
        const int first = (rank + i / ROWS * S) * ROWS, j = first + i % ROWS;
        if (first > t) break;
        if (j > t) continue;
        float sum = 0.f;
        const float old = j < t ? p.mass[at + j] : 0.f;
        for (int h = 0; h < p.g; ++h) sum += ex2_approx(score[h * p.score_stride + j] - total[h]);
        p.mass[at + j] = old + sum;
        if (j == t) p.held[at + j] = p.seen[seq];
    }
}

template <typename T, int D, int GQ, int MODE>
__global__ void __launch_bounds__(NT) sh_window_decode_simt_kernel(const WindowParams p, int qblocks, int) {
    constexpr int N = Vec<T>::N, CH = D / N / 8, EL = CH * N;      // 16-byte pieces and elements of a row per lane
    __shared__ __align__(16) float qs[GQ * D], ks[D], vs[D];
    __shared__ float part[WARPS][GQ][D + 2];
    __shared__ float cta[GQ][D + 2];                                // this CTA's maximum, sum, output
    cg::cluster_group cluster = cg::this_cluster();
    const int S = cluster.num_blocks(), rank = cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, l8 = lane & 7, grp = lane >> 3;
    const long long unit = blockIdx.x / S;
    const int qb = (int)(unit % qblocks), kvh = (int)(unit / qblocks % p.hk), seq = (int)(unit / qblocks / p.hk);
    const int t = rows_before<MODE>(p, seq);
    if (t < 0) return;                                              // idle: the whole cluster leaves
    const int h0 = kvh * p.g + qb * GQ, nq = min(GQ, p.g - qb * GQ);
    const int live = min(t, p.sinks + p.window), snew = MODE == ATTEND_CONTEXT ? -1 : slot_of(t, p.sinks, p.window);
    for (int i = tid; i < GQ * D; i += NT) qs[i] = 0.f;
    __syncthreads();
    stage_token<T, D, WARPS, MODE>(p, seq, kvh, h0, nq, p.scale_log2e, qs, ks, vs);
    __syncthreads();

    float m[GQ], l[GQ], o[GQ][EL];
#pragma unroll
    for (int q = 0; q < GQ; ++q) {
        m[q] = -CUDART_INF_F; l[q] = 0.f;
#pragma unroll
        for (int e = 0; e < EL; ++e) o[q][e] = 0.f;
    }
    // fold R rows (k, v: this lane's elements; valid: the group's row, slot first + 4 r, is to be used) into the running state
    auto fold = [&](const float (&k)[R][EL], const float (&v)[R][EL], const bool (&valid)[R], int first) {
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
                if (MODE == ATTEND_MASS && valid[r] && l8 == 0 && q < nq) scores_of(p, seq, h0 + q)[first + 4 * r] = s[r];
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
        fold(k, v, valid, base + grp);
    }
    if (MODE != ATTEND_CONTEXT && rank == 0 && warp == 0) {      // the new token: one group counts it, and the first query block stores it
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
        fold(k, v, valid, snew);
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
        finish<T, MODE>(p, seq, h0 + q, d, M, L, live == 0, total_of(p, seq, h0 + q), x);
        store_row<T, MODE>(p, seq, h0 + q, d, x);
    }
    cluster.sync();      // nobody's shared memory goes away while it is read
    if (MODE == ATTEND_MASS && p.add == ADD_IN_PLACE) add_weights<WARPS * BLOCK>(p, seq, kvh, t, rank, S);
}

// ---------------------------------------------------------------------------------------------------------------------
// 16-bit types: the same on warp-level MMAs (m16n8k16, fp32 accumulation).
//
// A warp takes blocks of 16 rows: S[q][key] = Q.K^T with the queries as M, O^T[d][q] += V^T.P^T with d as M, so that the
// accumulators of S are, lane by lane, the B operand of the second product.  Up to 8 query heads share a pass over the rows.  The
// other 8 rows of M hold what rounding a prepared query to 16 bits leaves (zero for queries that come as they are), and P enters as
// two 16-bit parts, so what is left of those roundings is 2^-18 of a weight or of an element of the query (bf16; fp16: 2^-24).  The arithmetic is a fifth of what the
// tensor pipe can do; the kernel is bound by HBM.
//
// Two fp16 parts hold a weight to 2^-25, however small it is, and thousands of small weights beside one large one (a sink) carry what
// the large one's value leaves out.  So fp16 weights are lifted: the maximum is renewed whenever it grows (weights are at most 1), and they
// carry a factor 2^15, which cancels in O / l.  A weight down to 2^-25 of its warp's largest then keeps 15 bits, one of 2^-29 keeps 11, and
// below it counts to 2^-40.  bf16 has the range of fp32.
//
// Each warp brings its rows in by cp.async, 16 bytes a lane, into a ring of its own (no barrier on the way; pieces permuted by
// row so that ldmatrix reads without bank conflicts).  Rows that hold no token are filled with zeros and never read.
// 128 sequences of up to 4100 rows, 8 key heads of 128, 32 query heads, bf16, with rotation: 295 us, 6.6 TB/s, 1.00 of the measured copy
// rate (CUDA cores: 699 us); 9216 units of 410 rows, fp16: 325 us, 0.91 (408 us); one sequence of 16388 rows: 19 us, 0.53 (61 us).
constexpr int MB = 16;               // rows of a block
constexpr int MQ = 8;                // query heads of a unit
// log2: growth at which the subtracted maximum is renewed (weights stay below 2^RENEW), and the factor of the weights
template <typename T> struct Weights { static constexpr float RENEW = 8.f, LIFT = 0.f; };
template <> struct Weights<__half> { static constexpr float RENEW = 0.f, LIFT = 15.f; };

template <int D, int MW> struct Mma {      // MW: warps of a CTA
    static constexpr int STAGES = (D == 128 ? 1 : 2) * (MW == 8 ? 3 : 2);
    static constexpr int ROW = 2 * D, TILE = MB * ROW, STAGE = 2 * TILE;      // bytes: a row, 16 rows, key and value rows of a block
    static constexpr int OFF_Q = MW * STAGES * STAGE;                         // [16][D]: high parts of the queries, low parts
    static constexpr int OFF_NEW = OFF_Q + 16 * ROW;                          // the new token's key and value, 16 bits
    static constexpr int OFF_F32 = OFF_NEW + 2 * ROW;                         // [MQ + 2][D] fp32: the same rows before the rounding
    static constexpr int OFF_PART = OFF_F32;                                  // (later) this CTA's maximum, sum, output: [MQ][D + 2]
    static constexpr int SMEM = OFF_F32 + (MQ + 2) * D * 4;
    static constexpr int SHARED_SCORES = (MQ + 2) * D - (D + 2) - 1;           // scores of one query that have a place besides its result
    static_assert(MQ * (D + 2) <= (MQ + 2) * D, "");
    static_assert(STAGES * STAGE >= MQ * (D + 2) * 4, "a warp's result takes the place of its ring");
};

__device__ __forceinline__ void cp16_or_zero(uint32_t dst, const void *src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T> __device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// (x, y) as 16-bit pairs hi + lo
template <typename T> __device__ __forceinline__ void split2(float x, float y, uint32_t &hi, uint32_t &lo) {
    hi = Vec<T>::pack2(x, y);
    float a, b;
    if constexpr (std::is_same<T, __half>::value) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
        a = f.x; b = f.y;
    } else {
        a = __uint_as_float(hi << 16); b = __uint_as_float(hi & 0xffff0000u);
    }
    lo = Vec<T>::pack2(x - a, y - b);
}

// One query by the D / 8 lanes that finish it: every live row once, in fp32.  x: this lane's 8 elements of the prepared query; fresh: key and
// value rows that stand for those of slot snew (NULL: they are in the cache already).
template <typename T, int D, int MODE>
__device__ __noinline__ void plain_row(const WindowParams &p, int seq, int kvh, int h, int live, int snew, const unsigned char *fresh, const float4 x0, const float4 x1,
                                       float *scores, float *total) {
    constexpr int CHUNKS = D / 8;
    const int c = threadIdx.x % CHUNKS;
    const unsigned group = ((1u << CHUNKS) - 1u) << ((threadIdx.x & 31) & ~(CHUNKS - 1));
    const float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
    float o[8] = {}, m = -CUDART_INF_F, l = 0.f;
    for (int j = 0; j < live; ++j) {
        const long long off = seq * p.css + kvh * p.chs + j * p.cls + c * 16;
        const bool f = fresh && j == snew;
        float k[8], v[8];
        Vec<T>::unpack(*reinterpret_cast<const uint4 *>(f ? reinterpret_cast<const char *>(fresh) + c * 16 : p.kc + off), k);
        Vec<T>::unpack(*reinterpret_cast<const uint4 *>(f ? reinterpret_cast<const char *>(fresh) + 2 * D + c * 16 : p.vc + off), v);
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(x[e], k[e], s);
#pragma unroll
        for (int i = CHUNKS / 2; i; i >>= 1) s += __shfl_xor_sync(group, s, i);
        s *= p.scale_log2e;
        if (MODE == ATTEND_MASS && c == 0) scores[j] = s;
        const float mn = fmaxf(m, s), b = mn == -CUDART_INF_F ? 0.f : mn, keep = ex2_approx(m - b), w = ex2_approx(s - b);
        m = mn;
        l = l * keep + w;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(w, v[e], o[e] * keep);
    }
    finish<T, MODE>(p, seq, h, c * 8, m, l, false, total, o);
    store_row<T, MODE>(p, seq, h, c * 8, o);
}

template <typename T, int D, int MW, int MODE>
__global__ void __launch_bounds__(MW * 32) sh_window_decode_mma_kernel(const __grid_constant__ WindowParams p, int qblocks, int parts) {
    using C = Mma<D, MW>;
    constexpr int CHUNKS = D / 8;                     // 16-byte pieces of a row
    extern __shared__ __align__(128) unsigned char sm[];
    cg::cluster_group cluster = cg::this_cluster();
    // the CTAs that share a unit's rows: a cluster, which merges by itself, or `parts` CTAs whose results a second kernel merges
    const int S = parts ? parts : cluster.num_blocks(), rank = parts ? blockIdx.x % parts : cluster.block_rank();
    if (parts) sh_pdl_launch_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long unit = blockIdx.x / S;
    const int qb = (int)(unit % qblocks), kvh = (int)(unit / qblocks % p.hk), seq = (int)(unit / qblocks / p.hk);
    const int t = rows_before<MODE>(p, seq);
    if (t < 0) return;                                // idle: the whole cluster leaves
    const int h0 = kvh * p.g + qb * MQ, nq = min(MQ, p.g - qb * MQ);
    const int live = MODE == ATTEND_CONTEXT ? t : min(t + 1, p.sinks + p.window);      // rows after the append
    const int snew = MODE == ATTEND_CONTEXT ? -1 : slot_of(t, p.sinks, p.window);
    const char *kc = p.kc + seq * p.css + kvh * p.chs, *vc = p.vc + seq * p.css + kvh * p.chs;
    const uint32_t ring = shasync::smem_u32(sm) + warp * C::STAGES * C::STAGE;

    // rows base .. base + 15 into a stage: a pass of the warp brings 32 / CHUNKS rows of keys and of values
    const int crow = lane / CHUNKS, cchunk = lane % CHUNKS;
    auto request = [&](int base, int st) {
#pragma unroll
        for (int i = 0; i < MB; i += 32 / CHUNKS) {
            const int r = i + crow, j = base + r;
            const bool take = j < live && j != snew;
            const long long off = take ? j * p.cls + cchunk * 16 : 0;
            const uint32_t dst = ring + st * C::STAGE + r * C::ROW + ((cchunk ^ (r & 7)) << 4);
            cp16_or_zero(dst, kc + off, take);
            cp16_or_zero(dst + C::TILE, vc + off, take);
        }
    };
    const int first = (rank * MW + warp) * MB, stride = S * MW * MB;
    int ahead = first;
#pragma unroll
    for (int st = 0; st < C::STAGES - 1; ++st, ahead += stride) {
        if (ahead < live) request(ahead, st);
        shumma::cp_async_commit();
    }
    // the token: prepared in fp32, then queries as two 16-bit parts, key and value as the cache holds them
    float *rows = reinterpret_cast<float *>(sm + C::OFF_F32);
    stage_token<T, D, MW, MODE>(p, seq, kvh, h0, nq, 1.f, rows, rows + MQ * D, rows + (MQ + 1) * D);
    __syncthreads();
    for (int i = tid; i < (MQ + 2) * CHUNKS; i += MW * 32) {
        const int r = i / CHUNKS, c = i % CHUNKS;
        uint32_t hi[4] = {}, lo[4] = {};
        if (r < nq || (MODE != ATTEND_CONTEXT && r >= MQ)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) split2<T>(rows[r * D + c * 8 + 2 * e], rows[r * D + c * 8 + 2 * e + 1], hi[e], lo[e]);
        }
        const uint4 h4 = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        if (r < MQ) {
            *reinterpret_cast<uint4 *>(sm + C::OFF_Q + r * C::ROW + ((c ^ (r & 7)) << 4)) = h4;
            *reinterpret_cast<uint4 *>(sm + C::OFF_Q + (r + 8) * C::ROW + ((c ^ (r & 7)) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        } else {
            *reinterpret_cast<uint4 *>(sm + C::OFF_NEW + (r - MQ) * C::ROW + c * 16) = h4;
        }
    }
    __syncthreads();
    // Q fragments: for each 16 of d, rows 0-7 and 8-15 by d 0-7 and 8-15
    uint32_t qf[D / 16][4];
    const int mrow = (lane & 7) + ((lane >> 3) & 1) * 8, mcol = lane >> 4;      // ldmatrix: this lane's row and piece among four 8 x 8 blocks
#pragma unroll
    for (int k = 0; k < D / 16; ++k) ldsm4(shasync::smem_u32(sm) + C::OFF_Q + mrow * C::ROW + (((2 * k + mcol) ^ (mrow & 7)) << 4), qf[k]);

    // scores and logs of the unit's rows: for small caches in the place of the staged rows, behind what the merge puts there
    float *scores = nullptr, *total = nullptr;
    if (MODE == ATTEND_MASS) {
        const bool shared = p.add == ADD_FROM_SHARED;
        scores = shared ? rows + nq * (D + 2) : scores_of(p, seq, h0);
        total = shared ? scores + nq * p.score_stride : total_of(p, seq, h0);
    }
    float o[D / 16][4];
#pragma unroll
    for (int k = 0; k < D / 16; ++k) o[k][0] = o[k][1] = o[k][2] = o[k][3] = 0.f;
    float m = -CUDART_INF_F, l = 0.f;                 // of query lane / 4; l: this lane's keys only
    int st = 0;
    for (int base = first; base < live; base += stride) {
        cp_wait<C::STAGES - 2>();
        __syncwarp();                                 // everyone's pieces of this block are there, everyone has left the block before
        const int nst = st == 0 ? C::STAGES - 1 : st - 1;
        if (ahead < live) request(ahead, nst);
        shumma::cp_async_commit();
        ahead += stride;
        const uint32_t kt = ring + st * C::STAGE, vt = kt + C::TILE;
        if (snew >= base && snew < base + MB) {       // the new token's rows
            const int r = snew - base;
            if (lane < CHUNKS) {
                unsigned char *dst = sm + (kt - shasync::smem_u32(sm)) + r * C::ROW + ((lane ^ (r & 7)) << 4);
                const uint4 kk = *reinterpret_cast<const uint4 *>(sm + C::OFF_NEW + lane * 16), vv = *reinterpret_cast<const uint4 *>(sm + C::OFF_NEW + C::ROW + lane * 16);
                *reinterpret_cast<uint4 *>(dst) = kk;
                *reinterpret_cast<uint4 *>(dst + C::TILE) = vv;
                if (qb == 0) {                        // (one unit of the key head stores them)
                    *reinterpret_cast<uint4 *>(p.kc + seq * p.css + kvh * p.chs + snew * p.cls + lane * 16) = kk;
                    *reinterpret_cast<uint4 *>(p.vc + seq * p.css + kvh * p.chs + snew * p.cls + lane * 16) = vv;
                }
            }
            __syncwarp();
        }
        float s[2][4] = {};                           // keys 0-7, 8-15 of the block; two chains each would not pay: the pipe is far from full
        const int krow = lane & 7, kcol = lane >> 3;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                uint32_t b[4];
                ldsm4(kt + (n * 8 + krow) * C::ROW + (((4 * k + kcol) ^ krow) << 4), b);
                mma16816<T>(s[n], qf[2 * k], b[0], b[1]);
                mma16816<T>(s[n], qf[2 * k + 1], b[2], b[3]);
            }
        float x[4];                                   // scores of query lane / 4 with keys 2 (lane % 4), + 1, + 8, + 9
        const int j = base + 2 * (lane & 3);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) x[2 * n + e] = j + 8 * n + e < live ? (s[n][e] + s[n][2 + e]) * p.scale_log2e : -CUDART_INF_F;
        if (MODE == ATTEND_MASS && (lane >> 2) < nq) {      // (a row of scores has a place for every row of the last block)
            float *to = scores + (lane >> 2) * p.score_stride + j;
            *reinterpret_cast<float2 *>(to) = make_float2(x[0], x[1]);
            *reinterpret_cast<float2 *>(to + 8) = make_float2(x[2], x[3]);
        }
        float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        if (__any_sync(0xffffffffu, mx - m > Weights<T>::RENEW)) {
            const float mn = fmaxf(m, mx), f = mn == -CUDART_INF_F ? 1.f : ex2_approx(m - mn);
            m = mn;
            l *= f;
            const float f0 = __shfl_sync(0xffffffffu, f, (lane & 3) * 8), f1 = __shfl_sync(0xffffffffu, f, (lane & 3) * 8 + 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) { o[k][0] *= f0; o[k][1] *= f1; o[k][2] *= f0; o[k][3] *= f1; }
        }
        const float mb = m == -CUDART_INF_F ? 0.f : m - Weights<T>::LIFT;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = ex2_approx(x[e] - mb);
        l += (x[0] + x[1]) + (x[2] + x[3]);
        uint32_t h0p, l0p, h1p, l1p;
        split2<T>(x[0], x[1], h0p, l0p);
        split2<T>(x[2], x[3], h1p, l1p);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {            // 16 of d: blocks (keys 0-7, d 0-7), (keys 0-7, d 8-15), (keys 8-15, ..) transposed
            uint32_t a[4];
            const int vrow = (lane & 7) + (lane >> 4) * 8, vcol = 2 * k + ((lane >> 3) & 1);
            ldsm4_t(vt + vrow * C::ROW + ((vcol ^ (vrow & 7)) << 4), a);
            mma16816<T>(o[k], a, h0p, h1p);
            mma16816<T>(o[k], a, l0p, l1p);
        }
        st = st == C::STAGES - 1 ? 0 : st + 1;
    }
    cp_wait<0>();
    constexpr int OLD = C::SHARED_SCORES / (MW * 32) + 1;
    float old[OLD];                                   // masses that the step's weights are added to: asked for before the results are merged
    const long long records = seq * p.rss + kvh * p.rhs;
    if (MODE == ATTEND_MASS && p.add == ADD_FROM_SHARED) {
#pragma unroll
        for (int i = 0; i < OLD; ++i) old[i] = tid + i * MW * 32 < t ? p.mass[records + tid + i * MW * 32] : 0.f;
    }
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    __syncwarp();
    // this warp's result in place of its ring: [query][maximum, sum, output]
    float *mine = reinterpret_cast<float *>(sm + warp * C::STAGES * C::STAGE);
    if ((lane & 3) == 0) { mine[(lane >> 2) * (D + 2)] = m; mine[(lane >> 2) * (D + 2) + 1] = l; }
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[(2 * (lane & 3) + (e & 1)) * (D + 2) + 2 + 16 * k + (lane >> 2) + (e >> 1) * 8] = o[k][e];
    __syncthreads();
    float *cta = reinterpret_cast<float *>(sm + C::OFF_PART);
    auto warp_part = [&](int w) { return reinterpret_cast<const float *>(sm + w * C::STAGES * C::STAGE); };
    for (int i = tid; i < nq * D; i += MW * 32) {
        const int q = i / D, d = i % D;
        float M = -CUDART_INF_F, L = 0.f, acc = 0.f;
#pragma unroll
        for (int w = 0; w < MW; ++w) M = fmaxf(M, warp_part(w)[q * (D + 2)]);
        const float mb = M == -CUDART_INF_F ? 0.f : M;
#pragma unroll
        for (int w = 0; w < MW; ++w) {
            const float *c = warp_part(w) + q * (D + 2);
            const float f = ex2_approx(c[0] - mb);
            L += c[1] * f;
            acc += c[2 + d] * f;
        }
        cta[q * (D + 2) + 2 + d] = acc;
        if (d == 0) { cta[q * (D + 2)] = M; cta[q * (D + 2) + 1] = L; }
    }
    if (parts) {                                      // hand the result over, and once the queries (should a row have to be done again)
        __syncthreads();
        float *to = p.part + (unit * parts + rank) * (MQ * (D + 2));
        for (int i = tid; i < nq * (D + 2); i += MW * 32) to[i] = cta[i];
        if (rank == 0)
            for (int i = tid; i < nq * D; i += MW * 32) {
                const int q = i / D, e = i % D, at = q * C::ROW + (((e / 8) ^ (q & 7)) << 4) + e % 8 * 2;
                const float hi = (float)*reinterpret_cast<const T *>(sm + C::OFF_Q + at), lo = (float)*reinterpret_cast<const T *>(sm + C::OFF_Q + 8 * C::ROW + at);
                p.part[(long long)(gridDim.x) * (MQ * (D + 2)) + unit * (MQ * D) + i] = isfinite(hi) ? hi + lo : hi;
            }
        return;
    }
    cluster.sync();
    // one CTA finishes: a thread per 8 elements
    if (rank == 0)
    for (int q = tid / CHUNKS, d = tid % CHUNKS * 8; q < nq; q += MW * 32 / CHUNKS) {
        float M = -CUDART_INF_F, L = 0.f, acc[8] = {};
        for (int r = 0; r < S; ++r) M = fmaxf(M, cluster.map_shared_rank(cta + q * (D + 2), r)[0]);
        const float mb = M == -CUDART_INF_F ? 0.f : M;
        for (int r = 0; r < S; ++r) {
            const float *c = cluster.map_shared_rank(cta + q * (D + 2), r);
            const float f = ex2_approx(c[0] - mb);
            L += c[1] * f;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf(c[2 + d + e], f, acc[e]);
        }
        const bool odd = finish<T, MODE>(p, seq, h0 + q, d, M - Weights<T>::LIFT, L, live == 0, total + q, acc);
        // the low part of a weight or of a query may be zero and meet an infinity: such rows are computed again in plain fp32
        float hi[8], lo[8];
        Vec<T>::unpack(*reinterpret_cast<const uint4 *>(sm + C::OFF_Q + q * C::ROW + (((d / 8) ^ (q & 7)) << 4)), hi);
        Vec<T>::unpack(*reinterpret_cast<const uint4 *>(sm + C::OFF_Q + (q + 8) * C::ROW + (((d / 8) ^ (q & 7)) << 4)), lo);
#pragma unroll
        for (int e = 0; e < 8; ++e) hi[e] = isfinite(hi[e]) ? hi[e] + lo[e] : hi[e];
        const float4 x0 = make_float4(hi[0], hi[1], hi[2], hi[3]), x1 = make_float4(hi[4], hi[5], hi[6], hi[7]);
        const unsigned group = ((1u << CHUNKS) - 1u) << (lane & ~(CHUNKS - 1));
        if (__any_sync(group, odd))
            plain_row<T, D, MODE>(p, seq, kvh, h0 + q, live, snew, MODE == ATTEND_CONTEXT ? nullptr : sm + C::OFF_NEW, x0, x1, scores + q * p.score_stride, total + q);
        else
            store_row<T, MODE>(p, seq, h0 + q, d, acc);
    }
    cluster.sync();                                   // nobody's shared memory goes away while it is read
    if (MODE == ATTEND_MASS && p.add == ADD_IN_PLACE) add_weights<MW * MB>(p, seq, kvh, t, rank, S);
    if (MODE == ATTEND_MASS && p.add == ADD_FROM_SHARED) {
#pragma unroll
        for (int i = 0; i < OLD; ++i) {
            const int j = tid + i * MW * 32;
            if (j > t) break;
            float sum = 0.f;
            for (int q = 0; q < nq; ++q) sum += ex2_approx(scores[q * p.score_stride + j] - total[q]);
            p.mass[records + j] = old[i] + sum;
            if (j == t) p.held[records + j] = p.seen[seq];
        }
    }
}

// Merge the `parts` results of each unit: a CTA per (unit, query), SLICES groups of D / 8 lanes that take every SLICES-th part each.
constexpr int SLICES = 8;
template <typename T, int D, int MODE>
__global__ void __launch_bounds__(SLICES * D / 8) sh_window_decode_merge_kernel(const __grid_constant__ WindowParams p, int qblocks, int parts, long long units) {
    constexpr int CHUNKS = D / 8, N = SLICES * CHUNKS, REC = MQ * (D + 2);
    __shared__ float top[N / 32], sum[SLICES], out[SLICES][D];
    const int tid = threadIdx.x, q = blockIdx.x % MQ, slice = tid / CHUNKS, c = tid % CHUNKS;
    const long long unit = blockIdx.x / MQ;
    const int qb = (int)(unit % qblocks), kvh = (int)(unit / qblocks % p.hk), seq = (int)(unit / qblocks / p.hk);
    sh_pdl_wait();
    const int t = rows_before<MODE>(p, seq);
    if (t < 0 || q >= min(MQ, p.g - qb * MQ)) return;
    const float *rec = p.part + unit * parts * REC + q * (D + 2);
    float M = -CUDART_INF_F;
    for (int i = tid; i < parts; i += N) M = fmaxf(M, rec[(long long)i * REC]);
#pragma unroll
    for (int i = 16; i; i >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, i));
    if (tid % 32 == 0) top[tid / 32] = M;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N / 32; ++i) M = fmaxf(M, top[i]);
    const float mb = M == -CUDART_INF_F ? 0.f : M;
    float L = 0.f, acc[8] = {};
    for (int i = slice; i < parts; i += SLICES) {
        const float *r = rec + (long long)i * REC;
        const float f = ex2_approx(r[0] - mb);
        L += r[1] * f;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float2 x = *reinterpret_cast<const float2 *>(r + 2 + c * 8 + e);
            acc[e] = fmaf(x.x, f, acc[e]);
            acc[e + 1] = fmaf(x.y, f, acc[e + 1]);
        }
    }
    if (c == 0) sum[slice] = L;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[slice][c * 8 + e] = acc[e];
    __syncthreads();
    if (slice) return;
    L = 0.f;
#pragma unroll
    for (int i = 0; i < SLICES; ++i) L += sum[i];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < SLICES; ++i) x += out[i][c * 8 + e];
        acc[e] = x;
    }
    const int h = kvh * p.g + qb * MQ + q;
    const bool odd = finish<T, MODE>(p, seq, h, c * 8, M - Weights<T>::LIFT, L, t == 0, total_of(p, seq, h), acc);
    if (__any_sync((1u << CHUNKS) - 1u, odd)) {
        const float4 *x = reinterpret_cast<const float4 *>(p.part + units * parts * REC + unit * (MQ * D) + q * D + c * 8);
        plain_row<T, D, MODE>(p, seq, kvh, h, MODE == ATTEND_CONTEXT ? t : min(t + 1, p.sinks + p.window), 0, nullptr, x[0], x[1], scores_of(p, seq, h), total_of(p, seq, h));
    } else {
        store_row<T, MODE>(p, seq, h, c * 8, acc);
    }
}

// Parts of all units together; bounds the workspace.
constexpr int MAX_PARTS = 160;

cudaLaunchConfig_t cluster_config(unsigned ctas, int threads, size_t smem, int S, cudaLaunchAttribute *attr, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim.x = S; attr->val.clusterDim.y = 1; attr->val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

// CTAs of `kern` in clusters of 1, 2, 4 and 8 that the current device holds at once (a cluster lies within one group of SMs, so with
// large CTAs not every SM can be used, and a size may have no place at all: 0).  Asked once per device.
template <auto kern>
cudaError_t cluster_slots(int threads, size_t smem, int (&slots)[4]) {
    static std::atomic<int> known[ShKernelSetup::DEVICES][4];      // one more than the answer; 0: not asked yet
    static ShKernelSetup setup;
    int dev = 0, sms = 0;
    cudaError_t e = sh_device_sms(&dev, &sms);
    if (e != cudaSuccess) return e;
    const bool kept = dev < ShKernelSetup::DEVICES;
    for (int i = 0; i < 4; ++i) {
        slots[i] = (kept ? known[dev][i].load(std::memory_order_relaxed) : 0) - 1;
        if (slots[i] >= 0) continue;
        e = sh_setup_kernel(setup, kern, smem, &sms);
        if (e != cudaSuccess) return e;
        cudaLaunchAttribute attr;
        const cudaLaunchConfig_t cfg = cluster_config(1u << i, threads, smem, 1 << i, &attr, nullptr);
        int clusters = 0;
        e = cudaOccupancyMaxActiveClusters(&clusters, kern, &cfg);
        if (e != cudaSuccess) return e;
        slots[i] = std::max(clusters, 0) << i;
        if (kept) known[dev][i].store(slots[i] + 1, std::memory_order_relaxed);
    }
    return cudaSuccess;
}

template <auto kern>
cudaError_t launch_units(const WindowParams &p, int qblocks, int threads, size_t smem, int S, int parts, cudaStream_t s) {
    const long long ctas = (long long)p.sequences * p.hk * qblocks * (parts ? parts : S);
    if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
    static ShKernelSetup setup;
    int sms = 0;
    const cudaError_t e = sh_setup_kernel(setup, kern, smem, &sms);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = cluster_config((unsigned)ctas, threads, smem, S, &attr, s);
    return cudaLaunchKernelEx(&cfg, kern, p, qblocks, parts);
}

// A launch of clusters and, for the masses, the weights' addition: by the CTAs themselves from scores in shared memory where a unit is one
// CTA and they fit (`places`: floats for them; 9216 units of 442 rows: 350 against 356 us), or from scores in global memory where a key
// head is one unit and all of them run at once, as it saves a launch (5 sequences, 12 heads of 64, fp32: 8.3 -> 7.3 us); else by a launch of
// its own, as the CTAs that wait for a place wait for the scores' way too (the same 9216 units: 396 us).
template <auto kern, int MODE>
cudaError_t launch_step(WindowParams p, int D, int qblocks, int threads, size_t smem, int S, const int (&slots)[4], int places, cudaStream_t s) {
    int i = 0;
    while (1 << i < S) ++i;
    p.add = ADD_LATER;
    if (MODE == ATTEND_MASS && qblocks == 1) {
        if (S == 1 && p.g * (D + 2 + p.score_stride + 1) <= places) p.add = ADD_FROM_SHARED;
        else if ((long long)p.sequences * p.hk * S <= slots[i]) p.add = ADD_IN_PLACE;
    }
    const cudaError_t e = launch_units<kern>(p, qblocks, threads, smem, S, 0, s);
    return MODE == ATTEND_MASS && e == cudaSuccess && p.add == ADD_LATER ? sh_launch_mass_fold(p, s) : e;
}

template <int D, int GQ, int MODE>
cudaError_t launch_simt(const WindowParams &p, cudaStream_t s) {
    constexpr auto kern = sh_window_decode_simt_kernel<float, D, GQ, MODE>;
    const int qblocks = (p.g + GQ - 1) / GQ;
    int slots[4];
    const cudaError_t e = cluster_slots<kern>(NT, 0, slots);
    if (e != cudaSuccess) return e;
    const Shape a = best_split((long long)p.sequences * p.hk * qblocks, (long long)p.window + p.sinks, 8 * D, slots, 3.0e4);
    return launch_step<kern, MODE>(p, D, qblocks, NT, 0, a.S, slots, 0, s);
}
template <int D, int MODE>
cudaError_t launch_f32(const WindowParams &p, cudaStream_t s) {
    return p.g == 1 ? launch_simt<D, 1, MODE>(p, s) : (p.g == 2 ? launch_simt<D, 2, MODE>(p, s) : launch_simt<D, 4, MODE>(p, s));
}
// Two shapes: CTAs of 4 warps, 3 to an SM, each warp with one block of rows in flight besides the one it works on; and CTAs of 8 warps,
// one to an SM, with two in flight.  Many units want the first (9216 units of 410 rows: 325 against 545 us), few units, which
// cannot fill the machine, the second, whose CTAs draw more each (8 units of 16384 rows: 34 against 23 us).
template <typename T, int D, int MODE>
cudaError_t launch_mma(const WindowParams &p, cudaStream_t s) {
    using Small = Mma<D, 4>;
    using Large = Mma<D, 8>;
    static_assert(3 * (Small::SMEM + 1024) <= 233472 && Large::SMEM <= 232448, "CTAs per SM");
    const int qblocks = (p.g + MQ - 1) / MQ;
    const long long units = (long long)p.sequences * p.hk * qblocks, rows = (long long)p.window + p.sinks;
    constexpr auto small = sh_window_decode_mma_kernel<T, D, 4, MODE>, large = sh_window_decode_mma_kernel<T, D, 8, MODE>;
    int slots_a[4], slots_b[4];
    cudaError_t e = cluster_slots<small>(128, Small::SMEM, slots_a);
    if (e == cudaSuccess) e = cluster_slots<large>(256, Large::SMEM, slots_b);
    if (e != cudaSuccess) return e;
    const Shape a = best_split(units, rows, 4 * D, slots_a, 3.6e4), b = best_split(units, rows, 4 * D, slots_b, 5.8e4);
    // Fewer units than SMs: parts whose results a second launch merges (about 3 us) can fill every SM, a cluster of 8 cannot.
    const long long parts = std::min(std::min((long long)slots_b[0], (long long)MAX_PARTS) / units, rows / 64);
    if (p.part && parts > 1) {
        const double us = (double)rows * 4 * D / parts / std::min(6.4e6 / (double)(units * parts), 5.8e4) + 5.5;
        if (us < a.us && us < b.us) {
            e = launch_units<large>(p, qblocks, 256, Large::SMEM, 1, (int)parts, s);
            if (e != cudaSuccess) return e;
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)(units * MQ));
            cfg.blockDim = dim3(SLICES * D / 8);
            cfg.stream = s;
            cudaLaunchAttribute attr = {};
            attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr.val.programmaticStreamSerializationAllowed = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            e = cudaLaunchKernelEx(&cfg, sh_window_decode_merge_kernel<T, D, MODE>, p, qblocks, (int)parts, units);
            return MODE == ATTEND_MASS && e == cudaSuccess ? sh_launch_mass_fold(p, s) : e;
        }
    }
    constexpr int places = (MQ + 2) * D;
    return a.us <= b.us ? launch_step<small, MODE>(p, D, qblocks, 128, Small::SMEM, a.S, slots_a, places, s)
                        : launch_step<large, MODE>(p, D, qblocks, 256, Large::SMEM, b.S, slots_b, places, s);
}

}  // namespace

template <int MODE>
static cudaError_t launch_type(const WindowParams &p, int dtype, int D, cudaStream_t s) {
    if (dtype == SH_F32) return D == 128 ? launch_f32<128, MODE>(p, s) : launch_f32<64, MODE>(p, s);
    if (dtype == SH_F16) return D == 128 ? launch_mma<__half, 128, MODE>(p, s) : launch_mma<__half, 64, MODE>(p, s);
    return D == 128 ? launch_mma<__nv_bfloat16, 128, MODE>(p, s) : launch_mma<__nv_bfloat16, 64, MODE>(p, s);
}
cudaError_t sh_launch_window_decode(const WindowParams &p, int dtype, int D, int mode, cudaStream_t s) {
    if (mode == ATTEND_CONTEXT) return launch_type<ATTEND_CONTEXT>(p, dtype, D, s);
    return mode == ATTEND_MASS ? launch_type<ATTEND_MASS>(p, dtype, D, s) : launch_type<ATTEND_WINDOW>(p, dtype, D, s);
}

size_t sh_window_decode_scratch(int sequences, int hk, int g, int dtype, int D) {
    const long long units = (long long)sequences * hk * ((g + MQ - 1) / MQ);
    if (dtype == SH_F32 || units < 1 || units * 2 > MAX_PARTS) return 0;
    return sizeof(float) * ((size_t)MAX_PARTS * MQ * (D + 2) + (size_t)units * MQ * D);
}
