// Truncated sampling: temperature, top-k, top-p and min-p, with the noise of the full-vocabulary
// sampler (sampler.hip).
//
// Tokens are ordered by logit, descending, equal ones by index.  Kept is the prefix of that order
// with rank < top_k, mass before the token < top_p times the mass of the first top_k, and
// logit >= largest + T ln(min_p); the draw is the argmax of l / T + g over what is kept, which is a
// draw from the kept tokens' renormalised softmax.
//
// top_k <= kTopMax: the top_k largest are selected in one pass (top_logits.h), and everything else
// happens on them, sorted, in LDS.
//
// No top-k: nothing is sorted.  The draw over a set that contains the kept tokens, if it is itself
// kept, is the draw over the kept tokens (the largest score of a superset); if not, no kept token
// comes after it in the order, and the draw is repeated over the tokens before it, a smaller set that
// still contains every kept one.  So a row costs one pass of noise, as dash_sample, then one
// pass that sums the mass before the winner, and a row's winner is kept with probability
// top_p; 1 + ln(1 / top_p) draws are expected from a flat row.  The mass is compared in float32
// exponentials first; only where it is within kMassTol of the border, the sums are repeated in
// float64, so the decision is that of float64 sums.
#include "kernels.h"
#include "sampler_screen.h"
#include "top_logits.h"

namespace dash {

namespace {

// Relative error of a row's float32 mass against exact exponentials: an entry at distance y (in
// powers of two) from the maximum is off by y ln 2 times three roundings of 2^-24 (difference,
// scale, product) and the exponential's 2^-23; averaged over a row's mass y is at most log2(vocab)
// <= 28.  Together below 4e-6 for either sum; sums in float64 add nothing.
constexpr double kMassTol = 1e-5;

struct Draw {
    const float* logits;
    int64_t ld;
    int vocab;
    const int32_t* row_of;
    const int32_t* uid;
    const int32_t* step;
    float temperature, scale;
    int top_k;
    double top_p, log_min_p;  // log_min_p: -inf keeps all
    uint32_t k0, k1;
    int32_t* tok_out;
    float* lp_out;
    uint32_t* status;
};

DASH_DEV void write_draw(const Draw& a, int b, int tok, double lp) {
    a.tok_out[b] = tok;
    if (a.lp_out) a.lp_out[b] = tok >= 0 ? (float)lp : NAN;
    if (tok < 0 && a.status) atomicOr(a.status, 2u);  // no finite logit: nothing can be drawn
}

DASH_DEV float noise_of(const Draw& a, int i, uint32_t step, uint32_t uid) {
    const U4 x = philox4x32_10(U4{(uint32_t)i >> 2, step, uid, 0u}, a.k0, a.k1);
    const uint32_t lo = i & 1 ? x.y : x.x, hi = i & 1 ? x.w : x.z;
    return gumbel_from_bits(i & 2 ? hi : lo);
}

// Largest score of the work-group, smallest index on ties (INT_MAX: none); every thread gets it.
struct BestShared {
    float s[kRowWaves];
    int i[kRowWaves];
};
DASH_DEV int block_best(float s, int i, BestShared& sh) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const float os = __shfl_xor(s, o, 64);
        const int oi = __shfl_xor(i, o, 64);
        if (better(os, oi, s, i)) {
            s = os;
            i = oi;
        }
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        sh.s[threadIdx.x >> 6] = s;
        sh.i[threadIdx.x >> 6] = i;
    }
    __syncthreads();
    s = sh.s[0];
    i = sh.i[0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w)
        if (better(sh.s[w], sh.i[w], s, i)) {
            s = sh.s[w];
            i = sh.i[w];
        }
    return i;
}

// Inclusive sum of v over the threads up to this one, and the total, in float64.
DASH_DEV double block_scan(double v, double* red, double& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 63) red[w] = v;
    __syncthreads();
    double before = 0.0;
    total = 0.0;
    for (int i = 0; i < kRowWaves; ++i) {
        if (i < w) before += red[i];
        total += red[i];
    }
    return v + before;
}

template <bool UNIT_T>
__global__ void __launch_bounds__(kRowThreads)
draw_top_k(Draw a) {
    __shared__ TopShared sh;
    __shared__ BestShared best;
    const int b = blockIdx.x;
    const float* row = a.logits + (int64_t)(a.row_of ? a.row_of[b] : b) * a.ld;
    TopState st;
    top_begin(sh);
    top_walk(sh, st, row, 0, a.vocab, a.top_k, a.scale);
    const int m = top_finish(sh, st, a.top_k, a.scale);
    const double T = a.temperature;
    float ref;
    const double rest = top_rest(sh, st, T, ref);
    const bool in = (int)threadIdx.x < m;
    const uint64_t word = in ? sh.c[threadIdx.x] : 0;
    const float l = word_value(word), l0 = word_value(sh.c[0]);
    const int i = word_index(word);
    const double w = in ? exp(((double)l - (double)l0) / T) : 0.0;
    double total;
    const double upto = block_scan(w, sh.red_d, total);
    bool keep = in && (a.top_p >= 1.0 || upto - w < a.top_p * total);
    keep = keep && (double)l >= (double)l0 + T * a.log_min_p;
    float s = -INFINITY;
    if (keep) s = (UNIT_T ? l : div_rn(l, a.temperature)) + noise_of(a, i, (uint32_t)a.step[b], (uint32_t)a.uid[b]);
    const int tok = block_best(s, keep ? i : 0x7FFFFFFF, best);
    if (threadIdx.x != 0) return;
    if (tok == 0x7FFFFFFF) {
        write_draw(a, b, -1, 0.0);
    } else {
        const double all = total + (rest > 0.0 ? rest * exp(((double)ref - (double)l0) / T) : 0.0);
        write_draw(a, b, tok, ((double)row[tok] - (double)l0) / T - log(all));
    }
}

// What a pass of noise may draw from: entries before (l, i) in the order, at or above `low`.
struct Before {
    float l;
    int i;
    float low;
};
DASH_DEV bool comes_before(float l, int i, const Before& w) {
    return (l > w.l || (l == w.l && i < w.i)) && l < INFINITY && l >= w.low;
}

// The draw over a row's entries (ALL: every finite one; else those that come before w), screened as
// in sampler.hip.  ALL also sums the row's exponentials and finds its largest logit.
template <bool UNIT_T, bool ALL>
DASH_DEV int draw_row(const Draw& a, const float* row, uint32_t step, uint32_t uid, const Before& w, float* floor_s,
                      BestShared& best, ExpSum& sum, float& top) {
    float best_s = -INFINITY;
    int best_i = 0x7FFFFFFF;
    const float inv_t = UNIT_T ? 1.f : div_rn(1.f, a.temperature);
    __syncthreads();
    if (threadIdx.x == 0) *floor_s = -INFINITY;
    __syncthreads();
    walk_row<2, false>(row, 0, a.vocab, [&](f32x4_t l, int i) {
        bool some = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = ALL ? fabsf(l[j]) < INFINITY : comes_before(l[j], i + j, w);
            l[j] = in ? l[j] : -INFINITY;
            some |= in;
        }
        if (!__any(some)) return;
        const float m4 = max4(l);
        if constexpr (ALL) {
            top = fmaxf(top, m4);
            exp_push4<false>(sum, l, m4, a.scale);
        }
        // Relaxed: a stale bound is a lower one, and only more entries are evaluated.
        const float floor_w = __hip_atomic_load(floor_s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        const U4 x = philox4x32_10(U4{(uint32_t)i >> 2, step, uid, 0u}, a.k0, a.k1);
        float sc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // l / T by a product and one corrected step, within the margin of the exact quotient, or
            // NaN where something overflows (then nothing is screened)
            const float q = l[j] * inv_t;
            sc[j] = UNIT_T ? l[j] : __builtin_fmaf(__builtin_fmaf(-q, a.temperature, l[j]), inv_t, q);
            if (l[j] == -INFINITY) sc[j] = -INFINITY;
        }
        float hi4 = sc[0];
#pragma unroll
        for (int j = 1; j < 4; ++j) hi4 = UNIT_T ? fmaxf(hi4, sc[j]) : __builtin_elementwise_maximum(hi4, sc[j]);
        hi4 += noise_bound(max(max(x.x, x.y), max(x.z, x.w)));
        if (!__any(!(hi4 + screen_margin(hi4) < floor_w) && hi4 != -INFINITY)) return;
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
        float floor_t = floor_w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (l[j] == -INFINITY) continue;
            const float hi = sc[j] + noise_bound(xs[j]);
            if (hi + screen_margin(hi) < floor_t) continue;
            const float sa = sc[j] + cheap_gumbel(xs[j]);
            const float mg = screen_margin(sa);
            if (!(sa + mg < floor_t)) {
                const float s = (UNIT_T ? l[j] : div_rn(l[j], a.temperature)) + gumbel_from_bits(xs[j]);
                // indices grow within a thread: the smallest stays on ties, also of quotients that overflow to -inf
                if (s > best_s || best_i == 0x7FFFFFFF) {
                    best_s = s;
                    best_i = i + j;
                }
                floor_t = fmaxf(floor_t, s);
            } else {
                floor_t = fmaxf(floor_t, sa - mg);
            }
        }
        const float f = wave_max_f(floor_t);
        if (f > floor_w && (threadIdx.x & 63) == 0)
            (void)__hip_atomic_fetch_max(floor_s, f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    });
    return block_best(best_s, best_i, best);
}

// Mass before w and of the row, relative to the largest logit, in float32 or (EXACT) float64 exponentials.
template <bool EXACT>
DASH_DEV void mass_before(const Draw& a, const float* row, const Before& w, float top, double* red, double& before,
                          double& all) {
    double sb = 0.0, sa = 0.0;
    walk_row<4, false>(row, 0, a.vocab, [&](const f32x4_t& l, int i) {
        if constexpr (EXACT) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!(fabsf(l[j]) < INFINITY)) continue;
                const double e = exp(((double)l[j] - (double)top) / (double)a.temperature);
                sa += e;
                if (l[j] > w.l || (l[j] == w.l && i + j < w.i)) sb += e;
            }
        } else {
            float ta = 0.f, tb = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float v = fabsf(l[j]) < INFINITY ? l[j] : -INFINITY;
                const float e = __builtin_amdgcn_exp2f((v - top) * a.scale);
                ta += e;
                tb += v > w.l || (v == w.l && i + j < w.i) ? e : 0.f;
            }
            sa += (double)ta;
            sb += (double)tb;
        }
    });
    before = block_sum_d(sb, red);
    all = block_sum_d(sa, red);
}

template <bool UNIT_T>
__global__ void __launch_bounds__(kRowThreads)
draw_top_p(Draw a) {
    __shared__ BestShared best;
    __shared__ double red_d[kRowWaves];
    __shared__ float red_f[kRowWaves];
    __shared__ float floor_s;
    const int b = blockIdx.x;
    const float* row = a.logits + (int64_t)(a.row_of ? a.row_of[b] : b) * a.ld;
    const uint32_t step = (uint32_t)a.step[b], uid = (uint32_t)a.uid[b];
    const double T = a.temperature;
    Before w{INFINITY, 0x7FFFFFFF, -INFINITY};
    ExpSum sum;
    float top = -INFINITY;
    int tok = draw_row<UNIT_T, true>(a, row, step, uid, w, &floor_s, best, sum, top);
    if (tok == 0x7FFFFFFF) {
        if (threadIdx.x == 0) write_draw(a, b, -1, 0.0);
        return;
    }
    top = block_max_f(top, red_f);
    const double z = block_sum_d(sum.z * exp(((double)sum.ref - (double)top) / T), red_d);
    {  // the least float at or above the min-p border
        const double t = (double)top + T * a.log_min_p;
        w.low = (float)t;
        if ((double)w.low < t) w.low = nextafterf(w.low, INFINITY);
    }
    for (;;) {
        w.l = row[tok];
        w.i = tok;
        bool kept = w.l >= w.low;
        if (kept && a.top_p < 1.0) {
            // all but the winner's own mass is at least what comes before it
            const double own = exp(((double)w.l - (double)top) / T) / z;
            if (!(1.0 - own < a.top_p - kMassTol)) {
                double before, all;
                mass_before<false>(a, row, w, top, red_d, before, all);
                if (fabs(before - a.top_p * all) <= kMassTol * all) mass_before<true>(a, row, w, top, red_d, before, all);
                kept = before < a.top_p * all;
            }
        }
        if (kept) break;
        tok = draw_row<UNIT_T, false>(a, row, step, uid, w, &floor_s, best, sum, top);
        if (tok == 0x7FFFFFFF) break;  // (the first token of the order is always kept)
    }
    if (threadIdx.x == 0) {
        if (tok == 0x7FFFFFFF) write_draw(a, b, -1, 0.0);
        else write_draw(a, b, tok, ((double)row[tok] - (double)top) / T - log(z));
    }
}

}  // namespace

hipError_t launch_sample_truncated(const float* logits, int64_t ld, int rows, int vocab, const int32_t* row_of,
                                   const int32_t* uid, const int32_t* step, float temperature, int top_k, double top_p,
                                   double min_p, uint64_t seed, int32_t* tok_out, float* lp_out, uint32_t* status,
                                   hipStream_t st) {
    if (rows <= 0) return hipSuccess;
    const Draw a{logits, ld, vocab, row_of, uid, step, temperature, exp2_scale(temperature), top_k, top_p,
                 log(min_p), (uint32_t)seed, (uint32_t)(seed >> 32), tok_out, lp_out, status};
    const bool unit = temperature == 1.0f;
    if (top_k > 0 && top_k < vocab) {
        if (unit) draw_top_k<true><<<rows, kRowThreads, 0, st>>>(a);
        else draw_top_k<false><<<rows, kRowThreads, 0, st>>>(a);
    } else {
        if (unit) draw_top_p<true><<<rows, kRowThreads, 0, st>>>(a);
        else draw_top_p<false><<<rows, kRowThreads, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace dash
