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
// still contains every kept one.
//   draw_first   the draw over the row, its exponential sum, and (top_p) a histogram of its mass over the
//                logit, 32 parts per power of two.  The histogram tells from the winner's logit
//                whether it is kept, unless it lies within two parts of the border.  Of rows of
//                151,936, peaked or flat, at T = 0.6 to 1, 89 to 97 in 100 end here at top_p = 0.95 and
//                82 to 93 at 0.9.  A row with an entry far above the sampled reference has no
//                histogram: of the peaked rows that stay open a quarter at T = 1, half to nine tenths
//                at 0.6.  With min-p the draw leaves out at once what is too far below the largest
//                logit so far.
//   draw_second  rows that did not end: the mass before the winner, and at once the draw over the
//                tokens before it that the histogram does not rule out; each row cut into stretches,
//                so that few rows still fill the GPU.
//   draw_last    joins these; the second winner is nearly always settled by the histogram, too.  What is
//                left takes another round of both, if there are many rows, and then further passes
//                of one work-group.
// Few rows are cut into stretches in the first pass as well, joined by draw_join.
// Vector instructions bound the first pass, most of them Philox's and the screening's (1024 rows of 151,936
// without truncation 153 us, the full-vocabulary sampler 130); the later ones are latency.  At top_p = 0.95
// 64 rows take 23, 11, 13 and 5 us in draw_first, draw_join, draw_second and draw_last; 1024 flat
// rows 177 us in the first and 8 to 30 in the rest.  With top-k = 64 1024 rows take 110 us in the
// selection (5.7 TB/s: memory) and 16 in the draw.
// Masses are float32 exponentials first; only where they are within kMassTol of the border, the sums
// are repeated in float64, so the decision is that of float64 sums.
#include <type_traits>

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

constexpr int kDrawTarget = 512;   // work-groups that fill the GPU: two per CU
// One per CU where draw_first leaves stretches: in registers for two it spilled a few, and a launch
// with scratch memory is slow to start (64 rows of 151,936 59 -> 55 us a call, 200 rows 78 -> 70).
constexpr int kSplitTarget = 256;
constexpr int kDrawStretch = 4096;  // least entries of a stretch

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

// Largest score of the work-group, smallest index on ties (kNone: none); every thread gets both.
constexpr int kNone = 0x7FFFFFFF;
struct BestShared {
    float s[kRowWaves];
    int i[kRowWaves];
};
template <int NT = kRowThreads>
DASH_DEV void block_best(float& s, int& i, BestShared& sh) {
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
    for (int w = 1; w < NT / 64; ++w)
        if (better(sh.s[w], sh.i[w], s, i)) {
            s = sh.s[w];
            i = sh.i[w];
        }
}

template <bool UNIT_T, int NT, int PER>
__global__ void __launch_bounds__(NT)
draw_top_k(Draw a, TopParts parts) {
    __shared__ TopShared<NT, PER> sh;
    __shared__ BestShared best;
    const int b = blockIdx.x;
    const float* row = a.logits + (int64_t)(a.row_of ? a.row_of[b] : b) * a.ld;
    TopState st;
    const int p = top_room(a.top_k);
    top_gather(sh, st, parts, b, row, a.vocab, a.top_k, p, a.scale);
    const int m = top_finish(sh, st, a.top_k, p, a.scale);
    const double T = a.temperature;
    float ref;
    const double rest = block_exp_sum<NT>(st.rest, T, sh.red_f, sh.red_d, ref);
    const bool in = (int)threadIdx.x < m;
    const uint64_t word = in ? sh.c[threadIdx.x] : 0;
    const float l = word_value(word), l0 = word_value(sh.c[0]);
    const double w = in ? exp(((double)l - (double)l0) / T) : 0.0;
    double total;
    const double upto = block_scan<NT>(w, sh.red_d, total);
    bool keep = in && (a.top_p >= 1.0 || upto - w < a.top_p * total);
    keep = keep && (double)l >= (double)l0 + T * a.log_min_p;
    float s = -INFINITY;
    int tok = kNone;
    if (keep) {
        tok = word_index(word);
        s = (UNIT_T ? l : div_rn(l, a.temperature)) + noise_of(a, tok, (uint32_t)a.step[b], (uint32_t)a.uid[b]);
    }
    block_best<NT>(s, tok, best);
    if (threadIdx.x != 0) return;
    if (tok == kNone) {
        write_draw(a, b, -1, 0.0);
    } else {
        const double all = total + (rest > 0.0 ? rest * exp(((double)ref - (double)l0) / T) : 0.0);
        write_draw(a, b, tok, ((double)row[tok] - (double)l0) / T - log(all));
    }
}

// ---- without top-k ----------------------------------------------------------------------------

// Histogram of a row's mass: an exponential e relative to a reference logit falls into the part that
// its exponent and the five bits below it name; there are 1024, one per thread, from 20 octaves
// below the reference to 12 above (an entry further above voids the histogram).  A part is summed in
// integers, the leading 14 bits of each e, so sums do not depend on order: 2^18 terms fit, and what is
// cut off is less than 2^-13 of each.  (Float atomics in LDS took five times as long as everything
// else.)  Lanes add to four copies.
constexpr int kBins = kRowThreads;
constexpr int kBinsPerOctave = 32;
constexpr int kBinsBelow = 20, kBinsAbove = kBins / kBinsPerOctave - kBinsBelow;  // octaves
constexpr uint32_t kBinBase = (127 - kBinsBelow) * kBinsPerOctave;
constexpr int kCopies = 4;
constexpr int kHistVocab = 1 << 18;
constexpr int kMostParts = 16;  // stretches of a row in the first pass: draw_join reads a histogram of each
constexpr double kBinTol = 1.3e-4;  // 2^-13, rounded up
DASH_DEV int bin_of(float e) { return min(max((int)(__float_as_uint(e) >> 18) - (int)kBinBase, 0), kBins - 1); }
DASH_DEV uint32_t bin_term(float e) { return __builtin_amdgcn_ubfe(__float_as_uint(e), 10, 13) | 0x2000u; }
// Value of a sum of terms of bin i.  (Entries below the lowest bin join it and count for more than they
// are, or are left out; that moves only the mass at or above bin 0, which rules nothing out and settles nothing.
// Peaked rows at T = 0.6 put nine entries in ten there and take no longer than flat ones: 1024 rows of 151,936 at
// top_p = 0.95 201 us against 202.)
DASH_DEV double bin_mass(uint32_t sum, int i) { return ldexp((double)sum, i / kBinsPerOctave - kBinsBelow - 13); }

// What a work-group that walked a stretch of a row in draw_first leaves.
struct FirstPart {
    double z;         // sum of e^((l - ref) / T)
    float ref, top;   // top: largest logit
    float bins_at;    // reference of the bins, octaves: a whole number; NaN: no histogram
    float s;          // largest score and its token
    int i, pad;
};
// A row that has not ended: its winner, and what it takes to settle it.
struct RowState {
    double z;         // sum of e^((l - top) / T)
    float l, top, low;  // the winner's logit, the largest, the least that min-p keeps
    float bin_ref;    // reference logit of the bins; NaN: no histogram
    int tok;
    int unsure;       // the winner may be kept
    int border, sure; // tokens of bins below border are not kept, of bins from sure on they are
};
struct SecondPart {
    double before;  // sum of e^((l - top) / T) before the winner
    float s;        // draw over the tokens before it
    int i;
};

// The logit that lies n octaves from zero.
DASH_DEV float octaves(float n, float temperature) { return (float)((double)n * 0.6931471805599453 * (double)temperature); }

DASH_DEV bool kept_by_own_mass(const Draw& a, float l, float top, double z) {
    // all but the winner's own mass is at least what comes before it
    return 1.0 - exp(((double)l - (double)top) / (double)a.temperature) / z < a.top_p - kMassTol;
}

// Settles a row after its first draw, or leaves its state.  bin: the mass of this thread's bin.
struct SettleShared {
    double red[kRowWaves];
    int red_i[kRowWaves];
};
DASH_DEV void settle(const Draw& a, int b, const float* row, int tok, float top, double z, float bin_ref, double bin,
                     SettleShared& sh, RowState* state, int* open) {
    bool done = true;
    RowState r{z, 0.f, top, -INFINITY, bin_ref, tok, 0, -kBins, 2 * kBins};
    if (tok != kNone) {
        const double T = a.temperature;
        r.l = row[tok];
        // the least float at or above the min-p border
        const double t = (double)top + T * a.log_min_p;
        r.low = (float)t;
        if ((double)r.low < t) r.low = nextafterf(r.low, INFINITY);
        const bool reaches = r.l >= r.low;
        done = reaches && (a.top_p >= 1.0 || kept_by_own_mass(a, r.l, top, z));
        if (!done && a.top_p < 1.0) {
            r.unsure = reaches;
            if (bin_ref == bin_ref) {
                // Mass at or above each bin, with one bin either way for logits that other stretches or
                // the exponential's last bit put into a neighbouring bin.
                double all;
                const double below = block_scan(bin, sh.red, all);
                const double from = all - below + bin, tol = (kMassTol + kBinTol) * z;
                auto most = [](int x, int y) { return max(x, y); };
                const int last = block_reduce(from >= a.top_p * z - tol ? (int)threadIdx.x : 0, sh.red_i, most);
                const int whole = block_reduce(from >= a.top_p * z + tol ? (int)threadIdx.x : 0, sh.red_i, most);
                r.sure = last + 2;
                r.border = whole - 1;
                const int at = bin_of(__builtin_amdgcn_exp2f(half_gap(r.l, 0.5f * bin_ref) * a.scale));
                done = reaches && at >= r.sure;
                r.unsure = reaches && at >= r.border;
            }
        }
    }
    if (threadIdx.x != 0) return;
    open[2 * b] = !done;  // for the first round of the later passes, and the second
    open[2 * b + 1] = 0;
    if (!done) state[b] = r;
    else if (tok == kNone) write_draw(a, b, -1, 0.0);
    else write_draw(a, b, tok, ((double)r.l - (double)top) / (double)a.temperature - log(z));
}

// Replaces what is no entry by -inf; whether the wave held such.  A finite sum of the four shows that all are.
DASH_DEV bool finite_or_low(f32x4_t& l) {
    const bool some = __any(!(fabsf((l[0] + l[1]) + (l[2] + l[3])) < INFINITY));
    if (some) {
#pragma unroll
        for (int j = 0; j < 4; ++j) l[j] = fabsf(l[j]) < INFINITY ? l[j] : -INFINITY;
    }
    return some;
}

// The draw over a stretch of a row, screened as in sampler.hip: thread and work-group state.
template <bool UNIT_T>
struct Drawing {
    float s = -INFINITY;
    int i = kNone;
    uint32_t step, uid;
    float inv_t;
    float* floor_s;  // lower bound on the best exact score that the work-group has seen

    // Clears the shared bound; the caller's next barrier is before the first score4.
    DASH_DEV Drawing(const Draw& a, int b, float* floor) : floor_s(floor) {
        step = (uint32_t)a.step[b];
        uid = (uint32_t)a.uid[b];
        inv_t = UNIT_T ? 1.f : div_rn(1.f, a.temperature);
        if (threadIdx.x == 0) *floor_s = -INFINITY;
    }
    // Entries i0 .. i0+3; those that are -inf (only if masked) take no part.
    DASH_DEV void score4(const Draw& a, const f32x4_t& l, int i0, bool masked) {
        // Relaxed: a stale bound is a lower one, and only more entries are evaluated.
        const float floor_w = __hip_atomic_load(floor_s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        uint32_t k0 = a.k0, k1 = a.k1;
        asm volatile("" : "+s"(k0), "+s"(k1));  // the round keys are derived here, not kept
        const U4 x = philox4x32_10(U4{(uint32_t)i0 >> 2, step, uid, 0u}, k0, k1);
        float sc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // l / T by a product and one corrected step, within the margin of the exact quotient, or
            // NaN where something overflows (then nothing is screened)
            const float q = l[j] * inv_t;
            sc[j] = UNIT_T ? l[j] : __builtin_fmaf(__builtin_fmaf(-q, a.temperature, l[j]), inv_t, q);
        }
        if (!UNIT_T && masked) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[j] = l[j] == -INFINITY ? -INFINITY : sc[j];
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
                const float e = (UNIT_T ? l[j] : div_rn(l[j], a.temperature)) + gumbel_from_bits(xs[j]);
                if (better(e, i0 + j, s, i)) {  // (a quotient that overflows to -inf still comes before none)
                    s = e;
                    i = i0 + j;
                }
                floor_t = fmaxf(floor_t, e);
            } else {
                floor_t = fmaxf(floor_t, sa - mg);
            }
        }
        const float f = wave_max_f(floor_t);
        if (f > floor_w && (threadIdx.x & 63) == 0)
            (void)__hip_atomic_fetch_max(floor_s, f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
};

// HIST: top_p < 1.  MINP: min_p > 0.  SPLIT: stretches of rows, left for draw_join.
template <bool UNIT_T, bool HIST, bool MINP, bool SPLIT>
__global__ void __launch_bounds__(kRowThreads, SPLIT ? 4 : 8)
draw_first(Draw a, RowSplit cut, FirstPart* __restrict__ part, uint32_t* __restrict__ hists, RowState* __restrict__ state,
           int* __restrict__ open) {
    __shared__ uint32_t hist[HIST ? kBins * kCopies : 1];
    __shared__ BestShared best;
    __shared__ SettleShared settled;
    __shared__ float red_f[kRowWaves];
    __shared__ float floor_s, top_s;
    __shared__ int far_s;
    const int b = SPLIT ? blockIdx.x / cut.n : blockIdx.x, n = SPLIT ? blockIdx.x % cut.n : 0;
    const float* row = a.logits + (int64_t)(a.row_of ? a.row_of[b] : b) * a.ld;
    Drawing<UNIT_T> draw(a, b, &floor_s);
    if (threadIdx.x == 0) {
        top_s = -INFINITY;
        far_s = 0;
    }
    if constexpr (HIST)
        for (int i = threadIdx.x; i < kBins * kCopies; i += kRowThreads) hist[i] = 0u;
    __syncthreads();
    const float min_gap = MINP ? (float)((double)a.temperature * a.log_min_p) : 0.f;
    const int copy = threadIdx.x & (kCopies - 1);
    float half = -0.5f * FLT_MAX, bins_at = NAN, top = -INFINITY;  // half: of the reference
    double z = 0.0;
    walk_row<2, true, false>(
        row, SPLIT ? n * cut.len : 0, SPLIT ? min(a.vocab, (n + 1) * cut.len) : a.vocab,
        [&](const f32x4_t (&buf)[2], int) {
            // The reference of the sums and of the bins: the largest of a sample of the row.
            float m = -INFINITY;
#pragma unroll
            for (int d = 0; d < 2; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) m = fmaxf(m, buf[d][j] < INFINITY ? buf[d][j] : -INFINITY);
            m = block_max_f(m, red_f);
            if (m == -INFINITY) return;
            half = 0.5f * m;
            if (HIST && fabsf(half * a.scale) < 16384.f) {  // (whole octaves: stretches share a grid of bins)
                const float at = rintf(half * a.scale), whole = octaves(at, a.temperature);
                if (fabsf(whole) < INFINITY) {  // (rounded up, it may lie past the largest float)
                    bins_at = at;
                    half = 0.5f * whole;
                }
            }
        },
        [&](f32x4_t l, int i) {
            bool masked = finite_or_low(l);
            const float m4 = max4(l);
            if (!__any(m4 > -INFINITY)) return;
            top = fmaxf(top, m4);
            const float above = half_gap(m4, half) * a.scale;
            const bool far = above >= (HIST ? (float)kBinsAbove : 40.f);
            if (__any(far)) {  // as in exp_push4; the histogram is void then
                if (far) {
                    z *= (double)__builtin_amdgcn_exp2f(-above);
                    half = 0.5f * m4;
                    far_s = 1;
                }
            }
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = __builtin_amdgcn_exp2f(half_gap(l[j], half) * a.scale);
            z += (double)((e[0] + e[1]) + (e[2] + e[3]));
            if constexpr (HIST) {
#pragma unroll
                for (int j = 0; j < 4; ++j) atomicAdd(&hist[bin_of(e[j]) * kCopies + copy], bin_term(e[j]));
            }
            if constexpr (MINP) {
                // No entry below the largest logit so far by more than the border's distance can be kept.
                float top_w = __hip_atomic_load(&top_s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                if (__any(m4 > top_w)) {
                    top_w = wave_max_f(m4);
                    if ((threadIdx.x & 63) == 0)
                        (void)__hip_atomic_fetch_max(&top_s, top_w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                }
                const float border = top_w + min_gap;
                const float low = border - fabsf(border) * 1e-6f - fabsf(min_gap) * 1e-6f;  // (not above it by rounding)
#pragma unroll
                for (int j = 0; j < 4; ++j) l[j] = l[j] < low ? -INFINITY : l[j];
                if (!__any(max4(l) > -INFINITY)) return;
                masked = true;
            }
            draw.score4(a, l, i, masked);
        },
        [](int) { return false; });
    block_best(draw.s, draw.i, best);
    top = block_max_f(top, red_f);
    const float ref = 2.f * half, at = block_max_f(z > 0.0 ? ref : -FLT_MAX, red_f);
    const double T = a.temperature;
    z = block_sum_d(z > 0.0 ? z * exp(((double)ref - (double)at) / T) : 0.0, settled.red);
    if (far_s) bins_at = NAN;
    uint32_t bin = 0;
    if constexpr (HIST) {
#pragma unroll
        for (int c = 0; c < kCopies; ++c) bin += hist[threadIdx.x * kCopies + c];
    }
    if constexpr (SPLIT) {
        if (HIST) hists[(int64_t)blockIdx.x * kBins + threadIdx.x] = bin;
        if (threadIdx.x == 0) part[blockIdx.x] = FirstPart{z, at, top, bins_at, draw.s, draw.i, 0};
    } else {
        const double by = exp(((double)at - (double)top) / T);  // sums relative to the largest logit
        settle(a, b, row, draw.i, top, z * by, bins_at == bins_at ? at : NAN, bin_mass(bin, threadIdx.x) * by, settled, state,
               open);
    }
}

// Joins the stretches of a row.
template <bool HIST>
__global__ void __launch_bounds__(kRowThreads)
draw_join(Draw a, const FirstPart* __restrict__ part, const uint32_t* __restrict__ hists, int parts,
          RowState* __restrict__ state, int* __restrict__ open) {
    __shared__ SettleShared settled;
    const int b = blockIdx.x, lane = threadIdx.x & 63;
    const float* row = a.logits + (int64_t)(a.row_of ? a.row_of[b] : b) * a.ld;
    part += (int64_t)b * parts;
    FirstPart p{0.0, -FLT_MAX, -INFINITY, NAN, -INFINITY, kNone, 0};
    if (lane < parts) p = part[lane];
    float top = p.top, s = p.s, ref = p.z > 0.0 ? p.ref : -FLT_MAX;
    int tok = p.i;
    // stretches without an entry have no part in the histogram
    const bool empty = !(p.z > 0.0);
    const bool whole = __all(lane >= parts || empty || p.bins_at == p.bins_at);
    float at = empty || p.bins_at != p.bins_at ? -FLT_MAX : p.bins_at;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        top = fmaxf(top, __shfl_xor(top, o, 64));
        ref = fmaxf(ref, __shfl_xor(ref, o, 64));
        at = fmaxf(at, __shfl_xor(at, o, 64));
        const float os = __shfl_xor(s, o, 64);
        const int oi = __shfl_xor(tok, o, 64);
        if (better(os, oi, s, tok)) {
            s = os;
            tok = oi;
        }
    }
    const double T = a.temperature;
    const double to_ref = p.z > 0.0 ? exp(((double)p.ref - (double)ref) / T) : 0.0;
    double z = p.z * to_ref;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) z += __shfl_xor(z, o, 64);
    const double by = exp(((double)ref - (double)top) / T);
    double bin = 0.0;
    if constexpr (HIST) {
        // Bins of all stretches lie on one grid; what lies below the row's lowest bin is left out.
        uint32_t sum[kMostParts];
        int from[kMostParts];
#pragma unroll
        for (int q = 0; q < kMostParts; ++q) {
            const float theirs = __shfl(p.bins_at, q, 64);
            from[q] = kBins;
            if (q < parts && !__shfl((int)empty, q, 64) && theirs == theirs)
                from[q] = (int)threadIdx.x + (int)fminf((at - theirs) * (float)kBinsPerOctave, (float)kBins);
            sum[q] = from[q] < kBins ? hists[((int64_t)b * parts + q) * kBins + from[q]] : 0;
        }
#pragma unroll
        for (int q = 0; q < kMostParts; ++q) bin += bin_mass(sum[q], from[q]) * __shfl(to_ref, q, 64);
        bin *= by;
    }
    settle(a, b, row, tok, top, z * by, whole ? octaves(at, a.temperature) : NAN, bin, settled, state,
           open);
}

// Over entries [lo, hi) of a row: the float32 mass that comes before the winner w.tok, and the draw over
// what comes before it and can be kept, in every thread.
template <int NT, bool UNIT_T>
DASH_DEV double draw_before(const Draw& a, int b, const float* row, int lo, int hi, const RowState& w, float* floor_s,
                            BestShared& best, double* red, float& s, int& tok) {
    __syncthreads();
    Drawing<UNIT_T> draw(a, b, floor_s);
    __syncthreads();
    double mass = 0.0;
    const float half_top = 0.5f * w.top, half_bins = 0.5f * w.bin_ref;
    // the least exponential of the border's bin (bin 0 holds all below it, too)
    const float border = w.bin_ref == w.bin_ref && w.border > 0 ? __uint_as_float((kBinBase + w.border) << 18) : 0.f;
    walk_row<2, false, NT>(row, lo, hi, [&](f32x4_t l, int i) {
        finite_or_low(l);
        if (!__any(max4(l) >= w.l)) return;
        float e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            l[j] = l[j] > w.l || (l[j] == w.l && i + j < w.tok) ? l[j] : -INFINITY;
            e[j] = __builtin_amdgcn_exp2f(half_gap(l[j], half_top) * a.scale);
        }
        mass += (double)((e[0] + e[1]) + (e[2] + e[3]));
#pragma unroll
        for (int j = 0; j < 4; ++j)
            l[j] = l[j] < w.low || __builtin_amdgcn_exp2f(half_gap(l[j], half_bins) * a.scale) < border ? -INFINITY : l[j];
        if (__any(max4(l) > -INFINITY)) draw.score4(a, l, i, true);
    });
    s = draw.s;
    tok = draw.i;
    block_best<NT>(s, tok, best);
    return block_sum_d<NT>(mass, red);
}

// The later passes have work-groups of kLater threads: with 1024 the last one needed more registers than
// there are, and a launch with scratch memory took 20 us with nothing to do.  They take rows by chunks.
constexpr int kLater = 512, kChunk = 1024;
// The rows that are open in a round (0 or 1) among rows [first, first + kChunk), in order; returns their number.
DASH_DEV int open_rows(const int* open, int round, int first, int rows, int* list, int* red) {
    constexpr int kOwn = kChunk / kLater;
    const int r = first + kOwn * (int)threadIdx.x;
    int mine[kOwn], sum = 0, total;
#pragma unroll
    for (int o = 0; o < kOwn; ++o) sum += mine[o] = r + o < rows && open[2 * (r + o) + round];
    int at = block_scan<kLater>(sum, red, total) - sum;
#pragma unroll
    for (int o = 0; o < kOwn; ++o)
        if (mine[o]) list[at++] = r + o;
    __syncthreads();
    return total;
}
// Stretches per open row: as many as its chunk of rows leaves work-groups for.
DASH_DEV int open_cuts(int n, int most) { return max(1, min(most, (int)gridDim.x / max(n, 1))); }

template <bool UNIT_T>
__global__ void __launch_bounds__(kLater)
draw_second(Draw a, int rows, const RowState* __restrict__ state, const int* __restrict__ open, int round,
            int most, SecondPart* __restrict__ second, int* __restrict__ cuts_of) {
    __shared__ BestShared best;
    __shared__ double red_d[kLater / 64];
    __shared__ int list[kChunk], red_i[kLater / 64];
    __shared__ float floor_s;
    for (int first = 0; first < rows; first += kChunk) {
        __syncthreads();
        const int n = open_rows(open, round, first, rows, list, red_i);
        const int cuts = open_cuts(n, most), len = ((a.vocab + cuts - 1) / cuts + 3) & ~3;
        for (int item = blockIdx.x; item < n * cuts; item += gridDim.x) {
            const int b = list[item / cuts], lo = min(a.vocab, item % cuts * len);
            const float* row = a.logits + (int64_t)(a.row_of ? a.row_of[b] : b) * a.ld;
            const RowState w = state[b];
            float s;
            int tok;
            const double before = draw_before<kLater, UNIT_T>(a, b, row, lo, min(a.vocab, lo + len), w, &floor_s, best, red_d, s, tok);
            if (threadIdx.x == 0) {
                second[(int64_t)b * most + item % cuts] = SecondPart{before, s, tok};
                cuts_of[b] = cuts;  // (the same from every stretch)
            }
        }
    }
}

// Whether the mass before (l, i) is below top_p of the row's, in float64 throughout.
DASH_DEV bool kept_exactly(const Draw& a, const float* row, float l0, int i0, float top, double* red) {
    double before = 0.0, all = 0.0;
    walk_row<2, false, kLater>(row, 0, a.vocab, [&](const f32x4_t& l, int i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (!(fabsf(l[j]) < INFINITY)) continue;
            const double e = exp(((double)l[j] - (double)top) / (double)a.temperature);
            all += e;
            if (l[j] > l0 || (l[j] == l0 && i + j < i0)) before += e;
        }
    });
    before = block_sum_d<kLater>(before, red);
    all = block_sum_d<kLater>(all, red);
    return before < a.top_p * all;
}

// LAST: rows that are still in doubt take further passes here; otherwise they stay open for another round.
template <bool UNIT_T, bool LAST>
__global__ void __launch_bounds__(kLater)
draw_last(Draw a, int rows, RowState* __restrict__ state, int* __restrict__ open, int round, int most,
          const SecondPart* __restrict__ second, const int* __restrict__ cuts_of) {
    __shared__ BestShared best;
    __shared__ double red_d[kLater / 64];
    __shared__ int list[kChunk], red_i[kLater / 64];
    __shared__ float floor_s;
    for (int first = 0; first < rows; first += kChunk) {
        __syncthreads();
        const int n = open_rows(open, round, first, rows, list, red_i);
        for (int item = blockIdx.x; item < n; item += gridDim.x) {
            const int b = list[item], cuts = cuts_of[b], lane = threadIdx.x & 63;
            const float* row = a.logits + (int64_t)(a.row_of ? a.row_of[b] : b) * a.ld;
            RowState w = state[b];
            double before = 0.0;
            float s = -INFINITY;
            int next = kNone;
            if (lane < cuts) {
                const SecondPart p = second[(int64_t)b * most + lane];
                before = p.before;
                s = p.s;
                next = p.i;
            }
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) {
                before += __shfl_xor(before, o, 64);
                const float os = __shfl_xor(s, o, 64);
                const int oi = __shfl_xor(next, o, 64);
                if (better(os, oi, s, next)) {
                    s = os;
                    next = oi;
                }
            }
            bool ended = true;
            for (;;) {
                bool kept = false;
                if (w.unsure) {
                    kept = before < a.top_p * w.z;
                    if (fabs(before - a.top_p * w.z) <= kMassTol * w.z) kept = kept_exactly(a, row, w.l, w.tok, w.top, red_d);
                }
                if (kept || next == kNone) break;  // (the first token of the order is kept: there is a next one)
                if constexpr (LAST && !UNIT_T) {
                    // A winner whose quotient overflows has no noise: the draws go down the row index by index, as many
                    // passes as there are such logits in ascending order.  The largest one's quotient overflows with it, any
                    // other logit is 2^103 T below that and without mass, so what is kept is among the entries equal
                    // to the largest, and the first of these is drawn.
                    if (fabsf(div_rn(w.l, a.temperature)) == INFINITY) {
                        w.l = value_below(top_key(w.top));
                        w.tok = 0;
                        draw_before<kLater, UNIT_T>(a, b, row, 0, a.vocab, w, &floor_s, best, red_d, s, next);
                        w.tok = next;
                        w.l = row[next];
                        break;
                    }
                }
                w.tok = next;
                w.l = row[next];
                if (a.top_p >= 1.0 || kept_by_own_mass(a, w.l, w.top, w.z)) break;
                if (w.bin_ref == w.bin_ref && bin_of(__builtin_amdgcn_exp2f(half_gap(w.l, 0.5f * w.bin_ref) * a.scale)) >= w.sure) break;
                w.unsure = 1;
                if constexpr (!LAST) {
                    ended = false;
                    break;
                }
                before = draw_before<kLater, UNIT_T>(a, b, row, 0, a.vocab, w, &floor_s, best, red_d, s, next);
            }
            if constexpr (!LAST) __syncthreads();  // every wave has read the row's state
            if (threadIdx.x != 0) continue;
            if (!ended) {
                state[b] = w;
                open[2 * b + 1] = 1;
            } else {
                write_draw(a, b, w.tok, ((double)w.l - (double)w.top) / (double)a.temperature - log(w.z));
            }
        }
    }
}

constexpr int kMostCuts = 64;   // in the second: a wave joins them
struct DrawPlan {
    RowSplit first;
    int most;  // room for stretches of the second pass, per row
    size_t hists, parts, states, seconds, opens, bytes;  // offsets in the workspace
};
// The number of stretches is 256 / rows, rounded down, so times step up where it changes: peaked rows of 151,936 at
// top_p = 0.95 take 62 us for 128, 71 for 129, 78 for 256, 99 for 257, 118 for 512, 135 for 513.
DrawPlan draw_plan(int rows, int vocab) {
    DrawPlan p;
    const int n = std::max(rows, 1);
    p.first = split_row(vocab, std::min({kMostParts, kSplitTarget / n, vocab / kDrawStretch}));
    p.most = std::max(1, std::min({kMostCuts, std::max(kDrawTarget / n, 8), vocab / kDrawStretch}));
    const size_t stretches = p.first.n > 1 ? (size_t)n * p.first.n : 0;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 15) / 16 * 16;
        return here;
    };
    p.hists = take(stretches * kBins * sizeof(uint32_t));
    p.parts = take(stretches * sizeof(FirstPart));
    p.states = take(n * sizeof(RowState));
    p.seconds = take((size_t)n * p.most * sizeof(SecondPart));
    p.opens = take(3 * (size_t)n * sizeof(int));
    p.bytes = at;
    return p;
}

}  // namespace

size_t sample_truncated_workspace_bytes(int rows, int vocab, int top_k) {
    if (top_k > 0 && top_k < vocab) return top_workspace_bytes(rows, vocab, top_k);
    return draw_plan(rows, vocab).bytes;
}

hipError_t launch_sample_truncated(const float* logits, int64_t ld, int rows, int vocab, const int32_t* row_of,
                                   const int32_t* uid, const int32_t* step, float temperature, int top_k, double top_p,
                                   double min_p, uint64_t seed, int32_t* tok_out, float* lp_out, uint32_t* status,
                                   void* ws, hipStream_t st) {
    if (rows <= 0) return hipSuccess;
    const Draw a{logits, ld, vocab, row_of, uid, step, temperature, exp2_scale(temperature), top_k, top_p,
                 log(min_p), (uint32_t)seed, (uint32_t)(seed >> 32), tok_out, lp_out, status};
    auto launch = [&](auto unit) -> hipError_t {
        constexpr bool U = decltype(unit)::value;
        if (top_k > 0 && top_k < vocab) {
            TopParts parts;
            if (hipError_t e = launch_top_parts(logits, ld, rows, vocab, row_of, top_k, temperature,
                                                top_plan(rows, vocab, top_k), ws, parts, st))
                return e;
            top_join_variant(top_k, [&](auto threads, auto per) {
                constexpr int NT = decltype(threads)::value, PER = decltype(per)::value;
                draw_top_k<U, NT, PER><<<rows, NT, 0, st>>>(a, parts);
            });
            return hipGetLastError();
        }
        const DrawPlan p = draw_plan(rows, vocab);
        char* at = (char*)ws;
        uint32_t* hists = (uint32_t*)(at + p.hists);
        FirstPart* parts = (FirstPart*)(at + p.parts);
        RowState* state = (RowState*)(at + p.states);
        SecondPart* second = (SecondPart*)(at + p.seconds);
        int* open = (int*)(at + p.opens);
        int* cuts_of = open + 2 * (size_t)rows;
        auto first = [&](auto hist, auto minp) {
            constexpr bool H = decltype(hist)::value, M = decltype(minp)::value;
            if (p.first.n == 1) {
                draw_first<U, H, M, false><<<rows, kRowThreads, 0, st>>>(a, p.first, parts, hists, state, open);
            } else {
                draw_first<U, H, M, true><<<rows * p.first.n, kRowThreads, 0, st>>>(a, p.first, parts, hists, state, open);
                draw_join<H><<<rows, kRowThreads, 0, st>>>(a, parts, hists, p.first.n, state, open);
            }
        };
        const bool hist = top_p < 1.0 && vocab <= kHistVocab;
        if (hist && min_p > 0.0) first(std::true_type{}, std::true_type{});
        else if (hist) first(std::true_type{}, std::false_type{});
        else if (min_p > 0.0) first(std::false_type{}, std::true_type{});
        else first(std::false_type{}, std::false_type{});
        if (top_p < 1.0 || min_p > 0.0) {  // (otherwise every row has ended)
            const int grid = std::min(rows, kDrawTarget / 2);
            // Of many rows one is likely to need a third pass, which takes one work-group as long as all the rest:
            // a second round costs 9 us and leaves that to few calls.
            const bool again = rows >= 256;
            draw_second<U><<<kDrawTarget, kLater, 0, st>>>(a, rows, state, open, 0, p.most, second, cuts_of);
            if (again) {
                draw_last<U, false><<<grid, kLater, 0, st>>>(a, rows, state, open, 0, p.most, second, cuts_of);
                draw_second<U><<<kDrawTarget, kLater, 0, st>>>(a, rows, state, open, 1, p.most, second, cuts_of);
            }
            draw_last<U, true><<<grid, kLater, 0, st>>>(a, rows, state, open, again, p.most, second, cuts_of);
        }
        return hipGetLastError();
    };
    return temperature == 1.0f ? launch(std::true_type{}) : launch(std::false_type{});
}

}  // namespace dash
