// Distillation from a teacher's K largest logits: the loss of every row of student logits, and its
// gradient.
//
// With p the teacher's probabilities of its K tokens and of all others together (the rest), and q
// the student's probabilities of the same outcomes, softmax at temperature T,
//   loss = sum p ln(p / q),
//   T dloss/ds_j = q_j - p_j for a teacher's token j,  (q_rest - p_rest) r_j for any other,
// r_j = q_j / q_rest its share of the others.
// A teacher without a rest has p_rest = 0: its K tokens renormalised, and q_j for every other token.
//
// q_rest is the sum over the other tokens themselves, not one minus the K tokens' mass, which
// loses every digit where a student is sure of itself: a bit per entry of a stretch of the row, in
// LDS, says which entries are the teacher's.  The K tokens' terms are float64 (one per thread), and
// an error of the rest's sum moves the loss by (q_rest - p_rest) times it only, since q is
// normalised with the same sum.
//
// Memory bounds all of it: the loss reads a row once (2048 rows of 151,936: 195 us, 6.4 TB/s), the
// gradient reads and writes one (701 x 50,257 in float32: 66 us, 4.3 TB/s), and both in one launch read
// and write one (2048 x 151,936 with bf16 gradients, a tenth of the rows without weight: 441 us).  Rows
// that are not read again and gradients go past the caches (217 and 477 us without).
#include <algorithm>

#include "kernels.h"
#include "row_walk.h"

namespace dash {

namespace {

// Work-groups that fill the GPU (four per CU for the loss, twice that for the gradient) and the least
// entries of a stretch.
constexpr int kDistillTarget = 1024, kDistillStretch = 4096, kGradTarget = 2048;
constexpr int kStretch = 1 << 18;  // entries of a row whose bits are in LDS at a time (32 KB)

// Work-groups that stream a row have kWide threads, four of them to a CU (2048 rows of 151,936 with 1024
// threads: 263 us, with 512 217); the one that joins a row's stretches has kNarrow: its reductions are
// over few entries (16 rows: 25 us a call with 1024, with 128 the host's 18).
constexpr int kWide = 512, kNarrow = 128;
template <int NT>
struct DistillShared {
    double red_d[NT / 64];
    float red_f[NT / 64];
    int twice;
};
struct MarkShared {
    uint32_t bits[kStretch / 32];
};

// The teacher of a row: a thread holds entries threadIdx.x, threadIdx.x + NT, ...
constexpr int kMostEntries = 1024;
template <int NT>
struct Teacher {
    static constexpr int kOwn = kMostEntries / NT;
    int idx[kOwn];      // token, -1: no entry
    float val[kOwn];
    double top, lz;     // ln p of an entry is val / T - top - lz
    double rest_lp, rest_p;
    int own;            // entries per thread that there may be
    bool none;          // no mass at all: the row has no teacher
    DASH_DEV double lp(int e, double T) const { return (double)val[e] / T - top - lz; }
};
template <int NT>
DASH_DEV void load_tokens(const DistillArgs& a, int64_t r, Teacher<NT>& t) {
    t.own = (a.k + NT - 1) / NT;
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e) {
        t.idx[e] = -1;
        t.val[e] = -INFINITY;
        const int k = e * NT + (int)threadIdx.x;
        if (k < a.k) {
            const int i = a.t_idx[r * a.k + k];
            const float v = a.t_val[r * a.k + k];
            if (i >= 0 && i < a.vocab) {
                t.idx[e] = i;
                t.val[e] = v;
            }
        }
    }
}
template <int NT>
DASH_DEV void normalise(const DistillArgs& a, int64_t r, Teacher<NT>& t, DistillShared<NT>& sh) {
    const double T = a.temperature;
    const double rest = a.t_rest ? (double)a.t_rest[r] : -INFINITY;
    // (a NaN is dropped by the maximum and comes back through the sum)
    float most = t.val[0];
#pragma unroll
    for (int e = 1; e < t.kOwn; ++e) most = fmaxf(most, t.val[e]);
    t.top = fmax((double)block_max_f<NT>(most, sh.red_f) / T, rest);
    if (t.top == -INFINITY) t.top = 0.0;
    double z = 0.0;
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e)
        if (e < t.own) z += exp((double)t.val[e] / T - t.top);
    z = block_sum_d<NT>(z, sh.red_d) + exp(rest - t.top);
    t.none = z == 0.0;
    t.lz = t.none ? 0.0 : log(z);
    t.rest_lp = rest - t.top - t.lz;
    t.rest_p = exp(t.rest_lp);
}

// Bits of the entries [base, base + n) that are the teacher's; an index that occurs twice is noted.
template <int NT>
DASH_DEV void mark_tokens(MarkShared& mark, int& twice, const Teacher<NT>& t, int base, int n) {
    __syncthreads();
    for (int i = threadIdx.x; i < (n + 31) >> 5; i += NT) mark.bits[i] = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e)
        if (t.idx[e] >= base && t.idx[e] < base + n) {
            const uint32_t bit = 1u << ((t.idx[e] - base) & 31);
            if (atomicOr(&mark.bits[(t.idx[e] - base) >> 5], bit) & bit) twice = 1;
        }
    __syncthreads();
}

// Sums of e^((s - top) / T) over all tokens and of e^((s - top_rest) / T) over the others.  Each has
// its own reference: where the student is sure of the teacher's tokens the others underflow
// relative to the row, but not among themselves, and p_rest is still spread over them.
struct Norm {
    float top, z, top_rest, z_rest;  // z_rest 0: no others
};

// Sum over the entries [lo, hi) that are not the teacher's; notes an index that occurs twice.
template <int NT>
DASH_DEV ExpSum sum_others(const DistillArgs& a, const float* row, const Teacher<NT>& t, int lo, int hi, MarkShared& mark,
                           int& twice) {
    ExpSum sum;
    if (threadIdx.x == 0) twice = 0;
    for (int base = lo; base < hi; base += kStretch) {
        const int end = min(hi, base + kStretch);
        walk_row<4, false, true, NT>(
            row, base, end,
            [&](const f32x4_t (&)[4], int) { mark_tokens(mark, twice, t, base, end - base); },  // (the first loads are under way)
            [&](f32x4_t l, int i) {
                const int at = min(i - base, kStretch - 4);
                const uint32_t mine = (mark.bits[at >> 5] >> (at & 31)) & 15u;
                if (__any(mine != 0)) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (mine >> j & 1u) l[j] = -INFINITY;
                }
                exp_push4<true>(sum, l, max4(l), a.scale, a.scale_low);
            },
            [](int) { return false; });
    }
    return sum;
}

// The student's logits of the thread's tokens (0 where it has none).
template <int NT>
DASH_DEV void load_student(const float* row, const Teacher<NT>& t, float (&s)[Teacher<NT>::kOwn]) {
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e) s[e] = t.idx[e] >= 0 ? row[t.idx[e]] : 0.f;
}

// Loss of a row (in every thread) and its normaliser, from the threads' sums over the other tokens.
template <int NT>
DASH_DEV float row_loss(const DistillArgs& a, const Teacher<NT>& t, const float (&s)[Teacher<NT>::kOwn], const ExpSum& sum,
                        bool twice, DistillShared<NT>& sh, Norm& n) {
    const double T = a.temperature;
    const double zr = block_exp_sum<NT>(sum, T, sh.red_f, sh.red_d, n.top_rest);
    float most = -INFINITY;
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e)
        if (t.idx[e] >= 0) most = fmaxf(most, s[e]);
    n.top = fmaxf(block_max_f<NT>(most, sh.red_f), zr > 0.0 ? n.top_rest : -INFINITY);
    const double top = n.top;
    double zs = 0.0;
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e)
        if (t.idx[e] >= 0) zs += exp(((double)s[e] - top) / T);
    zs = block_sum_d<NT>(zs, sh.red_d);
    const double far = ((double)n.top_rest - top) / T;  // <= 0, and 0 only counts with a rest
    double z = zs + (zr == 0.0 ? 0.0 : zr * exp(far));
    // a row of -inf alone has no distribution, and an index that occurs twice no meaning
    if (twice || top == -INFINITY) z = NAN;
    const double lz = log(z);
    double d = 0.0;
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e)
        if (t.idx[e] >= 0) {
            const double lp = t.lp(e, T), p = exp(lp);
            if (p != 0.0) d += p * (lp - (((double)s[e] - top) / T - lz));
        }
    d = block_sum_d<NT>(d, sh.red_d);
    if (t.rest_p != 0.0) d += t.rest_p * (t.rest_lp - (far + log(zr) - lz));
    n.z = (float)z;
    n.z_rest = (float)zr;
    return t.none ? 0.f : (float)d;
}

// Four gradient entries.
template <class G>
DASH_DEV void store4(G* p, const float (&v)[4], int n);
template <>
DASH_DEV void store4<float>(float* p, const float (&v)[4], int n) {
    if (n >= 4) {
        __builtin_nontemporal_store(f32x4_t{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4u_t*>(p));
    } else {
        for (int j = 0; j < n; ++j) p[j] = v[j];
    }
}
template <>
DASH_DEV void store4<bf16_t>(bf16_t* p, const float (&v)[4], int n) {
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    typedef u32x2_t u32x2u_t __attribute__((aligned(2)));
    if (n >= 4) {
        __builtin_nontemporal_store(u32x2_t{f2bf2(v[0], v[1]), f2bf2(v[2], v[3])}, reinterpret_cast<u32x2u_t*>(p));
    } else {
        for (int j = 0; j < n; ++j) p[j] = f2bf(v[j]);
    }
}
DASH_DEV void store1(float* p, float v) { *p = v; }
DASH_DEV void store1(bf16_t* p, float v) { *p = f2bf(v); }

// Gradient of a row's entries [lo, hi), w = its weight / T.  grad may be the row itself: a thread reads
// its entries before it writes them, and the teacher's tokens (s, read before) are written last.
struct GradTerms {
    float half, f, up;  // half: top_rest / 2; an other token's gradient: e^((s - top_rest) / T) 2^up f
};
template <int NT>
DASH_DEV GradTerms grad_terms(const DistillArgs& a, const Teacher<NT>& t, const float (&s)[Teacher<NT>::kOwn],
                              const Norm& n, double w, int lo, int hi, float (&g)[Teacher<NT>::kOwn]) {
    const double T = a.temperature;
    double f = 0.0;
    int up = 0;
    if (n.z_rest != 0.f) {
        const double q_rest = exp(((double)n.top_rest - (double)n.top) / T) * (double)n.z_rest / (double)n.z;
        f = w * (q_rest - t.rest_p) / (double)n.z_rest;
        // A factor past the largest float (w is, at T < 3e-39) would make 0 times it NaN: its powers of two join the exponent.
        if (fabs(f) > (double)FLT_MAX && fabs(f) < (double)INFINITY) {
            up = ilogb(f) - 126;
            f = ldexp(f, -up);
        }
    }
    if (n.z != n.z) f = n.z;
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e) {
        g[e] = 0.f;
        if (t.idx[e] >= lo && t.idx[e] < hi)
            g[e] = (float)(w * (exp(((double)s[e] - (double)n.top) / T) / (double)n.z - exp(t.lp(e, T))));
        asm volatile("" : "+v"(g[e]));  // s has arrived before any entry is written
    }
    return {0.5f * n.top_rest, (float)f, (float)up};
}
DASH_DEV void grad4(const DistillArgs& a, const GradTerms& q, const f32x4_t& l, float (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float d = half_gap(l[j], q.half);
        v[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(d, a.scale, __builtin_fmaf(fmaxf(d, -FLT_MAX), a.scale_low, q.up))) * q.f;
    }
}
template <int NT, class G>
DASH_DEV void store_tokens(G* grad, const Teacher<NT>& t, const float (&g)[Teacher<NT>::kOwn], int lo, int hi) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e)
        if (t.idx[e] >= lo && t.idx[e] < hi) store1(grad + t.idx[e], g[e]);
}
template <int NT, class G>
DASH_DEV void row_grad(const DistillArgs& a, const float* row, G* grad, int lo, int hi, const Teacher<NT>& t,
                       const float (&s)[Teacher<NT>::kOwn], const Norm& n, double w) {
    float g[Teacher<NT>::kOwn];
    const GradTerms q = grad_terms(a, t, s, n, w, lo, hi, g);
    __syncthreads();
    walk_row<4, true, NT>(row, lo, hi, [&](const f32x4_t& l, int i) {
        float v[4];
        grad4(a, q, l, v);
        store4(grad + i, v, hi - i);
    });
    store_tokens(grad, t, g, lo, hi);
}

template <int NT, class G>
DASH_DEV void zero_row(G* grad, int lo, int hi) {
    const float zero[4] = {};
    for (int i = lo + 4 * (int)threadIdx.x; i < hi; i += 4 * NT) store4(grad + i, zero, hi - i);
}

// Sum over the other tokens of one stretch of a row.
struct DistillPart {
    double z;
    float ref;
    int twice;
};
__global__ void __launch_bounds__(kWide, 8)
distill_part_k(DistillArgs a, RowSplit cut, DistillPart* __restrict__ part) {
    __shared__ DistillShared<kWide> sh;
    __shared__ MarkShared mark;
    const int64_t r = blockIdx.x / cut.n;
    const int lo = (int)(blockIdx.x % cut.n) * cut.len, hi = min(a.vocab, lo + cut.len);
    if (a.weight && a.weight[r] == 0.f) return;
    Teacher<kWide> t;
    load_tokens(a, r, t);
    const ExpSum sum = sum_others(a, a.logits + r * a.ld, t, lo, hi, mark, sh.twice);
    float ref;
    const double z = block_exp_sum<kWide>(sum, a.temperature, sh.red_f, sh.red_d, ref);
    if (threadIdx.x == 0) part[blockIdx.x] = DistillPart{z, ref, sh.twice};
}

DASH_DEV void write_norm(const DistillArgs& a, int64_t r, const Norm& n) {
    *reinterpret_cast<f32x4u_t*>(a.norm + 4 * r) = f32x4_t{n.top, n.z, n.top_rest, n.z_rest};
}

// A row per work-group.  A row of weight 0 has loss 0.
__global__ void __launch_bounds__(kWide, 8)
distill_loss_k(DistillArgs a) {
    __shared__ DistillShared<kWide> sh;
    __shared__ MarkShared mark;
    const int64_t r = blockIdx.x;
    const float* row = a.logits + r * a.ld;
    if (a.weight && a.weight[r] == 0.f) {
        if (threadIdx.x == 0) a.loss[r] = 0.f;
        return;
    }
    Teacher<kWide> t;
    float s[t.kOwn];
    load_tokens(a, r, t);
    const ExpSum sum = sum_others(a, row, t, 0, a.vocab, mark, sh.twice);
    normalise(a, r, t, sh);
    load_student(row, t, s);
    Norm n;
    const float loss = row_loss(a, t, s, sum, sh.twice, sh, n);
    if (threadIdx.x != 0) return;
    a.loss[r] = loss;
    write_norm(a, r, n);
}

// Joins the stretches of a row.
__global__ void __launch_bounds__(kNarrow)
distill_join_k(DistillArgs a, const DistillPart* __restrict__ part, int parts) {
    __shared__ DistillShared<kNarrow> sh;
    const int64_t r = blockIdx.x;
    if (a.weight && a.weight[r] == 0.f) {
        if (threadIdx.x == 0) a.loss[r] = 0.f;
        return;
    }
    Teacher<kNarrow> t;
    float s[t.kOwn];
    DistillPart p{0.0, -FLT_MAX, 0};
    if ((int)threadIdx.x < parts) p = part[r * parts + threadIdx.x];
    load_tokens(a, r, t);
    load_student(a.logits + r * a.ld, t, s);
    normalise(a, r, t, sh);
    ExpSum sum;
    if (p.z != 0.0) {
        sum.z = p.z;
        sum.half = 0.5f * p.ref;
    }
    Norm n;
    const float loss = row_loss(a, t, s, sum, __syncthreads_or(p.twice), sh, n);
    if (threadIdx.x != 0) return;
    a.loss[r] = loss;
    write_norm(a, r, n);
}

// One stretch of a row per work-group.
template <class G>
__global__ void __launch_bounds__(kWide, 8)
distill_grad_k(DistillArgs a, RowSplit cut) {
    __shared__ DistillShared<kWide> sh;
    const int64_t r = blockIdx.x / cut.n;
    const int lo = (int)(blockIdx.x % cut.n) * cut.len, hi = min(a.vocab, lo + cut.len);
    const float* row = a.logits + r * a.ld;
    G* grad = (G*)a.grad + r * a.ld_grad;
    const float weight = a.weight ? a.weight[r] : 1.f;
    if (weight == 0.f) return zero_row<kWide>(grad, lo, hi);
    Teacher<kWide> t;
    float s[t.kOwn];
    load_tokens(a, r, t);
    normalise(a, r, t, sh);
    if (t.none) return zero_row<kWide>(grad, lo, hi);
#pragma unroll
    for (int e = 0; e < t.kOwn; ++e) s[e] = t.idx[e] >= lo && t.idx[e] < hi ? row[t.idx[e]] : 0.f;
    const Norm n{a.norm[4 * r], a.norm[4 * r + 1], a.norm[4 * r + 2], a.norm[4 * r + 3]};
    row_grad(a, row, grad, lo, hi, t, s, n, (double)weight / (double)a.temperature);
}

// Loss and gradient of a row by one work-group, a CU to itself.  Both passes need the row, 608 KB of
// 151,936 entries; two of them per CU, in flight on 256 CUs, are more than the last-level cache holds, and
// with one the second reading still cost as much as the first (512 us for 2048 rows, 595 with
// two, 477 with what follows, 441 past the caches).  So the work-group keeps what it can: kInRegs tiles in the threads' registers (two waves per
// SIMD leave each 256) and kInLds in LDS; only the rest, a quarter of such a row, is read again.
// Every thread meets its entries in distill_loss_k's order: the same sums, bit for bit.
constexpr int kInRegs = 44, kInLds = 14;
struct KeepShared {
    f32x4_t tile[kInLds][kWide];
};
template <class G>
__global__ void __launch_bounds__(kWide, 2)
distill_loss_grad_k(DistillArgs a) {
    constexpr int kTile = 4 * kWide;
    __shared__ DistillShared<kWide> sh;
    __shared__ MarkShared mark;
    __shared__ KeepShared keep;
    const int64_t r = blockIdx.x;
    const float* row = a.logits + r * a.ld;
    G* grad = (G*)a.grad + r * a.ld_grad;
    const float weight = a.weight ? a.weight[r] : 1.f;
    if (weight == 0.f) {
        if (threadIdx.x == 0) a.loss[r] = 0.f;
        return zero_row<kWide>(grad, 0, a.vocab);
    }
    const int whole = a.vocab / kTile, at = 4 * (int)threadIdx.x;
    f32x4_t in[kInRegs];
#pragma unroll
    for (int d = 0; d < kInRegs; ++d)
        if (d < whole) in[d] = load_row4<true>(row, at + d * kTile);
    Teacher<kWide> t;
    float s[t.kOwn];
    load_tokens(a, r, t);
    if (threadIdx.x == 0) sh.twice = 0;
    mark_tokens(mark, sh.twice, t, 0, a.vocab);
    ExpSum sum;
    auto push = [&](f32x4_t l, int i) {
        const int b = min(i, kStretch - 4);
        const uint32_t mine = (mark.bits[b >> 5] >> (b & 31)) & 15u;
        if (__any(mine != 0)) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (mine >> j & 1u) l[j] = -INFINITY;
        }
        exp_push4<true>(sum, l, max4(l), a.scale, a.scale_low);
    };
#pragma unroll
    for (int d = 0; d < kInRegs; ++d)
        if (d < whole) push(in[d], at + d * kTile);
    const int from_lds = min(kInRegs, whole), from_row = min(kInRegs + kInLds, whole) * kTile;
    walk_row<4, false, kWide>(row, from_lds * kTile, from_row, [&](const f32x4_t& l, int i) {
        push(l, i);
        keep.tile[(i - at) / kTile - kInRegs][threadIdx.x] = l;
    });
    walk_row<4, false, kWide>(row, from_row, a.vocab, push);
    normalise(a, r, t, sh);
    if (t.none) {
        if (threadIdx.x == 0) a.loss[r] = 0.f;
        return zero_row<kWide>(grad, 0, a.vocab);
    }
    load_student(row, t, s);
    Norm n;
    const float loss = row_loss(a, t, s, sum, sh.twice, sh, n);
    if (threadIdx.x == 0) a.loss[r] = loss;
    float g[t.kOwn];
    const GradTerms q = grad_terms(a, t, s, n, (double)weight / (double)a.temperature, 0, a.vocab, g);
    __syncthreads();  // every thread has its tokens' logits: entries may be written
    auto write = [&](const f32x4_t& l, int i) {
        float v[4];
        grad4(a, q, l, v);
        store4(grad + i, v, a.vocab - i);
    };
    walk_row<4, false, kWide>(row, from_row, a.vocab, write);
#pragma unroll
    for (int d = 0; d < kInRegs; ++d)
        if (d < whole) write(in[d], at + d * kTile);
    for (int d = from_lds; d < from_row / kTile; ++d) write(keep.tile[d - kInRegs][threadIdx.x], at + d * kTile);
    store_tokens(grad, t, g, 0, a.vocab);
}

// Rows are cut where there are fewer of them than work-groups that fill the GPU.  From 513 on they are whole, with the
// first loads and the float64 sums at the end exposed once: 512 rows of 50,257 27 us, 513 30, 701 33, 1024 43; of
// 151,936 56, 67, 76, 102.
RowSplit loss_split(int rows, int vocab) {
    return split_row(vocab, std::min({64, kDistillTarget / std::max(rows, 1), vocab / kDistillStretch}));
}

// One work-group for loss and gradient of a row: where there are rows for every CU, the row's marks are in
// LDS at once, and what is not read again outweighs that a CU has one work-group instead of
// four.  2048 rows, pair of launches / one: 32,768 entries 159 / 164 us in float32 and 133 / 159 in bf16,
// 50,257 263 / 237 and 216 / 216, 80,000 360 / 311 and 293 / 282, 151,936 721 / 545 and 556 / 438; 706 47 / 87.
// Fewer rows, in float32: 513 of 50,257 79 / 82, 600 91 / 86, 769 111 / 112, 1024 136 / 125; 513 of 151,936 205 / 172,
// 769 279 / 232, in bf16 174 / 149 and 229 / 201.  So a round of 256 work-groups that is begun costs the one launch
// 4% at most.
bool fused(int rows, int vocab, bool bf16) {
    return loss_split(rows, vocab).n == 1 && vocab >= (bf16 ? 1 << 16 : 40960) && vocab <= kStretch;
}

}  // namespace

size_t distill_workspace_bytes(int rows, int vocab) {
    const RowSplit cut = loss_split(rows, vocab);
    const size_t parts = cut.n == 1 ? 0 : (size_t)rows * cut.n * sizeof(DistillPart);
    return parts + (fused(rows, vocab, true) ? 0 : (size_t)rows * 4 * sizeof(float));  // (float32 needs none where bf16 does not)
}

hipError_t launch_distill_loss(DistillArgs a, void* ws, hipStream_t st) {
    if (a.rows <= 0) return hipSuccess;
    a.scale = exp2_scale(a.temperature);
    a.scale_low = exp2_scale_low(a.temperature);
    const RowSplit cut = loss_split(a.rows, a.vocab);
    DistillPart* part = (DistillPart*)ws;
    if (cut.n == 1) {
        distill_loss_k<<<a.rows, kWide, 0, st>>>(a);
    } else {
        distill_part_k<<<a.rows * cut.n, kWide, 0, st>>>(a, cut, part);
        distill_join_k<<<a.rows, kNarrow, 0, st>>>(a, part, cut.n);
    }
    return hipGetLastError();
}

hipError_t launch_distill_grad(DistillArgs a, hipStream_t st) {
    if (a.rows <= 0) return hipSuccess;
    a.scale = exp2_scale(a.temperature);
    a.scale_low = exp2_scale_low(a.temperature);
    const RowSplit cut = split_row(a.vocab, std::min(kGradTarget / a.rows, a.vocab / kDistillStretch));
    if (a.grad_bf16) distill_grad_k<bf16_t><<<a.rows * cut.n, kWide, 0, st>>>(a, cut);
    else distill_grad_k<float><<<a.rows * cut.n, kWide, 0, st>>>(a, cut);
    return hipGetLastError();
}

hipError_t launch_distill_loss_grad(DistillArgs a, void* ws, hipStream_t st) {
    if (a.rows <= 0) return hipSuccess;
    const RowSplit cut = loss_split(a.rows, a.vocab);
    if (!fused(a.rows, a.vocab, a.grad_bf16)) {
        a.norm = (float*)((DistillPart*)ws + (cut.n == 1 ? 0 : (size_t)a.rows * cut.n));
        if (hipError_t e = launch_distill_loss(a, ws, st)) return e;
        return launch_distill_grad(a, st);
    }
    a.scale = exp2_scale(a.temperature);
    a.scale_low = exp2_scale_low(a.temperature);
    if (a.grad_bf16) distill_loss_grad_k<bf16_t><<<a.rows, kWide, 0, st>>>(a);
    else distill_loss_grad_k<float><<<a.rows, kWide, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace dash
