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
#include <algorithm>

#include "kernels.h"
#include "row_walk.h"

namespace dash {

namespace {

constexpr int kDistillTarget = 1024, kDistillStretch = 2048, kGradTarget = 2048;
constexpr int kStretch = 1 << 18;  // entries of a row whose bits are in LDS at a time (32 KB)

struct DistillShared {
    uint32_t bits[kStretch / 32];
    double red_d[kRowWaves];
    float red_f[kRowWaves];
    int twice;
};

// The teacher of a row: thread k < K holds entry k.
struct Teacher {
    int idx;          // token, -1: no entry
    double lp, p;     // ln p and p of the token (-inf and 0 without)
    double rest_lp, rest_p;
    bool none;        // no mass at all: the row has no teacher
};
DASH_DEV Teacher load_teacher(const DistillArgs& a, int64_t r, double* red_d) {
    Teacher t;
    const double T = a.temperature;
    double v = -INFINITY;
    t.idx = -1;
    if ((int)threadIdx.x < a.k) {
        const int i = a.t_idx[r * a.k + threadIdx.x];
        if (i >= 0 && i < a.vocab) {
            t.idx = i;
            v = (double)a.t_val[r * a.k + threadIdx.x] / T;
        }
    }
    const double rest = a.t_rest ? (double)a.t_rest[r] : -INFINITY;
    // (a NaN is dropped by the maximum and comes back through the sum)
    const double top = fmax(block_reduce(v, red_d, [](double x, double y) { return fmax(x, y); }), rest);
    const double ref = top == -INFINITY ? 0.0 : top;
    const double z = block_sum_d(exp(v - ref), red_d) + exp(rest - ref);
    t.none = z == 0.0;
    const double lz = t.none ? 0.0 : ref + log(z);
    t.lp = v - lz;
    t.p = exp(t.lp);
    t.rest_lp = rest - lz;
    t.rest_p = exp(t.rest_lp);
    return t;
}

// Bits of the entries [base, base + kStretch) that are the teacher's; an index that occurs twice is noted.
DASH_DEV void mark_tokens(DistillShared& sh, int idx, int base, int n) {
    __syncthreads();
    for (int i = threadIdx.x; i < (n + 31) >> 5; i += kRowThreads) sh.bits[i] = 0;
    __syncthreads();
    if (idx >= base && idx < base + n) {
        const uint32_t bit = 1u << ((idx - base) & 31);
        if (atomicOr(&sh.bits[(idx - base) >> 5], bit) & bit) sh.twice = 1;
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
DASH_DEV ExpSum sum_others(const DistillArgs& a, const float* row, int idx, int lo, int hi, DistillShared& sh) {
    ExpSum sum;
    if (threadIdx.x == 0) sh.twice = 0;
    for (int base = lo; base < hi; base += kStretch) {
        const int end = min(hi, base + kStretch);
        mark_tokens(sh, idx, base, end - base);
        walk_row<4, false>(row, base, end, [&](f32x4_t l, int i) {
            const int at = min(i - base, kStretch - 4);
            const uint32_t mine = (sh.bits[at >> 5] >> (at & 31)) & 15u;
            if (__any(mine != 0)) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (mine >> j & 1u) l[j] = -INFINITY;
            }
            exp_push4<true>(sum, l, max4(l), a.scale, a.scale_low);
        });
    }
    return sum;
}

// Loss of a row (in every thread) and its normaliser, from the threads' sums over the other tokens.
// s: the student's logit of this thread's token.
DASH_DEV float row_loss(const DistillArgs& a, const Teacher& t, float s, const ExpSum& sum, DistillShared& sh, Norm& n) {
    const double T = a.temperature;
    const bool has = t.idx >= 0;
    const double zr = block_exp_sum(sum, T, sh.red_f, sh.red_d, n.top_rest);
    n.top = fmaxf(block_max_f(has ? s : -INFINITY, sh.red_f), zr > 0.0 ? n.top_rest : -INFINITY);
    const double top = n.top;
    const double zs = block_sum_d(has ? exp(((double)s - top) / T) : 0.0, sh.red_d);
    const double far = ((double)n.top_rest - top) / T;  // <= 0, and 0 only counts with a rest
    double z = zs + (zr == 0.0 ? 0.0 : zr * exp(far));
    // a row of -inf alone has no distribution, and an index that occurs twice no meaning
    if (sh.twice || top == -INFINITY) z = NAN;
    const double lz = log(z);
    double d = 0.0;
    if (t.p != 0.0) d = t.p * (t.lp - (((double)s - top) / T - lz));
    d = block_sum_d(d, sh.red_d);
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
        *reinterpret_cast<f32x4u_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
    } else {
        for (int j = 0; j < n; ++j) p[j] = v[j];
    }
}
template <>
DASH_DEV void store4<bf16_t>(bf16_t* p, const float (&v)[4], int n) {
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    typedef u32x2_t u32x2u_t __attribute__((aligned(2)));
    if (n >= 4) {
        *reinterpret_cast<u32x2u_t*>(p) = u32x2_t{f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
    } else {
        for (int j = 0; j < n; ++j) p[j] = f2bf(v[j]);
    }
}
DASH_DEV void store1(float* p, float v) { *p = v; }
DASH_DEV void store1(bf16_t* p, float v) { *p = f2bf(v); }

// Gradient of a row's entries [lo, hi), w = its weight / T.  grad may be the row itself: a thread reads
// its entries before it writes them, and the teacher's tokens (s, read before) are written last.
template <class G>
DASH_DEV void row_grad(const DistillArgs& a, const float* row, G* grad, int lo, int hi, const Teacher& t, float s,
                       const Norm& n, float w) {
    const double T = a.temperature;
    float f = 0.f;
    if (n.z_rest != 0.f) {
        const double q_rest = exp(((double)n.top_rest - (double)n.top) / T) * (double)n.z_rest / (double)n.z;
        f = (float)((double)w * (q_rest - t.rest_p) / (double)n.z_rest);
    }
    if (n.z != n.z) f = n.z;
    float g = 0.f;
    if (t.idx >= lo && t.idx < hi) g = (float)((double)w * (exp(((double)s - (double)n.top) / T) / (double)n.z - t.p));
    asm volatile("" : "+v"(g));  // s has arrived before any entry is written
    __syncthreads();
    walk_row<4, false>(row, lo, hi, [&](const f32x4_t& l, int i) {
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float d = l[j] - n.top_rest;
            v[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(d, a.scale, fmaxf(d, -FLT_MAX) * a.scale_low)) * f;
        }
        store4(grad + i, v, hi - i);
    });
    __syncthreads();
    if (t.idx >= lo && t.idx < hi) store1(grad + t.idx, g);
}

template <class G>
DASH_DEV void zero_row(G* grad, int lo, int hi) {
    const float zero[4] = {};
    for (int i = lo + 4 * (int)threadIdx.x; i < hi; i += kRowTile) store4(grad + i, zero, hi - i);
}

// Sum over the other tokens of one stretch of a row.
struct DistillPart {
    double z;
    float ref;
    int twice;
};
__global__ void __launch_bounds__(kRowThreads, 8)
distill_part_k(DistillArgs a, RowSplit cut, DistillPart* __restrict__ part) {
    __shared__ DistillShared sh;
    const int64_t r = blockIdx.x / cut.n;
    const int lo = (int)(blockIdx.x % cut.n) * cut.len, hi = min(a.vocab, lo + cut.len);
    if (a.weight && a.weight[r] == 0.f) return;
    int idx = -1;
    if ((int)threadIdx.x < a.k) idx = a.t_idx[r * a.k + threadIdx.x];
    const ExpSum sum = sum_others(a, a.logits + r * a.ld, idx, lo, hi, sh);
    float ref;
    const double z = block_exp_sum(sum, a.temperature, sh.red_f, sh.red_d, ref);
    if (threadIdx.x == 0) part[blockIdx.x] = DistillPart{z, ref, sh.twice};
}

// A row per work-group, or (SPLIT) the joining of its stretches.  A row of weight 0 has loss 0.
template <bool SPLIT>
__global__ void __launch_bounds__(kRowThreads, 8)
distill_loss_k(DistillArgs a, const DistillPart* __restrict__ part, int parts) {
    __shared__ DistillShared sh;
    const int64_t r = blockIdx.x;
    if (a.weight && a.weight[r] == 0.f) {
        if (threadIdx.x == 0) a.loss[r] = 0.f;
        return;
    }
    const float* row = a.logits + r * a.ld;
    const Teacher t = load_teacher(a, r, sh.red_d);
    const float s = t.idx >= 0 ? row[t.idx] : 0.f;
    ExpSum sum;
    if constexpr (SPLIT) {
        if (threadIdx.x == 0) sh.twice = 0;
        __syncthreads();
        if ((int)threadIdx.x < parts) {
            const DistillPart p = part[r * parts + threadIdx.x];
            sum.z = p.z;
            sum.ref = p.ref;
            if (p.twice) sh.twice = 1;
        }
        __syncthreads();
    } else {
        sum = sum_others(a, row, t.idx, 0, a.vocab, sh);
    }
    Norm n;
    const float loss = row_loss(a, t, s, sum, sh, n);
    if (threadIdx.x != 0) return;
    a.loss[r] = loss;
    *reinterpret_cast<f32x4u_t*>(a.norm + 4 * r) = f32x4_t{n.top, n.z, n.top_rest, n.z_rest};
}

// One stretch of a row per work-group.
template <class G>
__global__ void __launch_bounds__(kRowThreads, 8)
distill_grad_k(DistillArgs a, RowSplit cut) {
    __shared__ double red_d[kRowWaves];
    const int64_t r = blockIdx.x / cut.n;
    const int lo = (int)(blockIdx.x % cut.n) * cut.len, hi = min(a.vocab, lo + cut.len);
    const float* row = a.logits + r * a.ld;
    G* grad = (G*)a.grad + r * a.ld_grad;
    const float weight = a.weight ? a.weight[r] : 1.f;
    if (weight == 0.f) return zero_row(grad, lo, hi);
    const Teacher t = load_teacher(a, r, red_d);
    if (t.none) return zero_row(grad, lo, hi);
    const Norm n{a.norm[4 * r], a.norm[4 * r + 1], a.norm[4 * r + 2], a.norm[4 * r + 3]};
    row_grad(a, row, grad, lo, hi, t, t.idx >= lo && t.idx < hi ? row[t.idx] : 0.f, n,
             (float)((double)weight / (double)a.temperature));
}

template <class G>
__global__ void __launch_bounds__(kRowThreads)
distill_loss_grad_k(DistillArgs a) {
    __shared__ DistillShared sh;
    const int64_t r = blockIdx.x;
    const float* row = a.logits + r * a.ld;
    G* grad = (G*)a.grad + r * a.ld_grad;
    const float weight = a.weight ? a.weight[r] : 1.f;
    if (weight == 0.f) {
        if (threadIdx.x == 0) a.loss[r] = 0.f;
        return zero_row(grad, 0, a.vocab);
    }
    const Teacher t = load_teacher(a, r, sh.red_d);
    if (t.none) {
        if (threadIdx.x == 0) a.loss[r] = 0.f;
        return zero_row(grad, 0, a.vocab);
    }
    const float s = t.idx >= 0 ? row[t.idx] : 0.f;
    const ExpSum sum = sum_others(a, row, t.idx, 0, a.vocab, sh);
    Norm n;
    const float loss = row_loss(a, t, s, sum, sh, n);
    if (threadIdx.x == 0) a.loss[r] = loss;
    row_grad(a, row, grad, 0, a.vocab, t, s, n, (float)((double)weight / (double)a.temperature));
}

RowSplit loss_split(int rows, int vocab) {
    return split_row(vocab, std::min({64, kDistillTarget / std::max(rows, 1), vocab / kDistillStretch}));
}

}  // namespace

size_t distill_workspace_bytes(int rows, int vocab) {
    const RowSplit cut = loss_split(rows, vocab);
    return cut.n == 1 ? 0 : (size_t)rows * (cut.n * sizeof(DistillPart) + 4 * sizeof(float));
}

hipError_t launch_distill_loss(DistillArgs a, void* ws, hipStream_t st) {
    if (a.rows <= 0) return hipSuccess;
    a.scale = exp2_scale(a.temperature);
    a.scale_low = exp2_scale_low(a.temperature);
    const RowSplit cut = loss_split(a.rows, a.vocab);
    DistillPart* part = (DistillPart*)ws;
    if (cut.n == 1) {
        distill_loss_k<false><<<a.rows, kRowThreads, 0, st>>>(a, nullptr, 1);
    } else {
        distill_part_k<<<a.rows * cut.n, kRowThreads, 0, st>>>(a, cut, part);
        distill_loss_k<true><<<a.rows, kRowThreads, 0, st>>>(a, part, cut.n);
    }
    return hipGetLastError();
}

hipError_t launch_distill_grad(DistillArgs a, hipStream_t st) {
    if (a.rows <= 0) return hipSuccess;
    a.scale = exp2_scale(a.temperature);
    a.scale_low = exp2_scale_low(a.temperature);
    const RowSplit cut = split_row(a.vocab, std::min(kGradTarget / a.rows, a.vocab / kDistillStretch));
    if (a.grad_bf16) distill_grad_k<bf16_t><<<a.rows * cut.n, kRowThreads, 0, st>>>(a, cut);
    else distill_grad_k<float><<<a.rows * cut.n, kRowThreads, 0, st>>>(a, cut);
    return hipGetLastError();
}

hipError_t launch_distill_loss_grad(DistillArgs a, void* ws, hipStream_t st) {
    if (a.rows <= 0) return hipSuccess;
    const RowSplit cut = loss_split(a.rows, a.vocab);
    if (cut.n > 1) {
        a.norm = (float*)((DistillPart*)ws + (size_t)a.rows * cut.n);
        if (hipError_t e = launch_distill_loss(a, ws, st)) return e;
        return launch_distill_grad(a, st);
    }
    a.scale = exp2_scale(a.temperature);
    a.scale_low = exp2_scale_low(a.temperature);
    if (a.grad_bf16) distill_loss_grad_k<bf16_t><<<a.rows, kRowThreads, 0, st>>>(a);
    else distill_loss_grad_k<float><<<a.rows, kRowThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace dash
