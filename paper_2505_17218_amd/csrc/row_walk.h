// One work-group walking a row of float32 logits (gfx950): loads, exponential sums, reductions.
// Shared by the kernels that read rows of the vocabulary once (top_logits.hip, truncate.hip,
// distill.hip).
#pragma once

#include <float.h>
#include <math.h>

#include "common.h"

namespace dash {

constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kRowTile = 4 * kRowThreads;  // entries of one step: four consecutive ones per thread

// Rows start on any float: gfx950 loads 16 bytes from a 4-byte aligned address in one instruction.
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
template <bool STREAM>
DASH_DEV f32x4_t load_row4(const float* p) {
    const f32x4u_t* q = reinterpret_cast<const f32x4u_t*>(p);
    if constexpr (STREAM) return __builtin_nontemporal_load(q);
    else return *q;
}

// Calls f(l, i) with entries i .. i+3 of row for every group of four in [lo, hi), whole tiles first,
// in ascending order; entries past hi are -inf.  Every thread of the work-group makes the same
// number of calls, so f may hold barriers.  DEPTH tiles are in flight: a thread's registers are
// used, then loaded again DEPTH tiles ahead (past the end: the last tile once more), so no wait
// covers a load younger than the one that is needed.  STREAM: rows that nothing reads again.
template <int DEPTH, bool STREAM, class F>
DASH_DEV void walk_row(const float* __restrict__ row, int lo, int hi, F&& f) {
    const int whole = (hi - lo) / kRowTile;
    const int end = lo + whole * kRowTile, at = lo + 4 * (int)threadIdx.x;
    f32x4_t last = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (end < hi) {  // the partial tile is loaded first and used last
        const int i = end + 4 * (int)threadIdx.x;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < hi) last[j] = row[i + j];
    }
    if (whole) {
        f32x4_t buf[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) buf[d] = load_row4<STREAM>(row + at + min(d, whole - 1) * kRowTile);
        for (int t0 = 0; t0 < whole; t0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int t = t0 + d;
                if (t >= whole) break;
                f(buf[d], at + t * kRowTile);
                buf[d] = load_row4<STREAM>(row + at + min(t + DEPTH, whole - 1) * kRowTile);
            }
        }
    }
    if (end < hi) f(last, end + 4 * (int)threadIdx.x);
}

// log2(e) / T, so that e^((x - m) / T) = 2^((x - m) scale); finite for every T > 0 (0 times it stays 0).
__host__ __device__ inline float exp2_scale(double temperature) {
    return (float)fmin(1.4426950408889634 / temperature, (double)FLT_MAX);
}
// What rounding that factor to float32 left out: with it exponents are right to their own rounding.
__host__ __device__ inline float exp2_scale_low(double temperature) {
    const double s = 1.4426950408889634 / temperature;
    return s < (double)FLT_MAX ? (float)(s - (double)(float)s) : 0.f;
}

// A thread's sum of e^((x - ref) / T).  ref follows the entries lazily: it is raised to a group's
// maximum only where that is 2^40 above it, so that most groups need no rescale and float32 terms
// neither overflow nor lose what matters; the sum itself is float64 (a thread may add 2^18 terms).
struct ExpSum {
    float ref = -FLT_MAX;
    double z = 0.0;
};

// Four terms; -inf adds nothing, NaN and +inf make the sum NaN.  LOW: with the scale's low part.
template <bool LOW>
DASH_DEV void exp_push4(ExpSum& s, const f32x4_t& x, float m4, float scale, float low = 0.f) {
    const bool far = (m4 - s.ref) * scale > 40.f;
    if (__any(far)) {
        if (far) {
            s.z *= (double)__builtin_amdgcn_exp2f((s.ref - m4) * scale);
            s.ref = m4;
        }
    }
    float e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float d = x[j] - s.ref;
        // (the low product is kept finite: -inf times a low part of either sign or zero)
        const float y = LOW ? __builtin_fmaf(d, scale, fmaxf(d, -FLT_MAX) * low) : d * scale;
        e[j] = __builtin_amdgcn_exp2f(y);
    }
    s.z += (double)((e[0] + e[1]) + (e[2] + e[3]));
}

DASH_DEV float max4(const f32x4_t& x) { return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])); }

// Reductions over the work-group's kRowThreads threads in a fixed order; every thread gets the
// result.  `red` is scratch of kRowWaves values that no other reduction is using: consecutive
// reductions through one scratch are separated by their own leading barrier.
template <class T, class OP>
DASH_DEV T block_reduce(T v, T* red, OP op) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = op(v, (T)__shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    T s = red[0];
#pragma unroll
    for (int i = 1; i < kRowWaves; ++i) s = op(s, red[i]);
    return s;
}
DASH_DEV double block_sum_d(double v, double* red) {
    return block_reduce(v, red, [](double a, double b) { return a + b; });
}
DASH_DEV float block_max_f(float v, float* red) {
    return block_reduce(v, red, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace dash
