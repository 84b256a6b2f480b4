// One work-group walking a row of float32 logits (gfx950): loads, exponential sums, reductions.
// Shared by the kernels that read rows of the vocabulary once (top_logits.hip, truncate.hip,
// distill.hip).
#pragma once

#include <float.h>
#include <math.h>

#include "common.h"

namespace dash {

// Threads of a work-group (NT below) unless a kernel says otherwise, and its waves.
constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / 64;
// Entries of one step of NT threads, a tile: four consecutive ones per thread.
constexpr int kRowTile = 4 * kRowThreads;

// Rows start on any float: gfx950 loads 16 bytes from a 4-byte aligned address in one instruction.
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
// (row is the same for the whole work-group: its address stays in scalar registers, and a lane
// holds a 32-bit offset.)
template <bool STREAM>
DASH_DEV f32x4_t load_row4(const float* row, int i) {
    const f32x4u_t* q = reinterpret_cast<const f32x4u_t*>(reinterpret_cast<const char*>(row) + (uint32_t)i * 4u);
    if constexpr (STREAM) return __builtin_nontemporal_load(q);
    else return *q;
}

// Calls f(l, i) with entries i .. i+3 of row for every group of four in [lo, hi); entries past hi are
// -inf.  Every thread of the work-group makes the same number of calls, so f may hold barriers.
// DEPTH tiles are in flight: a thread's registers are used, then loaded again (past the end: with a
// tile that is in bounds, unused), so no wait covers a load younger than the one that is needed.
// In order: whole tiles ascending, then the partial one.  STRIPES: the whole tiles as DEPTH stripes
// side by side, so that the first DEPTH tiles are a sample of the whole row.  start(buf, whole) sees
// these before f does; where there are fewer whole tiles than DEPTH, the last one (the partial one,
// if there is none) fills the places of the missing.  round(t) is called after the t-th DEPTH tiles
// (1, 2, ...) and ends the walk by returning true.  STREAM: rows that nothing reads again.
// f may write the entries that it was called with in their place, so row is not __restrict__.
template <int DEPTH, bool STRIPES, bool STREAM, int NT = kRowThreads, class START, class F, class ROUND>
DASH_DEV void walk_row(const float* row, int lo, int hi, START&& start, F&& f, ROUND&& round) {
    constexpr int kTile = 4 * NT;
    const int whole = (hi - lo) / kTile;
    const int end = lo + whole * kTile, at = lo + 4 * (int)threadIdx.x;
    f32x4_t last = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (end < hi) {  // the partial tile is loaded first and used last
        const int i = end + 4 * (int)threadIdx.x;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < hi) last[j] = row[i + j];
    }
    if (whole) {
        // Round t < rounds is tiles t of the stripes (or the next DEPTH tiles); the round after it, the
        // left-over tiles.
        const int rounds = whole / DEPTH, left = whole - rounds * DEPTH;
        auto tile = [&](int t, int d) {
            return t >= rounds ? min(rounds * DEPTH + d, whole - 1) : STRIPES ? d * rounds + t : t * DEPTH + d;
        };
        f32x4_t buf[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) buf[d] = load_row4<STREAM>(row, at + tile(0, d) * kTile);
        start(buf, whole);
        for (int t = 0; t < rounds; ++t) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                f(buf[d], at + tile(t, d) * kTile);
                buf[d] = load_row4<STREAM>(row, at + tile(t + 1, d) * kTile);
            }
            if (round(t + 1)) return;
        }
#pragma unroll
        for (int d = 0; d < DEPTH - 1; ++d) {
            if (d >= left) break;
            f(buf[d], at + tile(rounds, d) * kTile);
        }
    } else {
        f32x4_t buf[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) buf[d] = last;
        start(buf, 0);
    }
    if (end < hi) f(last, end + 4 * (int)threadIdx.x);
}
template <int DEPTH, bool STREAM, int NT = kRowThreads, class F>
DASH_DEV void walk_row(const float* row, int lo, int hi, F&& f) {
    walk_row<DEPTH, false, STREAM, NT>(row, lo, hi, [](const f32x4_t (&)[DEPTH], int) {}, (F&&)f, [](int) { return false; });
}

// Rows cut into n stretches of len entries (the last one shorter, none empty; len a multiple of four),
// each walked by a work-group of its own.
struct RowSplit {
    int n, len;
};
inline RowSplit split_row(int vocab, int n) {
    if (n <= 1) return {1, vocab};
    const int len = ((vocab + n - 1) / n + 3) & ~3;
    return {(vocab + len - 1) / len, len};
}

// Exponents are taken of half the difference of two logits: the whole one may lie past the largest
// float, and at T = 10^38 be worth a few octaves all the same.  Halving is exact (but for
// denormals) and one instruction with the difference, so the product below is that of the whole
// difference and log2(e) / T, bit for bit.
DASH_DEV float half_gap(float x, float half) { return __builtin_fmaf(x, 0.5f, -half); }
// 2 log2(e) / T, so that e^((x - m) / T) = 2^(half_gap(x, m / 2) scale); finite for every T > 0 (0 times it
// stays 0): below T = 8.5e-39, where logits less than 1e-36 apart would matter, it is that of 8.5e-39.
__host__ __device__ inline float exp2_scale(double temperature) {
    return (float)fmin(2.0 * 1.4426950408889634 / temperature, (double)FLT_MAX);
}
// What rounding that factor to float32 left out: with it exponents are right to their own rounding.
// Nothing above 2^25 (T < 8.6e-8), where the largest float times it could overflow against the product
// with the factor itself; it is worth 2^-25 of an exponent.
__host__ __device__ inline float exp2_scale_low(double temperature) {
    const double s = 2.0 * 1.4426950408889634 / temperature;
    return s <= 33554432.0 ? (float)(s - (double)(float)s) : 0.f;
}

// A thread's sum of e^((x - ref) / T).  ref follows the entries lazily: it is raised to a group's
// maximum only where that is 2^40 above it, so that most groups need no rescale and float32 terms
// neither overflow nor lose what matters; the sum itself is float64 (a thread may add 2^18 terms).
struct ExpSum {
    float half = -0.5f * FLT_MAX;  // ref / 2
    double z = 0.0;
    DASH_DEV float ref() const { return 2.f * half; }
};

// Four terms; -inf adds nothing, NaN and +inf make the sum NaN.  LOW: with the scale's low part.
template <bool LOW>
DASH_DEV void exp_push4(ExpSum& s, const f32x4_t& x, float m4, float scale, float low = 0.f) {
    const float above = half_gap(m4, s.half) * scale;
    const bool far = above > 40.f;
    if (__any(far)) {
        if (far) {
            s.z *= (double)__builtin_amdgcn_exp2f(-above);
            s.half = 0.5f * m4;
        }
    }
    float e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float d = half_gap(x[j], s.half);
        // (the low product is kept finite: -inf times a low part of either sign or zero)
        const float y = LOW ? __builtin_fmaf(d, scale, fmaxf(d, -FLT_MAX) * low) : d * scale;
        e[j] = __builtin_amdgcn_exp2f(y);
    }
    s.z += (double)((e[0] + e[1]) + (e[2] + e[3]));
}

// One finite term.
DASH_DEV void exp_push1(ExpSum& s, float x, float scale) {
    if (x > s.ref()) {
        s.z *= (double)__builtin_amdgcn_exp2f(-half_gap(x, s.half) * scale);
        s.half = 0.5f * x;
    }
    s.z += (double)__builtin_amdgcn_exp2f(half_gap(x, s.half) * scale);
}

// Inclusive sum over the threads up to this one (of NT), and the total.
template <int NT = kRowThreads, class T>
DASH_DEV T block_scan(T v, T* red, T& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 63) red[w] = v;
    __syncthreads();
    // every wave sums the waves' totals, a lane each
    T t = lane < NT / 64 ? red[lane] : (T)0;
#pragma unroll
    for (int o = 1; o < NT / 64; o <<= 1) {
        const T u = __shfl_up(t, o, 64);
        if (lane >= o) t += u;
    }
    total = __shfl(t, NT / 64 - 1, 64);
    const T before = __shfl(t, max(w - 1, 0), 64);
    return v + (w ? before : (T)0);
}

DASH_DEV float max4(const f32x4_t& x) { return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])); }

// Reductions over the work-group's NT threads in a fixed order; every thread gets the
// result.  `red` is scratch of NT / 64 values that no other reduction is using: consecutive
// reductions through one scratch are separated by their own leading barrier.
template <int NT = kRowThreads, class T, class OP>
DASH_DEV T block_reduce(T v, T* red, OP op) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = op(v, (T)__shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    T s = red[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) s = op(s, red[i]);
    return s;
}
template <int NT = kRowThreads>
DASH_DEV double block_sum_d(double v, double* red) {
    return block_reduce<NT>(v, red, [](double a, double b) { return a + b; });
}
template <int NT = kRowThreads>
DASH_DEV float block_max_f(float v, float* red) {
    return block_reduce<NT>(v, red, [](float a, float b) { return fmaxf(a, b); });
}

// Sum over the work-group's threads of e^((l - ref) / T) (0: nothing), and ref.
template <int NT = kRowThreads>
DASH_DEV double block_exp_sum(const ExpSum& s, double temperature, float* red_f, double* red_d, float& ref) {
    ref = block_max_f<NT>(s.z > 0.0 ? s.ref() : -FLT_MAX, red_f);
    // (a NaN sum stays one)
    return block_sum_d<NT>(s.z == 0.0 ? 0.0 : s.z * exp(((double)s.ref() - (double)ref) / temperature), red_d);
}

}  // namespace dash
