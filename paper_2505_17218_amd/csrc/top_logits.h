// Selection of a row's K largest logits by one work-group (gfx950), shared by dash_top_logits and
// the top-k draws of dash_sample_truncated.
//
// One pass: an entry above the bound `thr` (a value that K earlier entries reach) goes to a buffer
// in LDS, every other one into the sum of the rest at once, so the rest needs no subtraction of
// nearly equal sums.  After the first tile, then after doubling numbers of tiles, and whenever the
// buffer could overflow, the buffer is cut back to about its K largest and thr rises to the least
// of them.  Of random rows 1 + ln(V / 4096) times K entries then pass through the buffer; an
// ascending row fills it every tile and is slower, never wrong.
//
// Entries are held as one 64-bit word, key(l) : ~index, where key orders floats as unsigned
// integers: a larger word is a larger logit, or an equal one at a lower index, and no two are
// equal.  Cutting back bisects the words, seven pivots a step, counting with ballots.
#pragma once

#include "row_walk.h"

namespace dash {

constexpr int kTopMax = 1024;             // largest K: one sorted entry per thread
constexpr int kTopCap = 2 * kRowTile;     // buffer: what is kept and a whole tile, 64 KB of LDS
constexpr int kTopPer = kTopCap / kRowThreads;
constexpr float kEvictOne = 17592186044416.f;  // 2^44: evicted terms are summed as integers of 2^-44

struct TopShared {
    uint64_t c[kTopCap];
    uint64_t evict_z;
    int added[3];      // entries appended in a tile, by turns
    int piv[3][8];     // counts at or above the pivots, by turns
    unsigned evict_ref;
    int kept;
    double red_d[kRowWaves];
    float red_f[kRowWaves];
};

// Float order as unsigned order; -0 counts as +0 (equal values tie by index).
DASH_DEV uint32_t top_key(float l) {
    const uint32_t b = __float_as_uint(l + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
DASH_DEV float top_value(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }
DASH_DEV uint64_t top_word(float l, int i) { return (uint64_t)top_key(l) << 32 | (uint32_t)~i; }
DASH_DEV float word_value(uint64_t w) { return top_value((uint32_t)(w >> 32)); }
DASH_DEV int word_index(uint64_t w) { return (int)~(uint32_t)w; }

// A row's selection: uniform over the work-group but for `rest`.
struct TopState {
    int n = 0;                // words in the buffer
    int turn = 0;             // of `added`
    int pturn = 0;            // of `piv`
    float thr = -INFINITY;    // entries must exceed it
    uint64_t low = 0;         // every word in the buffer is at or above it
    ExpSum rest;              // the thread's share of the entries that were turned away
};

DASH_DEV void top_begin(TopShared& sh) {
    if (threadIdx.x < 3) sh.added[threadIdx.x] = 0;
    if (threadIdx.x < 24) (&sh.piv[0][0])[threadIdx.x] = 0;
    __syncthreads();
}

// A word b with k <= (words at or above b) <= k + slack, where n >= k words are held as e.
DASH_DEV uint64_t top_bound(TopShared& sh, TopState& st, const uint64_t (&e)[kTopPer], int k, int slack, int& count) {
    uint64_t lo = st.low, hi = 0xFF80000000000000ull;  // key(+inf): no word reaches it
    count = st.n;
    while (count > k + slack && hi - lo > 1) {
        const uint64_t step = max((hi - lo) >> 3, (uint64_t)1);
        int c[8] = {};
#pragma unroll
        for (int r = 0; r < kTopPer; ++r) {
            if (r * kRowThreads >= st.n) break;
#pragma unroll
            for (int j = 1; j < 8; ++j) c[j] += __popcll(__ballot(e[r] >= lo + j * step));
        }
        int* cnt = sh.piv[st.pturn];
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int j = 1; j < 8; ++j)
                if (c[j]) atomicAdd(&cnt[j], c[j]);
        }
        st.pturn = st.pturn == 2 ? 0 : st.pturn + 1;
        __syncthreads();
        // Cleared for the step after next: every thread has read it before this barrier, and adds to
        // it only after the next one.
        if (threadIdx.x < 8) sh.piv[st.pturn == 2 ? 0 : st.pturn + 1][threadIdx.x] = 0;
        uint64_t next_lo = lo, next_hi = lo + step;
#pragma unroll
        for (int j = 1; j < 8; ++j) {
            const int at = cnt[j];
            if (at >= k) {
                next_lo = lo + j * step;
                next_hi = j < 7 ? next_lo + step : hi;
                count = at;
            }
        }
        lo = next_lo;
        hi = min(hi, next_hi);
    }
    return lo;
}

// Cuts the buffer back to k .. k + slack words (n > k + slack); what falls out joins the rest.
DASH_DEV void top_cut(TopShared& sh, TopState& st, int k, int slack, float scale) {
    uint64_t e[kTopPer];
#pragma unroll
    for (int r = 0; r < kTopPer; ++r) {
        const int i = r * kRowThreads + (int)threadIdx.x;
        e[r] = i < st.n ? sh.c[i] : 0;
    }
    int count;
    const uint64_t b = top_bound(sh, st, e, k, slack, count);
    if (threadIdx.x == 0) {
        sh.evict_z = 0;
        sh.evict_ref = 0;
        sh.kept = 0;
    }
    __syncthreads();  // every word is in a register
    unsigned out = 0;  // the largest key that falls out
#pragma unroll
    for (int r = 0; r < kTopPer; ++r) {
        if (r * kRowThreads >= st.n) break;
        const uint64_t keep = __ballot(e[r] >= b);
        if (keep) {
            int at = 0;
            if ((threadIdx.x & 63) == 0) at = atomicAdd(&sh.kept, __popcll(keep));
            at = __builtin_amdgcn_readfirstlane(at);
            if (e[r] >= b) sh.c[at + __popcll(keep & ((1ull << (threadIdx.x & 63)) - 1))] = e[r];
        }
        if (e[r] && e[r] < b) out = max(out, (unsigned)(e[r] >> 32));
    }
    if (out) atomicMax(&sh.evict_ref, out);
    __syncthreads();
    // Integer terms relative to the largest: their sum does not depend on the order of the words,
    // which varies with the order in which waves appended them.
    const unsigned top = sh.evict_ref;
    if (top) {
        const float ref = top_value(top);
        uint64_t z = 0;
#pragma unroll
        for (int r = 0; r < kTopPer; ++r) {
            if (r * kRowThreads >= st.n) break;
            if (e[r] && e[r] < b) z += (uint64_t)(__builtin_amdgcn_exp2f((word_value(e[r]) - ref) * scale) * kEvictOne);
        }
        if (z) atomicAdd((unsigned long long*)&sh.evict_z, (unsigned long long)z);
        __syncthreads();
        if (threadIdx.x == 0) {
            const double zd = (double)sh.evict_z / (double)kEvictOne;
            if (ref > st.rest.ref) {
                st.rest.z = st.rest.z * exp2((double)(st.rest.ref - ref) * (double)scale) + zd;
                st.rest.ref = ref;
            } else {
                st.rest.z += zd * exp2((double)(ref - st.rest.ref) * (double)scale);
            }
        }
    }
    st.n = count;
    st.low = b;
    st.thr = word_value(b);
}

// One tile of the row (tile number t) into the selection.
DASH_DEV void top_tile(TopShared& sh, TopState& st, f32x4_t l, int i, int k, float scale) {
#pragma unroll
    for (int j = 0; j < 4; ++j) l[j] = fmaxf(l[j], -INFINITY);  // NaN is no entry
    float m4 = max4(l);
    if (__any(m4 > st.thr)) {
        uint64_t in[4];
        int total = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            in[j] = __ballot(l[j] > st.thr && l[j] < INFINITY);
            total += __popcll(in[j]);
        }
        int at = 0;
        if ((threadIdx.x & 63) == 0 && total) at = atomicAdd(&sh.added[st.turn], total);
        at = __builtin_amdgcn_readfirstlane(at) + st.n;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool mine = l[j] > st.thr;
            if (mine && l[j] < INFINITY)
                sh.c[at + __popcll(in[j] & ((1ull << (threadIdx.x & 63)) - 1))] = top_word(l[j], i + j);
            if (mine) l[j] = -INFINITY;  // +inf is no entry either
            at += __popcll(in[j]);
        }
        m4 = max4(l);
    }
    exp_push4<false>(st.rest, l, m4, scale);
    __syncthreads();
    st.n += sh.added[st.turn];
    // Cleared for the tile after next (as the pivots' counts).
    if (threadIdx.x == 0) sh.added[st.turn == 0 ? 2 : st.turn - 1] = 0;
    st.turn = st.turn == 2 ? 0 : st.turn + 1;
}

// Entries [lo, hi) of the row into the buffer, which ends with at most max(kTopCap - kRowTile, ...)
// words; thr and the rest as described above.
DASH_DEV void top_walk(TopShared& sh, TopState& st, const float* row, int lo, int hi, int k, float scale) {
    int tile = 0, next = 1;
    const int slack = (k >> 2) + 32;
    walk_row<4, true>(row, lo, hi, [&](const f32x4_t& l, int i) {
        top_tile(sh, st, l, i, k, scale);
        ++tile;
        if (st.n > kTopCap - kRowTile || (tile >= next && st.n > k + slack)) {
            top_cut(sh, st, k, slack, scale);
            next = 2 * tile;
        }
    });
}

// Leaves the m = min(n, k) largest words sorted in sh.c[0 .. m), descending; returns m.
DASH_DEV int top_finish(TopShared& sh, TopState& st, int k, float scale) {
    __syncthreads();
    if (st.n > k) top_cut(sh, st, k, 0, scale);
    const int m = st.n;
    int p = 2;
    while (p < m) p <<= 1;
    __syncthreads();
    for (int i = m + (int)threadIdx.x; i < p; i += kRowThreads) sh.c[i] = 0;
    __syncthreads();
    for (int size = 2; size <= p; size <<= 1) {
        for (int d = size >> 1; d >= 1; d >>= 1) {
            if ((int)threadIdx.x < p >> 1) {
                const int a = (((int)threadIdx.x & ~(d - 1)) << 1) | ((int)threadIdx.x & (d - 1));
                const uint64_t x = sh.c[a], y = sh.c[a + d];
                const bool down = (a & size) == 0;
                if (down ? x < y : x > y) {
                    sh.c[a] = y;
                    sh.c[a + d] = x;
                }
            }
            __syncthreads();
        }
    }
    return m;
}

// Sum of the rest over the work-group: e^((x - ref) / T) summed, and ref (0 and -FLT_MAX: nothing).
DASH_DEV double top_rest(TopShared& sh, const TopState& st, double temperature, float& ref) {
    ref = block_max_f(st.rest.z > 0.0 ? st.rest.ref : -FLT_MAX, sh.red_f);
    const double z = st.rest.z > 0.0 ? st.rest.z * exp(((double)st.rest.ref - (double)ref) / temperature) : 0.0;
    return block_sum_d(z, sh.red_d);
}

}  // namespace dash
