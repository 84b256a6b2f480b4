// Selection of a row's K largest logits (gfx950), shared by dash_top_logits and the top-k draws of
// dash_sample_truncated.  Two launches.
//
// The first walks the row (or stretches of it) once.  An entry above a bound that K entries reach goes
// to a list in the workspace, every other one into the sum of the rest at once, so the rest needs no
// subtraction of nearly equal sums.  The bound comes from four tiles spread over the row, which are
// in registers before any is used: of each thread's largest of two tiles and largest of the other two,
// the K-th.  About K / 16384 of a row is above it: 600 entries for K = 64.  This kernel does nothing else: with the
// cuts below in it, its loop reloaded spilled addresses, and every such reload waits for all loads
// in flight.
//
// The second gathers a row's lists in LDS, cuts them to the K largest and sorts those.  A list that
// overflowed (a row that holds one value many times, or whose large values the sample misses) sends
// it over the row itself, with a cut whenever the next tile might not fit.  That is slower, never wrong.
//
// Entries are held as one 64-bit word, key(l) : ~index, where key orders floats as unsigned
// integers: a larger word is a larger logit, or an equal one at a lower index, and no two are equal.
#pragma once

#include <algorithm>

#include "row_walk.h"

namespace dash {

constexpr int kTopMax = 1024;             // largest K: one sorted entry per thread
constexpr int kTopCap = 2 * kRowTile;     // words in LDS: 64 KB, two work-groups per CU
constexpr int kTopPer = kTopCap / kRowThreads;
constexpr int kTopStart = 4;              // tiles that give the bound
constexpr float kEvictOne = 17592186044416.f;  // 2^44: evicted terms are summed as integers of 2^-44

// Float order as unsigned order; -0 counts as +0 (equal values tie by index).
DASH_DEV uint32_t top_key(float l) {
    const uint32_t b = __float_as_uint(l + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
DASH_DEV float top_value(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }
DASH_DEV uint64_t top_word(float l, int i) { return (uint64_t)top_key(l) << 32 | (uint32_t)~i; }
DASH_DEV float word_value(uint64_t w) { return top_value((uint32_t)(w >> 32)); }
DASH_DEV int word_index(uint64_t w) { return (int)~(uint32_t)w; }
// The largest float below the one with this key (that of no entry but -0's: +0 comes after the negative numbers).
DASH_DEV float value_below(uint32_t key) { return top_value(key - (key == 0x80000000u ? 2u : 1u)); }
constexpr uint32_t kKeyInf = 0xFF800000u;      // key(+inf): above every entry's
constexpr uint32_t kKeyLowest = 0x00800000u;   // key of the lowest float

// What the first launch leaves of a stretch: its rest, and the number of its words in the list (more
// than the list's room: it overflowed).
struct TopPart {
    double z;  // sum of e^((l - ref) / T)
    float ref;
    int n;
};
// Stretches per row, and the room of a stretch's list: twice what the sampled bound lets
// through on average.
struct TopPlan {
    RowSplit cut;
    int room;
};
TopPlan top_plan(int rows, int vocab, int k);
struct TopParts {
    const TopPart* part;    // [rows][cut.n]
    const uint64_t* words;  // [rows][cut.n][room]
    int n, room;
};
hipError_t launch_top_parts(const float* logits, int64_t ld, int rows, int vocab, const int32_t* row_of, int k,
                            float temperature, const TopPlan& plan, void* ws, TopParts& out, hipStream_t st);

struct BoundShared {
    int hist[kRowThreads];
    int found[3];
    int red_i[kRowWaves];
};

// A bound b with k <= (words e at or above b), and at most k + slack unless equal words straddle that;
// lo <= b < hi, count words are at or above lo, none at or above hi.  The first `per` of a thread's
// words count.  A histogram of the range in 1024 parts, summed from the top, finds the part that holds
// the k-th word; that part is the range of the next round, if it holds too many.  Two rounds as a rule.
template <class W, int PER>
DASH_DEV W top_bound(BoundShared& sh, const W (&e)[PER], int per, int k, int slack, W lo, W hi, int& count) {
    int above = 0;  // words at or above hi
    while (count > k + slack && hi - lo > 1) {
        const int bits = (int)(8 * sizeof(uint64_t)) - __clzll((unsigned long long)(hi - lo - 1));
        const int shift = max(bits - 10, 0);
        __syncthreads();
        sh.hist[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            if (r >= per) break;
            if (e[r] >= lo && e[r] < hi) atomicAdd(&sh.hist[(int)((e[r] - lo) >> shift)], 1);
        }
        __syncthreads();
        const int part = kRowThreads - 1 - (int)threadIdx.x, here = sh.hist[part];
        int total;
        const int upto = above + block_scan(here, sh.red_i, total);
        if (upto >= k && upto - here < k) {
            sh.found[0] = part;
            sh.found[1] = upto;
            sh.found[2] = upto - here;
        }
        __syncthreads();
        lo += (W)sh.found[0] << shift;
        const W top = lo + ((W)1 << shift);
        hi = top < hi && top > lo ? top : hi;
        count = sh.found[1];
        above = sh.found[2];
    }
    return lo;
}

// ---- the second launch: a row's words in LDS ---------------------------------------------------

struct TopShared {
    uint64_t c[kTopCap];
    uint64_t evict_z;
    int count;         // words appended
    unsigned evict_ref;
    int kept;
    BoundShared bound;
    double red_d[kRowWaves];
    float red_f[kRowWaves];
};
// Uniform over the work-group but for `rest`.
struct TopState {
    int n = 0;       // words in the buffer, as of the last barrier that counted
    uint64_t low = 0;  // words must reach this
    ExpSum rest;     // the thread's share of the entries that were turned away
};

// Cuts the buffer from n > k + slack words to k .. k + slack; what falls out joins the rest, and the
// bound rises to the least word left.  Between barriers that separate it from appends.
DASH_DEV void top_cut(TopShared& sh, TopState& st, int k, int slack, float scale) {
    const int per = (st.n + kRowThreads - 1) / kRowThreads;
    uint64_t e[kTopPer];
#pragma unroll
    for (int r = 0; r < kTopPer; ++r) {
        const int i = r * kRowThreads + (int)threadIdx.x;
        e[r] = i < st.n ? sh.c[i] : 0;
    }
    int count = st.n;
    const uint64_t b = top_bound(sh.bound, e, per, k, slack, (uint64_t)kKeyLowest << 32, (uint64_t)kKeyInf << 32, count);
    if (threadIdx.x == 0) {
        sh.evict_z = 0;
        sh.evict_ref = 0;
        sh.kept = 0;
    }
    __syncthreads();  // every word is in a register
    unsigned out = 0;  // the largest key that falls out
#pragma unroll
    for (int r = 0; r < kTopPer; ++r) {
        if (r >= per) break;
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
            if (r >= per) break;
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
    if (threadIdx.x == 0) sh.count = count;
    st.n = count;
    st.low = b;
    __syncthreads();
}

// Appends the words of those lanes that have one (any lanes of a wave).
DASH_DEV void top_append(TopShared& sh, bool mine, uint64_t word) {
    const uint64_t in = __ballot(mine);
    if (!in) return;
    int at = 0;
    if ((threadIdx.x & 63) == 0) at = atomicAdd(&sh.count, __popcll(in));
    at = __builtin_amdgcn_readfirstlane(at);
    if (mine) sh.c[at + __popcll(in & ((1ull << (threadIdx.x & 63)) - 1))] = word;
}
// After at most kRowTile appends: room for as many again.
DASH_DEV void top_count(TopShared& sh, TopState& st, int k, float scale) {
    __syncthreads();
    st.n = sh.count;
    __syncthreads();
    if (st.n > kTopCap - kRowTile) top_cut(sh, st, k, (k >> 2) + 32, scale);
}

// The words of row b among them the k largest, and the rest of the row.
DASH_DEV void top_gather(TopShared& sh, TopState& st, const TopParts& p, int64_t b, const float* row, int vocab, int k,
                         float scale) {
    if (threadIdx.x == 0) sh.count = 0;
    const TopPart* part = p.part + b * p.n;
    const uint64_t* words = p.words + b * p.n * p.room;
    bool fits = true;
    if ((int)threadIdx.x < p.n) {
        const TopPart mine = part[threadIdx.x];
        fits = mine.n <= p.room;
        if (mine.z > 0.0) {
            st.rest.ref = mine.ref;
            st.rest.z = mine.z;
        }
    }
    if (__syncthreads_and(fits)) {
        for (int from = 0; from < p.n * p.room; from += kRowTile) {  // (room is a multiple of 64: a wave has one list)
#pragma unroll
            for (int r = 0; r < kRowTile / kRowThreads; ++r) {
                const int i = from + r * kRowThreads + (int)threadIdx.x;
                if (i >= p.n * p.room) break;
                const bool in = i % p.room < part[i / p.room].n;
                top_append(sh, in, in ? words[i] : 0);
            }
            top_count(sh, st, k, scale);
        }
        return;
    }
    st = TopState{};
    for (int at = 0; at < vocab; at += kRowTile) {
        walk_row<1, true>(row, at, min(vocab, at + kRowTile), [&](f32x4_t l, int i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool entry = fabsf(l[j]) < INFINITY;
                const uint64_t w = entry ? top_word(l[j], i + j) : 0;
                const bool in = entry && w >= st.low;
                top_append(sh, in, w);
                if (in || !entry) l[j] = -INFINITY;
            }
            exp_push4<false>(st.rest, l, max4(l), scale);
        });
        top_count(sh, st, k, scale);
    }
}

// Leaves the m = min(n, k) largest words sorted in sh.c[0 .. m), descending (what lies behind them in
// the buffer is added to the rest); returns m.
DASH_DEV int top_finish(TopShared& sh, TopState& st, int k, float scale) {
    int p = 64;
    while (p < k) p <<= 1;
    __syncthreads();
    if (st.n > p) top_cut(sh, st, k, p - k, scale);
    const int n = st.n;
    for (int i = n + (int)threadIdx.x; i < p; i += kRowThreads) sh.c[i] = 0;
    __syncthreads();
    if (p <= 128) {
        // A word's place is the number of larger ones (words differ; zeros fill what is left):
        // kRowThreads / p threads per word count over a share of the words each.
        const int i = (int)threadIdx.x & (p - 1), share = (int)threadIdx.x / p, len = p * p / kRowThreads;
        const uint64_t mine = sh.c[i];
        int place = 0;
        for (int j = share * len; j < (share + 1) * len; ++j) place += sh.c[j] > mine;
        sh.bound.hist[threadIdx.x] = place;
        __syncthreads();
        if ((int)threadIdx.x < p) {
            for (int q = 1; q < kRowThreads / p; ++q) place += sh.bound.hist[threadIdx.x + q * p];
            if (mine) sh.c[place] = mine;  // (each thread has its own word in a register)
        }
    } else {
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
    }
    __syncthreads();
    const int m = min(n, k);
    const int i = m + (int)threadIdx.x;
    if (__any(i < n)) {
        const float l = i < n ? word_value(sh.c[i]) : -INFINITY;
        exp_push4<false>(st.rest, f32x4_t{l, -INFINITY, -INFINITY, -INFINITY}, l, scale);
    }
    return m;
}

}  // namespace dash
