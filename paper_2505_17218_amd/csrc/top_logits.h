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
// The second reads a row's lists into registers, cuts them to the K largest and sorts those in LDS:
// 7.5 us for 8 rows and K = 20, 25 for 2048 and K = 64, 33 for 333 and K = 500, bound by one row's chain of
// barriers.
// Lists that do not fit are cut piece by piece, and one that overflowed (a row that holds one value
// many times, or whose large values the sample misses) sends it over the row itself, a cut whenever
// the next tile might not fit.  That is slower, never wrong.
//
// Entries are held as one 64-bit word, key(l) : ~index, where key orders floats as unsigned
// integers: a larger word is a larger logit, or an equal one at a lower index, and no two are equal.
#pragma once

#include <algorithm>
#include <type_traits>

#include "row_walk.h"

namespace dash {

constexpr int kTopMax = 1024;             // largest K: one sorted entry per thread
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

constexpr int kBoundParts = 1024;
template <int NT>
struct BoundShared {
    int hist[kBoundParts];
    int found[3];
    int red[NT / 64];
};

// A bound b with k <= (words e at or above b), and at most k + slack unless equal words straddle that;
// lo <= b < hi, count words are at or above lo, none at or above hi.  The first `per` of a thread's
// words count.  A histogram of the range in 1024 parts, summed from the top, finds the part that holds
// the k-th word; that part is the range of the next round, if it holds too many.  Two rounds as a rule.
template <int NT, class W, int PER>
DASH_DEV W top_bound(BoundShared<NT>& sh, const W (&e)[PER], int per, int k, int slack, W lo, W hi, int& count) {
    constexpr int kOwn = kBoundParts / NT;  // parts per thread, from the top
    int above = 0;  // words at or above hi
    while (count > k + slack && hi - lo > 1) {
        const int bits = (int)(8 * sizeof(uint64_t)) - __clzll((unsigned long long)(hi - lo - 1));
        const int shift = max(bits - 10, 0);
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kOwn; ++q) sh.hist[threadIdx.x + q * NT] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            if (r >= per) break;
            if (e[r] >= lo && e[r] < hi) atomicAdd(&sh.hist[(int)((e[r] - lo) >> shift)], 1);
        }
        __syncthreads();
        const int first = kBoundParts - 1 - kOwn * (int)threadIdx.x;
        int here[kOwn], sum = 0, total;
#pragma unroll
        for (int q = 0; q < kOwn; ++q) sum += here[q] = sh.hist[first - q];
        int upto = above + block_scan<NT>(sum, sh.red, total) - sum;  // words above this thread's parts
#pragma unroll
        for (int q = 0; q < kOwn; ++q) {
            if (upto < k && upto + here[q] >= k) {
                sh.found[0] = first - q;
                sh.found[1] = upto + here[q];
                sh.found[2] = upto;
            }
            upto += here[q];
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

// ---- the second launch -----------------------------------------------------------------------------

// A work-group of NT threads holds NT PER words, as many as a row's lists have together as a rule
// (k = 1000 of 151,936 cut piece by piece, 8192 words at a time: 672 us for 2048 rows, 568 whole).  It has as
// many threads as there may be results, but not fewer than 256: small ones share a CU, and their
// barriers are of few waves (333 rows and k = 500: 44 us with 1024 threads, 34 with 512).
constexpr int kTopSmall = 256;
template <class F>
void top_join_variant(int k, F&& join) {
    if (k <= 64) join(std::integral_constant<int, 256>{}, std::integral_constant<int, 8>{});
    else if (k <= kTopSmall) join(std::integral_constant<int, 256>{}, std::integral_constant<int, 16>{});
    else if (k <= 512) join(std::integral_constant<int, 512>{}, std::integral_constant<int, 16>{});
    else join(std::integral_constant<int, 1024>{}, std::integral_constant<int, 16>{});
}
inline int top_cap(int k) { return k <= 64 ? 256 * 8 : k <= kTopSmall ? 256 * 16 : k <= 512 ? 512 * 16 : 1024 * 16; }
template <int NT, int PER>
struct TopShared {
    uint64_t c[NT * PER];
    uint64_t evict_z;
    int count;         // words appended
    unsigned evict_ref;
    int kept;
    int at[64];        // where the words of each list begin
    BoundShared<NT> bound;
    double red_d[NT / 64];
    float red_f[NT / 64];
};
constexpr int kTopParts = 64;  // stretches of a row at most (a wave adds up their lists)
// Uniform over the work-group but for `rest`.
struct TopState {
    int n = 0;         // words in LDS, as of the last barrier that counted
    uint64_t low = 0;  // words must reach this
    ExpSum rest;       // the thread's share of the entries that were turned away
};

// The words that each(f) calls f with, all threads' together, join the rest; out is the largest key among
// the thread's.  Integer terms relative to the largest of all: their sum does not depend on the order
// of the words, which varies with the order in which waves appended them.  (sh.evict_z and
// sh.evict_ref are 0, set a barrier ago.)
template <int NT, int PER, class EACH>
DASH_DEV void top_turn_away(TopShared<NT, PER>& sh, TopState& st, unsigned out, float scale, EACH&& each) {
    if (__any(out != 0)) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) out = max(out, (unsigned)__shfl_xor((int)out, o, 64));
        if ((threadIdx.x & 63) == 0) atomicMax(&sh.evict_ref, out);
    }
    __syncthreads();
    const unsigned top = sh.evict_ref;
    if (!top) return;
    const float ref = top_value(top), half = 0.5f * ref;
    uint64_t z = 0;
    each([&](uint64_t w) { z += (uint64_t)(__builtin_amdgcn_exp2f(half_gap(word_value(w), half) * scale) * kEvictOne); });
    if (__any(z != 0)) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) z += (uint64_t)__shfl_xor((long long)z, o, 64);
        if ((threadIdx.x & 63) == 0) atomicAdd((unsigned long long*)&sh.evict_z, (unsigned long long)z);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        const double zd = (double)sh.evict_z / (double)kEvictOne;
        const double above = (double)half_gap(ref, st.rest.half) * (double)scale;
        if (above > 0.0) {
            st.rest.z = st.rest.z * exp2(-above) + zd;
            st.rest.half = half;
        } else {
            st.rest.z += zd * exp2(above);
        }
    }
}

// Of n words in the threads' registers (word r NT + thread is e[r]; 0: none) those at or above a bound
// that leaves k .. k + slack of them (all, if n is no more) go to LDS, the others (SUM) join the rest.
template <bool SUM, int NT, int PER>
DASH_DEV void top_keep(TopShared<NT, PER>& sh, TopState& st, const uint64_t (&e)[PER], int n, int k, int slack, float scale) {
    const int per = (n + NT - 1) / NT;
    int count = n;
    const uint64_t b = top_bound<NT>(sh.bound, e, per, k, slack, (uint64_t)kKeyLowest << 32, (uint64_t)kKeyInf << 32, count);
    __syncthreads();  // every word is in a register
    if (threadIdx.x == 0) {
        sh.evict_z = 0;
        sh.evict_ref = 0;
        sh.kept = 0;
    }
    __syncthreads();
    unsigned out = 0;  // the largest key that falls out
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const uint64_t keep = r < per ? __ballot(e[r] >= b) : 0;
        if (keep) {
            int at = 0;
            if ((threadIdx.x & 63) == 0) at = atomicAdd(&sh.kept, __popcll(keep));
            at = __builtin_amdgcn_readfirstlane(at);
            if (e[r] >= b) sh.c[at + __popcll(keep & ((1ull << (threadIdx.x & 63)) - 1))] = e[r];
        }
        if (e[r] && e[r] < b) out = max(out, (unsigned)(e[r] >> 32));
    }
    if constexpr (SUM)
        top_turn_away(sh, st, out, scale, [&](auto&& f) {
#pragma unroll
            for (int r = 0; r < PER; ++r) {
                if (r >= per) break;
                if (e[r] && e[r] < b) f(e[r]);
            }
        });
    if (threadIdx.x == 0) sh.count = count;
    st.n = count;
    st.low = max(st.low, b);  // (no cut was needed: b is the lowest word)
}

// Cuts the words in LDS to k .. k + slack.
template <bool SUM, int NT, int PER>
DASH_DEV void top_cut(TopShared<NT, PER>& sh, TopState& st, int k, int slack, float scale) {
    uint64_t e[PER];
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const int i = r * NT + (int)threadIdx.x;
        e[r] = i < st.n ? sh.c[i] : 0;
    }
    top_keep<SUM>(sh, st, e, st.n, k, slack, scale);
    __syncthreads();
}

// Appends the words of those lanes that have one.
template <int NT, int PER>
DASH_DEV void top_append(TopShared<NT, PER>& sh, bool mine, uint64_t word) {
    const uint64_t in = __ballot(mine);
    if (!in) return;
    int at = 0;
    if ((threadIdx.x & 63) == 0) at = atomicAdd(&sh.count, __popcll(in));
    at = __builtin_amdgcn_readfirstlane(at);
    if (mine) sh.c[at + __popcll(in & ((1ull << (threadIdx.x & 63)) - 1))] = word;
}

// Leaves the k largest words of row b in LDS, at most p >= k of them (st.n), unsorted, and the row's
// other entries in the rest.
template <int NT, int PER>
DASH_DEV void top_gather(TopShared<NT, PER>& sh, TopState& st, const TopParts& parts, int64_t b, const float* row,
                         int vocab, int k, int p, float scale) {
    constexpr int kCap = NT * PER, kTile = 4 * NT;
    const TopPart* part = parts.part + b * parts.n;
    const uint64_t* words = parts.words + b * parts.n * parts.room;
    const int lane = threadIdx.x & 63;
    // every wave adds up the lists
    int n = 0;
    if (lane < parts.n) {
        const TopPart mine = part[lane];
        n = mine.n;
        if (threadIdx.x < 64 && mine.z > 0.0) {
            st.rest.half = 0.5f * mine.ref;
            st.rest.z = mine.z;
        }
    }
    const bool fits = __all(n <= parts.room);
    int upto = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(upto, o, 64);
        if (lane >= o) upto += u;
    }
    const int total = __shfl(upto, 63, 64);
    if (threadIdx.x < 64) sh.at[lane] = upto - n;
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    auto word = [&](int i) {  // the i-th of all lists
        int s = 0;
        if (parts.n > 1) {
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1)
                if (s + o < parts.n && sh.at[s + o] <= i) s += o;
        }
        return words[(int64_t)s * parts.room + i - sh.at[s]];
    };
    if (fits && total <= kCap) {
        uint64_t e[PER];
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            const int i = r * NT + (int)threadIdx.x;
            e[r] = i < total ? word(i) : 0;
        }
        top_keep<true>(sh, st, e, total, k, total > p ? p - k : total, scale);
        __syncthreads();
        return;
    }
    const int slack = (k >> 2) + 32;
    auto count = [&](auto sum) {  // after at most kTile appends: room for as many again
        __syncthreads();
        st.n = sh.count;
        __syncthreads();
        if (st.n > kCap - kTile) top_cut<decltype(sum)::value>(sh, st, k, slack, scale);
    };
    if (fits) {
        // Which words share a piece depends on the order of the lists, so none joins the rest before
        // the k largest are known.
        for (int from = 0; from < total; from += kTile) {
#pragma unroll 1
            for (int i = from + (int)threadIdx.x; i - lane < min(total, from + kTile); i += NT) {
                const uint64_t w = i < total ? word(i) : 0;
                top_append(sh, w >= max(st.low, (uint64_t)1), w);
            }
            count(std::false_type{});
        }
        top_cut<false>(sh, st, k, 0, scale);
        unsigned out = 0;
        for (int i = threadIdx.x; i < total; i += NT) {
            const uint64_t w = word(i);
            if (w < st.low) out = max(out, (unsigned)(w >> 32));
        }
        top_turn_away(sh, st, out, scale, [&](auto&& f) {
            for (int i = threadIdx.x; i < total; i += NT) {
                const uint64_t w = word(i);
                if (w < st.low) f(w);
            }
        });
        __syncthreads();
        return;
    }
    st = TopState{};
#pragma unroll 1
    for (int at = 0; at < vocab; at += kTile) {
        walk_row<1, true, NT>(row, at, min(vocab, at + kTile), [&](f32x4_t l, int i) {
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
        count(std::true_type{});
    }
    if (st.n > p) top_cut<true>(sh, st, k, p - k, scale);
}

// Words that a row's selection leaves at most: sorting pads to it.
DASH_DEV int top_room(int k) {
    int p = 64;
    while (p < k) p <<= 1;
    return p;
}

// Sorts the st.n <= p words in LDS, descending; those behind the first m = min(n, k), which it returns,
// join the rest.
template <int NT, int PER>
DASH_DEV int top_finish(TopShared<NT, PER>& sh, TopState& st, int k, int p, float scale) {
    const int n = st.n;
    for (int i = n + (int)threadIdx.x; i < p; i += NT) sh.c[i] = 0;
    __syncthreads();
    if constexpr (NT <= kTopSmall) {
        // A word's place is the number of larger ones (words differ; zeros fill what is left):
        // NT / p threads per word count over a share of the words each.  (Quadratic: 333 rows and K = 500 take 103 us
        // by counting, 96 by the exchanges below.)
        const int i = (int)threadIdx.x & (p - 1), share = (int)threadIdx.x / p, len = p * p / NT;
        const uint64_t mine = sh.c[i];
        int place = 0;
#pragma unroll 8
        for (int j = share * len; j < (share + 1) * len; ++j) place += sh.c[j] > mine;
        sh.bound.hist[threadIdx.x] = place;
        __syncthreads();
        if ((int)threadIdx.x < p) {
            for (int q = 1; q < NT / p; ++q) place += sh.bound.hist[threadIdx.x + q * p];
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
    const int m = min(n, k), i = m + (int)threadIdx.x;  // (n - m <= p - k < NT)
    if (i < n) exp_push1(st.rest, word_value(sh.c[i]), scale);
    return m;
}

}  // namespace dash
