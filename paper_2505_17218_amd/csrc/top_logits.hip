// The K largest logits of every row, sorted, and the log-sum-exp of the rest: what a teacher's
// row of 151,936 logits is reduced to for distillation.  Selection: top_logits.h.
//
// Bound by reading the row: 2048 rows of 151,936 take 203 us for k = 1 (6.1 TB/s), 236 for k = 64 (210 and 25
// in the two launches) and 410 for k = 500: what grows with k are the entries above the sampled
// bound, 9 k of such a row, each put on a list.  With 512 threads and eight tiles in flight k = 64
// took 300 us, with 512 and four 311.
#include "kernels.h"
#include "top_logits.h"

namespace dash {

namespace {

// Work-groups that run at once (two per CU), shortest stretch, what a stretch costs beside its entries
// (its bound, its last sums) in entries, longest list.
constexpr int kTopSlots = 512, kTopStretch = 8192, kTopFixed = 24576, kTopRoom = 16384;

__global__ void __launch_bounds__(kRowThreads, 8)
top_part_k(const float* __restrict__ logits, int64_t ld, int vocab, const int32_t* __restrict__ row_of, int k,
           double temperature, float scale, TopPlan plan, TopPart* __restrict__ part, uint64_t* __restrict__ words) {
    __shared__ BoundShared<kRowThreads> bound;
    __shared__ int count;
    __shared__ double red_d[kRowWaves];
    __shared__ float red_f[kRowWaves];
    const int64_t b = blockIdx.x / plan.cut.n;
    const int lo = (int)(blockIdx.x % plan.cut.n) * plan.cut.len;
    const float* row = logits + (row_of ? (int64_t)row_of[b] : b) * ld;
    words += (int64_t)blockIdx.x * plan.room;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    float thr = -INFINITY;  // entries in the list exceed it
    ExpSum rest;
    walk_row<kTopStart, true, true>(
        row, lo, min(vocab, lo + plan.cut.len),
        [&](const f32x4_t (&buf)[kTopStart], int whole) {
            uint32_t e[kTopStart / 2];
            const int real = min(max(whole, 1), kTopStart);  // the places behind repeat a tile
#pragma unroll
            for (int h = 0; h < kTopStart / 2; ++h) {
                float m = -INFINITY;
#pragma unroll
                for (int d = 2 * h; d < 2 * h + 2; ++d)
#pragma unroll
                    for (int j = 0; j < 4; ++j) m = fmaxf(m, d < real && buf[d][j] < INFINITY ? buf[d][j] : -INFINITY);
                e[h] = m > -INFINITY ? top_key(m) : 0u;
            }
            int n = kTopStart / 2 * kRowThreads;
            // (no bound where the sample holds fewer than k entries)
            const uint32_t low = top_bound<kRowThreads>(bound, e, kTopStart / 2, k, k >> 3, 0u, kKeyInf, n);
            if (low >= kKeyLowest) thr = value_below(low);
            thr = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(thr)));
        },
        [&](f32x4_t l, int i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) l[j] = fmaxf(l[j], -INFINITY);  // NaN is no entry
            if (__any(max4(l) > thr)) {
                uint64_t in[4];
                int total = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    in[j] = __ballot(l[j] > thr && l[j] < INFINITY);
                    total += __popcll(in[j]);
                }
                int at = 0;
                if ((threadIdx.x & 63) == 0) at = atomicAdd(&count, total);
                at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (!in[j]) continue;
                    const uint32_t to = (uint32_t)at + __builtin_amdgcn_mbcnt_hi((uint32_t)(in[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in[j], 0u));
                    if (l[j] > thr && l[j] < INFINITY && to < (uint32_t)plan.room)
                        *reinterpret_cast<uint64_t*>(reinterpret_cast<char*>(words) + to * 8u) = top_word(l[j], i + j);
                    at += __popcll(in[j]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) l[j] = l[j] > thr ? -INFINITY : l[j];  // (+inf is no entry either)
            }
            exp_push4<false>(rest, l, max4(l), scale);
        },
        [](int) { return false; });
    float ref;
    const double z = block_exp_sum(rest, temperature, red_f, red_d, ref);
    if (threadIdx.x == 0) part[blockIdx.x] = TopPart{z, ref, count};
}

template <int NT, int PER>
__global__ void __launch_bounds__(NT)
top_logits_k(const float* __restrict__ logits, int64_t ld, int vocab, int k, double temperature, float scale,
             TopParts parts, float* __restrict__ values, int32_t* __restrict__ indices, float* __restrict__ rest) {
    __shared__ TopShared<NT, PER> sh;
    const int64_t r = blockIdx.x;
    TopState st;
    const int p = top_room(k);
    top_gather(sh, st, parts, r, logits + r * ld, vocab, k, p, scale);
    const int m = top_finish(sh, st, k, p, scale);
    if ((int)threadIdx.x < k) {
        const bool some = (int)threadIdx.x < m;
        const uint64_t w = some ? sh.c[threadIdx.x] : 0;
        values[r * k + threadIdx.x] = some ? word_value(w) : -INFINITY;
        indices[r * k + threadIdx.x] = some ? word_index(w) : -1;
    }
    if (!rest) return;
    float ref;
    const double z = block_exp_sum<NT>(st.rest, temperature, sh.red_f, sh.red_d, ref);
    if (threadIdx.x == 0) rest[r] = z > 0.0 ? (float)((double)ref / temperature + log(z)) : -INFINITY;
}

}  // namespace

int top_logits_max() { return kTopMax; }

TopPlan top_plan(int rows, int vocab, int k) {
    auto room = [&](int len) {  // words let through: about k in every kTopStart tiles
        const int64_t want = 2 * (int64_t)k * std::max(len / (kTopStart * kRowTile), 1) + 64;
        int r = 256;
        while (r < want && r < kTopRoom) r <<= 1;
        return r;
    };
    TopPlan p;
    // The number of stretches that ends soonest, of those whose lists fit in the second launch's registers: a
    // stretch lets about k words through however short it is, hence the 2 k each (64 rows and
    // k = 1000: 59 us, 192 with 16 stretches; and 31 us with 8, 44 with 16 for k = 64).
    const int most = std::min({kTopParts, 2 * kTopSlots / std::max(rows, 1), vocab / kTopStretch, top_cap(k) / (2 * k)});
    int best = 1;
    int64_t least = INT64_MAX;
    for (int n = 1; n <= most; ++n) {
        const int64_t rounds = ((int64_t)rows * n + kTopSlots - 1) / kTopSlots, cost = rounds * (vocab / n + kTopFixed);
        if (cost < least) {
            least = cost;
            best = n;
        }
    }
    p.cut = split_row(vocab, best);
    p.room = room(p.cut.len);
    return p;
}
size_t top_workspace_bytes(int rows, int vocab, int k) {
    const TopPlan p = top_plan(rows, vocab, k);
    return (size_t)rows * p.cut.n * (sizeof(TopPart) + sizeof(uint64_t) * p.room);
}

hipError_t launch_top_parts(const float* logits, int64_t ld, int rows, int vocab, const int32_t* row_of, int k,
                            float temperature, const TopPlan& plan, void* ws, TopParts& out, hipStream_t st) {
    TopPart* part = (TopPart*)ws;
    uint64_t* words = (uint64_t*)(part + (size_t)rows * plan.cut.n);
    out = TopParts{part, words, plan.cut.n, plan.room};
    top_part_k<<<rows * plan.cut.n, kRowThreads, 0, st>>>(logits, ld, vocab, row_of, k, (double)temperature,
                                                          exp2_scale(temperature), plan, part, words);
    return hipGetLastError();
}

hipError_t launch_top_logits(const float* logits, int64_t ld, int rows, int vocab, int k, float temperature,
                             float* values, int32_t* indices, float* rest, void* ws, hipStream_t st) {
    if (rows <= 0) return hipSuccess;
    TopParts p;
    if (hipError_t e = launch_top_parts(logits, ld, rows, vocab, nullptr, k, temperature, top_plan(rows, vocab, k), ws, p, st))
        return e;
    const float scale = exp2_scale(temperature);
    auto join = [&](auto threads, auto per) {
        constexpr int NT = decltype(threads)::value, PER = decltype(per)::value;
        top_logits_k<NT, PER><<<rows, NT, 0, st>>>(logits, ld, vocab, k, (double)temperature, scale, p, values, indices, rest);
    };
    top_join_variant(k, join);
    return hipGetLastError();
}

}  // namespace dash
