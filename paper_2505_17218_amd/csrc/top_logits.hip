// The K largest logits of every row, sorted, and the log-sum-exp of the rest: what a teacher's
// row of 151,936 logits is reduced to for distillation.  Selection: top_logits.h.
#include "kernels.h"
#include "top_logits.h"

namespace dash {

namespace {

__global__ void __launch_bounds__(kRowThreads)
top_logits_k(const float* __restrict__ logits, int64_t ld, int vocab, int k, double temperature, float scale,
             float* __restrict__ values, int32_t* __restrict__ indices, float* __restrict__ rest) {
    __shared__ TopShared sh;
    const int64_t r = blockIdx.x;
    TopState st;
    top_begin(sh);
    top_walk(sh, st, logits + r * ld, 0, vocab, k, scale);
    const int m = top_finish(sh, st, k, scale);
    if ((int)threadIdx.x < k) {
        const bool some = (int)threadIdx.x < m;
        const uint64_t w = some ? sh.c[threadIdx.x] : 0;
        values[r * k + threadIdx.x] = some ? word_value(w) : -INFINITY;
        indices[r * k + threadIdx.x] = some ? word_index(w) : -1;
    }
    if (!rest) return;
    float ref;
    const double z = top_rest(sh, st, temperature, ref);
    if (threadIdx.x == 0) rest[r] = z > 0.0 ? (float)((double)ref / temperature + log(z)) : -INFINITY;
}

}  // namespace

int top_logits_max() { return kTopMax; }

hipError_t launch_top_logits(const float* logits, int64_t ld, int rows, int vocab, int k, float temperature,
                             float* values, int32_t* indices, float* rest, hipStream_t st) {
    if (rows <= 0) return hipSuccess;
    top_logits_k<<<rows, kRowThreads, 0, st>>>(logits, ld, vocab, k, (double)temperature, exp2_scale(temperature),
                                               values, indices, rest);
    return hipGetLastError();
}

}  // namespace dash
