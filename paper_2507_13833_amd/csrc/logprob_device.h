// What a row of logits comes down to, and how its results are written: shared by the kernels that read logits and by those that
// make them.
#pragma once
#include "actor_device.h"

namespace dc {

// What a row comes down to: its largest logit, S = sum exp((x - M)/T), U = sum exp((x - M)/T) * (x - M)/T * log2(e).
struct RowSums { float m, s, u; };

struct RowResult { float m, inv_t, log_sum, entropy; bool good; };
__device__ __forceinline__ RowResult finish(const RowSums& r, float inv_t) {
    // the largest logit alone adds 1; a NaN, +infinity or nothing above -infinity makes the sum a NaN or 0
    const bool good = r.s >= 0.5f && r.s < INFINITY;
    RowResult w = {good ? r.m : NAN, inv_t, good ? logf(r.s) : NAN, 0.0f, good};
    w.entropy = w.log_sum - r.u / r.s * LN2;
    return w;
}
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t r, const RowResult& w, bool in, float x_token) {
    if (a.logprob) a.logprob[r] = in ? (x_token - w.m) * w.inv_t - w.log_sum : NAN;
    if (a.entropy) a.entropy[r] = w.good ? w.entropy : NAN;
    if (a.stat) { a.stat[2 * r] = w.m; a.stat[2 * r + 1] = w.log_sum; }
}
__device__ __forceinline__ void write_top(const LogprobArgs& a, int64_t r, int i, const RowResult& w, uint64_t key) {
    if (a.top_token) a.top_token[r * a.n_top + i] = w.good ? (int32_t)~(uint32_t)key : -1;
    if (a.top_logprob) a.top_logprob[r * a.n_top + i] = w.good ? (unsortable((uint32_t)(key >> 32)) - w.m) * w.inv_t - w.log_sum : NAN;
}
// A masked row.  Every thread of the workgroup comes here.
__device__ __forceinline__ void write_nothing(const LogprobArgs& a, int64_t r) {
    if (threadIdx.x == 0) {
        if (a.logprob) a.logprob[r] = 0.0f;
        if (a.entropy) a.entropy[r] = 0.0f;
        if (a.stat) { a.stat[2 * r] = 0.0f; a.stat[2 * r + 1] = 0.0f; }
    }
    for (int i = threadIdx.x; i < a.n_top; i += blockDim.x) {
        if (a.top_token) a.top_token[r * a.n_top + i] = -1;
        if (a.top_logprob) a.top_logprob[r * a.n_top + i] = 0.0f;
    }
}

}  // namespace dc
