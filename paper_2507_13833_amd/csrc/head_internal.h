// Host-side declarations of the head's log-probabilities without logits, and of the residual norm.
#pragma once
#include "actor_internal.h"

namespace dc {

struct HeadArgs {
    dc_matrix      hidden, weight;
    float          inv_t;           // 1 / temperature
    const int32_t* token;
    const uint8_t* mask;
    int32_t        n_top;
    float*         logprob;
    float*         stat;
    float*         entropy;
    int32_t*       top_token;
    float*         top_logprob;
    int32_t*       status;
};
size_t head_workspace_need(const dc_matrix& hidden, const dc_matrix& weight, int32_t n_top);    // of this call
size_t head_workspace_bytes(const dc_matrix& hidden, const dc_matrix& weight, int32_t n_top);   // of it and of those of fewer rows or alternatives
hipError_t launch_head(const HeadArgs& a, void* d_ws, hipStream_t st);

struct HeadGradArgs {
    dc_matrix      hidden, weight;
    float          inv_t;
    const int32_t* token;
    const uint8_t* mask;
    const float*   stat;
    const float*   entropy;
    const float*   grad_logprob;
    const float*   grad_entropy;
    dc_matrix      grad_hidden, grad_weight;     // d_data NULL: not wanted
    int32_t        accumulate;
    int32_t*       status;
};
size_t head_grad_workspace_bytes(const dc_matrix& hidden, const dc_matrix& weight, int32_t grad_weight_type);     // of this call and those of fewer rows
hipError_t launch_head_grad(const HeadGradArgs& a, void* d_ws, hipStream_t st);

// ---- the residual norm ----

// A row of factors for all rows (stride 0), or one for each.  p NULL: 1.
struct NormFactor { const void* p; int64_t stride; int32_t type; bool rows; };
struct NormStream { void* p; int64_t stride; };          // p NULL: there is none
struct NormArgs {
    int64_t    rows;
    int32_t    dim, act, res;       // types: of the block's and of the residual's streams
    float      eps, residual_scale, block_scale;
    NormFactor post, gate, pre;
    bool       has_post, has_pre;
    NormStream block, residual, residual_out, out;
    float*     stat;
};
hipError_t launch_residual_norm(const NormArgs& a, hipStream_t st);

struct NormSum { void* p; int32_t type; };               // a gradient of one row
struct NormGradArgs {
    int64_t     rows;
    int32_t     dim, act, res;
    float       residual_scale, block_scale;
    NormFactor  post, gate, pre;
    bool        has_post, has_pre;
    NormStream  block, residual_out, grad_residual_out, grad_out, grad_block, grad_residual, grad_gate;      // grad_gate: of a gate per row
    const float* stat;
    NormSum     sum[3];             // post, gate, pre
    int32_t     accumulate;
    float*      part;               // [block][3][dim]
};
size_t residual_norm_workspace_bytes(int64_t rows, int64_t dim);
hipError_t launch_residual_norm_grad(const NormGradArgs& a, hipStream_t st);

}  // namespace dc
