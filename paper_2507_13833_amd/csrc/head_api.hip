// C-ABI entry points of the head's log-probabilities without logits and of the residual norm: host-side validation and launches,
// nothing else.
#include <cmath>
#include <utility>
#include "api_checks.h"
#include "head_internal.h"

namespace dc {

static dc_status check_head(const dc_matrix* hidden, const dc_matrix* weight, double temperature) {
    for (const dc_matrix* m : {hidden, weight}) {
        const dc_status rc = check_matrix(m);
        if (rc != DC_OK) return rc;
    }
    if (hidden->type != weight->type || hidden->n_cols != weight->n_cols || hidden->n_cols < 1 || weight->n_rows < 1) return DC_ERR_INVALID_ARG;
    if (weight->n_rows > DC_MAX_VOCAB || hidden->n_cols > DC_MAX_DIM || hidden->n_rows > DC_MAX_HEAD_ROWS) return DC_ERR_UNSUPPORTED_SIZE;
    const float inv = (float)(1.0 / temperature);
    if (!(temperature > 0.0) || !(inv >= 0x1p-100f && inv <= 0x1p100f)) return DC_ERR_INVALID_ARG;
    return DC_OK;
}

static dc_status check_workspace(size_t need, const void* d_ws, size_t ws_bytes) {
    if (need > 0 && (!d_ws || !aligned_to(d_ws, 256))) return DC_ERR_INVALID_ARG;
    return ws_bytes < need ? DC_ERR_WORKSPACE : DC_OK;
}

// A matrix of the given shape and type; type < 0: any.
static dc_status check_shaped(const dc_matrix* m, int64_t rows, int64_t cols, int32_t type) {
    const dc_status rc = check_matrix(m);
    if (rc != DC_OK) return rc;
    return m->n_rows != rows || m->n_cols != cols || (type >= 0 && m->type != type) ? DC_ERR_INVALID_ARG : DC_OK;
}

// An array of a call: rows of so many bytes, `pitch` from one to the next.
struct Place { uintptr_t p; int64_t rows, bytes, pitch; };
static Place place_of(const dc_matrix* m) {
    if (!m) return Place{};
    const int64_t each = (int64_t)elem_bytes(m->type);
    return Place{reinterpret_cast<uintptr_t>(m->d_data), m->n_rows, m->n_cols * each, m->row_stride * each};
}
static Place place_of(const void* p, int64_t bytes) { return Place{reinterpret_cast<uintptr_t>(p), 1, bytes, bytes}; }

// Whether two arrays share a byte.  Rows that interleave, as columns of one matrix do, share none.  Not decided, and so not refused:
// two of several rows with different distances that do not begin in one place.
static bool overlap(Place a, Place b) {
    if (!a.p || !b.p || a.rows < 1 || b.rows < 1 || a.bytes < 1 || b.bytes < 1) return false;
    if (a.p > b.p) std::swap(a, b);
    const int64_t d = (int64_t)(b.p - a.p);
    if (d == 0) return true;
    if (d >= (a.rows - 1) * a.pitch + a.bytes) return false;
    if (a.rows == 1) return true;
    if (b.rows > 1 && a.pitch != b.pitch) return false;
    // b begins within a row of a, or between two and reaches the next
    return d % a.pitch < a.bytes || d % a.pitch + b.bytes > a.pitch;
}
// The same, but for an output that may lie in an input's place (of the same type and shape) row by row.
static bool overlap(const dc_matrix* out, const dc_matrix* in, bool in_place) {
    if (in_place && out && in && out->d_data == in->d_data && (out->n_rows <= 1 || out->row_stride == in->row_stride)) return false;
    return overlap(place_of(out), place_of(in));
}

static dc_status check_norm(const dc_matrix* block, const dc_matrix* post, const dc_matrix* gate, const dc_matrix* pre,
                            const dc_norm_params* prm) {
    dc_status rc = check_matrix(block);
    if (rc != DC_OK) return rc;
    if (block->n_cols > DC_MAX_DIM) return DC_ERR_UNSUPPORTED_SIZE;
    for (const dc_matrix* w : {post, pre})
        if (w && (rc = check_shaped(w, 1, block->n_cols, -1)) != DC_OK) return rc;
    if (!prm || prm->reserved != 0 || (prm->gate_rows != 0 && prm->gate_rows != 1)) return DC_ERR_INVALID_ARG;
    if (gate && (rc = prm->gate_rows ? check_shaped(gate, block->n_rows, block->n_cols, block->type) : check_shaped(gate, 1, block->n_cols, -1)) != DC_OK)
        return rc;
    if (!((float)prm->eps > 0.0f && std::isfinite((float)prm->eps)) || !std::isfinite((float)prm->residual_scale) ||
        !std::isfinite((float)prm->block_scale))
        return DC_ERR_INVALID_ARG;
    return DC_OK;
}

static NormStream stream_of(const dc_matrix* m) { return m ? NormStream{m->d_data, m->row_stride} : NormStream{nullptr, 0}; }
static NormFactor factor_of(const dc_matrix* m, bool rows = false) {
    return m ? NormFactor{m->d_data, rows ? m->row_stride : 0, m->type, rows} : NormFactor{nullptr, 0, DC_F32, false};
}

}  // namespace dc

using namespace dc;

extern "C" {

size_t dc_head_logprob_workspace_bytes(const dc_matrix* hidden, const dc_matrix* weight, int32_t n_top) {
    if (check_head(hidden, weight, 1.0) != DC_OK || n_top < 0 || n_top > DC_MAX_TOP || n_top > weight->n_rows) return 0;
    return head_workspace_bytes(*hidden, *weight, n_top);
}

dc_status dc_head_logprob(const dc_matrix* hidden, const dc_matrix* weight, double temperature, const int32_t* d_token,
                          const uint8_t* d_mask, int32_t n_top, float* d_logprob, float* d_row_stat, float* d_entropy,
                          int32_t* d_top_token, float* d_top_logprob, void* d_ws, size_t ws_bytes,
                          int32_t* d_status, void* hip_stream) {
    dc_status rc = check_head(hidden, weight, temperature);
    if (rc != DC_OK) return rc;
    if (n_top < 0 || n_top > weight->n_rows) return DC_ERR_INVALID_ARG;
    if (n_top > DC_MAX_TOP) return DC_ERR_UNSUPPORTED_SIZE;
    if (hidden->n_rows > 0) {
        if ((d_token == nullptr) != (d_logprob == nullptr) || (n_top > 0 && !d_top_token && !d_top_logprob)) return DC_ERR_INVALID_ARG;
        if (!d_logprob && !d_row_stat && !d_entropy && n_top == 0) return DC_ERR_INVALID_ARG;
    }
    for (const void* p : {(const void*)d_token, (const void*)d_logprob, (const void*)d_row_stat, (const void*)d_entropy,
                          (const void*)d_top_token, (const void*)d_top_logprob})
        if (!aligned_to(p, 4)) return DC_ERR_INVALID_ARG;
    rc = check_workspace(head_workspace_need(*hidden, *weight, n_top), d_ws, ws_bytes);
    if (rc != DC_OK) return rc;
    const HeadArgs a = {*hidden, *weight, (float)(1.0 / temperature), d_token, d_mask, n_top, d_logprob, d_row_stat, d_entropy,
                        n_top ? d_top_token : nullptr, n_top ? d_top_logprob : nullptr, d_status};
    return launch_head(a, d_ws, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? DC_OK : DC_ERR_HIP;
}

size_t dc_head_logprob_backward_workspace_bytes(const dc_matrix* hidden, const dc_matrix* weight, const dc_matrix* grad_weight) {
    if (check_head(hidden, weight, 1.0) != DC_OK) return 0;
    if (grad_weight && (grad_weight->type < DC_F32 || grad_weight->type > DC_F16)) return 0;
    return head_grad_workspace_bytes(*hidden, *weight, grad_weight ? grad_weight->type : hidden->type);
}

dc_status dc_head_logprob_backward(const dc_matrix* hidden, const dc_matrix* weight, double temperature, const int32_t* d_token,
                                   const uint8_t* d_mask, const float* d_row_stat, const float* d_entropy,
                                   const float* d_grad_logprob, const float* d_grad_entropy, const dc_matrix* grad_hidden,
                                   int32_t accumulate, const dc_matrix* grad_weight, void* d_ws, size_t ws_bytes,
                                   int32_t* d_status, void* hip_stream) {
    dc_status rc = check_head(hidden, weight, temperature);
    if (rc != DC_OK) return rc;
    if (!grad_hidden && !grad_weight) return DC_ERR_INVALID_ARG;
    if (grad_hidden && (rc = check_shaped(grad_hidden, hidden->n_rows, hidden->n_cols, hidden->type)) != DC_OK) return rc;
    if (grad_weight && (rc = check_shaped(grad_weight, weight->n_rows, weight->n_cols, -1)) != DC_OK) return rc;
    if (grad_weight && grad_weight->type != weight->type && grad_weight->type != DC_F32) return DC_ERR_INVALID_ARG;
    if (hidden->n_rows > 0 && (!d_row_stat || !d_grad_logprob || (d_grad_entropy && !d_entropy))) return DC_ERR_INVALID_ARG;
    for (const void* p : {(const void*)d_token, (const void*)d_row_stat, (const void*)d_entropy, (const void*)d_grad_logprob,
                          (const void*)d_grad_entropy})
        if (!aligned_to(p, 4)) return DC_ERR_INVALID_ARG;
    const int64_t n = hidden->n_rows;
    const Place ins[] = {place_of(hidden), place_of(weight), place_of(d_token, n * 4), place_of(d_mask, n), place_of(d_row_stat, n * 8),
                         place_of(d_entropy, n * 4), place_of(d_grad_logprob, n * 4), place_of(d_grad_entropy, n * 4)};
    for (const Place& in : ins)
        if (overlap(place_of(grad_hidden), in) || overlap(place_of(grad_weight), in)) return DC_ERR_INVALID_ARG;
    if (overlap(place_of(grad_hidden), place_of(grad_weight))) return DC_ERR_INVALID_ARG;
    const int32_t type = grad_weight ? grad_weight->type : hidden->type;
    rc = check_workspace(head_grad_workspace_bytes(*hidden, *weight, type), d_ws, ws_bytes);
    if (rc != DC_OK) return rc;
    const HeadGradArgs a = {*hidden, *weight, (float)(1.0 / temperature), d_token, d_mask, d_row_stat, d_entropy, d_grad_logprob,
                            d_grad_entropy, grad_hidden ? *grad_hidden : dc_matrix{}, grad_weight ? *grad_weight : dc_matrix{},
                            accumulate != 0, d_status};
    return launch_head_grad(a, d_ws, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? DC_OK : DC_ERR_HIP;
}

dc_status dc_residual_norm(const dc_matrix* block, const dc_matrix* post_weight, const dc_matrix* gate, const dc_matrix* residual,
                           const dc_matrix* pre_weight, const dc_norm_params* prm, const dc_matrix* residual_out,
                           const dc_matrix* out, float* d_row_stat, void* hip_stream) {
    dc_status rc = check_norm(block, post_weight, gate, pre_weight, prm);
    if (rc != DC_OK) return rc;
    if (!residual || (rc = check_shaped(residual, block->n_rows, block->n_cols, -1)) != DC_OK) return residual ? rc : DC_ERR_INVALID_ARG;
    if (!residual_out || (rc = check_shaped(residual_out, block->n_rows, block->n_cols, residual->type)) != DC_OK)
        return residual_out ? rc : DC_ERR_INVALID_ARG;
    if ((pre_weight == nullptr) != (out == nullptr)) return DC_ERR_INVALID_ARG;
    if (out && (rc = check_shaped(out, block->n_rows, block->n_cols, block->type)) != DC_OK) return rc;
    if (!aligned_to(d_row_stat, 4)) return DC_ERR_INVALID_ARG;
    const Place stat = place_of(d_row_stat, block->n_rows * 8);
    for (const dc_matrix* in : {block, post_weight, gate, residual, pre_weight, residual_out, out})
        if (overlap(stat, place_of(in))) return DC_ERR_INVALID_ARG;
    for (const dc_matrix* in : {post_weight, gate, pre_weight})
        if (overlap(residual_out, in, false) || overlap(out, in, false)) return DC_ERR_INVALID_ARG;
    if (overlap(residual_out, residual, true) || overlap(residual_out, block, false) || overlap(out, residual, false) ||
        overlap(out, block, true) || overlap(residual_out, out, false))
        return DC_ERR_INVALID_ARG;
    const NormArgs a = {block->n_rows, (int32_t)block->n_cols, block->type, residual->type, (float)prm->eps, (float)prm->residual_scale,
                        (float)prm->block_scale, factor_of(post_weight), factor_of(gate, prm->gate_rows), factor_of(pre_weight), post_weight != nullptr,
                        pre_weight != nullptr, stream_of(block), stream_of(residual), stream_of(residual_out), stream_of(out), d_row_stat};
    return launch_residual_norm(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? DC_OK : DC_ERR_HIP;
}

size_t dc_residual_norm_backward_workspace_bytes(const dc_matrix* block) {
    if (!block || block->n_rows < 0 || block->n_cols < 0 || block->n_cols > DC_MAX_DIM) return 0;
    return residual_norm_workspace_bytes(block->n_rows, block->n_cols);
}

dc_status dc_residual_norm_backward(const dc_matrix* block, const dc_matrix* post_weight, const dc_matrix* gate,
                                    const dc_matrix* residual_out, const dc_matrix* pre_weight, const dc_norm_params* prm,
                                    const float* d_row_stat, const dc_matrix* grad_residual_out, const dc_matrix* grad_out,
                                    const dc_matrix* grad_block, const dc_matrix* grad_residual, int32_t accumulate,
                                    const dc_matrix* grad_post_weight, const dc_matrix* grad_gate, const dc_matrix* grad_pre_weight,
                                    void* d_ws, size_t ws_bytes, void* hip_stream) {
    dc_status rc = check_norm(block, post_weight, gate, pre_weight, prm);
    if (rc != DC_OK) return rc;
    const int64_t rows = block->n_rows, cols = block->n_cols;
    // the residual's type is that of whichever of its matrices there is
    int32_t type = -1;
    for (const dc_matrix* m : {residual_out, grad_residual_out, grad_residual})
        if (m) {
            if ((rc = check_shaped(m, rows, cols, type)) != DC_OK) return rc;
            type = m->type;
        }
    for (const dc_matrix* m : {grad_out, grad_block})
        if (m && (rc = check_shaped(m, rows, cols, block->type)) != DC_OK) return rc;
    if ((pre_weight != nullptr) != (grad_out != nullptr) || (pre_weight && !residual_out)) return DC_ERR_INVALID_ARG;
    if ((grad_post_weight && !post_weight) || (grad_gate && !gate) || (grad_pre_weight && !pre_weight)) return DC_ERR_INVALID_ARG;
    for (const dc_matrix* m : {grad_post_weight, grad_pre_weight})
        if (m && (rc = check_shaped(m, 1, cols, -1)) != DC_OK) return rc;
    const bool gate_rows = gate && prm->gate_rows;
    if (grad_gate && (rc = check_shaped(grad_gate, gate->n_rows, cols, gate_rows ? block->type : -1)) != DC_OK) return rc;
    if (rows > 0 && (post_weight || pre_weight) && !d_row_stat) return DC_ERR_INVALID_ARG;
    if (!aligned_to(d_row_stat, 4)) return DC_ERR_INVALID_ARG;
    const Place stat = place_of(d_row_stat, rows * 8);
    const dc_matrix* const outs[] = {grad_block, grad_residual, grad_post_weight, grad_gate, grad_pre_weight};
    for (int o = 0; o < 5; ++o) {
        if (overlap(place_of(outs[o]), stat)) return DC_ERR_INVALID_ARG;
        for (const dc_matrix* in : {post_weight, gate, residual_out, pre_weight})
            if (overlap(outs[o], in, false)) return DC_ERR_INVALID_ARG;
        if (overlap(outs[o], block, o == 0) || overlap(outs[o], grad_out, o == 0) || overlap(outs[o], grad_residual_out, o == 1)) return DC_ERR_INVALID_ARG;
        for (int other = 0; other < o; ++other)
            if (overlap(outs[o], outs[other], false)) return DC_ERR_INVALID_ARG;
    }
    if (!grad_block && !grad_residual && !grad_post_weight && !grad_gate && !grad_pre_weight) return DC_ERR_INVALID_ARG;
    rc = check_workspace(residual_norm_workspace_bytes(rows, cols), d_ws, ws_bytes);
    if (rc != DC_OK) return rc;
    const auto sum_of = [](const dc_matrix* m) { return m ? NormSum{m->d_data, m->type} : NormSum{nullptr, DC_F32}; };
    const NormGradArgs a = {rows, (int32_t)cols, block->type, type < 0 ? (int32_t)DC_F32 : type, (float)prm->residual_scale,
                            (float)prm->block_scale, factor_of(post_weight), factor_of(gate, prm->gate_rows), factor_of(pre_weight), post_weight != nullptr,
                            pre_weight != nullptr, stream_of(block), stream_of(residual_out), stream_of(grad_residual_out),
                            stream_of(grad_out), stream_of(grad_block), stream_of(grad_residual), stream_of(gate_rows ? grad_gate : nullptr),
                            d_row_stat, {sum_of(grad_post_weight), sum_of(gate_rows ? nullptr : grad_gate), sum_of(grad_pre_weight)},
                            accumulate != 0, static_cast<float*>(d_ws)};
    return launch_residual_norm_grad(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? DC_OK : DC_ERR_HIP;
}

}  // extern "C"
