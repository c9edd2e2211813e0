// C-ABI entry points of the actor's update: host-side validation and launches, nothing else.
#include <cmath>
#include <cstring>
#include "api_checks.h"

namespace dc {

static dc_status check_logits(const dc_matrix* m, double temperature) {
    const dc_status rc = check_matrix(m);
    if (rc != DC_OK) return rc;
    if (m->n_cols < 1) return DC_ERR_INVALID_ARG;
    if (m->n_cols > DC_MAX_VOCAB) return DC_ERR_UNSUPPORTED_SIZE;
    const float inv = (float)(1.0 / temperature);
    if (!(temperature > 0.0) || !(inv >= 0x1p-100f && inv <= 0x1p100f)) return DC_ERR_INVALID_ARG;
    return DC_OK;
}

static dc_status check_tensors(const dc_adamw_tensor* t, int32_t n, int64_t* n_pieces) {
    if (n < 0 || (n > 0 && !t)) return DC_ERR_INVALID_ARG;
    if (n > DC_MAX_TENSORS) return DC_ERR_UNSUPPORTED_SIZE;
    int64_t pieces = 0;
    for (int32_t i = 0; i < n; ++i) {
        const dc_adamw_tensor& d = t[i];
        if (d.n < 0 || d.reserved != 0 || !(d.weight_decay >= 0.0 && std::isfinite(d.weight_decay))) return DC_ERR_INVALID_ARG;
        if (d.param_type < DC_F32 || d.param_type > DC_F16 || d.grad_type < DC_F32 || d.grad_type > DC_F16)
            return DC_ERR_INVALID_ARG;
        if (d.state_type != DC_F32 && d.state_type != DC_E4M3) return DC_ERR_INVALID_ARG;
        if (d.n > (1LL << 40)) return DC_ERR_UNSUPPORTED_SIZE;
        if (d.n == 0) continue;
        const size_t s = elem_bytes(d.state_type);
        if (!d.d_param || !d.d_grad || !d.d_exp_avg || !d.d_exp_avg_sq) return DC_ERR_INVALID_ARG;
        if (!aligned_to(d.d_param, elem_bytes(d.param_type)) || !aligned_to(d.d_master, 4) ||
            !aligned_to(d.d_grad, elem_bytes(d.grad_type)) || !aligned_to(d.d_exp_avg, s) || !aligned_to(d.d_exp_avg_sq, s))
            return DC_ERR_INVALID_ARG;
        if (d.state_type == DC_E4M3 && (!d.d_exp_avg_scale || !d.d_exp_avg_sq_scale || !aligned_to(d.d_exp_avg_scale, 4) ||
                                        !aligned_to(d.d_exp_avg_sq_scale, 4)))
            return DC_ERR_INVALID_ARG;
        pieces += (d.n + ADAMW_PIECE - 1) / ADAMW_PIECE;
        if (pieces > 0x7FFFFFFFLL) return DC_ERR_UNSUPPORTED_SIZE;
    }
    *n_pieces = pieces;
    return DC_OK;
}

// What dc_adamw_table writes and dc_adamw looks for at the table's start: 64 bits of everything that the kernel would take out of
// the table, so that one made for other tensors, or for these before they changed, is not used.
static AdamwHeader header_of(const dc_adamw_tensor* t, int32_t n, int64_t n_pieces) {
    uint64_t print = 0x9E3779B97F4A7C15u;
    const auto add = [&](uint64_t word) {        // (one to one in the word and in what came before)
        print = (print ^ word) * 0xD6E8FEB86659FD93u;
        print ^= print >> 32;
    };
    for (int32_t i = 0; i < n; ++i) {
        const dc_adamw_tensor& d = t[i];
        add((uint64_t)d.n);
        if (d.n == 0) continue;
        for (const void* p : {(const void*)d.d_param, (const void*)d.d_master, d.d_grad, (const void*)d.d_exp_avg, (const void*)d.d_exp_avg_sq})
            add(reinterpret_cast<uintptr_t>(p));
        if (d.state_type == DC_E4M3)
            for (const void* p : {(const void*)d.d_exp_avg_scale, (const void*)d.d_exp_avg_sq_scale}) add(reinterpret_cast<uintptr_t>(p));
        const double decay = d.weight_decay + 0.0;               // (a zero's sign does not count)
        uint64_t bits;
        std::memcpy(&bits, &decay, sizeof bits);
        add(bits);
        add((uint64_t)d.param_type << 16 | (uint64_t)d.grad_type << 8 | (uint64_t)d.state_type);
    }
    return AdamwHeader{n_pieces, print, n, 0};
}

}  // namespace dc

using namespace dc;

extern "C" {

size_t dc_token_logprob_workspace_bytes(const dc_matrix* logits, int32_t n_top) {
    if (check_logits(logits, 1.0) != DC_OK || n_top < 0 || n_top > DC_MAX_TOP) return 0;
    return logprob_workspace_bytes(logits->n_rows, (int32_t)logits->n_cols, logits->type, n_top);
}

dc_status dc_token_logprob(const dc_matrix* logits, double temperature, const int32_t* d_token, const uint8_t* d_mask,
                           int32_t n_top, float* d_logprob, float* d_row_stat, float* d_entropy,
                           int32_t* d_top_token, float* d_top_logprob, void* d_ws, size_t ws_bytes,
                           int32_t* d_status, void* hip_stream) {
    const dc_status rc = check_logits(logits, temperature);
    if (rc != DC_OK) return rc;
    if (n_top < 0 || n_top > logits->n_cols) return DC_ERR_INVALID_ARG;
    if (n_top > DC_MAX_TOP) return DC_ERR_UNSUPPORTED_SIZE;
    if (logits->n_rows > 0) {
        if ((d_token == nullptr) != (d_logprob == nullptr) || (n_top > 0 && !d_top_token && !d_top_logprob)) return DC_ERR_INVALID_ARG;
        if (!d_logprob && !d_row_stat && !d_entropy && n_top == 0) return DC_ERR_INVALID_ARG;
    }
    for (const void* p : {(const void*)d_token, (const void*)d_logprob, (const void*)d_row_stat, (const void*)d_entropy,
                          (const void*)d_top_token, (const void*)d_top_logprob})
        if (!aligned_to(p, 4)) return DC_ERR_INVALID_ARG;
    const size_t need = logprob_workspace_need(logits->n_rows, (int32_t)logits->n_cols, logits->type, n_top);
    if (need > 0 && (!d_ws || !aligned_to(d_ws, 256))) return DC_ERR_INVALID_ARG;
    if (ws_bytes < need) return DC_ERR_WORKSPACE;
    const LogprobArgs a = {logits->d_data, logits->row_stride, logits->n_rows, (int32_t)logits->n_cols, n_top,
                           (float)(1.0 / temperature), d_token, d_mask, d_logprob, d_row_stat, d_entropy,
                           n_top ? d_top_token : nullptr, n_top ? d_top_logprob : nullptr, d_status};
    const hipError_t e = launch_logprob(a, logits->type, d_ws, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? DC_OK : DC_ERR_HIP;
}

dc_status dc_token_logprob_backward(const dc_matrix* logits, double temperature, const int32_t* d_token,
                                    const uint8_t* d_mask, const float* d_row_stat, const float* d_entropy,
                                    const float* d_grad_logprob, const float* d_grad_entropy,
                                    const dc_matrix* grad_logits, int32_t* d_status, void* hip_stream) {
    dc_status rc = check_logits(logits, temperature);
    if (rc != DC_OK) return rc;
    rc = check_matrix(grad_logits);
    if (rc != DC_OK) return rc;
    if (grad_logits->n_rows != logits->n_rows || grad_logits->n_cols != logits->n_cols || grad_logits->type != logits->type)
        return DC_ERR_INVALID_ARG;
    if (grad_logits->d_data == logits->d_data && logits->n_rows > 1 && grad_logits->row_stride != logits->row_stride)
        return DC_ERR_INVALID_ARG;
    if (logits->n_rows > 0 && (!d_row_stat || !d_grad_logprob || (d_grad_entropy && !d_entropy))) return DC_ERR_INVALID_ARG;
    for (const void* p : {(const void*)d_token, (const void*)d_row_stat, (const void*)d_entropy,
                          (const void*)d_grad_logprob, (const void*)d_grad_entropy})
        if (!aligned_to(p, 4)) return DC_ERR_INVALID_ARG;
    const LogprobGradArgs a = {logits->d_data, grad_logits->d_data, logits->row_stride, grad_logits->row_stride,
                               logits->n_rows, (int32_t)logits->n_cols, (float)(1.0 / temperature), d_token, d_mask,
                               d_row_stat, d_entropy, d_grad_logprob, d_grad_entropy, d_status};
    const hipError_t e = launch_logprob_grad(a, logits->type, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? DC_OK : DC_ERR_HIP;
}

dc_status dc_embedding(const dc_matrix* weight, const int32_t* d_token, double scale, const dc_matrix* out,
                       int32_t* d_status, void* hip_stream) {
    dc_status rc = check_matrix(weight);
    if (rc != DC_OK) return rc;
    rc = check_matrix(out);
    if (rc != DC_OK) return rc;
    if (weight->n_cols != out->n_cols || !std::isfinite((float)scale)) return DC_ERR_INVALID_ARG;
    if (weight->n_rows > DC_MAX_VOCAB || weight->n_cols > DC_MAX_DIM) return DC_ERR_UNSUPPORTED_SIZE;
    if (out->n_rows > 0 && (!d_token || !aligned_to(d_token, 4))) return DC_ERR_INVALID_ARG;
    const EmbeddingArgs a = {weight->d_data, out->d_data, weight->row_stride, out->row_stride, out->n_rows, out->n_cols,
                             (int32_t)weight->n_rows, (float)scale, d_token, d_status};
    const hipError_t e = launch_embedding(a, weight->type, out->type, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? DC_OK : DC_ERR_HIP;
}

size_t dc_embedding_backward_workspace_bytes(const dc_matrix* grad_out, const dc_matrix* grad_weight) {
    if (!grad_out || !grad_weight || grad_out->n_rows < 0 || grad_out->n_rows > EMB_GRAD_MAX_TOKENS || grad_weight->n_rows < 0 ||
        grad_weight->n_rows > DC_MAX_VOCAB || grad_out->n_cols < 0 || grad_out->n_cols > DC_MAX_DIM)
        return 0;
    return embedding_grad_workspace_bytes(grad_out->n_rows, grad_out->n_cols);
}

dc_status dc_embedding_backward(const dc_matrix* grad_out, const int32_t* d_token, double scale, int32_t accumulate,
                                const dc_matrix* grad_weight, void* d_ws, size_t ws_bytes,
                                int32_t* d_status, void* hip_stream) {
    dc_status rc = check_matrix(grad_out);
    if (rc != DC_OK) return rc;
    rc = check_matrix(grad_weight);
    if (rc != DC_OK) return rc;
    if (grad_weight->n_cols != grad_out->n_cols || !std::isfinite((float)scale)) return DC_ERR_INVALID_ARG;
    if (grad_weight->n_rows > DC_MAX_VOCAB || grad_weight->n_cols > DC_MAX_DIM || grad_out->n_rows > EMB_GRAD_MAX_TOKENS ||
        grad_out->n_rows * grad_out->n_cols > 1LL << 38)                 // (a launch's threads)
        return DC_ERR_UNSUPPORTED_SIZE;
    if (grad_out->n_rows > 0 && (!d_token || !aligned_to(d_token, 4))) return DC_ERR_INVALID_ARG;
    const size_t need = embedding_grad_workspace_need(grad_out->n_rows, grad_out->n_cols);
    if (need > 0 && (!d_ws || !aligned_to(d_ws, 256))) return DC_ERR_INVALID_ARG;
    if (ws_bytes < need) return DC_ERR_WORKSPACE;
    const EmbeddingGradArgs a = {grad_out->d_data, grad_weight->d_data, grad_out->row_stride, grad_weight->row_stride,
                                 grad_out->n_cols, (int32_t)grad_out->n_rows, (int32_t)grad_weight->n_rows, (float)scale,
                                 accumulate != 0, d_token, d_status};
    const hipError_t e = launch_embedding_grad(a, grad_out->type, grad_weight->type, d_ws, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? DC_OK : DC_ERR_HIP;
}

size_t dc_adamw_table_bytes(const dc_adamw_tensor* tensors, int32_t n_tensors) {
    int64_t n_pieces = 0;
    if (check_tensors(tensors, n_tensors, &n_pieces) != DC_OK) return 0;
    return carve_adamw_table(nullptr, n_tensors, n_pieces).bytes;
}

dc_status dc_adamw_table(const dc_adamw_tensor* tensors, int32_t n_tensors, void* d_table, size_t table_bytes,
                         void* hip_stream) {
    int64_t n_pieces = 0;
    const dc_status rc = check_tensors(tensors, n_tensors, &n_pieces);
    if (rc != DC_OK) return rc;
    if (!d_table || !aligned_to(d_table, 256)) return DC_ERR_INVALID_ARG;
    const AdamwTable t = carve_adamw_table(d_table, n_tensors, n_pieces);
    if (table_bytes < t.bytes) return DC_ERR_WORKSPACE;
    const hipError_t e = launch_adamw_table(tensors, header_of(tensors, n_tensors, n_pieces), t, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? DC_OK : DC_ERR_HIP;
}

dc_status dc_adamw(const dc_adamw_tensor* tensors, int32_t n_tensors, const dc_adamw_params* prm, const float* d_grad_scale,
                   const void* d_table, size_t table_bytes, int32_t* d_status, void* hip_stream) {
    int64_t n_pieces = 0;
    const dc_status rc = check_tensors(tensors, n_tensors, &n_pieces);
    if (rc != DC_OK) return rc;
    if (!prm || !(prm->lr >= 0.0 && std::isfinite(prm->lr)) || !(prm->beta1 >= 0.0 && prm->beta1 < 1.0) ||
        !(prm->beta2 >= 0.0 && prm->beta2 < 1.0) || !(prm->eps >= 0x1p-100 && prm->eps <= 0x1p100) || prm->step < 1)
        return DC_ERR_INVALID_ARG;
    if (!d_table || !aligned_to(d_table, 256) || !aligned_to(d_grad_scale, 4)) return DC_ERR_INVALID_ARG;
    const AdamwTable t = carve_adamw_table(const_cast<void*>(d_table), n_tensors, n_pieces);
    if (table_bytes < t.bytes) return DC_ERR_WORKSPACE;
    const double bc1 = 1.0 - std::pow(prm->beta1, (double)prm->step), bc2 = 1.0 - std::pow(prm->beta2, (double)prm->step);
    // what the kernel multiplies by, in 32 bits
    if (!std::isfinite((float)(prm->lr / bc1))) return DC_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n_tensors; ++i)
        if (!std::isfinite((float)(1.0 - prm->lr * tensors[i].weight_decay))) return DC_ERR_INVALID_ARG;
    // the share that this step's gradient has in v, once the average is corrected for its start at 0
    const bool dither = (1.0 - prm->beta2) / bc2 < 1.0 / 24;
    uint64_t seed = (uint64_t)prm->step * 0x9E3779B97F4A7C15u;             // (an odd multiple of each step: all differ)
    seed = (seed ^ seed >> 32) * 0xD6E8FEB86659FD93u;
    const AdamwStep s = {(float)(prm->lr / bc1), (float)prm->beta1, (float)(1.0 - prm->beta1),
                         (float)prm->beta2, (float)(1.0 - prm->beta2), (float)(1.0 / std::sqrt(bc2)), (float)prm->eps,
                         prm->lr, dither, (uint32_t)(seed >> 32), d_grad_scale, d_status};
    const hipError_t e = launch_adamw(s, header_of(tensors, n_tensors, n_pieces), t, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? DC_OK : DC_ERR_HIP;
}

}  // extern "C"
