// Host-side declarations of the actor's update: what the entry points hand to the launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include "../../include/dc.h"

namespace dc {

struct LogprobArgs {
    const void*    x;               // logits
    int64_t        stride, n_rows;
    int32_t        vocab, n_top;
    float          inv_t;           // 1 / temperature
    const int32_t* token;
    const uint8_t* mask;
    float*         logprob;
    float*         stat;
    float*         entropy;
    int32_t*       top_token;
    float*         top_logprob;
    int32_t*       status;
};
size_t logprob_workspace_need(int64_t n_rows, int32_t vocab, int32_t type, int32_t n_top);       // of this call
size_t logprob_workspace_bytes(int64_t n_rows, int32_t vocab, int32_t type, int32_t n_top);      // of it and of those of fewer rows or alternatives
hipError_t launch_logprob(const LogprobArgs& a, int32_t type, void* d_ws, hipStream_t st);

struct LogprobGradArgs {
    const void*    x;
    void*          g;               // gradient of the logits
    int64_t        stride, g_stride, n_rows;
    int32_t        vocab;
    float          inv_t;
    const int32_t* token;
    const uint8_t* mask;
    const float*   stat;
    const float*   entropy;
    const float*   grad_logprob;
    const float*   grad_entropy;
    int32_t*       status;
};
hipError_t launch_logprob_grad(const LogprobGradArgs& a, int32_t type, hipStream_t st);

struct EmbeddingArgs {
    const void*    w;
    void*          out;
    int64_t        w_stride, out_stride, n_tokens, dim;
    int32_t        vocab;
    float          scale;
    const int32_t* token;
    int32_t*       status;
};
hipError_t launch_embedding(const EmbeddingArgs& a, int32_t w_type, int32_t out_type, hipStream_t st);

constexpr int64_t EMB_GRAD_MAX_TOKENS = 1 << 24;
struct EmbeddingGradArgs {
    const void*    g;
    void*          dw;
    int64_t        g_stride, dw_stride, dim;
    int32_t        n_tokens, vocab;
    float          scale;
    int32_t        accumulate;
    const int32_t* token;
    int32_t*       status;
    int32_t        dw_bytes, dw_aligned, dw_stream;        // the launcher's: of an element; rows on multiples of 16 bytes; past the caches
};
size_t embedding_grad_workspace_need(int64_t n_tokens, int64_t dim);      // of this call
size_t embedding_grad_workspace_bytes(int64_t n_tokens, int64_t dim);     // of it and of every smaller one
hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, int32_t g_type, int32_t dw_type, void* d_ws, hipStream_t st);

// The optimizer's table: a header, the tensors, and for every piece of ADAMW_PIECE elements its tensor and its place there.
constexpr int ADAMW_PIECE = 2048;
static_assert(ADAMW_PIECE % DC_STATE_BLOCK == 0, "a block of an 8-bit state lies in one piece");
struct AdamwHeader { int64_t n_pieces; uint64_t print; int32_t n_tensors, pad; };       // print: of the tensors that it was made for
struct AdamwPiece  { int32_t tensor, piece; };
struct AdamwTable  { AdamwHeader* head; dc_adamw_tensor* tensors; AdamwPiece* pieces; size_t bytes; };
AdamwTable carve_adamw_table(void* base, int32_t n_tensors, int64_t n_pieces);
struct AdamwStep {
    float step_size, beta1, one_minus_beta1, beta2, one_minus_beta2, inv_root_bc2, eps;
    double lr64;                    // the factor of the weight decay is 1 - lr * weight_decay, rounded once
    int32_t dither;                 // roots in 8 bits go up or down by chance; `seed`: the step's
    uint32_t seed;
    const float* grad_scale;
    int32_t* status;
};
hipError_t launch_adamw_table(const dc_adamw_tensor* tensors, const AdamwHeader& head, const AdamwTable& t, hipStream_t st);
hipError_t launch_adamw(const AdamwStep& s, const AdamwHeader& head, const AdamwTable& t, hipStream_t st);

}  // namespace dc
