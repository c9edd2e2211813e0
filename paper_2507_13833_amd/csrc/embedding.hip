// Embedding of token ids: rows of a table, scaled.
#include "actor_device.h"

namespace dc {

constexpr int EMB_THREADS = 256;

// One workgroup per token, element by element.
template <typename W, typename O>
__global__ __launch_bounds__(EMB_THREADS) void embedding_kernel(const EmbeddingArgs a) {
    for (int64_t t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
        const int32_t id = a.token[t];
        const bool in = id >= 0 && id < a.vocab;
        if (!in && id != DC_NO_TOKEN && threadIdx.x == 0) set_status(a.status, DC_ERR_TOKEN_RANGE);
        const W* w = static_cast<const W*>(a.w) + (in ? (int64_t)id * a.w_stride : 0);
        O* o = static_cast<O*>(a.out) + t * a.out_stride;
        for (int64_t c = threadIdx.x; c < a.dim; c += EMB_THREADS) o[c] = in ? (O)((float)w[c] * a.scale) : (O)0.0f;
    }
}

hipError_t launch_embedding(const EmbeddingArgs& a, int32_t w_type, int32_t out_type, hipStream_t st) {
    if (a.n_tokens == 0 || a.dim == 0) return hipSuccess;
    const unsigned grid = (unsigned)(a.n_tokens < (1 << 20) ? a.n_tokens : 1 << 20);
    return with_type(w_type, [&](auto w) {
        return with_type(out_type, [&](auto o) {
            embedding_kernel<typename decltype(w)::type, typename decltype(o)::type><<<grid, EMB_THREADS, 0, st>>>(a);
            return hipGetLastError();
        });
    });
}

}  // namespace dc
