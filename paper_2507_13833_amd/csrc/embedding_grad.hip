// Gradient of an embedding table.
#include "actor_device.h"

namespace dc {

constexpr int EG_THREADS = 256;

// One workgroup per row of the table and 256 columns: looks at every token, adds the rows of those that are its own.
template <typename G, typename W>
__global__ __launch_bounds__(EG_THREADS) void embedding_grad_kernel(const EmbeddingGradArgs a) {
    __shared__ uint64_t hit[EG_THREADS / WAVE];
    const int64_t c = (int64_t)blockIdx.y * EG_THREADS + threadIdx.x;
    for (int32_t v = blockIdx.x; v < a.vocab; v += gridDim.x) {
        float sum = 0.0f;
        bool any = false;
        for (int32_t t0 = 0; t0 < a.n_tokens; t0 += EG_THREADS) {
            const int32_t t = t0 + threadIdx.x, id = t < a.n_tokens ? a.token[t] : DC_NO_TOKEN;
            if (v == 0 && blockIdx.y == 0 && id != DC_NO_TOKEN && (id < 0 || id >= a.vocab)) set_status(a.status, DC_ERR_TOKEN_RANGE);
            const uint64_t b = __ballot(id == v);
            if (lane_id() == 0) hit[threadIdx.x / WAVE] = b;
            __syncthreads();
            for (int w = 0; w < EG_THREADS / WAVE; ++w)
                for (uint64_t left = hit[w]; left; left &= left - 1) {
                    any = true;
                    const int64_t row = t0 + w * WAVE + __builtin_ctzll(left);
                    if (c < a.dim) sum += (float)static_cast<const G*>(a.g)[row * a.g_stride + c];
                }
            __syncthreads();
        }
        if (c >= a.dim || (a.accumulate && !any)) continue;
        W* w = static_cast<W*>(a.dw) + (int64_t)v * a.dw_stride + c;
        *w = (W)(sum * a.scale + (a.accumulate ? (float)*w : 0.0f));
    }
}

size_t embedding_grad_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, int32_t g_type, int32_t dw_type, void*, hipStream_t st) {
    if (a.vocab == 0 || a.dim == 0) return hipSuccess;
    const dim3 grid((unsigned)(a.vocab < (1 << 20) ? a.vocab : 1 << 20), (unsigned)((a.dim + EG_THREADS - 1) / EG_THREADS));
    return with_type(g_type, [&](auto g) {
        return with_type(dw_type, [&](auto w) {
            embedding_grad_kernel<typename decltype(g)::type, typename decltype(w)::type><<<grid, EG_THREADS, 0, st>>>(a);
            return hipGetLastError();
        });
    });
}

}  // namespace dc
