// Log-probabilities of given tokens with entropy and top alternatives, and the gradient of the logits.
#include "actor_device.h"

namespace dc {

constexpr int LP_THREADS = 256;

// One workgroup per row; the row is read once for its maximum, once for the sums, once per alternative.
template <typename T>
__global__ __launch_bounds__(LP_THREADS) void logprob_kernel(const LogprobArgs a) {
    __shared__ float tmp[LP_THREADS / WAVE];
    __shared__ uint64_t tmp64[LP_THREADS / WAVE];
    for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
        if (a.mask && a.mask[r] == 0) {
            if (threadIdx.x == 0) {
                if (a.logprob) a.logprob[r] = 0.0f;
                if (a.entropy) a.entropy[r] = 0.0f;
                if (a.stat) { a.stat[2 * r] = 0.0f; a.stat[2 * r + 1] = 0.0f; }
            }
            for (int i = threadIdx.x; i < a.n_top; i += LP_THREADS) {
                if (a.top_token) a.top_token[r * a.n_top + i] = -1;
                if (a.top_logprob) a.top_logprob[r * a.n_top + i] = 0.0f;
            }
            continue;
        }
        const T* x = static_cast<const T*>(a.x) + r * a.stride;
        float m = -INFINITY;
        for (int v = threadIdx.x; v < a.vocab; v += LP_THREADS) m = fmaxf(m, (float)x[v]);
        m = block_reduce(m, tmp, wave_max, [](float p, float q) { return fmaxf(p, q); });
        float s = 0.0f, u = 0.0f;
        for (int v = threadIdx.x; v < a.vocab; v += LP_THREADS) {
            const float d = ((float)x[v] - m) * a.inv_t;
            const float e = __builtin_amdgcn_exp2f(d * LOG2E);
            s += e;
            u += e * fmaxf(d, -1e4f);               // e is 0 long before: -infinity adds 0, not a NaN
        }
        const auto add = [](float p, float q) { return p + q; };
        s = block_reduce(s, tmp, wave_sum, add);
        u = block_reduce(u, tmp, wave_sum, add);
        const bool good = s >= 1.0f;                // (the maximum alone adds 1; NaN, +infinity, nothing finite: a NaN)
        const float log_sum = good ? logf(s) : NAN;
        if (threadIdx.x == 0) {
            if (a.token) {
                const int32_t t = a.token[r];
                const bool in = t >= 0 && t < a.vocab;
                if (!in) set_status(a.status, DC_ERR_TOKEN_RANGE);
                a.logprob[r] = in ? ((float)x[t] - m) * a.inv_t - log_sum : NAN;
            }
            if (a.entropy) a.entropy[r] = log_sum - u / s;
            if (a.stat) { a.stat[2 * r] = good ? m : NAN; a.stat[2 * r + 1] = log_sum; }
        }
        uint64_t below = ~0ull;
        for (int i = 0; i < a.n_top; ++i) {
            uint64_t best = 0;
            for (int v = threadIdx.x; v < a.vocab; v += LP_THREADS) {
                const uint64_t key = ((uint64_t)sortable((float)x[v]) << 32) | (uint32_t)~v;
                if (key < below && key > best) best = key;
            }
            best = block_reduce(best, tmp64, wave_max_u64, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
            if (threadIdx.x == 0) {
                if (a.top_token) a.top_token[r * a.n_top + i] = good ? (int32_t)~(uint32_t)best : -1;
                if (a.top_logprob) a.top_logprob[r * a.n_top + i] = (unsortable((uint32_t)(best >> 32)) - m) * a.inv_t - log_sum;
            }
            below = best;
        }
    }
}

size_t logprob_workspace_bytes(int64_t, int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_logprob(const LogprobArgs& a, int32_t type, void*, hipStream_t st) {
    if (a.n_rows == 0) return hipSuccess;
    const unsigned grid = (unsigned)(a.n_rows < (1 << 20) ? a.n_rows : 1 << 20);
    return with_type(type, [&](auto e) {
        using T = typename decltype(e)::type;
        logprob_kernel<T><<<grid, LP_THREADS, 0, st>>>(a);
        return hipGetLastError();
    });
}

// One workgroup per row, element by element.
template <typename T>
__global__ __launch_bounds__(LP_THREADS) void logprob_grad_kernel(const LogprobGradArgs a) {
    for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.stride;
        T* g = static_cast<T*>(a.g) + r * a.g_stride;
        const float ga = a.grad_logprob[r], gb = a.grad_entropy ? a.grad_entropy[r] : 0.0f;
        if ((a.mask && a.mask[r] == 0) || (ga == 0.0f && gb == 0.0f)) {
            for (int v = threadIdx.x; v < a.vocab; v += LP_THREADS) g[v] = (T)0.0f;
            continue;
        }
        const float m = a.stat[2 * r], log_sum = a.stat[2 * r + 1], h = gb != 0.0f ? a.entropy[r] : 0.0f;
        int32_t token = -1;
        if (a.token) {
            token = a.token[r];
            if ((token < 0 || token >= a.vocab) && threadIdx.x == 0) set_status(a.status, DC_ERR_TOKEN_RANGE);
        }
        for (int v = threadIdx.x; v < a.vocab; v += LP_THREADS) {
            const float lp = ((float)x[v] - m) * a.inv_t - log_sum;
            const float p = __builtin_amdgcn_exp2f(lp * LOG2E);
            const float d = (v == token ? ga : 0.0f) - p * (ga + gb * (fmaxf(lp, -1e4f) + h));
            g[v] = (T)(d * a.inv_t);
        }
    }
}

hipError_t launch_logprob_grad(const LogprobGradArgs& a, int32_t type, hipStream_t st) {
    if (a.n_rows == 0) return hipSuccess;
    const unsigned grid = (unsigned)(a.n_rows < (1 << 20) ? a.n_rows : 1 << 20);
    return with_type(type, [&](auto e) {
        using T = typename decltype(e)::type;
        logprob_grad_kernel<T><<<grid, LP_THREADS, 0, st>>>(a);
        return hipGetLastError();
    });
}

}  // namespace dc
