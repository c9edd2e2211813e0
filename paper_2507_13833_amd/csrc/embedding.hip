// Embedding of token ids: rows of a table, scaled.
#include "actor_device.h"

namespace dc {

constexpr int EMB_THREADS = 256;

// One wave per ROWS tokens and 512 columns; the rows are asked for together.  Bound by the streams: a row of the table in,
// a row out.  Many rows leave past the caches, which then keep rows of the table that come again (131 072 tokens of 2048
// bf16 out of 152 064: 146 us, 5.3 TB/s; 162 us with plain stores; two or eight rows a wave: within 4 %).  Rows that do not start
// on 16 bytes or whose width is no multiple of 8 go element by element: 207 us for 2047 columns.
template <int ROWS, Layout L, typename W, typename O>
__global__ __launch_bounds__(EMB_THREADS) void embedding_kernel(const EmbeddingArgs a, int64_t units, int32_t slabs) {
    const int lane = lane_id();
    const int64_t step = (int64_t)gridDim.x * (EMB_THREADS / WAVE);
    for (int64_t unit = (int64_t)blockIdx.x * (EMB_THREADS / WAVE) + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE); unit < units;
         unit += step) {
        const int64_t group = unit / slabs, t0 = group * ROWS;
        const int32_t slab = (int32_t)(unit - group * slabs);
        const int n = (int)min((int64_t)ROWS, a.n_tokens - t0);
        int32_t id = DC_NO_TOKEN;
        if (lane < n) id = a.token[t0 + lane];
        const bool in = id >= 0 && id < a.vocab;
        if (!in && id != DC_NO_TOKEN && slab == 0) set_status(a.status, DC_ERR_TOKEN_RANGE);
        const uint64_t there = __ballot(in);
        Raw8<W> w[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if ((there >> j) & 1)
                load8<L>(static_cast<const W*>(a.w) + (int64_t)__builtin_amdgcn_readlane(id, j) * a.w_stride, slab, a.dim, w[j]);
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            if (j >= n) break;
            float f[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) f[c] = (there >> j) & 1 ? (float)w[j].e[c] * a.scale : 0.0f;
            store8<L, (ROWS > 1)>(static_cast<O*>(a.out) + (t0 + j) * a.out_stride, slab, a.dim, f);
        }
    }
}

hipError_t launch_embedding(const EmbeddingArgs& a, int32_t w_type, int32_t out_type, hipStream_t st) {
    if (a.n_tokens == 0 || a.dim == 0) return hipSuccess;
    const int32_t slabs = (int32_t)((a.dim + COLS - 1) / COLS);
    // a wave per token until there are enough of them to fill the chip
    const bool few = a.n_tokens * slabs < 8192;
    const int64_t units = (few ? a.n_tokens : (a.n_tokens + 3) / 4) * slabs, blocks = (units + EMB_THREADS / WAVE - 1) / (EMB_THREADS / WAVE);
    const unsigned grid = (unsigned)(blocks < (1 << 23) ? blocks : 1 << 23);
    return with_type(w_type, [&](auto we) {
        return with_type(out_type, [&](auto oe) {
            using W = typename decltype(we)::type;
            using O = typename decltype(oe)::type;
            const bool vec = a.dim % 8 == 0 && rows_aligned<W>(a.w, a.w_stride) && rows_aligned<O>(a.out, a.out_stride);
            constexpr Layout L = sizeof(O) == 4 ? FOURS : EIGHTS;
            if (few && vec) embedding_kernel<1, L, W, O><<<grid, EMB_THREADS, 0, st>>>(a, units, slabs);
            else if (few) embedding_kernel<1, APART, W, O><<<grid, EMB_THREADS, 0, st>>>(a, units, slabs);
            else if (vec) embedding_kernel<4, L, W, O><<<grid, EMB_THREADS, 0, st>>>(a, units, slabs);
            else embedding_kernel<4, APART, W, O><<<grid, EMB_THREADS, 0, st>>>(a, units, slabs);
            return hipGetLastError();
        });
    });
}

}  // namespace dc
