// Log-probabilities of given tokens straight from hidden states and the head's weights: the logits x = hidden weight^T are made
// tile by tile on the matrix cores and come down to a row's sums where they are.
//
// A workgroup keeps 128 rows and goes through its share of the vocabulary, 256 columns at a time.  A lane has four rows, and of
// each tile 32 logits of every one, all in registers: their largest M, S = sum 2^(k (x - M)) and U = sum 2^(k (x - M)) k (x - M)
// with k = log2(e) / T join what the lane has from the tiles before, and lanes and waves are joined at the end.  Products of
// 16-bit floats are exact and summed in 32 bits.  Numbers of 32 bits are taken apart into three of bf16 (24 bits together), and
// the six products of parts that reach 2^-24 are summed, the smallest first.
#include <algorithm>
#include "head_rows.h"

namespace dc {

struct HeadStatArgs {
    Operand        w, x;
    Parts          parts;
    int32_t        steps, v0, vocab_end, tiles;      // vocabulary entries v0 .. vocab_end - 1 are rows 0 .. of w; tiles: of PM
    int32_t        row_tiles, segments, n_rows;
    const int32_t* count;           // NULL: n_rows
    const int32_t* list;            // of the rows, for their tokens; NULL: as they lie
    const int32_t* token;
    float          k;
    bool           add;             // to what an earlier piece of the vocabulary left
    RowSums*       sums;            // [row][segment]
    float*         x_token;
};

template <typename T, bool ENTROPY>
__global__ __launch_bounds__(P_THREADS, 2) void head_stat_kernel(const HeadStatArgs h) {
    __shared__ __attribute__((aligned(1024))) char lds[P_LDS];
    const int32_t blocks = h.row_tiles * h.segments;
    const TilePair at = tile_pair(by_chiplet(blockIdx.x, blocks), h.row_tiles, h.segments);
    const int32_t n_rows = h.count ? *h.count : h.n_rows, first = at.first * PN;
    if (first >= n_rows) return;
    const int lane = lane_id(), wave = threadIdx.x / WAVE;
    const int32_t my_row = first + wave % 2 * (PN / 2) + (lane & 15);        // and 16, 32, 48 behind it
    int32_t token[P_NT];
    float m[P_NT], s[P_NT], u[P_NT];
#pragma unroll
    for (int j = 0; j < P_NT; ++j) {
        const int32_t r = my_row + 16 * j;
        token[j] = -1;
        if (h.token && r < n_rows) token[j] = h.token[h.list ? h.list[r] : r];
        m[j] = -INFINITY;
        s[j] = u[j] = 0.0f;
    }
    TileOfB b;
    place_tile(b, h.x, first, n_rows);
    for (int32_t t = at.second; t < h.tiles; t += h.segments) {
        TileOfA a;
        place_tile(a, h.w, t * PM, h.vocab_end - h.v0);
        f32x4 acc[P_MT][P_NT];
        product<T>(acc, a, b, h.parts, h.steps, lds);
        const int32_t v = h.v0 + t * PM + wave / 2 * (PM / 2) + (lane >> 4) * 4;     // of acc[0][.][0]
        if (h.v0 + (t + 1) * PM > h.vocab_end)
#pragma unroll
            for (int i = 0; i < P_MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (v + 16 * i + e >= h.vocab_end)
#pragma unroll
                        for (int j = 0; j < P_NT; ++j) acc[i][j][e] = -INFINITY;
#pragma unroll
        for (int j = 0; j < P_NT; ++j) {
            const uint32_t off = (uint32_t)(token[j] - v);
            if (off < PM / 2 && (off & 12) == 0) {
                float x = 0.0f;
#pragma unroll
                for (int i = 0; i < P_MT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x = off == (uint32_t)(16 * i + e) ? acc[i][j][e] : x;
                h.x_token[my_row + 16 * j] = x;
            }
            float most = m[j];
#pragma unroll
            for (int i = 0; i < P_MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, acc[i][j][e]);
            const float base = most > -INFINITY ? most : 0.0f;
            const float d0 = fmaxf((m[j] - base) * h.k, -1e4f), f = __builtin_amdgcn_exp2f(d0);
            if constexpr (ENTROPY) u[j] = f * (u[j] + d0 * s[j]);
            s[j] *= f;
            m[j] = most;
#pragma unroll
            for (int i = 0; i < P_MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float d = (acc[i][j][e] - base) * h.k, p = __builtin_amdgcn_exp2f(d);
                    s[j] += p;
                    if constexpr (ENTROPY) u[j] = fmaf(p, fmaxf(d, -1e4f), u[j]);     // (a logit of -infinity adds 0, not a NaN)
                }
        }
    }
    // the four lanes and the two waves that share a row
    const auto join = [&](RowSums p, RowSums q) {
        RowSums r = {fmaxf(p.m, q.m), 0.0f, 0.0f};
        const float base = r.m > -INFINITY ? r.m : 0.0f;
        const float dp = fmaxf((p.m - base) * h.k, -1e4f), dq = fmaxf((q.m - base) * h.k, -1e4f);
        const float fp = __builtin_amdgcn_exp2f(dp), fq = __builtin_amdgcn_exp2f(dq);
        r.s = fp * p.s + fq * q.s;
        r.u = fp * (p.u + dp * p.s) + fq * (q.u + dq * q.s);
        return r;
    };
    RowSums* tmp = reinterpret_cast<RowSums*>(lds);
    bare_barrier();
#pragma unroll
    for (int j = 0; j < P_NT; ++j) {
        RowSums r = {m[j], s[j], u[j]};
#pragma unroll
        for (int d = 16; d < 64; d <<= 1) r = join(r, RowSums{__shfl_xor(r.m, d), __shfl_xor(r.s, d), __shfl_xor(r.u, d)});
        if (lane < 16) tmp[wave * (PN / 2) + 16 * j + lane] = r;
    }
    __syncthreads();
    const int32_t row = first + threadIdx.x;
    if (threadIdx.x < PN && row < n_rows) {
        RowSums r = join(tmp[threadIdx.x], tmp[PN + threadIdx.x]);
        RowSums* to = h.sums + (int64_t)row * h.segments + at.second;
        if (h.add) r = join(*to, r);
        *to = r;
    }
}

// A row's logits in 32 bits, for rows whose alternatives are wanted.
template <typename T>
__global__ __launch_bounds__(P_THREADS, 2) void head_logits_kernel(const HeadStatArgs h, float* logits, int64_t pitch) {
    __shared__ __attribute__((aligned(1024))) char lds[P_LDS];
    const TilePair at = tile_pair(by_chiplet(blockIdx.x, h.row_tiles * h.tiles), h.row_tiles, h.tiles);
    const int32_t first = at.first * PN, t = at.second;
    const int lane = lane_id(), wave = threadIdx.x / WAVE;
    TileOfA a;
    TileOfB b;
    place_tile(a, h.w, t * PM, h.vocab_end - h.v0);
    place_tile(b, h.x, first, h.n_rows);
    f32x4 acc[P_MT][P_NT];
    product<T>(acc, a, b, h.parts, h.steps, lds);
    const int32_t v = h.v0 + t * PM + wave / 2 * (PM / 2) + (lane >> 4) * 4, row = first + wave % 2 * (PN / 2) + (lane & 15);
#pragma unroll
    for (int j = 0; j < P_NT; ++j)
        if (row + 16 * j < h.n_rows)
#pragma unroll
            for (int i = 0; i < P_MT; ++i)
                if (v + 16 * i < h.vocab_end)        // (the pitch is a multiple of 4)
                    *reinterpret_cast<f32x4*>(logits + (row + 16 * j) * pitch + v + 16 * i) = acc[i][j];
}

// A wave per row: its segments' sums as one, and the results.
__global__ __launch_bounds__(256) void head_join_kernel(const LogprobArgs a, const int32_t* pos, int32_t segments, const RowSums* sums,
                                                        const float* x_token) {
    const float k = a.inv_t * LOG2E;
    const int lane = lane_id();
    for (int64_t r = blockIdx.x * 4LL + threadIdx.x / WAVE; r < a.n_rows; r += gridDim.x * 4LL) {
        const int64_t at = pos ? pos[r] : r;
        if (at < 0) {
            if (lane == 0) {
                if (a.logprob) a.logprob[r] = 0.0f;
                if (a.entropy) a.entropy[r] = 0.0f;
                if (a.stat) { a.stat[2 * r] = 0.0f; a.stat[2 * r + 1] = 0.0f; }
            }
            continue;
        }
        RowSums all = {-INFINITY, 0.0f, 0.0f};
        for (int p = lane; p < segments; p += WAVE) all.m = fmaxf(all.m, sums[at * segments + p].m);
        all.m = wave_max(all.m);
        const float base = all.m > -INFINITY ? all.m : 0.0f;
        for (int p = lane; p < segments; p += WAVE) {
            const RowSums x = sums[at * segments + p];
            const float d = fmaxf((x.m - base) * k, -1e4f), f = __builtin_amdgcn_exp2f(d);
            all.s += f * x.s;
            all.u += f * (x.u + d * x.s);
        }
        all.s = wave_sum(all.s);
        all.u = wave_sum(all.u);
        if (lane == 0) {
            const int32_t token = a.token ? a.token[r] : 0;
            const bool in = token >= 0 && token < a.vocab;
            if (!in) set_status(a.status, DC_ERR_TOKEN_RANGE);
            write_row(a, r, finish(all, a.inv_t), in, in && a.token ? x_token[at] : 0.0f);
        }
    }
}

// How the vocabulary is shared out over workgroups: `segments` to each tile of rows, so that two to a compute unit finish at
// about the same time.
constexpr int32_t HEAD_SLOTS = 512, HEAD_MOST_BLOCKS = 4 * HEAD_SLOTS;
static int32_t segments_of(int64_t row_tiles, int32_t tiles) {
    int32_t best = 1;
    int64_t least = -1;
    for (int32_t s = 1; s <= tiles && row_tiles * s <= HEAD_MOST_BLOCKS; ++s) {
        const int64_t rounds = (row_tiles * s + HEAD_SLOTS - 1) / HEAD_SLOTS * ((tiles + s - 1) / s);
        if (least < 0 || rounds < least) { least = rounds; best = s; }
    }
    return best;
}

constexpr int64_t HEAD_TOP_ROWS = PN;            // rows whose logits are held at once
constexpr int64_t HEAD_PIECE_BYTES = 256LL << 20;    // of weights laid out at once
static int32_t weight_piece(const HeadShape& sh, const dc_matrix& w) {
    if (!sh.copy_weight) return (int32_t)w.n_rows;
    const int64_t row = sh.k_pad * 2LL * (w.type == DC_F32 ? 3 : 1);
    return (int32_t)std::min<int64_t>(whole(w.n_rows, PM), std::max<int64_t>(PM, HEAD_PIECE_BYTES / row / PM * PM));
}

namespace {
struct HeadWs {
    char*    hidden; int64_t hidden_plane;
    char*    weight; int64_t weight_plane; int32_t piece;
    LiveRows live;
    float*   x_token;
    RowSums* sums;
    float*   logits; int64_t pitch;
    char*    logprob;
    size_t   bytes;
};
}
// Areas for rows and sums grow with the rows; which of the two ways needs which does not matter for the layout.
static HeadWs carve(void* base, const dc_matrix& hidden, const dc_matrix& weight, int32_t n_top) {
    HeadWs w = {};
    const HeadShape sh = head_shape(hidden, weight, true);
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char* p = static_cast<char*>(base) + at;
        at += align256(bytes);
        return p;
    };
    const int64_t rows = hidden.n_rows, planes = hidden.type == DC_F32 ? 3 : 1;
    w.hidden_plane = rows * sh.k_pad * 2;
    w.hidden = take(sh.copy_hidden ? planes * w.hidden_plane : 0);
    w.piece = weight_piece(sh, weight);
    w.weight_plane = (int64_t)w.piece * sh.k_pad * 2;
    w.weight = take(sh.copy_weight ? planes * w.weight_plane : 0);
    w.pitch = whole(weight.n_rows, 4);
    if (n_top > 0) {
        w.logits = reinterpret_cast<float*>(take(std::min(rows, HEAD_TOP_ROWS) * w.pitch * 4));
        w.logprob = take((int64_t)logprob_workspace_bytes(std::min(rows, HEAD_TOP_ROWS), (int32_t)weight.n_rows, DC_F32, n_top));
    } else {
        w.live.list = reinterpret_cast<int32_t*>(take(rows * 4));
        w.live.pos = reinterpret_cast<int32_t*>(take(rows * 4));
        w.live.count = reinterpret_cast<int32_t*>(take(4));
        w.x_token = reinterpret_cast<float*>(take(rows * 4));
        // (as many segments as any number of tiles of rows up to this one's has: blocks never pass their limit, nor tiles of both)
        const int64_t row_tiles = sh.rows_pad / PN, tiles = whole(weight.n_rows, PM) / PM;
        const int64_t blocks = std::max<int64_t>(row_tiles, std::min<int64_t>(HEAD_MOST_BLOCKS, row_tiles * tiles));
        w.sums = reinterpret_cast<RowSums*>(take(blocks * PN * (int64_t)sizeof(RowSums)));
    }
    w.bytes = (size_t)at;
    return w;
}
size_t head_workspace_need(const dc_matrix& hidden, const dc_matrix& weight, int32_t n_top) {
    return hidden.n_rows > 0 ? carve(nullptr, hidden, weight, n_top).bytes : 0;
}
size_t head_workspace_bytes(const dc_matrix& hidden, const dc_matrix& weight, int32_t n_top) {
    return std::max(head_workspace_need(hidden, weight, 0), head_workspace_need(hidden, weight, n_top));
}

hipError_t launch_head(const HeadArgs& a, void* d_ws, hipStream_t st) {
    const int64_t rows = a.hidden.n_rows;
    if (rows == 0) return hipSuccess;
    const int32_t vocab = (int32_t)a.weight.n_rows, type = a.hidden.type;
    const HeadWs w = carve(d_ws, a.hidden, a.weight, a.n_top);
    const HeadShape sh = head_shape(a.hidden, a.weight, true);
    hipError_t e = hipSuccess;
    const bool live = a.n_top == 0 && a.mask;
    if (live) e = launch_live_rows(a.mask, nullptr, nullptr, rows, w.live, st);
    HeadStatArgs h = {};
    h.steps = sh.k_pad / PK;
    h.parts = parts_of(type, w.weight_plane, w.hidden_plane);
    h.k = a.inv_t * LOG2E;
    h.token = a.token;
    h.sums = w.sums;
    h.x_token = w.x_token;
    h.row_tiles = (int32_t)(sh.rows_pad / PN);
    h.n_rows = (int32_t)rows;
    h.count = live ? w.live.count : nullptr;
    h.list = live ? w.live.list : nullptr;
    h.segments = segments_of(h.row_tiles, (std::min(w.piece, vocab) + PM - 1) / PM);
    if (sh.copy_hidden) {
        if (e == hipSuccess) e = launch_lay_rows(a.hidden, 0, rows, h.list, h.count, sh.k_pad, w.hidden, w.hidden_plane, st);
        h.x = Operand{w.hidden, sh.k_pad * 2, nullptr};
    } else {
        h.x = Operand{static_cast<const char*>(a.hidden.d_data), a.hidden.row_stride * 2, h.list};
    }
    LogprobArgs out = {nullptr, w.pitch, rows, vocab, a.n_top, a.inv_t, a.token, a.mask, a.logprob, a.stat, a.entropy,
                       a.top_token, a.top_logprob, a.status};
    for (int64_t r0 = 0; r0 < rows && e == hipSuccess; r0 += HEAD_TOP_ROWS) {
        if (a.n_top > 0) {                       // so many rows at a time
            h.n_rows = (int32_t)std::min(HEAD_TOP_ROWS, rows - r0);
            h.row_tiles = 1;
        }
        for (int32_t v0 = 0; v0 < vocab && e == hipSuccess; v0 += w.piece) {
            const int32_t n = std::min(w.piece, vocab - v0);
            if (sh.copy_weight) {
                e = launch_lay_rows(a.weight, v0, n, nullptr, nullptr, sh.k_pad, w.weight, w.weight_plane, st);
                h.w = Operand{w.weight, sh.k_pad * 2, nullptr};
            } else {
                h.w = Operand{static_cast<const char*>(a.weight.d_data), a.weight.row_stride * 2, nullptr};
            }
            if (e != hipSuccess) break;
            h.v0 = v0;
            h.vocab_end = v0 + n;
            h.tiles = (n + PM - 1) / PM;
            h.add = v0 > 0;
            const auto go = [&](auto t) {
                using T = decltype(t);
                if (a.n_top > 0) head_logits_kernel<T><<<h.tiles, P_THREADS, 0, st>>>(h, w.logits, w.pitch);
                else if (a.entropy) head_stat_kernel<T, true><<<h.row_tiles * h.segments, P_THREADS, 0, st>>>(h);
                else head_stat_kernel<T, false><<<h.row_tiles * h.segments, P_THREADS, 0, st>>>(h);
            };
            if (type == DC_F16) go(_Float16{}); else go(__bf16{});
            e = hipGetLastError();
        }
        if (a.n_top == 0) break;
        LogprobArgs o = out;
        o.x = w.logits;
        o.n_rows = h.n_rows;
        const auto from = [&](auto* p, int64_t each) { return p ? p + r0 * each : p; };
        o.token = from(a.token, 1);
        o.mask = from(a.mask, 1);
        o.logprob = from(a.logprob, 1);
        o.stat = from(a.stat, 2);
        o.entropy = from(a.entropy, 1);
        o.top_token = from(a.top_token, a.n_top);
        o.top_logprob = from(a.top_logprob, a.n_top);
        if (e == hipSuccess) e = launch_logprob(o, DC_F32, w.logprob, st);
        h.x.p += HEAD_TOP_ROWS * h.x.pitch;
    }
    if (e != hipSuccess || a.n_top > 0) return e;
    head_join_kernel<<<(unsigned)std::min<int64_t>((rows + 3) / 4, 1 << 16), 256, 0, st>>>(out, live ? w.live.pos : nullptr, h.segments,
                                                                                          w.sums, w.x_token);
    return hipGetLastError();
}

}  // namespace dc
