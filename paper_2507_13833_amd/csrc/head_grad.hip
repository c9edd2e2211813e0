// Gradients of the hidden states and of the head's weights from those of the log-probabilities and entropies.  With
// G[r, v] = (1/T) (a_r ((v == token_r) - p_v) - b_r p_v (log p_v + H_r)), the gradient of the logits that are never kept:
//   grad_hidden = G weight,  grad_weight = G^T hidden.
//
// A piece of the vocabulary at a time: its logits are made again tile by tile and become G in the tile's registers, which goes to
// the workspace once along the rows and once along the vocabulary; two products of matrices read it there.  Rows that add nothing
// (masked, or a = b = 0) take part in none of it: the live rows are numbered first.
//
// G, the weights and the hidden states are held in f16 (11 bits, three more than bf16's), each times a power of two that takes its
// largest magnitude to just below 2^15: per row for G (from |a|, |b| and H, which bound it), undone in the row's hidden gradient and in
// the row's hidden state, per piece for the weights (f16 ones stay as they are).  G in one f16 is off by at most 2^-11 of each value, before sums of 32 bits that are
// rounded to 16 bits themselves; for a gradient of the weights in 32 bits it takes two (2^-22).  Operands of 32 bits are two f16 as
// well, and three of the four products of their parts are summed (the fourth is 2^-22).
#include <algorithm>
#include "head_rows.h"

namespace dc {

// ---- per row ----

struct TermArgs {
    const void*    x;
    int64_t        stride, n_rows;
    int32_t        dim, vocab;
    float          inv_t;
    const int32_t* token;
    const float*   stat;
    const float*   entropy;
    const float*   a;
    const float*   b;
    const int32_t* pos;
    RowTerm*       term;
    int32_t*       x_exp;
    int32_t*       top;             // [0]: of the hidden states, [1 ..]: of the pieces of the weights
    int32_t*       status;
};

// A wave per row.
template <typename T>
__global__ __launch_bounds__(256) void head_terms_kernel(const TermArgs t) {
    __shared__ int tmp[4];
    const int lane = lane_id();
    int most = NO_EXPONENT;
    for (int64_t r = blockIdx.x * 4LL + threadIdx.x / WAVE; r < t.n_rows; r += gridDim.x * 4LL) {
        const int32_t at = t.pos[r];
        if (at < 0) continue;
        // (in 64 bits: a / T may be subnormal in 32 or beyond them, and what it is multiplied with takes it back)
        const double a = (double)t.a[r] * t.inv_t, b = t.b ? (double)t.b[r] * t.inv_t : 0.0, h = b != 0.0 ? (double)t.entropy[r] : 0.0;
        // |p (log p + H)| <= max(1 / e, H)
        const double bound = fabs(a) + fabs(b) * (fabs(h) + 1.0);
        const int e = bound < INFINITY ? 14 - exponent_above(bound) : 0;
        const int x_exp = exponent_above(__uint_as_float(wave_top(row_top(static_cast<const T*>(t.x) + r * t.stride, t.dim))));
        most = max(most, x_exp - e);
        if (lane == 0) {
            t.x_exp[at] = x_exp;
            int32_t token = -1;
            if (t.token) {
                token = t.token[r];
                if (token < 0 || token >= t.vocab) {
                    set_status(t.status, DC_ERR_TOKEN_RANGE);
                    token = -1;
                }
            }
            t.term[at] = RowTerm{t.stat[2 * r], t.stat[2 * r + 1] * LOG2E, (float)ldexp(b != 0.0 ? -fma(b, h, a) : -a, e),
                                 (float)(ldexp(-b, e) * (double)LN2), (float)ldexp(a, e), token, e, x_exp};
        }
    }
    raise_top(most, tmp, t.top);
}

// ---- G of a piece ----

struct HeadPieceArgs {
    Operand        w, x;
    Parts          parts;
    int32_t        steps, v0, vocab_end, tiles, row_tiles;
    const int32_t* count;
    const RowTerm* term;
    const int32_t* w_top;           // numbers of 32 bits: of the weights; the rows' own are in their terms
    float          k;
    char*          g;               // [plane][row][width], NULL: not wanted
    char*          gt;              // [plane][vocabulary entry][rows_pad], NULL: not wanted
    int64_t        width, rows_pad;
};

// A tile to a workgroup: neighbours that share its rows or its entries run beside each other on a chiplet, and nothing is kept from
// one to the next.  Bound by the matrix cores for the product and then, while they wait, by the two writes.  8192 x 15360 x 2048 bf16
// (0.52 TFLOP, and both of G's layouts, 0.5 GB): 424 to 510 us, of which the product takes about 400; 6144 x 16384 x 1024 with two
// planes along the vocabulary (0.21 TFLOP, 0.6 GB) 350.  With one plane and Q = 8 the compiler spills 4 registers behind the product.
// G along the vocabulary could be read for the weights' gradient from the one layout with transposing loads: not tried.
// T: of the operands.  PLANES of G along the vocabulary (gt), ROW_PLANES along the rows.
template <typename T, int PLANES, int ROW_PLANES, int Q>
__global__ __launch_bounds__(P_THREADS, Q == 8 ? 1 : 2) void head_piece_kernel(const HeadPieceArgs h) {
    constexpr int SIDE = P_SIDE<Q>;
    __shared__ __attribute__((aligned(1024))) char lds[P_LDS<Q>];
    const TilePair at = tile_pair(by_chiplet(blockIdx.x, h.row_tiles * h.tiles), h.row_tiles, h.tiles);
    const int32_t n_rows = *h.count, first = at.first * SIDE, t = at.second;
    if (first >= n_rows) return;
    f32x4 acc[Q][Q];
    {
        TileOfA<Q> a;
        TileOfB<Q> b;
        place_tile(a, h.w, t * SIDE, h.vocab_end - h.v0);
        place_tile(b, h.x, first, n_rows);
        product<T, Q>(acc, a, b, h.parts, h.steps, lds);
    }
    const int32_t u = t * SIDE + place_a<Q>(), row = first + place_b<Q>();
    using D = _Float16;
    const int w_exp = h.w_top ? *h.w_top - 30 : 0;
    const int64_t g_plane = h.width * h.rows_pad * 2;
    // whole: all of the tile's rows and entries are there
    const auto put = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        RowTerm of[Q];
#pragma unroll
        for (int j = 0; j < Q; ++j) of[j] = h.term[WHOLE ? row + j : min(row + j, n_rows - 1)];
        float unit[Q];                               // of the row's sums
#pragma unroll
        for (int j = 0; j < Q; ++j) unit[j] = h.w_top ? ldexpf(1.0f, of[j].x_exp + w_exp) : 1.0f;
#pragma unroll
        for (int i = 0; i < Q; i += 2) {
            // eight entries of Q rows
            const int32_t v = u + along_a(i, 0);
            float f[8][Q];
#pragma unroll
            for (int j = 0; j < Q; ++j) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float l2 = fmaf(fmaf(acc[i + e / 4][j][e % 4], unit[j], -of[j].m), h.k, -of[j].l2), p = __builtin_amdgcn_exp2f(l2);
                    f[e][j] = p * fmaf(of[j].c1, WHOLE ? l2 : fmaxf(l2, -1e4f), of[j].c0);
                }
                const uint32_t own = (uint32_t)(of[j].token - h.v0 - v);
                if (own < 8)
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e][j] += own == (uint32_t)e ? of[j].ga : 0.0f;
                if constexpr (!WHOLE)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (row + j >= n_rows || h.v0 + v + e >= h.vocab_end) f[e][j] = 0.0f;
            }
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                Raw8<D> along[Q];                    // of a row
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int j = 0; j < Q; ++j) along[j].e[e] = take_part<D>(f[e][j]);
                if (h.g && p < ROW_PLANES)
#pragma unroll
                    for (int j = 0; j < Q; ++j)
                        *reinterpret_cast<u32x4*>(h.g + p * g_plane + ((row + j) * h.width + v) * 2) = along[j].q[0];
                if (h.gt)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        struct alignas(2 * Q) { D e[Q]; } down;      // of an entry
#pragma unroll
                        for (int j = 0; j < Q; ++j) down.e[j] = along[j].e[e];
                        *reinterpret_cast<decltype(down)*>(h.gt + p * g_plane + ((v + e) * h.rows_pad + row) * 2) = down;
                    }
            }
            __builtin_amdgcn_sched_barrier(0);       // (so many at a time in registers)
        }
    };
    if (first + SIDE <= n_rows && h.v0 + (t + 1) * SIDE <= h.vocab_end) put(std::true_type{}); else put(std::false_type{});
}

// ---- the two products ----

constexpr int32_t HG_MOST_SPLITS = 32;
struct HeadHiddenArgs {             // slab[split][row][col] (+)= sum over this split's share of the piece
    Operand        wt, g;
    Parts          parts;
    int32_t        steps, splits, col_tiles, row_tiles, dim;
    const int32_t* count;
    const RowTerm* term;
    const int32_t* top;
    bool           add;
    float*         slab;
    int64_t        pitch;
};
// The summed axis, a piece of the vocabulary, is long and the tiles are few (6144 x 1024: 96): `splits` workgroups take a share of it
// each, into slabs of their own that grow from piece to piece; atomics would make the order of sums change.  Bound by the matrix cores:
// 8192 x 2048 over 15360 entries 400 to 430 us (1.2 to 1.3 PFLOP/s), 6144 x 1024 over 16384 in shares 249 (0.83).
template <int Q>
__global__ __launch_bounds__(P_THREADS, Q == 8 ? 1 : 2) void head_hidden_kernel(const HeadHiddenArgs h) {
    constexpr int SIDE = P_SIDE<Q>;
    __shared__ __attribute__((aligned(1024))) char lds[P_LDS<Q>];
    const int32_t n_rows = *h.count, row_tiles = (n_rows + SIDE - 1) / SIDE;
    const int32_t splits = live_share(h.row_tiles * h.splits, row_tiles, HG_MOST_SPLITS), others = h.col_tiles * splits;
    if ((int32_t)blockIdx.x >= row_tiles * others) return;
    const TilePair at = tile_pair(by_chiplet(blockIdx.x, row_tiles * others), row_tiles, others);
    const int32_t first = at.first * SIDE, tile = at.second % h.col_tiles, split = at.second / h.col_tiles;
    const int32_t each = (h.steps + splits - 1) / splits, from = split * each, steps = min(each, h.steps - from);
    f32x4 acc[Q][Q];
    {
        TileOfA<Q> a;
        TileOfB<Q> b;
        place_tile(a, h.wt, tile * SIDE, h.dim);
        place_tile(b, h.g, first, n_rows);
        a.base += from * (PK * 2LL);
        b.base += from * (PK * 2LL);
        product<_Float16, Q>(acc, a, b, h.parts, max(steps, 0), lds);
    }
    const int32_t col = tile * SIDE + place_a<Q>(), row = first + place_b<Q>();
#pragma unroll
    for (int j = 0; j < Q; ++j)
        if (row + j < n_rows) {
            // (the slabs hold the gradient itself: a sum of pieces with the row's own power of two might leave the range)
            const int up = *h.top - 15 - h.term[row + j].exponent;
#pragma unroll
            for (int i = 0; i < Q; ++i)
                if (col + along_a(i, 0) < h.pitch) {         // (a multiple of 4)
                    f32x4* to = reinterpret_cast<f32x4*>(h.slab + ((int64_t)split * row_tiles * SIDE + row + j) * h.pitch + col + along_a(i, 0));
                    f32x4 v = acc[i][j];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = ldexpf(v[e], up);
                    if (h.add) v += *to;
                    *to = v;
                }
        }
}

// A row's hidden gradient: the slabs' sum, rounded once.  Rows that take no part: +0.  Bound by the slabs'
// bytes, eight asked for at once (8192 x 1024 in 6 slabs: 5 us, one at a time 13).
template <typename T>
__global__ __launch_bounds__(256) void head_hidden_join_kernel(const float* slab, const int32_t* count, int32_t side, int32_t blocks, int64_t pitch,
                                                               const int32_t* pos, T* out, int64_t stride, int64_t rows, int32_t dim) {
    const int64_t each = pitch / 4, row_tiles = (*count + side - 1) / side;
    const int32_t splits = live_share(blocks, (int32_t)row_tiles, HG_MOST_SPLITS);
    for (int64_t q = blockIdx.x * 256LL + threadIdx.x; q < rows * each; q += gridDim.x * 256LL) {
        const int64_t r = q / each;
        const int32_t c = (int32_t)(q - r * each) * 4, at = pos[r];
        f32x4 sum = {0, 0, 0, 0};
        if (at >= 0) {
#pragma unroll 8
            for (int32_t s = 0; s < splits; ++s) sum += *reinterpret_cast<const f32x4*>(slab + (s * row_tiles * side + at) * pitch + c);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < dim) out[r * stride + c + i] = (T)sum[i];
    }
}

struct HeadWeightArgs {             // grad_weight[v0 + row of gt][col] (+)= sum over the live rows
    Operand        xt, gt;
    Parts          parts;
    int32_t        n, row_tiles, col_tiles, dim;
    const int32_t* count;
    const int32_t* top;
    bool           add;
    void*          out;             // of the piece's first entry
    int64_t        stride;
};
// The sum goes over the rows, for all of them in one workgroup: there are many tiles (15360 x 2048: 480).  Bound by the matrix cores:
// those over 8192 rows 390 to 418 us (1.2 to 1.3 PFLOP/s), 16384 x 1024 over 6144 with two planes of G 320 (1.3).
template <typename T, int Q>
__global__ __launch_bounds__(P_THREADS, Q == 8 ? 1 : 2) void head_weight_kernel(const HeadWeightArgs h) {
    constexpr int SIDE = P_SIDE<Q>;
    __shared__ __attribute__((aligned(1024))) char lds[P_LDS<Q>];
    const TilePair at = tile_pair(by_chiplet(blockIdx.x, h.row_tiles * h.col_tiles), h.row_tiles, h.col_tiles);
    const int32_t first = at.first * SIDE, tile = at.second;
    f32x4 acc[Q][Q];
    {
        TileOfA<Q> a;
        TileOfB<Q> b;
        place_tile(a, h.xt, tile * SIDE, h.dim);
        place_tile(b, h.gt, first, h.n);
        product<_Float16, Q>(acc, a, b, h.parts, (*h.count + PK - 1) / PK, lds);
    }
    const int up = *h.top - 15;
    const int32_t col = tile * SIDE + place_a<Q>(), row = first + place_b<Q>();
#pragma unroll
    for (int j = 0; j < Q; ++j) {
        if (row + j >= h.n) continue;
        T* to = static_cast<T*>(h.out) + (row + j) * h.stride + col;
#pragma unroll
        for (int i = 0; i < Q; i += 2) {
            const int at = along_a(i, 0);
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = ldexpf(acc[i + e / 4][j][e % 4], up);
            if (col + at + 8 <= h.dim) {
                Raw8<T> r;
                auto* p = reinterpret_cast<u32x4_a2*>(to + at);
                if (h.add) {
#pragma unroll
                    for (int q = 0; q < (int)sizeof(T) / 2; ++q) r.q[q] = p[q];
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] += (float)r.e[e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) r.e[e] = (T)f[e];
#pragma unroll
                for (int q = 0; q < (int)sizeof(T) / 2; ++q) p[q] = r.q[q];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + at + e < h.dim) to[at + e] = (T)(h.add ? f[e] + (float)to[at + e] : f[e]);
            }
        }
    }
}

// ---- the workspace ----

constexpr int64_t HG_AREA = 1 << 27;             // elements of G, or of the weights laid out, held at once

namespace {
struct HeadGradWs {
    LiveRows live;
    RowTerm* term;
    int32_t* x_exp;
    int32_t* top;
    int32_t  pieces, piece;         // entries of the vocabulary to a piece, a multiple of P_MOST_SIDE
    char*    hidden; int64_t hidden_plane;
    char*    weight; int64_t weight_plane;
    char*    xt;     int64_t xt_plane;
    char*    wt;     int64_t wt_plane;
    char*    g;
    char*    gt;     int64_t g_plane;
    float*   slab;   int64_t pitch; ProductCut cut_hidden;
    size_t   bytes;
};
}
static int64_t g_area(int64_t rows_pad, int64_t vocab_pad) {
    return std::min(rows_pad * vocab_pad, std::max(HG_AREA, rows_pad * 8 * P_MOST_SIDE));
}
// Every area grows with the rows, so that what serves a call serves those of fewer.
static HeadGradWs carve_grad(void* base, const dc_matrix& hidden, const dc_matrix& weight, int32_t grad_weight_type) {
    HeadGradWs w = {};
    const HeadShape sh = head_shape(hidden, weight, true);
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char* p = static_cast<char*>(base) + at;
        at += align256(bytes);
        return p;
    };
    const bool f32 = hidden.type == DC_F32;
    const int64_t rows = hidden.n_rows, dim = hidden.n_cols, planes = f32 ? 2 : 1, g_planes = grad_weight_type == DC_F32 ? 2 : 1;
    const int64_t vocab_pad = whole(weight.n_rows, P_MOST_SIDE);
    w.live.list = reinterpret_cast<int32_t*>(take(rows * 4));
    w.live.pos = reinterpret_cast<int32_t*>(take(rows * 4));
    w.live.count = reinterpret_cast<int32_t*>(take(4));
    w.term = reinterpret_cast<RowTerm*>(take(rows * (int64_t)sizeof(RowTerm)));
    w.x_exp = reinterpret_cast<int32_t*>(take(rows * 4));
    w.top = reinterpret_cast<int32_t*>(take((vocab_pad / P_MOST_SIDE + 1) * 4));
    const int64_t area = g_area(sh.rows_pad, vocab_pad);
    // (the weights laid out along the columns: at most HG_AREA elements too)
    const int64_t width = std::min(area / sh.rows_pad, std::max<int64_t>(HG_AREA / whole(dim, P_MOST_SIDE), 8 * P_MOST_SIDE));
    w.piece = (int32_t)std::min<int64_t>(vocab_pad, width / P_MOST_SIDE * P_MOST_SIDE);
    w.pieces = (int32_t)((vocab_pad + w.piece - 1) / w.piece);
    w.piece = (int32_t)whole((vocab_pad + w.pieces - 1) / w.pieces, P_MOST_SIDE);
    w.pieces = (int32_t)((vocab_pad + w.piece - 1) / w.piece);
    const int64_t widest = std::min(vocab_pad, std::max<int64_t>(HG_AREA / whole(dim, P_MOST_SIDE), 8 * P_MOST_SIDE));
    w.hidden_plane = rows * sh.k_pad * 2;
    w.hidden = take(sh.copy_hidden ? planes * w.hidden_plane : 0);
    w.weight_plane = (int64_t)w.piece * sh.k_pad * 2;
    w.weight = take(sh.copy_weight ? planes * widest * sh.k_pad * 2 : 0);
    w.xt_plane = dim * sh.rows_pad * 2;
    w.xt = take(planes * w.xt_plane);
    w.wt_plane = dim * w.piece * 2;
    w.wt = take(planes * dim * widest * 2);
    w.g_plane = sh.rows_pad * w.piece * 2;
    w.g = take(planes * area * 2);
    w.gt = take(g_planes * area * 2);
    w.pitch = whole(dim, 4);
    w.cut_hidden = cut_product(rows, dim, w.piece / PK * parts_of(hidden.type, 0, 0).n, HG_MOST_SPLITS);
    w.slab = reinterpret_cast<float*>(take(most_split_rows(sh.rows_pad, dim, HG_MOST_SPLITS) * w.pitch * 4));
    w.bytes = (size_t)at;
    return w;
}
size_t head_grad_workspace_bytes(const dc_matrix& hidden, const dc_matrix& weight, int32_t grad_weight_type) {
    return hidden.n_rows > 0 ? carve_grad(nullptr, hidden, weight, grad_weight_type).bytes : 0;
}

// grad_weight of a call without rows.
template <typename T>
__global__ __launch_bounds__(256) void head_no_rows_kernel(T* out, int64_t stride, int64_t rows, int32_t dim) {
    for (int64_t q = blockIdx.x * 256LL + threadIdx.x; q < rows * dim; q += gridDim.x * 256LL) out[q / dim * stride + q % dim] = (T)0.0f;
}

hipError_t launch_head_grad(const HeadGradArgs& a, void* d_ws, hipStream_t st) {
    const int64_t rows = a.hidden.n_rows;
    const dc_matrix &gh = a.grad_hidden, &gw = a.grad_weight;
    const int32_t vocab = (int32_t)a.weight.n_rows, dim = (int32_t)a.hidden.n_cols, type = a.hidden.type;
    if (rows == 0) {
        if (!gw.d_data || a.accumulate) return hipSuccess;
        return with_type(gw.type, [&](auto e) {
            using T = typename decltype(e)::type;
            head_no_rows_kernel<T><<<2048, 256, 0, st>>>(static_cast<T*>(gw.d_data), gw.row_stride, vocab, dim);
            return hipGetLastError();
        });
    }
    const HeadGradWs w = carve_grad(d_ws, a.hidden, a.weight, gw.d_data ? gw.type : type);
    const HeadShape sh = head_shape(a.hidden, a.weight, true);
    const bool f32 = type == DC_F32;
    hipError_t e = launch_live_rows(a.mask, a.grad_logprob, a.grad_entropy, rows, w.live, {w.top, w.pieces + 1, type == DC_F16}, st);
    const TermArgs t = {a.hidden.d_data, a.hidden.row_stride, rows, dim, vocab, a.inv_t, a.token, a.stat, a.entropy,
                        a.grad_logprob, a.grad_entropy, w.live.pos, w.term, w.x_exp, w.top, a.status};
    const unsigned waves4 = (unsigned)std::min<int64_t>((rows + 3) / 4, TOP_BLOCKS);
    if (e == hipSuccess) e = with_type(type, [&](auto el) {
        head_terms_kernel<typename decltype(el)::type><<<waves4, 256, 0, st>>>(t);
        return hipGetLastError();
    });
    HeadPieceArgs p = {};
    p.steps = sh.k_pad / PK;
    p.parts = parts_of(type, w.weight_plane, w.hidden_plane);
    p.count = w.live.count;
    p.term = w.term;
    p.k = a.inv_t * LOG2E;
    p.g = gh.d_data ? w.g : nullptr;
    p.gt = gw.d_data ? w.gt : nullptr;
    p.width = w.piece;
    p.rows_pad = sh.rows_pad;
    if (sh.copy_hidden) {
        if (e == hipSuccess) e = launch_lay_rows(a.hidden, 0, rows, w.live.list, w.live.count, sh.k_pad, w.hidden, w.hidden_plane, F16S, w.x_exp, nullptr, st);
        p.x = Operand{w.hidden, sh.k_pad * 2, nullptr};
    } else {
        p.x = Operand{static_cast<const char*>(a.hidden.d_data), a.hidden.row_stride * 2, w.live.list};
    }
    if (gw.d_data && e == hipSuccess)
        e = launch_lay_columns(a.hidden, 0, rows, w.live.list, w.live.count, sh.rows_pad, w.top, w.term, w.xt, w.xt_plane, st);
    HeadHiddenArgs hh = {};
    hh.wt = Operand{w.wt, w.piece * 2LL, nullptr};
    hh.g = Operand{w.g, w.piece * 2LL, nullptr};
    hh.parts = parts_of(type, w.wt_plane, w.g_plane);
    hh.splits = w.cut_hidden.splits;
    const auto tiles_of = [](int64_t n, bool small) { return (int32_t)((n + (small ? P_SIDE<4> : P_SIDE<8>) - 1) / (small ? P_SIDE<4> : P_SIDE<8>)); };
    hh.col_tiles = tiles_of(dim, w.cut_hidden.small);
    hh.row_tiles = tiles_of(rows, w.cut_hidden.small);
    hh.dim = dim;
    hh.count = w.live.count;
    hh.term = w.term;
    hh.slab = w.slab;
    hh.pitch = w.pitch;
    HeadWeightArgs hw = {};
    hw.xt = Operand{w.xt, sh.rows_pad * 2, nullptr};
    hw.gt = Operand{w.gt, sh.rows_pad * 2, nullptr};
    hw.parts = parts_of(type, w.xt_plane, w.g_plane);
    const bool two = gw.d_data && !f32 && gw.type == DC_F32;
    if (two) hw.parts = Parts{2, 0, 1, 0, w.g_plane};        // the small one first
    hw.dim = dim;
    hw.count = w.live.count;
    hw.top = w.top;
    hw.add = a.accumulate;
    hw.stride = gw.row_stride;
    const int64_t out_bytes = gw.type == DC_F32 ? 4 : 2;
    for (int32_t i = 0; i < w.pieces && e == hipSuccess; ++i) {
        const int32_t v0 = i * w.piece, n = std::min(w.piece, vocab - v0);
        int32_t* const top_w = w.top + 1 + i;
        if (f32 || (gh.d_data && type == DC_BF16)) e = launch_top_exponent(a.weight, v0, n, top_w, st);
        if (gh.d_data && e == hipSuccess) e = launch_lay_columns(a.weight, v0, n, nullptr, nullptr, w.piece, top_w, nullptr, w.wt, w.wt_plane, st);
        if (sh.copy_weight) {
            if (e == hipSuccess) e = launch_lay_rows(a.weight, v0, n, nullptr, nullptr, sh.k_pad, w.weight, w.weight_plane, F16S, nullptr, top_w, st);
            p.w = Operand{w.weight, sh.k_pad * 2, nullptr};
        } else {
            p.w = Operand{static_cast<const char*>(a.weight.d_data) + v0 * a.weight.row_stride * 2, a.weight.row_stride * 2, nullptr};
        }
        p.w_top = f32 ? top_w : nullptr;
        if (e != hipSuccess) break;
        p.v0 = v0;
        p.vocab_end = v0 + n;
        const bool small_piece = cut_product(rows, n, p.steps * p.parts.n, 1).small,
                   small_weight = cut_product(n, dim, sh.rows_pad / PK * hw.parts.n, 1).small;
        p.tiles = tiles_of(n, small_piece);
        p.row_tiles = tiles_of(rows, small_piece);
        const auto piece = [&](auto t, auto planes, auto row_planes) {
            using T = decltype(t);
            constexpr int PLANES = decltype(planes)::value, ROW_PLANES = decltype(row_planes)::value;
            const unsigned blocks = (unsigned)(p.row_tiles * p.tiles);
            if (small_piece) head_piece_kernel<T, PLANES, ROW_PLANES, 4><<<blocks, P_THREADS, 0, st>>>(p);
            else head_piece_kernel<T, PLANES, ROW_PLANES, 8><<<blocks, P_THREADS, 0, st>>>(p);
        };
        using One = std::integral_constant<int, 1>;
        using Two = std::integral_constant<int, 2>;
        if (f32) piece(_Float16{}, Two{}, Two{});
        else if (type == DC_BF16 && two) piece(__bf16{}, Two{}, One{});
        else if (type == DC_BF16) piece(__bf16{}, One{}, One{});
        else if (two) piece(_Float16{}, Two{}, One{});
        else piece(_Float16{}, One{}, One{});
        if (gh.d_data) {
            hh.steps = (n + PK - 1) / PK;
            hh.top = top_w;
            hh.add = i > 0;
            const unsigned b = (unsigned)(hh.row_tiles * hh.col_tiles * hh.splits);
            if (w.cut_hidden.small) head_hidden_kernel<4><<<b, P_THREADS, 0, st>>>(hh);
            else head_hidden_kernel<8><<<b, P_THREADS, 0, st>>>(hh);
        }
        if (gw.d_data) {
            hw.n = n;
            hw.row_tiles = tiles_of(n, small_weight);
            hw.col_tiles = tiles_of(dim, small_weight);
            hw.out = static_cast<char*>(gw.d_data) + v0 * gw.row_stride * out_bytes;
            const unsigned b = (unsigned)(hw.row_tiles * hw.col_tiles);
            e = with_type(gw.type, [&](auto el) {
                using T = typename decltype(el)::type;
                if (small_weight) head_weight_kernel<T, 4><<<b, P_THREADS, 0, st>>>(hw);
                else head_weight_kernel<T, 8><<<b, P_THREADS, 0, st>>>(hw);
                return hipGetLastError();
            });
        }
        if (e == hipSuccess) e = hipGetLastError();
    }
    if (gh.d_data && e == hipSuccess)
        e = with_type(gh.type, [&](auto el) {
            using T = typename decltype(el)::type;
            head_hidden_join_kernel<T><<<(unsigned)std::min<int64_t>((rows * (w.pitch / 4) + 255) / 256, 1 << 14), 256, 0, st>>>(
                w.slab, w.live.count, w.cut_hidden.small ? P_SIDE<4> : P_SIDE<8>, hh.row_tiles * hh.splits, w.pitch, w.live.pos, static_cast<T*>(gh.d_data), gh.row_stride, rows, dim);
            return hipGetLastError();
        });
    return e;
}

}  // namespace dc
