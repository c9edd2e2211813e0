// Log-probabilities of given tokens straight from hidden states and the head's weights: the logits x = hidden weight^T are made
// tile by tile on the matrix cores and come down to a row's sums where they are.
//
// A workgroup keeps 256 (128) rows and goes through its share of the vocabulary, as many entries at a time.  A lane has Q rows, and of
// each tile 4 Q logits of every one, all in registers: their largest M, S = sum 2^(k (x - M)) and U = sum 2^(k (x - M)) k (x - M)
// with k = log2(e) / T join what the lane has from the tiles before, and lanes and waves are joined at the end.  Products of
// 16-bit floats are exact and summed in 32 bits.  Numbers of 32 bits, times powers of two that take a row's, or the weights', largest to
// just below 2^15, are taken apart into two of f16 (22 bits together), and three of the four products are summed, the smallest first.
// Up to 64 rows they are three of bf16 (24 bits) and six products: that is bound by memory.
#include <algorithm>
#include "head_rows.h"

namespace dc {

struct HeadStatArgs {
    Operand        w, x;
    Parts          parts;
    int32_t        steps, v0, vocab_end, tiles;      // vocabulary entries v0 .. vocab_end - 1 are rows 0 .. of w; tiles: of P_SIDE
    int32_t        row_tiles, segments, n_rows, most_tiles;      // for all rows; most_tiles: of the first piece
    const int32_t* count;           // NULL: n_rows
    const int32_t* list;            // of the rows, for their tokens; NULL: as they lie
    const int32_t* token;
    const int32_t* x_exp;           // numbers of 32 bits: of the rows, and of the weights, as launch_lay_rows has them; else NULL
    const int32_t* w_exp;
    float          k;
    bool           add;             // to what an earlier piece of the vocabulary left
    RowSums*       sums;            // [row][segment]
    float*         x_token;
};

// What a lane's sums of a row are relative to, in powers of two: k m for its largest logit m until now, rounded (k x less it is one
// operation then), or from LOGIT_FAR on, where that rounding would be felt, k m itself, by differences taken first.
constexpr float LOGIT_FAR = 0x1p24f;
// How far what a lane's sums were relative to (for the largest logit m until now) lies below what they become relative to.
__device__ __forceinline__ float less_reference(float m, float k, float base, float base2, bool far) {
    const float m2 = m * k;
    const bool was_far = fabsf(m2) >= LOGIT_FAR;
    if (far) return was_far ? (m - base) * k : fmaf(-base, k, m2);
    return was_far ? fmaf(m, k, -base2) : m2 - base2;
}

// Bound by the matrix cores, and by the clock that the card holds under them (1.5 to 1.6 of 2.4 GHz): the next tile's first operands
// come while a tile's sums are taken.  us a call, Q = 8: 8192 rows x 152064 x 2048 bf16 3660 to 3830 (1.33 to 1.39 PFLOP/s; a
// library's product of these sizes alone 3580), 6144 of 8192 x 32000 x 1024 345 (1.17); 200 of 333 x 32003 x 515 f32 115,
// of which it takes 52.  With entropies and Q = 8 the compiler spills 6 registers, outside the products.
// Also measured on the large one: 128 rows by 256 entries, two workgroups to a compute unit, 5500; eight waves of 128 by 64 with four
// shorter stages 4650; sums that the compiler places 12 700 (copied from and to their registers).
template <typename T, bool ENTROPY, int Q>
__global__ __launch_bounds__(P_THREADS, Q == 8 ? 1 : 2) void head_stat_kernel(const HeadStatArgs h) {
    constexpr int SIDE = P_SIDE<Q>;
    __shared__ __attribute__((aligned(1024))) char lds[P_LDS<Q>];
    const int32_t n_rows = h.count ? *h.count : h.n_rows, row_tiles = (n_rows + SIDE - 1) / SIDE;
    const int32_t segments = live_share(h.row_tiles * h.segments, row_tiles, h.most_tiles);
    if ((int32_t)blockIdx.x >= row_tiles * segments) return;
    const TilePair at = tile_pair(by_chiplet(blockIdx.x, row_tiles * segments), row_tiles, segments);
    const int32_t first = at.first * SIDE;
    const int lane = lane_id(), wave = threadIdx.x / WAVE;
    const int32_t my_row = first + place_b<Q>();        // and the Q - 1 behind it
    // sums of products of numbers of 32 bits are in units of the row's own: kr takes those to powers of two, as k does logits
    int32_t token[Q];
    float m[Q], s[Q], u[Q], kr[Q];
    const auto unit_of = [&](int32_t r) { return h.x_exp ? h.x_exp[min(r, n_rows - 1)] + *h.w_exp - 30 : 0; };
#pragma unroll
    for (int j = 0; j < Q; ++j) {
        const int32_t r = my_row + j;
        token[j] = -1;
        if (h.token && r < n_rows) token[j] = h.token[h.list ? h.list[r] : r];
        m[j] = -INFINITY;
        kr[j] = ldexpf(h.k, unit_of(r));
        s[j] = u[j] = 0.0f;
    }
    Product<T, Q> product;
    product.parts = h.parts;
    product.steps = h.steps;
    int32_t asked = at.second;                   // the tile whose numbers are on their way
    const auto next = [&] {
        if (asked + segments < h.tiles) place_tile(product.a, h.w, (asked += segments) * SIDE, h.vocab_end - h.v0);
    };
    if (asked < h.tiles) {                       // (the last piece of a vocabulary may have fewer tiles than there are segments)
        place_tile(product.a, h.w, asked * SIDE, h.vocab_end - h.v0);
        place_tile(product.b, h.x, first, n_rows);
        product.begin(lds, next);
    }
    for (int32_t t = at.second; t < h.tiles; t += segments) {
        f32x4 acc[Q][Q];
        product.tile(acc, next);
        const int32_t v = h.v0 + t * SIDE + place_a<Q>();       // of acc[0][.][0]
        const bool whole = h.v0 + (t + 1) * SIDE <= h.vocab_end;
#pragma unroll
        for (int j = 0; j < Q; ++j) {             // a row at a time
            float x[Q][4];
#pragma unroll
            for (int i = 0; i < Q; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i][e] = sum_of(acc[i][j][e]);
            const uint32_t off = (uint32_t)(token[j] - v);
            if (off < SIDE / 2 && off % 32 < 8) {
                float own = 0.0f;
#pragma unroll
                for (int i = 0; i < Q; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) own = off == (uint32_t)along_a(i, e) ? x[i][e] : own;
                h.x_token[my_row + j] = ldexpf(own, unit_of(my_row + j));
            }
            if (!whole)
#pragma unroll
                for (int i = 0; i < Q; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][e] = v + along_a(i, e) < h.vocab_end ? x[i][e] : -INFINITY;
            float most = m[j];
#pragma unroll
            for (int i = 0; i < Q; ++i)
#pragma unroll
                for (int e = 0; e < 4; e += 2) most = fmaxf(fmaxf(x[i][e], x[i][e + 1]), most);
            const float base = most > -INFINITY ? most : 0.0f, base2 = base * kr[j];
            const bool far = fabsf(base2) >= LOGIT_FAR;
            const float d0 = fmaxf(less_reference(m[j], kr[j], base, base2, far), -1e4f), f = __builtin_amdgcn_exp2f(d0);
            if constexpr (ENTROPY) u[j] = f * (u[j] + d0 * s[j]);
            s[j] *= f;
            m[j] = most;
            const auto take_in = [&](auto plain) {
                constexpr bool PLAIN = decltype(plain)::value;
#pragma unroll
                for (int i = 0; i < Q; ++i) {
                    float d[4], p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[e] = !PLAIN && far ? (x[i][e] - base) * kr[j] : fmaf(x[i][e], kr[j], -base2);
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(d[e]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[j] += p[e];
                        // (outside the vocabulary 0 is added, not a NaN)
                        if constexpr (ENTROPY) u[j] = fmaf(p[e], PLAIN ? d[e] : fmaxf(d[e], -1e4f), u[j]);
                    }
                }
            };
            if (whole && !__any(far)) take_in(std::true_type{}); else take_in(std::false_type{});
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // the four lanes and the two waves that share a row
    // (from here on relative to the largest logit itself)
#pragma unroll
    for (int j = 0; j < Q; ++j) {
        const float base = m[j] > -INFINITY ? m[j] : 0.0f, base2 = base * kr[j];
        const float d = fabsf(base2) >= LOGIT_FAR ? 0.0f : fmaf(-base, kr[j], base2), f = __builtin_amdgcn_exp2f(d);
        u[j] = f * (u[j] + d * s[j]);
        s[j] *= f;
        m[j] = ldexpf(m[j], unit_of(my_row + j));
    }
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
    product.end();
#pragma unroll
    for (int j = 0; j < Q; ++j) {
        RowSums r = {m[j], s[j], u[j]};
#pragma unroll
        for (int d = 16; d < 64; d <<= 1) r = join(r, RowSums{__shfl_xor(r.m, d), __shfl_xor(r.s, d), __shfl_xor(r.u, d)});
        if (lane < 16) tmp[wave * (SIDE / 2) + Q * lane + j] = r;
    }
    __syncthreads();
    for (int32_t i = threadIdx.x; i < SIDE && first + i < n_rows; i += P_THREADS) {
        const int32_t row = first + i;
        RowSums r = join(tmp[i], tmp[SIDE + i]);
        RowSums* to = h.sums + (int64_t)row * segments + at.second;
        if (h.add) r = join(*to, r);
        *to = r;
    }
}

// A row's logits in 32 bits, for rows whose alternatives are wanted.
template <typename T, int Q>
__global__ __launch_bounds__(P_THREADS, Q == 8 ? 1 : 2) void head_logits_kernel(const HeadStatArgs h, float* logits, int64_t pitch) {
    constexpr int SIDE = P_SIDE<Q>;
    __shared__ __attribute__((aligned(1024))) char lds[P_LDS<Q>];
    const TilePair at = tile_pair(by_chiplet(blockIdx.x, h.row_tiles * h.tiles), h.row_tiles, h.tiles);
    const int32_t first = at.first * SIDE, t = at.second;
    TileOfA<Q> a;
    TileOfB<Q> b;
    place_tile(a, h.w, t * SIDE, h.vocab_end - h.v0);
    place_tile(b, h.x, first, h.n_rows);
    f32x4 acc[Q][Q];
    product<T, Q>(acc, a, b, h.parts, h.steps, lds);
    const int32_t v = h.v0 + t * SIDE + place_a<Q>(), row = first + place_b<Q>();
#pragma unroll
    for (int j = 0; j < Q; ++j)
        if (row + j < h.n_rows) {
            const int unit = h.x_exp ? h.x_exp[row + j] + *h.w_exp - 30 : 0;
#pragma unroll
            for (int i = 0; i < Q; ++i)
                if (v + along_a(i, 0) < h.vocab_end)         // (the pitch is a multiple of 4)
                    {
                    f32x4 x = acc[i][j];
                    if (h.x_exp)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = ldexpf(x[e], unit);
                    *reinterpret_cast<f32x4*>(logits + (row + j) * pitch + v + along_a(i, 0)) = x;
                }
        }
}

// ---- few rows: bound by reading the weights ----

struct FewArgs {
    const void*  w;
    int64_t      w_stride;
    int32_t      vocab, dim;
    const char*  x;
    int64_t      x_pitch, x_plane;
    int32_t      n_rows;
    float*       logits;
    int64_t      pitch;
};
template <typename W> struct FewTypes { using T = W; static constexpr int PLANES = 1; };
template <> struct FewTypes<float> { using T = __bf16; static constexpr int PLANES = 3; };

// Eight numbers as one of 16 bits each, or as three of bf16.
template <typename W> union Eight { u32x4 q[sizeof(W) / 2]; W e[8]; };
template <typename W>
__device__ __forceinline__ void take_apart(const Eight<W>& from, Raw8<typename FewTypes<W>::T> (&part)[FewTypes<W>::PLANES]) {
    if constexpr (sizeof(W) == 2) {
        part[0].q[0] = from.q[0];
    } else {
        // the upper 16 bits of a number, of what they leave, and of what those leave: 24 bits, cut and not rounded, so exactly all of it
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float x = from.e[e], y = from.e[e + 1];
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                part[p].q[0][e / 2] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
                x -= __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
                y -= __uint_as_float(__float_as_uint(y) & 0xFFFF0000u);
            }
        }
    }
}
// sum += a b, all parts
template <typename W>
__device__ __forceinline__ void multiply_parts(const Raw8<typename FewTypes<W>::T> (&a)[FewTypes<W>::PLANES],
                                               const Raw8<typename FewTypes<W>::T> (&b)[FewTypes<W>::PLANES], f32x4& sum) {
    using M = Mfma<typename FewTypes<W>::T>;
    using Frag = typename M::Frag;
    const auto one = [&](int i, int j) { sum = M::sum(__builtin_bit_cast(Frag, a[i].q[0]), __builtin_bit_cast(Frag, b[j].q[0]), sum); };
    if constexpr (sizeof(W) == 4) { one(0, 2); one(2, 0); one(1, 1); one(0, 1); one(1, 0); }
    one(0, 0);
}

// A workgroup goes through its share of the vocabulary, TILE entries at a time: BYTES of each, and of every row, at a time come into the
// LDS, STAGES - 1 of them ahead and on into the next tile, so that memory never waits.  A wave has a quarter of the entries and all
// rows.  Numbers of 32 bits lie in the LDS as they are and are taken apart on the way to the matrix cores.
// 152064 x 2048 bf16 (622 MB), us, one row: 512 bytes of 64 entries and one workgroup to a compute unit 99 (6.3 TB/s), 256 of 64 and two
// 106, 128 of 128 and two 120; without the loads' hint not to keep the weights 119 instead of 106.  64 rows, which come out of the L2
// once per stage: 128 bytes of 128 entries and two workgroups 151, 256 bytes of 64 entries 159; a wave of its own that asks 170.  f32
// (1.25 GB), the whole call: 4 rows 250 (5.0 TB/s), 32 rows 343, 64 rows 386.
template <typename W, int NB, int BYTES, int W_STAGE, int GROUPS>
__global__ __launch_bounds__(256) void head_few_kernel(const FewArgs f) {
    constexpr int TILE = W_STAGE / BYTES, MT = TILE / 64, LANES = BYTES / 16, AT_ONCE = 256 / LANES;     // rows of BYTES that a load of all threads fills
    constexpr int ROWS = NB * 16 < AT_ONCE ? AT_ONCE : NB * 16, STAGE = (TILE + ROWS) * BYTES, LOADS = (TILE + ROWS) / AT_ONCE;
    constexpr int STAGES = 163840 / (GROUPS / 256) / STAGE;      // GROUPS / 256 workgroups fill a compute unit's LDS
    constexpr int STEP = BYTES / sizeof(W), HALVES = STEP / 32;
    static_assert(STAGES >= 2 && (STAGES - 2) * LOADS < 64 && TILE % 64 == 0, "what a wave can wait for");
    __shared__ __attribute__((aligned(1024))) char lds[STAGES * STAGE];
    const int lane = lane_id(), tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
    // a share in whole 16 entries
    const int32_t units = (f.vocab + 15) / 16;
    const int32_t first = (int32_t)((int64_t)units * blockIdx.x / gridDim.x) * 16;
    const int32_t end = min((int32_t)((int64_t)units * (blockIdx.x + 1) / gridDim.x) * 16, f.vocab);
    const int32_t tiles = (end - first + TILE - 1) / TILE, steps = f.dim / STEP;
    if (tiles <= 0) return;
    const int place = tid / LANES, piece = tid % LANES ^ (place & 7);
    static_assert(AT_ONCE % 8 == 0, "a thread's pieces are the same in all its rows");
    const char* const w0 = static_cast<const char*>(f.w) + first * f.w_stride * (int64_t)sizeof(W);
    int64_t w_at[TILE / AT_ONCE], x_at[ROWS / AT_ONCE];
    int32_t asked_tile = 0, asked_step = 0, to = 0;
    const auto place_entries = [&](int32_t tile) {
#pragma unroll
        for (int j = 0; j < TILE / AT_ONCE; ++j)
            w_at[j] = min(tile * TILE + place + AT_ONCE * j, end - first - 1) * f.w_stride * (int64_t)sizeof(W) + 16 * piece;
    };
    place_entries(0);
#pragma unroll
    for (int j = 0; j < ROWS / AT_ONCE; ++j) x_at[j] = min(place + AT_ONCE * j, f.n_rows - 1) * f.x_pitch + 16 * piece;
    const auto ask = [&] {
        char* s = lds + to * STAGE + wave * 1024;
#pragma unroll
        for (int j = 0; j < TILE / AT_ONCE; ++j) load_to_lds<true>(w0 + w_at[j] + asked_step * BYTES, s + j * 4096);
#pragma unroll
        for (int j = 0; j < ROWS / AT_ONCE; ++j) load_to_lds(f.x + x_at[j] + asked_step * BYTES, s + TILE * BYTES + j * 4096);
        to = to + 1 == STAGES ? 0 : to + 1;
        if (++asked_step == steps) {             // (behind the last tile: that one again, for nobody)
            asked_step = 0;
            if (asked_tile + 1 < tiles) place_entries(++asked_tile);
        }
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) ask();
    const int row = lane & 15;
    const auto read = [&](const char* rows, int first_piece, Eight<W>& e) {          // neighbouring pieces of a row
#pragma unroll
        for (int q = 0; q < (int)sizeof(W) / 2; ++q)
            e.q[q] = *reinterpret_cast<const u32x4*>(rows + row * BYTES + ((first_piece + q) ^ (row & 7)) * 16);
    };
    int32_t now = 0;
    for (int32_t tile = 0; tile < tiles; ++tile) {
        f32x4 acc[MT][NB] = {};
        for (int32_t k = 0; k < steps; ++k) {
            wait_loads<(STAGES - 2) * LOADS>();
            bare_barrier();
            ask();
            const char* stage = lds + now * STAGE;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const int at = h * (int)(2 * sizeof(W)) + (lane >> 4) * (int)(sizeof(W) / 2);
                Raw8<typename FewTypes<W>::T> a[MT][FewTypes<W>::PLANES], b[NB][FewTypes<W>::PLANES];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    Eight<W> e;
                    read(stage + (wave * 16 * MT + 16 * i) * BYTES, at, e);
                    take_apart<W>(e, a[i]);
                }
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    Eight<W> e;
                    read(stage + (TILE + 16 * j) * BYTES, at, e);
                    take_apart<W>(e, b[j]);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NB; ++j) multiply_parts<W>(a[i], b[j], acc[i][j]);
            }
            now = now + 1 == STAGES ? 0 : now + 1;
        }
        const int32_t v = first + tile * TILE + wave * 16 * MT + (lane >> 4) * 4;
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (16 * j + row < f.n_rows)
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    if (v + 16 * i < end)        // (the pitch is a multiple of 4)
                        *reinterpret_cast<f32x4*>(f.logits + (16 * j + row) * f.pitch + v + 16 * i) = acc[i][j];
    }
    wait_loads<0>();
}

// The same for weights and rows that lie anyhow: a wave per 16 MT entries and 16 NB rows, the weights straight into the places that the
// matrix cores want, AHEAD steps of 32 elements before they are multiplied; the rows, laid out with k_pad columns, 0 behind the last
// one, come out of the L2.  Bound by its loads, 16 bytes a lane across the lines' borders: 152064 x 2048 bf16 in rows of 2049, us, one row
// 307 (2.0 TB/s), 64 rows 420; f32 304 (4.1 TB/s); 32003 x 515 bf16 23 and 31.
template <typename W, int MT, int NB, int AHEAD>
__global__ __launch_bounds__(256) void head_few_any_kernel(const FewArgs f) {
    using T = typename FewTypes<W>::T;
    constexpr int PLANES = FewTypes<W>::PLANES;
    using Piece = std::conditional_t<sizeof(W) == 4, u32x4_a4, u32x4_a2>;
    const int lane = lane_id();
    const int32_t v0 = (blockIdx.x * 4 + threadIdx.x / WAVE) * 16 * MT;
    if (v0 >= f.vocab) return;
    const W* w[MT];
    const char* x[NB];
#pragma unroll
    for (int i = 0; i < MT; ++i) w[i] = static_cast<const W*>(f.w) + min(v0 + 16 * i + (lane & 15), f.vocab - 1) * f.w_stride + (lane >> 4) * 8;
#pragma unroll
    for (int j = 0; j < NB; ++j) x[j] = f.x + min(16 * j + (lane & 15), f.n_rows - 1) * f.x_pitch + (lane >> 4) * 16;
    f32x4 acc[MT][NB] = {};
    struct Steps { Eight<W> a[AHEAD][MT]; Raw8<T> b[AHEAD][NB][PLANES]; } first, second;
    const int32_t steps = f.dim / 32;
    const auto ask = [&](Steps& s, int32_t k) {              // (behind the last step: that one again)
#pragma unroll
        for (int h = 0; h < AHEAD; ++h) {
            const int32_t at = min(k + h, steps - 1) * 32;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int q = 0; q < (int)sizeof(W) / 2; ++q)
                    s.a[h][i].q[q] = *(reinterpret_cast<const Piece*>(w[i] + at) + q);
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
#pragma unroll
                for (int j = 0; j < NB; ++j) s.b[h][j][p].q[0] = *reinterpret_cast<const u32x4*>(x[j] + p * f.x_plane + at * 2);
        }
    };
    const auto multiply = [&](const Eight<W> (&a)[MT], const Raw8<T> (&b)[NB][PLANES]) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            Raw8<T> part[PLANES];
            take_apart<W>(a[i], part);
#pragma unroll
            for (int j = 0; j < NB; ++j) multiply_parts<W>(part, b[j], acc[i][j]);
        }
    };
    const auto multiply_all = [&](const Steps& s, int32_t k) {
#pragma unroll
        for (int h = 0; h < AHEAD; ++h)
            if (k + h < steps) multiply(s.a[h], s.b[h]);
    };
    if (steps > 0) ask(first, 0);
    for (int32_t k = 0; k < steps; k += 2 * AHEAD) {
        ask(second, k + AHEAD);
        multiply_all(first, k);
        if (k + AHEAD >= steps) break;
        ask(first, k + 2 * AHEAD);
        multiply_all(second, k + AHEAD);
    }
    if (steps * 32 < f.dim) {                    // what is left, an element at a time
        Eight<W> a[MT];
        Raw8<T> b[NB][PLANES];
        const int32_t left = f.dim - steps * 32 - (lane >> 4) * 8;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) a[i].e[e] = e < left ? w[i][steps * 32 + e] : (W)0.0f;
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
#pragma unroll
            for (int j = 0; j < NB; ++j) b[j][p].q[0] = *reinterpret_cast<const u32x4*>(x[j] + p * f.x_plane + steps * 64);
        multiply(a, b);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j)
        if (16 * j + (lane & 15) < f.n_rows)
#pragma unroll
            for (int i = 0; i < MT; ++i)
                if (v0 + 16 * i + (lane >> 4) * 4 < f.vocab)         // (the pitch is a multiple of 4)
                    *reinterpret_cast<f32x4*>(f.logits + (16 * j + (lane & 15)) * f.pitch + v0 + 16 * i + (lane >> 4) * 4) = acc[i][j];
}

constexpr int64_t FEW_ROWS = 64;
// Rows that are read 128 bytes at a time.
static bool in_whole_steps(const dc_matrix& m) {
    const int64_t each = m.type == DC_F32 ? 4 : 2;
    return reinterpret_cast<uintptr_t>(m.d_data) % 16 == 0 && m.row_stride * each % 16 == 0 && m.n_cols * each % 128 == 0;
}
template <int BYTES, int STAGE, int GROUPS, typename F>
static void launch_with(F&& f) {
    f(std::integral_constant<int, BYTES>{}, std::integral_constant<int, STAGE>{}, std::integral_constant<int, GROUPS>{});
}
static hipError_t launch_few(const FewArgs& f, int32_t type, bool any, hipStream_t st) {
    return with_type(type, [&](auto el) {
        using W = typename decltype(el)::type;
        using std::integral_constant;
        constexpr bool F32 = std::is_same_v<W, float>;
        const auto go = [&](auto mt, auto nb, auto ahead) {
            constexpr int MT = decltype(mt)::value, NB = decltype(nb)::value, AHEAD = decltype(ahead)::value;
            if (any) head_few_any_kernel<W, MT, NB, AHEAD><<<(unsigned)((f.vocab + 64 * MT - 1) / (64 * MT)), 256, 0, st>>>(f);
            else {
                const auto launch = [&](auto bytes, auto stage, auto groups) {
                    constexpr int GROUPS = decltype(groups)::value;
                    head_few_kernel<W, NB, decltype(bytes)::value, decltype(stage)::value, GROUPS><<<(unsigned)std::min((f.vocab + 15) / 16, GROUPS), 256, 0, st>>>(f);
                };
                if constexpr (NB < 4)
                    if (f.dim * sizeof(W) % 512 == 0) {
                        launch_with<512, 32768, 256>(launch);
                        return;
                    }
                launch_with<128, 16384, 512>(launch);
            }
        };
        if (f.n_rows <= 16) go(integral_constant<int, 1>{}, integral_constant<int, 1>{}, integral_constant<int, F32 ? 2 : 8>{});
        else if (f.n_rows <= 32) go(integral_constant<int, F32 ? 1 : 2>{}, integral_constant<int, 2>{}, integral_constant<int, 2>{});
        else go(integral_constant<int, 2>{}, integral_constant<int, 4>{}, integral_constant<int, F32 ? 1 : 2>{});
        return hipGetLastError();
    });
}

// A wave per row: its segments' sums as one, and the results.
__global__ __launch_bounds__(256) void head_join_kernel(const LogprobArgs a, const int32_t* pos, const int32_t* count, int32_t side, int32_t blocks,
                                                        int32_t most_tiles, const RowSums* sums, const float* x_token) {
    const int32_t segments = live_share(blocks, (int32_t)(((count ? *count : a.n_rows) + side - 1) / side), most_tiles);
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
        if (!(fabsf(all.u) < INFINITY)) all.s = NAN;         // (an infinite logit)
        if (lane == 0) {
            const int32_t token = a.token ? a.token[r] : 0;
            const bool in = token >= 0 && token < a.vocab;
            if (!in) set_status(a.status, DC_ERR_TOKEN_RANGE);
            write_row(a, r, finish(all, a.inv_t), in, in && a.token ? x_token[at] : 0.0f);
        }
    }
}

// How the vocabulary is shared out over workgroups: `segments` to each tile of rows, as many as make the fewest tiles one after another
// for `slots` workgroups at once.
constexpr int32_t HEAD_MOST_BLOCKS = 2048;
static int32_t segments_of(int64_t row_tiles, int32_t tiles, int32_t slots) {
    int32_t best = 1;
    int64_t least = -1;
    for (int32_t s = 1; s <= tiles && row_tiles * s <= HEAD_MOST_BLOCKS; ++s) {
        const int64_t rounds = (row_tiles * s + slots - 1) / slots * ((tiles + s - 1) / s);
        if (least < 0 || rounds < least) { least = rounds; best = s; }
    }
    return best;
}

constexpr int64_t HEAD_TOP_ROWS = 256;           // rows whose logits are held at once, where alternatives are wanted
constexpr int64_t HEAD_PIECE_BYTES = 256LL << 20;    // of weights laid out at once
static int32_t weight_piece(const HeadShape& sh, const dc_matrix& w) {
    if (!sh.copy_weight) return (int32_t)w.n_rows;
    const int64_t row = sh.k_pad * 2LL * (w.type == DC_F32 ? 2 : 1);
    return (int32_t)std::min<int64_t>(whole(w.n_rows, P_MOST_SIDE), std::max<int64_t>(P_MOST_SIDE, HEAD_PIECE_BYTES / row / P_MOST_SIDE * P_MOST_SIDE));
}

namespace {
struct HeadWs {
    char*    hidden; int64_t hidden_plane;
    char*    weight; int64_t weight_plane; int32_t piece;
    int32_t *x_exp, *w_exp;         // w_exp: one to a piece
    LiveRows live;
    float*   x_token;
    RowSums* sums;
    float*   logits; int64_t pitch;
    char*    logprob;
    size_t   bytes;
};
}
// Up to FEW_ROWS rows, and HEAD_TOP_ROWS at a time with alternatives, go through their logits, others straight to sums.
static HeadWs carve(void* base, const dc_matrix& hidden, const dc_matrix& weight, int32_t n_top) {
    HeadWs w = {};
    const HeadShape sh = head_shape(hidden, weight, true);
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char* p = static_cast<char*>(base) + at;
        at += align256(bytes);
        return p;
    };
    const int64_t rows = hidden.n_rows, planes = hidden.type == DC_F32 ? 2 : 1;
    const bool few = rows <= FEW_ROWS;
    w.hidden_plane = rows * sh.k_pad * 2;
    w.hidden = take(sh.copy_hidden || few ? (few && planes == 2 ? 3 : planes) * w.hidden_plane : 0);
    w.piece = weight_piece(sh, weight);
    w.weight_plane = (int64_t)w.piece * sh.k_pad * 2;
    w.weight = take(sh.copy_weight && !few ? planes * w.weight_plane : 0);
    w.x_exp = reinterpret_cast<int32_t*>(take(planes == 2 ? rows * 4 : 0));
    w.w_exp = reinterpret_cast<int32_t*>(take(planes == 2 && !few ? whole(weight.n_rows, w.piece) / w.piece * 4 : 0));
    w.pitch = whole(weight.n_rows, 4);
    if (few || n_top > 0) {
        w.logits = reinterpret_cast<float*>(take(std::min(rows, HEAD_TOP_ROWS) * w.pitch * 4));
        w.logprob = take((int64_t)logprob_workspace_bytes(std::min(rows, HEAD_TOP_ROWS), (int32_t)weight.n_rows, DC_F32, n_top));
    } else {
        w.live.list = reinterpret_cast<int32_t*>(take(rows * 4));
        w.live.pos = reinterpret_cast<int32_t*>(take(rows * 4));
        w.live.count = reinterpret_cast<int32_t*>(take(4));
        w.x_token = reinterpret_cast<float*>(take(rows * 4));
        // (as many segments as any number of tiles of rows up to this one's has: blocks never pass their limit, nor tiles of both)
        int64_t sums = 0;
        for (const int64_t side : {P_SIDE<4>, P_SIDE<8>}) {
            const int64_t row_tiles = whole(rows, side) / side, tiles = whole(weight.n_rows, side) / side;
            sums = std::max(sums, side * std::max<int64_t>(row_tiles, std::min<int64_t>(HEAD_MOST_BLOCKS, row_tiles * tiles)));
        }
        w.sums = reinterpret_cast<RowSums*>(take(sums * (int64_t)sizeof(RowSums)));
    }
    w.bytes = (size_t)at;
    return w;
}
size_t head_workspace_need(const dc_matrix& hidden, const dc_matrix& weight, int32_t n_top) {
    return hidden.n_rows > 0 ? carve(nullptr, hidden, weight, n_top).bytes : 0;
}
size_t head_workspace_bytes(const dc_matrix& hidden, const dc_matrix& weight, int32_t n_top) {
    dc_matrix fewer = hidden;
    fewer.n_rows = std::min(hidden.n_rows, FEW_ROWS);
    return std::max(std::max(head_workspace_need(hidden, weight, 0), head_workspace_need(hidden, weight, n_top)),
                    std::max(head_workspace_need(fewer, weight, 0), head_workspace_need(fewer, weight, n_top)));
}

hipError_t launch_head(const HeadArgs& a, void* d_ws, hipStream_t st) {
    const int64_t rows = a.hidden.n_rows;
    if (rows == 0) return hipSuccess;
    const int32_t vocab = (int32_t)a.weight.n_rows, type = a.hidden.type;
    const HeadWs w = carve(d_ws, a.hidden, a.weight, a.n_top);
    const HeadShape sh = head_shape(a.hidden, a.weight, true);
    hipError_t e = hipSuccess;
    LogprobArgs out = {nullptr, w.pitch, rows, vocab, a.n_top, a.inv_t, a.token, a.mask, a.logprob, a.stat, a.entropy,
                       a.top_token, a.top_logprob, a.status};
    if (rows <= FEW_ROWS) {
        const bool any = !in_whole_steps(a.hidden) || !in_whole_steps(a.weight);
        FewArgs f = {a.weight.d_data, a.weight.row_stride, vocab, (int32_t)a.hidden.n_cols, static_cast<const char*>(a.hidden.d_data),
                     a.hidden.row_stride * (type == DC_F32 ? 4 : 2), 0, (int32_t)rows, w.logits, w.pitch};
        if (any) {
            e = launch_lay_rows(a.hidden, 0, rows, nullptr, nullptr, sh.k_pad, w.hidden, w.hidden_plane, BF16S, nullptr, nullptr, st);
            f.x = w.hidden;
            f.x_pitch = sh.k_pad * 2;
            f.x_plane = w.hidden_plane;
        }
        if (e == hipSuccess) e = launch_few(f, type, any, st);
        out.x = w.logits;
        return e == hipSuccess ? launch_logprob(out, DC_F32, w.logprob, st) : e;
    }
    const bool live = a.n_top == 0 && a.mask;
    const bool f32 = type == DC_F32;
    const FirstExponents none = {w.w_exp, f32 ? (vocab + w.piece - 1) / w.piece : 0, false};
    if (live) e = launch_live_rows(a.mask, nullptr, nullptr, rows, w.live, none, st);
    else if (f32) e = launch_first_exponents(none, st);
    HeadStatArgs h = {};
    h.x_exp = f32 ? w.x_exp : nullptr;
    h.steps = sh.k_pad / PK;
    h.parts = parts_of(type, w.weight_plane, w.hidden_plane);
    h.k = a.inv_t * LOG2E;
    h.token = a.token;
    h.sums = w.sums;
    h.x_token = w.x_token;
    const bool small = cut_product(a.n_top > 0 ? std::min(rows, HEAD_TOP_ROWS) : rows, std::min(w.piece, vocab), h.steps * h.parts.n, 1).small;
    const int32_t side = small ? P_SIDE<4> : P_SIDE<8>;
    h.row_tiles = (int32_t)((rows + side - 1) / side);
    h.n_rows = (int32_t)rows;
    h.count = live ? w.live.count : nullptr;
    h.list = live ? w.live.list : nullptr;
    h.most_tiles = (std::min(w.piece, vocab) + side - 1) / side;
    h.segments = segments_of(h.row_tiles, h.most_tiles, small ? P_SLOTS<4> : P_SLOTS<8>);
    if (sh.copy_hidden) {
        if (e == hipSuccess && f32) e = launch_row_exponents(a.hidden, rows, h.list, h.count, w.x_exp, st);
        if (e == hipSuccess) e = launch_lay_rows(a.hidden, 0, rows, h.list, h.count, sh.k_pad, w.hidden, w.hidden_plane, F16S, w.x_exp, nullptr, st);
        h.x = Operand{w.hidden, sh.k_pad * 2, nullptr};
    } else {
        h.x = Operand{static_cast<const char*>(a.hidden.d_data), a.hidden.row_stride * 2, h.list};
    }
    for (int64_t r0 = 0; r0 < rows && e == hipSuccess; r0 += HEAD_TOP_ROWS) {
        // so many rows at a time (copied weights are copied for each: 4096 x 32003 x 515 f32 1295 us, without alternatives 427)
        if (a.n_top > 0) {
            h.n_rows = (int32_t)std::min(HEAD_TOP_ROWS, rows - r0);
            h.row_tiles = (h.n_rows + side - 1) / side;
        }
        for (int32_t v0 = 0; v0 < vocab && e == hipSuccess; v0 += w.piece) {
            const int32_t n = std::min(w.piece, vocab - v0);
            if (sh.copy_weight) {
                h.w_exp = w.w_exp + v0 / w.piece;
                if (f32 && r0 == 0) e = launch_top_exponent(a.weight, v0, n, w.w_exp + v0 / w.piece, st);
                if (e == hipSuccess)
                    e = launch_lay_rows(a.weight, v0, n, nullptr, nullptr, sh.k_pad, w.weight, w.weight_plane, F16S, nullptr, h.w_exp, st);
                h.w = Operand{w.weight, sh.k_pad * 2, nullptr};
            } else {
                h.w = Operand{static_cast<const char*>(a.weight.d_data), a.weight.row_stride * 2, nullptr};
            }
            if (e != hipSuccess) break;
            h.v0 = v0;
            h.vocab_end = v0 + n;
            h.tiles = (n + side - 1) / side;
            h.add = v0 > 0;
            const auto go = [&](auto t, auto q) {
                using T = decltype(t);
                constexpr int Q = decltype(q)::value;
                if (a.n_top > 0) head_logits_kernel<T, Q><<<h.row_tiles * h.tiles, P_THREADS, 0, st>>>(h, w.logits, w.pitch);
                else if (a.entropy) head_stat_kernel<T, true, Q><<<h.row_tiles * h.segments, P_THREADS, 0, st>>>(h);
                else head_stat_kernel<T, false, Q><<<h.row_tiles * h.segments, P_THREADS, 0, st>>>(h);
            };
            const auto with_q = [&](auto t) {
                if (small) go(t, std::integral_constant<int, 4>{}); else go(t, std::integral_constant<int, 8>{});
            };
            if (type == DC_BF16) with_q(__bf16{}); else with_q(_Float16{});
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
        if (f32) h.x_exp += HEAD_TOP_ROWS;
    }
    if (e != hipSuccess || a.n_top > 0) return e;
    head_join_kernel<<<(unsigned)std::min<int64_t>((rows + 3) / 4, 1 << 16), 256, 0, st>>>(
        out, live ? w.live.pos : nullptr, h.count, side, h.row_tiles * h.segments, h.most_tiles, w.sums, w.x_token);
    return hipGetLastError();
}

}  // namespace dc
