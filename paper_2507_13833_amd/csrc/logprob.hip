// Log-probabilities of given tokens with entropy and top alternatives, and the gradient of the logits.
//
// One pass over a row, every thread on its own: with k = log2(e) / T a thread keeps M2 = k * (its largest logit), rounded,
// s = sum 2^(k x - M2) and u = sum 2^(k x - M2) (k x - M2); both are scaled when M2 grows.  k x - M2 is one fused
// multiply-add, so M2's rounding is no error: whatever M2 is, it is taken off exactly at the end.
// The n_top largest: a thread also keeps where the 16 bytes with its largest logit begin.  An
// element below the n_top-th greatest of these (logit, place) has no place among the n_top largest.  The threads whose own
// is not below a bound on it read their logits once more (out of the caches); what is not below it is ranked by counting.
// A workgroup takes a row; few rows get larger workgroups, and long ones are cut into parts that a second launch joins.
// Bound by reading the logits where there are many rows (8192 x 152064 bf16, 2.5 GB: 0.37 ms, 6.7 TB/s), by two launches' trips to
// memory where there are few (1 x 152064: 7.5 + 4.6 us).
#include <algorithm>
#include "logprob_device.h"

namespace dc {

constexpr int LP_THREADS = 256, LP_WIDE = 1024;  // of a workgroup: where there are many rows, where there are few
constexpr int LP_AT_ONCE = 4;                    // 16-byte loads asked for at once
constexpr int LP_CANDIDATES = 1024;              // of the largest that are ranked in the LDS; more: one by one
// |k M| from here on: the sums are made again with differences taken first.  Below it M2's rounding is at most 1/2, so the
// exponents k x - M2 stay as small as the true ones; at 2^31 it would be 128, which no float has the power of.
constexpr float LP_FAR = 0x1p24f;

template <typename T> constexpr int CHUNK_ELEMS = 16 / sizeof(T);

// 16 bytes of logits as floats.
template <typename T>
__device__ __forceinline__ void unpack(u32x4 q, float (&f)[CHUNK_ELEMS<T>]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(q[i]);
    } else if constexpr (std::is_same_v<T, __bf16>) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(q[i] << 16);
            f[2 * i + 1] = __uint_as_float(q[i] & 0xFFFF0000u);
        }
    } else {
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        const h8 h = __builtin_bit_cast(h8, q);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)h[i];
    }
}

// A logit and its place as one number: greater for a larger logit, and among equal ones for the lower place.
__device__ __forceinline__ uint64_t top_key(float x, int32_t place) { return (uint64_t)sortable(x) << 32 | (uint32_t)~place; }

template <int THREADS>
struct TopLds {
    static constexpr int WAVES = THREADS / WAVE;
    uint64_t candidate[LP_CANDIDATES];
    uint64_t tmp[WAVES];
    int32_t  chosen[THREADS];
    uint32_t n_candidates, n_chosen;
};

// The largest v of `bits` bits that n lanes' numbers are no smaller than; `in`: the lanes that count.  0 where there are fewer.
__device__ __forceinline__ uint32_t wave_nth(uint32_t number, uint64_t in, int bits, int n) {
    uint32_t v = 0;
    for (int b = bits - 1; b >= 0; --b) {
        const uint32_t t = v | 1u << b;
        if (__popcll(__ballot(number >= t) & in) >= n) v = t;
    }
    return v;
}
// The n-th greatest of a wave's keys, 0 where there are fewer (0 is no key; all others differ).  The place counts among
// equal logits alone.  BITS: of a logit as a sortable number that tell logits of its type apart.
template <typename T> constexpr int SORT_BITS = std::is_same_v<T, __bf16> ? 16 : std::is_same_v<T, _Float16> ? 20 : 32;
template <int BITS>
__device__ __forceinline__ uint64_t wave_nth_key(uint64_t key, int n) {
    const uint32_t value = (uint32_t)(key >> 32) >> (32 - BITS), place = (uint32_t)key;
    const uint32_t v = wave_nth(value, ~0ull, BITS, n);
    if (v == 0) return 0;
    const uint64_t same = __ballot(value == v);
    const int left = n - __popcll(__ballot(value > v));      // so many of those with this logit
    const uint64_t least = (uint64_t)v << (64 - BITS);
    if (__popcll(same) == left) return least;
    static_assert(DC_MAX_VOCAB <= 1 << 24, "the upper 8 bits of ~place are set");
    return least | 0xFF000000u | wave_nth(place & 0xFFFFFFu, same, 24, left);
}
// A key that n of the workgroup's keys are not below, near the n-th greatest: every wave's nth key has nth keys that are not
// below it, so many waves together have n.  Where too few waves have as many (a short row), one that has n by itself.  0 where
// there is none either.  Every thread gets it; the candidates and the chosen are none.
template <int BITS, int THREADS>
__device__ __forceinline__ uint64_t least_key(TopLds<THREADS>& t, uint64_t key, int n) {
    constexpr int WAVES = THREADS / WAVE;
    const int nth = min(n, (2 * n + WAVES - 1) / WAVES), of_waves = (n + nth - 1) / nth;
    const uint64_t mine = wave_nth_key<BITS>(key, nth);
    if (lane_id() == 0) t.tmp[threadIdx.x / WAVE] = mine;
    if (threadIdx.x == 0) { t.n_candidates = 0; t.n_chosen = 0; }
    __syncthreads();
    uint64_t least = wave_nth_key<BITS>(lane_id() < WAVES ? t.tmp[lane_id()] : 0ull, of_waves);
    if (least != 0) return least;
    __syncthreads();
    const uint64_t alone = wave_nth_key<BITS>(key, n);
    if (lane_id() == 0) t.tmp[threadIdx.x / WAVE] = alone;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) least = t.tmp[w] > least ? t.tmp[w] : least;
    return least;
}
template <int THREADS>
__device__ __forceinline__ void add_candidate(TopLds<THREADS>& t, uint64_t key) {
    const uint32_t at = atomicAdd(&t.n_candidates, 1u);
    if (at < LP_CANDIDATES) t.candidate[at] = key;
}
// The n_top greatest keys, in order, to put(i, key); all keys differ.  all(visit) hands every key there is to visit: used
// where there are more candidates than the LDS takes, once for every place in the list.
template <int THREADS, typename All, typename Put>
__device__ __forceinline__ void rank_candidates(TopLds<THREADS>& t, int n_top, All all, Put put) {
    __syncthreads();
    const int n = (int)t.n_candidates;
    if (n <= LP_CANDIDATES) {
        for (int i = threadIdx.x; i < n; i += THREADS) {
            const uint64_t key = t.candidate[i];
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < n; ++j) rank += t.candidate[j] > key ? 1 : 0;
            if (rank < n_top) put(rank, key);
        }
        for (int i = n + threadIdx.x; i < n_top; i += THREADS) put(i, 0ull);
    } else {
        uint64_t below = ~0ull;
        for (int i = 0; i < n_top; ++i) {
            uint64_t best = 0;
            all([&](uint64_t key) { if (key < below && key > best) best = key; });
            best = block_reduce(best, t.tmp, wave_max_u64, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
            if (threadIdx.x == 0) put(i, best);
            below = best;
        }
    }
    __syncthreads();                             // the LDS is free again
}

// What a part leaves for the join: its sums, then n_top keys, greatest first (0: the part has no more elements).
struct PartHead { RowSums sums; float pad; };
static __host__ __device__ size_t part_bytes(int n_top) { return sizeof(PartHead) + (size_t)n_top * sizeof(uint64_t); }

template <int THREADS, typename T, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(THREADS) void logprob_kernel(const LogprobArgs a, int32_t parts, int32_t per_part, char* ws) {
    constexpr int N = CHUNK_ELEMS<T>, WAVES = THREADS / WAVE;
    __shared__ float red[3][WAVES];
    __shared__ __attribute__((aligned(16))) char top_lds[TOP ? sizeof(TopLds<THREADS>) : 16];
    TopLds<THREADS>& top = *reinterpret_cast<TopLds<THREADS>*>(top_lds);
    const float k = a.inv_t * LOG2E;
    const int tid = threadIdx.x;
    for (int64_t unit = blockIdx.x; unit < a.n_rows * parts; unit += gridDim.x) {
        const int64_t r = unit / parts;
        const int32_t part = (int32_t)(unit - r * parts);
        if (a.mask && a.mask[r] == 0) {
            if (parts == 1) write_nothing(a, r);
            continue;
        }
        const T* row = static_cast<const T*>(a.x) + r * a.stride;
        // the given token's logit is asked for before everything else
        const int32_t token = parts == 1 && a.token ? a.token[r] : 0;
        const bool in = token >= 0 && token < a.vocab;
        const float x_token = parts == 1 && a.token ? (float)row[in ? token : 0] : 0.0f;

        const int32_t v0 = part * per_part, n = min(per_part, a.vocab - v0);
        const T* x = row + v0;
        // up to the first multiple of 16 bytes and behind the last one: an element to a thread
        const int32_t head = min(n, (int32_t)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int32_t)sizeof(T));
        const int32_t chunks = (n - head) / N, tail = n - head - chunks * N, tail_at = head + chunks * N;
        const u32x4* body = reinterpret_cast<const u32x4*>(x + head);

        float m = -INFINITY, m2 = -LP_FAR, s = 0.0f, u = 0.0f;
        int32_t at = -1;                         // TOP: where the 16 bytes with the first largest logit begin
        const auto scale_to = [&](float new_m) {
            m = new_m;
            const float new_m2 = fmaxf(m * k, -LP_FAR), d = m2 - new_m2, f = __builtin_amdgcn_exp2f(d);
            if constexpr (ENTROPY) u = f * (u + d * s);
            s *= f;
            m2 = new_m2;
        };
        const auto one = [&](float v, int32_t place) {
            if (TOP && (v > m || at < 0)) at = place;
            if (v > m) scale_to(v);
            const float d = fmaf(v, k, -m2), e = __builtin_amdgcn_exp2f(d);
            s += e;
            if constexpr (ENTROPY) u += e * fmaxf(d, -1e4f);               // (a logit of -infinity adds 0, not a NaN)
        };
        u32x4 next[LP_AT_ONCE];
        const auto ask = [&](int32_t c) {
#pragma unroll
            for (int j = 0; j < LP_AT_ONCE; ++j) {
                const u32x4* p = body + min(c + j * THREADS, chunks - 1);
                if constexpr (TOP) next[j] = *p;               // (the caches keep what may be read again)
                else next[j] = __builtin_nontemporal_load(p);
            }
        };
        if (tid < chunks) ask(tid);
        if (tid < head) one((float)x[tid], v0 + tid);
        for (int32_t c = tid; c < chunks; c += LP_AT_ONCE * THREADS) {
            float f[LP_AT_ONCE][N], most[LP_AT_ONCE];
#pragma unroll
            for (int j = 0; j < LP_AT_ONCE; ++j) {
                unpack<T>(next[j], f[j]);
                if (c + j * THREADS >= chunks)
#pragma unroll
                    for (int i = 0; i < N; ++i) f[j][i] = -INFINITY;
                most[j] = f[j][0];
#pragma unroll
                for (int i = 1; i < N; ++i) most[j] = fmaxf(most[j], f[j][i]);
            }
            if (c + LP_AT_ONCE * THREADS < chunks) ask(c + LP_AT_ONCE * THREADS);
            float all = most[0];
#pragma unroll
            for (int j = 1; j < LP_AT_ONCE; ++j) all = fmaxf(all, most[j]);
            if constexpr (TOP) {
                int32_t first = c;
#pragma unroll
                for (int j = LP_AT_ONCE - 1; j > 0; --j) first = most[j] == all ? c + j * THREADS : first;
                first = most[0] == all ? c : first;
                if (all > m || at < 0) at = v0 + head + first * N;
            }
            if (all > m) scale_to(all);
#pragma unroll
            for (int j = 0; j < LP_AT_ONCE; ++j) {
                float sj = 0.0f, uj = 0.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float d = fmaf(f[j][i], k, -m2), e = __builtin_amdgcn_exp2f(d);
                    sj += e;
                    if constexpr (ENTROPY) uj = fmaf(e, fmaxf(d, -1e4f), uj);
                }
                s += sj;
                if constexpr (ENTROPY) u += uj;
            }
        }
        if (tid < tail) one((float)x[tail_at + tid], v0 + tail_at + tid);

        // the workgroup's: sums relative to the largest logit itself
        RowSums sums;
        {
            const float wm = wave_max(m);
            if (lane_id() == 0) red[0][tid / WAVE] = wm;
            __syncthreads();
            sums.m = red[0][0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) sums.m = fmaxf(sums.m, red[0][i]);
            // (nothing above -infinity: sums of 0)
            const float d = sums.m > -INFINITY ? fmaxf(fmaf(-sums.m, k, m2), -1e4f) : 0.0f, f = __builtin_amdgcn_exp2f(d);
            float ws_ = wave_sum(f * s), wu = ENTROPY ? wave_sum(f * (u + d * s)) : 0.0f;
            if (fabsf(sums.m * k) >= LP_FAR && fabsf(sums.m) < INFINITY) {           // (the same in every thread)
                s = u = 0.0f;
                for (int32_t v = tid; v < n; v += THREADS) {
                    const float dv = ((float)x[v] - sums.m) * k, e = __builtin_amdgcn_exp2f(dv);
                    s += e;
                    if constexpr (ENTROPY) u += e * fmaxf(dv, -1e4f);
                }
                ws_ = wave_sum(s);
                wu = ENTROPY ? wave_sum(u) : 0.0f;
            }
            if (lane_id() == 0) { red[1][tid / WAVE] = ws_; red[2][tid / WAVE] = wu; }
            __syncthreads();
            sums.s = red[1][0];
            sums.u = red[2][0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) { sums.s += red[1][i]; sums.u += red[2][i]; }
        }
        const RowResult w = finish(sums, a.inv_t);
        char* mine = ws + unit * part_bytes(a.n_top);
        if (tid == 0) {
            if (parts == 1) {
                if (!in) set_status(a.status, DC_ERR_TOKEN_RANGE);
                write_row(a, r, w, in, x_token);
            } else {
                reinterpret_cast<PartHead*>(mine)->sums = sums;
            }
        }
        if constexpr (TOP) {
            const auto put = [&](int i, uint64_t key) {
                if (parts == 1) write_top(a, r, i, w, key);
                else reinterpret_cast<uint64_t*>(mine + sizeof(PartHead))[i] = key;
            };
            const uint64_t me = at < 0 ? 0ull : top_key(m, at), least = least_key<SORT_BITS<T>>(top, me, a.n_top);
            // (a NaN's row has no list; what is ranked for it stays inside the row all the same)
            if (me != 0 && me >= least) {
                top.chosen[atomicAdd(&top.n_chosen, 1u)] = tid;
                if (tid < head && top_key((float)x[tid], v0 + tid) >= least) add_candidate(top, top_key((float)x[tid], v0 + tid));
                if (tid < tail && top_key((float)x[tail_at + tid], v0 + tail_at + tid) >= least)
                    add_candidate(top, top_key((float)x[tail_at + tid], v0 + tail_at + tid));
            }
            __syncthreads();
            const int32_t chosen = (int32_t)top.n_chosen;
            const int32_t turns = (chunks + THREADS - 1) / THREADS, again = chosen * turns;
            for (int32_t q = tid; q < again; q += LP_AT_ONCE * THREADS) {
                int32_t c[LP_AT_ONCE];
#pragma unroll
                for (int j = 0; j < LP_AT_ONCE; ++j) {
                    const int32_t at_q = min(q + j * THREADS, again - 1), turn = at_q / chosen;
                    c[j] = q + j * THREADS < again ? turn * THREADS + top.chosen[at_q - turn * chosen] : chunks;
                    next[j] = body[min(c[j], chunks - 1)];
                }
#pragma unroll
                for (int j = 0; j < LP_AT_ONCE; ++j) {
                    if (c[j] >= chunks) continue;
                    float f[N];
                    unpack<T>(next[j], f);
                    const int32_t place = v0 + head + c[j] * N;
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (top_key(f[i], place) >= least) add_candidate(top, top_key(f[i], place + i));
                }
            }
            rank_candidates(top, a.n_top, [&](auto visit) {
                for (int32_t v = tid; v < n; v += THREADS) visit(top_key((float)x[v], v0 + v));
            }, put);
        }
        __syncthreads();                         // red is free again
    }
}

// One wave per row: its parts' sums and lists as one.
constexpr int LJ_AT_ONCE = 8;                    // keys asked for at once
template <typename T>
__global__ __launch_bounds__(WAVE) void logprob_join_kernel(const LogprobArgs a, int32_t parts, const char* __restrict__ ws) {
    __shared__ TopLds<WAVE> top;
    const float k = a.inv_t * LOG2E;
    const int lane = threadIdx.x;
    for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
        if (a.mask && a.mask[r] == 0) {
            write_nothing(a, r);
            continue;
        }
        const int32_t token = a.token ? a.token[r] : 0;
        const bool in = token >= 0 && token < a.vocab;
        const float x_token = a.token ? (float)(static_cast<const T*>(a.x) + r * a.stride)[in ? token : 0] : 0.0f;
        const size_t bytes = part_bytes(a.n_top);
        const char* first = ws + r * parts * bytes;
        const auto sums_of = [&](int p) { return reinterpret_cast<const PartHead*>(first + p * bytes)->sums; };
        const auto keys_of = [&](int p) { return reinterpret_cast<const uint64_t*>(first + p * bytes + sizeof(PartHead)); };
        // every part's nth key has nth keys of that part that are not below it: so many parts together have n_top (of the
        // first parts alone where there are more than lanes)
        const int nth = max(1, min(a.n_top, (2 * a.n_top + parts - 1) / min(parts, WAVE))), of_parts = (a.n_top + nth - 1) / nth;
        const uint64_t bound = a.n_top > 0 && lane < parts ? keys_of(lane)[nth - 1] : 0ull;
        RowSums all = {-INFINITY, 0.0f, 0.0f};
        for (int p = lane; p < parts; p += WAVE) all.m = fmaxf(all.m, sums_of(p).m);
        all.m = wave_max(all.m);
        for (int p = lane; p < parts; p += WAVE) {
            const RowSums x = sums_of(p);
            const float d = (x.m - all.m) * k, f = __builtin_amdgcn_exp2f(d);
            all.s += f * x.s;
            all.u += f * (x.u + fmaxf(d, -1e4f) * x.s);
        }
        all.s = wave_sum(all.s);
        all.u = wave_sum(all.u);
        const RowResult w = finish(all, a.inv_t);
        if (lane == 0) {
            if (!in) set_status(a.status, DC_ERR_TOKEN_RANGE);
            write_row(a, r, w, in, x_token);
            top.n_candidates = 0;
        }
        if (a.n_top == 0) continue;
        const uint64_t least = wave_nth_key<SORT_BITS<T>>(bound, of_parts);
        __syncthreads();
        const int32_t n_keys = parts * a.n_top;
        for (int32_t q = lane; q < n_keys; q += LJ_AT_ONCE * WAVE) {
            uint64_t key[LJ_AT_ONCE];
#pragma unroll
            for (int j = 0; j < LJ_AT_ONCE; ++j) {
                const int32_t at = min(q + j * WAVE, n_keys - 1), p = at / a.n_top;
                key[j] = keys_of(p)[at - p * a.n_top];
            }
#pragma unroll
            for (int j = 0; j < LJ_AT_ONCE; ++j)
                if (q + j * WAVE < n_keys && key[j] != 0 && key[j] >= least) add_candidate(top, key[j]);
        }
        rank_candidates(top, a.n_top, [&](auto visit) {
            for (int32_t q = lane; q < n_keys; q += WAVE) visit(keys_of(q / a.n_top)[q % a.n_top]);
        }, [&](int i, uint64_t key) { write_top(a, r, i, w, key); });
    }
}

// How a row is cut.  Many rows: a workgroup of LP_THREADS each, several to a compute unit, so that one's reductions and
// ranking run beside another's loads (a larger one for alternatives of rows above 512 KB, whose second look it shortens).  At
// most one row to a compute unit: a larger workgroup, or, where one unit's loads take longer than a second launch does, parts
// of at least LP_LEAST logits, about LP_GROUPS of them.  Measured, us, no alternatives / 20 of them, the two sides of each
// border:
//   300 x 32000 bf16      narrow  8.7 / 15.3   wide  11.7 / 20.8
//   64 x 32000 f32        wide    7.4 / 11.3   narrow 8.8 / 14.5
//   64 x 12000 f32        narrow  8.0 /  9.0   wide   7.5 /  9.9
//   1000 x 152064 f32     narrow 91.6 /  171   wide  95.5 /  130
//   1000 x 152064 bf16    narrow 51.0 / 83.8   wide  62.8 / 87.1
//   1 x 152064 f32        parts   9.6 / 13.9   wide  15.1 / 20.9
//   64 x 152064 f32       parts  13.8 / 19.2   wide  16.8 / 24.3
//   256 x 152064 f32      wide   27.7 / 35.5   parts 31.1 / 51.3
//   1 x 32000 f32         wide    7.4 / 10.3   parts  9.8 / 13.8
// The row of 12000 is narrow for the sake of its alternatives; 65 to 255 long rows, between the two sides of their border, were not
// measured.  1024 parts in all instead of 512: 64 x 152064 f32 with 20 alternatives 21.2 us.
constexpr int64_t LP_GROUPS = 512, LP_LEAST = 4096, LP_CUT_ROWS = 64;
struct Cut { int32_t parts, per_part; bool wide; };
static Cut cut_of(int64_t n_rows, int32_t vocab, int32_t type, int32_t n_top) {
    const int64_t bytes = (int64_t)vocab * (type == DC_F32 ? 4 : 2);
    if (n_rows > 256 || bytes <= 1 << 16) return Cut{1, vocab, n_top > 0 && bytes > 1 << 19};
    if (n_rows > LP_CUT_ROWS || bytes <= 1 << 17) return Cut{1, vocab, true};
    int64_t parts = n_rows > 0 ? (LP_GROUPS + n_rows - 1) / n_rows : 1;
    const int64_t most = (vocab + LP_LEAST - 1) / LP_LEAST;
    parts = parts < most ? parts : most;
    const int32_t per = (int32_t)(((vocab + parts - 1) / parts + 63) / 64 * 64);
    return Cut{(vocab + per - 1) / per, per, false};
}

size_t logprob_workspace_need(int64_t n_rows, int32_t vocab, int32_t type, int32_t n_top) {
    const Cut c = cut_of(n_rows, vocab, type, n_top);
    return c.parts > 1 ? (size_t)n_rows * c.parts * part_bytes(n_top) : 0;
}
// As much as any call of at most these rows and alternatives needs: the number of parts in all goes up and down with the rows, and
// many rows have none.
size_t logprob_workspace_bytes(int64_t n_rows, int32_t vocab, int32_t type, int32_t n_top) {
    size_t most = 0;
    for (int64_t n = 1; n <= std::min(n_rows, LP_CUT_ROWS); ++n) most = std::max(most, logprob_workspace_need(n, vocab, type, n_top));
    return most;
}

hipError_t launch_logprob(const LogprobArgs& a, int32_t type, void* d_ws, hipStream_t st) {
    if (a.n_rows == 0) return hipSuccess;
    const Cut c = cut_of(a.n_rows, a.vocab, type, a.n_top);
    const int64_t units = a.n_rows * c.parts;
    const unsigned grid = (unsigned)(units < (1 << 20) ? units : 1 << 20), rows = (unsigned)(a.n_rows < (1 << 20) ? a.n_rows : 1 << 20);
    return with_type(type, [&](auto e) {
        using T = typename decltype(e)::type;
        char* ws = static_cast<char*>(d_ws);
        const auto go = [&](auto entropy, auto top) {
            constexpr bool ENTROPY = decltype(entropy)::value, TOP = decltype(top)::value;
            if (c.wide) logprob_kernel<LP_WIDE, T, ENTROPY, TOP><<<grid, LP_WIDE, 0, st>>>(a, c.parts, c.per_part, ws);
            else logprob_kernel<LP_THREADS, T, ENTROPY, TOP><<<grid, LP_THREADS, 0, st>>>(a, c.parts, c.per_part, ws);
        };
        if (a.entropy && a.n_top) go(std::true_type{}, std::true_type{});
        else if (a.entropy) go(std::true_type{}, std::false_type{});
        else if (a.n_top) go(std::false_type{}, std::true_type{});
        else go(std::false_type{}, std::false_type{});
        if (c.parts > 1) logprob_join_kernel<T><<<rows, WAVE, 0, st>>>(a, c.parts, ws);
        return hipGetLastError();
    });
}

// ---- the gradient: dx = p * -(a + b (log p + H)) / T, and a / T more at the given token ----

constexpr int LG_THREADS = 256, LG_AT_ONCE = 4;
template <typename T> constexpr int LG_PIECE = LG_THREADS * LG_AT_ONCE * CHUNK_ELEMS<T>;

template <typename T>
__device__ __forceinline__ u32x4 pack(const float (&f)[CHUNK_ELEMS<T>]) {
    union { T e[CHUNK_ELEMS<T>]; u32x4 q; } r;
#pragma unroll
    for (int i = 0; i < CHUNK_ELEMS<T>; ++i) r.e[i] = (T)f[i];
    return r.q;
}

// One workgroup per piece of a row: 16 bytes in, 16 bytes out, four times a thread.  Bound by the two streams: 8192 x 152064 in
// bf16, 5.0 GB, in 0.82 ms, 6.1 TB/s, what a large copy reaches; with a quarter of the rows masked 5.8 TB/s.  64 registers, so that
// a SIMD holds 8 waves: 1 to 4 % quicker than 7 of them, although two registers are spilled for 16-bit logits with an entropy.
// Half as much a workgroup: 5 % slower.  Rows of x and of the gradient that lie differently to 16 bytes go element by element:
// 8192 x 152063 in 1.96 ms (0.90 where they lie alike).
template <typename T, bool ENTROPY>
__global__ __launch_bounds__(LG_THREADS, 8) void logprob_grad_kernel(const LogprobGradArgs a, int32_t pieces) {
    constexpr int N = CHUNK_ELEMS<T>;
    const int tid = threadIdx.x;
    for (int64_t unit = blockIdx.x; unit < a.n_rows * pieces; unit += gridDim.x) {
        const int64_t r = unit / pieces;
        const int32_t v0 = (int32_t)(unit - r * pieces) * LG_PIECE<T>, n = min(LG_PIECE<T>, a.vocab - v0);
        const T* x = static_cast<const T*>(a.x) + r * a.stride + v0;
        T* g = static_cast<T*>(a.g) + r * a.g_stride + v0;
        const float ga = a.grad_logprob[r] * a.inv_t, gb = ENTROPY ? a.grad_entropy[r] * a.inv_t : 0.0f;
        const bool zero = (a.mask && a.mask[r] == 0) || (a.grad_logprob[r] == 0.0f && (!ENTROPY || a.grad_entropy[r] == 0.0f));
        // both streams in whole 16 bytes where they can be: up to the first and behind the last of those an element to a thread
        const uint32_t xa = (uint32_t)reinterpret_cast<uintptr_t>(x) & 15, ga16 = (uint32_t)reinterpret_cast<uintptr_t>(g) & 15;
        const bool together = zero || xa == ga16;
        const int32_t head = together ? min(n, (int32_t)((16 - ga16) & 15) / (int32_t)sizeof(T)) : 0;
        const int32_t chunks = together ? (n - head) / N : 0;
        const u32x4* from = reinterpret_cast<const u32x4*>(x + head);
        u32x4* to = reinterpret_cast<u32x4*>(g + head);
        if (zero) {
            for (int32_t c = tid; c < chunks; c += LG_THREADS) store16(to + c, u32x4{0, 0, 0, 0});
            if (tid < head) g[tid] = (T)0.0f;
            for (int32_t v = head + chunks * N + tid; v < n; v += LG_THREADS) g[v] = (T)0.0f;
            continue;
        }
        u32x4 q[LG_AT_ONCE];
        if (chunks > 0)
#pragma unroll
            for (int j = 0; j < LG_AT_ONCE; ++j) q[j] = __builtin_nontemporal_load(from + min(tid + j * LG_THREADS, chunks - 1));
        int32_t token = -1;
        if (a.token) {
            token = a.token[r];
            if ((token < 0 || token >= a.vocab) && tid == 0 && v0 == 0) set_status(a.status, DC_ERR_TOKEN_RANGE);
            token -= v0;                         // (outside the piece: no element has it)
        }
        const float k = a.inv_t * LOG2E, m = a.stat[2 * r], log_sum2 = a.stat[2 * r + 1] * LOG2E;
        const float c0 = ENTROPY && gb != 0.0f ? -fmaf(gb, a.entropy[r], ga) : -ga, c1 = -gb * LN2;
        const auto one = [&](float v) {
            const float lp2 = fmaf(v - m, k, -log_sum2), p = __builtin_amdgcn_exp2f(lp2);
            // (a logit of -infinity: 0 times a number, not times -infinity)
            return p * (ENTROPY ? fmaf(c1, fmaxf(lp2, -1e4f), c0) : c0);
        };
#pragma unroll
        for (int j = 0; j < LG_AT_ONCE; ++j) {
            const int32_t c = tid + j * LG_THREADS;
            if (c < chunks) {
                float f[N];
                unpack<T>(q[j], f);
#pragma unroll
                for (int i = 0; i < N; ++i) f[i] = one(f[i]);
                const uint32_t at = (uint32_t)(token - head - c * N);
                if (at < (uint32_t)N)
#pragma unroll
                    for (int i = 0; i < N; ++i) f[i] += at == (uint32_t)i ? ga : 0.0f;
                store16(to + c, pack<T>(f));
            }
        }
        if (tid < head) g[tid] = (T)(one((float)x[tid]) + (tid == token ? ga : 0.0f));
        for (int32_t v = head + chunks * N + tid; v < n; v += LG_THREADS) g[v] = (T)(one((float)x[v]) + (v == token ? ga : 0.0f));
    }
}

hipError_t launch_logprob_grad(const LogprobGradArgs& a, int32_t type, hipStream_t st) {
    if (a.n_rows == 0) return hipSuccess;
    return with_type(type, [&](auto e) {
        using T = typename decltype(e)::type;
        const int32_t pieces = (a.vocab + LG_PIECE<T> - 1) / LG_PIECE<T>;
        const int64_t units = a.n_rows * pieces;
        const unsigned grid = (unsigned)(units < (1 << 23) ? units : 1 << 23);
        if (a.grad_entropy) logprob_grad_kernel<T, true><<<grid, LG_THREADS, 0, st>>>(a, pieces);
        else logprob_grad_kernel<T, false><<<grid, LG_THREADS, 0, st>>>(a, pieces);
        return hipGetLastError();
    });
}

}  // namespace dc
