// Gradient of an embedding table: dW[v, :] = scale * sum of g[t, :] over the tokens t with id v.
//
// The tokens are sorted by id (stable, so the tokens of one id stay in ascending order), and the sorted sequence is cut
// into chunks of CHUNK entries: a hot id costs as much per token as a rare one, and no float goes through an atomic.
//   sort_portions   PORTION tokens per workgroup, radix sort in the LDS
//   merge_runs      up to MERGE_WAYS sorted runs into one: an entry's place is its own plus, for every other run, how many
//                   entries there come before it (a binary search each); once for every factor of MERGE_WAYS
//   add_rows        one wave per chunk and 512 columns: sums the rows of the segments (entries of one id) that start in the
//                   chunk, each in ascending token order, and writes them.  A segment of more than CHUNK entries is
//                   summed in pieces, one per chunk that it touches, into workspace memory.  Further waves write the rows
//                   without a token (a bit per id, set where the tokens are sorted).
//   join_pieces     the pieces of the long segments, in ascending order
#include "actor_device.h"

namespace dc {

constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / WAVE;
constexpr int PORTION = 4096, PER_THREAD = PORTION / SORT_THREADS;
constexpr int MERGE_WAYS = 32, MERGE_THREADS = 256;
constexpr int CHUNK = 64;
constexpr int COLS = 512;                        // columns of a wave: eight to a lane
constexpr int ADD_THREADS = 256;
constexpr int FILL_ROWS = 8;                     // rows of the table per wave that looks for those without a token
constexpr int JOIN_THREADS = 256;

static inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

struct EmbGradWs {
    uint32_t* key[2];                            // ids, sorted; an entry without a token has the id `vocab`
    int32_t*  pos[2];                            // the tokens' places
    uint32_t* present;                           // a bit per id
    int32_t*  n_long;                            // long segments, and the chunks that they start in
    int32_t*  long_at;
    float*    piece;                             // [2 * n_chunks][dim]: of the segment that reaches into the chunk, of the one that leaves it
    size_t    bytes;
};
static EmbGradWs carve_emb_grad(void* base, int64_t n_tokens, int64_t vocab, int64_t dim) {
    EmbGradWs w;
    char* p = static_cast<char*>(base);
    size_t off = 0;
    const int64_t chunks = (n_tokens + CHUNK - 1) / CHUNK;
    const auto take = [&](size_t n) { char* q = p + off; off += round_up(n, 256); return q; };
    for (int i = 0; i < 2; ++i) {
        w.key[i] = reinterpret_cast<uint32_t*>(take((size_t)n_tokens * 4));
        w.pos[i] = reinterpret_cast<int32_t*>(take((size_t)n_tokens * 4));
    }
    w.present = reinterpret_cast<uint32_t*>(take((size_t)(vocab + 31) / 32 * 4));
    w.n_long = reinterpret_cast<int32_t*>(take(4));
    w.long_at = reinterpret_cast<int32_t*>(take((size_t)chunks * 4));
    // segments are cut only where there are more tokens than a chunk
    w.piece = reinterpret_cast<float*>(take(n_tokens > CHUNK ? (size_t)chunks * 2 * (size_t)dim * 4 : 0));
    w.bytes = off;
    return w;
}
size_t embedding_grad_workspace_bytes(int64_t n_tokens, int64_t vocab, int64_t dim) {
    return carve_emb_grad(nullptr, n_tokens, vocab, dim).bytes;
}

// A portion's tokens by id: least significant digit first, `digit_bits` (at most 8) at a time.  A wave ranks 64 entries by
// ballots over the digit's bits; counts are kept per digit and wave, so the order within a digit is that of the tokens.
__global__ __launch_bounds__(SORT_THREADS) void sort_portions_kernel(const EmbeddingGradArgs a, EmbGradWs w, int digit_bits, int passes,
                                                                     int set_present) {
    __shared__ uint32_t keys[PORTION];
    __shared__ uint16_t places[PORTION];
    __shared__ uint32_t counts[256 * SORT_WAVES];
    __shared__ uint32_t tmp[SORT_WAVES];
    const int lane = lane_id(), wave = threadIdx.x / WAVE;
    const int32_t first = blockIdx.x * PORTION;
    const int32_t words = (a.vocab + 31) / 32;
    if (!a.accumulate)
        for (int32_t i = blockIdx.x * SORT_THREADS + threadIdx.x; i < words; i += gridDim.x * SORT_THREADS) w.present[i] = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.n_long = 0;

    uint32_t key[PER_THREAD];
    uint16_t place[PER_THREAD];
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
        const int at = wave * (WAVE * PER_THREAD) + j * WAVE + lane;
        const int32_t t = first + at;
        key[j] = 0xFFFFFFFFu;                    // behind the last token: last in every pass
        place[j] = (uint16_t)at;
        if (t < a.n_tokens) {
            const int32_t id = a.token[t];
            const bool in = id >= 0 && id < a.vocab;
            if (!in && id != DC_NO_TOKEN) set_status(a.status, DC_ERR_TOKEN_RANGE);
            key[j] = in ? (uint32_t)id : (uint32_t)a.vocab;
        }
    }
    const uint32_t digits = 1u << digit_bits;
    const uint64_t below = (1ull << lane) - 1;
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * digit_bits;
        for (uint32_t i = threadIdx.x; i < digits * SORT_WAVES; i += SORT_THREADS) counts[i] = 0;
        __syncthreads();
        uint32_t rank[PER_THREAD];
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
            const uint32_t d = (key[j] >> shift) & (digits - 1);
            uint64_t same = ~0ull;
            for (int b = 0; b < digit_bits; ++b) {
                const uint64_t set = __ballot((d >> b) & 1);
                same &= (d >> b) & 1 ? set : ~set;
            }
            volatile uint32_t* c = &counts[d * SORT_WAVES + wave];        // this wave's own count
            const uint32_t before = *c;
            __builtin_amdgcn_wave_barrier();
            rank[j] = before + (uint32_t)__popcll(same & below);
            if ((same & below) == 0) *c = before + (uint32_t)__popcll(same);
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        // exclusive prefix over (digit, wave): every thread takes as many neighbouring counts as there are per thread
        const uint32_t per = (digits * SORT_WAVES + SORT_THREADS - 1) / SORT_THREADS, from = threadIdx.x * per;
        uint32_t sum = 0, total;
        for (uint32_t i = 0; i < per; ++i)
            if (from + i < digits * SORT_WAVES) sum += counts[from + i];
        uint32_t run = block_excl_scan_add<uint32_t>(sum, tmp, &total);
        for (uint32_t i = 0; i < per; ++i)
            if (from + i < digits * SORT_WAVES) {
                const uint32_t c = counts[from + i];
                counts[from + i] = run;
                run += c;
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
            const uint32_t d = (key[j] >> shift) & (digits - 1);
            const uint32_t to = counts[d * SORT_WAVES + wave] + rank[j];
            keys[to] = key[j];
            places[to] = place[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
            const int at = wave * (WAVE * PER_THREAD) + j * WAVE + lane;
            key[j] = keys[at];
            place[j] = places[at];
        }
        __syncthreads();
    }
    const int32_t n = min(PORTION, a.n_tokens - first);
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
        const int at = wave * (WAVE * PER_THREAD) + j * WAVE + lane;
        if (at < n) {
            w.key[0][first + at] = key[j];
            w.pos[0][first + at] = first + place[j];
        }
    }
    if (set_present) {                           // (one workgroup: its zeros above are in place)
        __threadfence();
        __syncthreads();
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j)
            if (key[j] < (uint32_t)a.vocab) atomicOr(&w.present[key[j] >> 5], 1u << (key[j] & 31));
    }
}

// Runs of `run` sorted entries, MERGE_WAYS neighbouring ones into one; one thread per entry.
__global__ __launch_bounds__(MERGE_THREADS) void merge_runs_kernel(const EmbeddingGradArgs a, const uint32_t* __restrict__ key_in,
                                                                   const int32_t* __restrict__ pos_in, uint32_t* __restrict__ key_out,
                                                                   int32_t* __restrict__ pos_out, uint32_t* present, int64_t run,
                                                                   int set_present) {
    const int64_t i = (int64_t)blockIdx.x * MERGE_THREADS + threadIdx.x;
    if (i >= a.n_tokens) return;
    const uint32_t key = key_in[i];
    const int64_t mine = i / run, group = mine / MERGE_WAYS;
    const int64_t first = group * MERGE_WAYS, last = min(first + MERGE_WAYS, ((int64_t)a.n_tokens + run - 1) / run);
    int64_t to = first * run + (i - mine * run);
    for (int64_t q = first; q < last; ++q) {
        if (q == mine) continue;
        // entries of an earlier run come first among equals
        int64_t lo = q * run, hi = min(lo + run, (int64_t)a.n_tokens);
        const int64_t base = lo;
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            const uint32_t k = key_in[mid];
            if (k < key || (k == key && q < mine)) lo = mid + 1; else hi = mid;
        }
        to += lo - base;
    }
    key_out[to] = key;
    pos_out[to] = pos_in[i];
    if (set_present && key < (uint32_t)a.vocab && (i == mine * run || key_in[i - 1] != key))
        atomicOr(&present[key >> 5], 1u << (key & 31));
}

// ---- eight columns of a row: neighbours where rows are aligned (VEC), 64 apart where they are not ----
template <typename T> struct alignas(16) Pack { T v[16 / sizeof(T)]; };

template <bool VEC>
__device__ __forceinline__ int64_t column(int64_t slab, int j) {
    return slab * COLS + (VEC ? (int64_t)lane_id() * 8 + j : (int64_t)j * WAVE + lane_id());
}
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* row, int64_t slab, int64_t dim, float (&f)[8]) {
    if constexpr (VEC) {
        if (column<VEC>(slab, 0) < dim) {
            constexpr int N = 16 / sizeof(T);
#pragma unroll
            for (int h = 0; h < 8 / N; ++h) {
                const Pack<T> p = *reinterpret_cast<const Pack<T>*>(row + column<VEC>(slab, 0) + h * N);
#pragma unroll
                for (int j = 0; j < N; ++j) f[h * N + j] = (float)p.v[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = 0.0f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t c = column<VEC>(slab, j);
            f[j] = c < dim ? (float)row[c] : 0.0f;
        }
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* row, int64_t slab, int64_t dim, const float (&f)[8]) {
    if constexpr (VEC) {
        if (column<VEC>(slab, 0) < dim) {
            constexpr int N = 16 / sizeof(T);
#pragma unroll
            for (int h = 0; h < 8 / N; ++h) {
                Pack<T> p;
#pragma unroll
                for (int j = 0; j < N; ++j) p.v[j] = (T)f[h * N + j];
                *reinterpret_cast<Pack<T>*>(row + column<VEC>(slab, 0) + h * N) = p;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t c = column<VEC>(slab, j);
            if (c < dim) row[c] = (T)f[j];
        }
    }
}

// A finished sum to its row of the table.
template <bool VEC, typename W>
__device__ __forceinline__ void write_row(const EmbeddingGradArgs& a, uint32_t id, int64_t slab, const float (&sum)[8]) {
    W* row = static_cast<W*>(a.dw) + (int64_t)id * a.dw_stride;
    float out[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = sum[j] * a.scale;
    if (a.accumulate) {
        float old[8];
        load8<VEC>(row, slab, a.dim, old);
#pragma unroll
        for (int j = 0; j < 8; ++j) out[j] += old[j];
    }
    store8<VEC>(row, slab, a.dim, out);
}

constexpr int ROWS_AT_ONCE = 8;

template <bool VEC, typename G, typename W>
__global__ __launch_bounds__(ADD_THREADS) void add_rows_kernel(const EmbeddingGradArgs a, const uint32_t* __restrict__ skey,
                                                               const int32_t* __restrict__ spos, const uint32_t* __restrict__ present,
                                                               int32_t* n_long, int32_t* long_at, float* __restrict__ piece,
                                                               int64_t chunks, int64_t slabs) {
    const int64_t unit = (int64_t)blockIdx.x * (ADD_THREADS / WAVE) + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int lane = lane_id();
    if (unit >= chunks * slabs) {                // rows without a token
        const int64_t v0 = (unit - chunks * slabs) * FILL_ROWS;
        if (a.accumulate || v0 >= a.vocab) return;
        const uint32_t bits = present[v0 >> 5] >> (v0 & 31);
        const float zero[8] = {};
        for (int r = 0; r < FILL_ROWS && v0 + r < a.vocab; ++r) {
            if ((bits >> r) & 1) continue;
            W* row = static_cast<W*>(a.dw) + (v0 + r) * a.dw_stride;
            for (int64_t s = 0; s < slabs; ++s) store8<VEC>(row, s, a.dim, zero);
        }
        return;
    }
    const int64_t chunk = unit / slabs, slab = unit % slabs;
    const int32_t c0 = (int32_t)(chunk * CHUNK);
    // the chunk's entries, those behind it that a segment of it may reach, those before it
    constexpr uint32_t NONE = 0xFFFFFFFFu;       // (an id that no entry has)
    const uint32_t k1 = c0 + lane < a.n_tokens ? skey[c0 + lane] : NONE;
    const uint32_t k2 = c0 + CHUNK + lane < a.n_tokens ? skey[c0 + CHUNK + lane] : NONE;
    const uint32_t k0 = c0 > 0 ? skey[c0 - CHUNK + lane] : NONE;
    const int32_t p1 = c0 + lane < a.n_tokens ? spos[c0 + lane] : 0;
    const int32_t p2 = c0 + CHUNK + lane < a.n_tokens ? spos[c0 + CHUNK + lane] : 0;
    const uint32_t vocab = (uint32_t)a.vocab;
    const uint32_t before = __shfl(k0, CHUNK - 1), up1 = __shfl_up(k1, 1), up2 = __shfl_up(k2, 1), last1 = __shfl(k1, CHUNK - 1);
    const uint64_t start1 = __ballot(k1 != (lane ? up1 : before)), start2 = __ballot(k2 != (lane ? up2 : last1));
    const uint64_t valid1 = __ballot(k1 < vocab);
    const int n_valid = valid1 ? 64 - __builtin_clzll(valid1) : 0;         // valid entries come first
    if (n_valid == 0) return;

    float sum[8];
    const auto clear = [&] {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    };
    // entries [from, to); `ends`: whether entry i is the last of its segment; done(i) writes the sum there
    const auto walk = [&](int from, int to, auto ends, auto done) {
        clear();
        for (int i = from; i < to; i += ROWS_AT_ONCE) {
            float g[ROWS_AT_ONCE][8];
#pragma unroll
            for (int j = 0; j < ROWS_AT_ONCE; ++j) {
                const int e = min(i + j, to - 1);
                const int32_t t = e < WAVE ? __builtin_amdgcn_readlane(p1, e) : __builtin_amdgcn_readlane(p2, e - WAVE);
                load8<VEC>(static_cast<const G*>(a.g) + (int64_t)t * a.g_stride, slab, a.dim, g[j]);
            }
#pragma unroll
            for (int j = 0; j < ROWS_AT_ONCE; ++j) {
                if (i + j >= to) break;
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] += g[j][c];
                if (ends(i + j)) { done(i + j); clear(); }
            }
        }
    };
    const auto to_piece = [&](int which) {
        store8<VEC>(piece + (chunk * 2 + which) * a.dim, slab, a.dim, sum);
    };

    // the segment that reaches into the chunk: another chunk's, unless it is long
    const int first_start = start1 ? __builtin_ctzll(start1) : CHUNK;
    if (first_start > 0) {
        const int r = min(first_start, n_valid);
        // r - 1 is its last entry here; it is long if it has CHUNK entries before that one
        const bool is_long = r == CHUNK || __builtin_amdgcn_readlane(k0, (r - 1) & 63) == __builtin_amdgcn_readfirstlane(k1);
        if (is_long) walk(0, r, [&](int i) { return i == r - 1; }, [&](int) { to_piece(0); });
    }
    if (first_start >= n_valid) return;
    // the segments that start here; the last of them may go on behind the chunk
    const uint64_t own = start1 & (n_valid == 64 ? ~0ull : (1ull << n_valid) - 1);
    const int s = 63 - __builtin_clzll(own);
    const uint32_t last_key = __builtin_amdgcn_readlane(k1, s);
    int to = n_valid;
    bool is_long = false;
    if (n_valid == CHUNK) {
        is_long = __builtin_amdgcn_readlane(k2, s) == last_key;            // entry s + CHUNK
        if (!is_long) to = CHUNK + (start2 ? __builtin_ctzll(start2) : CHUNK);
    }
    const auto ends = [&](int i) {
        if (i == to - 1) return true;
        return i + 1 < CHUNK ? ((start1 >> (i + 1)) & 1) != 0 : false;
    };
    walk(first_start, to, ends, [&](int i) {
        if (is_long && i == to - 1) {
            to_piece(1);
            if (slab == 0 && lane == 0) long_at[atomicAdd(n_long, 1)] = (int32_t)chunk;
        } else {
            const uint32_t id = i < CHUNK ? __builtin_amdgcn_readlane(k1, i) : __builtin_amdgcn_readlane(k2, i - CHUNK);
            write_row<VEC, W>(a, id, slab, sum);
        }
    });
}

// One workgroup per long segment and 512 columns, round and round; its waves take every fourth piece each.
template <bool VEC, typename W>
__global__ __launch_bounds__(JOIN_THREADS) void join_pieces_kernel(const EmbeddingGradArgs a, const uint32_t* __restrict__ skey,
                                                                   const int32_t* __restrict__ n_long, const int32_t* __restrict__ long_at,
                                                                   const float* __restrict__ piece, int64_t chunks, int64_t slabs) {
    constexpr int WAVES = JOIN_THREADS / WAVE;
    __shared__ float part[WAVES][8][WAVE];
    const int lane = lane_id(), wave = threadIdx.x / WAVE;
    const int64_t units = (int64_t)*n_long * slabs;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t c0 = long_at[u / slabs], slab = u % slabs;
        const uint32_t id = skey[c0 * CHUNK + CHUNK - 1];
        // the last chunk whose first entry is of this segment: 64 looks at a time
        int64_t lo = c0, hi = chunks;            // (lo is in it, hi is not)
        while (hi - lo > 1) {
            const int64_t step = (hi - lo + WAVE - 1) / WAVE;
            const int64_t at = lo + (int64_t)(lane + 1) * step;
            const uint64_t in = __ballot(at < hi && skey[at * CHUNK] == id);
            lo += (int64_t)__popcll(in) * step;
            hi = min(hi, lo + step);
        }
        float sum[8] = {};
        for (int64_t c = c0 + wave; c <= lo; c += WAVES) {
            float f[8];
            load8<VEC>(piece + (c * 2 + (c == c0)) * a.dim, slab, a.dim, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += f[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) part[wave][j][lane] = sum[j];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                for (int w = 1; w < WAVES; ++w) sum[j] += part[w][j][lane];
            write_row<VEC, W>(a, id, slab, sum);
        }
        __syncthreads();
    }
}

hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, int32_t g_type, int32_t dw_type, void* d_ws, hipStream_t st) {
    if (a.vocab == 0 || a.dim == 0 || (a.n_tokens == 0 && a.accumulate)) return hipSuccess;
    EmbGradWs w = carve_emb_grad(d_ws, a.n_tokens, a.vocab, a.dim);
    const int64_t portions = a.n_tokens > 0 ? ((int64_t)a.n_tokens + PORTION - 1) / PORTION : 1;
    int bits = 1;
    while ((1 << bits) <= a.vocab) ++bits;       // ids up to and with `vocab`
    const int passes = (bits + 7) / 8, digit_bits = (bits + passes - 1) / passes;
    sort_portions_kernel<<<(unsigned)portions, SORT_THREADS, 0, st>>>(a, w, digit_bits, passes, portions == 1 && !a.accumulate);
    int at = 0;
    for (int64_t run = PORTION; run < a.n_tokens; run *= MERGE_WAYS) {
        const bool final = run * MERGE_WAYS >= a.n_tokens;
        merge_runs_kernel<<<(unsigned)((a.n_tokens + MERGE_THREADS - 1) / MERGE_THREADS), MERGE_THREADS, 0, st>>>(
            a, w.key[at], w.pos[at], w.key[at ^ 1], w.pos[at ^ 1], w.present, run, final && !a.accumulate);
        at ^= 1;
    }
    const int64_t chunks = ((int64_t)a.n_tokens + CHUNK - 1) / CHUNK, slabs = (a.dim + COLS - 1) / COLS;
    const int64_t fill = a.accumulate ? 0 : ((int64_t)a.vocab + FILL_ROWS - 1) / FILL_ROWS;
    const int64_t units = chunks * slabs + fill, blocks = (units + ADD_THREADS / WAVE - 1) / (ADD_THREADS / WAVE);
    if (blocks > 0x7FFFFFFFLL) return hipErrorInvalidValue;
    return with_type(g_type, [&](auto ge) {
        return with_type(dw_type, [&](auto we) {
            using G = typename decltype(ge)::type;
            using W = typename decltype(we)::type;
            const auto aligned = [&](const void* p, int64_t stride, size_t size) {
                return (reinterpret_cast<uintptr_t>(p) % 16 == 0) && (size_t)stride * size % 16 == 0;
            };
            const bool vec = a.dim % 8 == 0 && aligned(a.g, a.g_stride, sizeof(G)) && aligned(a.dw, a.dw_stride, sizeof(W));
            const auto go = [&](auto v) {
                constexpr bool VEC = decltype(v)::value;
                add_rows_kernel<VEC, G, W><<<(unsigned)blocks, ADD_THREADS, 0, st>>>(a, w.key[at], w.pos[at], w.present, w.n_long,
                                                                                     w.long_at, w.piece, chunks, slabs);
                if (a.n_tokens > CHUNK) {
                    const int64_t most = (int64_t)a.n_tokens / (CHUNK + 1) * slabs;      // long segments there can be
                    join_pieces_kernel<VEC, W><<<(unsigned)(most < 1024 ? most : 1024), JOIN_THREADS, 0, st>>>(
                        a, w.key[at], w.n_long, w.long_at, w.piece, chunks, slabs);
                }
            };
            if (vec) go(std::true_type{}); else go(std::false_type{});
            return hipGetLastError();
        });
    });
}

}  // namespace dc
