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
//                   without a token.
//   join_pieces     the pieces of the long segments, in ascending order
#include "actor_device.h"

namespace dc {

constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / WAVE;
constexpr int PORTION = 4096, PER_THREAD = PORTION / SORT_THREADS;
constexpr int MERGE_WAYS = 32, MERGE_THREADS = 256;
constexpr int CHUNK = 64;
constexpr int COLS = 512;                        // columns of a wave: eight to a lane
constexpr int ADD_THREADS = 256;
constexpr int FILL_ROWS = 8, FILL_LANES = WAVE / FILL_ROWS;      // rows of the table per wave that looks for those without a token
constexpr int JOIN_THREADS = 256;

static inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

struct EmbGradWs {
    uint32_t* key[2];                            // ids, sorted; an entry without a token has the id `vocab`
    int32_t*  pos[2];                            // the tokens' places
    int32_t*  n_long;                            // long segments, and the chunks that they start in
    int32_t*  long_at;
    float*    piece;                             // [2 * n_chunks][dim]: of the segment that reaches into the chunk, of the one that leaves it
    size_t    bytes;
};
static EmbGradWs carve_emb_grad(void* base, int64_t n_tokens, int64_t dim) {
    EmbGradWs w;
    char* p = static_cast<char*>(base);
    size_t off = 0;
    const int64_t chunks = (n_tokens + CHUNK - 1) / CHUNK;
    const auto take = [&](size_t n) { char* q = p + off; off += round_up(n, 256); return q; };
    for (int i = 0; i < 2; ++i) {
        w.key[i] = reinterpret_cast<uint32_t*>(take((size_t)n_tokens * 4));
        w.pos[i] = reinterpret_cast<int32_t*>(take((size_t)n_tokens * 4));
    }
    w.n_long = reinterpret_cast<int32_t*>(take(4));
    w.long_at = reinterpret_cast<int32_t*>(take((size_t)chunks * 4));
    // segments are cut only where there are more tokens than a chunk
    w.piece = reinterpret_cast<float*>(take(n_tokens > CHUNK ? (size_t)chunks * 2 * (size_t)dim * 4 : 0));
    w.bytes = off;
    return w;
}
size_t embedding_grad_workspace_bytes(int64_t n_tokens, int64_t dim) {
    return carve_emb_grad(nullptr, n_tokens, dim).bytes;
}

// A portion's tokens by id: least significant digit first, `digit_bits` (at most 8) at a time.  A wave ranks 64 entries by
// ballots over the digit's bits; counts are kept per digit and wave, so the order within a digit is that of the tokens.
__global__ __launch_bounds__(SORT_THREADS) void sort_portions_kernel(const EmbeddingGradArgs a, EmbGradWs w, int digit_bits, int passes) {
    __shared__ uint32_t keys[PORTION];
    __shared__ uint16_t places[PORTION];
    __shared__ uint32_t counts[256 * SORT_WAVES];
    __shared__ uint32_t tmp[SORT_WAVES];
    const int lane = lane_id(), wave = threadIdx.x / WAVE;
    const int32_t first = blockIdx.x * PORTION;
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
}

// Runs of `run` sorted entries, MERGE_WAYS neighbouring ones into one.  Four lanes share an entry, each with a quarter of the
// runs: its searches go side by side, one look in each run per step.
constexpr int MERGE_LANES = 4, MERGE_EACH = MERGE_WAYS / MERGE_LANES, MERGE_ENTRIES = MERGE_THREADS / MERGE_LANES;
__global__ __launch_bounds__(MERGE_THREADS) void merge_runs_kernel(const EmbeddingGradArgs a, const uint32_t* __restrict__ key_in,
                                                                   const int32_t* __restrict__ pos_in, uint32_t* __restrict__ key_out,
                                                                   int32_t* __restrict__ pos_out, int32_t run) {
    const int lane = lane_id(), part = lane / (WAVE / MERGE_LANES);
    const int32_t at = blockIdx.x * MERGE_ENTRIES + (threadIdx.x / WAVE) * (WAVE / MERGE_LANES) + lane % (WAVE / MERGE_LANES);
    const int32_t i = min(at, a.n_tokens - 1);
    const uint32_t key = key_in[i];
    const int32_t mine = i / run, first = mine / MERGE_WAYS * MERGE_WAYS;
    int32_t lo[MERGE_EACH], len[MERGE_EACH];
#pragma unroll
    for (int j = 0; j < MERGE_EACH; ++j) {
        const int64_t from = (int64_t)(first + part * MERGE_EACH + j) * run;      // (may lie behind the last run)
        lo[j] = (int32_t)min(from, (int64_t)a.n_tokens);
        len[j] = first + part * MERGE_EACH + j == mine ? 0 : min(run, a.n_tokens - lo[j]);
    }
    // entries of an earlier run come first among equals: there the first greater one is looked for
    int32_t to = 0;
#pragma unroll
    for (int j = 0; j < MERGE_EACH; ++j) to -= lo[j];
    for (int32_t step = run; step > 0; step = step > 1 ? (step + 1) >> 1 : 0) {
#pragma unroll
        for (int j = 0; j < MERGE_EACH; ++j) {
            const int32_t half = (len[j] + 1) >> 1;
            const uint32_t k = key_in[min(lo[j] + (half > 0 ? half - 1 : 0), a.n_tokens - 1)];
            const bool less = k < key || (k == key && first + part * MERGE_EACH + j < mine);
            if (half > 0) {
                lo[j] += less ? half : 0;
                len[j] = less ? len[j] - half : half - 1;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < MERGE_EACH; ++j) to += lo[j];
    to += __shfl_xor(to, WAVE / MERGE_LANES);
    to += __shfl_xor(to, WAVE / MERGE_LANES * 2);
    to += first * run + (i - mine * run);
    if (at >= a.n_tokens || part != 0) return;
    key_out[to] = key;
    pos_out[to] = pos_in[i];
}

// ---- eight columns of a row per lane: neighbours where rows are aligned (VEC), 64 apart where they are not ----
template <bool VEC>
__device__ __forceinline__ int64_t column(int64_t slab, int j) {
    return slab * COLS + (VEC ? (int64_t)lane_id() * 8 + j : (int64_t)j * WAVE + lane_id());
}
// Eight elements as they lie in memory.
template <typename T>
union Raw8 {
    T e[8];
    u32x4 q[sizeof(T) / 2];
};
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* row, int64_t slab, int64_t dim, Raw8<T>& r) {
    if constexpr (VEC) {
        // (behind the row's end: its last columns again, which nobody stores)
        const u32x4* p = reinterpret_cast<const u32x4*>(row + min(column<VEC>(slab, 0), dim - 8));
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) r.q[h] = p[h];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.e[j] = row[min(column<VEC>(slab, j), dim - 1)];
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* row, int64_t slab, int64_t dim, const float (&f)[8]) {
    if constexpr (VEC) {
        if (column<VEC>(slab, 0) < dim) {
            Raw8<T> r;
#pragma unroll
            for (int j = 0; j < 8; ++j) r.e[j] = (T)f[j];
            u32x4* p = reinterpret_cast<u32x4*>(row + column<VEC>(slab, 0));
#pragma unroll
            for (int h = 0; h < (int)sizeof(T) / 2; ++h) p[h] = r.q[h];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t c = column<VEC>(slab, j);
            if (c < dim) row[c] = (T)f[j];
        }
    }
}
// A finished sum to its row of the table, added to what `old` holds of it.
template <bool VEC, bool ACC, typename W>
__device__ __forceinline__ void write_row(const EmbeddingGradArgs& a, uint32_t id, int64_t slab, const float (&sum)[8], const Raw8<W>& old) {
    float out[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = sum[j] * a.scale + (ACC ? (float)old.e[j] : 0.0f);
    store8<VEC>(static_cast<W*>(a.dw) + (int64_t)id * a.dw_stride, slab, a.dim, out);
}

template <bool VEC, bool ACC, typename G, typename W>
__global__ __launch_bounds__(ADD_THREADS) void add_rows_kernel(const EmbeddingGradArgs a, const uint32_t* __restrict__ skey,
                                                               const int32_t* __restrict__ spos,
                                                               int32_t* n_long, int32_t* long_at, float* __restrict__ piece,
                                                               int32_t chunks, int32_t slabs) {
    constexpr int AT_ONCE = ACC ? 4 : 8;         // rows asked for before the ones before them are added
    const int64_t unit = (int64_t)blockIdx.x * (ADD_THREADS / WAVE) + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int lane = lane_id();
    const int64_t adders = (int64_t)chunks * slabs;
    if (unit >= adders) {                        // rows without a token
        const int64_t v0 = (unit - adders) * FILL_ROWS;
        if (ACC || v0 >= a.vocab) return;
        // eight lanes look for each row's id among the sorted ones, eight places at a time
        const int sub = lane % FILL_LANES;
        const uint32_t id = (uint32_t)(v0 + lane / FILL_LANES);
        int32_t lo = 0, hi = a.n_tokens;         // the first entry that is not below it lies in [lo, hi]
        while (__ballot(lo < hi)) {
            const int32_t step = (hi - lo + FILL_LANES) / (FILL_LANES + 1);
            const int32_t at = lo + (sub + 1) * step - 1;
            const bool below = at < hi && skey[at] < id;
            const int n = __popc((uint32_t)(__ballot(below) >> (lane - sub)) & ((1u << FILL_LANES) - 1));
            if (lo < hi) {
                const int32_t next = lo + n * step;
                hi = n < FILL_LANES ? min(hi, next + step - 1) : hi;
                lo = next;
            }
        }
        const uint64_t there = __ballot(lo < a.n_tokens && skey[min(lo, a.n_tokens - 1)] == id);
        const float zero[8] = {};
        for (int r = 0; r < FILL_ROWS && v0 + r < a.vocab; ++r) {
            if ((there >> (r * FILL_LANES)) & 1) continue;
            W* row = static_cast<W*>(a.dw) + (v0 + r) * a.dw_stride;
            for (int32_t s = 0; s < slabs; ++s) store8<VEC>(row, s, a.dim, zero);
        }
        return;
    }
    const int32_t chunk = (int32_t)((uint64_t)unit / (uint32_t)slabs), slab = (int32_t)(unit - (int64_t)chunk * slabs);
    const int32_t c0 = chunk * CHUNK;
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
    if (!valid1) return;
    const int n_valid = 64 - __builtin_clzll(valid1);                      // valid entries come first

    // entries [from, to) are this wave's; a bit of `end1` / `end2` where one is the last of its segment
    int from, to = n_valid;
    bool lead_long = false, tail_long = false;
    const int first_start = start1 ? __builtin_ctzll(start1) : CHUNK;
    if (first_start > 0) {                       // a segment reaches into the chunk: another chunk's, unless it is long,
        const int r = min(first_start, n_valid); // that is, has CHUNK entries before its last one here
        lead_long = r == CHUNK || __builtin_amdgcn_readlane(k0, (r - 1) & 63) == __builtin_amdgcn_readfirstlane(k1);
    }
    from = lead_long ? 0 : first_start;
    if (first_start < n_valid && n_valid == CHUNK) {                       // the last segment may go on behind the chunk
        const int s = 63 - __builtin_clzll(start1);
        tail_long = __builtin_amdgcn_readlane(k2, s) == __builtin_amdgcn_readlane(k1, s);      // entry s + CHUNK
        if (!tail_long) to = CHUNK + (start2 ? __builtin_ctzll(start2) : 0);
    }
    if (from >= to) return;
    uint64_t end1 = start1 >> 1, end2 = 0;
    if (to <= CHUNK) end1 |= 1ull << (to - 1); else end2 = 1ull << (to - 1 - CHUNK);

    const G* grad = static_cast<const G*>(a.g);
    const auto entry_pos = [&](int e) { return e < WAVE ? __builtin_amdgcn_readlane(p1, e) : __builtin_amdgcn_readlane(p2, e - WAVE); };
    const auto entry_id = [&](int e) { return (uint32_t)(e < WAVE ? __builtin_amdgcn_readlane(k1, e) : __builtin_amdgcn_readlane(k2, e - WAVE)); };
    Raw8<G> next[AT_ONCE];
    Raw8<W> next_old[ACC ? AT_ONCE : 1];
    const auto ask = [&](int i) {
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int e = min(i + j, to - 1);
            load8<VEC>(grad + (int64_t)entry_pos(e) * a.g_stride, slab, a.dim, next[j]);
            // (all of a segment's entries ask for its row, the last one's answer is used: the others come out of the cache)
            if constexpr (ACC) load8<VEC>(static_cast<const W*>(a.dw) + (int64_t)entry_id(e) * a.dw_stride, slab, a.dim, next_old[j]);
        }
    };
    float sum[8] = {};
    ask(from);
    for (int i = from; i < to; i += AT_ONCE) {
        Raw8<G> now[AT_ONCE];
        Raw8<W> old[ACC ? AT_ONCE : 1];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            now[j] = next[j];
            if constexpr (ACC) old[j] = next_old[j];
        }
        if (i + AT_ONCE < to) ask(i + AT_ONCE);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int e = i + j;
            if (e < to) {
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] += (float)now[j].e[c];
                if ((e < CHUNK ? end1 >> e : end2 >> (e - CHUNK)) & 1) {
                    const bool lead = lead_long && e < first_start, tail = tail_long && e == CHUNK - 1 && !lead;
                    if (lead || tail) {
                        store8<VEC>(piece + ((int64_t)chunk * 2 + tail) * a.dim, slab, a.dim, sum);
                        if (tail && slab == 0 && lane == 0) long_at[atomicAdd(n_long, 1)] = chunk;
                    } else {
                        write_row<VEC, ACC, W>(a, entry_id(e), slab, sum, old[ACC ? j : 0]);
                    }
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum[c] = 0.0f;
                }
            }
        }
    }
}

// One workgroup per long segment and 512 columns, round and round; its waves take every fourth piece each.
template <bool VEC, bool ACC, typename W>
__global__ __launch_bounds__(JOIN_THREADS) void join_pieces_kernel(const EmbeddingGradArgs a, const uint32_t* __restrict__ skey,
                                                                   const int32_t* __restrict__ n_long, const int32_t* __restrict__ long_at,
                                                                   const float* __restrict__ piece, int32_t chunks, int32_t slabs) {
    constexpr int WAVES = JOIN_THREADS / WAVE, AT_ONCE = 4;
    __shared__ float part[WAVES][8][WAVE];
    const int lane = lane_id(), wave = threadIdx.x / WAVE;
    const int64_t units = (int64_t)*n_long * slabs;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int32_t c0 = long_at[u / slabs], slab = (int32_t)(u % slabs);
        const uint32_t id = skey[(int64_t)c0 * CHUNK + CHUNK - 1];
        // the last chunk whose first entry is of this segment: 64 looks at a time
        int32_t lo = c0, hi = chunks;            // (lo is in it, hi is not)
        while (hi - lo > 1) {
            const int32_t step = (hi - lo + WAVE - 1) / WAVE;
            const int64_t at = lo + (int64_t)(lane + 1) * step;
            const uint64_t in = __ballot(at < hi && skey[at * CHUNK] == id);
            lo += __popcll(in) * step;
            hi = min(hi, lo + step);
        }
        Raw8<W> old;
        if constexpr (ACC) load8<VEC>(static_cast<const W*>(a.dw) + (int64_t)id * a.dw_stride, slab, a.dim, old);
        float sum[8] = {};
        for (int64_t c = (int64_t)c0 + wave; c <= lo; c += WAVES * AT_ONCE) {
            Raw8<float> f[AT_ONCE];
#pragma unroll
            for (int q = 0; q < AT_ONCE; ++q) {
                const int64_t at = min(c + q * WAVES, (int64_t)lo);
                load8<VEC>(piece + (at * 2 + (at == c0)) * a.dim, slab, a.dim, f[q]);
            }
#pragma unroll
            for (int q = 0; q < AT_ONCE; ++q)
                if (c + q * WAVES <= lo)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] += f[q].e[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) part[wave][j][lane] = sum[j];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                for (int w = 1; w < WAVES; ++w) sum[j] += part[w][j][lane];
            write_row<VEC, ACC, W>(a, id, slab, sum, old);
        }
        __syncthreads();
    }
}

hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, int32_t g_type, int32_t dw_type, void* d_ws, hipStream_t st) {
    if (a.vocab == 0 || a.dim == 0 || (a.n_tokens == 0 && a.accumulate)) return hipSuccess;
    EmbGradWs w = carve_emb_grad(d_ws, a.n_tokens, a.dim);
    const int64_t portions = a.n_tokens > 0 ? ((int64_t)a.n_tokens + PORTION - 1) / PORTION : 1;
    int bits = 1;
    while ((1 << bits) <= a.vocab) ++bits;       // ids up to and with `vocab`
    const int passes = (bits + 7) / 8, digit_bits = (bits + passes - 1) / passes;
    sort_portions_kernel<<<(unsigned)portions, SORT_THREADS, 0, st>>>(a, w, digit_bits, passes);
    int at = 0;
    for (int64_t run = PORTION; run < a.n_tokens; run *= MERGE_WAYS) {
        merge_runs_kernel<<<(unsigned)((a.n_tokens + MERGE_ENTRIES - 1) / MERGE_ENTRIES), MERGE_THREADS, 0, st>>>(
            a, w.key[at], w.pos[at], w.key[at ^ 1], w.pos[at ^ 1], (int32_t)run);
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
            const auto go = [&](auto v, auto acc) {
                constexpr bool VEC = decltype(v)::value, ACC = decltype(acc)::value;
                add_rows_kernel<VEC, ACC, G, W><<<(unsigned)blocks, ADD_THREADS, 0, st>>>(
                    a, w.key[at], w.pos[at], w.n_long, w.long_at, w.piece, (int32_t)chunks, (int32_t)slabs);
                if (a.n_tokens > CHUNK) {
                    const int64_t most = (int64_t)a.n_tokens / (CHUNK + 1) * slabs;      // long segments there can be
                    join_pieces_kernel<VEC, ACC, W><<<(unsigned)(most < 1024 ? most : 1024), JOIN_THREADS, 0, st>>>(
                        a, w.key[at], w.n_long, w.long_at, w.piece, (int32_t)chunks, (int32_t)slabs);
                }
            };
            if (vec && a.accumulate) go(std::true_type{}, std::true_type{});
            else if (vec) go(std::true_type{}, std::false_type{});
            else if (a.accumulate) go(std::false_type{}, std::true_type{});
            else go(std::false_type{}, std::false_type{});
            return hipGetLastError();
        });
    });
}

}  // namespace dc
