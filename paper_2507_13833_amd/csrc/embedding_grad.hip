// Gradient of an embedding table: dW[v, :] = scale * sum of g[t, :] over the tokens t with id v.
//
// Few tokens: one launch (few_tokens).  Otherwise the tokens are sorted by id (stable, so the tokens of one id stay in
// ascending order), and the sorted sequence is cut into chunks of CHUNK entries, so that a hot id's rows are summed by many
// waves; no float goes through an atomic.  131 072 tokens of 2048 columns, bf16 added to f32, ids as text has them / all the
// same: 364 / 271 us; a table of 152 064 rows written anew 373 / 462 (one id's 4096 pieces are joined by four workgroups, one per
// 512 columns, and then all rows but one are without a token).
//   sort_portions   1024 to 8192 tokens per workgroup, radix sort in the LDS
//   merge_runs      up to MERGE_WAYS sorted runs into one: an entry's place is its own plus, for every other run, how many
//                   entries there come before it (a binary search each); once for every factor of MERGE_WAYS
//   add_rows        one wave per chunk and 512 columns: sums the rows of the segments (entries of one id) that start in the
//                   chunk, each in ascending token order, and writes them.  A segment of more than CHUNK entries is
//                   summed in pieces, one per chunk that it touches, into workspace memory
//   join_pieces     the pieces of the long segments, in ascending order
// The rows without a token, most of a large table, are written beside other work that leaves the memory idle: sort_portions
// has workgroups for as many as fit into its time (they look through all tokens), add_rows and join_pieces have them for the
// others (they search the sorted ids).
#include <algorithm>
#include "actor_device.h"

namespace dc {

constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / WAVE;
constexpr int MAX_PORTION = 8192, PER_THREAD = MAX_PORTION / SORT_THREADS;
constexpr int MERGE_WAYS = 32, MERGE_THREADS = 512, MERGE_SAMPLES = 64;
constexpr int ADD_THREADS = 256;
constexpr int FILL_ROWS = 4, FILL_LANES = WAVE / FILL_ROWS;      // rows of the table per wave that looks for those without a token
constexpr int FILL_GROUPS = 240, FILL_MOST = 4096;               // workgroups that write rows before the sort is done, rows of each
constexpr int JOIN_THREADS = 512;

static inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

struct EmbGradWs {
    uint32_t* key[2];                            // ids, sorted; an entry without a token has the id `vocab`
    int32_t*  pos[2];                            // the tokens' places
    int32_t*  n_long;                            // long segments, and the chunks that they start in
    int32_t*  long_at;
    float*    piece;                             // [2 * n_chunks][dim]: of the segment that reaches into the chunk, of the one that leaves it
    size_t    bytes;
};
// Entries of a chunk: fewer where there would be too few waves to hide the loads' latency.
constexpr int64_t FEW_WAVES = 32768 * 4;
static int chunk_of(int64_t n_tokens, int64_t dim) { return n_tokens * ((dim + COLS - 1) / COLS) < FEW_WAVES ? 16 : 32; }
static EmbGradWs carve_emb_grad(void* base, int64_t n_tokens, int64_t dim) {
    const int64_t CHUNK = chunk_of(n_tokens, dim);
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
size_t embedding_grad_workspace_need(int64_t n_tokens, int64_t dim) { return carve_emb_grad(nullptr, n_tokens, dim).bytes; }
// As much as any call of at most these tokens and columns needs.  Chunks of either size need no more for fewer of both; but the
// short ones, of calls below the border, may need more than the long ones of this call: for each number of slabs as wide a row
// and as many tokens as still have them.
size_t embedding_grad_workspace_bytes(int64_t n_tokens, int64_t dim) {
    size_t most = embedding_grad_workspace_need(n_tokens, dim);
    for (int64_t slabs = 1; (slabs - 1) * COLS < dim; ++slabs)
        most = std::max(most, embedding_grad_workspace_need(std::min(n_tokens, (FEW_WAVES - 1) / slabs), std::min<int64_t>(dim, slabs * COLS)));
    return most;
}

// +0 to a row of the table.  Every lane of the wave comes here.
__device__ __forceinline__ void zero_row(const EmbeddingGradArgs& a, int64_t v) {
    char* row = static_cast<char*>(a.dw) + v * a.dw_stride * a.dw_bytes;
    const int64_t bytes = a.dim * a.dw_bytes, whole = a.dw_aligned ? bytes & ~15LL : 0;
    // (two loops: in one the compiler makes the two stores a plain one)
    if (a.dw_stream)
        for (int64_t o = lane_id() * 16; o < whole; o += WAVE * 16) store16(reinterpret_cast<u32x4*>(row + o), u32x4{0, 0, 0, 0});
    else
        for (int64_t o = lane_id() * 16; o < whole; o += WAVE * 16) *reinterpret_cast<u32x4*>(row + o) = u32x4{0, 0, 0, 0};
    if (a.dw_bytes == 4)
        for (int64_t o = whole + lane_id() * 4; o < bytes; o += WAVE * 4) *reinterpret_cast<uint32_t*>(row + o) = 0;
    else
        for (int64_t o = whole + lane_id() * 2; o < bytes; o += WAVE * 2) *reinterpret_cast<uint16_t*>(row + o) = 0;
}
// A workgroup's rows [v0, v0 + rows) that no token names, rows at most FILL_MOST: a bit in the LDS for each, set by a look at
// all tokens (out of the L2, 16 bytes to a thread eight times over).
typedef int32_t i32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));
template <int THREADS>
__device__ __forceinline__ void fill_unnamed(const EmbeddingGradArgs& a, int64_t v0, int32_t rows, uint32_t* bits) {
    constexpr int AT_ONCE = 8;
    for (int i = threadIdx.x; i < FILL_MOST / 32; i += THREADS) bits[i] = 0;
    __syncthreads();
    const auto name = [&](int32_t id) {
        const uint32_t r = (uint32_t)id - (uint32_t)v0;
        if (r < (uint32_t)rows && ((bits[r / 32] >> (r % 32)) & 1) == 0) atomicOr(&bits[r / 32], 1u << (r % 32));
    };
    const i32x4_by4* four = reinterpret_cast<const i32x4_by4*>(a.token);
    const int32_t fours = a.n_tokens / 4;
    for (int32_t i = threadIdx.x; i < fours; i += AT_ONCE * THREADS) {
        i32x4_by4 q[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) q[j] = four[min(i + j * THREADS, fours - 1)];        // (the last ones again: set twice)
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) name(q[j][c]);
    }
    if ((int32_t)threadIdx.x < a.n_tokens - fours * 4) name(a.token[fours * 4 + threadIdx.x]);
    __syncthreads();
    const int32_t each = (rows + THREADS / WAVE - 1) / (THREADS / WAVE), mine = (int32_t)(threadIdx.x / WAVE) * each;
    for (int32_t r = mine; r < min(rows, mine + each); ++r)                // (neighbours to a wave)
        if (((bits[r / 32] >> (r % 32)) & 1) == 0) zero_row(a, v0 + r);
}
// Rows [first, first + rows) of the table by `groups` workgroups; `group`: this one.
struct Fill { int64_t first, rows; int32_t groups; };
template <int THREADS>
__device__ __forceinline__ void fill_part(const EmbeddingGradArgs& a, const Fill& f, int32_t group, uint32_t* bits) {
    const int64_t per = (f.rows + f.groups - 1) / f.groups, from = group * per;
    if (from < f.rows) fill_unnamed<THREADS>(a, f.first + from, (int32_t)min(per, f.rows - from), bits);
}

// `per` times SORT_THREADS tokens by id: least significant digit first, `digit_bits` (at most 8) at a time.  A wave ranks 64 entries by
// ballots over the digit's bits; counts are kept per digit and wave, so the order within a digit is that of the tokens.
__global__ __launch_bounds__(SORT_THREADS) void sort_portions_kernel(const EmbeddingGradArgs a, EmbGradWs w, int per_thread, int digit_bits,
                                                                     int passes, Fill fill) {
    __shared__ uint32_t keys[MAX_PORTION];
    __shared__ uint16_t places[MAX_PORTION];
    __shared__ uint16_t counts[256 * SORT_WAVES];
    __shared__ uint32_t tmp[SORT_WAVES];
    const int32_t portions = (int32_t)gridDim.x - fill.groups;
    if ((int32_t)blockIdx.x >= portions) return fill_part<SORT_THREADS>(a, fill, (int32_t)blockIdx.x - portions, keys);
    const int lane = lane_id(), wave = threadIdx.x / WAVE;
    const int32_t portion = per_thread * SORT_THREADS, first = blockIdx.x * portion;
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.n_long = 0;

    uint32_t key[PER_THREAD];
    uint16_t place[PER_THREAD];
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
        if (j >= per_thread) break;
        const int at = wave * (WAVE * per_thread) + j * WAVE + lane;
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
            if (j >= per_thread) break;
            const uint32_t d = (key[j] >> shift) & (digits - 1);
            uint32_t same_lo = ~0u, same_hi = ~0u;
            for (int b = 0; b < digit_bits; ++b) {
                const uint32_t mine = (uint32_t)((int32_t)(d << (31 - b)) >> 31);        // the bit in every place
                const uint64_t set = __ballot(mine != 0);
                same_lo &= ~((uint32_t)set ^ mine);
                same_hi &= ~((uint32_t)(set >> 32) ^ mine);
            }
            const uint64_t same = (uint64_t)same_hi << 32 | same_lo;
            volatile uint16_t* c = &counts[d * SORT_WAVES + wave];        // this wave's own count
            const uint32_t before = *c;
            __builtin_amdgcn_wave_barrier();
            rank[j] = before + (uint32_t)__popcll(same & below);
            if ((same & below) == 0) *c = (uint16_t)(before + (uint32_t)__popcll(same));
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
                counts[from + i] = (uint16_t)run;
                run += c;
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
            if (j >= per_thread) break;
            const uint32_t d = (key[j] >> shift) & (digits - 1);
            const uint32_t to = counts[d * SORT_WAVES + wave] + rank[j];
            keys[to] = key[j];
            places[to] = place[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
            if (j >= per_thread) break;
            const int at = wave * (WAVE * per_thread) + j * WAVE + lane;
            key[j] = keys[at];
            place[j] = places[at];
        }
        __syncthreads();
    }
    const int32_t n = min(portion, a.n_tokens - first);
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) {
        if (j >= per_thread) break;
        const int at = wave * (WAVE * per_thread) + j * WAVE + lane;
        if (at < n) {
            w.key[0][first + at] = key[j];
            w.pos[0][first + at] = first + place[j];
        }
    }
}

// Runs of `run` sorted entries, MERGE_WAYS neighbouring ones into one.  Four lanes share an entry, each takes every fourth
// run, MERGE_SIDE searches side by side.  The first steps look at MERGE_SAMPLES entries of every run, which the workgroup has
// fetched into the LDS at once.  What bounds it is the instructions of the searches: their number is that of the runs times
// that of the entries, which is why portions are as long as one workgroup sorts well.
constexpr int MERGE_LANES = 4, MERGE_SIDE = 4, MERGE_ENTRIES = MERGE_THREADS / MERGE_LANES;
__global__ __launch_bounds__(MERGE_THREADS) void merge_runs_kernel(const EmbeddingGradArgs a, const uint32_t* __restrict__ key_in,
                                                                   const int32_t* __restrict__ pos_in, uint32_t* __restrict__ key_out,
                                                                   int32_t* __restrict__ pos_out, int32_t run) {
    static_assert(SORT_THREADS % MERGE_SAMPLES == 0 && SORT_THREADS % MERGE_ENTRIES == 0, "a workgroup's entries are of one run");
    static_assert(MERGE_WAYS % (MERGE_LANES * MERGE_SIDE) == 0, "searches side by side");
    __shared__ uint32_t samples[MERGE_WAYS * (MERGE_SAMPLES + 1)];         // (a run's apart from the next one's by a bank)
    const int lane = lane_id(), part = lane / (WAVE / MERGE_LANES);
    const int32_t at = blockIdx.x * MERGE_ENTRIES + (threadIdx.x / WAVE) * (WAVE / MERGE_LANES) + lane % (WAVE / MERGE_LANES);
    const int32_t i = min(at, a.n_tokens - 1);
    const int32_t mine = (int32_t)(blockIdx.x * MERGE_ENTRIES) / run, first = mine / MERGE_WAYS * MERGE_WAYS;
    const int32_t begin = first * run, rest = a.n_tokens - begin;          // the group's entries: [begin, begin + rest) or fewer
    const int ways = (int)min((int64_t)MERGE_WAYS, ((int64_t)rest + run - 1) / run);
    const int32_t window = run / MERGE_SAMPLES;  // a sample is the last entry of its window
    for (int q = threadIdx.x; q < ways * MERGE_SAMPLES; q += MERGE_THREADS) {
        const int64_t from = (int64_t)(q + 1) * window - 1;
        samples[q / MERGE_SAMPLES * (MERGE_SAMPLES + 1) + q % MERGE_SAMPLES] = from < rest ? key_in[begin + from] : 0xFFFFFFFFu;
    }
    const uint32_t key = key_in[i];
    __syncthreads();
    int32_t to = 0;
    for (int j0 = 0; j0 * MERGE_LANES < ways; j0 += MERGE_SIDE) {
        int32_t lo[MERGE_SIDE], len[MERGE_SIDE];
        uint32_t least[MERGE_SIDE];              // entries of an earlier run come first among equals: those below key + 1
#pragma unroll
        for (int j = 0; j < MERGE_SIDE; ++j) {
            const int q = (j0 + j) * MERGE_LANES + part;
            const bool there = q < ways && first + q != mine;
            least[j] = key + (first + q < mine ? 1 : 0);
            const uint32_t* run_samples = samples + (q < ways ? q : 0) * (MERGE_SAMPLES + 1);
            int w = 0;                           // windows that lie before the entry as a whole
#pragma unroll
            for (int step = MERGE_SAMPLES / 2; step > 0; step >>= 1) w += run_samples[w + step - 1] < least[j] ? step : 0;
            w += run_samples[w] < least[j] ? 1 : 0;
            const int64_t from = (int64_t)q * run + (int64_t)w * window, end = min((int64_t)(q + 1) * run, (int64_t)rest);
            lo[j] = there ? (int32_t)min(from, end) : 0;
            len[j] = there ? (int32_t)min((int64_t)window, end - lo[j]) : 0;
            to -= there ? q * run : 0;
        }
        for (int32_t step = window; step > 0; step >>= 1) {
#pragma unroll
            for (int j = 0; j < MERGE_SIDE; ++j) {
                const int32_t half = (len[j] + 1) >> 1;
                const bool less = half > 0 && key_in[begin + lo[j] + (half > 0 ? half - 1 : 0)] < least[j];
                lo[j] += less ? half : 0;
                len[j] = less ? len[j] - half : max(half - 1, 0);
            }
        }
#pragma unroll
        for (int j = 0; j < MERGE_SIDE; ++j) to += lo[j];
    }
#pragma unroll
    for (int d = WAVE / MERGE_LANES; d < WAVE; d <<= 1) to += __shfl_xor(to, d);
    to += begin + (i - mine * run);
    if (at >= a.n_tokens || part != 0) return;
    key_out[to] = key;
    pos_out[to] = pos_in[i];
}

// FILL_ROWS rows of the table by a wave, those without a token: sixteen lanes look for each row's id among the sorted ones,
// sixteen places at a time.
__device__ __forceinline__ void fill_sought(const EmbeddingGradArgs& a, const uint32_t* __restrict__ skey, int64_t v0, int64_t end) {
    const int lane = lane_id(), sub = lane % FILL_LANES;
    const uint32_t id = (uint32_t)(v0 + lane / FILL_LANES);
    int32_t lo = 0, hi = a.n_tokens;             // the first entry that is not below it lies in [lo, hi]
    while (__ballot(lo < hi)) {
        const int32_t step = (hi - lo + FILL_LANES) / (FILL_LANES + 1);
        const int32_t at = lo + (sub + 1) * step - 1;
        const bool below = at >= lo && at < hi && skey[at] < id;           // (a row that is found asks for nothing)
        const int n = __popc((uint32_t)(__ballot(below) >> (lane - sub)) & ((1u << FILL_LANES) - 1));
        if (lo < hi) {
            const int32_t next = lo + n * step;
            hi = n < FILL_LANES ? min(hi, next + step - 1) : hi;
            lo = next;
        }
    }
    const uint64_t there = __ballot(lo < a.n_tokens && skey[min(lo, a.n_tokens - 1)] == id);
    for (int r = 0; r < FILL_ROWS && v0 + r < end; ++r)
        if (((there >> (r * FILL_LANES)) & 1) == 0) zero_row(a, v0 + r);
}

// A finished sum to its row of the table, added to what `old` holds of it.
template <Layout L, bool ACC, typename W>
__device__ __forceinline__ void write_row(const EmbeddingGradArgs& a, uint32_t id, int64_t slab, const float (&sum)[8], const Raw8<W>& old) {
    float out[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = sum[j] * a.scale + (ACC ? (float)old.e[j] : 0.0f);
    store8<L, !ACC>(static_cast<W*>(a.dw) + (int64_t)id * a.dw_stride, slab, a.dim, out);
}

// Few tokens in one launch: a workgroup per token and 512 columns that sums the rows of all tokens of its id, if no earlier
// token has it, and workgroups for FEW_FILL rows each for those without a token.  Every wave compares all ids with its own, a
// ballot per 64; above AT_ONCE rows the waves take equal shares, in ascending order, and join in that order.  Bound by trips to
// memory in a row, four where the sorted way has a dozen in three launches.  Measured, us, gradients in bf16 added to a table in
// f32, this way / sorted: 30 tokens of 512 columns 7.5 / 13.6, 300 of 2048 8.2 / 17, 512 of 2048 10.8 / 15.5, 512 of one id 12.4 /
// 12.6, 1000 of 2048 26 / 19; 300 tokens and a table of 32 000 x 2048 written anew 37 / 50.
constexpr int FEW_TOKENS = 512, FEW_GROUPS = 2048, FEW_THREADS = 512, FEW_FILL = 32;
template <Layout L, bool ACC, typename G, typename W>
__global__ __launch_bounds__(FEW_THREADS) void few_tokens_kernel(const EmbeddingGradArgs a, int32_t slabs, int32_t adders, Fill fill) {
    constexpr int WAVES = FEW_THREADS / WAVE, WORDS = FEW_TOKENS / WAVE, AT_ONCE = 8;
    __shared__ float part[WAVES][8][WAVE];
    __shared__ int32_t place[FEW_TOKENS];
    static_assert(FILL_MOST / 32 <= FEW_TOKENS, "the bits fit as well");
    if ((int32_t)blockIdx.x >= adders)
        return fill_part<FEW_THREADS>(a, fill, (int32_t)blockIdx.x - adders, reinterpret_cast<uint32_t*>(place));
    const int32_t t = (int32_t)blockIdx.x / slabs, slab = (int32_t)blockIdx.x - t * slabs;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    int32_t ids[WORDS];
#pragma unroll
    for (int w = 0; w < WORDS; ++w) ids[w] = w * WAVE < a.n_tokens ? a.token[min(w * WAVE + lane, a.n_tokens - 1)] : DC_NO_TOKEN;
    const int32_t id = a.token[t];
    if (id < 0 || id >= a.vocab) {
        if (id != DC_NO_TOKEN && slab == 0 && threadIdx.x == 0) set_status(a.status, DC_ERR_TOKEN_RANGE);
        return;
    }
    Raw8<W> old;
    if constexpr (ACC) load8<L>(static_cast<const W*>(a.dw) + (int64_t)id * a.dw_stride, slab, a.dim, old);
    const uint64_t below = (1ull << lane) - 1;
    int32_t count = 0, before = 0;               // tokens of this id; those before token t
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        const uint64_t same = __ballot(w * WAVE + lane < a.n_tokens && ids[w] == id);
        if (wave == w % WAVES && (same >> lane) & 1) place[count + __popcll(same & below)] = w * WAVE + lane;
        const int32_t left = t - w * WAVE;
        before += __popcll(left >= WAVE ? same : left > 0 ? same & ((1ull << left) - 1) : 0ull);
        count += __popcll(same);
    }
    if (before > 0) return;
    __syncthreads();
    const int32_t per = max(AT_ONCE, (count + WAVES - 1) / WAVES), from = wave * per, to = min(count, from + per);
    float sum[8] = {};
    for (int32_t k = from; k < to; k += AT_ONCE) {
        Raw8<G> g[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
            load8<L>(static_cast<const G*>(a.g) + (int64_t)__builtin_amdgcn_readfirstlane(place[min(k + j, to - 1)]) * a.g_stride,
                     slab, a.dim, g[j]);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
            if (k + j < to)
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] += (float)g[j].e[c];
    }
    if (count > per) {
#pragma unroll
        for (int c = 0; c < 8; ++c) part[wave][c][lane] = sum[c];
        __syncthreads();
        if (wave == 0)
            for (int w = 1; w * per < count; ++w)
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] += part[w][c][lane];
    }
    if (wave == 0) write_row<L, ACC, W>(a, (uint32_t)id, slab, sum, old);
}

// Bound by the memory: 131 072 rows of 2048 in bf16 in, 58 000 rows in f32 out and 67 000 written as +0 in 0.30 ms of the
// call's 0.37 (5.2 TB/s; a large copy reaches 6.2).
template <int CHUNK, Layout L, bool ACC, typename G, typename W>
__global__ __launch_bounds__(ADD_THREADS) void add_rows_kernel(const EmbeddingGradArgs a, const uint32_t* __restrict__ skey,
                                                               const int32_t* __restrict__ spos,
                                                               int32_t* n_long, int32_t* long_at, float* __restrict__ piece,
                                                               int32_t chunks, int32_t slabs, Fill fill) {
    constexpr int AT_ONCE = ACC ? 4 : 8;         // rows asked for before the ones before them are added
    const int64_t unit = (int64_t)blockIdx.x * (ADD_THREADS / WAVE) + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int lane = lane_id();
    const int64_t adders = (int64_t)chunks * slabs;
    if (unit >= adders) {
        const int64_t v0 = fill.first + (unit - adders) * FILL_ROWS, end = fill.first + fill.rows;
        if (v0 < end) fill_sought(a, skey, v0, end);
        return;
    }
    const int32_t chunk = (int32_t)((uint64_t)unit / (uint32_t)slabs), slab = (int32_t)(unit - (int64_t)chunk * slabs);
    const int32_t c0 = chunk * CHUNK;
    // the chunk's entries and those behind it that a segment of it may reach, and the entries before it
    static_assert(2 * CHUNK <= WAVE, "a lane for every entry");
    constexpr uint32_t NONE = 0xFFFFFFFFu;       // (an id that no entry has)
    constexpr uint64_t IN_CHUNK = (1ull << CHUNK) - 1;
    const uint32_t k1 = c0 + lane < a.n_tokens ? skey[c0 + lane] : NONE;
    const uint32_t k0 = c0 > 0 ? skey[c0 - CHUNK + lane % CHUNK] : NONE;
    const int32_t p1 = c0 + lane < a.n_tokens ? spos[c0 + lane] : 0;
    const uint32_t before = __shfl(k0, CHUNK - 1), up1 = __shfl_up(k1, 1);
    const uint64_t start = __ballot(k1 != (lane ? up1 : before));
    const uint64_t valid = __ballot(k1 < (uint32_t)a.vocab) & IN_CHUNK;
    if (!valid) return;
    const int n_valid = 64 - __builtin_clzll(valid);                       // valid entries come first

    // entries [from, to) are this wave's; a bit of `ends` where one is the last of its segment
    int from, to = n_valid;
    bool lead_long = false, tail_long = false;
    const int first_start = start & IN_CHUNK ? __builtin_ctzll(start) : CHUNK;
    if (first_start > 0) {                       // a segment reaches into the chunk: another chunk's, unless it is long,
        const int r = min(first_start, n_valid); // that is, has CHUNK entries before its last one here
        lead_long = __builtin_amdgcn_readlane(k0, r - 1) == __builtin_amdgcn_readfirstlane(k1);
    }
    from = lead_long ? 0 : first_start;
    if (first_start < n_valid && n_valid == CHUNK) {                       // the last segment may go on behind the chunk
        const int s = 63 - __builtin_clzll(start & IN_CHUNK);
        tail_long = __builtin_amdgcn_readlane(k1, s + CHUNK) == __builtin_amdgcn_readlane(k1, s);
        if (!tail_long) to = __builtin_ctzll(start & ~IN_CHUNK);           // (there is one up to entry s + CHUNK)
    }
    if (from >= to) return;
    const uint64_t ends = start >> 1 | 1ull << (to - 1);

    const G* grad = static_cast<const G*>(a.g);
    const auto entry_pos = [&](int e) { return __builtin_amdgcn_readlane(p1, e); };
    const auto entry_id = [&](int e) { return (uint32_t)__builtin_amdgcn_readlane(k1, e); };
    Raw8<G> next[AT_ONCE];
    Raw8<W> next_old[ACC ? AT_ONCE : 1];
    const auto ask = [&](int i) {
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int e = min(i + j, to - 1);
            load8<L>(grad + (int64_t)entry_pos(e) * a.g_stride, slab, a.dim, next[j]);
            // (all of a segment's entries ask for its row, the last one's answer is used: the others come out of the cache)
            if constexpr (ACC) load8<L>(static_cast<const W*>(a.dw) + (int64_t)entry_id(e) * a.dw_stride, slab, a.dim, next_old[j]);
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
                if ((ends >> e) & 1) {
                    const bool lead = lead_long && e < first_start, tail = tail_long && e == CHUNK - 1 && !lead;
                    if (lead || tail) {
                        store8<L>(piece + ((int64_t)chunk * 2 + tail) * a.dim, slab, a.dim, sum);
                        if (tail && slab == 0 && lane == 0) long_at[atomicAdd(n_long, 1)] = chunk;
                    } else {
                        write_row<L, ACC, W>(a, entry_id(e), slab, sum, old[ACC ? j : 0]);
                    }
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum[c] = 0.0f;
                }
            }
        }
    }
}

// One workgroup per long segment and 512 columns, round and round; its waves take every eighth piece each.
template <int CHUNK, Layout L, bool ACC, typename W>
__global__ __launch_bounds__(JOIN_THREADS) void join_pieces_kernel(const EmbeddingGradArgs a, const uint32_t* __restrict__ skey,
                                                                   const int32_t* __restrict__ n_long, const int32_t* __restrict__ long_at,
                                                                   const float* __restrict__ piece, int32_t chunks, int32_t slabs,
                                                                   int32_t joiners, int64_t fill_from, int64_t fill_end) {
    constexpr int WAVES = JOIN_THREADS / WAVE, AT_ONCE = 8;
    __shared__ float part[WAVES][8][WAVE];
    if ((int32_t)blockIdx.x >= joiners) {
        const int64_t v0 = fill_from + ((int64_t)((int32_t)blockIdx.x - joiners) * WAVES + threadIdx.x / WAVE) * FILL_ROWS;
        if (v0 < fill_end) fill_sought(a, skey, v0, fill_end);
        return;
    }
    const int lane = lane_id(), wave = threadIdx.x / WAVE;
    const int64_t units = (int64_t)*n_long * slabs;
    for (int64_t u = blockIdx.x; u < units; u += joiners) {
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
        if constexpr (ACC) load8<L>(static_cast<const W*>(a.dw) + (int64_t)id * a.dw_stride, slab, a.dim, old);
        float sum[8] = {};
        for (int64_t c = (int64_t)c0 + wave; c <= lo; c += WAVES * AT_ONCE) {
            Raw8<float> f[AT_ONCE];
#pragma unroll
            for (int q = 0; q < AT_ONCE; ++q) {
                const int64_t at = min(c + q * WAVES, (int64_t)lo);
                load8<L>(piece + (at * 2 + (at == c0)) * a.dim, slab, a.dim, f[q]);
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
            write_row<L, ACC, W>(a, id, slab, sum, old);
        }
        __syncthreads();
    }
}

// Bytes of rows without a token that are written beside the sort (which takes longer the more tokens a thread has) and beside
// the join; the rest beside add_rows.  Measured, us, gradients in bf16, a table in f32; all of it beside add_rows / beside the
// sort, 70 MB / 160 MB, no more at the join / 120 MB at the sort (80 MB at the second), 100 MB at the join / everything at
// the sort:
//   131072 tokens, 152064 x 2048   391.9 / 380.2 / 377.6 / 374.5 / 397.2
//   33000 tokens, 152064 x 512      90.6 /  80.4 /  82.3 /  76.8 /  86.3
// From the table's start instead of its end, where most rows have tokens: nothing gained.  Beside the merge as well: 1 % slower
// (its own work takes all compute units).
constexpr double FILL_SORT = 60e6, FILL_SORT_EACH = 8e6, FILL_JOIN = 100e6;
// f(layout, whether to accumulate, element types of the gradient and of the table).  Rows that do not start on 16 bytes or whose
// width is no multiple of 8 go element by element: 131 072 tokens of 2047 columns, a table of 152 064 in f32 written anew, 428 us
// (373 for 2048), 8192 of 1023 added to 32 000 33 us (29).
template <typename F>
static hipError_t with_layout(const EmbeddingGradArgs& a, int32_t g_type, int32_t dw_type, F&& f) {
    return with_type(g_type, [&](auto ge) {
        return with_type(dw_type, [&](auto we) {
            using G = typename decltype(ge)::type;
            using W = typename decltype(we)::type;
            const auto go = [&](auto layout) {
                return a.accumulate ? f(layout, std::true_type{}, ge, we) : f(layout, std::false_type{}, ge, we);
            };
            if (a.dim % 8 == 0 && rows_aligned<G>(a.g, a.g_stride) && rows_aligned<W>(a.dw, a.dw_stride))
                return go(std::integral_constant<Layout, sizeof(W) == 4 ? FOURS : EIGHTS>{});
            return go(std::integral_constant<Layout, APART>{});
        });
    });
}

hipError_t launch_embedding_grad(const EmbeddingGradArgs& args, int32_t g_type, int32_t dw_type, void* d_ws, hipStream_t st) {
    EmbeddingGradArgs a = args;
    a.dw_bytes = dw_type == DC_F32 ? 4 : 2;
    // rows of +0 past the caches where the table is several times the Infinity Cache's 256 MB: 1245 MB 375 us (through the caches
    // 405); through them otherwise: 623 MB 111 us (past them 114), 311 MB 74 (77), 262 MB 37 (48)
    a.dw_stream = (size_t)a.vocab * a.dw_stride * a.dw_bytes > 768u << 20;
    a.dw_aligned = reinterpret_cast<uintptr_t>(a.dw) % 16 == 0 && (size_t)a.dw_stride * a.dw_bytes % 16 == 0;
    if (a.vocab == 0 || a.dim == 0 || (a.n_tokens == 0 && a.accumulate)) return hipSuccess;
    const int64_t slabs = (a.dim + COLS - 1) / COLS;
    if (a.n_tokens <= FEW_TOKENS && a.n_tokens * slabs <= FEW_GROUPS) {
        const int64_t rows = a.accumulate ? 0 : a.vocab, groups = (rows + FEW_FILL - 1) / FEW_FILL;
        const Fill fill = {0, rows, (int32_t)groups};
        const int32_t adders = a.n_tokens * (int32_t)slabs;
        return with_layout(a, g_type, dw_type, [&](auto layout, auto acc, auto ge, auto we) {
            few_tokens_kernel<decltype(layout)::value, decltype(acc)::value, typename decltype(ge)::type, typename decltype(we)::type>
                <<<(unsigned)(adders + groups), FEW_THREADS, 0, st>>>(a, (int32_t)slabs, adders, fill);
            return hipGetLastError();
        });
    }
    EmbGradWs w = carve_emb_grad(d_ws, a.n_tokens, a.dim);
    // short portions keep more workgroups busy, long ones leave the merge fewer runs (one level of it either way up to
    // 2^18 tokens): 8192 tokens sorted and merged
    const int per_thread = a.n_tokens <= SORT_THREADS ? 1 : a.n_tokens <= 16384 ? 2 : a.n_tokens <= 65536 ? 4 : 8;
    const int64_t portion = (int64_t)per_thread * SORT_THREADS;
    const int64_t portions = (a.n_tokens + portion - 1) / portion;
    int bits = 1;
    while ((1 << bits) <= a.vocab) ++bits;       // ids up to and with `vocab`
    const int passes = (bits + 7) / 8, digit_bits = (bits + passes - 1) / passes;
    // rows without a token, from the table's end, where ids are rare
    const double row = (double)a.dim * a.dw_bytes;
    int64_t left = a.accumulate ? 0 : a.vocab;   // rows [0, left) are still to be looked at
    Fill by_sort = {0, 0, 0};
    if (portions + FILL_GROUPS <= 256)           // (a compute unit for each)
        by_sort.rows = std::min({left, (int64_t)((FILL_SORT + FILL_SORT_EACH * per_thread) / row), (int64_t)FILL_GROUPS * FILL_MOST});
    by_sort.first = left -= by_sort.rows;
    by_sort.groups = (int32_t)std::min<int64_t>(by_sort.rows, FILL_GROUPS);
    sort_portions_kernel<<<(unsigned)(portions + by_sort.groups), SORT_THREADS, 0, st>>>(a, w, per_thread, digit_bits, passes, by_sort);
    int at = 0;
    for (int64_t run = portion; run < a.n_tokens; run *= MERGE_WAYS) {
        merge_runs_kernel<<<(unsigned)((a.n_tokens + MERGE_ENTRIES - 1) / MERGE_ENTRIES), MERGE_THREADS, 0, st>>>(
            a, w.key[at], w.pos[at], w.key[at ^ 1], w.pos[at ^ 1], (int32_t)run);
        at ^= 1;
    }
    const int chunk = chunk_of(a.n_tokens, a.dim);
    const int64_t chunks = ((int64_t)a.n_tokens + chunk - 1) / chunk;
    const int64_t by_join = std::min<int64_t>(left, (int64_t)(FILL_JOIN / row));
    const Fill by_add = {0, left - by_join, 0};
    const int64_t units = chunks * slabs + (by_add.rows + FILL_ROWS - 1) / FILL_ROWS;
    const int64_t blocks = (units + ADD_THREADS / WAVE - 1) / (ADD_THREADS / WAVE);
    if (blocks > 0x7FFFFFFFLL) return hipErrorInvalidValue;
    const int64_t per_join = JOIN_THREADS / WAVE * FILL_ROWS, fillers = (by_join + per_join - 1) / per_join;
    return with_layout(a, g_type, dw_type, [&](auto layout, auto acc, auto ge, auto we) {
        using G = typename decltype(ge)::type;
        using W = typename decltype(we)::type;
        constexpr Layout L = decltype(layout)::value;
        constexpr bool ACC = decltype(acc)::value;
        const auto launch = [&](auto c) {
            constexpr int CHUNK = decltype(c)::value;
            add_rows_kernel<CHUNK, L, ACC, G, W><<<(unsigned)blocks, ADD_THREADS, 0, st>>>(
                a, w.key[at], w.pos[at], w.n_long, w.long_at, w.piece, (int32_t)chunks, (int32_t)slabs, by_add);
            const int64_t most = (int64_t)a.n_tokens / (CHUNK + 1) * slabs;              // long segments there can be
            const int32_t joiners = (int32_t)(most < 1024 ? most : 1024);
            join_pieces_kernel<CHUNK, L, ACC, W><<<(unsigned)(joiners + fillers), JOIN_THREADS, 0, st>>>(
                a, w.key[at], w.n_long, w.long_at, w.piece, (int32_t)chunks, (int32_t)slabs, joiners, left - by_join, left);
        };
        if (chunk == 16) launch(std::integral_constant<int, 16>{});
        else launch(std::integral_constant<int, 32>{});
        return hipGetLastError();
    });
}

}  // namespace dc
