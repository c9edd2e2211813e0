// Operands of the head laid out for the product on the matrix cores.
#include <algorithm>
#include "head_rows.h"

namespace dc {

static bool readable(const dc_matrix& m, bool listed) {
    if (m.type == DC_F32 || m.n_cols % PK != 0 || reinterpret_cast<uintptr_t>(m.d_data) % 16 != 0) return false;
    const int64_t pitch = m.row_stride * 2;
    return pitch % 16 == 0 && pitch <= P_MOST_PITCH && (!listed || pitch * m.n_rows < 1LL << 32);
}

// A round of tiles takes, in us, about 1.4 a step and 14 around them with Q = 8, 0.85 and 5 with Q = 4, and a split's sums 0.6 a MB.
// Measured, the two sides, us: 1000 x 32000, 16 steps, Q = 8 66, Q = 4 73; 2048 x 32000, 32 steps 207, 245; 300 x 32003, 8 steps
// 31.7, 27.5; 100 x 152064, 32 steps 176, 144; 4096 x 10000, 8 steps 57, 52; 500 x 32000, 48 steps 111, 125.
ProductCut cut_product(int64_t m, int64_t n, int64_t steps, int32_t most_splits) {
    ProductCut best = {false, 1};
    double least = -1;
    for (const bool small : {false, true}) {
        const int64_t side = small ? P_SIDE<4> : P_SIDE<8>, slots = small ? P_SLOTS<4> : P_SLOTS<8>;
        const int64_t tiles = whole(m, side) / side * (whole(n, side) / side);
        for (int32_t s = 1; s <= most_splits && (s == 1 || tiles * s <= 2 * slots); ++s) {
            const double round = (double)((steps + s - 1) / s) * (small ? 0.85 : 1.4) + (small ? 5 : 14);
            const double all = (double)((tiles * s + slots - 1) / slots) * round + (s - 1) * (double)m * n * 2.5e-6;
            if (least < 0 || all < least) { least = all; best = ProductCut{small, s}; }
        }
    }
    return best;
}

HeadShape head_shape(const dc_matrix& hidden, const dc_matrix& weight, bool listed) {
    return HeadShape{whole(hidden.n_rows, P_MOST_SIDE), (int32_t)whole(hidden.n_cols, PK), !readable(hidden, listed), !readable(weight, false)};
}

// A thread takes eight neighbouring columns.  Bound by the bytes; sources of any alignment are read an element at a time.
template <typename S, typename D, int PARTS>
__global__ __launch_bounds__(256) void lay_rows_kernel(const S* src, int64_t stride, int64_t first, int64_t n, int32_t cols,
                                                       const int32_t* list, const int32_t* count, int32_t k_pad, char* dst, int64_t plane,
                                                       const int32_t* row_exp, const int32_t* all_exp) {
    const int64_t rows = count ? *count : n;
    const int32_t each = k_pad / 8;
    for (int64_t q = blockIdx.x * 256LL + threadIdx.x; q < rows * each; q += gridDim.x * 256LL) {
        const int64_t r = q / each;
        const int32_t c = (int32_t)(q - r * each) * 8;
        const S* from = src + (list ? list[r] : first + r) * stride + c;
        float f[8];
        if (reinterpret_cast<uintptr_t>(from) % 16 == 0 && c + 8 <= cols) {
            Raw8<S> in;
#pragma unroll
            for (int h = 0; h < (int)sizeof(S) / 2; ++h) in.q[h] = reinterpret_cast<const u32x4*>(from)[h];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = (float)in.e[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = c + j < cols ? (float)from[j] : 0.0f;
        }
        if constexpr (PARTS == 2) {
            const int up = 15 - (row_exp ? row_exp[r] : *all_exp);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = ldexpf(f[j], up);
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            Raw8<D> out;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (PARTS == 1) out.e[j] = (D)f[j];
                else out.e[j] = take_part<D>(f[j]);
            }
            *reinterpret_cast<u32x4*>(dst + p * plane + (r * k_pad + c) * 2) = out.q[0];
        }
    }
}

hipError_t launch_lay_rows(const dc_matrix& src, int64_t first, int64_t n, const int32_t* list, const int32_t* count, int32_t k_pad,
                           char* dst, int64_t plane, Apart apart, const int32_t* row_exp, const int32_t* all_exp, hipStream_t st) {
    const int64_t blocks = std::min<int64_t>((n * (k_pad / 8) + 255) / 256, 8192);
    if (blocks == 0) return hipSuccess;
    const auto go = [&](auto s, auto d, auto parts) {
        using S = decltype(s);
        lay_rows_kernel<S, decltype(d), decltype(parts)::value><<<(unsigned)blocks, 256, 0, st>>>(
            static_cast<const S*>(src.d_data), src.row_stride, first, n, (int32_t)src.n_cols, list, count, k_pad, dst, plane, row_exp, all_exp);
    };
    if (src.type == DC_F32 && apart == F16S) go(float{}, _Float16{}, std::integral_constant<int, 2>{});
    else if (src.type == DC_F32) go(float{}, __bf16{}, std::integral_constant<int, 3>{});
    else if (src.type == DC_BF16) go(__bf16{}, __bf16{}, std::integral_constant<int, 1>{});
    else go(_Float16{}, _Float16{}, std::integral_constant<int, 1>{});
    return hipGetLastError();
}

// ---- powers of two ----

__device__ __forceinline__ void write_first(const FirstExponents& x) {
    for (int32_t i = threadIdx.x; i < x.n; i += blockDim.x) x.top[i] = i > 0 && x.exact ? 15 : NO_EXPONENT;
}
__global__ __launch_bounds__(256) void first_exponents_kernel(const FirstExponents x) { write_first(x); }
hipError_t launch_first_exponents(const FirstExponents& x, hipStream_t st) {
    first_exponents_kernel<<<1, 256, 0, st>>>(x);
    return hipGetLastError();
}

// A wave per row.
__global__ __launch_bounds__(256) void row_exponents_kernel(const float* x, int64_t stride, int64_t n, int32_t cols, const int32_t* list,
                                                            const int32_t* count, int32_t* out) {
    const int64_t rows = count ? *count : n;
    for (int64_t r = blockIdx.x * 4LL + threadIdx.x / WAVE; r < rows; r += gridDim.x * 4LL) {
        const uint32_t big = wave_top(row_top(x + (list ? list[r] : r) * stride, cols));
        if (lane_id() == 0) out[r] = exponent_above(__uint_as_float(big));
    }
}
hipError_t launch_row_exponents(const dc_matrix& src, int64_t n, const int32_t* list, const int32_t* count, int32_t* out, hipStream_t st) {
    row_exponents_kernel<<<(unsigned)std::min<int64_t>((n + 3) / 4, 1 << 14), 256, 0, st>>>(static_cast<const float*>(src.d_data), src.row_stride, n,
                                                                                           (int32_t)src.n_cols, list, count, out);
    return hipGetLastError();
}

template <typename T>
__global__ __launch_bounds__(256) void top_exponent_kernel(const T* w, int64_t stride, int64_t rows, int32_t cols, int32_t last_cols, int32_t* top) {
    __shared__ int tmp[4];
    uint32_t big = 0;
    for (int64_t r = blockIdx.x * 4LL + threadIdx.x / WAVE; r < rows; r += gridDim.x * 4LL) big = max(big, row_top(w + r * stride, r + 1 < rows ? cols : last_cols));
    raise_top(exponent_above(__uint_as_float(wave_top(big))), tmp, top);
}
hipError_t launch_top_exponent(const dc_matrix& src, int64_t first, int64_t n, int32_t* top, hipStream_t st) {
    // (rows that follow each other directly: as pieces of 8192 elements, the last one shorter)
    const bool together = src.row_stride == src.n_cols;
    const int64_t all = n * src.n_cols, rows = together ? (all + 8191) / 8192 : n, stride = together ? 8192 : src.row_stride;
    const int32_t cols = together ? 8192 : (int32_t)src.n_cols, last = together ? (int32_t)(all - (rows - 1) * 8192) : cols;
    const auto launch = [&](auto el) {
        using T = decltype(el);
        const T* from = static_cast<const T*>(src.d_data) + first * src.row_stride;
        top_exponent_kernel<T><<<(unsigned)std::min<int64_t>(TOP_BLOCKS, (rows + 3) / 4), 256, 0, st>>>(from, stride, rows, cols, last, top);
    };
    if (src.type == DC_F32) launch(float{}); else launch(__bf16{});
    return hipGetLastError();
}

// Tiles of 64 x 64 through the LDS: read along the rows, written along the columns.  WIDE: rows on multiples of 16 bytes.  Bound by the
// bytes: 15360 x 2048 bf16 (126 MB in and out) in 19 us.
template <typename S, int PARTS, bool WIDE>
__global__ __launch_bounds__(256) void lay_columns_kernel(const S* src, int64_t stride, int64_t first, int64_t n, int32_t cols,
                                                          const int32_t* list, const int32_t* count, int64_t rows_pad, const int32_t* top,
                                                          const RowTerm* term, char* dst, int64_t plane) {
    __shared__ __attribute__((aligned(16))) float tile[64][68];
    const int64_t rows = count ? *count : n, r0 = blockIdx.x * 64LL;
    if (r0 >= rows) return;
    const int32_t c0 = blockIdx.y * 64, tid = threadIdx.x;
    const int up = 15 - *top;
    if (WIDE && c0 + 64 <= cols) {
        constexpr int N = 16 / sizeof(S), LANES = 64 / N, ROWS = 256 / LANES;
        u32x4 q[64 / ROWS];
#pragma unroll
        for (int h = 0; h < 64 / ROWS; ++h) {
            const int64_t r = min(r0 + tid / LANES + h * ROWS, rows - 1);
            q[h] = *reinterpret_cast<const u32x4*>(src + (list ? list[r] : first + r) * stride + c0 + tid % LANES * N);
        }
#pragma unroll
        for (int h = 0; h < 64 / ROWS; ++h) {
            const int i = tid / LANES + h * ROWS;
            const int64_t r = r0 + i;
            const int x = up - (term && r < rows ? term[r].exponent : 0);
            union { u32x4 q; S e[N]; } in = {q[h]};
#pragma unroll
            for (int j = 0; j < N; ++j) tile[i][tid % LANES * N + j] = r < rows ? ldexpf((float)in.e[j], x) : 0.0f;
        }
    } else {
        const int32_t c = c0 + (tid & 63);
        S in[16];
#pragma unroll
        for (int h = 0; h < 16; ++h) {
            const int64_t r = min(r0 + tid / 64 + 4 * h, rows - 1);
            in[h] = src[(list ? list[r] : first + r) * stride + min(c, cols - 1)];
        }
#pragma unroll
        for (int h = 0; h < 16; ++h) {
            const int64_t r = r0 + tid / 64 + 4 * h;
            tile[tid / 64 + 4 * h][tid & 63] = r < rows && c < cols ? ldexpf((float)in[h], up - (term ? term[r].exponent : 0)) : 0.0f;
        }
    }
    __syncthreads();
    const int32_t c = tid / 4;
    if (c0 + c >= cols) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int32_t i = tid % 4 * 8 + h * 32;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = tile[i + j][c];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            Raw8<_Float16> out;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (PARTS == 1) out.e[j] = (_Float16)f[j];
                else out.e[j] = take_part<_Float16>(f[j]);
            }
            *reinterpret_cast<u32x4*>(dst + p * plane + ((c0 + c) * rows_pad + r0 + i) * 2) = out.q[0];
        }
    }
}

hipError_t launch_lay_columns(const dc_matrix& src, int64_t first, int64_t n, const int32_t* list, const int32_t* count, int64_t rows_pad,
                              const int32_t* top, const RowTerm* term, char* dst, int64_t plane, hipStream_t st) {
    if (n == 0) return hipSuccess;
    const dim3 grid((unsigned)((n + 63) / 64), (unsigned)((src.n_cols + 63) / 64));
    return with_type(src.type, [&](auto el) {
        using S = typename decltype(el)::type;
        const auto launch = [&](auto wide) {
            lay_columns_kernel<S, sizeof(S) == 4 ? 2 : 1, decltype(wide)::value><<<grid, 256, 0, st>>>(
                static_cast<const S*>(src.d_data), src.row_stride, first, n, (int32_t)src.n_cols, list, count, rows_pad, top, term, dst, plane);
        };
        if (rows_aligned<S>(src.d_data, src.row_stride)) launch(std::true_type{}); else launch(std::false_type{});
        return hipGetLastError();
    });
}

// One workgroup, eight neighbouring rows to a thread: a chain of scans, 8192 rows each, and as many trips to memory (8192 rows: 8 us;
// more rows have products that take a hundred times as long).
constexpr int LIVE_THREADS = 1024, LIVE_EACH = 8;
__global__ __launch_bounds__(LIVE_THREADS) void live_rows_kernel(const uint8_t* mask, const float* a, const float* b, int64_t n, LiveRows l,
                                                                 const FirstExponents x) {
    __shared__ int32_t tmp[LIVE_THREADS / WAVE];
    write_first(x);
    int32_t before = 0;
    for (int64_t r0 = 0; r0 < n; r0 += LIVE_THREADS * LIVE_EACH) {
        const int64_t r = r0 + threadIdx.x * LIVE_EACH;
        uint32_t live = 0;
#pragma unroll
        for (int e = 0; e < LIVE_EACH; ++e) {
            bool is = r + e < n && (!mask || mask[r + e] != 0);
            if (is && a) is = a[r + e] != 0.0f || (b && b[r + e] != 0.0f);
            live |= (uint32_t)is << e;
        }
        int32_t total;
        int32_t at = before + block_excl_scan_add((int32_t)__popc(live), tmp, &total);
#pragma unroll
        for (int e = 0; e < LIVE_EACH; ++e) {
            if (r + e >= n) break;
            const bool is = live >> e & 1;
            l.pos[r + e] = is ? at : -1;
            if (is) l.list[at++] = (int32_t)(r + e);
        }
        before += total;
    }
    if (threadIdx.x == 0) *l.count = before;
}
hipError_t launch_live_rows(const uint8_t* mask, const float* a, const float* b, int64_t n, const LiveRows& l, const FirstExponents& x, hipStream_t st) {
    live_rows_kernel<<<1, LIVE_THREADS, 0, st>>>(mask, a, b, n, l, x);
    return hipGetLastError();
}

Parts parts_of(int32_t type, int64_t a_plane, int64_t b_plane) {
    if (type != DC_F32) return Parts{1, 0, 0, a_plane, b_plane};
    return Parts{3, 0u | 1u << 2 | 0u << 4, 1u | 0u << 2 | 0u << 4, a_plane, b_plane};       // the small ones first
}

}  // namespace dc
