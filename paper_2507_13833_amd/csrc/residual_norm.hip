// The residual stream from one block to the next, and its gradient.
//
// A workgroup (a wave, for short rows) takes a row, eight columns to a thread, and holds it in registers from the first sum to the
// last store: each stream is read once and written once.  The factors that all rows share stay in registers from row to row, and so do
// their gradients' sums, which a second launch joins.  Bound by the streams' bytes.
#include <algorithm>
#include "actor_device.h"
#include "head_internal.h"

namespace dc {

constexpr int NORM_WIDEST = 1024 * 8;            // columns that a workgroup's registers hold
constexpr int64_t NORM_GRID = 1024, NORM_PARTS = 512, NORM_WIDE_PARTS = 256;      // workgroups of the gradient: their sums are joined

// E columns of a thread.  WIDE (rows on multiples of 16 bytes and dim a multiple of 8): eight neighbours, and eight more 8 P further on;
// else P apart (16 bytes at a time from wherever they lie: 131072 x 1365 bf16 559 us for 354).
template <int P, bool WIDE>
__device__ __forceinline__ int32_t norm_column(int t, int j) { return WIDE ? j / 8 * (8 * P) + t * 8 + j % 8 : j * P + t; }

template <int P, bool WIDE, int G, typename T>
__device__ __forceinline__ void norm_load(const T* row, int t, int32_t dim, Raw8<T> (&r)[G]) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
        if constexpr (WIDE) {
            const u32x4* p = reinterpret_cast<const u32x4*>(row + min(norm_column<P, WIDE>(t, 8 * g), dim - 8));
#pragma unroll
            for (int h = 0; h < (int)sizeof(T) / 2; ++h) r[g].q[h] = __builtin_nontemporal_load(p + h);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) r[g].e[j] = row[min(norm_column<P, WIDE>(t, 8 * g + j), dim - 1)];
        }
    }
}
// (columns behind the last one: 0)
template <int P, bool WIDE, int G, int E, typename T>
__device__ __forceinline__ void norm_values(const Raw8<T> (&r)[G], int t, int32_t dim, float (&f)[E]) {
#pragma unroll
    for (int j = 0; j < E; ++j) f[j] = norm_column<P, WIDE>(t, j) < dim ? (float)r[j / 8].e[j % 8] : 0.0f;
}
template <int P, bool WIDE, int E, typename T>
__device__ __forceinline__ void norm_store(T* row, int t, int32_t dim, const float (&f)[E]) {
#pragma unroll
    for (int g = 0; g < E / 8; ++g) {
        Raw8<T> r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r.e[j] = (T)f[8 * g + j];
        if constexpr (WIDE) {
            const int32_t c = norm_column<P, WIDE>(t, 8 * g);
            if (c < dim)
#pragma unroll
                for (int h = 0; h < (int)sizeof(T) / 2; ++h) store16(reinterpret_cast<u32x4*>(row + c) + h, r.q[h]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (norm_column<P, WIDE>(t, 8 * g + j) < dim) row[norm_column<P, WIDE>(t, 8 * g + j)] = r.e[j];
        }
    }
}
__device__ __forceinline__ float factor_at(const NormFactor& f, int64_t r, int32_t c) {
    if (!f.p) return 1.0f;
    const int64_t at = r * f.stride + c;
    return f.type == DC_F32 ? static_cast<const float*>(f.p)[at] : f.type == DC_BF16 ? (float)static_cast<const __bf16*>(f.p)[at]
                                                                                     : (float)static_cast<const _Float16*>(f.p)[at];
}
// A thread's factors that all rows share.
template <int P, bool WIDE, int E>
__device__ __forceinline__ void factors_of(const NormFactor& w, int t, int32_t dim, float (&f)[E]) {
#pragma unroll
    for (int j = 0; j < E; ++j) f[j] = factor_at(w, 0, min(norm_column<P, WIDE>(t, j), dim - 1));
}

__device__ __forceinline__ float wave_read_lane_f(float v) { return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v))); }
// Sums over the P threads of a row; `tmp`: N floats per wave, of its own for every call between two barriers.
template <int P, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* tmp) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (P > WAVE) {
        constexpr int WAVES = P / WAVE;
        if (lane_id() == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) tmp[i * WAVES + threadIdx.x / WAVE] = v[i];
        lds_barrier();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = lane_id() < WAVES ? tmp[i * WAVES + lane_id()] : 0.0f;
#pragma unroll
            for (int d = 1; d < WAVES; d <<= 1) v[i] += __shfl_xor(v[i], d);
            v[i] = wave_read_lane_f(v[i]);
        }
    }
}
// 1 / sqrt, rounded twice
__device__ __forceinline__ float inverse_root(float x) { return 1.0f / sqrtf(x); }

// us: 131072 x 2048, block and out bf16, the stream f32 (3.2 GB) 681 (4.7 TB/s; a large copy reaches 4.9); one row 11, mostly
// the host's: the kernel takes 6.
template <typename A, typename R, int P, bool WIDE>
__global__ __launch_bounds__(P < 256 ? 256 : P) void residual_norm_kernel(const NormArgs a) {
    constexpr int THREADS = P < 256 ? 256 : P, ROWS = THREADS / P;
    __shared__ float tmp[2][2][THREADS / WAVE];
    const int t = threadIdx.x % P;
    const int32_t dim = a.dim;
    const bool gate_rows = a.gate.p && a.gate.rows;
    float post[8], gate[8], pre[8];
    factors_of<P, WIDE>(a.post, t, dim, post);
    if (!gate_rows) factors_of<P, WIDE>(a.gate, t, dim, gate);
    factors_of<P, WIDE>(a.pre, t, dim, pre);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (!gate_rows) post[j] *= gate[j];
        post[j] *= a.block_scale;
    }
    const float each = 1.0f / (float)dim;
    int turn = 0;
    Raw8<A> rb[1], rg[1];
    Raw8<R> rr[1];
    const auto ask = [&](int64_t r) {
        norm_load<P, WIDE>(static_cast<const A*>(a.block.p) + r * a.block.stride, t, dim, rb);
        norm_load<P, WIDE>(static_cast<const R*>(a.residual.p) + r * a.residual.stride, t, dim, rr);
        if (gate_rows) norm_load<P, WIDE>(static_cast<const A*>(a.gate.p) + r * a.gate.stride, t, dim, rg);
    };
    const int64_t step = gridDim.x * (int64_t)ROWS;
    int64_t r = blockIdx.x * (int64_t)ROWS + threadIdx.x / P;
    if (r < a.rows) ask(r);
    for (; r < a.rows; r += step, turn ^= 1) {
        float b[8], h[8];
        norm_values<P, WIDE>(rb, t, dim, b);
        norm_values<P, WIDE>(rr, t, dim, h);
        if (gate_rows) norm_values<P, WIDE>(rg, t, dim, gate);
        if (r + step < a.rows) ask(r + step);    // (the next row is on its way while this one is summed and stored)
        float r1 = 0.0f, r2 = 0.0f, s[1] = {0.0f};
        if (a.has_post) {
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] = fmaf(b[j], b[j], s[0]);
            row_sums<P>(s, tmp[turn][0]);
            r1 = inverse_root(fmaf(s[0], each, a.eps));
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] *= r1;
        }
        if (gate_rows)
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] *= gate[j];
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = fmaf(b[j], post[j], h[j] * a.residual_scale);
        norm_store<P, WIDE>(static_cast<R*>(a.residual_out.p) + r * a.residual_out.stride, t, dim, h);
        if (a.has_pre) {
            s[0] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] = fmaf(h[j], h[j], s[0]);
            row_sums<P>(s, tmp[turn][1]);
            r2 = inverse_root(fmaf(s[0], each, a.eps));
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] *= r2 * pre[j];
            norm_store<P, WIDE>(static_cast<A*>(a.out.p) + r * a.out.stride, t, dim, h);
        }
        if (a.stat && t == 0) {
            a.stat[2 * r] = r1;
            a.stat[2 * r + 1] = r2;
        }
    }
}

// Rows longer than a workgroup's registers: read again from the caches for each sum and for the stores, an element at a time, which is
// what bounds it (16384 x 16384 bf16, 2.1 GB: 2766 us, 0.8 TB/s; the gradient, whose sums over rows go through memory, 4747, 0.7).
template <typename A, typename R>
__global__ __launch_bounds__(1024) void residual_norm_wide_kernel(const NormArgs a) {
    __shared__ float tmp[2][16];
    const float each = 1.0f / (float)a.dim;
    const int t = threadIdx.x;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const A* block = static_cast<const A*>(a.block.p) + r * a.block.stride;
        const R* residual = static_cast<const R*>(a.residual.p) + r * a.residual.stride;
        float r1 = 0.0f, r2 = 0.0f, s[1] = {0.0f};
        if (a.has_post) {
            for (int32_t c = t; c < a.dim; c += 1024) s[0] = fmaf((float)block[c], (float)block[c], s[0]);
            row_sums<1024>(s, tmp[0]);
            r1 = inverse_root(fmaf(s[0], each, a.eps));
        }
        const auto h_at = [&](int32_t c) {
            float b = (float)block[c];
            if (a.has_post) b *= r1 * factor_at(a.post, 0, c);
            return fmaf(b * factor_at(a.gate, r, c), a.block_scale, (float)residual[c] * a.residual_scale);
        };
        if (a.has_pre) {
            s[0] = 0.0f;
            for (int32_t c = t; c < a.dim; c += 1024) { const float h = h_at(c); s[0] = fmaf(h, h, s[0]); }
            row_sums<1024>(s, tmp[1]);
            r2 = inverse_root(fmaf(s[0], each, a.eps));
        }
        for (int32_t c = t; c < a.dim; c += 1024) {
            const float h = h_at(c);
            if (a.has_pre) (static_cast<A*>(a.out.p) + r * a.out.stride)[c] = (A)(h * (r2 * factor_at(a.pre, 0, c)));
            (static_cast<R*>(a.residual_out.p) + r * a.residual_out.stride)[c] = (R)h;
        }
        if (a.stat && t == 0) { a.stat[2 * r] = r1; a.stat[2 * r + 1] = r2; }
        __syncthreads();                         // tmp is free again
    }
}

// Threads to a row, eight columns each; short rows share a workgroup.  The longest rows' gradient has half the threads and twice the
// columns: 1024 threads have 128 registers each, of which it would spill 90 (32768 x 8192 bf16: 1641 us for 639, 5.0 TB/s).  Where one of
// the streams has 32 bits 36 to 65 registers are spilled all the same (stream in f32 1094 us, 4.4 TB/s; both 1512, 4.3), and where rows
// are odd, on 1024 threads, 50 to 65 (32768 x 5001 bf16: 1383 us, 1.4 TB/s; stream in f32 3292, 0.9).
template <bool GRAD, typename F>
static hipError_t with_threads(int32_t dim, bool wide, F&& f) {
    using std::integral_constant;
    const auto go = [&](auto p, auto e) { return wide ? f(p, e, std::true_type{}) : f(p, e, std::false_type{}); };
    using Eight = integral_constant<int, 8>;
    if (dim <= 512) return go(integral_constant<int, 64>{}, Eight{});
    if (dim <= 2048) return go(integral_constant<int, 256>{}, Eight{});
    if (dim <= 4096) return go(integral_constant<int, 512>{}, Eight{});
    if constexpr (GRAD)
        return wide ? f(integral_constant<int, 512>{}, integral_constant<int, 16>{}, std::true_type{})
                    : f(integral_constant<int, 1024>{}, Eight{}, std::false_type{});
    else
        return go(integral_constant<int, 1024>{}, Eight{});
}
static bool lies_wide(const NormStream& s, int32_t type) {
    return reinterpret_cast<uintptr_t>(s.p) % 16 == 0 && s.stride * (type == DC_F32 ? 4 : 2) % 16 == 0;
}

hipError_t launch_residual_norm(const NormArgs& a, hipStream_t st) {
    if (a.rows == 0 || a.dim == 0) return hipSuccess;
    const bool wide = a.dim % 8 == 0 && lies_wide(a.block, a.act) && lies_wide(a.residual, a.res) && lies_wide(a.residual_out, a.res) &&
                      lies_wide(a.out, a.act) && (!a.gate.p || !a.gate.rows || lies_wide(NormStream{const_cast<void*>(a.gate.p), a.gate.stride}, a.act));
    return with_type(a.act, [&](auto ea) {
        return with_type(a.res, [&](auto er) {
            using A = typename decltype(ea)::type;
            using R = typename decltype(er)::type;
            if (a.dim > NORM_WIDEST) {
                residual_norm_wide_kernel<A, R><<<(unsigned)std::min<int64_t>(a.rows, 2048), 1024, 0, st>>>(a);
                return hipGetLastError();
            }
            return with_threads<false>(a.dim, wide, [&](auto p, auto, auto w) {
                constexpr int P = decltype(p)::value, THREADS = P < 256 ? 256 : P, ROWS = THREADS / P;
                const unsigned grid = (unsigned)std::min<int64_t>((a.rows + ROWS - 1) / ROWS, NORM_GRID * 256 / THREADS);
                residual_norm_kernel<A, R, P, decltype(w)::value><<<grid, THREADS, 0, st>>>(a);
                return hipGetLastError();
            });
        });
    });
}

// ---- the gradient ----

// One round of sums to a row: with x = dy pre, n2 = h r2, n1 = b r1 (b without a norm), w = gate post n1 (0 without a norm),
//   S1 = sum x n2,  Sa = sum (dh + r2 x) w,  Sb = sum n2 w:  sum dh' w = Sa - r2 S1 Sb / dim for dh' = dh + r2 (x - n2 S1 / dim).
// 131072 x 2048 bf16, all gradients (3.2 GB): 652 us (4.9 TB/s), 12 of them the join's; 777 x 1365 f32 23, two launches and the host.
template <typename A, typename R, int P, int E, bool WIDE>
__global__ __launch_bounds__(P < 256 ? 256 : P) void residual_norm_grad_kernel(const NormGradArgs a) {
    constexpr int THREADS = P < 256 ? 256 : P, ROWS = THREADS / P;
    constexpr bool AHEAD = E == 8 && P < 1024;   // the next row is on its way while one is summed and stored (else: too many registers)
    __shared__ float tmp[2][3][THREADS / WAVE];
    __shared__ float sums[ROWS > 1 ? ROWS * 3 * P * E : 1];
    const int t = threadIdx.x % P;
    const int32_t dim = a.dim;
    const bool gate_rows = a.gate.p && a.gate.rows;
    float post[E], gate[E], pre[E], sum_post[E] = {}, sum_gate[E] = {}, sum_pre[E] = {};
    factors_of<P, WIDE>(a.post, t, dim, post);
    if (!gate_rows) factors_of<P, WIDE>(a.gate, t, dim, gate);
    factors_of<P, WIDE>(a.pre, t, dim, pre);
    const float each = 1.0f / (float)dim;
    int turn = 0;
    Raw8<A> rb[E / 8], rg[E / 8], ry[E / 8];
    Raw8<R> rh[E / 8], rd[E / 8];
    float next1 = 1.0f, next2 = 0.0f;
    const auto ask = [&](int64_t r) {
        norm_load<P, WIDE>(static_cast<const A*>(a.block.p) + r * a.block.stride, t, dim, rb);
        if (a.grad_residual_out.p) norm_load<P, WIDE>(static_cast<const R*>(a.grad_residual_out.p) + r * a.grad_residual_out.stride, t, dim, rd);
        if (a.has_pre) {
            norm_load<P, WIDE>(static_cast<const R*>(a.residual_out.p) + r * a.residual_out.stride, t, dim, rh);
            norm_load<P, WIDE>(static_cast<const A*>(a.grad_out.p) + r * a.grad_out.stride, t, dim, ry);
            next2 = a.stat[2 * r + 1];
        }
        if (gate_rows) norm_load<P, WIDE>(static_cast<const A*>(a.gate.p) + r * a.gate.stride, t, dim, rg);
        if (a.has_post) next1 = a.stat[2 * r];
    };
    const int64_t step = gridDim.x * (int64_t)ROWS;
    int64_t r = blockIdx.x * (int64_t)ROWS + threadIdx.x / P;
    if (AHEAD && r < a.rows) ask(r);
    for (; r < a.rows; r += step, turn ^= 1) {
        if (!AHEAD) ask(r);
        const float r1 = next1, r2 = next2;
        float n1[E], dh[E], n2[E], x[E];
        norm_values<P, WIDE>(rb, t, dim, n1);
        if (a.grad_residual_out.p) norm_values<P, WIDE>(rd, t, dim, dh);
        else
#pragma unroll
            for (int j = 0; j < E; ++j) dh[j] = 0.0f;
        if (gate_rows) norm_values<P, WIDE>(rg, t, dim, gate);
        if (a.has_pre) {
            norm_values<P, WIDE>(rh, t, dim, n2);
            norm_values<P, WIDE>(ry, t, dim, x);
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) n2[j] = x[j] = 0.0f;
        }
        if (AHEAD && r + step < a.rows) ask(r + step);
#pragma unroll
        for (int j = 0; j < E; ++j) n1[j] *= r1;
        if (a.has_pre) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                n2[j] *= r2;
                sum_pre[j] = fmaf(x[j], n2[j], sum_pre[j]);
                x[j] *= pre[j];
                dh[j] = fmaf(r2, x[j], dh[j]);
            }
        }
        float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < E; ++j) {
            s[0] = fmaf(x[j], n2[j], s[0]);
            if (a.has_post) {
                const float w = gate[j] * post[j] * n1[j];
                s[1] = fmaf(dh[j], w, s[1]);
                s[2] = fmaf(n2[j], w, s[2]);
            }
        }
        row_sums<P>(s, tmp[turn][0]);
        const float along2 = r2 * s[0] * each, along1 = a.has_post ? (s[1] - along2 * s[2]) * each * a.block_scale : 0.0f;
        float out[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            dh[j] = fmaf(-along2, n2[j], dh[j]);
            out[j] = dh[j] * a.residual_scale;
        }
        if (a.grad_residual.p) norm_store<P, WIDE>(static_cast<R*>(a.grad_residual.p) + r * a.grad_residual.stride, t, dim, out);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float du = dh[j] * a.block_scale, dg = du * n1[j] * post[j];
            sum_gate[j] += dg;
            out[j] = dg;
            dh[j] = du * gate[j];
            sum_post[j] = fmaf(dh[j], n1[j], sum_post[j]);
        }
        if (a.grad_gate.p) norm_store<P, WIDE>(static_cast<A*>(a.grad_gate.p) + r * a.grad_gate.stride, t, dim, out);
        if (a.grad_block.p) {
#pragma unroll
            for (int j = 0; j < E; ++j) out[j] = r1 * fmaf(-along1, n1[j], dh[j] * post[j]);
            norm_store<P, WIDE>(static_cast<A*>(a.grad_block.p) + r * a.grad_block.stride, t, dim, out);
        }
    }
    float* part = a.part + (int64_t)blockIdx.x * 3 * dim;
    const auto put = [&](int i, const float (&v)[E]) {
        if (!a.sum[i].p) return;
        if constexpr (ROWS == 1) {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (norm_column<P, WIDE>(t, j) < dim) part[(int64_t)i * dim + norm_column<P, WIDE>(t, j)] = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) sums[(threadIdx.x / P * 3 + i) * P * E + norm_column<P, WIDE>(t, j)] = v[j];
        }
    };
    put(0, sum_post);
    put(1, sum_gate);
    put(2, sum_pre);
    if constexpr (ROWS > 1) {
        __syncthreads();
        for (int i = 0; i < 3; ++i)
            if (a.sum[i].p)
                for (int32_t c = threadIdx.x; c < dim; c += THREADS) {
                    float v = 0.0f;
                    for (int w = 0; w < ROWS; ++w) v += sums[(w * 3 + i) * P * E + c];
                    part[(int64_t)i * dim + c] = v;
                }
    }
}

template <typename A, typename R>
__global__ __launch_bounds__(1024) void residual_norm_grad_wide_kernel(const NormGradArgs a) {
    __shared__ float tmp[3][16];
    const float each = 1.0f / (float)a.dim;
    const int t = threadIdx.x;
    float* part = a.part + (int64_t)blockIdx.x * 3 * a.dim;
    bool first = true;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, first = false) {
        const float r1 = a.has_post ? a.stat[2 * r] : 1.0f, r2 = a.has_pre ? a.stat[2 * r + 1] : 0.0f;
        const A* block = static_cast<const A*>(a.block.p) + r * a.block.stride;
        struct Column { float n1, n2, x, y, dh, gate, post; };
        const auto column = [&](int32_t c) {
            Column q = {(float)block[c] * r1, 0.0f, 0.0f, 0.0f, 0.0f, factor_at(a.gate, r, c), factor_at(a.post, 0, c)};
            if (a.grad_residual_out.p) q.dh = (float)(static_cast<const R*>(a.grad_residual_out.p) + r * a.grad_residual_out.stride)[c];
            if (a.has_pre) {
                q.n2 = (float)(static_cast<const R*>(a.residual_out.p) + r * a.residual_out.stride)[c] * r2;
                q.y = (float)(static_cast<const A*>(a.grad_out.p) + r * a.grad_out.stride)[c];
                q.x = q.y * factor_at(a.pre, 0, c);
                q.dh = fmaf(r2, q.x, q.dh);
            }
            return q;
        };
        float s[3] = {0.0f, 0.0f, 0.0f};
        for (int32_t c = t; c < a.dim; c += 1024) {
            const Column q = column(c);
            s[0] = fmaf(q.x, q.n2, s[0]);
            if (a.has_post) {
                const float w = q.gate * q.post * q.n1;
                s[1] = fmaf(q.dh, w, s[1]);
                s[2] = fmaf(q.n2, w, s[2]);
            }
        }
        row_sums<1024>(s, tmp[0]);
        const float along2 = r2 * s[0] * each, along1 = a.has_post ? (s[1] - along2 * s[2]) * each * a.block_scale : 0.0f;
        for (int32_t c = t; c < a.dim; c += 1024) {
            const Column q = column(c);
            const float dh = fmaf(-along2, q.n2, q.dh), du = dh * a.block_scale, dg = du * q.n1 * q.post, db = du * q.gate;
            const float add[3] = {db * q.n1, dg, q.y * q.n2};
            for (int i = 0; i < 3; ++i)
                if (a.sum[i].p) part[(int64_t)i * a.dim + c] = first ? add[i] : part[(int64_t)i * a.dim + c] + add[i];
            if (a.grad_residual.p) (static_cast<R*>(a.grad_residual.p) + r * a.grad_residual.stride)[c] = (R)(dh * a.residual_scale);
            if (a.grad_gate.p) (static_cast<A*>(a.grad_gate.p) + r * a.grad_gate.stride)[c] = (A)dg;
            if (a.grad_block.p) (static_cast<A*>(a.grad_block.p) + r * a.grad_block.stride)[c] = (A)(r1 * fmaf(-along1, q.n1, db * q.post));
        }
        __syncthreads();                         // tmp is free again
    }
}

// The workgroups' sums as one: 16 columns to a workgroup, 16 threads to a column.
struct NormJoinArgs { NormSum sum[3]; const float* part; int32_t dim, parts, accumulate; };
__global__ __launch_bounds__(256) void residual_norm_join_kernel(const NormJoinArgs a) {
    __shared__ float tmp[16][17];
    const NormSum out = a.sum[blockIdx.y];
    if (!out.p) return;
    const int32_t c = blockIdx.x * 16 + threadIdx.x % 16, strip = threadIdx.x / 16;
    float v = 0.0f;
    if (c < a.dim)
        for (int32_t p = strip; p < a.parts; p += 16) v += a.part[((int64_t)p * 3 + blockIdx.y) * a.dim + c];
    tmp[strip][threadIdx.x % 16] = v;
    __syncthreads();
    if (strip > 0 || c >= a.dim) return;
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += tmp[i][threadIdx.x];
    const auto put = [&](auto* to) {
        if (a.accumulate) v += (float)to[c];
        to[c] = (std::remove_reference_t<decltype(*to)>)v;
    };
    if (out.type == DC_F32) put(static_cast<float*>(out.p));
    else if (out.type == DC_BF16) put(static_cast<__bf16*>(out.p));
    else put(static_cast<_Float16*>(out.p));
}

size_t residual_norm_workspace_bytes(int64_t rows, int64_t dim) {
    return (size_t)std::max(std::min(rows, NORM_PARTS) * std::min<int64_t>(dim, NORM_WIDEST), std::min(rows, NORM_WIDE_PARTS) * dim) * 3 * sizeof(float);
}

hipError_t launch_residual_norm_grad(const NormGradArgs& a, hipStream_t st) {
    if (a.dim == 0) return hipSuccess;
    unsigned parts = 0;
    if (a.rows > 0) {
        bool wide = a.dim % 8 == 0;
        for (const NormStream* s : {&a.block, &a.grad_out, &a.grad_block, &a.grad_gate}) wide = wide && lies_wide(*s, a.act);
        for (const NormStream* s : {&a.residual_out, &a.grad_residual_out, &a.grad_residual}) wide = wide && lies_wide(*s, a.res);
        if (a.gate.p && a.gate.rows) wide = wide && lies_wide(NormStream{const_cast<void*>(a.gate.p), a.gate.stride}, a.act);
        const hipError_t e = with_type(a.act, [&](auto ea) {
            return with_type(a.res, [&](auto er) {
                using A = typename decltype(ea)::type;
                using R = typename decltype(er)::type;
                if (a.dim > NORM_WIDEST) {
                    parts = (unsigned)std::min(a.rows, NORM_WIDE_PARTS);
                    residual_norm_grad_wide_kernel<A, R><<<parts, 1024, 0, st>>>(a);
                    return hipGetLastError();
                }
                return with_threads<true>(a.dim, wide, [&](auto p, auto e, auto w) {
                    constexpr int P = decltype(p)::value, THREADS = P < 256 ? 256 : P, ROWS = THREADS / P;
                    parts = (unsigned)std::min<int64_t>((a.rows + ROWS - 1) / ROWS, NORM_PARTS * 256 / THREADS);
                    residual_norm_grad_kernel<A, R, P, decltype(e)::value, decltype(w)::value><<<parts, THREADS, 0, st>>>(a);
                    return hipGetLastError();
                });
            });
        });
        if (e != hipSuccess) return e;
    }
    if (!a.sum[0].p && !a.sum[1].p && !a.sum[2].p) return hipSuccess;
    const NormJoinArgs j = {{a.sum[0], a.sum[1], a.sum[2]}, a.part, a.dim, (int32_t)parts, a.accumulate};
    residual_norm_join_kernel<<<dim3((unsigned)(a.dim + 15) / 16, 3), 256, 0, st>>>(j);
    return hipGetLastError();
}

}  // namespace dc
