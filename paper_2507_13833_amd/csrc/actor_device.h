// Device-side building blocks of the actor's update: number formats and reductions over a wave and a workgroup.
#pragma once
#include "dc_device.h"
#include "actor_internal.h"

namespace dc {

// ---- number formats: every kernel computes in float and rounds once, to nearest, ties to even ----
template <int TYPE> struct Elem;
template <> struct Elem<DC_F32>  { using type = float; };
template <> struct Elem<DC_BF16> { using type = __bf16; };
template <> struct Elem<DC_F16>  { using type = _Float16; };

template <typename F>
hipError_t with_type(int32_t type, F&& f) {
    switch (type) {
        case DC_F32:  return f(Elem<DC_F32>{});
        case DC_BF16: return f(Elem<DC_BF16>{});
        case DC_F16:  return f(Elem<DC_F16>{});
    }
    return hipErrorInvalidValue;
}

// ---- reductions over a wave: every lane gets the result ----
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)v, d);
        v = o > v ? o : v;
    }
    return v;
}
// Over a workgroup, in the same order in every thread; `tmp` holds one T per wave and is free again on return.
template <typename T, typename WaveOp, typename Op>
__device__ __forceinline__ T block_reduce(T v, T* tmp, WaveOp wave_op, Op op) {
    v = wave_op(v);
    if (lane_id() == 0) tmp[threadIdx.x / WAVE] = v;
    __syncthreads();
    T all = tmp[0];
    for (unsigned w = 1; w < blockDim.x / WAVE; ++w) all = op(all, tmp[w]);
    __syncthreads();
    return all;
}

// ---- rows of a table: a wave takes COLS columns, eight to a lane ----
// EIGHTS: neighbours, for results of 2 bytes; FOURS: twice four neighbours, so that a wave's 16-byte stores of 4-byte results
// lie side by side and fill whole lines (both need aligned rows and dim % 8 == 0); APART: 64 apart.
constexpr int COLS = 512;
enum Layout { APART, EIGHTS, FOURS };

template <typename T>
inline bool rows_aligned(const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (size_t)stride * sizeof(T) % 16 == 0;
}
template <Layout L>
__device__ __forceinline__ int64_t column(int64_t slab, int j) {
    return slab * COLS + (L == EIGHTS ? lane_id() * 8 + j : L == FOURS ? j / 4 * (COLS / 2) + lane_id() * 4 + j % 4 : j * WAVE + lane_id());
}
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// Eight elements as they lie in memory.
template <typename T>
union Raw8 {
    T e[8];
    u32x4 q[sizeof(T) / 2];
    u32x2 d[sizeof(T)];
};
template <Layout L, typename T>
__device__ __forceinline__ void load8(const T* row, int64_t slab, int64_t dim, Raw8<T>& r) {
    // (behind the row's end: its last columns again, which nobody stores)
    if constexpr (L == EIGHTS) {
        const u32x4* p = reinterpret_cast<const u32x4*>(row + min(column<L>(slab, 0), dim - 8));
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) r.q[h] = p[h];
    } else if constexpr (L == FOURS) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const T* p = row + min(column<L>(slab, 4 * h), dim - 4);
            if constexpr (sizeof(T) == 4) r.q[h] = *reinterpret_cast<const u32x4*>(p);
            else r.d[h] = *reinterpret_cast<const u32x2*>(p);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.e[j] = row[min(column<L>(slab, j), dim - 1)];
    }
}
template <Layout L, bool STREAM = false, typename T>           // STREAM: past the caches
__device__ __forceinline__ void store8(T* row, int64_t slab, int64_t dim, const float (&f)[8]) {
    Raw8<T> r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.e[j] = (T)f[j];
    if constexpr (L == EIGHTS) {
        if (column<L>(slab, 0) < dim) {
            u32x4* p = reinterpret_cast<u32x4*>(row + column<L>(slab, 0));
#pragma unroll
            for (int h = 0; h < (int)sizeof(T) / 2; ++h)
                if constexpr (STREAM) store16(p + h, r.q[h]); else p[h] = r.q[h];
        }
    } else if constexpr (L == FOURS) {
        static_assert(sizeof(T) == 4, "whole lines");
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (column<L>(slab, 4 * h) < dim) {
                u32x4* p = reinterpret_cast<u32x4*>(row + column<L>(slab, 4 * h));
                if constexpr (STREAM) store16(p, r.q[h]); else *p = r.q[h];
            }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t c = column<L>(slab, j);
            if (c < dim) row[c] = r.e[j];
        }
    }
}
constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LN2 = 0.69314718055994530942f;

// A float as an unsigned integer that sorts like it (a zero's sign does not count).
__device__ __forceinline__ uint32_t sortable(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unsortable(uint32_t s) {
    return __uint_as_float(s & 0x80000000u ? s & 0x7FFFFFFFu : ~s);
}

}  // namespace dc
