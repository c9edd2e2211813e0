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
