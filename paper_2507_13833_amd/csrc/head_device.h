// Products of matrices on the matrix cores for the head: both operands have their rows' elements along the summed axis side by
// side, 16-bit floats in, 32-bit sums out.
#pragma once
#include "logprob_device.h"
#include "head_internal.h"

namespace dc {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// D[i, j] += sum_k A[i, k] B[j, k] for 16 x 16 places and 32 k.  Lane l brings A[l % 16, 8 (l / 16) ..] and B likewise, and holds
// D[4 (l / 16) + 0..3, l % 16].
template <typename T> struct Mfma;
template <> struct Mfma<__bf16> {
    using Frag = bf16x8;
    static __device__ __forceinline__ f32x4 add(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<_Float16> {
    using Frag = f16x8;
    static __device__ __forceinline__ f32x4 add(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// A workgroup makes PM rows of A times PN rows of B: four waves, two by two, 128 x 64 each.
constexpr int PM = 256, PN = 128, PK = 32, P_THREADS = 256;
constexpr int P_STAGES = 3, P_STAGE = (PM + PN) * PK * 2, P_LDS = P_STAGES * P_STAGE;
constexpr int P_MT = PM / 32, P_NT = PN / 32;            // 16 x 16 places of a wave
constexpr int P_MOST_PARTS = 6;

struct Operand {
    const char*    p;               // 16-byte aligned
    int64_t        pitch;           // bytes from a row to the next, a multiple of 16 and at most P_MOST_PITCH
    const int32_t* list;            // which rows, by their numbers (the last one's end below 4 GB then); NULL: as they lie
};
constexpr int64_t P_MOST_PITCH = 1 << 23;
// The sum goes over parts: pairs of places, in bytes from the operands' starts, with `steps` times PK elements each.
struct Parts { int32_t n; int64_t a[P_MOST_PARTS], b[P_MOST_PARTS]; };

typedef const __attribute__((address_space(1))) void GlobalVoid;
typedef __attribute__((address_space(3))) void LdsVoid;
// 16 bytes a lane from memory to the LDS, lane after lane from `to` on (the same in every lane).
__device__ __forceinline__ void load_to_lds(const char* from, char* to) {
    __builtin_amdgcn_global_load_lds((GlobalVoid*)from, (LdsVoid*)to, 16, 0, 0);
}
// Waits until at most `N` of the wave's loads and stores are under way, and all its LDS reads are done.
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4);
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void bare_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// What of a tile a thread loads: rows tid / 4 + 64 j, 16 bytes each.  The four 16-byte pieces of a row's 64 bytes lie in the LDS at
// piece ^ (row / 2 % 4), so that eight rows' same piece fills all banks.
struct TileOfA { const char* base; uint32_t at[PM / 64]; };
struct TileOfB { const char* base; uint32_t at[PN / 64]; };
template <typename Tile>
__device__ __forceinline__ void place_tile(Tile& t, const Operand& o, int32_t first, int32_t n_rows) {
    const int row = threadIdx.x / 4, piece = (threadIdx.x & 3) ^ (row >> 1 & 3);
    t.base = o.list ? o.p : o.p + first * o.pitch;
#pragma unroll
    for (int j = 0; j < (int)(sizeof(t.at) / 4); ++j) {
        const int32_t r = min(first + row + 64 * j, n_rows - 1);         // (behind the last row: that one again)
        t.at[j] = (uint32_t)(o.list ? o.list[r] : r - first) * (uint32_t)o.pitch + 16 * piece;
    }
}

// acc = the tile's sums (0 without steps).  Three stages of PK elements: while one is multiplied the next two are on their way.
template <typename T>
__device__ __forceinline__ void product(f32x4 (&acc)[P_MT][P_NT], const TileOfA& a, const TileOfB& b, const Parts& parts, int32_t steps,
                                        char* lds) {
    using Frag = typename Mfma<T>::Frag;
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
#pragma unroll
    for (int i = 0; i < P_MT; ++i)
#pragma unroll
        for (int j = 0; j < P_NT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    const int32_t all = steps * parts.n;
    if (all <= 0) return;
    int32_t part = 0, left = steps;
    const char *pa = a.base + parts.a[0], *pb = b.base + parts.b[0];
    char* to = lds + wave * 1024;
    const auto ask = [&](char* stage) {
#pragma unroll
        for (int j = 0; j < PM / 64; ++j) load_to_lds(pa + a.at[j], stage + j * 4096);
#pragma unroll
        for (int j = 0; j < PN / 64; ++j) load_to_lds(pb + b.at[j], stage + PM * 64 + j * 4096);
        pa += PK * 2;
        pb += PK * 2;
        if (--left == 0 && ++part < parts.n) {
            pa = a.base + parts.a[part];
            pb = b.base + parts.b[part];
            left = steps;
        }
    };
    bare_barrier();                              // (the LDS may still be read)
    ask(to);
    if (all > 1) ask(to + P_STAGE);
    const int row = lane & 15, piece = (lane >> 4) ^ (row >> 1 & 3);
    const char* from_a = lds + (wave / 2 * (PM / 2) + row) * 64 + piece * 16;
    const char* from_b = lds + PM * 64 + (wave % 2 * (PN / 2) + row) * 64 + piece * 16;
    int32_t now = 0, then = 2 * P_STAGE;
    for (int32_t k = 0; k < all; ++k) {
        if (k + 1 < all) wait_loads<(PM + PN) / 64>(); else wait_loads<0>();
        bare_barrier();
        if (k + 2 < all) ask(to + then);
        Frag fa[P_MT], fb[P_NT];
#pragma unroll
        for (int j = 0; j < P_NT; ++j) fb[j] = *reinterpret_cast<const Frag*>(from_b + now + j * 1024);
#pragma unroll
        for (int i = 0; i < P_MT; ++i) fa[i] = *reinterpret_cast<const Frag*>(from_a + now + i * 1024);
#pragma unroll
        for (int i = 0; i < P_MT; ++i)
#pragma unroll
            for (int j = 0; j < P_NT; ++j) acc[i][j] = Mfma<T>::add(fa[i], fb[j], acc[i][j]);
        now = now == 2 * P_STAGE ? 0 : now + P_STAGE;
        then = then == 2 * P_STAGE ? 0 : then + P_STAGE;
    }
    wait_loads<0>();
}

// Workgroups are handed to the eight chiplets in turn.  The n-th of those that share a chiplet (and its L2) come to lie side by side.
__device__ __forceinline__ int32_t by_chiplet(int32_t block, int32_t blocks) {
    const int32_t each = blocks / 8, more = blocks % 8, x = block % 8;
    return x * each + min(x, more) + block / 8;
}
// Of `first` times `second` tiles the at-th: eight firsts beside each other for each second, so that neighbours share both.
struct TilePair { int32_t first, second; };
__device__ __forceinline__ TilePair tile_pair(int32_t at, int32_t first, int32_t second) {
    const int32_t group = at / (8 * second), in = at - group * 8 * second, wide = min(8, first - group * 8);
    return TilePair{group * 8 + in % wide, in / wide};
}

// ---- operands laid out for the product ----

// The first of how many 16-bit numbers a value is taken apart into: together they are it, to 8 or 11 bits a number.
template <typename D>
__device__ __forceinline__ D take_part(float& rest) {
    D d = (D)rest;
    // (the largest numbers of 32 bits are infinite in bf16: cut those instead of rounding them)
    if constexpr (std::is_same_v<D, __bf16>)
        if (fabsf(rest) < INFINITY && fabsf((float)d) == INFINITY) d = __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(rest) >> 16));
    rest = fabsf(rest) < INFINITY ? rest - (float)d : 0.0f;
    return d;
}

}  // namespace dc
