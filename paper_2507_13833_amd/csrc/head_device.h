// Products of matrices on the matrix cores for the head: both operands have their rows' elements along the summed axis side by
// side, 16-bit floats in, 32-bit sums out.
#pragma once
#include "logprob_device.h"
#include "head_internal.h"

namespace dc {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));         // 16 bytes wherever a 16-bit element may lie
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// D[i, j] += sum_k A[i, k] B[j, k] for 16 x 16 places and 32 k.  Lane l brings A[l % 16, 8 (l / 16) ..] and B likewise, and holds
// D[4 (l / 16) + 0..3, l % 16].  The sums stay in the accumulation registers, which the compiler would share out otherwise and copy
// from and to in the loop (add; sum is the ordinary way).  It does not know these instructions for what they are, so settle_sums() keeps
// their distance from ordinary ones that write or read the sums.
template <typename T> struct Mfma;
template <> struct Mfma<__bf16> {
    using Frag = bf16x8;
    static __device__ __forceinline__ void add(const Frag& a, const Frag& b, f32x4& c) {
        asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    }
    static __device__ __forceinline__ f32x4 sum(const Frag& a, const Frag& b, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<_Float16> {
    using Frag = f16x8;
    static __device__ __forceinline__ void add(const Frag& a, const Frag& b, f32x4& c) {
        asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    }
    static __device__ __forceinline__ f32x4 sum(const Frag& a, const Frag& b, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
// A sum out of its register, read where this stands and not kept.
__device__ __forceinline__ float sum_of(float c) {
    float v;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(c));
    return v;
}
// 32 cycles: more than any of the distances (18 at most, behind the longest of these instructions).
__device__ __forceinline__ void settle_sums() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A workgroup makes 32 Q rows of A times 32 Q rows of B: four waves, two by two, Q by Q places of 16 x 16 each.  Q = 8: a wave to a SIMD,
// all 256 sums of its lanes in registers, the most products for what is read.  Q = 4: two workgroups to a compute unit, one begins
// and ends beside the other's products, where there are few tiles or few steps.
constexpr int PK = 64, P_THREADS = 256;
template <int Q> constexpr int P_SIDE = 32 * Q;
template <int Q> constexpr int P_STAGE = 2 * P_SIDE<Q> * PK * 2;
template <int Q> constexpr int P_LDS = 2 * P_STAGE<Q>;
template <int Q> constexpr int P_SLOTS = Q == 8 ? 256 : 512;         // workgroups at once
constexpr int P_MOST_SIDE = P_SIDE<8>;

struct Operand {
    const char*    p;               // 16-byte aligned
    int64_t        pitch;           // bytes from a row to the next, a multiple of 16 and at most P_MOST_PITCH
    const int32_t* list;            // which rows, by their numbers (the last one's end below 4 GB then); NULL: as they lie
};
constexpr int64_t P_MOST_PITCH = 1 << 23;
// Second planes of f16 hold what the first leave off times so much: as exact down to 2^-28 of the largest value as near it.
constexpr float SMALL_PART = 2048.0f;
// The sum goes over n parts of `steps` times PK elements each: part i multiplies plane (a >> 2 i) % 4 of A, planes a_plane bytes apart,
// by plane (b >> 2 i) % 4 of B.  All but the last hold one second plane.
struct Parts { int32_t n; uint32_t a, b; int64_t a_plane, b_plane; };

typedef const __attribute__((address_space(1))) void GlobalVoid;
typedef __attribute__((address_space(3))) void LdsVoid;
// 16 bytes a lane from memory to the LDS, lane after lane from `to` on (the same in every lane).
// STREAM: not kept in the caches.
template <bool STREAM = false>
__device__ __forceinline__ void load_to_lds(const char* from, char* to) {
    __builtin_amdgcn_global_load_lds((GlobalVoid*)from, (LdsVoid*)to, 16, 0, STREAM ? 2 : 0);
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

// What of a tile a thread loads: the rows that lie at tid / 8 + 32 j in the LDS, 16 bytes each.  The eight 16-byte pieces of a row's
// 128 bytes lie there at piece ^ (place % 8), so that eight rows' same piece fills all banks.  Rows of the tile are dealt out to the
// places so that a lane comes to hold neighbours, which its stores want: of each 16 Q rows of A, place 16 i + p takes row
// 32 (i / 2) + 8 (p / 4) + 4 (i % 2) + p % 4; of each 16 Q of B, place 16 j + q row Q q + j.
template <int Q> struct Tile { const char* base; uint32_t at[Q]; };
template <int Q> struct TileOfA : Tile<Q> {
    static __device__ __forceinline__ int row_at(int x) { return (x & ~31) + (x >> 2 & 3) * 8 + (x >> 4 & 1) * 4 + (x & 3); }
};
template <int Q> struct TileOfB : Tile<Q> {
    static __device__ __forceinline__ int row_at(int x) { return (x & -16 * Q) + (x & 15) * Q + (x >> 4 & (Q - 1)); }
};
template <typename T>
__device__ __forceinline__ void place_tile(T& t, const Operand& o, int32_t first, int32_t n_rows) {
    const int place = threadIdx.x / 8, piece = (threadIdx.x ^ place) & 7;
    t.base = o.list ? o.p : o.p + first * o.pitch;
#pragma unroll
    for (int j = 0; j < (int)(sizeof(t.at) / 4); ++j) {
        const int32_t r = min(first + T::row_at(place + 32 * j), n_rows - 1);        // (behind the last row: that one again)
        t.at[j] = (uint32_t)(o.list ? o.list[r] : r - first) * (uint32_t)o.pitch + 16 * piece;
    }
}

// Where a lane's rows begin in a tile of A and of B: acc[i][j][e] is of A's row place_a() + along_a(i, e) and B's place_b() + j.
template <int Q> __device__ __forceinline__ int place_a() { return threadIdx.x / (2 * WAVE) * (16 * Q) + (lane_id() >> 4) * 8; }
template <int Q> __device__ __forceinline__ int place_b() { return threadIdx.x / WAVE % 2 * (16 * Q) + (lane_id() & 15) * Q; }
constexpr __device__ __host__ int along_a(int i, int e) { return i / 2 * 32 + i % 2 * 4 + e; }

// The workgroup's tiles one after the other.  Two stages of PK elements lie in the LDS, each multiplied in two halves; a half's numbers
// are read into registers while the half before is multiplied.  Once the second half of a stage is in registers its place is free:
// the stage after next is asked for there, a whole stage ahead and on into the next tile.  next() makes a and b that next tile (or
// leaves them: what is asked for then is not used).  Steps and parts are the same for all tiles, and there is at least one of each.
template <typename T, int Q>
struct Product {
    using Frag = typename Mfma<T>::Frag;
    static constexpr int STAGE = P_STAGE<Q>, B_AT = P_SIDE<Q> * 128;     // where B's rows lie in a stage
    TileOfA<Q>  a;
    TileOfB<Q>  b;
    Parts       parts;
    int32_t     steps, part, left, stage;
    const char *pa, *pb;
    char*       to;
    const char *from_a, *from_b;
    int         at_half[2];
    Frag        fa[2][Q], fb[2][Q];

    __device__ __forceinline__ void start_of(int32_t i) {
        part = i;
        left = steps;
        pa = a.base + (parts.a >> 2 * i & 3) * parts.a_plane;
        pb = b.base + (parts.b >> 2 * i & 3) * parts.b_plane;
    }
    __device__ __forceinline__ void ask_a(int j) { load_to_lds(pa + a.at[j], to + (stage & 1) * STAGE + j * 4096); }
    __device__ __forceinline__ void ask_b(int j) { load_to_lds(pb + b.at[j], to + (stage & 1) * STAGE + B_AT + j * 4096); }
    template <typename Next>
    __device__ __forceinline__ void asked(Next&& next) {
        pa += PK * 2;
        pb += PK * 2;
        ++stage;
        if (--left == 0) {
            if (part + 1 < parts.n) {
                start_of(part + 1);
            } else {
                next();
                start_of(0);
            }
        }
    }
    __device__ __forceinline__ void read_a(int32_t s, int h, int i) {
        fa[h][i] = *reinterpret_cast<const Frag*>(from_a + (s & 1) * STAGE + at_half[h] + i * 2048);
    }
    __device__ __forceinline__ void read_b(int32_t s, int h, int j) {
        fb[h][j] = *reinterpret_cast<const Frag*>(from_b + (s & 1) * STAGE + at_half[h] + j * 2048);
    }

    // a, b, parts and steps are set
    template <typename Next>
    __device__ __forceinline__ void begin(char* lds, Next&& next) {
        const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
        const int row = lane & 15, piece = (lane >> 4) ^ (row & 7);
        to = lds + wave * 1024;
        from_a = lds + (wave / 2 * (16 * Q) + row) * 128;
        from_b = lds + B_AT + (wave % 2 * (16 * Q) + row) * 128;
        at_half[0] = piece * 16;
        at_half[1] = (piece ^ 4) * 16;
        stage = 0;
        start_of(0);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int j = 0; j < Q; ++j) ask_a(j);
#pragma unroll
            for (int j = 0; j < Q; ++j) ask_b(j);
            asked(next);
        }
        wait_loads<2 * Q>();
        bare_barrier();
#pragma unroll
        for (int i = 0; i < Q; ++i) read_a(0, 0, i);
#pragma unroll
        for (int j = 0; j < Q; ++j) read_b(0, 0, j);
    }

    // acc = the sums of the tile whose turn it is
    template <typename Next>
    __device__ __forceinline__ void tile(f32x4 (&acc)[Q][Q], Next&& next) {
#pragma unroll
        for (int i = 0; i < Q; ++i)
#pragma unroll
            for (int j = 0; j < Q; ++j) {
                acc[i][j] = f32x4{0, 0, 0, 0};
                asm volatile("" : "+a"(acc[i][j]));  // (in their registers from here on)
            }
        settle_sums();
        int32_t s = stage - 2;
        const int32_t end = s + steps * parts.n;
        const auto run = [&](int32_t to) {
            for (; s < to; ++s) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = 0; q < 2 * Q; ++q) {    // half a row of places to a read
#pragma unroll
                    for (int e = 0; e < Q / 2; ++e) Mfma<T>::add(fa[0][q / 2], fb[0][q % 2 * (Q / 2) + e], acc[q / 2][q % 2 * (Q / 2) + e]);
                    // (the first products of the next half want all of B and the first of A)
                    if (q < Q) read_b(s, 1, q); else read_a(s, 1, q - Q);
                    __builtin_amdgcn_sched_barrier(0);
                }
                wait_loads<0>();
                bare_barrier();
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = 0; q < 2 * Q; ++q) {
#pragma unroll
                    for (int e = 0; e < Q / 2; ++e) Mfma<T>::add(fa[1][q / 2], fb[1][q % 2 * (Q / 2) + e], acc[q / 2][q % 2 * (Q / 2) + e]);
                    if (q < Q) ask_a(q); else ask_b(q - Q);
                    if (q < Q) read_b(s + 1, 0, q); else read_a(s + 1, 0, q - Q);
                    __builtin_amdgcn_sched_barrier(0);
                }
                asked(next);
            }
        };
        if (parts.n > 1) {                       // the small parts' products are SMALL_PART times too large
            run(end - steps);
            settle_sums();
#pragma unroll
            for (int i = 0; i < Q; ++i)
#pragma unroll
                for (int j = 0; j < Q; ++j) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = sum_of(acc[i][j][e]) * (1.0f / SMALL_PART);
                    asm volatile("" : "+a"(acc[i][j]));              // (back where they belong, four at a time)
                    __builtin_amdgcn_sched_barrier(0);
                }
            settle_sums();
        }
        run(end);
        settle_sums();
    }

    // the LDS is free again
    __device__ __forceinline__ void end() {
        wait_loads<0>();
        bare_barrier();
    }
};
// One tile alone, already placed.
template <typename T, int Q>
__device__ __forceinline__ void product(f32x4 (&acc)[Q][Q], const TileOfA<Q>& a, const TileOfB<Q>& b, const Parts& parts, int32_t steps,
                                        char* lds) {
    if (steps <= 0) {
#pragma unroll
        for (int i = 0; i < Q; ++i)
#pragma unroll
            for (int j = 0; j < Q; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
        return;
    }
    Product<T, Q> p;
    p.a = a;
    p.b = b;
    p.parts = parts;
    p.steps = steps;
    const auto next = [] {};
    p.begin(lds, next);
    p.tile(acc, next);
    p.end();
}

// Workgroups are handed to the eight chiplets in turn.  The n-th of those that share a chiplet (and its L2) come to lie side by side.
__device__ __forceinline__ int32_t by_chiplet(int32_t block, int32_t blocks) {
    const int32_t each = blocks / 8, more = blocks % 8, x = block % 8;
    return x * each + min(x, more) + block / 8;
}
// Of `blocks` workgroups that were launched for all rows, how many come to each tile of those that take part; at most `most`.
__device__ __forceinline__ int32_t live_share(int32_t blocks, int32_t tiles, int32_t most) {
    return tiles > 0 ? min(blocks / tiles, most) : 0;
}
// Of `first` times `second` tiles the at-th: eight firsts beside each other for each second, so that neighbours share both.
struct TilePair { int32_t first, second; };
__device__ __forceinline__ TilePair tile_pair(int32_t at, int32_t first, int32_t second) {
    const int32_t group = at / (8 * second), in = at - group * 8 * second, wide = min(8, first - group * 8);
    return TilePair{group * 8 + in % wide, in / wide};
}

// ---- operands laid out for the product ----

// The first of how many 16-bit numbers a value is taken apart into, 11 (f16) or 8 (bf16) bits each; rest: what the next are made of.
template <typename D>
__device__ __forceinline__ D take_part(float& rest) {
    D d = (D)rest;
    // (the largest numbers of 32 bits are infinite in bf16: cut those instead of rounding them)
    if constexpr (std::is_same_v<D, __bf16>)
        if (fabsf(rest) < INFINITY && fabsf((float)d) == INFINITY) d = __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(rest) >> 16));
    rest = fabsf(rest) < INFINITY ? rest - (float)d : 0.0f;
    if constexpr (std::is_same_v<D, _Float16>) rest *= SMALL_PART;
    return d;
}

// ---- powers of two of operands ----

constexpr int NO_EXPONENT = -100000;
__device__ __forceinline__ int exponent_above(float magnitude) { return (int)(__float_as_uint(magnitude) >> 23) - 126; }     // 2^it is above
__device__ __forceinline__ int exponent_above(double magnitude) { return (int)((uint64_t)__double_as_longlong(magnitude) >> 52) - 1022; }
// A wave's largest finite magnitude of a row, as bits (those of a float without a sign sort like it).
template <typename T>
__device__ __forceinline__ uint32_t row_top(const T* row, int32_t cols) {
    constexpr int N = 16 / sizeof(T);
    const int lane = lane_id();
    uint32_t big = 0;
    const auto one = [&](T v) {
        const uint32_t bits = __float_as_uint(fabsf((float)v));
        big = max(big, bits < 0x7F800000u ? bits : 0u);
    };
    const int32_t head = min(cols, (int32_t)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int32_t)sizeof(T)), chunks = (cols - head) / N;
    if (lane < head) one(row[lane]);
    const u32x4* body = reinterpret_cast<const u32x4*>(row + head);
    for (int32_t c = lane; c < chunks; c += 4 * WAVE) {
        union { u32x4 q; T e[N]; } in[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) in[j].q = body[min(c + j * WAVE, chunks - 1)];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) one(in[j].e[i]);
    }
    if (head + chunks * N + lane < cols) one(row[head + chunks * N + lane]);
    return big;
}
__device__ __forceinline__ uint32_t wave_top(uint32_t big) {
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) big = max(big, (uint32_t)__shfl_xor((int)big, d));
    return big;
}
// The largest of the four waves' exponents goes to *top: one atomic a workgroup, and few of those (8192 waves' own took 98 us).
constexpr int64_t TOP_BLOCKS = 512;
__device__ __forceinline__ void raise_top(int most, int* tmp, int32_t* top) {
    if (lane_id() == 0) tmp[threadIdx.x / WAVE] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        most = max(max(tmp[0], tmp[1]), max(tmp[2], tmp[3]));
        if (most != NO_EXPONENT) atomicMax(top, most);
    }
}

}  // namespace dc
