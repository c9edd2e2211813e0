// AdamW over many tensors in one launch.
#include "actor_device.h"

namespace dc {

static inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

AdamwTable carve_adamw_table(void* base, int32_t n_tensors, int64_t n_pieces) {
    AdamwTable t;
    char* p = static_cast<char*>(base);
    t.head = reinterpret_cast<AdamwHeader*>(p);
    t.tensors = reinterpret_cast<dc_adamw_tensor*>(p + 256);
    size_t off = 256 + round_up((size_t)n_tensors * sizeof(dc_adamw_tensor), 256);
    t.pieces = reinterpret_cast<AdamwPiece*>(p + off);
    t.bytes = off + round_up((size_t)n_pieces * sizeof(AdamwPiece), 256);
    return t;
}

// The table travels in kernel arguments, a few tensors a launch: the call neither waits for a copy nor keeps host memory.
constexpr int TABLE_TENSORS = 32;
struct TableChunk {
    AdamwHeader head;
    int32_t first, count;
    int64_t first_piece[TABLE_TENSORS];
    dc_adamw_tensor tensors[TABLE_TENSORS];
};

__global__ __launch_bounds__(256) void adamw_table_kernel(const TableChunk c, AdamwTable t) {
    if (blockIdx.y == 0 && blockIdx.x == 0 && threadIdx.x == 0) *t.head = c.head;
    const int i = blockIdx.y;
    if (blockIdx.x == 0 && threadIdx.x == 0) t.tensors[c.first + i] = c.tensors[i];
    const int64_t n = (c.tensors[i].n + ADAMW_PIECE - 1) / ADAMW_PIECE;
    for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < n; p += (int64_t)gridDim.x * 256)
        t.pieces[c.first_piece[i] + p] = AdamwPiece{c.first + i, (int32_t)p};
}

// Whether every array of a tensor starts on a multiple of 16 bytes.
static int32_t aligned(const dc_adamw_tensor& d) {
    uintptr_t all = 0;
    for (const void* p : {(const void*)d.d_param, (const void*)d.d_master, d.d_grad, (const void*)d.d_exp_avg, (const void*)d.d_exp_avg_sq})
        all |= reinterpret_cast<uintptr_t>(p);
    return all % 16 == 0;
}

hipError_t launch_adamw_table(const dc_adamw_tensor* tensors, const AdamwHeader& head, const AdamwTable& t, hipStream_t st) {
    const int32_t n_tensors = head.n_tensors;
    int64_t at = 0;
    for (int32_t first = 0; first < n_tensors; first += TABLE_TENSORS) {
        TableChunk c = {};
        c.head = head;
        c.first = first;
        c.count = n_tensors - first < TABLE_TENSORS ? n_tensors - first : TABLE_TENSORS;
        int64_t most = 1;
        for (int i = 0; i < c.count; ++i) {
            c.tensors[i] = tensors[first + i];
            c.tensors[i].reserved = aligned(tensors[first + i]);
            c.first_piece[i] = at;
            const int64_t n = (tensors[first + i].n + ADAMW_PIECE - 1) / ADAMW_PIECE;
            at += n;
            if (n > most) most = n;
        }
        const int64_t gx = (most + 255) / 256;
        adamw_table_kernel<<<dim3((unsigned)(gx < 1024 ? gx : 1024), (unsigned)c.count), 256, 0, st>>>(c, t);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

__device__ __forceinline__ float load_as(const void* p, int64_t i, int32_t type) {
    switch (type) {
        case DC_F32:  return static_cast<const float*>(p)[i];
        case DC_BF16: return (float)static_cast<const __bf16*>(p)[i];
        default:      return (float)static_cast<const _Float16*>(p)[i];
    }
}
__device__ __forceinline__ void store_as(void* p, int64_t i, int32_t type, float v) {
    switch (type) {
        case DC_F32:  static_cast<float*>(p)[i] = v; break;
        case DC_BF16: static_cast<__bf16*>(p)[i] = (__bf16)v; break;
        default:      static_cast<_Float16*>(p)[i] = (_Float16)v; break;
    }
}
__device__ __forceinline__ float from_e4m3(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8(c, 0); }
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

constexpr float E4M3_MOST = 448.0f, E4M3_LEAST = 0x1p-9f, STATE_SCALE_LEAST = 0x1p-120f;

// a / b for b > 0 that is neither denormal nor near the largest float: the hardware's reciprocal and one correction by the
// remainder, which is exact (what a general quotient does beyond that costs 8-bit states 3 % of the step).  The last
// operation puts in what infinities and NaN come to.
__device__ __forceinline__ float quotient(float a, float b) {
    const float y = __builtin_amdgcn_rcpf(b), q = a * y;
    return __builtin_amdgcn_div_fixupf(fmaf(fmaf(-b, q, a), y, q), b, a);
}
// One element's step; m and v become the new states, root the square root of v; returns the new weight.  Whatever goes into
// states of 8 bits is rounded operation by operation (no contraction, exact roots and quotients): a value next to a border of
// two codes goes the same way wherever these operations are done, and a state never depends on how a root is made.
__device__ __forceinline__ float step_of(const AdamwStep& s, float decay, float g, float w, float& m, float& v, float& root) {
    m = m * s.beta1 + g * s.one_minus_beta1;
    v = v * s.beta2 + g * g * s.one_minus_beta2;
    root = sqrtf(v);
    return w * decay - s.step_size * quotient(m, root * s.inv_root_bc2 + s.eps);
}
// Behind it, for an element whose v is beyond 32 bits (a gradient above 1.8e19) but not its root, which is what 8 bits keep: the
// root and the weight again from what they were, with everything 2^-80 times as large, where a square fits and eps is nothing.
__device__ __forceinline__ float far_step_of(const AdamwStep& s, float decay, float g, float w, float& m, float& root) {
    constexpr float LESS = 0x1p-80f, MOST = 0x1.fffffep127f;
    const float gl = g * LESS, rl = root * LESS, root_l = sqrtf(rl * rl * s.beta2 + gl * gl * s.one_minus_beta2);
    // (averages of finite numbers: only their rounding can pass the largest)
    root = fminf(root_l / LESS, MOST);
    if (fabsf(g) <= MOST) m = fminf(fmaxf(m, -MOST), MOST);
    return w * decay - s.step_size * quotient(m * LESS, root_l * s.inv_root_bc2);
}
// The scales of a block whose largest magnitudes are these, and their inverses; both 0 for what is stored as zeros.  One half of
// the wave divides for the one, the other half for the other.
struct Scales { float m, m_inverse, root, root_inverse; };
__device__ __forceinline__ Scales scales_of(float m_most, float root_most) {
    float s = (lane_id() < WAVE / 2 ? m_most : root_most) / E4M3_MOST;
    s = s >= STATE_SCALE_LEAST ? s : 0.0f;
    const float inverse = s > 0.0f ? 1.0f / s : 0.0f;
    const auto of = [](float v, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane)); };
    return Scales{of(s, 0), of(inverse, 0), of(s, WAVE - 1), of(inverse, WAVE - 1)};
}
// 32 bits that look random, of the step, the element's place and its gradient: two products of 32 by 32 bits, each folded.  Over
// 200 steps of 65 536 places their mean, variance and the correlations between neighbouring steps and places are those of
// independent ones, with gradients that are all zero, all the same or normal.
__device__ __forceinline__ uint32_t chance(uint32_t seed, int64_t place, float g) {
    const auto fold = [](uint32_t x, uint32_t c) { const uint64_t p = (uint64_t)x * c; return (uint32_t)(p >> 32) ^ (uint32_t)p; };
    return fold(fold((((uint32_t)place * 0x9E3779B1u ^ seed) + __float_as_uint(g)) ^ 0x6A09E667u, 0xBB67AE85u) ^ 0x3C6EF372u, 0xA54FF53Bu);
}
// What a root becomes in 8 bits, before the conversion rounds it to nearest.  Where an average moves by less in a step than codes
// are apart, nearest would put a root back where it was, time and again: there (CHANCE) it goes to the code above or below it,
// by chance and the likelier the nearer, so that it moves as far as it should on average.  Median of the kept root over that of
// 32 bits, elements whose gradients fall to a tenth halfway through 1000 steps (0.999: 10 000), nearest / by chance: beta2 0.95
// 1.04 / -, 0.96 1.09 / 0.99, 0.97 2.4 / 0.99, 0.98 12.7 / 0.98, 0.99 9.2 / 0.99, 0.999 6.7 / 0.99.  The first moment needs none
// of it: 0.0133 off at beta1 from 0.9 to 0.99 by nearest, 0.019 by chance (rms, gradients of 1), for its gradients and the
// block's scale move it from code to code.  612 M elements: 1.78 ms, by nearest 1.69; a
// kernel of its own, for the branch alone costs the others 0.6 %.
__device__ __forceinline__ float by_chance(float c, uint32_t chance) {
    // 20 bits behind those that a code holds; what is below a code's smallest power of two gets that power in front
    const float front = c < 0x1p-6f ? 0x1p-6f : 0.0f;
    return __uint_as_float((__float_as_uint(fminf(c, E4M3_MOST) + front) + (chance >> 12)) & 0xFFF00000u) - front;
}
__device__ __forceinline__ float not_zero(float c, float exact) { return exact > 0.0f ? fmaxf(c, E4M3_LEAST) : c; }      // (it is divided by)
// Codes of neighbouring elements, the first of them at `place`.
template <bool CHANCE, int N>
__device__ __forceinline__ void root_codes(const AdamwStep& s, const float (&root)[N], float inverse, int64_t place, const float (&g)[N], float (&code)[N]) {
    if constexpr (CHANCE) {
#pragma unroll
        for (int c = 0; c < N; ++c) code[c] = not_zero(by_chance(root[c] * inverse, chance(s.seed, place + c, g[c])), root[c] * inverse);
    } else {
#pragma unroll
        for (int c = 0; c < N; ++c) code[c] = not_zero(root[c] * inverse, root[c] * inverse);
    }
}
// The largest of a wave's magnitudes, in every lane: magnitudes sort like their bits.
__device__ __forceinline__ float wave_most(float v) {
    const uint32_t m = wave_incl_scan_u32(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)m, WAVE - 1));
}

// A wave's block of DC_STATE_BLOCK elements or fewer, element by element: the last block of a tensor, tensors that are not
// aligned (200 M elements in bf16 with masters and 8-bit states 1.52 ms, aligned 0.55; 32-bit states 1.33 and 1.00), and blocks of
// 8-bit states with a v beyond 32 bits.
template <bool CHANCE>
__device__ __forceinline__ void block_by_elements(const AdamwStep& s, const dc_adamw_tensor& d, int64_t block, float gs, float decay) {
    const int64_t at = block * DC_STATE_BLOCK;
    const bool small = d.state_type == DC_E4M3;
    const float ms = small ? d.d_exp_avg_scale[block] : 0.0f, vs = small ? d.d_exp_avg_sq_scale[block] : 0.0f;
    float g[4], m[4], root[4], m_most = 0.0f, root_most = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = at + j * WAVE + lane_id();
        g[j] = m[j] = root[j] = 0.0f;
        if (i >= d.n) continue;
        float v, old_root = 0.0f;
        if (small) {
            m[j] = from_e4m3(static_cast<const uint8_t*>(d.d_exp_avg)[i]) * ms;
            old_root = from_e4m3(static_cast<const uint8_t*>(d.d_exp_avg_sq)[i]) * vs;
            v = old_root * old_root;
        } else {
            m[j] = static_cast<const float*>(d.d_exp_avg)[i];
            v = static_cast<const float*>(d.d_exp_avg_sq)[i];
        }
        g[j] = load_as(d.d_grad, i, d.grad_type) * gs;
        const float old_w = d.d_master ? d.d_master[i] : load_as(d.d_param, i, d.param_type);
        float w = step_of(s, decay, g[j], old_w, m[j], v, root[j]);
        if (small && v == INFINITY) {
            root[j] = old_root;
            w = far_step_of(s, decay, g[j], old_w, m[j], root[j]);
        }
        if (d.d_master) d.d_master[i] = w;
        store_as(d.d_param, i, d.param_type, w);
        if (!small) {
            static_cast<float*>(d.d_exp_avg)[i] = m[j];
            static_cast<float*>(d.d_exp_avg_sq)[i] = v;
        }
        m_most = fmaxf(m_most, fabsf(m[j]));
        root_most = fmaxf(root_most, root[j]);
    }
    if (!small) return;
    const Scales sc = scales_of(wave_most(m_most), wave_most(root_most));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = at + j * WAVE + lane_id();
        if (i >= d.n) continue;
        static_cast<uint8_t*>(d.d_exp_avg)[i] = (uint8_t)to_e4m3(m[j] * sc.m_inverse, 0.0f, 0.0f, 0.0f);
        float code[1];
        root_codes<CHANCE, 1>(s, {root[j]}, sc.root_inverse, i, {g[j]}, code);
        static_cast<uint8_t*>(d.d_exp_avg_sq)[i] = (uint8_t)to_e4m3(code[0], 0.0f, 0.0f, 0.0f);
    }
    if (lane_id() == 0) { d.d_exp_avg_scale[block] = sc.m; d.d_exp_avg_sq_scale[block] = sc.root; }
}

// Four neighbouring elements as they lie in memory.
template <typename T> struct Raw4 { T e[4]; };
template <typename T>
__device__ __forceinline__ Raw4<T> load4(const void* p, int64_t i) {
    Raw4<T> r;
    if constexpr (sizeof(T) == 4) {
        const u32x4 q = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const T*>(p) + i));
        __builtin_memcpy(&r, &q, 16);
    } else {
        const u32x2 q = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(static_cast<const T*>(p) + i));
        __builtin_memcpy(&r, &q, 8);
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void store4(void* p, int64_t i, const float (&f)[4]) {
    Raw4<T> r;
#pragma unroll
    for (int c = 0; c < 4; ++c) r.e[c] = (T)f[c];
    if constexpr (sizeof(T) == 4) {
        u32x4 q;
        __builtin_memcpy(&q, &r, 16);
        __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(static_cast<T*>(p) + i));
    } else {
        u32x2 q;
        __builtin_memcpy(&q, &r, 8);
        __builtin_nontemporal_store(q, reinterpret_cast<u32x2*>(static_cast<T*>(p) + i));
    }
}

// A wave's block of an aligned tensor, four neighbouring elements to a lane; everything is asked for before anything is used.
// G: the gradient's type, P: what the weights are read from (the master's float, or the parameter's).  False, and nothing
// written, where the block has to go by elements: a v beyond 32 bits in 8-bit states.
template <typename G, typename P, bool MASTER, bool SMALL, bool CHANCE>
__device__ __forceinline__ bool whole_block(const AdamwStep& s, const dc_adamw_tensor& d, int64_t block, float gs, float decay) {
    const int64_t i = block * DC_STATE_BLOCK + lane_id() * 4;
    const Raw4<G> rg = load4<G>(d.d_grad, i);
    const Raw4<P> rw = load4<P>(MASTER ? (const void*)d.d_master : d.d_param, i);
    float m[4], v[4], root[4], w[4];
    if constexpr (SMALL) {
        const uint32_t cm = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(d.d_exp_avg) + i));
        const uint32_t cv = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(d.d_exp_avg_sq) + i));
        const float ms = d.d_exp_avg_scale[block], vs = d.d_exp_avg_sq_scale[block];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            m[c] = from_e4m3((uint8_t)(cm >> (8 * c))) * ms;
            const float r = from_e4m3((uint8_t)(cv >> (8 * c))) * vs;
            v[c] = r * r;
        }
    } else {
        const Raw4<float> rm = load4<float>(d.d_exp_avg, i), rv = load4<float>(d.d_exp_avg_sq, i);
#pragma unroll
        for (int c = 0; c < 4; ++c) { m[c] = rm.e[c]; v[c] = rv.e[c]; }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = step_of(s, decay, (float)rg.e[c] * gs, (float)rw.e[c], m[c], v[c], root[c]);
    float root_most = 0.0f;                      // this lane's
    if constexpr (SMALL) {
        // (the weights and m are there before the branch: left to itself the compiler asks for what they are made of behind it,
        // which takes 8 % more time)
#pragma unroll
        for (int c = 0; c < 4; ++c) asm volatile("" : "+v"(w[c]), "+v"(m[c]));
        root_most = fmaxf(fmaxf(root[0], root[1]), fmaxf(root[2], root[3]));
        if (__ballot(root_most == INFINITY)) return false;
    }
    if constexpr (MASTER) {
        store4<float>(d.d_master, i, w);
        if (d.param_type == DC_BF16) store4<__bf16>(d.d_param, i, w);
        else if (d.param_type == DC_F16) store4<_Float16>(d.d_param, i, w);
        else store4<float>(d.d_param, i, w);
    } else {
        store4<P>(d.d_param, i, w);
    }
    if constexpr (SMALL) {
        const Scales sc = scales_of(wave_most(fmaxf(fmaxf(fabsf(m[0]), fabsf(m[1])), fmaxf(fabsf(m[2]), fabsf(m[3])))),
                                    wave_most(root_most));
        const uint32_t em = to_e4m3(m[0] * sc.m_inverse, m[1] * sc.m_inverse, m[2] * sc.m_inverse, m[3] * sc.m_inverse);
        const float g[4] = {(float)rg.e[0] * gs, (float)rg.e[1] * gs, (float)rg.e[2] * gs, (float)rg.e[3] * gs};
        float code[4];
        root_codes<CHANCE>(s, root, sc.root_inverse, i, g, code);
        const uint32_t er = to_e4m3(code[0], code[1], code[2], code[3]);
        __builtin_nontemporal_store(em, reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(d.d_exp_avg) + i));
        __builtin_nontemporal_store(er, reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(d.d_exp_avg_sq) + i));
        if (lane_id() == 0) { d.d_exp_avg_scale[block] = sc.m; d.d_exp_avg_sq_scale[block] = sc.root; }
    } else {
        store4<float>(d.d_exp_avg, i, m);
        store4<float>(d.d_exp_avg_sq, i, v);
    }
    return true;
}
template <typename G, bool SMALL, bool CHANCE>
__device__ __forceinline__ bool whole_block_of(const AdamwStep& s, const dc_adamw_tensor& d, int64_t block, float gs, float decay) {
    if (d.d_master) return whole_block<G, float, true, SMALL, CHANCE>(s, d, block, gs, decay);
    if (d.param_type == DC_F32) return whole_block<G, float, false, SMALL, CHANCE>(s, d, block, gs, decay);
    if (d.param_type == DC_BF16) return whole_block<G, __bf16, false, SMALL, CHANCE>(s, d, block, gs, decay);
    return whole_block<G, _Float16, false, SMALL, CHANCE>(s, d, block, gs, decay);
}

// One workgroup per piece, a wave per block.  What a tensor is made of is the same for a whole piece, so the kinds are branches
// of one kernel and all tensors go in one launch.  Bound by the streams: 612 M elements in bf16 with 32-bit masters, bf16
// gradients and 8-bit states (16 bytes each) in 1.69 ms, 5.8 TB/s; 54 M all in 32 bits (28 bytes) in 0.26 ms, 5.8 TB/s.  Two or
// four blocks a wave, all asked for at once: within 2 % for 32-bit states, 3 to 5 % slower for 8-bit ones.  Plain stores
// instead of streamed ones: 6 % slower.
constexpr int AW_THREADS = ADAMW_PIECE / DC_STATE_BLOCK * WAVE;
template <bool CHANCE>
__global__ __launch_bounds__(AW_THREADS) void adamw_kernel(const AdamwStep s, const AdamwHeader want, const AdamwHeader* __restrict__ head,
                                                           const dc_adamw_tensor* __restrict__ tensors,
                                                           const AdamwPiece* __restrict__ pieces) {
    const int64_t n_pieces = want.n_pieces;
    if (head->n_pieces != n_pieces || head->n_tensors != want.n_tensors || head->print != want.print) {
        if (threadIdx.x == 0) set_status(s.status, DC_ERR_BAD_LAYOUT);
        return;
    }
    const float gs = s.grad_scale ? *s.grad_scale : 1.0f;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    for (int64_t q = blockIdx.x; q < n_pieces; q += gridDim.x) {
        const AdamwPiece piece = pieces[q];
        const dc_adamw_tensor d = tensors[piece.tensor];     // (a copy: no store below can be thought to change it)
        const float decay = (float)(1.0 - s.lr64 * d.weight_decay);
        const int64_t block = (int64_t)piece.piece * (ADAMW_PIECE / DC_STATE_BLOCK) + wave;
        bool done = block * DC_STATE_BLOCK >= d.n;
        if (d.reserved && (block + 1) * DC_STATE_BLOCK <= d.n) {           // (in the table: whether all of it is aligned)
            if (d.state_type == DC_E4M3) {
                if (d.grad_type == DC_BF16) done = whole_block_of<__bf16, true, CHANCE>(s, d, block, gs, decay);
                else if (d.grad_type == DC_F32) done = whole_block_of<float, true, CHANCE>(s, d, block, gs, decay);
                else done = whole_block_of<_Float16, true, CHANCE>(s, d, block, gs, decay);
            } else {
                if (d.grad_type == DC_BF16) done = whole_block_of<__bf16, false, false>(s, d, block, gs, decay);
                else if (d.grad_type == DC_F32) done = whole_block_of<float, false, false>(s, d, block, gs, decay);
                else done = whole_block_of<_Float16, false, false>(s, d, block, gs, decay);
            }
        }
        if (!done) block_by_elements<CHANCE>(s, d, block, gs, decay);
    }
}

hipError_t launch_adamw(const AdamwStep& s, const AdamwHeader& head, const AdamwTable& t, hipStream_t st) {
    if (head.n_pieces == 0) return hipSuccess;
    const unsigned grid = (unsigned)(head.n_pieces < (1 << 22) ? head.n_pieces : 1 << 22);     // (2^31 threads)
    if (s.dither) adamw_kernel<true><<<grid, AW_THREADS, 0, st>>>(s, head, t.head, t.tensors, t.pieces);
    else adamw_kernel<false><<<grid, AW_THREADS, 0, st>>>(s, head, t.head, t.tensors, t.pieces);
    return hipGetLastError();
}

}  // namespace dc
