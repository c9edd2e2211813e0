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

hipError_t launch_adamw_table(const dc_adamw_tensor* tensors, int32_t n_tensors, const AdamwTable& t, int64_t n_pieces, hipStream_t st) {
    int64_t at = 0;
    for (int32_t first = 0; first < n_tensors; first += TABLE_TENSORS) {
        TableChunk c = {};
        c.head = AdamwHeader{n_pieces, n_tensors, 0};
        c.first = first;
        c.count = n_tensors - first < TABLE_TENSORS ? n_tensors - first : TABLE_TENSORS;
        int64_t most = 1;
        for (int i = 0; i < c.count; ++i) {
            c.tensors[i] = tensors[first + i];
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
__device__ __forceinline__ uint8_t to_e4m3(float v) { return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false) & 0xFF); }

constexpr float E4M3_MOST = 448.0f, E4M3_LEAST = 0x1p-9f, STATE_SCALE_LEAST = 0x1p-120f;

// One wave per block of DC_STATE_BLOCK elements, four to a lane, element by element.  Every operation on m, v and the
// scales is rounded by itself (no contraction), so that what is stored in 8 bits is a function of the inputs alone.
constexpr int AW_THREADS = 256;
__global__ __launch_bounds__(AW_THREADS) void adamw_kernel(const AdamwStep s, const AdamwTable t, int64_t n_pieces, int32_t n_tensors) {
    if (t.head->n_pieces != n_pieces || t.head->n_tensors != n_tensors) {
        if (threadIdx.x == 0) set_status(s.status, DC_ERR_BAD_LAYOUT);
        return;
    }
    const float gs = s.grad_scale ? *s.grad_scale : 1.0f;
    for (int64_t q = blockIdx.x; q < n_pieces; q += gridDim.x) {
        const AdamwPiece piece = t.pieces[q];
        const dc_adamw_tensor& d = t.tensors[piece.tensor];
        const float decay = (float)(1.0 - s.lr64 * d.weight_decay);
        const bool small = d.state_type == DC_E4M3;
        for (int b = threadIdx.x / WAVE; b < ADAMW_PIECE / DC_STATE_BLOCK; b += AW_THREADS / WAVE) {
            const int64_t block = (int64_t)piece.piece * (ADAMW_PIECE / DC_STATE_BLOCK) + b, at = block * DC_STATE_BLOCK;
            if (at >= d.n) break;
            const float ms = small ? d.d_exp_avg_scale[block] : 0.0f, vs = small ? d.d_exp_avg_sq_scale[block] : 0.0f;
            float m[4], root[4], m_most = 0.0f, root_most = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t i = at + j * WAVE + lane_id();
                m[j] = root[j] = 0.0f;
                if (i >= d.n) continue;
                float v;
                if (small) {
                    m[j] = from_e4m3(static_cast<const uint8_t*>(d.d_exp_avg)[i]) * ms;
                    const float r = from_e4m3(static_cast<const uint8_t*>(d.d_exp_avg_sq)[i]) * vs;
                    v = r * r;
                } else {
                    m[j] = static_cast<const float*>(d.d_exp_avg)[i];
                    v = static_cast<const float*>(d.d_exp_avg_sq)[i];
                }
                const float g = load_as(d.d_grad, i, d.grad_type) * gs;
                m[j] = m[j] * s.beta1 + g * s.one_minus_beta1;
                v = v * s.beta2 + g * g * s.one_minus_beta2;
                root[j] = sqrtf(v);
                float w = d.d_master ? d.d_master[i] : load_as(d.d_param, i, d.param_type);
                w = w * decay - s.step_size * (m[j] / (root[j] * s.inv_root_bc2 + s.eps));
                if (d.d_master) d.d_master[i] = w;
                store_as(d.d_param, i, d.param_type, w);
                if (!small) {
                    static_cast<float*>(d.d_exp_avg)[i] = m[j];
                    static_cast<float*>(d.d_exp_avg_sq)[i] = v;
                }
                m_most = fmaxf(m_most, fabsf(m[j]));
                root_most = fmaxf(root_most, root[j]);
            }
            if (!small) continue;
            float m_scale = wave_max(m_most) / E4M3_MOST, r_scale = wave_max(root_most) / E4M3_MOST;
            if (!(m_scale >= STATE_SCALE_LEAST)) m_scale = 0.0f;
            if (!(r_scale >= STATE_SCALE_LEAST)) r_scale = 0.0f;
            const float m_inv = m_scale > 0.0f ? 1.0f / m_scale : 0.0f, r_inv = r_scale > 0.0f ? 1.0f / r_scale : 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t i = at + j * WAVE + lane_id();
                if (i >= d.n) continue;
                const float mc = m[j] * m_inv;
                float rc = root[j] * r_inv;
                if (rc > 0.0f) rc = fmaxf(rc, E4M3_LEAST);
                static_cast<uint8_t*>(d.d_exp_avg)[i] = to_e4m3(mc);
                static_cast<uint8_t*>(d.d_exp_avg_sq)[i] = to_e4m3(rc);
            }
            if (lane_id() == 0) { d.d_exp_avg_scale[block] = m_scale; d.d_exp_avg_sq_scale[block] = r_scale; }
        }
    }
}

hipError_t launch_adamw(const AdamwStep& s, int32_t n_tensors, const AdamwTable& t, int64_t n_pieces, hipStream_t st) {
    if (n_pieces == 0) return hipSuccess;
    const unsigned grid = (unsigned)(n_pieces < (1 << 20) ? n_pieces : 1 << 20);
    adamw_kernel<<<grid, AW_THREADS, 0, st>>>(s, t, n_pieces, n_tensors);
    return hipGetLastError();
}

}  // namespace dc
