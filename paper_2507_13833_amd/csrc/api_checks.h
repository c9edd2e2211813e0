// Host-side checks that the entry points of the actor's update share.
#pragma once
#include "actor_internal.h"

namespace dc {

inline size_t elem_bytes(int32_t type) { return type == DC_F32 ? 4 : type == DC_E4M3 ? 1 : 2; }
inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// A matrix that can be addressed: its last byte lies below 2^62.
inline dc_status check_matrix(const dc_matrix* m) {
    if (!m || m->reserved != 0 || m->type < DC_F32 || m->type > DC_F16) return DC_ERR_INVALID_ARG;
    if (m->n_rows < 0 || m->n_cols < 0 || m->row_stride < m->n_cols) return DC_ERR_INVALID_ARG;
    if (m->n_rows > 0 && m->n_cols > 0 && (!m->d_data || !aligned_to(m->d_data, elem_bytes(m->type)))) return DC_ERR_INVALID_ARG;
    if (m->n_rows > (1LL << 40) || m->row_stride > (1LL << 40) ||
        (m->n_rows > 0 && m->row_stride > (1LL << 60) / m->n_rows)) return DC_ERR_UNSUPPORTED_SIZE;
    return DC_OK;
}

}  // namespace dc
