// Internal: what the host sides of the library's source files share.
#ifndef FLASHOPTIM_HOST_H
#define FLASHOPTIM_HOST_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "flashoptim.h"

// Returns from the function with the status of `expr` if that is not FLASHOPTIM_OK.
#define FO_TRY(expr)                          \
    do {                                      \
        const int rc_ = (int)(expr);          \
        if (rc_ != FLASHOPTIM_OK) return rc_; \
    } while (0)

namespace fo {

// FLASHOPTIM_OK, or FLASHOPTIM_ERR_HIP after noting `e` for flashoptim_last_hip_error.
int hip_status(hipError_t e);

constexpr int64_t kMaxElems = (int64_t)1 << 40;

inline bool aligned_to(const void* p, uintptr_t unit) { return reinterpret_cast<uintptr_t>(p) % unit == 0; }
inline int elem_bytes(int dtype) { return dtype == FLASHOPTIM_FP32 ? 4 : 2; }

// Checks a matrix of `rows` by `cols` values of type FLASHOPTIM_BF16 or FLASHOPTIM_FP32.  Its rows may start anywhere that is aligned
// to a value.
inline int check_matrix(const flashoptim_matrix* m) {
    if (!m || m->rows < 0 || m->cols < 0 || (m->dtype != FLASHOPTIM_BF16 && m->dtype != FLASHOPTIM_FP32))
        return FLASHOPTIM_ERR_INVALID_ARG;
    if (m->rows >= ((int64_t)1 << 31) || m->cols >= ((int64_t)1 << 31)) return FLASHOPTIM_ERR_NUMEL_RANGE;
    if (m->rows == 0 || m->cols == 0) return FLASHOPTIM_OK;
    if (!m->data || (m->rows > 1 && m->stride < m->cols)) return FLASHOPTIM_ERR_INVALID_ARG;
    if (m->rows > 1 && m->stride >= kMaxElems / m->rows) return FLASHOPTIM_ERR_NUMEL_RANGE;
    if (!aligned_to(m->data, (uintptr_t)elem_bytes(m->dtype))) return FLASHOPTIM_ERR_MISALIGNED;
    return FLASHOPTIM_OK;
}

}  // namespace fo
#endif
