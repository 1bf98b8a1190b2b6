// What the two host layers of the head's operators share (api_head.hip, api_answer.hip).
#pragma once

#include "../../include/huge.h"
#include "head.hpp"

namespace huge {

constexpr int64_t kMaxRows = 0x7FFFFFFF;

#define HEAD_TRY(expr)                                  \
    do {                                                \
        if ((expr) != hipSuccess) return HUGE_ERR_HIP;  \
    } while (0)

inline bool dtype_ok(int32_t t) { return t == HUGE_DTYPE_F32 || t == HUGE_DTYPE_BF16; }

inline size_t elem(int32_t dtype) { return dtype == HUGE_DTYPE_BF16 ? 2 : 4; }

inline bool on(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Whether rows can be read four elements at a time.
inline bool fours(const void* p, int64_t ld, int32_t dtype) {
    return on(p, 4 * elem(dtype)) && ld % 4 == 0;
}

// AdamW: the checks of a step, and the step, whose gradients are multiplied by d_factor[0]
// d_factor[1] where that is given, and by cfg->grad_scale otherwise.
huge_status adamw_args(const huge_adamw_config* cfg, const huge_adamw_tensor* h_tensors,
                       int32_t count, const int32_t* d_status);
huge_status adamw_step(const huge_adamw_config* cfg, const huge_adamw_tensor* h_tensors,
                       int32_t count, const float* d_factor, int32_t* d_status, void* stream);

}  // namespace huge
