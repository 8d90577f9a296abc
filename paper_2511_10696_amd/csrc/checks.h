// checks.h -- argument checks that the parts of the C ABI share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/pi_attn.h"

namespace pi_attn {

constexpr int64_t kMaxRows = (int64_t)1 << 31;   // B*H*N (and S*H) limit

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline int elem_size(int32_t dtype) { return dtype == PI_ATTN_F32 ? 4 : dtype == PI_ATTN_BF16 ? 2 : 0; }

inline bool stride16(int64_t stride_elems, int es) { return stride_elems >= 0 && ((stride_elems * es) & 15) == 0; }

inline int from_hip(hipError_t e) { return e == hipSuccess ? PI_ATTN_OK : PI_ATTN_EHIP; }

}  // namespace pi_attn
