// Argument checks that the entry points share.
#pragma once
#include "../../include/molora.h"
#include "common.h"

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned256(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }
inline size_t round256(size_t b) { return (b + 255u) & ~size_t(255); }

inline bool apply_sizes_ok(int64_t N, int32_t d_in, int32_t d_out, int32_t C, int32_t rank) {
    return N >= 0 && N < (int64_t(1) << 31) && d_in >= 8 && d_in % 8 == 0 && d_out >= 8 &&
           d_out % 8 == 0 && C >= 1 && C <= MOLORA_MAX_TARGETS && rank >= 8 && rank % 8 == 0 &&
           rank <= MOLORA_MAX_RANK;
}

inline molora_status from_hip(hipError_t e) { return e == hipSuccess ? MOLORA_OK : MOLORA_EHIP; }

}  // namespace
