// The scaled matrix instruction on operands in the layout of mx.h.
#pragma once
#include "mx.h"

namespace molora {
namespace {

// Codes as the instruction's operand: 16 bytes a lane, the format's upper half is not read.
__device__ __forceinline__ i32x8 mx_operand(u32x4 c) {
    return i32x8{(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0};
}
// acc += W tile (first operand: a lane then holds four columns of one row of h) x x tile, scales from byte J
template <int J>
__device__ __forceinline__ f32x4 mx_mfma(u32x4 w, u32x4 x, f32x4 acc, uint32_t sw, uint32_t sx) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(w), mx_operand(x), acc, 4, 4, J, (int)sw, J, (int)sx);
}

}  // namespace
}  // namespace molora
