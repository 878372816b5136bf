// Quantisation of rows to 4-bit microscaled blocks, as part of a launch.
//
//   X = floor(log2 max |v|) - 2 over a block of 32 along k, at least -127: the largest value then lies in
//       [4, 8) 2^X, the top binade of e2m1 (4 and 6) and what saturates to 6
//   code = e2m1(v 2^-X), to the nearest, the even code in the middle, at most 6
//   a block that holds a NaN or an infinity gets the scale byte 255, which stands for NaN
//
// The exponent of the maximum is a shift of its bits: the maximum is taken over the absolute values' bits as
// integers, whose order is that of the numbers and puts infinities and NaN on top.  The rounding is the matrix
// core's own conversion instruction.
#pragma once
#include "mx.h"

namespace molora {
namespace {

__device__ __forceinline__ uint32_t max_u32(uint32_t a, uint32_t b) { return a > b ? a : b; }

// the scale byte of a block whose largest absolute value has these fp32 bits
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const uint32_t e = top >> 23;
    return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}
// the power of two that the byte stands for, as the conversion instructions take it (its exponent field)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float((byte == 255 ? 254u : byte) << 23); }

// eight values -> eight codes in a dword
__device__ __forceinline__ uint32_t codes8(const float *v, float scale) {
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], scale, 3);
    return q;
}

// Rows.  A workgroup takes 16 rows x 512 k, a wavefront one k tile of it: four lanes share a block, eight values
// each, so that a load instruction covers 256 (512) contiguous bytes of a row, and the four rows of an
// instruction leave as 64 contiguous bytes per block.  The scales of the four wavefronts meet in LDS.
template <bool F32>
__device__ __forceinline__ void mx_quantize_body(int64_t block, const void *__restrict__ src, const int32_t *__restrict__ perm,
                                                 uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, int64_t rows, int K,
                                                 int kt_n, int kg_n, uint8_t *sc) {  // sc: 256 bytes of LDS
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rt = block / kg_n;
    const int kg = (int)(block % kg_n);
    const int kt = kg * 4 + wave;
    const int sub = lane >> 4, kb = (lane >> 2) & 3, part = lane & 3;
    const int k = kt * 128 + kb * 32 + part * 8;
    const bool k_in = k < K;  // (K is a multiple of 8)
    u32x4 raw[4][F32 ? 2 : 1];
#pragma unroll
    for (int g = 0; g < 4; ++g) {  // addresses are clamped, what is outside is masked below
        int64_t p = rt * 16 + g * 4 + sub;
        if (p >= rows) p = rows - 1;
        const int64_t row = perm != nullptr ? perm[p] : p;
        const int64_t at = row * K + (k_in ? k : 0);
        if constexpr (F32) {
            raw[g][0] = *(const u32x4 *)((const float *)src + at);
            raw[g][1] = *(const u32x4 *)((const float *)src + at + 4);
        } else {
            raw[g][0] = *(const u32x4 *)((const uint16_t *)src + at);
        }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const bool in = k_in && rt * 16 + g * 4 + sub < rows;
        float v[8];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t bits;
            if constexpr (F32)
                bits = raw[g][i >> 2][i & 3];
            else
                bits = i & 1 ? raw[g][0][i >> 1] & 0xFFFF0000u : raw[g][0][i >> 1] << 16;
            bits = in ? bits : 0u;
            top = max_u32(top, bits & 0x7FFFFFFFu);
            v[i] = __uint_as_float(bits);
        }
        top = max_u32(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));
        top = max_u32(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));
        const uint32_t byte = scale_byte(top);
        const int entry = kb * 16 + g * 4 + sub;
        if (kt < kt_n)
            *(uint32_t *)(codes + ((rt * kt_n + kt) * 64 + entry) * 16 + part * 4) = codes8(v, scale_of(byte));
        if (part == 0) sc[entry * 4 + wave] = (uint8_t)byte;
    }
    __syncthreads();
    if (threadIdx.x < 64)
        *(uint32_t *)(scales + ((rt * kg_n + kg) * 64 + threadIdx.x) * 4) = *(const uint32_t *)(sc + threadIdx.x * 4);
}

}  // namespace
}  // namespace molora
