// Quantisation to 4-bit microscaled blocks and back (layout in mx.h).
// The row kernel and a decode step's first launch share mx_quant_body.h.  All kernels here are bound by HBM: 16384 x 4096
// bf16 in 29 us (170 MB), back to fp32 in 42 us (304 MB).
#include "mx_quant_body.h"

namespace molora {

namespace {

template <bool F32>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const void *__restrict__ src, const int32_t *__restrict__ perm,
                                                          uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                          int64_t rows, int K, int kt_n, int kg_n) {
    __shared__ uint8_t sc[256];
    mx_quantize_body<F32>(blockIdx.x, src, perm, codes, scales, rows, K, kt_n, kg_n, sc);
}

// A base weight [d_in][d_out]: rows of the operand are its columns, blocks run down them.  A lane takes two
// columns, so that a wavefront's load covers 256 contiguous bytes of a row of W and a block's maximum and codes
// stay in the lane; wavefront b takes block b of four k tiles, which makes up its columns' dwords of scales.
__global__ __launch_bounds__(256) void mx_quantize_w_kernel(const uint16_t *__restrict__ W, uint8_t *__restrict__ codes,
                                                            uint8_t *__restrict__ scales, int d_in, int d_out, int kt_n,
                                                            int kg_n) {
    const int lane = threadIdx.x & 63, kb = threadIdx.x >> 6;
    const int kg = (int)(blockIdx.x % kg_n);
    const int col = (int)(blockIdx.x / kg_n) * 128 + lane * 2;
    const bool col_in = col < d_out;
    const int padded = (d_out + 15) & ~15;
    uint32_t dword[2] = {0, 0};
    for (int j = 0; j < 4; ++j) {
        const int kt = kg * 4 + j, k0 = kt * 128 + kb * 32;
        if (kt >= kt_n) break;
        uint32_t raw[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int k = k0 + i < d_in ? k0 + i : d_in - 1;
            raw[i] = *(const uint32_t *)(W + (int64_t)k * d_out + (col_in ? col : 0));
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float v[32];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                uint32_t bits = c ? raw[i] & 0xFFFF0000u : raw[i] << 16;
                bits = col_in && k0 + i < d_in ? bits : 0u;
                top = max_u32(top, bits & 0x7FFFFFFFu);
                v[i] = __uint_as_float(bits);
            }
            const uint32_t byte = scale_byte(top);
            const float scale = scale_of(byte);
            dword[c] |= byte << (8 * j);
            if (col + c < padded) {
                const int64_t tile = (int64_t)((col + c) >> 4) * kt_n + kt;
                *(u32x4 *)(codes + (tile * 64 + kb * 16 + ((col + c) & 15)) * 16) =
                    u32x4{codes8(v, scale), codes8(v + 8, scale), codes8(v + 16, scale), codes8(v + 24, scale)};
            }
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (col + c < padded)
            *(uint32_t *)(scales + (((int64_t)((col + c) >> 4) * kg_n + kg) * 64 + kb * 16 + ((col + c) & 15)) * 4) = dword[c];
}

// Back to the values, fp32 rows.  A wavefront takes two rows of a tile at a time, four values a lane, and
// stores 512 contiguous bytes of each; a workgroup of four takes a tile.
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint8_t *__restrict__ codes,
                                                            const uint8_t *__restrict__ scales, float *__restrict__ dst,
                                                            int64_t rows, int K, int kt_n, int kg_n) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rt = blockIdx.x / kt_n;
    const int kt = (int)(blockIdx.x % kt_n);
    const int kb = (lane >> 3) & 3, k = kt * 128 + (lane & 31) * 4;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const int row = wave * 4 + g * 2 + (lane >> 5), entry = kb * 16 + row;
        const uint32_t q = *(const uint16_t *)(codes + ((rt * kt_n + kt) * 64 + entry) * 16 + (lane & 7) * 2);
        const uint32_t byte = scales[((rt * kg_n + (kt >> 2)) * 64 + entry) * 4 + (kt & 3)];
        // 2^(byte - 127) in two factors, both normal numbers: the value may be below the smallest one
        const float s1 = __uint_as_float((byte < 64 ? byte + 64 : byte) << 23);
        const float s2 = byte < 64 ? 5.421010862427522e-20f : 1.0f;  // 2^-64
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t c = q >> (4 * i), m = c & 7;
            const float a = m < 4 ? (float)m * 0.5f : m < 6 ? (float)(m - 2) : (float)(2 * m - 8);
            v[i] = byte == 255 ? __uint_as_float(0x7FC00000u) : (c & 8 ? -a : a) * s1 * s2;
        }
        if (rt * 16 + row < rows && k < K) __builtin_nontemporal_store(v, (f32x4 *)(dst + (rt * 16 + row) * K + k));
    }
}

}  // namespace

hipError_t launch_mx_quantize(const void *src, bool src_f32, const int32_t *perm, uint8_t *codes, uint8_t *scales,
                              int64_t rows, int K, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const int kt = mx_k_tiles(K), kg = mx_k_groups(K);
    const int64_t blocks = mx_row_tiles(rows) * kg;
    if (blocks >= kMxMaxBlocks) return hipErrorInvalidValue;
    if (src_f32)
        hipLaunchKernelGGL((mx_quantize_kernel<true>), dim3((unsigned)blocks), dim3(256), 0, s, src, perm, codes, scales, rows, K, kt, kg);
    else
        hipLaunchKernelGGL((mx_quantize_kernel<false>), dim3((unsigned)blocks), dim3(256), 0, s, src, perm, codes, scales, rows, K, kt, kg);
    return hipGetLastError();
}

hipError_t launch_mx_quantize_w(const uint16_t *W, uint8_t *codes, uint8_t *scales, int d_in, int d_out, hipStream_t s) {
    const int kg = mx_k_groups(d_in);
    const int64_t blocks = (((int64_t)d_out + 127) / 128) * kg;
    if (blocks >= kMxMaxBlocks) return hipErrorInvalidValue;
    hipLaunchKernelGGL(mx_quantize_w_kernel, dim3((unsigned)blocks), dim3(256), 0, s, W, codes, scales, d_in, d_out,
                       mx_k_tiles(d_in), kg);
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(const uint8_t *codes, const uint8_t *scales, float *dst, int64_t rows, int K,
                                hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const int64_t blocks = mx_row_tiles(rows) * mx_k_tiles(K);
    if (blocks >= kMxMaxBlocks) return hipErrorInvalidValue;
    hipLaunchKernelGGL(mx_dequantize_kernel, dim3((unsigned)blocks), dim3(256), 0, s, codes, scales, dst, rows, K,
                       mx_k_tiles(K), mx_k_groups(K));
    return hipGetLastError();
}

}  // namespace molora
