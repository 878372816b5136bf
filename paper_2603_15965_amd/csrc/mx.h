// 4-bit microscaled operands (blocks of 32 e2m1 values under one power of two), as the kernels of
// mx_quant.hip write them and those of mx_gemm.hip read them.
//
// Codes: [rows / 16][K / 128][64][16 bytes].  A tile of 16 rows x 128 k is the 1 KB that one wavefront
// hands to v_mfma_scale_f32_16x16x128_f8f6f4: entry (lane) 16 b + i holds the 32 codes of row i, block b,
// the even k of a byte in its low half.  One 16-byte load per lane, contiguous over the wavefront, from
// memory or from LDS without bank conflicts, and no swizzle anywhere.
// Scales: [rows / 16][K / 512][64][4 bytes]: the dword of entry 16 b + i holds the exponents (+ 127) of that
// row and block in four k tiles one after the other; the instruction picks the byte.
// Rows are padded to 16, codes along k to 128 and scales to 512, with zero codes under zero bytes.
#pragma once
#include "../../include/molora.h"
#include "common.h"

namespace molora {

typedef __attribute__((ext_vector_type(8))) int i32x8;

inline __host__ __device__ int64_t mx_row_tiles(int64_t rows) { return (rows + 15) / 16; }
inline __host__ __device__ int mx_k_tiles(int K) { return (int)(((int64_t)K + 127) / 128); }
inline __host__ __device__ int mx_k_groups(int K) { return (int)(((int64_t)K + 511) / 512); }  // dwords of scales
// one workgroup of 256 a tile at most: the runtime counts a launch's threads in 32 bits
constexpr int64_t kMxMaxBlocks = int64_t(1) << 24;

// perm != nullptr: row i of the operand is row perm[i] of src
hipError_t launch_mx_quantize(const void *src, bool src_f32, const int32_t *perm, uint8_t *codes, uint8_t *scales,
                              int64_t rows, int K, hipStream_t s);
hipError_t launch_mx_quantize_w(const uint16_t *W, uint8_t *codes, uint8_t *scales, int d_in, int d_out, hipStream_t s);
hipError_t launch_mx_dequantize(const uint8_t *codes, const uint8_t *scales, float *dst, int64_t rows, int K,
                                hipStream_t s);

// h[perm[p]][:] = Q(x)_p Q(W) + t_p B_c for every position p (perm == nullptr: h[p], C = 0: without adapters).
// xc, xs: the rows in the order of the positions.
hipError_t launch_mx_gemm(const uint8_t *xc, const uint8_t *xs, const uint8_t *wc, const uint8_t *ws, const uint16_t *B,
                          const uint16_t *t2, const int32_t *offsets, const int32_t *perm, float *h, int64_t N, int d_in,
                          int d_out, int C, int rank, hipStream_t s);

// A batch of at most 64 tokens in two launches (mx_decode.hip).  The first: the rows' codes and scales, in token order,
// and x_i A_{r(i)} in slices of K (decode_body.h), planes [slices][64][rank] fp32 (rows of tokens without adapter
// are not written).  The second: h = Q(x) Q(W) + (x A_r) B_r; with C = 0 the product alone.
hipError_t launch_mx_decode_first(const uint16_t *x, const uint16_t *A, const int32_t *r, uint8_t *codes, uint8_t *scales,
                                  float *planes, int64_t N, int d_in, int C, int rank, hipStream_t s);
hipError_t launch_mx_decode(const uint8_t *xc, const uint8_t *xs, const uint8_t *wc, const uint8_t *ws, const uint16_t *B,
                            const int32_t *r, const float *planes, float *h, int64_t N, int d_in, int d_out, int C, int rank,
                            hipStream_t s);

int mx_decode_cols(int d_out);  // columns of a workgroup of the second
// the kernel that a product takes: rows, columns and stages of its tiles; 0 stages: at most 64 tokens
void mx_gemm_tile(int64_t N, int d_in, int d_out, int32_t *tile);

}  // namespace molora
