// The backward pass of the gated block z = act(g) u, [g | u] = h = x W + (x A_r) B_r, beside its GEMMs:
//
//     dh = [dz u act'(g) | dz act(g)],   dA_c = x_c^T (dh_c B_c^T),   dB_c = (x_c A_c)^T dh_c
#include "gate.h"
#include "lds_dma.h"

namespace molora {

namespace {

// One thread takes four columns of a row.
// dh is rounded to bf16 here: it is an operand of the matrix instructions in every gradient that follows.  (h comes
// in fp32: with g and u rounded too, the gradients would be 1.9 instead of 1.4 times as far from their exact
// values as their own rounding to bf16 puts them.)
__global__ __launch_bounds__(256) void gate_backward_kernel(const uint16_t *__restrict__ dz, const float *__restrict__ pre,
                                                            uint16_t *__restrict__ dh, int64_t N, int64_t items, int F, int act) {
    const int64_t it = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (it >= items) return;
    const int per = F / 4;
    const int64_t row = it / per;
    const int col = (int)(it % per) * 4;
    uint16_t *out = dh + row * 2 * F + col;
    if (row >= N) {
        *(u32x2 *)out = u32x2{0, 0};
        *(u32x2 *)(out + F) = u32x2{0, 0};
        return;
    }
    const float *h = pre + row * 2 * F + col;
    const f32x4 g = *(const f32x4 *)h, u = *(const f32x4 *)(h + F);
    const u32x2 d2 = *(const u32x2 *)(dz + row * F + col);
    f32x4 dg, du;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float d = bf16_bits_to_f32((d2[i >> 1] >> (16 * (i & 1))) & 0xFFFF);
        float slope;
        const float p = gate_factor<true>(g[i], act, slope);
        dg[i] = d * u[i] * (p + g[i] * slope);
        du[i] = d * g[i] * p;
    }
    *(u32x2 *)out = bf16x4_bits(dg);
    *(u32x2 *)(out + F) = bf16x4_bits(du);
}

__global__ __launch_bounds__(256) void zero_kernel(u32x4 *__restrict__ dst, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) dst[i] = u32x4{0, 0, 0, 0};
}

// 64 x 64 elements through LDS; rows and columns are multiples of 8 (rows of the padded side).
__global__ __launch_bounds__(256) void transpose_kernel(const uint16_t *__restrict__ src, uint16_t *__restrict__ dst,
                                                        int64_t rows, int64_t cols, int64_t padded, int64_t tiles_c,
                                                        int64_t tiles) {
    __shared__ uint16_t t[64][66];
    const int64_t b = blockIdx.x / tiles, in = blockIdx.x % tiles;
    const int64_t r0 = in / tiles_c * 64, c0 = in % tiles_c * 64;
    src += b * rows * cols;
    dst += b * cols * padded;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = (threadIdx.x >> 3) + i * 32, c = (threadIdx.x & 7) * 8;
        u32x4 v = {0, 0, 0, 0};
        if (r0 + r < rows && c0 + c < cols) v = *(const u32x4 *)(src + (r0 + r) * cols + c0 + c);
#pragma unroll
        for (int j = 0; j < 4; ++j) *(uint32_t *)&t[r][c + 2 * j] = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = (threadIdx.x >> 3) + i * 32, r = (threadIdx.x & 7) * 8;
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (uint32_t)t[r + 2 * j][c] | (uint32_t)t[r + 2 * j + 1][c] << 16;
        if (c0 + c < cols && r0 + r < padded) *(u32x4 *)(dst + (c0 + c) * padded + r0 + r) = v;
    }
}

// out_c = Y_c^T S_c over the rows of a bucket.  A workgroup takes 64 columns of Y and 32 of S (the hi and the lo
// half of each); its four wavefronts take 32 rows at a time in turn, bring them to LDS as they lie in memory and
// read both operands through the transpose read (k of the product runs down the rows).  Sums are added in
// wavefront order.
constexpr int kOuterCols = 64, kOuterR = 32;
template <bool FLAT>
__global__ __launch_bounds__(256) void grouped_outer_kernel(const uint16_t *__restrict__ y, const uint16_t *__restrict__ s2,
                                                            const int32_t *__restrict__ offsets,
                                                            const int32_t *__restrict__ perm, uint16_t *__restrict__ out,
                                                            int D, int R) {
    constexpr int YS = kOuterCols * 2 + 32, SS = kOuterR * 4 + 32;  // bytes per row in LDS
    constexpr int SLAB = 32 * (YS + SS);
    constexpr int PART = kOuterCols * (kOuterR + 1) * 4;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * (SLAB > PART ? SLAB : PART)];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int kq = lane >> 4, l16 = lane & 15;
    const int c = blockIdx.z, d0 = blockIdx.x * kOuterCols, r0 = blockIdx.y * kOuterR;
    const int lo = offsets[c], hi = offsets[c + 1];
    unsigned char *ys = lds + wave * SLAB, *ss = ys + 32 * YS;
    f32x4 acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto frag = [&](const unsigned char *base, int stride, int col) __attribute__((always_inline)) {
        const unsigned char *p = base + (kq * 8 + (l16 >> 2)) * stride + col * 2 + (l16 & 3) * 8;
        const i16x4 u = lds_read_tr16((const MOLORA_LDS void *)p), v = lds_read_tr16((const MOLORA_LDS void *)(p + 4 * stride));
        return __builtin_bit_cast(bf16x8, i16x8{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]});
    };
    for (int p0 = lo + wave * 32; p0 < hi; p0 += 128) {
        u32x4 yv[4], sv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // 8 rows at a time, 8 columns a lane
            const int r = i * 8 + (lane >> 3), col = (lane & 7) * 8;
            const int p = min(p0 + r, hi - 1);
            const int64_t tok = perm[p];
            yv[i] = *(const u32x4 *)(y + tok * D + min(d0 + col, D - 8));
            const int half = col >> 5, sc = min(r0 + (col & 31), R - 8);
            sv[i] = *(const u32x4 *)(s2 + (int64_t)p * 2 * R + half * R + sc);
            if (p0 + r >= hi) {  // rows of the next bucket count as zero, on both sides
                yv[i] = u32x4{0, 0, 0, 0};
                sv[i] = u32x4{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 8 + (lane >> 3), col = (lane & 7) * 8;
            *(u32x4 *)(ys + r * YS + col * 2) = yv[i];
            *(u32x4 *)(ss + r * SS + col * 2) = sv[i];
        }
        bf16x8 fy[4], fs[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fy[i] = frag(ys, YS, i * 16);
            fs[i] = frag(ss, SS, i * 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[i][j & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fy[i], fs[j], acc[i][j & 1], 0, 0, 0);
    }
    __syncthreads();
    float *part = (float *)(lds + wave * PART);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) part[(i * 16 + kq * 4 + v) * (kOuterR + 1) + j * 16 + l16] = acc[i][j][v];
    __syncthreads();
    for (int it = tid; it < kOuterCols * kOuterR / 2; it += 256) {  // two neighbours of the output's rows
        const int d = FLAT ? it % (kOuterCols / 2) * 2 : it / (kOuterR / 2), r = FLAT ? it / (kOuterCols / 2) : it % (kOuterR / 2) * 2;
        float v[2] = {0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                v[k] += ((const float *)(lds + w * PART))[(d + (FLAT ? k : 0)) * (kOuterR + 1) + r + (FLAT ? 0 : k)];
        if (d0 + d < D && r0 + r < R) {
            const int64_t at = FLAT ? ((int64_t)c * R + r0 + r) * D + d0 + d : ((int64_t)c * D + d0 + d) * R + r0 + r;
            *(uint32_t *)(out + at) = bf16x2_bits(v[0], v[1]);
        }
    }
}

}  // namespace

hipError_t launch_zero(void *dst, int64_t bytes, hipStream_t s) {
    const int64_t n = bytes / 16, blocks = (n + 255) / 256;
    if (n > 0)
        hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s, (u32x4 *)dst, n);
    return hipGetLastError();
}

hipError_t launch_gate_backward(const uint16_t *dz, const float *pre, uint16_t *dh, int64_t N, int64_t padded, int F,
                                int act, hipStream_t s) {
    const int64_t items = padded * (F / 4), blocks = (items + 255) / 256;
    if (blocks >= (int64_t(1) << 24)) return hipErrorInvalidValue;
    if (blocks > 0)
        hipLaunchKernelGGL(gate_backward_kernel, dim3((unsigned)blocks), dim3(256), 0, s, dz, pre, dh, N, items, F, act);
    return hipGetLastError();
}

hipError_t launch_transpose(const uint16_t *src, uint16_t *dst, int64_t batch, int64_t rows, int64_t cols, int64_t padded,
                            hipStream_t s) {
    const int64_t tiles_c = (cols + 63) / 64, tiles = tiles_c * ((padded + 63) / 64), blocks = batch * tiles;
    if (blocks >= (int64_t(1) << 24)) return hipErrorInvalidValue;
    if (blocks > 0)
        hipLaunchKernelGGL(transpose_kernel, dim3((unsigned)blocks), dim3(256), 0, s, src, dst, rows, cols, padded, tiles_c, tiles);
    return hipGetLastError();
}

hipError_t launch_grouped_outer(const uint16_t *y, const uint16_t *s2, const int32_t *offsets, const int32_t *perm,
                                uint16_t *out, int64_t N, int D, int C, int R, bool flat, hipStream_t s) {
    (void)N;
    const dim3 grid((unsigned)((D + kOuterCols - 1) / kOuterCols), (unsigned)((R + kOuterR - 1) / kOuterR), (unsigned)C);
    if (flat)
        hipLaunchKernelGGL((grouped_outer_kernel<true>), grid, dim3(256), 0, s, y, s2, offsets, perm, out, D, R);
    else
        hipLaunchKernelGGL((grouped_outer_kernel<false>), grid, dim3(256), 0, s, y, s2, offsets, perm, out, D, R);
    return hipGetLastError();
}

}  // namespace molora
