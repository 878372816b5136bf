// The backward pass of the gated block z = act(g) u, [g | u] = h = x W + (x A_r) B_r, beside its GEMMs:
//
//     dh = [dz u act'(g) | dz act(g)],   dA_c = x_c^T (dh_c B_c^T),   dB_c = (x_c A_c)^T dh_c
#include "gate.h"
#include "lds_dma.h"

namespace molora {

namespace {

typedef __attribute__((ext_vector_type(2))) float f32x2_t;

// The activation and the product by themselves, where the projection leaves fp32 sums.  One thread takes four columns.
__global__ __launch_bounds__(256) void gate_kernel(const float *planes, int count, uint16_t *__restrict__ z, float *pre, int64_t items,
                                                   int F, int act) {
    const int64_t it = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (it >= items) return;
    const int per = F / 4;
    const int64_t row = it / per, all = items * 8;  // floats of a plane
    const int col = (int)(it % per) * 4;
    const int64_t at = row * 2 * F + col;
    f32x4 g = *(const f32x4 *)(planes + at), u = *(const f32x4 *)(planes + at + F);
    for (int i = 1; i < count; ++i) {
        g += *(const f32x4 *)(planes + i * all + at);
        u += *(const f32x4 *)(planes + i * all + at + F);
    }
    if (pre != nullptr) {
        *(f32x4 *)(pre + at) = g;
        *(f32x4 *)(pre + at + F) = u;
    }
    *(u32x2 *)(z + row * F + col) = bf16x4_bits(gate4(g, u, act));
}

// One thread takes four columns of a row.  dh is rounded to bf16 here: it is an operand of the matrix instructions
// in every gradient that follows.  (h comes in fp32: with g and u rounded too, the gradients would be 1.9 instead of
// 1.4 times as far from their exact values as their own rounding to bf16 puts them.)
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

// Several matrices transposed in one launch, 64 x 64 elements at a time through LDS.  Rows and columns are multiples of 8
// (rows of the padded side).  (t is padded to 66: a column is read without bank conflicts.)
struct TransposeJobs {
    TransposeJob job[kMaxTransposes];
    int first[kMaxTransposes];  // its first workgroup (past the last one: behind it)
};
__global__ __launch_bounds__(256) void transpose_kernel(TransposeJobs jobs) {
    __shared__ uint16_t t[64][66];
    int j = 0;
#pragma unroll
    for (int i = 1; i < kMaxTransposes; ++i) j += (int)blockIdx.x >= jobs.first[i] ? 1 : 0;
    const TransposeJob m = jobs.job[j];
    const int64_t tiles_c = (m.cols + 63) / 64, tiles = tiles_c * ((m.padded + 63) / 64);
    const int64_t at = (int)blockIdx.x - jobs.first[j], b = at / tiles, in = at % tiles;
    const int64_t r0 = in / tiles_c * 64, c0 = in % tiles_c * 64;
    const uint16_t *const src = m.src + b * m.rows * m.cols;
    uint16_t *const dst = m.dst + b * m.cols * m.padded;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = (threadIdx.x >> 3) + i * 32, c = (threadIdx.x & 7) * 8;
        u32x4 v = {0, 0, 0, 0};
        if (r0 + r < m.rows && c0 + c < m.cols) v = *(const u32x4 *)(src + (r0 + r) * m.cols + c0 + c);
#pragma unroll
        for (int k = 0; k < 4; ++k) *(uint32_t *)&t[r][c + 2 * k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = (threadIdx.x >> 3) + i * 32, r = (threadIdx.x & 7) * 8;
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (uint32_t)t[r + 2 * k][c] | (uint32_t)t[r + 2 * k + 1][c] << 16;
        if (c0 + c < m.cols && r0 + r < m.padded) *(u32x4 *)(dst + (c0 + c) * m.padded + r0 + r) = v;
    }
}

// out_c = Y_c^T S_c over the rows of a bucket.  A workgroup takes 64 columns of Y and 32 of S (the hi and the lo
// half of each); its four wavefronts take 32 rows at a time in turn, the next ones on their way while these are
// multiplied, bring them to LDS as they lie in memory and read both operands through the transpose read (k of the product
// runs down the rows).  Sums are added in wavefront order.  Where the columns leave the chip idle, the rows of a bucket
// are cut into `cuts` pieces of their own workgroups: fp32 sums to planes, added by a second launch in a fixed order.
constexpr int kOuterCols = 64, kOuterR = 32;
struct OuterJob {
    const uint16_t *y, *s2;
    uint16_t *out;
    float *planes;  // [cuts][C][D][R] (flat: [R][D]) where cuts > 1
    int D, flat, cuts, tiles;  // tiles: column tiles of Y
};
struct OuterJobs {
    OuterJob job[2];
    int first;  // the second one's first workgroup
};
__device__ __forceinline__ void grouped_outer_body(const OuterJob &m, int block, const int32_t *__restrict__ offsets,
                                                   const int32_t *__restrict__ perm, int C, int R, unsigned char *lds) {
    constexpr int YS = kOuterCols * 2 + 32, SS = kOuterR * 4 + 32;  // bytes per row in LDS
    constexpr int SLAB = 32 * (YS + SS);
    constexpr int PART = kOuterCols * (kOuterR + 1) * 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int kq = lane >> 4, l16 = lane & 15;
    const int D = m.D, parts = (R + kOuterR - 1) / kOuterR;
    const int d0 = block % m.tiles * kOuterCols, r0 = block / m.tiles % parts * kOuterR;
    const int cut = block / (m.tiles * parts) % m.cuts, c = block / (m.tiles * parts * m.cuts);
    int lo = offsets[c], hi = offsets[c + 1];
    if (m.cuts > 1) {  // pieces of whole steps
        const int per = ((hi - lo + m.cuts - 1) / m.cuts + 127) & ~127;
        lo = min(lo + cut * per, hi);
        hi = min(lo + per, hi);
    }
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
    u32x4 yv[4], sv[4];
    const int row = lane >> 3, col = (lane & 7) * 8;  // 8 rows at a time, 8 columns a lane
    const uint16_t *const y_col = m.y + min(d0 + col, D - 8), *const s_col = m.s2 + (col >> 5) * R + min(r0 + (col & 31), R - 8);
    auto load = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = min(p0 + i * 8 + row, hi - 1);
            yv[i] = *(const u32x4 *)(y_col + (int64_t)perm[p] * D);
            sv[i] = *(const u32x4 *)(s_col + (int64_t)p * 2 * R);
        }
    };
    int p0 = lo + wave * 32;
    if (p0 < hi) load(p0);
    for (; p0 < hi; p0 += 128) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (p0 + i * 8 + row >= hi) {  // rows of the next bucket count as zero, on both sides
                yv[i] = u32x4{0, 0, 0, 0};
                sv[i] = u32x4{0, 0, 0, 0};
            }
            *(u32x4 *)(ys + (i * 8 + row) * YS + col * 2) = yv[i];
            *(u32x4 *)(ss + (i * 8 + row) * SS + col * 2) = sv[i];
        }
        if (p0 + 128 < hi) load(p0 + 128);
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
        const int d = m.flat ? it % (kOuterCols / 2) * 2 : it / (kOuterR / 2), r = m.flat ? it / (kOuterCols / 2) : it % (kOuterR / 2) * 2;
        float v[2] = {0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                v[k] += ((const float *)(lds + w * PART))[(d + (m.flat ? k : 0)) * (kOuterR + 1) + r + (m.flat ? 0 : k)];
        if (d0 + d < D && r0 + r < R) {
            const int64_t at = m.flat ? ((int64_t)c * R + r0 + r) * D + d0 + d : ((int64_t)c * D + d0 + d) * R + r0 + r;
            if (m.cuts > 1)
                *(f32x2_t *)(m.planes + (int64_t)cut * C * D * R + at) = f32x2_t{v[0], v[1]};
            else
                *(uint32_t *)(m.out + at) = bf16x2_bits(v[0], v[1]);
        }
    }
}
__global__ __launch_bounds__(256) void grouped_outer_kernel(OuterJobs jobs, const int32_t *__restrict__ offsets,
                                                            const int32_t *__restrict__ perm, int C, int R) {
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * 32 * (kOuterCols * 2 + kOuterR * 4 + 64)];
    static_assert(32 * (kOuterCols * 2 + kOuterR * 4 + 64) >= kOuterCols * (kOuterR + 1) * 4, "the sums take the slabs' place");
    const bool second = (int)blockIdx.x >= jobs.first;
    grouped_outer_body(jobs.job[second ? 1 : 0], (int)blockIdx.x - (second ? jobs.first : 0), offsets, perm, C, R, lds);
}

// bf16 sums of fp32 planes, eight values to a thread; two arrays in one launch.
struct SumJob {
    const float *planes;
    uint16_t *out;
    int64_t n;  // values, a multiple of 8
    int planes_n;
};
struct SumJobs {
    SumJob job[2];
    int first;
};
__global__ __launch_bounds__(256) void sum_planes_kernel(SumJobs jobs) {
    const bool second = (int)blockIdx.x >= jobs.first;
    const SumJob &m = jobs.job[second ? 1 : 0];
    const int64_t at = ((int64_t)((int)blockIdx.x - (second ? jobs.first : 0)) * 256 + threadIdx.x) * 8;
    if (at >= m.n) return;
    f32x4 a = *(const f32x4 *)(m.planes + at), b = *(const f32x4 *)(m.planes + at + 4);
    for (int i = 1; i < m.planes_n; ++i) {
        a += *(const f32x4 *)(m.planes + i * m.n + at);
        b += *(const f32x4 *)(m.planes + i * m.n + at + 4);
    }
    const u32x2 lo = bf16x4_bits(a), hi = bf16x4_bits(b);
    *(u32x4 *)(m.out + at) = u32x4{lo[0], lo[1], hi[0], hi[1]};
}

int outer_cuts(int64_t N, int D, int C, int R) {
    const int64_t blocks = (int64_t)((D + kOuterCols - 1) / kOuterCols) * ((R + kOuterR - 1) / kOuterR) * C;
    // enough workgroups for two to a compute unit, and four steps of 128 rows to a piece of an average bucket
    int64_t cuts = 512 / blocks, most = N / ((int64_t)C * 512);
    if (cuts > most) cuts = most;
    return (int)(cuts < 1 ? 1 : cuts > 16 ? 16 : cuts);
}

}  // namespace

hipError_t launch_zero(void *dst, int64_t bytes, hipStream_t s) {
    const int64_t n = bytes / 16, blocks = (n + 255) / 256;
    if (n > 0)
        hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s, (u32x4 *)dst, n);
    return hipGetLastError();
}

hipError_t launch_gate(const float *planes, int count, uint16_t *z, float *pre, int64_t N, int F, int act, hipStream_t s) {
    const int64_t items = N * (F / 4), blocks = (items + 255) / 256;
    if (blocks >= (int64_t(1) << 24)) return hipErrorInvalidValue;
    if (blocks > 0) hipLaunchKernelGGL(gate_kernel, dim3((unsigned)blocks), dim3(256), 0, s, planes, count, z, pre, items, F, act);
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

hipError_t launch_transposes(const TransposeJob *jobs, int n, hipStream_t s) {
    if (n == 0) return hipSuccess;
    if (n > kMaxTransposes) return hipErrorInvalidValue;
    TransposeJobs all{};
    int64_t blocks = 0;
    for (int i = 0; i < kMaxTransposes; ++i) {
        all.first[i] = (int)blocks;
        if (i >= n) continue;
        all.job[i] = jobs[i];
        blocks += jobs[i].batch * ((jobs[i].cols + 63) / 64) * ((jobs[i].padded + 63) / 64);
        if (blocks >= (int64_t(1) << 24)) return hipErrorInvalidValue;
    }
    hipLaunchKernelGGL(transpose_kernel, dim3((unsigned)blocks), dim3(256), 0, s, all);
    return hipGetLastError();
}

size_t grouped_outer_floats(int64_t N, int D, int C, int R) {
    const int cuts = outer_cuts(N, D, C, R);
    return cuts > 1 ? (size_t)cuts * C * D * R : 0;
}

hipError_t launch_sum_planes(const float *planes, uint16_t *out, int64_t n, int count, hipStream_t s) {
    const int64_t blocks = (n + 2047) / 2048;
    if (blocks >= (int64_t(1) << 24)) return hipErrorInvalidValue;
    SumJobs jobs{};
    jobs.job[0] = SumJob{planes, out, n, count};
    jobs.first = (int)blocks;
    hipLaunchKernelGGL(sum_planes_kernel, dim3((unsigned)blocks), dim3(256), 0, s, jobs);
    return hipGetLastError();
}

hipError_t launch_grouped_outers(const GroupedOuter *want, int n, const int32_t *offsets, const int32_t *perm, int64_t N, int C,
                                 int R, hipStream_t s) {
    if (n < 1 || n > 2) return n == 0 ? hipSuccess : hipErrorInvalidValue;
    OuterJobs jobs{};
    SumJobs sums{};
    int64_t blocks = 0, sum_blocks = 0;
    int n_sums = 0;
    for (int i = 0; i < n; ++i) {
        OuterJob &m = jobs.job[i];
        m = OuterJob{want[i].y, want[i].s2, want[i].out, want[i].planes, want[i].D, want[i].flat ? 1 : 0, outer_cuts(N, want[i].D, C, R),
                     (want[i].D + kOuterCols - 1) / kOuterCols};
        if (i == 1) jobs.first = (int)blocks;
        blocks += (int64_t)m.tiles * ((R + kOuterR - 1) / kOuterR) * m.cuts * C;
        if (m.cuts > 1) {
            if (n_sums == 1) sums.first = (int)sum_blocks;
            sums.job[n_sums++] = SumJob{m.planes, m.out, (int64_t)C * m.D * R, m.cuts};
            sum_blocks += ((int64_t)C * m.D * R + 2047) / 2048;
        }
    }
    if (n == 1) jobs.first = (int)blocks;
    if (blocks >= (int64_t(1) << 24) || sum_blocks >= (int64_t(1) << 24)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(grouped_outer_kernel, dim3((unsigned)blocks), dim3(256), 0, s, jobs, offsets, perm, C, R);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || n_sums == 0) return e;
    if (n_sums == 1) sums.first = (int)sum_blocks;
    hipLaunchKernelGGL(sum_planes_kernel, dim3((unsigned)sum_blocks), dim3(256), 0, s, sums);
    return hipGetLastError();
}

}  // namespace molora
