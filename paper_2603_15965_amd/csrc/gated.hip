// The backward pass of the gated block z = act(g) u, [g | u] = h = x W + (x A_r) B_r, beside its GEMMs:
//
//     dh = [dz u act'(g) | dz act(g)],   dA_c = x_c^T (dh_c B_c^T),   dB_c = (x_c A_c)^T dh_c
#include <algorithm>

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
struct GateBackward {
    const uint16_t *dz;
    const float *pre;
    uint16_t *dh;
    int64_t N, items;
    int F, act;
};
__device__ __forceinline__ void gate_backward_body(const GateBackward &m, int64_t block) {
    const int64_t it = block * 256 + threadIdx.x;
    if (it >= m.items) return;
    const int F = m.F;
    const int per = F / 4;
    const int64_t row = it / per;
    const int col = (int)(it % per) * 4;
    uint16_t *out = m.dh + row * 2 * F + col;
    if (row >= m.N) {
        *(u32x2 *)out = u32x2{0, 0};
        *(u32x2 *)(out + F) = u32x2{0, 0};
        return;
    }
    const float *h = m.pre + row * 2 * F + col;
    const f32x4 g = *(const f32x4 *)h, u = *(const f32x4 *)(h + F);
    const u32x2 d2 = *(const u32x2 *)(m.dz + row * F + col);
    f32x4 dg, du;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float d = bf16_bits_to_f32((d2[i >> 1] >> (16 * (i & 1))) & 0xFFFF);
        float slope;
        const float p = gate_factor<true>(g[i], m.act, slope);
        dg[i] = d * u[i] * (p + g[i] * slope);
        du[i] = d * g[i] * p;
    }
    *(u32x2 *)out = bf16x4_bits(dg);
    *(u32x2 *)(out + F) = bf16x4_bits(du);
}

__global__ __launch_bounds__(256) void zero_kernel(u32x4 *__restrict__ dst, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) dst[i] = u32x4{0, 0, 0, 0};
}

// The first launch of a backward pass: dh, and matrices transposed, 64 x 64 elements at a time through LDS (a step of
// 515 tokens takes 4 us less than with two launches).  Rows and columns are multiples of 8 (rows of the padded side).
// (t is padded to 66: a column is read without bank conflicts.)
struct TransposeJobs {
    TransposeJob job[kMaxTransposes];
    int first[kMaxTransposes + 1];  // its first workgroup (past the last one: behind it); behind all: the gate's
};
__global__ __launch_bounds__(256) void gate_backward_kernel(GateBackward gate, TransposeJobs jobs) {
    __shared__ uint16_t t[64][66];
    if ((int)blockIdx.x >= jobs.first[kMaxTransposes]) {
        gate_backward_body(gate, (int)blockIdx.x - jobs.first[kMaxTransposes]);
        return;
    }
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
// runs down the rows).  Sums are added in wavefront order.
// A bucket of more than `rows` rows is cut into even pieces of their own workgroups, whose fp32 sums go to planes and are
// added by a second launch in a fixed order.  The launch has a piece for every bucket and then as many more as there
// can be (N / rows), whichever buckets turn out to be the long ones; `rows` is what the workgroups of a compute unit
// share evenly.  It is bound by reading dh and x: 8192 x 2048 -> 2 x 6144, 8 adapters of rank 16, level routing, 41 us
// (235 MB) and 5 for the sums.  16384 x 512 -> 2 x 1024, 48 of rank 128 and one of them for all tokens: 84 us, in whole buckets 129; with
// level routing cut buckets cost the second launch, 5 us.
// Where the buckets are short on average (kWideRows) and the columns many, the wavefronts take 64 columns of Y each instead,
// all rows and no sum: with one step of rows to a bucket three of four had nothing to do.  168 x 1792 -> 2 x 1536, 59 of
// rank 40: 33 -> 20 us; 8192 x 2048 -> 2 x 6144, 64 of rank 16: 72 -> 56; at 4096 rows and 64 skewed ones of rank 32 31 -> 35;
// up to 512 rows to a bucket nothing is gained.
constexpr int kOuterCols = 64, kOuterR = 32, kOuterRows = 1024, kWideRows = 128;
struct OuterJob {
    const uint16_t *y, *s2;
    uint16_t *out;
    float *planes;  // [2 extra][D][R] (flat: [R][D]): the further pieces, then the first ones of the same buckets
    int D, flat, tiles, rows, extra, wide;  // tiles: column tiles of Y
};
struct OuterJobs {
    OuterJob job[2];
    int first, first_sum;  // the second one's first workgroup, of the products and of the sums
};
// A piece of a bucket: its cut-th of n; `first`: the place of the bucket's second piece among all further ones.
struct Piece {
    int c, cut, n, first;
};
// The further piece j of all, or (j < 0) the first one of bucket c; c = -1: there are fewer.
__device__ __forceinline__ Piece find_piece(const int32_t *__restrict__ offsets, int C, int rows, int j, int c, int lane) {
    int before = 0;
    for (int c0 = 0; c0 < C; c0 += 64) {
        const int at = min(c0 + lane, C - 1), len = offsets[at + 1] - offsets[at];
        const int more = c0 + lane < C && len > 0 ? (len - 1) / rows : 0;
        int sum = more;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(sum, d);
            if (lane >= d) sum += up;
        }
        sum += before;
        const uint64_t here = __ballot(j < 0 ? c0 + lane == c : sum > j);
        if (here != 0) {
            const int l = __builtin_ctzll(here);
            const int n = __builtin_amdgcn_readlane(more, l) + 1, first = __builtin_amdgcn_readlane(sum, l) - n + 1;
            return Piece{c0 + l, j < 0 ? 0 : j - first + 1, n, first};
        }
        before = __builtin_amdgcn_readlane(sum, 63);
    }
    return Piece{-1, 0, 0, 0};
}
__device__ __forceinline__ void grouped_outer_body(const OuterJob &m, int block, const int32_t *__restrict__ offsets,
                                                   const int32_t *__restrict__ perm, int C, int R, unsigned char *lds) {
    constexpr int YS = kOuterCols * 2 + 32, SS = kOuterR * 4 + 32;  // bytes per row in LDS
    constexpr int SLAB = 32 * (YS + SS);
    constexpr int PART = kOuterCols * (kOuterR + 1) * 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int kq = lane >> 4, l16 = lane & 15;
    const int D = m.D, parts = (R + kOuterR - 1) / kOuterR;
    const int d0 = (block % m.tiles * (m.wide ? 4 : 1) + (m.wide ? wave : 0)) * kOuterCols, r0 = block / m.tiles % parts * kOuterR;
    const int p_at = block / (m.tiles * parts);
    Piece piece{p_at, 0, 1, 0};
    if (p_at >= C)
        piece = find_piece(offsets, C, m.rows, p_at - C, -1, lane);
    else if (offsets[p_at + 1] - offsets[p_at] > m.rows)
        piece = find_piece(offsets, C, m.rows, -1, p_at, lane);
    const int c = piece.c;
    if (c < 0) return;
    int lo = offsets[c], hi = offsets[c + 1];
    if (piece.n > 1) {  // pieces of whole steps
        const int per = ((hi - lo + piece.n - 1) / piece.n + 127) & ~127;
        lo = min(lo + piece.cut * per, hi);
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
    int p0 = m.wide ? lo : lo + wave * 32;
    const int step = m.wide ? 32 : 128;
    if (p0 < hi) load(p0);
    for (; p0 < hi; p0 += step) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (p0 + i * 8 + row >= hi) {  // rows of the next bucket count as zero, on both sides
                yv[i] = u32x4{0, 0, 0, 0};
                sv[i] = u32x4{0, 0, 0, 0};
            }
            *(u32x4 *)(ys + (i * 8 + row) * YS + col * 2) = yv[i];
            *(u32x4 *)(ss + (i * 8 + row) * SS + col * 2) = sv[i];
        }
        if (p0 + step < hi) load(p0 + step);
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
    constexpr int ITEMS = kOuterCols * kOuterR / 2;  // two neighbours of the output's rows each
    const int first_d = d0 - (m.wide ? wave * kOuterCols : 0);
    for (int at = tid; at < (m.wide ? 4 * ITEMS : ITEMS); at += 256) {
        const int it = at % ITEMS, from = at / ITEMS;
        int d = m.flat ? it % (kOuterCols / 2) * 2 : it / (kOuterR / 2), r = m.flat ? it / (kOuterCols / 2) : it % (kOuterR / 2) * 2;
        const int place = d * (kOuterR + 1) + r, next = m.flat ? kOuterR + 1 : 1;
        const float *const p = (const float *)(lds + from * PART) + place;
        float v[2] = {p[0], p[next]};
        if (!m.wide) {
#pragma unroll
            for (int w = 1; w < 4; ++w) {
                v[0] += ((const float *)(lds + w * PART))[place];
                v[1] += ((const float *)(lds + w * PART))[place + next];
            }
        }
        d += first_d + from * kOuterCols;
        if (d < D && r0 + r < R) {
            const int64_t to = m.flat ? (int64_t)(r0 + r) * D + d : (int64_t)d * R + r0 + r, all = (int64_t)D * R;
            if (piece.n > 1)
                *(f32x2_t *)(m.planes + (piece.cut > 0 ? piece.first + piece.cut - 1 : m.extra + piece.first) * all + to) = f32x2_t{v[0], v[1]};
            else
                *(uint32_t *)(m.out + c * all + to) = bf16x2_bits(v[0], v[1]);
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

// bf16 sums of fp32 planes, eight values to a thread.
__global__ __launch_bounds__(256) void sum_planes_kernel(const float *__restrict__ planes, uint16_t *__restrict__ out, int64_t n,
                                                         int count) {
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= n) return;
    f32x4 a = *(const f32x4 *)(planes + at), b = *(const f32x4 *)(planes + at + 4);
    for (int i = 1; i < count; ++i) {
        a += *(const f32x4 *)(planes + i * n + at);
        b += *(const f32x4 *)(planes + i * n + at + 4);
    }
    const u32x2 lo = bf16x4_bits(a), hi = bf16x4_bits(b);
    *(u32x4 *)(out + at) = u32x4{lo[0], lo[1], hi[0], hi[1]};
}
// The same of the pieces of the buckets that were cut: 2048 values to the workgroup of a bucket's second piece.
__global__ __launch_bounds__(256) void sum_pieces_kernel(OuterJobs jobs, const int32_t *__restrict__ offsets, int C, int R) {
    const bool second = (int)blockIdx.x >= jobs.first_sum;
    const OuterJob &m = jobs.job[second ? 1 : 0];
    const int block = (int)blockIdx.x - (second ? jobs.first_sum : 0);
    const int64_t n = (int64_t)m.D * R;
    const int chunks = (int)((n + 2047) / 2048);
    const Piece piece = find_piece(offsets, C, m.rows, block / chunks, -1, threadIdx.x & 63);
    const int64_t at = ((int64_t)(block % chunks) * 256 + threadIdx.x) * 8;
    if (piece.c < 0 || piece.cut != 1 || at >= n) return;
    const float *p = m.planes + (m.extra + piece.first) * n + at;
    f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
    p = m.planes + piece.first * n + at;
    for (int i = 1; i < piece.n; ++i, p += n) {
        a += *(const f32x4 *)p;
        b += *(const f32x4 *)(p + 4);
    }
    const u32x2 lo = bf16x4_bits(a), hi = bf16x4_bits(b);
    *(u32x4 *)(m.out + piece.c * n + at) = u32x4{lo[0], lo[1], hi[0], hi[1]};
}

// workgroups of a piece
int64_t outer_tiles(int D, int R) { return (int64_t)((D + kOuterCols - 1) / kOuterCols) * ((R + kOuterR - 1) / kOuterR); }
// columns of Y to a workgroup, in tiles: where the buckets are short on average and the columns many, one for each wavefront
bool outer_wide(int64_t N, int D, int C, int R) { return N <= (int64_t)C * kWideRows && outer_tiles(D, R) * C > 1024; }
// rows of a piece: so many that two workgroups to a compute unit share all rows, and eight steps at least
int outer_rows(int64_t N, int D, int R) {
    const int64_t rows = (N * outer_tiles(D, R) + 511) / 512;
    return (int)(rows <= kOuterRows ? kOuterRows : (rows + 127) / 128 * 128);
}
// workgroups of an outer product, of the sums behind it, and of matrices transposed
int64_t outer_blocks(int64_t N, int D, int C, int R) {
    const int64_t tiles = outer_wide(N, D, C, R) ? ((D + kOuterCols - 1) / kOuterCols + 3) / 4 : (D + kOuterCols - 1) / kOuterCols;
    return tiles * ((R + kOuterR - 1) / kOuterR) * (C + N / outer_rows(N, D, R));
}
int64_t sum_blocks(int64_t N, int D, int R) { return ((int64_t)D * R + 2047) / 2048 * (N / outer_rows(N, D, R)); }
int64_t transpose_blocks(int64_t batch, int64_t cols, int64_t padded) { return batch * ((cols + 63) / 64) * ((padded + 63) / 64); }
constexpr int64_t kMaxBlocks = int64_t(1) << 24;  // of 256 threads: the runtime counts a launch's threads in 32 bits

}  // namespace

hipError_t launch_zero(void *dst, int64_t bytes, hipStream_t s) {
    const int64_t n = bytes / 16, blocks = (n + 255) / 256;
    if (n > 0)
        hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s, (u32x4 *)dst, n);
    return hipGetLastError();
}

hipError_t launch_gate(const float *planes, int count, uint16_t *z, float *pre, int64_t N, int F, int act, hipStream_t s) {
    const int64_t items = N * (F / 4), blocks = (items + 255) / 256;
    if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
    if (blocks > 0) hipLaunchKernelGGL(gate_kernel, dim3((unsigned)blocks), dim3(256), 0, s, planes, count, z, pre, items, F, act);
    return hipGetLastError();
}

hipError_t launch_gate_backward(const uint16_t *dz, const float *pre, uint16_t *dh, int64_t N, int64_t padded, int F,
                                int act, const TransposeJob *jobs, int n, hipStream_t s) {
    if (n > kMaxTransposes) return hipErrorInvalidValue;
    TransposeJobs all{};
    int64_t blocks = 0;
    for (int i = 0; i < kMaxTransposes; ++i) {
        all.first[i] = (int)blocks;
        if (i >= n) continue;
        all.job[i] = jobs[i];
        blocks += transpose_blocks(jobs[i].batch, jobs[i].cols, jobs[i].padded);
        if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
    }
    all.first[kMaxTransposes] = (int)blocks;
    const GateBackward gate{dz, pre, dh, N, padded * (F / 4), F, act};
    blocks += (gate.items + 255) / 256;
    if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
    hipLaunchKernelGGL(gate_backward_kernel, dim3((unsigned)blocks), dim3(256), 0, s, gate, all);
    return hipGetLastError();
}

bool gated_backward_sizes_ok(int64_t N, int64_t padded, int d_in, int F, int C, int R) {
    const int64_t turned = transpose_blocks(C, 2 * (int64_t)F, R) + transpose_blocks(C, R, d_in) + transpose_blocks(1, d_in, padded);
    if (turned + (padded * (F / 4) + 255) / 256 >= kMaxBlocks) return false;
    return C == 0 || (outer_blocks(N, d_in, C, R) + outer_blocks(N, 2 * F, C, R) < kMaxBlocks && sum_blocks(N, d_in, R) + sum_blocks(N, 2 * F, R) < kMaxBlocks);
}

size_t grouped_outer_floats(int64_t N, int D, int R) {  // (never less for more rows: what outer_rows gives at most)
    return (size_t)(std::min(N / kOuterRows, 512 / outer_tiles(D, R)) * 2) * D * R;
}

hipError_t launch_sum_planes(const float *planes, uint16_t *out, int64_t n, int count, hipStream_t s) {
    const int64_t blocks = (n + 2047) / 2048;
    if (blocks >= kMaxBlocks) return hipErrorInvalidValue;
    hipLaunchKernelGGL(sum_planes_kernel, dim3((unsigned)blocks), dim3(256), 0, s, planes, out, n, count);
    return hipGetLastError();
}

hipError_t launch_grouped_outers(const GroupedOuter *want, int n, const int32_t *offsets, const int32_t *perm, int64_t N, int C,
                                 int R, hipStream_t s) {
    if (n < 1 || n > 2) return n == 0 ? hipSuccess : hipErrorInvalidValue;
    OuterJobs jobs{};
    int64_t blocks = 0, sums = 0;
    for (int i = 0; i < n; ++i) {
        OuterJob &m = jobs.job[i];
        const int rows = outer_rows(N, want[i].D, R), extra = (int)(N / rows);
        const int tiles = (want[i].D + kOuterCols - 1) / kOuterCols;
        const bool wide = outer_wide(N, want[i].D, C, R);
        m = OuterJob{want[i].y, want[i].s2, want[i].out, want[i].planes, want[i].D, want[i].flat ? 1 : 0,
                     wide ? (tiles + 3) / 4 : tiles, rows, extra, wide ? 1 : 0};
        blocks += outer_blocks(N, m.D, C, R);
        sums += sum_blocks(N, m.D, R);
        if (i == 0) jobs.first = (int)blocks, jobs.first_sum = (int)sums;
        if (blocks >= kMaxBlocks || sums >= kMaxBlocks) return hipErrorInvalidValue;
    }
    hipLaunchKernelGGL(grouped_outer_kernel, dim3((unsigned)blocks), dim3(256), 0, s, jobs, offsets, perm, C, R);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || sums == 0) return e;
    hipLaunchKernelGGL(sum_pieces_kernel, dim3((unsigned)sums), dim3(256), 0, s, jobs, offsets, C, R);
    return hipGetLastError();
}

}  // namespace molora
