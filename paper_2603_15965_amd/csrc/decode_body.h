// A batch of at most 64 tokens in token order: which tokens share an adapter is a ballot over the batch's 64
// targets, taken wherever it is needed, so nothing waits for a sort.  Shared by the decode steps on a 4-bit base
// weight and of the gated block.
#pragma once
#include "../../include/molora.h"
#include "common.h"

namespace molora {

// x_i A_{r(i)} comes in this many slices of K at most: planes [slices][64][R] fp32
constexpr int kMaxSlices = 4;

namespace {

// The adapter of place j: the j-th among the batch's distinct ones in the order of their first token; -1: fewer
// than that.  `mine`: its tokens.  target: the lane's token's, -1 without.
__device__ __forceinline__ int place_adapter(int target, int place, uint64_t &mine) {
    uint64_t left = __ballot(target >= 0);
    int c = -1;
    mine = 0;
    for (int j = 0; j <= place && left != 0; ++j) {
        c = __builtin_amdgcn_readlane(target, __builtin_ctzll(left));
        mine = __ballot(target == c);
        left &= ~mine;
        if (j < place) c = -1;
    }
    return c;
}
__device__ __forceinline__ int target_of(const int32_t *r, int i, int N, int C) {
    if (i >= N) return -1;
    const int c = r[i];
    return c >= 0 && c < C ? c : -1;
}

constexpr int kShrinkCols = 32, kSlabStride = kShrinkCols * 2 + 32;  // bytes of a row of A in LDS: distinct banks

// t = x A_c of one adapter's tokens for 32 columns of A_c over one slice of K.  Four wavefronts take steps of 32 k
// in turn, four of them in flight; A comes in rows of k and is turned by the transpose read.
__device__ __forceinline__ void decode_shrink_body(int block, const uint16_t *__restrict__ x, const uint16_t *__restrict__ A,
                                                   const int32_t *__restrict__ r, float *__restrict__ planes, int N, int d_in,
                                                   int C, int R, int slices, unsigned char *lds) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kq = lane >> 4, l16 = lane & 15;
    const int groups = (R + kShrinkCols - 1) / kShrinkCols;
    const int slice = block % slices, g = block / slices % groups;
    uint64_t mine;
    const int c = place_adapter(target_of(r, lane, N, C), block / (slices * groups), mine);
    if (c < 0) return;
    const int count = __popcll(mine), tiles = (count + 15) / 16;
    // lane -> its token in each row tile (past the last: the last one again, not stored)
    int tok[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int want = min(i * 16 + l16, count - 1);
        int at = 0;  // position of the want-th bit
#pragma unroll
        for (int width = 32; width > 0; width >>= 1) {
            const int below = __popcll(mine & ((uint64_t(1) << (at + width)) - 1));
            if (below <= want) at += width;
        }
        tok[i] = min(at, 63);
    }
    const int steps = (d_in + 31) / 32, per = (steps + slices - 1) / slices;
    const int end = min((slice + 1) * per, steps);
    f32x4 acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    unsigned char *const slab = lds + wave * 32 * kSlabStride;
    const uint16_t *const Ac = A + (int64_t)c * d_in * R;
    for (int st = slice * per + wave; st < end; st += 16) {
        u32x4 a[4][2];
        i16x8 xv[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k0 = min(st + u * 4, steps - 1) * 32;
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int row = lane / 4 + v * 16, col = g * kShrinkCols + lane % 4 * 8;
                a[u][v] = *(const u32x4 *)(Ac + (int64_t)min(k0 + row, d_in - 1) * R + min(col, R - 8));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < tiles) xv[u][i] = *(const i16x8 *)(x + (int64_t)tok[i] * d_in + min(k0 + kq * 8, d_in - 8));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int s = st + u * 4;
            if (s >= end) break;
#pragma unroll
            for (int v = 0; v < 2; ++v) *(u32x4 *)(slab + (lane / 4 + v * 16) * kSlabStride + lane % 4 * 16) = a[u][v];
            bf16x8 fa[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const unsigned char *p = slab + (kq * 8 + (l16 >> 2)) * kSlabStride + j * 32 + (l16 & 3) * 8;
                const i16x4 v0 = lds_read_tr16((const MOLORA_LDS void *)p), v1 = lds_read_tr16((const MOLORA_LDS void *)(p + 4 * kSlabStride));
                fa[j] = __builtin_bit_cast(bf16x8, i16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]});
            }
            const bool in = s * 32 + kq * 8 < d_in;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= tiles) break;
                const i16x8 xf = in ? xv[u][i] : i16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[j], __builtin_bit_cast(bf16x8, xf), acc[i][j], 0, 0, 0);
            }
        }
    }
    __syncthreads();
    f32x4 *const part = (f32x4 *)lds;  // [wave][tile][column block][lane]
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) part[((wave * 4 + i) * 2 + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    // one row tile to a wavefront
    if (wave < tiles) {
        int row = tok[0];  // (a register array wants a constant index)
#pragma unroll
        for (int i = 1; i < 4; ++i) row = wave == i ? tok[i] : row;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            f32x4 sum = part[(wave * 2 + j) * 64 + lane];
#pragma unroll
            for (int w = 1; w < 4; ++w) sum += part[((w * 4 + wave) * 2 + j) * 64 + lane];
            const int col = g * kShrinkCols + j * 16 + kq * 4;
            if (wave * 16 + l16 < count && col < R) *(f32x4 *)(planes + ((int64_t)slice * 64 + row) * R + col) = sum;
        }
    }
}

constexpr int kDecodeShrinkLds = 4 * 4 * 2 * 64 * 16;  // the partial sums; the slabs of A take less
static_assert(4 * 32 * kSlabStride <= kDecodeShrinkLds, "slabs");

// As many slices of K as leave a workgroup to one and a half compute units, and a slice 512 k
inline int decode_slices(int64_t N, int d_in, int C, int rank) {
    const int64_t blocks = (N < C ? N : C) * ((rank + kShrinkCols - 1) / kShrinkCols);
    int64_t s = blocks > 0 ? 384 / blocks : 1;
    if (s > d_in / 512) s = d_in / 512;
    return (int)(s < 1 ? 1 : s > kMaxSlices ? kMaxSlices : s);
}
inline int decode_shrink_blocks(int64_t N, int d_in, int C, int rank) {
    return (int)(N < C ? N : C) * ((rank + kShrinkCols - 1) / kShrinkCols) * decode_slices(N, d_in, C, rank);
}

// The batch's adapters, one to a lane, with their tokens.
struct BatchAdapters {
    int c = 0, n = 0;
    uint64_t mine = 0;
    __device__ __forceinline__ void find(int target, int lane) {
        for (uint64_t left = __ballot(target >= 0); left != 0; ++n) {
            const int first = __builtin_amdgcn_readlane(target, __builtin_ctzll(left));
            const uint64_t own = __ballot(target == first);
            left &= ~own;
            if (lane == n) {
                c = first;
                mine = own;
            }
        }
    }
    // slab `turn`: 16 rows of the B of an adapter, `parts` to each
    __device__ __forceinline__ void slab(int turn, int parts, int &adapter, int &part, uint64_t &tokens) const {
        const int at = turn / parts;
        part = turn - at * parts;
        adapter = __builtin_amdgcn_readlane(c, at);
        tokens = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), at) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)mine, at);
    }
};

// t of NR * 16 rows, the slices added, as bf16 halves [hi | lo] to LDS; zeros where there is no adapter.  512 threads.
// (Two halves, as in the larger batches: the product takes bf16 operands, and what a third half would hold is 2^-16 of
// t at most; h of 64 x 4096 -> 12288 is 6e-7 of its norm off, 8e-8 with t in fp32.)
inline __host__ __device__ constexpr int t_row_bytes(int R) { return 4 * R + 16; }  // (+16: bank shift)
template <int NR>
__device__ __forceinline__ void t_to_lds(const float *__restrict__ planes, int slices, int target, int R, unsigned char *t_lds) {
    constexpr int ITEMS = (NR * 16 * (MOLORA_MAX_RANK / 8) + 511) / 512;  // eight columns of a row
    const int tid = threadIdx.x, lane = tid & 63;
    const int per_row = R / 8, items = NR * 16 * per_row;
    const uint64_t routed = __ballot(target >= 0);  // the tokens with an adapter (asked of all lanes: a lane that is off has no answer)
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        const int it = min(tid + u * 512, items - 1), row = it / per_row, col = it % per_row * 8;
        f32x4 v[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
        if (tid + u * 512 - lane >= items) break;  // nothing left for the wavefront
#pragma unroll
        for (int sl = 0; sl < kMaxSlices; ++sl) {
            const float *p = planes + ((int64_t)min(sl, slices - 1) * 64 + row) * R + col;
            const f32x4 v0 = *(const f32x4 *)p, v1 = *(const f32x4 *)(p + 4);
            if (sl < slices) {
                v[0] += v0;
                v[1] += v1;
            }
        }
        const bool own = routed >> row & 1;
        u32x4 hi, lo;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t h2[2], l2[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float f = own ? v[k >> 1][(k & 1) * 2 + e] : 0.f;
                h2[e] = f32_to_bf16_bits(f);
                l2[e] = f32_to_bf16_bits(f - bf16_bits_to_f32(h2[e]));
            }
            hi[k] = h2[0] | h2[1] << 16;
            lo[k] = l2[0] | l2[1] << 16;
        }
        if (tid + u * 512 < items) {
            *(u32x4 *)(t_lds + row * t_row_bytes(R) + col * 2) = hi;
            *(u32x4 *)(t_lds + row * t_row_bytes(R) + (R + col) * 2) = lo;
        }
    }
}
// 16 columns of t from column k0 on, of row tile i, as [hi | lo] (the operand against 16 rows of B twice); rows
// that are not among `tokens` count as zero
__device__ __forceinline__ bf16x8 t_operand(const unsigned char *t_lds, int i, int k0, int R, uint64_t tokens, int lane) {
    const int kq = lane >> 4, row = i * 16 + (lane & 15), kc = k0 + (kq & 1) * 8;
    i16x8 v = *(const i16x8 *)(t_lds + row * t_row_bytes(R) + ((kq >> 1) * R + min(kc, R - 8)) * 2);
    if (!(tokens >> row & 1) || kc >= R) v = i16x8{0, 0, 0, 0, 0, 0, 0, 0};
    return __builtin_bit_cast(bf16x8, v);
}
// What a lane keeps of a product with the B of an adapter whose tokens these are: row tile i's sum for a row of the
// adapter, what was there before for any other
__device__ __forceinline__ f32x4 own_row(uint64_t tokens, int i, int lane, f32x4 sum, f32x4 before) {
    return tokens >> (i * 16 + (lane & 15)) & 1 ? sum : before;
}
// the columns [16] x 8 k of a slab that lies k-row by k-row in LDS, k-rows 8 kg .. 8 kg + 7 from p on
__device__ __forceinline__ bf16x8 turned(const unsigned char *slab, int stride, int kg, int col_bytes, int lane) {
    const unsigned char *p = slab + (kg * 8 + ((lane & 15) >> 2)) * stride + col_bytes + (lane & 3) * 8;
    const i16x4 v0 = lds_read_tr16((const MOLORA_LDS void *)p), v1 = lds_read_tr16((const MOLORA_LDS void *)(p + 4 * stride));
    return __builtin_bit_cast(bf16x8, i16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]});
}

}  // namespace
}  // namespace molora
