// The routed projection of at most 64 tokens on a 4-bit base weight, in two launches.  Such a step is one read of
// the codes of W and of the adapters in use, so everything runs in token order and nothing waits for a sort:
// which tokens share an adapter is a ballot over the batch's 64 targets, taken wherever it is needed.
//
//   first   x to codes, beside t = x A_r in slices of K (fp32 partial sums): both only read x, and the handful
//           of adapters in use alone would leave most of the chip idle
//   second  h = Q(x) Q(W) + t B_r, the slices of t added on the way
#include <type_traits>

#include "mx_mfma.h"
#include "mx_quant_body.h"

namespace molora {

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

constexpr int kFirstLds = 4 * 4 * 2 * 64 * 16;  // the partial sums; the slabs of A and the scales take less
static_assert(4 * 32 * kSlabStride <= kFirstLds, "slabs");

__global__ __launch_bounds__(256) void mx_decode_first_kernel(const uint16_t *__restrict__ x, const uint16_t *__restrict__ A,
                                                              const int32_t *__restrict__ r, uint8_t *__restrict__ codes,
                                                              uint8_t *__restrict__ scales, float *__restrict__ planes, int N,
                                                              int d_in, int C, int R, int slices, int shrink_blocks, int kt_n,
                                                              int kg_n) {
    __shared__ __attribute__((aligned(16))) unsigned char lds[kFirstLds];
    if ((int)blockIdx.x < shrink_blocks)  // (the longer ones first)
        decode_shrink_body((int)blockIdx.x, x, A, r, planes, N, d_in, C, R, slices, lds);
    else
        mx_quantize_body<false>((int)blockIdx.x - shrink_blocks, x, nullptr, codes, scales, N, d_in, kt_n, kg_n, lds);
}

// A workgroup owns CT * 16 columns.  Its eight wavefronts take groups of 512 k of W in turn, straight from memory into
// registers (a code tile is 1 KB, contiguous), then slabs of 16 rows of the B_c in use in turn, and add their
// sums in LDS in a fixed order.  Every trip to memory that depends on no other is sent for before the first is waited
// for: the slices of t, the first codes, the targets, then the first slabs of B.
template <int NR, int CT>
struct DecodeLds {
    static constexpr int PART = CT * NR * 1024;  // a wavefront's sums; before, the slab of B that it turns
    static constexpr int STRIDE = CT * 32 + 32;  // bytes of a row of that slab: distinct banks
    static_assert(16 * STRIDE <= PART, "slab");
    static __host__ __device__ constexpr int t_stride(int R) { return 4 * R + 16; }
    static constexpr int bytes(int R) { return 8 * PART + NR * 16 * t_stride(R); }
};

template <int NR, int CT>
__global__ __launch_bounds__(512, 2) void mx_decode_kernel(const uint8_t *__restrict__ xc, const uint8_t *__restrict__ xs,
                                                           const uint8_t *__restrict__ wc, const uint8_t *__restrict__ ws,
                                                           const uint16_t *__restrict__ B, const int32_t *__restrict__ r,
                                                           const float *__restrict__ planes, float *__restrict__ h, int N, int d_out,
                                                           int kt_n, int kg_n, int C, int R, int slices) {
    using Lds = DecodeLds<NR, CT>;
    constexpr int STRIDE = Lds::STRIDE, LPR = CT * 2, LOADS = (16 * LPR + 63) / 64;  // 16-byte chunks of a row, loads of a slab
    constexpr int ITEMS = (NR * 16 * (MOLORA_MAX_RANK / 8) + 511) / 512;             // eight columns of a row of t
    constexpr int BATCH = 4;                                                         // slabs of a wavefront in flight
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kq = lane >> 4, l16 = lane & 15;
    const int64_t ct0 = (int64_t)blockIdx.x * CT, ct_last = (d_out + 15) / 16 - 1, n0 = ct0 * 16;
    const int t_stride = Lds::t_stride(R);
    unsigned char *const t_lds = lds + 8 * Lds::PART;
    f32x4 acc[CT][NR];
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
        for (int i = 0; i < NR; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};

    int target = -1;
    if (C > 0) target = target_of(r, lane, N, C);
    u32x4 w[CT][4], x[NR][4];
    uint32_t sw[CT], sx[NR];
    auto load = [&](int kg) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < CT; ++j) {
            const int64_t ct = min(ct0 + j, ct_last);
            sw[j] = *(const uint32_t *)(ws + ((ct * kg_n + kg) * 64 + lane) * 4);
#pragma unroll
            for (int q = 0; q < 4; ++q)  // past the last k tile: that one again, not multiplied
                w[j][q] = *(const u32x4 *)(wc + ((ct * kt_n + min(kg * 4 + q, kt_n - 1)) * 64 + lane) * 16);
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            sx[i] = *(const uint32_t *)(xs + (((int64_t)i * kg_n + kg) * 64 + lane) * 4);
#pragma unroll
            for (int q = 0; q < 4; ++q) x[i][q] = *(const u32x4 *)(xc + (((int64_t)i * kt_n + min(kg * 4 + q, kt_n - 1)) * 64 + lane) * 16);
        }
    };
    auto multiply = [&](int kg) __attribute__((always_inline)) {
        auto tile = [&](auto q_c) __attribute__((always_inline)) {
            constexpr int Q = decltype(q_c)::value;
            if (kg * 4 + Q >= kt_n) return;
#pragma unroll
            for (int i = 0; i < NR; ++i)
#pragma unroll
                for (int j = 0; j < CT; ++j) acc[j][i] = mx_mfma<Q>(w[j][Q], x[i][Q], acc[j][i], sw[j], sx[i]);
        };
        tile(std::integral_constant<int, 0>{});
        tile(std::integral_constant<int, 1>{});
        tile(std::integral_constant<int, 2>{});
        tile(std::integral_constant<int, 3>{});
    };
    int kg = wave;
    if (C == 0) {
        for (; kg < kg_n; kg += 8) {
            load(kg);
            multiply(kg);
        }
    } else {
        // ---- the batch's adapters, one to a lane, with their tokens ----
        int list_c = 0, n_list = 0;
        uint64_t list_mine = 0;
        const int parts = (R + 15) / 16;
        u32x4 b[BATCH][LOADS];
        auto slab_of = [&](int turn, int &c, int &q, uint64_t &mine) __attribute__((always_inline)) {
            const int at = turn / parts;
            q = turn - at * parts;
            c = __builtin_amdgcn_readlane(list_c, at);
            mine = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(list_mine >> 32), at) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)list_mine, at);
        };
        auto load_slabs = [&](int turn) __attribute__((always_inline)) {  // (past the last one: that one again)
#pragma unroll
            for (int s = 0; s < BATCH; ++s) {
                int c, q;
                uint64_t mine;
                slab_of(min(turn + s * 8, n_list * parts - 1), c, q, mine);
#pragma unroll
                for (int u = 0; u < LOADS; ++u) {
                    const int at = lane + u * 64, row = min(at / LPR, 15);
                    b[s][u] = *(const u32x4 *)(B + ((int64_t)c * R + min(q * 16 + row, R - 1)) * d_out + min(n0 + at % LPR * 8, (int64_t)d_out - 8));
                }
            }
        };
        if (kg < kg_n) load(kg);
        for (uint64_t left = __ballot(target >= 0); left != 0; ++n_list) {
            const int c = __builtin_amdgcn_readlane(target, __builtin_ctzll(left));
            const uint64_t mine = __ballot(target == c);
            left &= ~mine;
            if (lane == n_list) {
                list_c = c;
                list_mine = mine;
            }
        }
        if (n_list > 0) load_slabs(wave);
        // ---- t: the slices added, bf16 halves [hi | lo] to LDS, zeros where there is no adapter ----
        const int per_row = R / 8, items = NR * 16 * per_row;
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) {
            const int it = min(tid + u * 512, items - 1), row = it / per_row, col = it % per_row * 8;
            f32x4 v[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
            if (tid + u * 512 - lane >= items) break;  // nothing left for the wavefront
#pragma unroll
            for (int sl = 0; sl < kMxMaxSlices; ++sl) {
                const float *p = planes + ((int64_t)min(sl, slices - 1) * 64 + row) * R + col;
                const f32x4 v0 = *(const f32x4 *)p, v1 = *(const f32x4 *)(p + 4);
                if (sl < slices) {
                    v[0] += v0;
                    v[1] += v1;
                }
            }
            const bool own = row < N && __shfl(target, row & 63) >= 0;
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
                *(u32x4 *)(t_lds + row * t_stride + col * 2) = hi;
                *(u32x4 *)(t_lds + row * t_stride + (R + col) * 2) = lo;
            }
        }
        while (kg < kg_n) {
            multiply(kg);
            kg += 8;
            if (kg < kg_n) load(kg);
        }
        __syncthreads();
        // ---- expand ----
        unsigned char *const slab = lds + wave * Lds::PART;  // the wavefront's own until its sums go there
        for (int turn = wave; turn < n_list * parts; turn += 8 * BATCH) {
            u32x4 now[BATCH][LOADS];
#pragma unroll
            for (int s = 0; s < BATCH; ++s)
#pragma unroll
                for (int u = 0; u < LOADS; ++u) now[s][u] = b[s][u];
            if (turn + 8 * BATCH < n_list * parts) load_slabs(turn + 8 * BATCH);
#pragma unroll
            for (int s = 0; s < BATCH; ++s) {
                if (turn + s * 8 >= n_list * parts) break;
                int c, q;
                uint64_t mine;
                slab_of(turn + s * 8, c, q, mine);
#pragma unroll
                for (int u = 0; u < LOADS; ++u) {
                    const int at = lane + u * 64;
                    if (at < 16 * LPR) *(u32x4 *)(slab + at / LPR * STRIDE + at % LPR * 16) = now[s][u];
                }
                // 16 columns of t as [hi | lo] against the slab twice
                const int kc = q * 16 + (kq & 1) * 8;
                bf16x8 t[NR];
#pragma unroll
                for (int i = 0; i < NR; ++i) {
                    const int row = i * 16 + l16;
                    i16x8 v = *(const i16x8 *)(t_lds + row * t_stride + ((kq >> 1) * R + min(kc, R - 8)) * 2);
                    if (!(mine >> row & 1) || kc >= R) v = i16x8{0, 0, 0, 0, 0, 0, 0, 0};
                    t[i] = __builtin_bit_cast(bf16x8, v);
                }
#pragma unroll
                for (int j = 0; j < CT; ++j) {
                    const unsigned char *p = slab + ((kq & 1) * 8 + (l16 >> 2)) * STRIDE + j * 32 + (l16 & 3) * 8;
                    const i16x4 v0 = lds_read_tr16((const MOLORA_LDS void *)p), v1 = lds_read_tr16((const MOLORA_LDS void *)(p + 4 * STRIDE));
                    const bf16x8 fb = __builtin_bit_cast(bf16x8, i16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]});
#pragma unroll
                    for (int i = 0; i < NR; ++i) acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb, t[i], acc[j][i], 0, 0, 0);
                }
            }
        }
    }

#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
        for (int i = 0; i < NR; ++i) *(f32x4 *)(lds + wave * Lds::PART + ((j * NR + i) * 64 + lane) * 16) = acc[j][i];
    __syncthreads();
    for (int f = wave; f < CT * NR; f += 8) {
        f32x4 sum = *(const f32x4 *)(lds + (f * 64 + lane) * 16);
#pragma unroll
        for (int v = 1; v < 8; ++v) sum += *(const f32x4 *)(lds + v * Lds::PART + (f * 64 + lane) * 16);
        const int row = f % NR * 16 + l16;
        const int64_t col = (ct0 + f / NR) * 16 + kq * 4;
        if (row < N && col < d_out) *(f32x4 *)(h + (int64_t)row * d_out + col) = sum;
    }
}

template <int NR, int CT>
struct DecodeKernel {
    static inline LdsRegistrar lds{(const void *)mx_decode_kernel<NR, CT>, (size_t)DecodeLds<NR, CT>::bytes(MOLORA_MAX_RANK)};
};
template <int NR, int CT, class... Args>
void launch_decode(unsigned blocks, int rank, hipStream_t s, Args... args) {
    (void)&DecodeKernel<NR, CT>::lds;  // instantiates the registration
    constexpr auto kernel = mx_decode_kernel<NR, CT>;
    const int bytes = DecodeLds<NR, CT>::bytes(rank);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(512), bytes, s, args...);
}

}  // namespace

// As many slices of K as leave a workgroup to a compute unit and half, and a slice 512 k
int mx_decode_slices(int64_t N, int d_in, int C, int rank) {
    const int64_t blocks = (N < C ? N : C) * ((rank + kShrinkCols - 1) / kShrinkCols);
    int64_t s = blocks > 0 ? 384 / blocks : 1;
    if (s > d_in / 512) s = d_in / 512;
    return (int)(s < 1 ? 1 : s > kMxMaxSlices ? kMxMaxSlices : s);
}

hipError_t launch_mx_decode_first(const uint16_t *x, const uint16_t *A, const int32_t *r, uint8_t *codes, uint8_t *scales,
                                  float *planes, int64_t N, int d_in, int C, int rank, hipStream_t s) {
    if (N < 1 || N > 64) return hipErrorInvalidValue;
    const int slices = mx_decode_slices(N, d_in, C, rank), kg = mx_k_groups(d_in);
    const int shrink = (int)(N < C ? N : C) * ((rank + kShrinkCols - 1) / kShrinkCols) * slices;
    const unsigned blocks = (unsigned)(shrink + mx_row_tiles(N) * kg);
    hipLaunchKernelGGL(mx_decode_first_kernel, dim3(blocks), dim3(256), 0, s, x, A, r, codes, scales, planes, (int)N, d_in, C,
                       rank, slices, shrink, mx_k_tiles(d_in), kg);
    return hipGetLastError();
}

hipError_t launch_mx_decode(const uint8_t *xc, const uint8_t *xs, const uint8_t *wc, const uint8_t *ws, const uint16_t *B,
                            const int32_t *r, const float *planes, float *h, int64_t N, int d_in, int d_out, int C, int rank,
                            hipStream_t s) {
    if (N < 1 || N > 64) return hipErrorInvalidValue;
    const int kt = mx_k_tiles(d_in), kg = mx_k_groups(d_in), slices = C > 0 ? mx_decode_slices(N, d_in, C, rank) : 1;
    const int64_t tiles = ((int64_t)d_out + 15) / 16;
    // as many columns to a workgroup as leave one for every compute unit: what else would run in its place would
    // read all of x and of t again
    const int ct = tiles <= 256 ? 1 : tiles <= 512 ? 2 : 3;
    const unsigned blocks = (unsigned)((tiles + ct - 1) / ct);
#define MOLORA_MX_DECODE(NR, CT) launch_decode<NR, CT>(blocks, rank, s, xc, xs, wc, ws, B, r, planes, h, (int)N, d_out, kt, kg, C, rank, slices)
#define MOLORA_MX_DECODE_ROWS(NR)                    \
    do {                                             \
        if (ct == 1) MOLORA_MX_DECODE(NR, 1);        \
        else if (ct == 2) MOLORA_MX_DECODE(NR, 2);   \
        else MOLORA_MX_DECODE(NR, 3);                \
    } while (0)
    switch ((N + 15) / 16) {
        case 1: MOLORA_MX_DECODE_ROWS(1); break;
        case 2: MOLORA_MX_DECODE_ROWS(2); break;
        case 3: MOLORA_MX_DECODE_ROWS(3); break;
        default: MOLORA_MX_DECODE_ROWS(4); break;
    }
#undef MOLORA_MX_DECODE_ROWS
#undef MOLORA_MX_DECODE
    return hipGetLastError();
}

}  // namespace molora
