// The routed projection of at most 64 tokens on a 4-bit base weight, in two launches.  Such a step is one read of
// the codes of W and of the adapters in use; everything runs in token order and nothing waits for a sort.
//
//   first   x to codes, beside t = x A_r in slices of K (fp32 partial sums): both only read x, and the handful
//           of adapters in use alone would leave most of the chip idle
//   second  h = Q(x) Q(W) + t B_r, the slices of t added on the way
//
// 64 x 4096 -> 12288, 16 adapters of rank 64 under skewed routing: 26 us, 7 of the first launch and 19 of the second for
// 46 MB (27 of codes and scales, 19 of B, whose lines neighbouring workgroups on two XCDs both fetch: 73 are read): three
// trips to memory one after the other (codes of W and t, then B in two batches) in the one workgroup of a compute unit.  With a sort and the tiled product: 40 us.  The product alone of one
// token, 4096 -> 4096: 3.5 us, a launch.
#include <type_traits>

#include "decode_body.h"
#include "mx_mfma.h"
#include "mx_quant_body.h"

namespace molora {

namespace {

__global__ __launch_bounds__(256) void mx_decode_first_kernel(const uint16_t *__restrict__ x, const uint16_t *__restrict__ A,
                                                              const int32_t *__restrict__ r, uint8_t *__restrict__ codes,
                                                              uint8_t *__restrict__ scales, float *__restrict__ planes, int N,
                                                              int d_in, int C, int R, int slices, int shrink_blocks, int kt_n,
                                                              int kg_n) {
    __shared__ __attribute__((aligned(16))) unsigned char lds[kDecodeShrinkLds];
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
    static constexpr int bytes(int R) { return 8 * PART + NR * 16 * t_row_bytes(R); }
};

// (false: a sum is not finite; CAREFUL: common.h, find_not_finite)
template <int NR, int CT, bool CAREFUL>
__device__ __forceinline__ bool mx_decode_body(const uint8_t *__restrict__ xc, const uint8_t *__restrict__ xs,
                                               const uint8_t *__restrict__ wc, const uint8_t *__restrict__ ws,
                                               const uint16_t *__restrict__ B, const int32_t *__restrict__ r,
                                               const float *__restrict__ planes, float *__restrict__ h, int N, int d_out, int kt_n,
                                               int kg_n, int C, int R, int slices, int *not_finite) {
    using Lds = DecodeLds<NR, CT>;
    constexpr int STRIDE = Lds::STRIDE, LPR = CT * 2, LOADS = (16 * LPR + 63) / 64;  // 16-byte chunks of a row, loads of a slab
    constexpr int BATCH = 4;  // slabs of a wavefront in flight
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = fresh_thread<512>(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kq = lane >> 4, l16 = lane & 15;
    const int64_t ct0 = (int64_t)blockIdx.x * CT, ct_last = (d_out + 15) / 16 - 1, n0 = ct0 * 16;
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
        BatchAdapters batch;
        const int parts = (R + 15) / 16;
        u32x4 b[BATCH][LOADS];
        auto load_slabs = [&](int turn) __attribute__((always_inline)) {  // (past the last one: that one again)
#pragma unroll
            for (int s = 0; s < BATCH; ++s) {
                int c, q;
                uint64_t mine;
                batch.slab(min(turn + s * 8, batch.n * parts - 1), parts, c, q, mine);
#pragma unroll
                for (int u = 0; u < LOADS; ++u) {
                    const int at = lane + u * 64, row = min(at / LPR, 15);
                    b[s][u] = *(const u32x4 *)(B + ((int64_t)c * R + min(q * 16 + row, R - 1)) * d_out + min(n0 + at % LPR * 8, (int64_t)d_out - 8));
                }
            }
        };
        if (kg < kg_n) load(kg);
        batch.find(target, lane);
        if (batch.n > 0) load_slabs(wave);
        t_to_lds<NR>(planes, slices, target, R, t_lds);
        while (kg < kg_n) {
            multiply(kg);
            kg += 8;
            if (kg < kg_n) load(kg);
        }
        __syncthreads();
        // ---- expand ----
        unsigned char *const slab = lds + wave * Lds::PART;  // the wavefront's own until its sums go there
        for (int turn = wave; turn < batch.n * parts; turn += 8 * BATCH) {
            u32x4 now[BATCH][LOADS];
#pragma unroll
            for (int s = 0; s < BATCH; ++s)
#pragma unroll
                for (int u = 0; u < LOADS; ++u) now[s][u] = b[s][u];
            if (turn + 8 * BATCH < batch.n * parts) load_slabs(turn + 8 * BATCH);
#pragma unroll
            for (int s = 0; s < BATCH; ++s) {
                if (turn + s * 8 >= batch.n * parts) break;
                int c, q;
                uint64_t mine;
                batch.slab(turn + s * 8, parts, c, q, mine);
#pragma unroll
                for (int u = 0; u < LOADS; ++u) {
                    const int at = lane + u * 64;
                    if (at < 16 * LPR) *(u32x4 *)(slab + at / LPR * STRIDE + at % LPR * 16) = now[s][u];
                }
                bf16x8 t[NR];
#pragma unroll
                for (int i = 0; i < NR; ++i) t[i] = t_operand(t_lds, i, q * 16, R, mine, lane);
#pragma unroll
                for (int j = 0; j < CT; ++j) {
                    const bf16x8 fb = turned(slab, STRIDE, kq & 1, j * 32, lane);
#pragma unroll
                    for (int i = 0; i < NR; ++i) {
                        const f32x4 sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb, t[i], acc[j][i], 0, 0, 0);
                        acc[j][i] = CAREFUL ? own_row(mine, i, lane, sum, acc[j][i]) : sum;
                    }
                }
            }
        }
    }

#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
        for (int i = 0; i < NR; ++i) *(f32x4 *)(lds + wave * Lds::PART + ((j * NR + i) * 64 + lane) * 16) = acc[j][i];
    __syncthreads();
    float seen = 0.f;
    for (int f = wave; f < CT * NR; f += 8) {
        f32x4 sum = *(const f32x4 *)(lds + (f * 64 + lane) * 16);
#pragma unroll
        for (int v = 1; v < 8; ++v) sum += *(const f32x4 *)(lds + v * Lds::PART + (f * 64 + lane) * 16);
        const int row = f % NR * 16 + l16;
        const int64_t col = (ct0 + f / NR) * 16 + kq * 4;
        if (row < N && col < d_out) *(f32x4 *)(h + (int64_t)row * d_out + col) = sum;
        find_not_finite(seen, sum);
    }
    if (CAREFUL || C == 0) return true;
    if (seen != 0.f) *not_finite = 1;
    __syncthreads();
    return *not_finite == 0;
}

template <int NR, int CT>
__global__ __launch_bounds__(512, 2) void mx_decode_kernel(const uint8_t *__restrict__ xc, const uint8_t *__restrict__ xs,
                                                           const uint8_t *__restrict__ wc, const uint8_t *__restrict__ ws,
                                                           const uint16_t *__restrict__ B, const int32_t *__restrict__ r,
                                                           const float *__restrict__ planes, float *__restrict__ h, int N, int d_out,
                                                           int kt_n, int kg_n, int C, int R, int slices) {
    __shared__ int not_finite;
    if (threadIdx.x == 0) not_finite = 0;  // (a barrier follows before it is set)
    if (!mx_decode_body<NR, CT, false>(xc, xs, wc, ws, B, r, planes, h, N, d_out, kt_n, kg_n, C, R, slices, &not_finite))
        mx_decode_body<NR, CT, true>(xc, xs, wc, ws, B, r, planes, h, N, d_out, kt_n, kg_n, C, R, slices, nullptr);
}

template <int NR, int CT>
struct DecodeKernel {
    static inline LdsRegistrar lds{(const void *)mx_decode_kernel<NR, CT>, (size_t)DecodeLds<NR, CT>::bytes(MOLORA_MAX_RANK)};
};
template <int NR, int CT, class... Args>
void launch_decode(unsigned blocks, int rank, hipStream_t s, Args... args) {
    (void)&DecodeKernel<NR, CT>::lds;  // instantiates the registration
    constexpr auto kernel = mx_decode_kernel<NR, CT>;
    launch_base_kernel(kernel, dim3(blocks), dim3(512), (size_t)DecodeLds<NR, CT>::bytes(rank), s, args...);
}

}  // namespace

hipError_t launch_mx_decode_first(const uint16_t *x, const uint16_t *A, const int32_t *r, uint8_t *codes, uint8_t *scales,
                                  float *planes, int64_t N, int d_in, int C, int rank, hipStream_t s) {
    if (N < 1 || N > 64) return hipErrorInvalidValue;
    const int slices = decode_slices(N, d_in, C, rank), shrink = decode_shrink_blocks(N, d_in, C, rank), kg = mx_k_groups(d_in);
    const unsigned blocks = (unsigned)(shrink + mx_row_tiles(N) * kg);
    hipLaunchKernelGGL(mx_decode_first_kernel, dim3(blocks), dim3(256), 0, s, x, A, r, codes, scales, planes, (int)N, d_in, C,
                       rank, slices, shrink, mx_k_tiles(d_in), kg);
    return hipGetLastError();
}

// as many columns to a workgroup as leave one for every compute unit: what else would run in its place would
// read all of x and of t again
int mx_decode_cols(int d_out) { return d_out <= 4096 ? 16 : d_out <= 8192 ? 32 : 48; }

hipError_t launch_mx_decode(const uint8_t *xc, const uint8_t *xs, const uint8_t *wc, const uint8_t *ws, const uint16_t *B,
                            const int32_t *r, const float *planes, float *h, int64_t N, int d_in, int d_out, int C, int rank,
                            hipStream_t s) {
    if (N < 1 || N > 64) return hipErrorInvalidValue;
    const int kt = mx_k_tiles(d_in), kg = mx_k_groups(d_in), slices = C > 0 ? decode_slices(N, d_in, C, rank) : 1;
    const int64_t tiles = ((int64_t)d_out + 15) / 16;
    const int ct = mx_decode_cols(d_out) / 16;
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
