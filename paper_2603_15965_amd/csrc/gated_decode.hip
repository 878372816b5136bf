// The gated block of at most 64 tokens, second of two launches.  The first is the decode step's (small_batch.hip): x W,
// its K range in slices where the columns alone would not occupy the chip, beside dispatch and t = x A_r.  This one
//
//     h = sum of the slices + t B_r,   z = act(h[:, :F]) * h[:, F:]
//
// ends in z; h is stored only where it is asked for.  It is bound by reading the B_c in use: 64 x 4096 -> 2 x 12288, 16
// adapters of rank 64 under skewed routing, 20 us behind the first launch's 59 (201 MB of W, 3.4 TB/s).  Streaming both
// halves of W in this kernel, without the first launch's slices of K: 84 us in all.
#include "decode_body.h"
#include "gate.h"

namespace molora {

namespace {

template <int NR, int CT>
struct FinishLds {
    static constexpr int CPR = CT * 4;              // 16-byte chunks of a row of a slab: gate columns, then up columns
    static constexpr int STRIDE = CT * 64 + 32;     // its bytes (+32: four consecutive rows on distinct banks)
    static constexpr int SLAB = 16 * STRIDE;
    static constexpr int PART = 2 * CT * NR * 1024; // a wavefront's sums; they are added in two halves of four
    static constexpr int T_AT = 8 * SLAB;           // t lies behind the slabs; the sums take the place of both
    static constexpr int bytes(int R) { return T_AT + NR * 16 * t_row_bytes(R) > 4 * PART ? T_AT + NR * 16 * t_row_bytes(R) : 4 * PART; }
};

// A workgroup owns the same CT * 16 columns of the gate and of the up half, so that both factors of a z meet in it.  Its
// eight wavefronts take slabs of 16 rows of the B_c in use in turn, in token order (decode_body.h), and add their sums
// in LDS in a fixed order.
// (false: a sum is not finite, nothing is stored; CAREFUL: common.h, find_not_finite)
template <int NR, int CT, bool CAREFUL>
__device__ __forceinline__ bool gated_finish_body(const float *base, const float *__restrict__ planes, int slices,
                                                  const uint16_t *__restrict__ B, const int32_t *__restrict__ r,
                                                  const uint16_t *__restrict__ t2, const int32_t *__restrict__ perm,
                                                  uint16_t *__restrict__ z, float *pre, int N, int F, int C, int R, int act,
                                                  int *not_finite) {
    using Lds = FinishLds<NR, CT>;
    constexpr int CPR = Lds::CPR, STRIDE = Lds::STRIDE;
    constexpr int BL = (16 * CPR + 63) / 64, BATCH = CT < 4 ? 4 : 2;  // loads of a slab, slabs of a wavefront in flight
    constexpr int OUTS = (CT * NR + 7) / 8;              // 16 x 16 tiles of z per wavefront
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = fresh_thread<512>(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kq = lane >> 4, l16 = lane & 15;
    const int n0 = (int)blockIdx.x * (CT * 16);
    const int64_t pitch = 2 * (int64_t)F;
    unsigned char *const slab = lds + wave * Lds::SLAB, *const t_lds = lds + Lds::T_AT;

    // what x W gave, for the tiles of z that this wavefront will end
    f32x4 sum[OUTS][2];
#pragma unroll
    for (int o = 0; o < OUTS; ++o) {
        const int f = min(wave + o * 8, CT * NR - 1);
        const int row = min(f % NR * 16 + l16, N - 1), col = min(n0 + f / NR * 16 + kq * 4, F - 4);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int64_t at = row * pitch + half * F + col;
            sum[o][half] = *(const f32x4 *)(base + at);
            for (int sl = 1; sl < slices; ++sl) sum[o][half] += *(const f32x4 *)(planes + (int64_t)(sl - 1) * N * pitch + at);
        }
    }

    if (C > 0) {
        f32x4 acc[2 * CT][NR];  // gate columns, then up columns
#pragma unroll
        for (int j = 0; j < 2 * CT; ++j)
#pragma unroll
            for (int i = 0; i < NR; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        BatchAdapters batch;
        batch.find(target_of(r, lane, N, C), lane);
        const int parts = (R + 15) / 16, turns = batch.n * parts;
        // chunk `at` of a slab: its row is at / CPR, this its column of B
        auto chunk_col = [&](int at) __attribute__((always_inline)) {
            const int ch = at % CPR;
            return min(n0 + ch % (CPR / 2) * 8, F - 8) + (ch >= CPR / 2 ? F : 0);
        };
        u32x4 b[BATCH][BL];
        auto load_slabs = [&](int turn) __attribute__((always_inline)) {  // (past the last one: that one again)
#pragma unroll
            for (int s = 0; s < BATCH; ++s) {
                int c, q;
                uint64_t tokens;
                batch.slab(min(turn + s * 8, turns - 1), parts, c, q, tokens);
#pragma unroll
                for (int u = 0; u < BL; ++u) {
                    const int at = min(lane + u * 64, 16 * CPR - 1);
                    b[s][u] = *(const u32x4 *)(B + ((int64_t)c * R + min(q * 16 + at / CPR, R - 1)) * pitch + chunk_col(at));
                }
            }
        };
        if (turns > 0) load_slabs(wave);
        // rows of t to their tokens (those of tokens without adapter hold anything: t_operand takes none of them)
        const int per_row = R / 4, items = N * per_row;  // 16-byte chunks
        for (int it = tid; it < items; it += 512) {
            const int p = it / per_row, ch = it % per_row;
            *(u32x4 *)(t_lds + perm[p] * t_row_bytes(R) + ch * 16) = *(const u32x4 *)(t2 + (int64_t)p * 2 * R + ch * 8);
        }
        __syncthreads();
        for (int turn = wave; turn < turns; turn += 8 * BATCH) {
            u32x4 now[BATCH][BL];
#pragma unroll
            for (int s = 0; s < BATCH; ++s)
#pragma unroll
                for (int u = 0; u < BL; ++u) now[s][u] = b[s][u];
            if (turn + 8 * BATCH < turns) load_slabs(turn + 8 * BATCH);
#pragma unroll
            for (int s = 0; s < BATCH; ++s) {
                if (turn + s * 8 >= turns) break;
                int c, q;
                uint64_t tokens;
                batch.slab(turn + s * 8, parts, c, q, tokens);
#pragma unroll
                for (int u = 0; u < BL; ++u) {
                    const int at = lane + u * 64;
                    if (at < 16 * CPR) *(u32x4 *)(slab + at / CPR * STRIDE + at % CPR * 16) = now[s][u];
                }
                bf16x8 t[NR];
#pragma unroll
                for (int i = 0; i < NR; ++i) t[i] = t_operand(t_lds, i, q * 16, R, tokens, lane);
#pragma unroll
                for (int j = 0; j < 2 * CT; ++j) {
                    const bf16x8 fb = turned(slab, STRIDE, kq & 1, j * 32, lane);
#pragma unroll
                    for (int i = 0; i < NR; ++i) {
                        const f32x4 all = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb, t[i], acc[j][i], 0, 0, 0);
                        acc[j][i] = CAREFUL ? own_row(tokens, i, lane, all, acc[j][i]) : all;
                    }
                }
            }
        }
        // the wavefronts' sums: 4 .. 7 are added to 0 .. 3, then those four
        __syncthreads();  // no slab is in use, nor t
        unsigned char *const part = lds + (wave & 3) * Lds::PART + lane * 16;
        if (wave >= 4) {
#pragma unroll
            for (int j = 0; j < 2 * CT; ++j)
#pragma unroll
                for (int i = 0; i < NR; ++i) *(f32x4 *)(part + (j * NR + i) * 1024) = acc[j][i];
        }
        __syncthreads();
        if (wave < 4) {
#pragma unroll
            for (int j = 0; j < 2 * CT; ++j)
#pragma unroll
                for (int i = 0; i < NR; ++i) *(f32x4 *)(part + (j * NR + i) * 1024) = acc[j][i] + *(const f32x4 *)(part + (j * NR + i) * 1024);
        }
        __syncthreads();
    }

    if (C > 0) {
        float seen = 0.f;
#pragma unroll
        for (int o = 0; o < OUTS; ++o) {
            const int f = min(wave + o * 8, CT * NR - 1);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int v = 0; v < 4; ++v) sum[o][half] += *(const f32x4 *)(lds + v * Lds::PART + (half * CT * NR + f) * 1024 + lane * 16);
                find_not_finite(seen, sum[o][half]);
            }
        }
        if (!CAREFUL) {  // (before anything is stored: base may be pre)
            if (seen != 0.f) *not_finite = 1;
            __syncthreads();
            if (*not_finite != 0) return false;
        }
    }
#pragma unroll
    for (int o = 0; o < OUTS; ++o) {
        const int f = wave + o * 8, row = f % NR * 16 + l16, col = n0 + f / NR * 16 + kq * 4;
        if (f < CT * NR && row < N && col < F) {
            if (pre != nullptr) {
                *(f32x4 *)(pre + row * pitch + col) = sum[o][0];
                *(f32x4 *)(pre + row * pitch + F + col) = sum[o][1];
            }
            *(u32x2 *)(z + (int64_t)row * F + col) = bf16x4_bits(gate4(sum[o][0], sum[o][1], act));
        }
    }
    return true;
}

template <int NR, int CT>
__global__ __launch_bounds__(512, 2) void gated_finish_kernel(const float *base, const float *__restrict__ planes,
                                                              int slices, const uint16_t *__restrict__ B,
                                                              const int32_t *__restrict__ r, const uint16_t *__restrict__ t2,
                                                              const int32_t *__restrict__ perm, uint16_t *__restrict__ z,
                                                              float *pre, int N, int F, int C, int R, int act) {
    __shared__ int not_finite;
    if (threadIdx.x == 0) not_finite = 0;  // (a barrier follows before it is set)
    if (!gated_finish_body<NR, CT, false>(base, planes, slices, B, r, t2, perm, z, pre, N, F, C, R, act, &not_finite))
        gated_finish_body<NR, CT, true>(base, planes, slices, B, r, t2, perm, z, pre, N, F, C, R, act, nullptr);
}

template <int NR, int CT>
struct FinishKernel {
    static inline LdsRegistrar lds{(const void *)gated_finish_kernel<NR, CT>, (size_t)FinishLds<NR, CT>::bytes(MOLORA_MAX_RANK)};
};
template <int NR, int CT, class... Args>
void launch_finish(unsigned blocks, int rank, hipStream_t s, Args... args) {
    (void)&FinishKernel<NR, CT>::lds;  // instantiates the registration
    constexpr auto kernel = gated_finish_kernel<NR, CT>;
    const int bytes = FinishLds<NR, CT>::bytes(rank);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(512), bytes, s, args...);
}

}  // namespace

// as many columns to a workgroup as leave one for every compute unit: pieces of B's rows are longer (three tiles, one
// workgroup to each unit at F = 12288, instead of four: 20 us at best and more at the median)
int gated_finish_cols(int F) { return F <= 4096 ? 16 : F <= 8192 ? 32 : 64; }

hipError_t launch_gated_finish(const float *base, const float *planes, int slices, const uint16_t *B, const int32_t *r,
                               const uint16_t *t2, const int32_t *perm, uint16_t *z, float *pre, int64_t N, int F, int C, int rank,
                               int act, hipStream_t s) {
    if (N < 1 || N > 64) return hipErrorInvalidValue;
    const int tiles = (F + 15) / 16, ct = gated_finish_cols(F) / 16;
    const unsigned blocks = (unsigned)((tiles + ct - 1) / ct);
#define MOLORA_FINISH(NR, CT) launch_finish<NR, CT>(blocks, rank, s, base, planes, slices, B, r, t2, perm, z, pre, (int)N, F, C, rank, act)
#define MOLORA_FINISH_ROWS(NR)                  \
    do {                                        \
        if (ct == 1) MOLORA_FINISH(NR, 1);      \
        else if (ct == 2) MOLORA_FINISH(NR, 2); \
        else MOLORA_FINISH(NR, 4);              \
    } while (0)
    switch ((N + 15) / 16) {
        case 1: MOLORA_FINISH_ROWS(1); break;
        case 2: MOLORA_FINISH_ROWS(2); break;
        case 3: MOLORA_FINISH_ROWS(3); break;
        default: MOLORA_FINISH_ROWS(4); break;
    }
#undef MOLORA_FINISH_ROWS
#undef MOLORA_FINISH
    return hipGetLastError();
}

}  // namespace molora
