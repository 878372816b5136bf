// Products of 4-bit microscaled operands (layout in mx.h), with the grouped expand of routed adapters:
//
//     h[perm[p]][:] = Q(x)_p Q(W)  +  t_p B_{c(p)}
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 codes by 128 x 16, applies both blocks' scales and adds in
// fp32.  The products of two codes and their block sums are exact in fp32 (codes are multiples of 1/2 up to 6), so
// only the order of the additions over blocks is this kernel's.
#include <type_traits>

#include "lds_dma.h"
#include "mx.h"

namespace molora {

namespace {

// Codes as the instruction's operand: 16 bytes a lane, the format's upper half is not read.
__device__ __forceinline__ i32x8 mx_operand(u32x4 c) {
    return i32x8{(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0};
}
// acc += W tile (first operand: a lane then holds four columns of one row of h) x x tile, scales from byte J
template <int J>
__device__ __forceinline__ f32x4 mx_mfma(u32x4 w, u32x4 x, f32x4 acc, uint32_t sw, uint32_t sx) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(w), mx_operand(x), acc, 4, 4, J, (int)sw, J, (int)sx);
}

// ---- a batch of at most 64 rows: one read of W ----
// A workgroup owns 16 columns, its eight wavefronts take groups of 512 k in turn, straight from memory into
// registers (a code tile is 1 KB, contiguous), and add their sums in LDS in a fixed order.
template <int NR>
__global__ __launch_bounds__(512) void mx_stream_kernel(const uint8_t *__restrict__ xc, const uint8_t *__restrict__ xs,
                                                        const uint8_t *__restrict__ wc, const uint8_t *__restrict__ ws,
                                                        float *__restrict__ h, int N, int d_out, int kt_n, int kg_n) {
    __shared__ f32x4 part[8][NR][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t ct = blockIdx.x;
    f32x4 acc[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int kg = wave; kg < kg_n; kg += 8) {
        u32x4 w[4], x[NR][4];
        uint32_t sw, sx[NR];
        sw = *(const uint32_t *)(ws + ((ct * kg_n + kg) * 64 + lane) * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // past the last tile: its codes again, under scales of zero codes (masked below)
            const int kt = min(kg * 4 + j, kt_n - 1);
            w[j] = *(const u32x4 *)(wc + ((ct * kt_n + kt) * 64 + lane) * 16);
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            sx[i] = *(const uint32_t *)(xs + (((int64_t)i * kg_n + kg) * 64 + lane) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int kt = min(kg * 4 + j, kt_n - 1);
                x[i][j] = *(const u32x4 *)(xc + (((int64_t)i * kt_n + kt) * 64 + lane) * 16);
            }
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            acc[i] = mx_mfma<0>(w[0], x[i][0], acc[i], sw, sx[i]);
            if (kg * 4 + 1 < kt_n) acc[i] = mx_mfma<1>(w[1], x[i][1], acc[i], sw, sx[i]);
            if (kg * 4 + 2 < kt_n) acc[i] = mx_mfma<2>(w[2], x[i][2], acc[i], sw, sx[i]);
            if (kg * 4 + 3 < kt_n) acc[i] = mx_mfma<3>(w[3], x[i][3], acc[i], sw, sx[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < NR; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave < NR) {
        f32x4 sum = part[0][wave][lane];
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += part[w][wave][lane];
        const int row = wave * 16 + (lane & 15);
        const int64_t col = ct * 16 + (lane >> 4) * 4;
        if (row < N && col < d_out) *(f32x4 *)(h + (int64_t)row * d_out + col) = sum;
    }
}

// ---- larger batches: output tiles ----
// BM x BN output tile, WM x WN wavefronts.  A stage is 256 k of both sides (two code tiles per 16 rows or
// columns) brought to LDS as it lies in memory; two stages, one travelling while the other is multiplied.
// The scales of 512 k come with every second stage, into one of two places of their own.
template <int WM_, int WN_, int TM_, int TN_>
struct MxCfg {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_;
    static constexpr int NW = WM * WN, NT = NW * 64;
    static constexpr int RT = WM * TM, CT = WN * TN;  // 16-row and 16-column tiles
    static constexpr int BM = RT * 16, BN = CT * 16;
    static constexpr int PIECES = 2 * (RT + CT), LPW = PIECES / NW;
    static constexpr int STAGE = PIECES * 1024;
    static constexpr int SP = (RT + CT) / 4, SLPW = (SP + NW - 1) / NW;  // 1 KB holds the scales of four tiles
    static constexpr int SCALES = SP * 1024;
    static constexpr int B_STRIDE = BN * 2 + 32;  // a row of B in LDS: four consecutive rows on distinct banks
    static constexpr size_t LDS_BYTES = 2 * (STAGE + SCALES) + (1024 + 4) * 4;
    static_assert(PIECES % NW == 0 && RT % 4 == 0 && CT % 4 == 0, "pieces split evenly");
    static_assert(16 * B_STRIDE <= STAGE, "a slab of B fits a stage");
};

template <class Cfg>
__global__ __launch_bounds__(Cfg::NT, 2) void mx_gemm_kernel(
    const uint8_t *__restrict__ xc, const uint8_t *__restrict__ xs, const uint8_t *__restrict__ wc,
    const uint8_t *__restrict__ ws, const uint16_t *__restrict__ B, const uint16_t *__restrict__ t2,
    const int32_t *__restrict__ offsets, const int32_t *__restrict__ perm, float *__restrict__ h, int N, int d_out,
    int kt_n, int kg_n, int C, int R, int tiles_m, int tiles_n) {
    constexpr int TM = Cfg::TM, TN = Cfg::TN, RT = Cfg::RT, CT = Cfg::CT, NW = Cfg::NW;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    unsigned char *const scales = smem + 2 * Cfg::STAGE;
    int32_t *const off = (int32_t *)(scales + 2 * Cfg::SCALES);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / Cfg::WN, wn = wave % Cfg::WN;

    // XCDs take runs of tiles, eight row tiles wide, so that each one's L2 holds its rows and columns
    const int total = tiles_m * tiles_n, share = (total + 7) / 8;
    const int logical = (int)(blockIdx.x % 8) * share + (int)(blockIdx.x / 8);
    if (blockIdx.x / 8 >= (unsigned)share || logical >= total) return;
    const int group = logical / (8 * tiles_n), first = group * 8;
    const int width = min(8, tiles_m - first), in_group = logical - first * tiles_n;
    const int tile_m = first + in_group % width, tile_n = in_group / width;
    const int p0 = tile_m * Cfg::BM;
    const int64_t rt_last = (N + 15) / 16 - 1, ct_last = (d_out + 15) / 16 - 1;
    const int64_t rt0 = (int64_t)tile_m * RT, ct0 = (int64_t)tile_n * CT;

    auto issue = [&](int st) __attribute__((always_inline)) {
        unsigned char *stage = smem + (st & 1) * Cfg::STAGE;
#pragma unroll
        for (int i = 0; i < Cfg::LPW; ++i) {
            const int piece = i * NW + wave;  // [tile][two k tiles], rows first
            const int kt = min(2 * st + (piece & 1), kt_n - 1);
            const int tile = piece >> 1;
            const bool is_x = tile < RT;
            const int64_t at = is_x ? min(rt0 + tile, rt_last) : min(ct0 + tile - RT, ct_last);
            load_to_lds16((is_x ? xc : wc) + (at * kt_n + kt) * 1024, lane * 16, stage + piece * 1024);
        }
        if (st & 1) return;
        unsigned char *place = scales + ((st >> 1) & 1) * Cfg::SCALES;
#pragma unroll
        for (int i = 0; i < Cfg::SLPW; ++i) {
            const int piece = (i * NW + wave) % Cfg::SP;  // (twice the same where there are more wavefronts than pieces)
            const int tile = piece * 4 + (lane >> 4);
            const bool is_x = piece * 4 < RT;
            const int64_t at = is_x ? min(rt0 + tile, rt_last) : min(ct0 + tile - RT, ct_last);
            load_to_lds16_ptr((is_x ? xs : ws) + (at * kg_n + (st >> 1)) * 256 + (lane & 15) * 16, place + piece * 1024);
        }
    };

    for (int i = tid; i <= C && C > 0; i += Cfg::NT) off[i] = offsets[i];

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int nst = (kt_n + 1) / 2;
    __syncthreads();
    issue(0);
    if (nst > 1) issue(1);
    auto multiply = [&](int st, auto half_c) __attribute__((always_inline)) {
        constexpr int HALF = decltype(half_c)::value;  // which two bytes of the scales
        if (st + 1 < nst)
            wait_vmcnt<Cfg::LPW + (HALF ? Cfg::SLPW : 0)>();  // the next stage may be on its way
        else
            wait_vmcnt<0>();
        wg_barrier();
        const unsigned char *stage = smem + HALF * Cfg::STAGE;
        const unsigned char *place = scales + ((st >> 1) & 1) * Cfg::SCALES;
        uint32_t sx[TM], sw[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) sx[i] = *(const uint32_t *)(place + (wm * TM + i) * 256 + lane * 4);
#pragma unroll
        for (int j = 0; j < TN; ++j) sw[j] = *(const uint32_t *)(place + (RT + wn * TN + j) * 256 + lane * 4);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k == 1 && 2 * st + 1 >= kt_n) break;
            u32x4 w[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) w[j] = *(const u32x4 *)(stage + ((RT + wn * TN + j) * 2 + k) * 1024 + lane * 16);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const u32x4 x = *(const u32x4 *)(stage + ((wm * TM + i) * 2 + k) * 1024 + lane * 16);
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = k ? mx_mfma<HALF * 2 + 1>(w[j], x, acc[i][j], sw[j], sx[i])
                                  : mx_mfma<HALF * 2>(w[j], x, acc[i][j], sw[j], sx[i]);
            }
        }
        wait_lds();
        wg_barrier();  // every wavefront has read the stage: it can be filled again
        if (st + 2 < nst) issue(st + 2);
    };
    for (int st = 0; st < nst; st += 2) {
        multiply(st, std::integral_constant<int, 0>{});
        if (st + 1 < nst) multiply(st + 1, std::integral_constant<int, 1>{});
    }

    // ---- expand: the buckets that own rows of the tile, 16 columns of t at a time ----
    // A fragment of 32 k is [hi | lo] of 16 columns of t against the same 16 rows of B twice.
    const int kq = lane >> 4, l16 = lane & 15;
    if (C > 0) {
        int lo_c = 0, hi_c = C;  // first bucket that ends behind the tile's first row
        while (lo_c < hi_c) {
            const int mid = (lo_c + hi_c) >> 1;
            if (off[mid + 1] > p0) hi_c = mid; else lo_c = mid + 1;
        }
        const int64_t n0 = ct0 * 16;
        for (int c = lo_c; c < C && off[c] < p0 + Cfg::BM; ++c) {
            const int lo = off[c], hi = off[c + 1];
            if (lo == hi) continue;
            for (int k0 = 0; k0 < R; k0 += 16) {
                __syncthreads();
                for (int i = tid; i < 16 * (Cfg::BN / 8); i += Cfg::NT) {
                    const int row = i / (Cfg::BN / 8), at = i % (Cfg::BN / 8);
                    const int64_t col = min(n0 + at * 8, (int64_t)d_out - 8);
                    *(u32x4 *)(smem + row * Cfg::B_STRIDE + at * 16) =
                        *(const u32x4 *)(B + ((int64_t)c * R + min(k0 + row, R - 1)) * d_out + col);
                }
                __syncthreads();
                bf16x8 b[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const unsigned char *p = smem + ((kq & 1) * 8 + (l16 >> 2)) * Cfg::B_STRIDE + (wn * TN + j) * 32 + (l16 & 3) * 8;
                    const i16x4 u = lds_read_tr16((const MOLORA_LDS void *)p), v = lds_read_tr16((const MOLORA_LDS void *)(p + 4 * Cfg::B_STRIDE));
                    b[j] = __builtin_bit_cast(bf16x8, i16x8{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]});
                }
                const int kc = k0 + (kq & 1) * 8;
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const int first_row = p0 + (wm * TM + i) * 16, p = first_row + l16;
                    if (hi <= first_row || lo >= first_row + 16) continue;
                    const bool mine = p >= lo && p < hi && kc < R;
                    i16x8 t = *(const i16x8 *)(t2 + (int64_t)min(p, N - 1) * 2 * R + (kq >> 1) * R + min(kc, R - 8));
                    if (!mine) t = i16x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], __builtin_bit_cast(bf16x8, t), acc[i][j], 0, 0, 0);
                }
            }
        }
    }

#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int p = p0 + (wm * TM + i) * 16 + l16;
        if (p >= N) continue;
        const int64_t row = perm != nullptr ? perm[p] : p;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t col = (ct0 + wn * TN + j) * 16 + kq * 4;
            if (col < d_out) __builtin_nontemporal_store(acc[i][j], (f32x4 *)(h + row * d_out + col));
        }
    }
}

template <class Cfg>
struct MxKernel {
    static inline LdsRegistrar lds{(const void *)mx_gemm_kernel<Cfg>, Cfg::LDS_BYTES};
};

template <class Cfg>
hipError_t launch_mx_tiles(const uint8_t *xc, const uint8_t *xs, const uint8_t *wc, const uint8_t *ws, const uint16_t *B,
                           const uint16_t *t2, const int32_t *offsets, const int32_t *perm, float *h, int64_t N, int d_in,
                           int d_out, int C, int rank, hipStream_t s) {
    (void)&MxKernel<Cfg>::lds;  // instantiates the registration
    const int64_t tiles_m = (N + Cfg::BM - 1) / Cfg::BM, tiles_n = (d_out + Cfg::BN - 1) / Cfg::BN;
    const int64_t blocks = (tiles_m * tiles_n + 7) / 8 * 8;
    if (blocks * Cfg::NT >= (int64_t(1) << 32)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(mx_gemm_kernel<Cfg>, dim3((unsigned)blocks), dim3(Cfg::NT), Cfg::LDS_BYTES, s, xc, xs, wc, ws, B, t2,
                       offsets, perm, h, (int)N, d_out, mx_k_tiles(d_in), mx_k_groups(d_in), C, rank, (int)tiles_m, (int)tiles_n);
    return hipGetLastError();
}

}  // namespace

using MxBig = MxCfg<2, 4, 8, 4>;    // 256 x 256, one workgroup per compute unit
using MxSmall = MxCfg<2, 2, 4, 4>;  // 128 x 128, two

hipError_t launch_mx_gemm(const uint8_t *xc, const uint8_t *xs, const uint8_t *wc, const uint8_t *ws, const uint16_t *B,
                          const uint16_t *t2, const int32_t *offsets, const int32_t *perm, float *h, int64_t N, int d_in,
                          int d_out, int C, int rank, hipStream_t s) {
    if (N == 0) return hipSuccess;
    if (N <= 64 && C == 0 && perm == nullptr) {
        const dim3 grid((unsigned)((d_out + 15) / 16)), block(512);
        const int kt = mx_k_tiles(d_in), kg = mx_k_groups(d_in);
#define MOLORA_MX_STREAM(NR) hipLaunchKernelGGL((mx_stream_kernel<NR>), grid, block, 0, s, xc, xs, wc, ws, h, (int)N, d_out, kt, kg)
        if (N <= 16) MOLORA_MX_STREAM(1);
        else if (N <= 32) MOLORA_MX_STREAM(2);
        else if (N <= 48) MOLORA_MX_STREAM(3);
        else MOLORA_MX_STREAM(4);
#undef MOLORA_MX_STREAM
        return hipGetLastError();
    }
    const int64_t big = ((N + 255) / 256) * (((int64_t)d_out + 255) / 256);
    if (big >= 256) return launch_mx_tiles<MxBig>(xc, xs, wc, ws, B, t2, offsets, perm, h, N, d_in, d_out, C, rank, s);
    return launch_mx_tiles<MxSmall>(xc, xs, wc, ws, B, t2, offsets, perm, h, N, d_in, d_out, C, rank, s);
}

}  // namespace molora
