// The fused GEMM writing h in fp32: choice of the tiles and launch.
#include <math.h>

#include "gemm_kernel.h"

namespace molora {

namespace {

template <class Cfg>
hipError_t launch_cfg(const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                           const int32_t *offsets, const int32_t *perm, float *h, int64_t N, int d_in,
                           int d_out, int C, int rank, Mix mix, hipStream_t s) {
    auto kern = fused_gemm_kernel<Cfg>;
    (void)&GemmKernel<Cfg>::lds;  // instantiates the registration
    const int tiles_m = (int)((N + Cfg::BM - 1) / Cfg::BM);
    const int tiles_n = (d_out + Cfg::BN - 1) / Cfg::BN;
    const int total = tiles_m * tiles_n;
    const unsigned blocks = (unsigned)(((total + 7) / 8) * 8);
    launch_base_kernel(kern, dim3(blocks), dim3(Cfg::NT), Cfg::LDS_BYTES, s, x, W, B, t2, offsets, perm, h,
                       (int)N, d_in, d_out, C, rank, tiles_m, tiles_n, mix, GemmEpilogue{});
    return hipGetLastError();
}

}  // namespace

constexpr int kSmallBatchMax = 512;  // up to here the small-batch kernel takes operands of any size

bool fused_gemm_sizes_ok(int64_t N, int d_in, int d_out, int force_tile) {
    const bool tiled = force_tile == 128 || force_tile == 256 || (force_tile == 0 && N > kSmallBatchMax);
    if (!tiled) return true;  // the small-batch kernel checks its own offsets
    const uint64_t lim = uint64_t(1) << 32;
    return (uint64_t)N * (uint64_t)d_in * 2 < lim && (uint64_t)d_in * (uint64_t)d_out * 2 < lim;
}

namespace {
// Kernel and tile choice from static shapes only (no host read of the histogram): the smallest of
// the costs below.  Every configuration runs in rounds of (256 compute units x workgroups per
// unit) tiles; a round costs a start and an end, a time per K tile of 64 that grows from `k_few`
// to `k_few + k_full` with the share of the places in use, and the expand phase's batches and chunks.
// The coefficients are fitted (non-negative least squares of the relative error) to 270 shapes of
// 65 .. 16384 rows, 256 .. 12288 wide, 2 .. 64 adapters of rank 8 .. 64, every configuration forced on
// each (events around back-to-back launches, rotating inputs, us); the expand's were then lowered, the tiles' by
// a fifth, the streaming kernel's from 0.1 to 0.06, on 1600 random shapes of 1 .. 300 adapters up to rank 128,
// half of them with skewed routing.  Over those the choice is 1.25 % behind the best configuration (geometric
// mean; 4 % of them are more than 10 % behind, where the skew, which the rule cannot see, or a wide rank against a
// short K decides).  With the fitted ones it was 1.43 %, and up to 1.6x where 40 .. 200 adapters
// of rank 96 and more outweigh the product (311 x 256 -> 7168, 62 of rank 128: streaming 41, 64-row
// tiles 64 us; 528 x 1664 -> 5120, 180 of rank 128 88 / 121 us).  Fixed thresholds between 64, 128, 128 x 256
// and 256 rows are 8 % behind (5003 x 2728 -> 3176 in 256-row tiles, 260 of them for 256 units: 154 us,
// in 320-row tiles 109 us; 1333 x 2048 -> 6144 67 -> 55 us).
// These are fits of the kernels before their loop took 16x16x32 products, but for the row of 128 x 256: unrolled by three
// its loop gained more than the others, and of 8700 random shapes, every configuration forced with inputs from HBM and
// from the Infinity Cache, those that took 128 x 128 two-stage tiles were 3.3 and 3.5 % behind the best one, in half of
// them 128 x 256.  That row is lowered by 6 %: 4.6 % of the shapes go there, which take 0.954 (HBM) and 0.948 of the time
// (4096 x 2048 -> 2048 behind a shrink, W from HBM: 41 -> 35.5 us); 0.4 and 0.25 % of all are more than 3 % slower, one
// by 11 %, 2.9 % more than 3 % faster.  The choice is then 1.0 and 1.3 % behind the best configuration (1.2 and 1.6
// before; on 2300 other shapes the same).  A refit of all rows gains 0.7 % more on average and loses more than 3 % on
// more shapes: wide ranks and skewed routing against a short K.
struct GemmCost {
    int bm, bn, per_cu;
    double once, per_round, partial, k_round, k_few, k_full, expand;
};
constexpr GemmCost kGemmCosts[] = {
    {64, 128, 2, 4.7, 1.6, 0.0, 0.62, 0.28, 0.38, 1.11},
    {128, 128, 1, 1.9, 3.9, 3.6, 0.52, 0.37, 0.16, 0.91},
    {128, 128, 2, 0.0, 5.3, 5.2, 0.86, 0.55, 0.36, 1.02},
    {128, 256, 1, 0.0, 6.6, 6.5, 0.79, 0.545, 0.254, 1.06},
    {192, 256, 1, 2.1, 9.1, 4.5, 1.13, 0.85, 0.36, 1.29},
    {256, 256, 1, 3.7, 12.5, 4.2, 1.42, 0.98, 0.51, 1.54},
    {320, 256, 1, 4.9, 15.8, 5.8, 1.78, 1.18, 0.59, 1.58},
};
constexpr int kGemmConfigs = sizeof(kGemmCosts) / sizeof(kGemmCosts[0]);

double tiled_cost(const GemmCost &g, int64_t N, int d_in, int d_out, int C, int R, int slices = 1) {
    const int64_t tiles = ((N + g.bm - 1) / g.bm) * ((d_out + g.bn - 1) / g.bn) * slices;
    const int64_t slots = (int64_t)256 * g.per_cu, full = tiles / slots;
    const double last = (double)(tiles % slots) / (double)slots, part = last > 0 ? 1 : 0;
    const double kt = (d_in + 64 * slices - 1) / (64 * slices);
    const double segs = fmin((double)C, 1.0 + (double)g.bm * C / (double)N);  // buckets that own rows of a tile
    const double expand = segs / slices * ((R + 15) / 16) / 4 + (R + 31) / 32;
    return g.once + g.per_round * (double)full + g.partial * part + kt * (g.k_round * (double)full + g.k_few * part + g.k_full * last) +
           g.expand * ((double)full + part) * expand;
}
// the streaming kernel: rounds of 256 workgroups, column groups of 64 (of 32 when that leaves at most
// 128) x row tiles of 64
double streaming_cost(int64_t N, int d_in, int d_out, int C, int R) {
    int64_t wgs = (int64_t)((d_out + 63) / 64) * ((N + 63) / 64);
    if (wgs <= 128) wgs *= 2;
    const double rounds = (double)((wgs + 255) / 256);
    const double segs = fmin((double)C, 1.0 + 64.0 * C / (double)N);
    return 0.6 + rounds * (5.6 + 3.26 * d_in / 1024.0 + 0.06 * segs * R / 16.0);
}
// -1: the streaming kernel, else the place in kGemmCosts
int gemm_choice(int64_t N, int d_in, int d_out, int C, int R, bool streaming = true) {
    const uint64_t lim = uint64_t(1) << 32;
    // one row tile always streams; so do operands beyond the tiled kernel's 32-bit offsets
    // (fused_gemm_sizes_ok refuses them above kSmallBatchMax)
    if (streaming && (N <= 64 || (N <= kSmallBatchMax && ((uint64_t)N * d_in * 2 >= lim || (uint64_t)d_in * d_out * 2 >= lim))))
        return -1;
    double best = streaming && N <= 4096 ? streaming_cost(N, d_in, d_out, C, R) : 1e30;
    int pick = -1;
    for (int i = 0; i < kGemmConfigs; ++i) {
        const double cost = tiled_cost(kGemmCosts[i], N, d_in, d_out, C, R);
        if (cost < best) {
            best = cost;
            pick = i;
        }
    }
    return pick;
}
}  // namespace

// The cheapest way to an output that is not h itself: one launch that ends in it, or fp32 sums in memory, of the
// streaming kernel (many wide adapters against a small batch: its expand is the cheaper one) or of K in slices (few
// output tiles, long K), and a second launch that ends them.  1459 x 9216 -> 2 x 256, gated: 76 us in one launch, 53 in
// slices; a training step of 381 x 256 -> 2 x 512 with 29 adapters of rank 64 90 / 66 us.  (Sixteen slices at most instead of eight: no
// difference over thirty random shapes.)
// The costs are the fits above, of fp32 h.  For these outputs, every tile and two, four and eight slices of K forced on 60
// random shapes (65 .. 16384 tokens, 256 .. 8192 wide, 1 .. 64 adapters, times of the whole call): the choice is behind the
// best way by 1.7 % for z, 2.1 % for z with h, 1.3 % for dx and 1.8 % for dW (geometric means; 3 to 7 % of the shapes by
// more than 10 %: 410 x 7608 -> 2 x 2912 85 us, in two slices 68; dW of 207 x 7168 -> 2 x 5376 92, in 128 x 128 tiles 67).
GemmSlices sliced_gemm_choice(int64_t N, int d_in, int d_out, int C, int R, bool streaming) {
    GemmSlices pick{1, gemm_choice(N, d_in, d_out, C, R, false)};
    double best = tiled_cost(kGemmCosts[pick.config], N, d_in, d_out, C, R);
    const double floats = (double)N * d_out;
    const auto second = [&](int slices) { return 4.0 + slices * floats * 8 / 4e6; };  // (4 MB a microsecond, written and read)
    if (streaming && N <= kSmallBatchMax && floats <= (double)kMaxPlaneFloats) {
        const double cost = streaming_cost(N, d_in, d_out, C, R) + second(1);
        if (cost < best) {
            best = cost;
            pick = GemmSlices{1, -1};
        }
    }
    for (int slices = 2; slices <= kMaxGemmSlices; ++slices) {
        if (slices * floats > (double)kMaxPlaneFloats || d_in < slices * 256) break;
        for (int i = 0; i <= kMaxSlicedConfig; ++i) {
            const double cost = tiled_cost(kGemmCosts[i], N, d_in, d_out, C, R, slices) + second(slices);
            if (cost < best) {
                best = cost;
                pick = GemmSlices{slices, i};
            }
        }
    }
    return pick;
}

namespace {
void name_tile(int pick, int64_t N, int d_out, int32_t *tile) {
    static constexpr int stages[kGemmConfigs] = {Gemm64::STAGES,   GemmMid::STAGES, GemmSmall::STAGES, GemmWide::STAGES,
                                                 Gemm192::STAGES, GemmBig::STAGES, Gemm320::STAGES};  // the order of kGemmCosts
    tile[0] = pick < 0 ? 64 : kGemmCosts[pick].bm;
    tile[1] = pick < 0 ? small_batch_cols(N, d_out) : kGemmCosts[pick].bn;
    tile[2] = pick < 0 ? 0 : stages[pick];
}
}  // namespace
void fused_gemm_tile(int64_t N, int d_in, int d_out, int C, int R, int32_t *tile) {
    name_tile(gemm_choice(N, d_in, d_out, C, R), N, d_out, tile);
}
void sliced_gemm_tile(int64_t N, int d_in, int d_out, int C, int R, bool streaming, int32_t *tile) {
    const GemmSlices pick = sliced_gemm_choice(N, d_in, d_out, C, R, streaming);
    name_tile(pick.config, N, d_out, tile);
    const int k_slice = gemm_k_slice(d_in, pick.slices);
    tile[3] = pick.config < 0 ? 1 : (d_in + k_slice - 1) / k_slice;
}

// force_tile: 0 = the choice below; 64 / 128 / 256 = that row-tile height whatever the shape
// (the tiling ablation compares the choice with fixed tiles).
hipError_t launch_fused_gemm(const uint16_t *x, const uint16_t *W, const uint16_t *B,
                             const uint16_t *t2, const int32_t *offsets, const int32_t *perm,
                             float *h, int64_t N, int d_in, int d_out, int C, int rank, Mix mix,
                             hipStream_t s, int force_tile) {
    if (N == 0) return hipSuccess;
    // the token-order intermediate is read by the kernels chosen below, for a batch of several row tiles
    if (mix.t_dense && (force_tile == 64 || N <= 64 || mix.k != 1)) return hipErrorInvalidValue;
#define MOLORA_GEMM_ARGS x, W, B, t2, offsets, perm, h, N, d_in, d_out, C, rank, mix, s
    if (force_tile == 64) return launch_small_batch_gemm(MOLORA_GEMM_ARGS);
    if (force_tile == 128) return launch_cfg<GemmSmall>(MOLORA_GEMM_ARGS);
    if (force_tile == 256) return launch_cfg<GemmBig>(MOLORA_GEMM_ARGS);
    switch (gemm_choice(N, d_in, d_out, C, mix.k * rank)) {  // the order of kGemmCosts
        case 0: return launch_cfg<Gemm64>(MOLORA_GEMM_ARGS);
        case 1: return launch_cfg<GemmMid>(MOLORA_GEMM_ARGS);
        case 2: return launch_cfg<GemmSmall>(MOLORA_GEMM_ARGS);
        case 3: return launch_cfg<GemmWide>(MOLORA_GEMM_ARGS);
        case 4: return launch_cfg<Gemm192>(MOLORA_GEMM_ARGS);
        case 5: return launch_cfg<GemmBig>(MOLORA_GEMM_ARGS);
        case 6: return launch_cfg<Gemm320>(MOLORA_GEMM_ARGS);
        default: return launch_small_batch_gemm(MOLORA_GEMM_ARGS);
    }
#undef MOLORA_GEMM_ARGS
}

}  // namespace molora
