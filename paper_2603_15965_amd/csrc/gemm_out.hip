// The fused GEMM with outputs other than fp32 h: bf16 (gradients) and the gated block's z.
#include "gemm_kernel.h"

namespace molora {

namespace {

template <class Cfg, int OUT>
hipError_t launch_out(const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2, const int32_t *offsets,
                      const int32_t *perm, float *h, int64_t N, int d_in, int d_out, int C, int rank, GemmEpilogue ep, int slices,
                      hipStream_t s) {
    (void)&GemmKernel<Cfg, OUT>::lds;  // instantiates the registration
    const int tiles_m = (int)((N + Cfg::BM - 1) / Cfg::BM);
    const int cols = OUT == kOutGated ? d_out / 2 : d_out, per = OUT == kOutGated ? Cfg::BN / 2 : Cfg::BN;
    const int tiles_n = (cols + per - 1) / per;
    const unsigned blocks = (unsigned)(((int64_t)tiles_m * tiles_n + 7) / 8 * 8);
    constexpr auto kernel = fused_gemm_kernel<Cfg, OUT>;
    hipLaunchKernelGGL(kernel, dim3(blocks, (unsigned)slices), dim3(Cfg::NT), Cfg::LDS_BYTES, s, x, W, B, t2, offsets, perm, h, (int)N, d_in, d_out, C, rank, tiles_m, tiles_n, Mix{1, C, nullptr, nullptr}, ep);
    return hipGetLastError();
}

template <int OUT>
hipError_t launch_config(int config, const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                         const int32_t *offsets, const int32_t *perm, float *h, int64_t N, int d_in, int d_out, int C, int rank,
                         GemmEpilogue ep, int slices, hipStream_t s) {
#define MOLORA_OUT_ARGS x, W, B, t2, offsets, perm, h, N, d_in, d_out, C, rank, ep, slices, s
    switch (config) {  // the order of kGemmCosts
        case 0: return launch_out<Gemm64, OUT>(MOLORA_OUT_ARGS);
        case 1: return launch_out<GemmMid, OUT>(MOLORA_OUT_ARGS);
        case 2: return launch_out<GemmSmall, OUT>(MOLORA_OUT_ARGS);
        case 3: return launch_out<GemmWide, OUT>(MOLORA_OUT_ARGS);
        case 4: return launch_out<Gemm192, OUT>(MOLORA_OUT_ARGS);
        case 5: return launch_out<GemmBig, OUT>(MOLORA_OUT_ARGS);
        default: return launch_out<Gemm320, OUT>(MOLORA_OUT_ARGS);
    }
#undef MOLORA_OUT_ARGS
}

}  // namespace

namespace {
// fp32 sums of x W + t B_c to planes, `count` of them
hipError_t launch_planes(const GemmSlices &pick, const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                         const int32_t *offsets, const int32_t *perm, float *planes, int64_t N, int d_in, int d_out, int C,
                         int rank, int &count, hipStream_t s) {
    count = 1;
    if (pick.config < 0) return launch_small_batch_gemm(x, W, B, t2, offsets, perm, planes, N, d_in, d_out, C, rank, Mix{1, C, nullptr, nullptr}, s);
    const int k_slice = ((d_in + pick.slices - 1) / pick.slices + 63) / 64 * 64;
    count = (d_in + k_slice - 1) / k_slice;
    return launch_config<kOutPlanes>(pick.config, x, W, B, t2, offsets, perm, planes, N, d_in, d_out, C, rank,
                                     GemmEpilogue{nullptr, 0, k_slice}, count, s);
}
}  // namespace

hipError_t launch_gemm_bf16(const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                            const int32_t *offsets, const int32_t *perm, uint16_t *out, float *planes, int64_t N, int d_in,
                            int d_out, int C, int rank, hipStream_t s) {
    if (N == 0) return hipSuccess;
    GemmSlices pick = sliced_gemm_choice(N, d_in, d_out, C, rank);
    if (perm == nullptr && pick.config < 0) pick = GemmSlices{1, tiled_gemm_choice(N, d_in, d_out, C, rank)};  // it wants a dispatch
    if (pick.slices == 1 && pick.config >= 0)
        return launch_config<kOutBf16>(pick.config, x, W, B, t2, offsets, perm, nullptr, N, d_in, d_out, C, rank,
                                       GemmEpilogue{out}, 1, s);
    int count;
    const hipError_t e = launch_planes(pick, x, W, B, t2, offsets, perm, planes, N, d_in, d_out, C, rank, count, s);
    return e != hipSuccess ? e : launch_sum_planes(planes, out, N * d_out, count, s);
}

hipError_t launch_gemm_gated(const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                             const int32_t *offsets, const int32_t *perm, float *pre, uint16_t *z, float *planes, int64_t N,
                             int d_in, int F, int C, int rank, int act, hipStream_t s) {
    if (N == 0) return hipSuccess;
    GemmSlices pick = sliced_gemm_choice(N, d_in, 2 * F, C, rank);
    if (perm == nullptr && pick.config < 0) pick = GemmSlices{1, tiled_gemm_choice(N, d_in, 2 * F, C, rank)};
    if (pick.slices == 1 && pick.config >= 0)
        return launch_config<kOutGated>(pick.config, x, W, B, t2, offsets, perm, pre, N, d_in, 2 * F, C, rank, GemmEpilogue{z, act}, 1, s);
    int count;
    const hipError_t e = launch_planes(pick, x, W, B, t2, offsets, perm, planes, N, d_in, 2 * F, C, rank, count, s);
    return e != hipSuccess ? e : launch_gate(planes, count, z, pre, N, F, act, s);
}

}  // namespace molora
