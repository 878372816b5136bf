// Launches of the fused GEMM with outputs other than fp32 h, shared by the translation units that instantiate them.
#pragma once
#include "gemm_kernel.h"

namespace molora {

namespace {

template <class Cfg, int OUT, bool WT>
hipError_t launch_out(const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2, const int32_t *offsets,
                      const int32_t *perm, float *h, int64_t N, int d_in, int d_out, int C, int rank, GemmEpilogue ep, int slices,
                      hipStream_t s) {
    (void)&GemmKernel<Cfg, OUT, WT>::lds;  // instantiates the registration
    const int tiles_m = (int)((N + Cfg::BM - 1) / Cfg::BM);
    const int cols = OUT == kOutGated ? d_out / 2 : d_out, per = OUT == kOutGated ? Cfg::BN / 2 : Cfg::BN;
    const int tiles_n = (cols + per - 1) / per;
    const unsigned blocks = (unsigned)(((int64_t)tiles_m * tiles_n + 7) / 8 * 8);
    constexpr auto kernel = fused_gemm_kernel<Cfg, OUT, WT>;
    const dim3 grid(blocks, (unsigned)slices), block(Cfg::NT);
    const Mix plain{1, C, nullptr, nullptr};
    if (ep.base)
        launch_base_kernel(kernel, grid, block, Cfg::LDS_BYTES, s, x, W, B, t2, offsets, perm, h, (int)N, d_in, d_out, C, rank, tiles_m, tiles_n, plain, ep);
    else
        hipLaunchKernelGGL(kernel, grid, block, Cfg::LDS_BYTES, s, x, W, B, t2, offsets, perm, h, (int)N, d_in, d_out, C, rank, tiles_m, tiles_n, plain, ep);
    return hipGetLastError();
}

template <int OUT, bool WT>
hipError_t launch_config(int config, const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                         const int32_t *offsets, const int32_t *perm, float *h, int64_t N, int d_in, int d_out, int C, int rank,
                         GemmEpilogue ep, int slices, hipStream_t s) {
#define MOLORA_OUT_ARGS x, W, B, t2, offsets, perm, h, N, d_in, d_out, C, rank, ep, slices, s
    if constexpr (OUT != kOutPlanes) {  // (kMaxSlicedConfig)
        if (config == 5) return launch_out<GemmBig, OUT, WT>(MOLORA_OUT_ARGS);
        if (config == 6) return launch_out<Gemm320, OUT, WT>(MOLORA_OUT_ARGS);
    }
    switch (config) {  // the order of kGemmCosts
        case 0: return launch_out<Gemm64, OUT, WT>(MOLORA_OUT_ARGS);
        case 1: return launch_out<GemmMid, OUT, WT>(MOLORA_OUT_ARGS);
        case 2: return launch_out<GemmSmall, OUT, WT>(MOLORA_OUT_ARGS);
        case 3: return launch_out<GemmWide, OUT, WT>(MOLORA_OUT_ARGS);
        case 4: return launch_out<Gemm192, OUT, WT>(MOLORA_OUT_ARGS);
        default: return hipErrorInvalidValue;
    }
#undef MOLORA_OUT_ARGS
}

}  // namespace

// fp32 sums of x W + t B_c over slices of K to planes, `count` of them (gemm_planes.hip)
hipError_t launch_gemm_planes(const GemmSlices &pick, const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                              const int32_t *offsets, const int32_t *perm, float *planes, int64_t N, int d_in, int d_out, int C,
                              int rank, bool wt, bool base, int &count, hipStream_t s);

}  // namespace molora
