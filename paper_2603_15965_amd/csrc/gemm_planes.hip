// The fused GEMM over slices of K: fp32 sums of each to a plane of its own, for outputs of few tiles.
#include "gemm_out.h"

namespace molora {

hipError_t launch_gemm_planes(const GemmSlices &pick, const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                              const int32_t *offsets, const int32_t *perm, float *planes, int64_t N, int d_in, int d_out, int C,
                              int rank, bool wt, bool base, int &count, hipStream_t s) {
    const int k_slice = gemm_k_slice(d_in, pick.slices);
    count = (d_in + k_slice - 1) / k_slice;
    const GemmEpilogue ep{nullptr, 0, k_slice, base};
    return wt ? launch_config<kOutPlanes, true>(pick.config, x, W, B, t2, offsets, perm, planes, N, d_in, d_out, C, rank, ep, count, s)
              : launch_config<kOutPlanes, false>(pick.config, x, W, B, t2, offsets, perm, planes, N, d_in, d_out, C, rank, ep, count, s);
}

}  // namespace molora
