// The fused GEMM with bf16 outputs: gradients in their parameters' type.  8192 tokens, W 2048 x 12288: dx 289 us, dW 317
// (1.43 and 1.30 PFLOP/s, by power).
#include "gemm_out.h"

namespace molora {

hipError_t launch_gemm_bf16(const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                            const int32_t *offsets, const int32_t *perm, uint16_t *out, float *planes, int64_t N, int d_in,
                            int d_out, int C, int rank, bool wt, hipStream_t s) {
    if (N == 0) return hipSuccess;
    // (the streaming kernel wants a dispatch, which dW has not, and W by rows of d_out)
    const GemmSlices pick = sliced_gemm_choice(N, d_in, d_out, C, rank, false);
    const GemmEpilogue ep{out};
    if (pick.slices == 1)
        return wt ? launch_config<kOutBf16, true>(pick.config, x, W, B, t2, offsets, perm, nullptr, N, d_in, d_out, C, rank, ep, 1, s)
                  : launch_config<kOutBf16, false>(pick.config, x, W, B, t2, offsets, perm, nullptr, N, d_in, d_out, C, rank, ep, 1, s);
    int count;
    const hipError_t e = launch_gemm_planes(pick, x, W, B, t2, offsets, perm, planes, N, d_in, d_out, C, rank, wt, false, count, s);
    return e != hipSuccess ? e : launch_sum_planes(planes, out, N * d_out, count, s);
}

}  // namespace molora
