// The fused GEMM that ends in the gated block's z; where K goes in slices, or the streaming kernel is the cheaper one, fp32 sums
// and a second launch that ends them.  (gemm_planes.hip: the slices.  gemm_grad.hip: bf16 gradients.)
//
// 8192 x 2048 -> 2 x 6144, 8 adapters of rank 16, launch timer: 329 us (1.25 PFLOP/s, by power) where h is not wanted, 385
// with its 403 MB, whose stores meet no products: every compute unit holds one workgroup.  Back to back with the rest of a
// training step it is 430; when it was 455, two workgroups of 128 x 128 each took 510 and 320 x 256 tiles 452.
#include "gemm_out.h"

namespace molora {

hipError_t launch_gemm_gated(const uint16_t *x, const uint16_t *W, const uint16_t *B, const uint16_t *t2,
                             const int32_t *offsets, const int32_t *perm, float *pre, uint16_t *z, float *planes, int64_t N,
                             int d_in, int F, int C, int rank, int act, hipStream_t s) {
    if (N == 0) return hipSuccess;
    const GemmSlices pick = sliced_gemm_choice(N, d_in, 2 * F, C, rank, perm != nullptr);
    if (pick.slices == 1 && pick.config >= 0)
        return launch_config<kOutGated, false>(pick.config, x, W, B, t2, offsets, perm, pre, N, d_in, 2 * F, C, rank,
                                               GemmEpilogue{z, act, 0, true}, 1, s);
    int count = 1;
    const hipError_t e =
        pick.config < 0
            ? launch_small_batch_gemm_own_rows(x, W, B, t2, offsets, perm, planes, N, d_in, 2 * F, C, rank, s)
            : launch_gemm_planes(pick, x, W, B, t2, offsets, perm, planes, N, d_in, 2 * F, C, rank, false, true, count, s);
    return e != hipSuccess ? e : launch_gate(planes, count, z, pre, N, F, act, s);
}

}  // namespace molora
