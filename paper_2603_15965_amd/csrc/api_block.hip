// C ABI of the feed-forward block: 4-bit microscaled products and the gated block.  Argument checking and the
// order of launches, no arithmetic.
#include "api_util.h"
#include "decode_body.h"
#include "mx.h"

#include <algorithm>

namespace {

// Rows and k of a microscaled operand.
inline bool mx_sizes_ok(int64_t rows, int32_t K) {
    return rows >= 0 && rows < (int64_t(1) << 31) && K >= 8 && K % 8 == 0 &&
           molora::mx_row_tiles(rows) * molora::mx_k_tiles(K) < molora::kMxMaxBlocks;
}
inline size_t mx_codes(int64_t rows, int32_t K) {
    return size_t(molora::mx_row_tiles(rows)) * size_t(molora::mx_k_tiles(K)) * 1024;
}
inline size_t mx_scales(int64_t rows, int32_t K) {
    return size_t(molora::mx_row_tiles(rows)) * size_t(molora::mx_k_groups(K)) * 256;
}
inline bool mx_product_ok(int64_t N, int32_t d_in, int32_t d_out) {
    return d_out >= 8 && d_out % 8 == 0 && mx_sizes_ok(N, d_in) && mx_sizes_ok(d_out, d_in) &&
           ((N + 127) / 128) * ((int64_t(d_out) + 127) / 128) < molora::kMxMaxBlocks;
}

constexpr int64_t kDecode = 64;  // batches that are one read of the base weight

// Scratch of a shrink of any batch of up to N tokens (it does not grow with the batch).
inline size_t shrink_scratch_up_to(int64_t N, int32_t d_in, int32_t C, int32_t rank) {
    int64_t peaks[molora::kShrinkPeaks];
    const int n = molora::shrink_scratch_peaks(N, d_in, C, rank, peaks);
    size_t most = molora::shrink_scratch_bytes(N, d_in, C, rank);
    for (int i = 0; i < n; ++i) most = std::max(most, molora::shrink_scratch_bytes(peaks[i], d_in, C, rank));
    return most;
}

struct Cutter {  // pieces of a workspace, each 256-byte aligned
    unsigned char *base;
    size_t at = 0;
    template <class T>
    T *take(size_t bytes) {
        T *p = reinterpret_cast<T *>(base + at);
        at += round256(bytes);
        return p;
    }
};

// ---- routed projection on a microscaled base weight ----
struct MxWorkspace {
    int32_t *offsets, *perm;
    uint16_t *t2;
    uint8_t *codes, *scales;
    float *planes;  // x A_r in slices of K
    size_t bytes;
};
inline MxWorkspace carve_mx(void *base, int64_t N, int32_t d_in, int32_t C, int32_t rank) {
    Cutter c{static_cast<unsigned char *>(base)};
    MxWorkspace w{};
    w.codes = c.take<uint8_t>(mx_codes(N, d_in));
    w.scales = c.take<uint8_t>(mx_scales(N, d_in));
    if (N <= kDecode) {
        w.planes = c.take<float>(size_t(molora::kMaxSlices) * 64 * rank * 4);
    } else {
        w.offsets = c.take<int32_t>(size_t(C + 1) * 4);
        w.perm = c.take<int32_t>(size_t(N) * 4);
        w.t2 = c.take<uint16_t>(size_t(N) * 2 * rank * 2);
        w.planes = c.take<float>(shrink_scratch_up_to(N, d_in, C, rank));
    }
    w.bytes = c.at;
    return w;
}

// ---- gated block ----
inline bool gated_sizes_ok(int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank, int32_t act) {
    if (act < MOLORA_ACT_SILU || act > MOLORA_ACT_GELU_TANH || F < 8 || F % 8 != 0 || F > (1 << 29)) return false;
    const bool bare = C == 0 && rank == 0;
    if (!apply_sizes_ok(N, d_in, 2 * F, bare ? 1 : C, bare ? 8 : rank)) return false;
    // the tiled kernel's 32-bit offsets into x and W, also as operands of the backward pass
    return molora::fused_gemm_sizes_ok(N + 7, d_in, 2 * F, 256) && molora::fused_gemm_sizes_ok(N + 7, 2 * F, 8, 256);
}
inline bool adapters_given(const void *A, const void *B, const int32_t *r, int32_t C) {
    return C == 0 ? !A && !B && !r : A && B && r;
}

struct GatedWorkspace {
    int32_t *offsets, *perm;
    uint16_t *t2;
    float *base, *planes;  // at most 64 tokens: x W, in slices of K; more: fp32 sums where the GEMM does not end in z
    int slices;
    size_t bytes;
};
inline GatedWorkspace carve_gated(void *base, int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank) {
    Cutter c{static_cast<unsigned char *>(base)};
    GatedWorkspace w{};
    if (C > 0) {
        w.offsets = c.take<int32_t>(size_t(C + 1) * 4);
        w.perm = c.take<int32_t>(size_t(N) * 4);
        w.t2 = c.take<uint16_t>(size_t(N) * 2 * rank * 2);
    }
    if (N <= kDecode) {
        const size_t plane = size_t(N) * 2 * F * 4;
        w.slices = molora::small_base_slices_rounds(N, d_in, 2 * F, C);
        w.base = c.take<float>(plane);
        if (w.slices > 1) w.planes = c.take<float>(plane * (w.slices - 1));
    } else {
        size_t bytes = size_t(molora::gemm_plane_floats(N, 2 * int64_t(F))) * 4;
        if (C > 0) bytes = std::max(bytes, shrink_scratch_up_to(N, d_in, C, rank));
        w.planes = c.take<float>(bytes);
    }
    w.bytes = c.at;
    return w;
}
inline int64_t padded_rows(int64_t N) { return (N + 7) & ~int64_t(7); }
inline bool backward_sizes_ok(int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank, int32_t act) {
    return gated_sizes_ok(N, d_in, F, C, rank, act) && molora::gated_backward_sizes_ok(N, padded_rows(N), d_in, F, C, rank);
}
// Room for any batch of up to N tokens: one of a few tokens may be cut into more slices than one of 64.
inline size_t gated_workspace_up_to(int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank) {
    size_t most = carve_gated(nullptr, N, d_in, F, C, rank).bytes;
    for (int64_t n = 1; n <= N && n <= kDecode; ++n) {
        const size_t b = carve_gated(nullptr, n, d_in, F, C, rank).bytes;
        most = b > most ? b : most;
    }
    return most;
}

struct BackwardWorkspace {
    int32_t *offsets, *perm;
    uint16_t *t2, *s2, *dh, *xt, *at, *bt;
    float *planes;
    size_t outer_a;  // floats of planes that dA takes
    size_t bytes;
};
inline BackwardWorkspace carve_backward(void *base, int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank) {
    Cutter c{static_cast<unsigned char *>(base)};
    BackwardWorkspace w{};
    if (C > 0) {
        w.offsets = c.take<int32_t>(size_t(C + 1) * 4);
        w.perm = c.take<int32_t>(size_t(N) * 4);
        w.t2 = c.take<uint16_t>(size_t(N) * 2 * rank * 2);
        w.s2 = c.take<uint16_t>(size_t(N) * 2 * rank * 2);
        w.at = c.take<uint16_t>(size_t(C) * rank * d_in * 2);
        w.bt = c.take<uint16_t>(size_t(C) * rank * 2 * F * 2);
    }
    w.dh = c.take<uint16_t>(size_t(padded_rows(N)) * 2 * F * 2);
    w.xt = c.take<uint16_t>(size_t(padded_rows(N)) * d_in * 2);
    // fp32 sums of one product at a time: slices of K of t, s, dx and dW, pieces of the rows of dA and dB
    size_t floats = size_t(molora::gemm_plane_floats(N, d_in));
    floats = std::max(floats, size_t(molora::gemm_plane_floats(d_in, 2 * int64_t(F))));
    w.outer_a = C > 0 ? round256(molora::grouped_outer_floats(N, d_in, rank) * 4) / 4 : 0;
    if (C > 0) {
        floats = std::max(floats, w.outer_a + molora::grouped_outer_floats(N, 2 * F, rank));
        floats = std::max(floats, std::max(shrink_scratch_up_to(N, d_in, C, rank), shrink_scratch_up_to(N, 2 * F, C, rank)) / 4);
    }
    w.planes = c.take<float>(floats * 4);
    w.bytes = c.at;
    return w;
}

// The dispatch step and t = x A_c of a batch of more than 64 tokens: one launch where that pays, as in molora_apply.
inline hipError_t dispatch_shrink(const int32_t *r, const uint16_t *x, const uint16_t *A, int32_t *offsets, int32_t *perm,
                                  uint16_t *t2, float *scratch, int64_t N, int32_t d_in, int32_t C, int32_t rank,
                                  hipStream_t s) {
    const molora::Mix plain{1, C, nullptr, nullptr};
    molora::SortArgs sort;
    if (molora::sort_large_in_shrink(N, d_in, C, rank)) {
        sort = molora::SortArgs{r, offsets, perm, nullptr};
    } else {
        const hipError_t e = molora::launch_bucket(r, offsets, perm, N, C, nullptr, s);
        if (e != hipSuccess) return e;
    }
    return molora::launch_shrink(x, A, offsets, perm, t2, N, d_in, C, rank, plain, s, scratch, sort);
}

#define MOLORA_TRY(call)                              \
    do {                                              \
        if ((call) != hipSuccess) return MOLORA_EHIP; \
    } while (0)

}  // namespace

extern "C" {

size_t molora_mx_codes_bytes(int64_t rows, int32_t K) { return mx_sizes_ok(rows, K) ? mx_codes(rows, K) : 0; }
size_t molora_mx_scales_bytes(int64_t rows, int32_t K) { return mx_sizes_ok(rows, K) ? mx_scales(rows, K) : 0; }

molora_status molora_mx_quantize(const void *src, int32_t src_type, void *codes, void *scales, int64_t rows, int32_t K,
                                 void *stream) {
    if (!mx_sizes_ok(rows, K) || (src_type != MOLORA_BF16 && src_type != MOLORA_F32)) return MOLORA_EINVAL;
    if (rows == 0) return MOLORA_OK;
    if (!src || !codes || !scales) return MOLORA_EINVAL;
    if (!aligned16(src) || !aligned16(codes) || !aligned16(scales)) return MOLORA_EALIGN;
    if (molora::ensure_device_ready() != hipSuccess) return MOLORA_EHIP;
    return from_hip(molora::launch_mx_quantize(src, src_type == MOLORA_F32, nullptr, static_cast<uint8_t *>(codes),
                                               static_cast<uint8_t *>(scales), rows, K, static_cast<hipStream_t>(stream)));
}

molora_status molora_mx_quantize_w(const void *W, void *codes, void *scales, int32_t d_in, int32_t d_out, void *stream) {
    if (d_out < 8 || d_out % 8 != 0 || !mx_sizes_ok(d_out, d_in)) return MOLORA_EINVAL;
    if (!W || !codes || !scales) return MOLORA_EINVAL;
    if (!aligned16(W) || !aligned16(codes) || !aligned16(scales)) return MOLORA_EALIGN;
    if (molora::ensure_device_ready() != hipSuccess) return MOLORA_EHIP;
    return from_hip(molora::launch_mx_quantize_w(static_cast<const uint16_t *>(W), static_cast<uint8_t *>(codes),
                                                 static_cast<uint8_t *>(scales), d_in, d_out,
                                                 static_cast<hipStream_t>(stream)));
}

molora_status molora_mx_dequantize(const void *codes, const void *scales, float *dst, int64_t rows, int32_t K,
                                   void *stream) {
    if (!mx_sizes_ok(rows, K)) return MOLORA_EINVAL;
    if (rows == 0) return MOLORA_OK;
    if (!codes || !scales || !dst) return MOLORA_EINVAL;
    if (!aligned16(codes) || !aligned16(scales) || !aligned16(dst)) return MOLORA_EALIGN;
    if (molora::ensure_device_ready() != hipSuccess) return MOLORA_EHIP;
    return from_hip(molora::launch_mx_dequantize(static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales),
                                                 dst, rows, K, static_cast<hipStream_t>(stream)));
}

molora_status molora_mx_matmul(const void *xc, const void *xs, const void *wc, const void *ws, float *h, int64_t N,
                               int32_t d_in, int32_t d_out, void *stream) {
    if (!mx_product_ok(N, d_in, d_out)) return MOLORA_EINVAL;
    if (N == 0) return MOLORA_OK;
    if (!xc || !xs || !wc || !ws || !h) return MOLORA_EINVAL;
    if (!aligned16(xc) || !aligned16(xs) || !aligned16(wc) || !aligned16(ws) || !aligned16(h)) return MOLORA_EALIGN;
    if (molora::ensure_device_ready() != hipSuccess) return MOLORA_EHIP;
    return from_hip(molora::launch_mx_gemm(static_cast<const uint8_t *>(xc), static_cast<const uint8_t *>(xs),
                                           static_cast<const uint8_t *>(wc), static_cast<const uint8_t *>(ws), nullptr,
                                           nullptr, nullptr, nullptr, h, N, d_in, d_out, 0, 0,
                                           static_cast<hipStream_t>(stream)));
}

molora_status molora_mx_matmul_tile(int64_t N, int32_t d_in, int32_t d_out, int32_t *tile) {
    if (!tile || N < 1 || !mx_product_ok(N, d_in, d_out)) return MOLORA_EINVAL;
    molora::mx_gemm_tile(N, d_in, d_out, tile);
    return MOLORA_OK;
}

size_t molora_apply_mx_workspace_bytes(int64_t N, int32_t d_in, int32_t d_out, int32_t C, int32_t rank) {
    if (!apply_sizes_ok(N, d_in, d_out, C, rank) || !mx_product_ok(N, d_in, d_out)) return 0;
    const size_t a = carve_mx(nullptr, N, d_in, C, rank).bytes, b = carve_mx(nullptr, N < kDecode ? N : kDecode, d_in, C, rank).bytes;
    return a > b ? a : b;
}

molora_status molora_apply_mx(const void *x, const void *wc, const void *ws, const void *A, const void *B, const int32_t *r,
                              float *h, int64_t N, int32_t d_in, int32_t d_out, int32_t C, int32_t rank, void *workspace,
                              size_t workspace_bytes, void *stream) {
    if (!apply_sizes_ok(N, d_in, d_out, C, rank) || !mx_product_ok(N, d_in, d_out)) return MOLORA_EINVAL;
    if (N == 0) return MOLORA_OK;
    if (!x || !wc || !ws || !A || !B || !r || !h || !workspace) return MOLORA_EINVAL;
    if (!aligned16(x) || !aligned16(wc) || !aligned16(ws) || !aligned16(A) || !aligned16(B) || !aligned16(r) ||
        !aligned16(h) || !aligned256(workspace))
        return MOLORA_EALIGN;
    const MxWorkspace w = carve_mx(workspace, N, d_in, C, rank);
    if (workspace_bytes < w.bytes) return MOLORA_EWORKSPACE;
    if (molora::ensure_device_ready() != hipSuccess) return MOLORA_EHIP;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint16_t *xb = static_cast<const uint16_t *>(x), *Ab = static_cast<const uint16_t *>(A);
    const uint8_t *wcb = static_cast<const uint8_t *>(wc), *wsb = static_cast<const uint8_t *>(ws);
    const uint16_t *Bb = static_cast<const uint16_t *>(B);
    if (N <= kDecode) {
        MOLORA_TRY(molora::launch_mx_decode_first(xb, Ab, r, w.codes, w.scales, w.planes, N, d_in, C, rank, s));
        return from_hip(molora::launch_mx_decode(w.codes, w.scales, wcb, wsb, Bb, r, w.planes, h, N, d_in, d_out, C, rank, s));
    }
    MOLORA_TRY(dispatch_shrink(r, xb, Ab, w.offsets, w.perm, w.t2, w.planes, N, d_in, C, rank, s));
    MOLORA_TRY(molora::launch_mx_quantize(x, false, w.perm, w.codes, w.scales, N, d_in, s));
    return from_hip(molora::launch_mx_gemm(w.codes, w.scales, wcb, wsb, Bb, w.t2, w.offsets, w.perm, h, N, d_in, d_out, C, rank, s));
}

size_t molora_apply_gated_workspace_bytes(int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank) {
    if (!gated_sizes_ok(N, d_in, F, C, rank, 0)) return 0;
    return gated_workspace_up_to(N, d_in, F, C, rank);
}

molora_status molora_apply_gated(const void *x, const void *W, const void *A, const void *B, const int32_t *r, void *z,
                                 float *pre, int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank, int32_t act,
                                 void *workspace, size_t workspace_bytes, void *stream) {
    if (!gated_sizes_ok(N, d_in, F, C, rank, act)) return MOLORA_EINVAL;
    if (N == 0) return MOLORA_OK;
    if (!x || !W || !z || !workspace || !adapters_given(A, B, r, C)) return MOLORA_EINVAL;
    if (!aligned16(x) || !aligned16(W) || !aligned16(A) || !aligned16(B) || !aligned16(r) || !aligned16(z) ||
        !aligned16(pre) || !aligned256(workspace))
        return MOLORA_EALIGN;
    const GatedWorkspace w = carve_gated(workspace, N, d_in, F, C, rank);
    if (workspace_bytes < w.bytes) return MOLORA_EWORKSPACE;
    if (molora::ensure_device_ready() != hipSuccess) return MOLORA_EHIP;
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint16_t *zb = static_cast<uint16_t *>(z);
    const uint16_t *xb = static_cast<const uint16_t *>(x), *Wb = static_cast<const uint16_t *>(W);
    const uint16_t *Ab = static_cast<const uint16_t *>(A), *Bb = static_cast<const uint16_t *>(B);
    if (N <= kDecode) {
        float *base = pre != nullptr ? pre : w.base;
        MOLORA_TRY(molora::launch_small_shrink_base(xb, Wb, Ab, base, w.t2, N, d_in, 2 * F, C, C > 0 ? rank : 8,
                                                    molora::Mix{1, C, nullptr, nullptr},
                                                    molora::SortArgs{r, w.offsets, w.perm, nullptr}, s, false, w.planes, w.slices));
        return from_hip(molora::launch_gated_finish(base, w.planes, w.slices, Bb, r, w.t2, w.perm, zb, pre, N, F, C, rank, act, s));
    }
    if (C > 0) MOLORA_TRY(dispatch_shrink(r, xb, Ab, w.offsets, w.perm, w.t2, w.planes, N, d_in, C, rank, s));
    return from_hip(molora::launch_gemm_gated(xb, Wb, Bb, w.t2, w.offsets, w.perm, pre, zb, w.planes, N, d_in, F, C, rank, act, s));
}

molora_status molora_apply_gated_tile(int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank, int32_t *tile) {
    if (!tile || N < 1 || !gated_sizes_ok(N, d_in, F, C, rank, 0)) return MOLORA_EINVAL;
    if (N <= kDecode) {
        tile[0] = (int32_t)(N + 15) / 16 * 16;
        tile[1] = 2 * molora::gated_finish_cols(F);
        tile[2] = 0;
        tile[3] = molora::small_base_slices_rounds(N, d_in, 2 * F, C);
    } else {
        molora::sliced_gemm_tile(N, d_in, 2 * F, C, rank, C > 0, tile);
    }
    return MOLORA_OK;
}

molora_status molora_gated_backward_tile(int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank, int32_t *dx_tile, int32_t *dW_tile) {
    if (!dx_tile || !dW_tile || N < 1 || !backward_sizes_ok(N, d_in, F, C, rank, 0)) return MOLORA_EINVAL;
    molora::sliced_gemm_tile(N, 2 * F, d_in, C, rank, false, dx_tile);
    molora::sliced_gemm_tile(d_in, (int)padded_rows(N), 2 * F, 0, 0, false, dW_tile);
    return MOLORA_OK;
}

size_t molora_gated_backward_workspace_bytes(int64_t N, int32_t d_in, int32_t F, int32_t C, int32_t rank) {
    return backward_sizes_ok(N, d_in, F, C, rank, 0) ? carve_backward(nullptr, N, d_in, F, C, rank).bytes : 0;
}

molora_status molora_gated_backward(const void *dz, const void *x, const void *W, const void *A, const void *B,
                                    const int32_t *r, const float *pre, void *dx, void *dW, void *dA, void *dB, int64_t N,
                                    int32_t d_in, int32_t F, int32_t C, int32_t rank, int32_t act, void *workspace,
                                    size_t workspace_bytes, void *stream) {
    if (!backward_sizes_ok(N, d_in, F, C, rank, act)) return MOLORA_EINVAL;
    if (C == 0 && (dA || dB)) return MOLORA_EINVAL;
    if (N == 0) {  // sums over no tokens
        if (!aligned16(dW) || !aligned16(dA) || !aligned16(dB)) return MOLORA_EALIGN;
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (dW) MOLORA_TRY(molora::launch_zero(dW, int64_t(d_in) * F * 4, s));
        if (dA) MOLORA_TRY(molora::launch_zero(dA, int64_t(C) * d_in * rank * 2, s));
        if (dB) MOLORA_TRY(molora::launch_zero(dB, int64_t(C) * rank * F * 4, s));
        return MOLORA_OK;
    }
    if (!dz || !x || !W || !pre || !adapters_given(A, B, r, C) || !workspace) return MOLORA_EINVAL;
    if (!aligned16(dz) || !aligned16(x) || !aligned16(W) || !aligned16(A) || !aligned16(B) || !aligned16(r) ||
        !aligned16(pre) || !aligned16(dx) || !aligned16(dW) || !aligned16(dA) || !aligned16(dB) || !aligned256(workspace))
        return MOLORA_EALIGN;
    const BackwardWorkspace w = carve_backward(workspace, N, d_in, F, C, rank);
    if (workspace_bytes < w.bytes) return MOLORA_EWORKSPACE;
    if (molora::ensure_device_ready() != hipSuccess) return MOLORA_EHIP;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint16_t *xb = static_cast<const uint16_t *>(x), *Wb = static_cast<const uint16_t *>(W);
    const uint16_t *Ab = static_cast<const uint16_t *>(A), *Bb = static_cast<const uint16_t *>(B);
    const molora::Mix plain{1, C, nullptr, nullptr};
    const int64_t Np = padded_rows(N);
    // the operands whose k runs down their columns, turned
    molora::TransposeJob turn[molora::kMaxTransposes];
    int turns = 0;
    if (C > 0 && (dx || dA)) turn[turns++] = {Bb, w.bt, C, rank, 2 * F, rank};
    if (C > 0 && dx) turn[turns++] = {Ab, w.at, C, d_in, rank, d_in};
    if (dW) turn[turns++] = {xb, w.xt, 1, N, d_in, Np};
    MOLORA_TRY(molora::launch_gate_backward(static_cast<const uint16_t *>(dz), pre, w.dh, N, Np, F, act, turn, turns, s));
    if (C > 0 && (dx || dA || dB)) {
        if (dB && N > kDecode)
            MOLORA_TRY(dispatch_shrink(r, xb, Ab, w.offsets, w.perm, w.t2, w.planes, N, d_in, C, rank, s));
        else
            MOLORA_TRY(molora::launch_bucket(r, w.offsets, w.perm, N, C, nullptr, s));
        if (dB && N <= kDecode) MOLORA_TRY(molora::launch_shrink(xb, Ab, w.offsets, w.perm, w.t2, N, d_in, C, rank, plain, s, w.planes));
        if (dx || dA)  // s = dh B^T
            MOLORA_TRY(molora::launch_shrink(w.dh, w.bt, w.offsets, w.perm, w.s2, N, 2 * F, C, rank, plain, s, w.planes));
        molora::GroupedOuter outer[2];
        int outers = 0;
        if (dA) outer[outers++] = {xb, w.s2, static_cast<uint16_t *>(dA), w.planes, d_in, false};
        if (dB) outer[outers++] = {w.dh, w.t2, static_cast<uint16_t *>(dB), w.planes + w.outer_a, 2 * F, true};
        MOLORA_TRY(molora::launch_grouped_outers(outer, outers, w.offsets, w.perm, N, C, rank, s));
    }
    if (dx)
        MOLORA_TRY(molora::launch_gemm_bf16(w.dh, Wb, w.at, w.s2, w.offsets, C > 0 ? w.perm : nullptr,
                                            static_cast<uint16_t *>(dx), w.planes, N, 2 * F, d_in, C, rank, true, s));
    if (dW)
        MOLORA_TRY(molora::launch_gemm_bf16(w.xt, w.dh, nullptr, nullptr, nullptr, nullptr, static_cast<uint16_t *>(dW), w.planes,
                                            d_in, (int)Np, 2 * F, 0, 0, false, s));
    return MOLORA_OK;
}

}  // extern "C"
