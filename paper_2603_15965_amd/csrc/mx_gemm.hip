// Products of 4-bit microscaled operands (layout in mx.h), with the grouped expand of routed adapters:
//
//     h[perm[p]][:] = Q(x)_p Q(W)  +  t_p B_{c(p)}
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 codes by 128 x 16, applies both blocks' scales and adds in
// fp32.  The products of two codes and their block sums are exact in fp32 (codes are multiples of 1/2 up to 6), so
// only the order of the additions over blocks is this kernel's.
#include <type_traits>

#include "lds_dma.h"
#include "mx_mfma.h"

namespace molora {

namespace {

// ---- larger batches: output tiles ----
// BM x BN output tile, WM x WN wavefronts of TM x TN tiles of 16 x 16.  A stage is 128 k of both sides, brought to
// LDS as it lies in memory; of three or four stages one is multiplied while the others travel, and a k tile costs one
// barrier.  The scales of 512 k have one place: a wavefront holds its own in registers for four k tiles, and
// the next ones are sent for when every wavefront has passed the barrier behind that read.
// 8192 x 12288 -> 4096: 176 us, 4.7 PFLOP/s.  On random codes the instruction sustains 6.9 from registers and 6.2 with its
// operands read from LDS at this tile's rate (zeros 9.7 and 8.3: power); without the loads of the loop the kernel takes
// 161 us.  Reads in front of a k tile's products instead of behind the products before: 204 us; two barriers and
// stages of 256 k, 258.  With d_in = 4096 the stores of h count: 16384 x 4096 -> 12288 takes 420 us in steady
// runs (403 at best; 440 to 490 under a kernel trace), 805 MB of them.
template <int WM_, int WN_, int TM_, int TN_, int STAGES_>
struct MxCfg {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, STAGES = STAGES_;
    static constexpr int NW = WM * WN, NT = NW * 64;
    static constexpr int RT = WM * TM, CT = WN * TN;  // 16-row and 16-column tiles
    static constexpr int BM = RT * 16, BN = CT * 16;
    static constexpr int PIECES = RT + CT, LPW = PIECES / NW;
    static constexpr int STAGE = PIECES * 1024;
    static constexpr int SP = PIECES / 4, SLPW = (SP + NW - 1) / NW;  // 1 KB holds the scales of four tiles
    static constexpr int B_STRIDE = BN * 2 + 32;  // a row of B in LDS: four consecutive rows on distinct banks
    static constexpr int OUT_STRIDE = TN * 64 + 16;  // a row of a wavefront's 16 rows on their way to h
    static constexpr size_t LDS_BYTES = STAGES * STAGE + SP * 1024;
    static_assert(STAGES >= 3 && STAGES <= 4, "scales are sent for after their place was read");
    static_assert(PIECES % NW == 0 && RT % 4 == 0 && CT % 4 == 0, "pieces split evenly");
    static_assert(2 * 32 * B_STRIDE <= STAGES * STAGE, "two slabs of B fit the stages");
    static_assert(NW * 16 * OUT_STRIDE <= STAGES * STAGE, "the epilogue fits the stages");
};

// (false: a sum is not finite; CAREFUL: common.h, find_not_finite)
template <class Cfg, bool CAREFUL>
__device__ __forceinline__ bool mx_gemm_body(
    const uint8_t *__restrict__ xc, const uint8_t *__restrict__ xs, const uint8_t *__restrict__ wc,
    const uint8_t *__restrict__ ws, const uint16_t *__restrict__ B, const uint16_t *__restrict__ t2,
    const int32_t *__restrict__ offsets, const int32_t *__restrict__ perm, float *__restrict__ h, int N, int d_out,
    int kt_n, int kg_n, int C, int R, int tiles_m, int tiles_n) {
    constexpr int TM = Cfg::TM, TN = Cfg::TN, RT = Cfg::RT, NW = Cfg::NW, STAGES = Cfg::STAGES;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    unsigned char *const scales = smem + STAGES * Cfg::STAGE;
    const int tid = fresh_thread<Cfg::NT>(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / Cfg::WN, wn = wave % Cfg::WN;

    // XCDs take runs of tiles, eight row tiles wide, so that each one's L2 holds its rows and columns
    const int total = tiles_m * tiles_n, share = (total + 7) / 8;
    const int logical = (int)(blockIdx.x % 8) * share + (int)(blockIdx.x / 8);
    if (blockIdx.x / 8 >= (unsigned)share || logical >= total) return true;
    const int group = logical / (8 * tiles_n), first = group * 8;
    const int width = min(8, tiles_m - first), in_group = logical - first * tiles_n;
    const int tile_m = first + in_group % width, tile_n = in_group / width;
    const int p0 = tile_m * Cfg::BM;
    const int64_t rt_last = (N + 15) / 16 - 1, ct_last = (d_out + 15) / 16 - 1;
    const int64_t rt0 = (int64_t)tile_m * RT, ct0 = (int64_t)tile_n * Cfg::CT;

    // this wavefront's pieces (rows first, then columns; a tile past the last one: the last one again) at k tile 0
    const uint8_t *src[Cfg::LPW];
#pragma unroll
    for (int i = 0; i < Cfg::LPW; ++i) {
        const int tile = i * NW + wave;
        const bool is_x = tile < RT;
        src[i] = (is_x ? xc : wc) + (is_x ? min(rt0 + tile, rt_last) : min(ct0 + tile - RT, ct_last)) * kt_n * 1024;
    }
    // piece i of k tile kt, to its stage
    auto issue_piece = [&](int kt, unsigned char *stage, int i) __attribute__((always_inline)) {
        load_to_lds16(src[i] + (int64_t)kt * 1024, lane * 16, stage + (i * NW + wave) * 1024);
    };
    const uint8_t *scale_src[Cfg::SLPW];  // this lane's
#pragma unroll
    for (int i = 0; i < Cfg::SLPW; ++i) {
        const int tile = (i * NW + wave) % Cfg::SP * 4 + (lane >> 4);  // (twice the same where there are more wavefronts than pieces)
        scale_src[i] = (tile < RT ? xs + min(rt0 + tile, rt_last) * kg_n * 256 : ws + min(ct0 + tile - RT, ct_last) * kg_n * 256) + (lane & 15) * 16;
    }
    auto issue_scales = [&](int kt) __attribute__((always_inline)) {  // of the four k tiles from kt on
#pragma unroll
        for (int i = 0; i < Cfg::SLPW; ++i)
            load_to_lds16_ptr(scale_src[i] + (int64_t)(kt >> 2) * 256, scales + (i * NW + wave) % Cfg::SP * 1024);
    };

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // A k tile is TM places, one x fragment times the TN of W each.  Behind a place's products the x fragment NA
    // places ahead is read, and in the last NA places the W fragments of the next k tile.  The workgroup barrier
    // sits in front of these: there every wavefront holds the last fragments of its k tile, so the stage is
    // filled again (k tile kt + STAGES) and the first fragments of the next one are read behind products.
    constexpr int NA = TM < 4 ? TM : 4;
    static_assert(TM % NA == 0, "a place's fragment is in register set place % NA");
    u32x4 x[NA], w[2][TN];
    uint32_t sx[TM], sw[TN], sw_next[TN];
    const unsigned char *const x_lane = smem + wm * TM * 1024 + lane * 16;
    const unsigned char *const w_lane = smem + (RT + wn * TN) * 1024 + lane * 16;
    const unsigned char *const s_lane = scales + lane * 4;
    auto read_x = [&](int stage, int i) __attribute__((always_inline)) { x[i % NA] = *(const u32x4 *)(x_lane + stage + i * 1024); };
    auto read_sx = [&](int i) __attribute__((always_inline)) { sx[i] = *(const uint32_t *)(s_lane + (wm * TM + i) * 256); };
    auto read_sw = [&](int j) __attribute__((always_inline)) { sw_next[j] = *(const uint32_t *)(s_lane + (RT + wn * TN + j) * 256); };

#pragma unroll
    for (int st = 0; st < STAGES; ++st) {
        if (st >= kt_n) break;
#pragma unroll
        for (int i = 0; i < Cfg::LPW; ++i) issue_piece(st, smem + st * Cfg::STAGE, i);
        if (st == 0) issue_scales(0);
    }
    if (kt_n >= STAGES)
        wait_vmcnt<(STAGES - 1) * Cfg::LPW>();
    else
        wait_vmcnt<0>();
    wg_barrier();
#pragma unroll
    for (int i = 0; i < NA; ++i) read_x(0, i);
#pragma unroll
    for (int j = 0; j < TN; ++j) w[0][j] = *(const u32x4 *)(w_lane + j * 1024);
#pragma unroll
    for (int i = 0; i < TM; ++i) read_sx(i);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        read_sw(j);
        sw[j] = sw_next[j];
    }

    // the first bucket that ends behind the tile's first row
    int c_first = C, lo_first = 0, hi_first = 0;
    for (int c0 = 0; c0 < C; c0 += 64) {
        const int end = offsets[min(c0 + lane, C - 1) + 1];
        const uint64_t behind = __ballot(end > p0);
        if (behind == 0) continue;
        const int first = __builtin_ctzll(behind);
        c_first = c0 + first;
        hi_first = __builtin_amdgcn_readlane(end, first);
        lo_first = __builtin_amdgcn_readfirstlane(offsets[c_first]);
        if (lo_first >= p0 + Cfg::BM) c_first = C;
        break;
    }
    int cur = 0;  // the k tile's stage, its offset
    // J: the k tile's byte of the scales, and the parity of its register set.  Without a branch inside, or the
    // compiler moves products behind later reads.
    auto multiply = [&](int kt, auto j_c) __attribute__((always_inline)) {
        constexpr int J = decltype(j_c)::value, LATE = TM - NA, PER = (Cfg::LPW + NA - 1) / NA;
        const int nxt = cur == (STAGES - 1) * Cfg::STAGE ? 0 : cur + Cfg::STAGE;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            if (i == LATE) {
                wait_lds();  // this wavefront has read the stage
                // its part of the next one is there; those behind it may be on their way
                wait_vmcnt<(STAGES - 2) * Cfg::LPW + (J == 2 || (STAGES == 4 && J == 1) ? Cfg::SLPW : 0)>();
                wg_barrier();
            }
            if (i >= LATE) {
#pragma unroll
                for (int j = i - LATE; j < TN; j += NA) w[(J + 1) & 1][j] = *(const u32x4 *)(w_lane + nxt + j * 1024);
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mx_mfma<J>(w[J & 1][j], x[i % NA], acc[i][j], sw[j], sx[i]);
            if (i < LATE) {
                read_x(cur, i + NA);
            } else {
                read_x(nxt, i - LATE);
                if (J == 3) {
#pragma unroll
                    for (int k = i % NA; k < TM; k += NA) read_sx(k);
#pragma unroll
                    for (int j = i - LATE; j < TN; j += NA) read_sw(j);
                }
#pragma unroll
                for (int u = (i - LATE) * PER; u < (i - LATE + 1) * PER && u < Cfg::LPW; ++u) issue_piece(kt + STAGES, smem + cur, u);
                if ((J + STAGES) % 4 == 0 && i == TM - 1) issue_scales(kt + STAGES);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (J == 3) {
#pragma unroll
            for (int j = 0; j < TN; ++j) sw[j] = sw_next[j];
        }
        cur = nxt;
    };
    int kt = 0;
    for (; kt + 3 + STAGES < kt_n; kt += 4) {
        multiply(kt, std::integral_constant<int, 0>{});
        multiply(kt + 1, std::integral_constant<int, 1>{});
        multiply(kt + 2, std::integral_constant<int, 2>{});
        multiply(kt + 3, std::integral_constant<int, 3>{});
    }
    // the last k tiles, at most STAGES + 3, one at a time; kt is a multiple of four, stage cur is there
    for (const int kt0 = kt; kt < kt_n; ++kt) {
        if (kt != kt0) {
            const int before = cur;
            cur = cur == (STAGES - 1) * Cfg::STAGE ? 0 : cur + Cfg::STAGE;
            wait_lds();
            if (kt + STAGES - 2 < kt_n)
                wait_vmcnt<(STAGES - 2) * Cfg::LPW>();
            else
                wait_vmcnt<0>();
            wg_barrier();
            if (const int next = kt - 1 + STAGES; next < kt_n) {
#pragma unroll
                for (int i = 0; i < Cfg::LPW; ++i) issue_piece(next, smem + before, i);
                if (next % 4 == 0) issue_scales(next);
            }
            if (kt % 4 == 0) {
#pragma unroll
                for (int i = 0; i < TM; ++i) read_sx(i);
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    read_sw(j);
                    sw[j] = sw_next[j];
                }
            }
        }
        u32x4 wt[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) wt[j] = *(const u32x4 *)(w_lane + cur + j * 1024);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const u32x4 xt = *(const u32x4 *)(x_lane + cur + i * 1024);
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mx_mfma<0>(wt[j], xt, acc[i][j], sw[j], sx[i]);
            sx[i] >>= 8;
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) sw[j] >>= 8;
    }
    // a tile that buckets have rows of, but no bucket all
    const bool look = !CAREFUL && c_first < C && !(lo_first <= p0 && hi_first >= min(p0 + Cfg::BM, N));
    int *const not_finite = (int *)scales;
    __syncthreads();  // the stages and the scales are free
    if (look && tid == 0) *not_finite = 0;  // (a barrier follows before it is set)

    // ---- expand: the buckets that own rows of the tile, 32 columns of t at a time ----
    // A fragment of 32 k is [hi | lo] of 16 columns of t against the same 16 rows of B twice.  The next step's rows of
    // B are on their way while one is multiplied; they go through LDS, which turns them, in two places.
    const int kq = lane >> 4, l16 = lane & 15;
    if (C > 0) {
        constexpr int PER = (32 * (Cfg::BN / 8) + Cfg::NT - 1) / Cfg::NT;  // 16-byte chunks of B per thread and step
        const int64_t n0 = ct0 * 16;
        u32x4 b_next[PER];
        i16x8 t[2][TM];
        auto fetch_b = [&](int c, int k0) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int i = tid + u * Cfg::NT, row = i / (Cfg::BN / 8), at = i % (Cfg::BN / 8);
                b_next[u] = *(const u32x4 *)(B + ((int64_t)c * R + min(k0 + row, R - 1)) * d_out + min(n0 + at * 8, (int64_t)d_out - 8));
            }
        };
        auto fetch_t = [&](int k0, int lo, int hi) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int first_row = p0 + (wm * TM + i) * 16, p = first_row + l16;
                if (hi <= first_row || lo >= first_row + 16) continue;
                const uint16_t *row = t2 + (int64_t)min(p, N - 1) * 2 * R + (kq >> 1) * R;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int kc = k0 + u * 16 + (kq & 1) * 8;
                    t[u][i] = *(const i16x8 *)(row + min(kc, R - 8));
                    if ((!CAREFUL && (p < lo || p >= hi)) || kc >= R) t[u][i] = i16x8{0, 0, 0, 0, 0, 0, 0, 0};
                }
            }
        };
        int c = c_first, lo = lo_first, hi = hi_first, place = 0;
        if (c < C) fetch_b(c, 0);
        for (int k0 = 0; c < C;) {
            unsigned char *const slab = smem + place * (32 * Cfg::B_STRIDE);
            place ^= 1;
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int i = tid + u * Cfg::NT, row = i / (Cfg::BN / 8), at = i % (Cfg::BN / 8);
                if (i < 32 * (Cfg::BN / 8)) *(u32x4 *)(slab + row * Cfg::B_STRIDE + at * 16) = b_next[u];
            }
            fetch_t(k0, lo, hi);
            const int lo_now = lo, hi_now = hi, parts = R - k0 > 16 ? 2 : 1;
            k0 += 32;
            if (k0 >= R) {  // the next bucket with rows, as long as it begins in the tile
                k0 = 0;
                do {
                    ++c;
                    lo = hi;
                    if (c < C) hi = __builtin_amdgcn_readfirstlane(offsets[c + 1]);
                } while (c < C && lo < p0 + Cfg::BM && lo == hi);
                if (lo >= p0 + Cfg::BM) c = C;
            }
            if (c < C) fetch_b(c, k0);
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (u >= parts) break;
                bf16x8 b[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const unsigned char *p = slab + (u * 16 + (kq & 1) * 8 + (l16 >> 2)) * Cfg::B_STRIDE + (wn * TN + j) * 32 + (l16 & 3) * 8;
                    const i16x4 v0 = lds_read_tr16((const MOLORA_LDS void *)p), v1 = lds_read_tr16((const MOLORA_LDS void *)(p + 4 * Cfg::B_STRIDE));
                    b[j] = __builtin_bit_cast(bf16x8, i16x8{v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]});
                }
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const int first_row = p0 + (wm * TM + i) * 16;
                    if (hi_now <= first_row || lo_now >= first_row + 16) continue;
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const f32x4 sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], __builtin_bit_cast(bf16x8, t[u][i]), acc[i][j], 0, 0, 0);
                        acc[i][j] = !CAREFUL || (uint32_t)(l16 + (first_row - lo_now)) < (uint32_t)(hi_now - lo_now) ? sum : acc[i][j];
                    }
                }
            }
        }
        if (look) {
            float seen = 0.f;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) find_not_finite(seen, acc[i][j]);
            if (seen != 0.f) *not_finite = 1;
        }
        __syncthreads();
    }

    // ---- epilogue: 16 rows at a time through a region of the wavefront's own, so that a store instruction
    // covers TN * 64 contiguous bytes of each of its rows ----
    unsigned char *const own = smem + wave * (16 * Cfg::OUT_STRIDE);
    constexpr int LPR = TN * 4, RPI = 64 / LPR;  // lanes to a row, rows to an instruction
    const int64_t col = (ct0 + wn * TN) * 16 + lane % LPR * 4;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j) *(f32x4 *)(own + l16 * Cfg::OUT_STRIDE + j * 64 + kq * 16) = acc[i][j];
#pragma unroll
        for (int k = 0; k < 16 / RPI; ++k) {
            const int in = k * RPI + lane / LPR, p = p0 + (wm * TM + i) * 16 + in;
            const f32x4 v = *(const f32x4 *)(own + in * Cfg::OUT_STRIDE + lane % LPR * 16);
            if (p < N && col < d_out) {
                const int64_t row = perm != nullptr ? perm[p] : p;
                __builtin_nontemporal_store(v, (f32x4 *)(h + row * d_out + col));
            }
        }
    }
    return !look || *not_finite == 0;
}

template <class Cfg>
__global__ __launch_bounds__(Cfg::NT, 2) void mx_gemm_kernel(
    const uint8_t *__restrict__ xc, const uint8_t *__restrict__ xs, const uint8_t *__restrict__ wc,
    const uint8_t *__restrict__ ws, const uint16_t *__restrict__ B, const uint16_t *__restrict__ t2,
    const int32_t *__restrict__ offsets, const int32_t *__restrict__ perm, float *__restrict__ h, int N, int d_out,
    int kt_n, int kg_n, int C, int R, int tiles_m, int tiles_n) {
    if (mx_gemm_body<Cfg, false>(xc, xs, wc, ws, B, t2, offsets, perm, h, N, d_out, kt_n, kg_n, C, R, tiles_m, tiles_n)) return;
    __syncthreads();  // nothing in LDS is read any more
    mx_gemm_body<Cfg, true>(xc, xs, wc, ws, B, t2, offsets, perm, h, N, d_out, kt_n, kg_n, C, R, tiles_m, tiles_n);
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
    launch_base_kernel(mx_gemm_kernel<Cfg>, dim3((unsigned)blocks), dim3(Cfg::NT), Cfg::LDS_BYTES, s, xc, xs, wc, ws, B, t2,
                       offsets, perm, h, (int)N, d_out, mx_k_tiles(d_in), mx_k_groups(d_in), C, rank, (int)tiles_m, (int)tiles_n);
    return hipGetLastError();
}

}  // namespace

using Mx256 = MxCfg<2, 4, 8, 4, 4>;   // 256 x 256, one workgroup per compute unit
using MxWide = MxCfg<2, 2, 8, 4, 3>;  // 256 x 128, two
using Mx128 = MxCfg<2, 2, 4, 4, 3>;   // 128 x 128, three
using Mx128Deep = MxCfg<2, 2, 4, 4, 4>;  // the same with a stage more, two
using MxLow = MxCfg<1, 4, 4, 2, 4>;   // 64 x 128, four
using Mx64 = MxCfg<2, 2, 2, 2, 4>;    // 64 x 64, five

namespace {
// The tile from the sizes: the least of the costs below (us).  Tiles run in rounds of 256 compute units x workgroups per
// unit; a whole round costs a start and an end and a time per k tile of 128, the last one parts of both that
// grow with its share of the places.  Coefficients: non-negative least squares of the relative error over 128
// shapes, 65 .. 16384 rows, 256 .. 12288 deep, 1024 .. 12288 wide, every configuration timed on each with its operands
// from HBM.  The choice is 3 % behind the best configuration there (geometric mean, but for a few timings that were
// disturbed at most 26 %).  Over 60 products of 8 .. 1024 columns, which the fit has not seen, it is 1.3 % behind (at most
// 21 %: 12586 x 768 -> 488 13.2 us, in 64 x 64 tiles 10.9).
struct MxCost {
    int bm, bn, per_cu;
    double once, round, part, last, k_round, k_part, k_last;
};
constexpr MxCost kMxCosts[] = {
    {256, 256, 1, 2.2, 12.0, 5.4, 4.3, 0.762, 0.523, 0.163}, {256, 128, 2, 7.3, 9.5, 0.0, 4.4, 0.774, 0.322, 0.341},
    {128, 128, 3, 3.5, 6.3, 1.2, 4.3, 0.651, 0.232, 0.364},  {128, 128, 2, 4.4, 4.4, 0.7, 2.5, 0.457, 0.185, 0.197},
    {64, 128, 4, 3.7, 3.9, 0.0, 3.0, 0.588, 0.125, 0.389},   {64, 64, 5, 3.0, 2.4, 0.0, 2.2, 0.447, 0.100, 0.337}};

int mx_tile_choice(int64_t N, int d_in, int d_out) {
    const double kt = mx_k_tiles(d_in);
    double best = 1e30;
    int pick = 0;
    for (int i = 0; i < 6; ++i) {
        const MxCost &c = kMxCosts[i];
        const int64_t tiles = ((N + c.bm - 1) / c.bm) * (((int64_t)d_out + c.bn - 1) / c.bn), slots = 256 * c.per_cu;
        const double full = (double)(tiles / slots), last = (double)(tiles % slots) / (double)slots, part = last > 0 ? 1 : 0;
        const double cost = c.once + full * (c.round + kt * c.k_round) + part * (c.part + kt * c.k_part) + last * (c.last + kt * c.k_last);
        if (cost < best) {
            best = cost;
            pick = i;
        }
    }
    return pick;
}
}  // namespace

void mx_gemm_tile(int64_t N, int d_in, int d_out, int32_t *tile) {
    static constexpr int stages[] = {Mx256::STAGES, MxWide::STAGES, Mx128::STAGES, Mx128Deep::STAGES, MxLow::STAGES, Mx64::STAGES};  // the order of kMxCosts
    const int pick = N <= 64 ? -1 : mx_tile_choice(N, d_in, d_out);
    tile[0] = pick < 0 ? (int)mx_row_tiles(N) * 16 : kMxCosts[pick].bm;
    tile[1] = pick < 0 ? mx_decode_cols(d_out) : kMxCosts[pick].bn;
    tile[2] = pick < 0 ? 0 : stages[pick];
}

hipError_t launch_mx_gemm(const uint8_t *xc, const uint8_t *xs, const uint8_t *wc, const uint8_t *ws, const uint16_t *B,
                          const uint16_t *t2, const int32_t *offsets, const int32_t *perm, float *h, int64_t N, int d_in,
                          int d_out, int C, int rank, hipStream_t s) {
    if (N == 0) return hipSuccess;
    if (N <= 64 && C == 0) return launch_mx_decode(xc, xs, wc, ws, nullptr, nullptr, nullptr, h, N, d_in, d_out, 0, 0, s);
#define MOLORA_MX_TILES(CFG) launch_mx_tiles<CFG>(xc, xs, wc, ws, B, t2, offsets, perm, h, N, d_in, d_out, C, rank, s)
    switch (mx_tile_choice(N, d_in, d_out)) {  // the order of kMxCosts
        case 0: return MOLORA_MX_TILES(Mx256);
        case 1: return MOLORA_MX_TILES(MxWide);
        case 2: return MOLORA_MX_TILES(Mx128);
        case 3: return MOLORA_MX_TILES(Mx128Deep);
        case 4: return MOLORA_MX_TILES(MxLow);
        default: return MOLORA_MX_TILES(Mx64);
    }
#undef MOLORA_MX_TILES
}

}  // namespace molora
