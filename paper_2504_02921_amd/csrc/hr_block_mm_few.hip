// Products of 8-bit matrices with few rows (hr_block_matmul): the weights' bytes are what counts.
//
// A workgroup has a tile of y and its wavefronts share the sum over k: wavefront ks takes the 128-column blocks ks, ks + KS, .. of both
// operands straight into registers, in the order that the matrix instruction wants (a lane has 16 codes of either half of one row's block; the columns come in
// another order than the instruction's own, the same for both operands).  Codes become halves, which are exact, and
// a block's sum of 128 products starts at zero and is added in fp32 with the product of the two scales.  At the end the wavefronts' sums meet in LDS,
// which also turns them into rows for what follows.
//
// y[m][n] = sum over blocks b of a.scale[m][b] w.scale[n / 128][b] sum over k in b of a[m][k] w[n][k].  A row of y reads all of w once, so its bytes at the
// memory's rate are what a call cannot do without; 16 x 16 or 16 x 32 tiles are the most workgroups that still read whole lines of w, and eight
// wavefronts with two blocks each under way ask for up to 64 KB a compute unit at once.  1 x 4096 x 4096 (17 MB): 5.7 us, 2.9 TB/s, of which 2.3 to 3.2 are the
// launch, the first answer from memory and the join; 1 x 4096 x 14336 (59 MB) 11.8 us, 5.0 TB/s.  Rows share w's lines in the L2s only: from a dozen or two rows on, and
// for weights of more than 256 tiles, the tiles through LDS are faster.
#include <hip/hip_runtime.h>

#include "hr_block_mm.h"

namespace hr {

namespace {

constexpr int KS = 8, DEPTH = 2;         // wavefronts along k; blocks that a wavefront has under way

// 16 rows x NT times 16 columns of y (with a gate NT times 16 of either half)
template <int NT, bool GATE, typename OUT>
__global__ void __launch_bounds__(KS * 64) block_mm_few_kernel(MatmulArgs a) {
    constexpr int H = GATE ? 2 : 1, BM = 16, BN = 16 * NT, PITCH = H * BN + 4;
    __shared__ __attribute__((aligned(16))) float sums[KS * BM * PITCH];
    const int tiles_m = (int)((a.M + BM - 1) / BM), tiles_n = (a.N + BN - 1) / BN;
    const TileCoord tc = map_tile(blockIdx.x, tiles_m, tiles_n);
    if (!tc.valid) return;
    const int64_t m0 = (int64_t)tc.tm * BM;
    const int n0 = tc.tn * BN;
    const int lane = threadIdx.x & 63, ks = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, fq = lane >> 4;
    const int nk = (int)blocks_of(a.K);

    // rows behind the last one are read as that, and not stored
    const int64_t m = min(m0 + r, a.M - 1);
    const uint8_t *pa = a.a + m * a.a_stride + 16 * fq, *pw[H][NT];
    const float *sa = a.a_scales + m * a.a_scale_stride, *sw[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
#pragma unroll
        for (int j = 0; j < NT; ++j) pw[h][j] = a.w + (min(n0 + 16 * j + r, a.N - 1) + (int64_t)h * a.half) * a.w_stride + 16 * fq;
        sw[h] = a.w_scales + (n0 + (int64_t)h * a.half) / kBlockCols * a.w_scale_stride;
    }

    struct Block {
        mm_i4 a[2], w[H][NT][2];
        float sa, sw[H];
    } blk[DEPTH];
    auto load = [&](Block& b, int kt) {
        const int at = kt * kBlockCols;
        if (at + kBlockCols <= a.K) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int j = 0; j < NT; ++j) b.w[h][j][c] = *(const mm_i4*)(pw[h][j] + at + 64 * c);
                b.a[c] = *(const mm_i4*)(pa + at + 64 * c);
            }
        } else {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int left = a.K - (at + 16 * fq + 64 * c);
                const bool some = left > 0;
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int j = 0; j < NT; ++j) b.w[h][j][c] = some ? first_codes(*(const mm_i4*)(pw[h][j] + at + 64 * c), left) : mm_i4{0, 0, 0, 0};
                b.a[c] = some ? first_codes(*(const mm_i4*)(pa + at + 64 * c), left) : mm_i4{0, 0, 0, 0};
            }
        }
        b.sa = sa[kt];
#pragma unroll
        for (int h = 0; h < H; ++h) b.sw[h] = sw[h][kt];
    };

    mm_f4 acc[H][NT];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[h][j] = mm_f4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Block& b) {
        mm_h8 ah[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) ah[s] = halves(b.a[s / 2][s % 2 * 2], b.a[s / 2][s % 2 * 2 + 1]);
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                mm_f4 part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const mm_h8 wh = halves(b.w[h][j][s / 2][s % 2 * 2], b.w[h][j][s / 2][s % 2 * 2 + 1]);
                    part = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh, ah[s], part, 0, 0, 0);
                }
                const float scale = b.sa * b.sw[h];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[h][j][e] = fmaf(part[e], scale, acc[h][j][e]);
            }
    };

#pragma unroll
    for (int p = 0; p < DEPTH; ++p)
        if (ks + p * KS < nk) load(blk[p], ks + p * KS);
    for (int k0 = ks; k0 < nk; k0 += KS * DEPTH) {
#pragma unroll
        for (int p = 0; p < DEPTH; ++p) {
            const int kt = k0 + p * KS;
            if (kt < nk) {
                multiply(blk[p]);
                if (kt + KS * DEPTH < nk) load(blk[p], kt + KS * DEPTH);
            }
        }
    }

    // a lane has row r of a tile and four of its columns
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int j = 0; j < NT; ++j) *(mm_f4*)(sums + (ks * BM + r) * PITCH + h * BN + 16 * j + 4 * fq) = acc[h][j];
    __syncthreads();
    constexpr int Q = BN / 4;
    if (threadIdx.x >= BM * Q) return;
    const int row = threadIdx.x / Q, col = threadIdx.x % Q * 4;
    mm_f4 c = {0.f, 0.f, 0.f, 0.f}, up = c;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        c += *(const mm_f4*)(sums + (s * BM + row) * PITCH + col);
        if (GATE) up += *(const mm_f4*)(sums + (s * BM + row) * PITCH + BN + col);
    }
    if (m0 + row < a.M && n0 + col < a.N) store4<OUT>(a, m0 + row, n0 + col, finish4<GATE>(a, n0 + col, c, up));
}

template <int NT, bool GATE, typename OUT>
hipError_t launch(const MatmulArgs& a, hipStream_t st) {
    const int64_t tiles = (a.M + 15) / 16 * ((a.N + 16 * NT - 1) / (16 * NT));
    block_mm_few_kernel<NT, GATE, OUT><<<(unsigned)((tiles + kXcds - 1) / kXcds * kXcds), KS * 64, 0, st>>>(a);
    return hipGetLastError();
}

template <int NT>
hipError_t launch_shape(const MatmulArgs& a, int dtype, hipStream_t st) {
    if (dtype == HR_F32) return a.half > 0 ? launch<NT, true, float>(a, st) : launch<NT, false, float>(a, st);
    return a.half > 0 ? launch<NT, true, bf16_t>(a, st) : launch<NT, false, bf16_t>(a, st);
}

}  // namespace

hipError_t launch_block_matmul_few(const MatmulArgs& a, int dtype, int shape, hipStream_t st) {
    return shape == MM_FEW_16 ? launch_shape<1>(a, dtype, st) : launch_shape<2>(a, dtype, st);
}

}  // namespace hr
