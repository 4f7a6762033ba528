// Products of 8-bit matrices with few rows (hr_block_matmul): the weights' bytes are what counts.
//
// A workgroup has a tile of y and its wavefronts share the sum over k: wavefront ks takes the 128-column blocks ks, ks + KS, .. of both
// operands straight into registers, in the order that the matrix instruction wants (a lane has 16 codes of either half of one row's block; the columns come in
// another order than the instruction's own, the same for both operands).  Codes become halves, which are exact, and
// a block's sum of 128 products starts at zero and is added in fp32 with the product of the two scales.  At the end the wavefronts' sums meet in LDS,
// which also turns them into rows for what follows.
#include <hip/hip_runtime.h>

#include "hr_block_mm.h"

namespace hr {

namespace {

// MT x NT tiles of 16 x 16 of y a workgroup (with a gate NT of either half), KS wavefronts along k times CS along the columns, DEPTH blocks under way
template <int MT, int NT, int KS, int CS, int DEPTH, bool GATE, typename OUT, bool CODES>
__global__ void __launch_bounds__(KS * CS * 64) block_mm_few_kernel(MatmulArgs a) {
    constexpr int NW = NT / CS, H = GATE ? 2 : 1, BM = 16 * MT, BN = 16 * NT, PITCH = H * BN + 4;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float* sums = (float*)smem;                           // [KS][BM][PITCH]
    const int tiles_m = (int)((a.M + BM - 1) / BM), tiles_n = (a.N + BN - 1) / BN;
    const TileCoord tc = map_tile(blockIdx.x, tiles_m, tiles_n);
    if (!tc.valid) return;
    const int64_t m0 = (int64_t)tc.tm * BM;
    const int n0 = tc.tn * BN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ks = wave / CS, cs = wave % CS, r = lane & 15, fq = lane >> 4;
    const int nk = (int)blocks_of(a.K);

    // rows behind the last one are read as that, and not stored
    const uint8_t *pa[MT], *pw[H][NW];
    const float *sa[MT], *sw[H];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = min(m0 + 16 * i + r, a.M - 1);
        pa[i] = a.a + m * a.a_stride + 16 * fq;
        sa[i] = a.a_scales + m * a.a_scale_stride;
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
#pragma unroll
        for (int j = 0; j < NW; ++j) pw[h][j] = a.w + (int64_t)(min(n0 + 16 * (cs * NW + j) + r, a.N - 1) + h * a.half) * a.w_stride + 16 * fq;
        sw[h] = a.w_scales + (int64_t)((n0 + h * a.half) / kBlockCols) * a.w_scale_stride;
    }

    struct Block {
        mm_i4 a[MT][2], w[H][NW][2];
        float sa[MT], sw[H];
    } blk[DEPTH];
    auto load = [&](Block& b, int kt) {
        const int at = kt * kBlockCols;
        if (at + kBlockCols <= a.K) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int j = 0; j < NW; ++j) b.w[h][j][c] = *(const mm_i4*)(pw[h][j] + at + 64 * c);
#pragma unroll
                for (int i = 0; i < MT; ++i) b.a[i][c] = *(const mm_i4*)(pa[i] + at + 64 * c);
            }
        } else {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int left = a.K - (at + 16 * fq + 64 * c);
                const bool some = left > 0;
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int j = 0; j < NW; ++j) b.w[h][j][c] = some ? first_codes(*(const mm_i4*)(pw[h][j] + at + 64 * c), left) : mm_i4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < MT; ++i) b.a[i][c] = some ? first_codes(*(const mm_i4*)(pa[i] + at + 64 * c), left) : mm_i4{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) b.sa[i] = sa[i][kt];
#pragma unroll
        for (int h = 0; h < H; ++h) b.sw[h] = sw[h][kt];
    };

    mm_f4 acc[MT][H][NW];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < NW; ++j) acc[i][h][j] = mm_f4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Block& b) {
        mm_h8 ah[MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s) ah[i][s] = halves(b.a[i][s / 2][s % 2 * 2], b.a[i][s / 2][s % 2 * 2 + 1]);
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < NW; ++j) {
                mm_f4 part[MT];
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const mm_h8 wh = halves(b.w[h][j][s / 2][s % 2 * 2], b.w[h][j][s / 2][s % 2 * 2 + 1]);
#pragma unroll
                    for (int i = 0; i < MT; ++i)
                        part[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh, ah[i][s], s == 0 ? mm_f4{0.f, 0.f, 0.f, 0.f} : part[i], 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const float scale = b.sa[i] * b.sw[h];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][h][j][e] = fmaf(part[i][e], scale, acc[i][h][j][e]);
                }
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
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < NW; ++j) *(mm_f4*)(sums + (ks * BM + 16 * i + r) * PITCH + h * BN + 16 * (cs * NW + j) + 4 * fq) = acc[i][h][j];
    __syncthreads();
    constexpr int Q = BN / 4;
    for (int u = threadIdx.x; u < BM * Q; u += KS * CS * 64) {
        const int row = u / Q, col = u % Q * 4;
        mm_f4 c = {0.f, 0.f, 0.f, 0.f}, up = c;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            c += *(const mm_f4*)(sums + (s * BM + row) * PITCH + col);
            if (GATE) up += *(const mm_f4*)(sums + (s * BM + row) * PITCH + BN + col);
        }
        const int64_t m = m0 + row;
        const mm_f4 y = finish4<GATE>(a, n0 + col, c, up);
        if constexpr (CODES) store_block4(a, m, n0 + col, y, m < a.M);
        else if (m < a.M) store4<OUT>(a, m, n0 + col, y);
    }
}

template <int MT, int NT, int KS, int CS, int DEPTH, bool GATE, typename OUT, bool CODES>
hipError_t launch(const MatmulArgs& a, hipStream_t st) {
    constexpr size_t lds = (size_t)KS * 16 * MT * ((GATE ? 2 : 1) * 16 * NT + 4) * sizeof(float);
    const auto kernel = block_mm_few_kernel<MT, NT, KS, CS, DEPTH, GATE, OUT, CODES>;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    const int64_t tiles = (a.M + 16 * MT - 1) / (16 * MT) * ((a.N + 16 * NT - 1) / (16 * NT));
    kernel<<<(unsigned)((tiles + kXcds - 1) / kXcds * kXcds), KS * CS * 64, lds, st>>>(a);
    return hipGetLastError();
}

template <int MT, int DEPTH>
hipError_t launch_rows(const MatmulArgs& a, int dtype, hipStream_t st) {
    const bool gate = a.half > 0;
    if (a.codes) {
        constexpr int KS = MT == 4 ? 2 : 4;
        return gate ? launch<MT, 8, KS, 4, 1, true, float, true>(a, st) : launch<MT, 8, KS, 4, 2, false, float, true>(a, st);
    }
    if (dtype == HR_F32) return gate ? launch<MT, 1, 8, 1, DEPTH, true, float, false>(a, st) : launch<MT, 2, 8, 1, DEPTH, false, float, false>(a, st);
    return gate ? launch<MT, 1, 8, 1, DEPTH, true, bf16_t, false>(a, st) : launch<MT, 2, 8, 1, DEPTH, false, bf16_t, false>(a, st);
}

}  // namespace

hipError_t launch_block_matmul_few(const MatmulArgs& a, int dtype, const MatmulTile& t, hipStream_t st) {
    switch (t.bm) {
        case 16: return launch_rows<1, 4>(a, dtype, st);
        case 32: return launch_rows<2, 3>(a, dtype, st);
        default: return launch_rows<4, 2>(a, dtype, st);
    }
}

}  // namespace hr
