// The operators of a layer's projections in 8 bits (hr_rms_norm, hr_block_quantize, hr_block_matmul): what their host and device parts share.
#pragma once

#include <cstddef>
#include <cstdint>

#include "hr_internal.h"
#include "hr_layout.h"

namespace hr {

constexpr int kBlockCols = HR_BLOCK_COLS;
constexpr float kE4m3Top = 448.0f, kLeastScale = 1.17549435e-38f;      // 2^-126: its reciprocal is finite
// Of a launch, whose lanes are counted in 32 bits: workgroups of 256 lanes, and of up to 1024
constexpr int64_t kMaxWorkgroups = (1 << 24) - 512, kMaxWideWorkgroups = (1 << 22) - 512;
HR_HD int64_t blocks_of(int64_t n) { return (n + kBlockCols - 1) / kBlockCols; }

// ---- norm
// How a head's channels are spread: `lanes` lanes have a head (16, 32 or 64 of a wavefront, or a workgroup's 128 to 1024), `chunks` times 8 channels each;
// chunks = 0: more channels than that holds, read twice.
struct NormShape { int lanes, chunks; };
NormShape norm_shape(int channels, int64_t rows);
int norm_check(const hr_norm_args* a);

// ---- codes
int block8_check(const hr_block8* b, int block_rows);
int quantize_check(int dtype, const void* x, int64_t x_stride, const hr_block8* out);

// ---- product
int matmul_check(const hr_block8* a, const hr_block8* w, const hr_matmul_args* args);
struct MatmulArgs {
    const uint8_t *a, *w;
    const float *a_scales, *w_scales;
    int64_t a_stride, a_scale_stride, w_stride, w_scale_stride;
    int64_t M;
    int32_t N, K;              // N: columns of y (half of w's rows with a gate)
    int32_t half;              // rows of w from a gate's row to the row it multiplies; 0: no gate
    int32_t gate;
    bool eight;                // the 8-bit instruction
    const float* bias;
    const void* add;
    void* out;
    int64_t add_stride, out_stride;
    uint8_t* codes;            // block8
    float* scales;
    int64_t code_stride, scale_stride;
};
MatmulArgs matmul_args(const hr_block8& a, const hr_block8& w, const hr_matmul_args& m);

// Tiles of a product: rows x rows of w (with a gate half as many columns of y), _n: n groups of wavefronts that take turns along k
enum MatmulShape {
    MM_FEW_16, MM_FEW_32,            // no LDS on the way in: 16 rows x 16 or 32 columns of y
    MM_16x32_8, MM_32x32_8, MM_16x64_4, MM_32x64_2, MM_64x64, MM_64x64_2, MM_64x128, MM_64x128_2, MM_64x256, MM_128x128, MM_128x128_2, MM_128x256, MM_256x256,
    MM_16x128_4, MM_32x128_2, MM_16x256, MM_32x256,      // into codes only
    MM_SHAPES
};
struct MatmulPlan { int shape; int64_t rows; int rest; };      // the first `rows` rows, and the shape of what is left
MatmulPlan matmul_plan(const MatmulArgs& a);
int64_t matmul_tiles(int shape, const MatmulArgs& a, int64_t rows);
MatmulArgs matmul_rows(const MatmulArgs& a, int dtype, int64_t first, int64_t rows);

}  // namespace hr
