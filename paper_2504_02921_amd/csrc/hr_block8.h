// The operators of a layer's projections in 8 bits (hr_rms_norm, hr_block_quantize, hr_block_matmul): what their host and device parts share.
#pragma once

#include <cstddef>
#include <cstdint>

#include "hr_internal.h"
#include "hr_layout.h"

namespace hr {

constexpr int kBlockCols = HR_BLOCK_COLS;
constexpr float kE4m3Top = 448.0f, kLeastScale = 1.17549435e-38f;      // 2^-126: its reciprocal is finite
constexpr int64_t kMaxWorkgroups = (1 << 24) - 512;                    // of a launch
HR_HD int64_t blocks_of(int64_t n) { return (n + kBlockCols - 1) / kBlockCols; }

// ---- norm
// How a head's channels are spread: `lanes` lanes have a head (16, 32 or 64 of a wavefront, or a workgroup's 256), `chunks` times 8 channels each;
// chunks = 0: more channels than that holds, read twice
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
    const float* bias;
    const void* add;
    void* out;
    int64_t add_stride, out_stride;
    uint8_t* codes;            // block8
    float* scales;
    int64_t code_stride, scale_stride;
};
MatmulArgs matmul_args(const hr_block8& a, const hr_block8& w, const hr_matmul_args& m);

// A product's tile: BM rows x BN columns of y
struct MatmulTile { int bm, bn; bool few; };
MatmulTile matmul_tile(int64_t M, int N, int K, int dtype, int gate, bool block8);

}  // namespace hr
