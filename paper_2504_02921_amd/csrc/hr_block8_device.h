// Device side of codes and scales: what the norm, the quantisers and the products' epilogues have in common.
#pragma once

#include <hip/hip_runtime.h>

#include "hr_block8.h"
#include "hr_device_types.h"

namespace hr {

// Largest value over groups of 16 lanes, in every lane of the group
__device__ __forceinline__ float max16(float v) {
    v = fmaxf(v, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x128, 0xF, 0xF, true)));      // row_ror:8
    v = fmaxf(v, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x124, 0xF, 0xF, true)));      // row_ror:4
    v = fmaxf(v, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x4E, 0xF, 0xF, true)));       // quad_perm:[2,3,0,1]
    v = fmaxf(v, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0xB1, 0xF, 0xF, true)));       // quad_perm:[1,0,3,2]
    return v;
}
__device__ __forceinline__ float sum16(float v) {
    v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x128, 0xF, 0xF, true));
    v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x124, 0xF, 0xF, true));
    v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x4E, 0xF, 0xF, true));
    v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0xB1, 0xF, 0xF, true));
    return v;
}

// Largest magnitude among finite values.  NaN loses every comparison of fmaxf; an infinity is looked for behind it, since there hardly ever is one
template <int N>
__device__ __forceinline__ float finite_top(const float (&v)[N]) {
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) top = fmaxf(top, fabsf(v[e]));
    if (top == __builtin_inff()) {
        top = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) top = fmaxf(top, fabsf(v[e]) < __builtin_inff() ? fabsf(v[e]) : 0.0f);
    }
    return top;
}

__device__ __forceinline__ float scale_of(float top) { return top == 0.0f ? 1.0f : fmaxf(top / kE4m3Top, kLeastScale); }

// Four values' codes, the first in the lowest byte.  The conversion rounds to nearest, ties to the even code; finite values are at most 448 (1 + 2^-22)
// here, which is nearer to 448 than to what would follow it, and what is not finite becomes the code NaN
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}

}  // namespace hr
