// Products of 8-bit matrices (hr_block_matmul): what their kernels have in common.
#pragma once

#include <hip/hip_runtime.h>

#include "hr_block8_device.h"
#include "hr_gemm_tiles.h"

namespace hr {

constexpr int kCus = 256;

typedef __attribute__((ext_vector_type(4))) float mm_f4;
typedef __attribute__((ext_vector_type(2))) _Float16 mm_h2;
typedef __attribute__((ext_vector_type(8))) _Float16 mm_h8;
typedef __attribute__((ext_vector_type(4))) int mm_i4;

// Eight codes as halves: every E4M3 value is one
__device__ __forceinline__ mm_h8 halves(int lo, int hi) {
    const mm_h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const mm_h2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return mm_h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The codes at `at` .. `at` + 15 of a row, those behind its last one as zeros: `left` = columns from `at` to the row's end, of 1 .. 15
__device__ __forceinline__ mm_i4 first_codes(mm_i4 w, int left) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int keep = left - q * 4;
        w[q] = keep >= 4 ? w[q] : keep <= 0 ? 0 : w[q] & (int)(0xFFFFFFFFu >> (32 - 8 * keep));
    }
    return w;
}

// A gate's act(z) u.  Both acts are z / (1 + exp(-t)): silu with t = z, gelu with t = 2 sqrt(2 / pi) (z + 0.044715 z^3).  exp(-t) is 2^x with
// x = -t / ln 2 in two parts, as one would lose |x| 2^-24 of the result; both instructions are good to their last digit.  Beyond +-200 it is infinite or zero
__device__ __forceinline__ float gated(float z, float u, int gate) {
    float t = gate == HR_GATE_SILU ? z : 1.5957691216057308f * fmaf(0.044715f * z * z, z, z);
    t = fminf(fmaxf(t, -200.0f), 200.0f);
    const float x = -1.44269504088896341f * t, rest = fmaf(-1.44269504088896341f, t, -x) - 1.9259629911e-8f * t;
    const float power = __builtin_amdgcn_exp2f(x);
    return z * __builtin_amdgcn_rcpf(1.0f + (power < __builtin_inff() ? fmaf(power, 0.69314718f * rest, power) : power)) * u;
}

// Values n .. n + 3 of y's row m, from c and, with a gate, from what it multiplies
template <bool GATE>
__device__ __forceinline__ mm_f4 finish4(const MatmulArgs& a, int n, mm_f4 c, mm_f4 up) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (a.bias) {
            c[e] += n + e < a.N ? a.bias[n + e] : 0.0f;
            if (GATE) up[e] += n + e < a.N ? a.bias[a.half + n + e] : 0.0f;
        }
        if (GATE) c[e] = gated(c[e], up[e], a.gate);
    }
    return c;
}

// ... + add, into out
template <typename T>
__device__ __forceinline__ void store4(const MatmulArgs& a, int64_t m, int n, mm_f4 y) {
    T* out = (T*)a.out + m * a.out_stride + n;
    const T* add = (const T*)a.add + m * a.add_stride + n;
    if (n + 4 <= a.N) {
        Loose<T, 4> w;
        if (a.add) {
            w = *(const Loose<T, 4>*)add;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] += to_float<T>(w.w[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) w.w[e] = from_float<T>(y[e]);
        *(Loose<T, 4>*)out = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.N) out[e] = from_float<T>(a.add ? y[e] + to_float<T>(add[e]) : y[e]);
    }
}

template <typename T>
__device__ __forceinline__ void store8(const MatmulArgs& a, int64_t m, int n, mm_f4 lo, mm_f4 hi) {
    if (n + 8 <= a.N) {
        T* out = (T*)a.out + m * a.out_stride + n;
        const T* add = (const T*)a.add + m * a.add_stride + n;
        Loose<T, 8> w;
        if (a.add) {
            w = *(const Loose<T, 8>*)add;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] += to_float<T>(w.w[e]);
                hi[e] += to_float<T>(w.w[4 + e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w.w[e] = from_float<T>(lo[e]);
            w.w[4 + e] = from_float<T>(hi[e]);
        }
        *(Loose<T, 8>*)out = w;
    } else {
        if (n < a.N) store4<T>(a, m, n, lo);
        if (n + 4 < a.N) store4<T>(a, m, n + 4, hi);
    }
}

// Largest value over the lanes l, l ^ 16, l ^ 32 and l ^ 48, in each of them
__device__ __forceinline__ float max_over_fq(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// A row's codes in NY blocks of 16 columns from n0 on, of which a lane has columns 4 fq .. 4 fq + 3 in w[block]: swapped among the four lanes of a row until
// a lane has what NY of them had of one block
template <int NY>
__device__ __forceinline__ void store_codes(const MatmulArgs& a, int64_t m, int n0, int fq, uint32_t (&w)[NY]) {
    static_assert(NY == 1 || NY == 2 || NY == 4, "blocks of a wavefront");
    int n = n0 + 4 * fq;
    if constexpr (NY == 4) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const auto x = __builtin_amdgcn_permlane32_swap(w[j], w[j + 2], false, false);
            w[j] = x[0];
            w[j + 2] = x[1];
        }
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            const auto x = __builtin_amdgcn_permlane16_swap(w[j], w[j + 1], false, false);
            w[j] = x[0];
            w[j + 1] = x[1];
        }
        n = n0 + 16 * fq;
    } else if constexpr (NY == 2) {
        const auto x = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
        w[0] = x[0];
        w[1] = x[1];
        n = n0 + (fq & 1) * 16 + (fq >> 1) * 8;
    }
    if (m >= a.M) return;
    uint8_t* out = a.codes + m * a.code_stride + n;
    if (n + 4 * NY <= a.N) {
        if constexpr (NY == 4) *(uint4*)out = uint4{w[0], w[1], w[2], w[3]};
        else if constexpr (NY == 2) *(uint2*)out = uint2{w[0], w[1]};
        else *(uint32_t*)out = w[0];
    } else {
#pragma unroll
        for (int e = 0; e < 4 * NY; ++e)
            if (n + e < a.N) out[e] = (uint8_t)(w[e / 4] >> (e % 4 * 8));
    }
}

// ... into codes: 32 lanes have a row's 128 columns from n / 128 * 128 on, and all of them come here.  on: the row is one of y's
__device__ __forceinline__ void store_block4(const MatmulArgs& a, int64_t m, int n, mm_f4 y, bool on) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = n + e < a.N ? y[e] : 0.0f;
    float top = max16(finite_top(v));
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    const float scale = scale_of(top), by = 1.0f / scale;
    if (!on || n >= a.N) return;
    const uint32_t w = codes4(v[0] * by, v[1] * by, v[2] * by, v[3] * by);
    uint8_t* out = a.codes + m * a.code_stride + n;
    if (n + 4 <= a.N) {
        *(uint32_t*)out = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.N) out[e] = (uint8_t)(w >> (8 * e));
    }
    if (n % kBlockCols == 0) a.scales[m * a.scale_stride + n / kBlockCols] = scale;
}

hipError_t launch_block_matmul_few(const MatmulArgs& a, int dtype, int shape, hipStream_t st);
hipError_t launch_block_matmul_bf16(const MatmulArgs& a, int shape, hipStream_t st);
hipError_t launch_block_matmul_bf16_fast(const MatmulArgs& a, int shape, hipStream_t st);
hipError_t launch_block_matmul_f32(const MatmulArgs& a, int shape, hipStream_t st);
hipError_t launch_block_matmul_f32_fast(const MatmulArgs& a, int shape, hipStream_t st);
hipError_t launch_block_matmul_codes(const MatmulArgs& a, int shape, hipStream_t st);
hipError_t launch_block_matmul_codes_fast(const MatmulArgs& a, int shape, hipStream_t st);

}  // namespace hr
