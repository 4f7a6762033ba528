// Device pieces that the half-precision kernels of hr_pair_attention share.
#pragma once

#include "hr_pair_attn.h"

namespace hr {

template <int HD, bool FP8>
struct PairGeo {
    static constexpr int KC = HD / 16, MB = HD / 32;
    static constexpr int ESZ = FP8 ? 1 : 2;
    static constexpr int BLOCK = kPageTokens * HD * ESZ;      // bytes of a K or V block
    using Piece = std::conditional_t<FP8, uint2, halfx8>;     // 8 elements of a page
};

// 8 consecutive E4M3 codes as halves of 2^-8 of their values, exactly (fp8x8_to_half without its factor): a code in the upper byte of a half,
// shifted down by one with its sign kept, has exponent and mantissa in a half's fields, and between them and the sign a copy of the sign to clear.
// K's factor goes into the scores' scale.  Three instructions for two codes: tiles of fp8 pools are bound by what is issued.
__device__ __forceinline__ halfx8 fp8x8_low(uint2 w) {
    typedef __attribute__((ext_vector_type(2))) short shortx2;
    auto pair = [&](unsigned x, unsigned sel) {
        return __builtin_bit_cast(unsigned, __builtin_bit_cast(shortx2, __builtin_amdgcn_perm(x, 0u, sel)) >> 1) & 0xBFFFBFFFu;
    };
    const uint4 r = make_uint4(pair(w.x, 0x050c040cu), pair(w.x, 0x070c060cu), pair(w.y, 0x050c040cu), pair(w.y, 0x070c060cu));
    return __builtin_bit_cast(halfx8, r);
}
// ... times a power of two and 2^8 (fp8_expand_factor)
__device__ __forceinline__ halfx8 fp8x8_times(uint2 w, halfx2 f) {
    return fp8x8_low(w) * __builtin_shufflevector(f, f, 0, 1, 0, 1, 0, 1, 0, 1);
}
constexpr float kFp8Low = 256.0f;      // what fp8x8_low leaves for the scores

__device__ __forceinline__ halfx8 to_half8(VecN<bf16_t, 8> x) {
    halfx8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (half_t)(float)x[e];         // beyond the half range: infinity
    return r;
}
__device__ __forceinline__ halfx8 bf16x8_to_half(const bf16_t* p) { return to_half8(((const Loose<bf16_t, 8>*)p)->w); }

// the lane's 16 probabilities as the B operands of two products over 16 keys each, rounded to half: 2^-11 of a weight (nothing of one below 2^-25, the
// largest being 1 or more), an eighth of what an output loses in bf16; as fp32 the product would run at the seventh part of the rate.  Their sum is that
// of the unrounded ones
__device__ __forceinline__ void pack_p(const floatx16& s, halfx8 (&pf)[2], float f0, float f1) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const halfx2 x = __builtin_convertvector(floatx2{s[e] * f0, s[e + 1] * f0}, halfx2);
        const halfx2 y = __builtin_convertvector(floatx2{s[8 + e] * f1, s[9 + e] * f1}, halfx2);
        pf[0][e] = x[0]; pf[0][e + 1] = x[1];
        pf[1][e] = y[0]; pf[1][e + 1] = y[1];
    }
}

// Hides the keys of a sub-tile outside [lo, hi), relative to the lane's first
__device__ __forceinline__ void hide_keys(floatx16& s, int lo, int hi) {
    const unsigned n = (unsigned)max(hi - lo, 0);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = (unsigned)(8 * (r >> 2) + (r & 3) - lo) < n ? s[r] : -INFINITY;
}

// O^T += V^T P^T over a sub-tile that not every row sees whole.  A hidden key's V counts for nothing, whatever it holds, and 0 times infinity is
// not nothing: where a value is not finite (rarely: 0 times all of them is summed, and is NaN then) the product has zeros for those, and they are added
// value by value to the rows that see them, [lo, hi) of the first `exist` keys.  frag(mb, e): the lane's V operand; value(key, ch): one value.
template <int MB, typename Frag, typename Value>
__device__ __forceinline__ void add_pv_masked(floatx16 (&o)[MB], const halfx8 (&pf)[2], int lo, int hi, int exist, int hh, Frag frag, Value value) {
    halfx2 none[4] = {};
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const halfx8 v = frag(mb, e);
#pragma unroll
            for (int i = 0; i < 4; ++i) none[i] = __builtin_elementwise_fma(halfx2{v[2 * i], v[2 * i + 1]}, halfx2{}, none[i]);
        }
    const halfx2 odd = (none[0] + none[1]) + (none[2] + none[3]);
    const bool fix = __any(odd[0] != odd[0] || odd[1] != odd[1]);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            halfx8 v = frag(mb, e);
            if (fix) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __builtin_fabsf16(v[i]) < (half_t)INFINITY ? v[i] : (half_t)0.0f;
            }
            o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pf[e], o[mb], 0, 0, 0);
        }
    if (!fix) return;
#pragma unroll 1
    for (int key = 0; key < exist; ++key) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float v = (float)value(key, mb * 32 + 8 * (r >> 2) + 4 * hh + (r & 3));
                o[mb][r] += key >= lo && key < hi && !(fabsf(v) < INFINITY) ? v : 0.0f;
            }
    }
}

}  // namespace hr
