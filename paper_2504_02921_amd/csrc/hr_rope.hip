// Rotary positions of q and k of a batch of tokens (hr_rope_apply): one launch, every channel read and written once.
//
// Pair i of a token at position p is turned by p f_i.  The angle is taken in quarter turns in fp64 (p f_i reaches 10^6 turns, of which
// fp32 would keep nothing), reduced to [-1/2, 1/2] of a quarter, and only that remainder is fp32; sine and cosine are their series there.
// A lane keeps one chunk of pairs of one token and walks the heads, so a chunk's angles are computed once for all of its heads.  What bounds it is
// the copy: 12800 tokens of 40 heads of 128 channels in bf16, 262 MB, take 59 us, 4.5 TB/s (a plain copy of 4 GiB makes 4.8); 16800 rows of 4 heads
// in fp32, 34 MB, 10 us, 3.5 TB/s; 65 tokens the 4 us of a launch that waits for its loads once.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "hr_device_types.h"
#include "hr_kernels.h"
#include "hr_pair.h"

namespace hr {

namespace {

constexpr int kHeadsAhead = 4;      // heads whose loads are in flight together

struct RopeSide {
    const void* in;
    void* out;
    int64_t in_ts, in_hs, out_ts, out_hs;
};
struct RopeArgs {
    const int32_t* positions;
    int64_t n_tokens;
    int32_t first, period;
    int32_t rot_chunks, chunks, heads, tokens;      // RopeShape; rot_chunks: of the rotated channels
    int32_t n_heads[2];                             // heads of the first tensor, of both
    int32_t rotary, head_dim;
    float amplitude, sign;
    RopeSide side[2];
    double quarters[kMaxRotaryPairs];               // quarter turns per position
};

// sine and cosine of pi/2 x for |x| <= 1/2: their series, whose next terms are below 2^-29 there
__device__ __forceinline__ void sincos_quarter(float x, float& s, float& c) {
    const float t = x * 1.57079632679489662f, u = t * t;
    s = fmaf(t * u, fmaf(u, fmaf(u, fmaf(u, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), t);
    c = fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
}

template <typename T, bool INTERLEAVED, int VEC>
__global__ void __launch_bounds__(kRopeWaves * 64) rope_apply_kernel(RopeArgs a) {
    constexpr int W = INTERLEAVED ? 2 * VEC : VEC;               // channels of one load
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)blockIdx.x * kRopeWaves + (threadIdx.x >> 6);
    // lane -> (token, head, chunk); heads with more than 64 chunks are walked 64 at a time
    const int wide = min(a.chunks, 64);
    const int unit = lane / wide, chunk0 = lane - unit * wide;
    const int tok = unit / a.heads, head0 = unit - tok * a.heads;
    const int64_t t = wave * a.tokens + tok;
    if (tok >= a.tokens || t >= a.n_tokens) return;
    const int pos = a.positions ? a.positions[t] : a.first + (int)(a.period > 0 ? t % a.period : t);
    if (pos < 0) return;
    using V = Loose<T, W>;
    for (int chunk = chunk0; chunk < a.chunks; chunk += 64) {
        const bool turned = chunk < a.rot_chunks;
        const RopeChunk own = rope_chunk(chunk, a.rot_chunks, VEC, INTERLEAVED ? HR_ROPE_INTERLEAVED : HR_ROPE_HALF, a.rotary, a.head_dim);
        const int at = own.at;
        const bool alone = INTERLEAVED && VEC == 1 && own.n == 1;      // other widths divide what they copy (rope_shape)
        float cs[VEC], sn[VEC];
        if (turned) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const double turns = (double)pos * a.quarters[chunk * VEC + e] * 0.25;
                const double x = (turns - floor(turns)) * 4.0, q = rint(x);
                float s, c;
                sincos_quarter((float)(x - q), s, c);
                const int quad = (int)q & 3;
                const float s2 = quad & 1 ? c : s, c2 = quad & 1 ? s : c;
                sn[e] = (quad & 2 ? -s2 : s2) * a.sign * a.amplitude;
                cs[e] = ((quad + 1) & 2 ? -c2 : c2) * a.amplitude;
            }
        }
        for (int h0 = head0; h0 < a.n_heads[1]; h0 += kHeadsAhead * a.heads) {
            V x1[kHeadsAhead], x2[kHeadsAhead];
#pragma unroll
            for (int u = 0; u < kHeadsAhead; ++u) {
                const int h = h0 + u * a.heads;
                if (h >= a.n_heads[1]) break;
                const RopeSide& d = a.side[h >= a.n_heads[0]];
                const T* p = (const T*)d.in + t * d.in_ts + (h >= a.n_heads[0] ? h - a.n_heads[0] : h) * d.in_hs + at;
                if (alone) x1[u].w[0] = *p;
                else x1[u] = *(const V*)p;
                if (!INTERLEAVED && turned) x2[u] = *(const V*)(p + a.rotary / 2);
            }
#pragma unroll
            for (int u = 0; u < kHeadsAhead; ++u) {
                const int h = h0 + u * a.heads;
                if (h >= a.n_heads[1]) break;
                const RopeSide& d = a.side[h >= a.n_heads[0]];
                T* p = (T*)d.out + t * d.out_ts + (h >= a.n_heads[0] ? h - a.n_heads[0] : h) * d.out_hs + at;
                if (turned) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        if constexpr (INTERLEAVED) {
                            const float lo = to_float<T>(x1[u].w[2 * e]), hi = to_float<T>(x1[u].w[2 * e + 1]);
                            x1[u].w[2 * e] = from_float<T>(rope_lo(lo, hi, cs[e], sn[e]));
                            x1[u].w[2 * e + 1] = from_float<T>(rope_hi(lo, hi, cs[e], sn[e]));
                        } else {
                            const float lo = to_float<T>(x1[u].w[e]), hi = to_float<T>(x2[u].w[e]);
                            x1[u].w[e] = from_float<T>(rope_lo(lo, hi, cs[e], sn[e]));
                            x2[u].w[e] = from_float<T>(rope_hi(lo, hi, cs[e], sn[e]));
                        }
                    }
                    if (!INTERLEAVED) *(V*)(p + a.rotary / 2) = x2[u];
                }
                if (alone) *p = x1[u].w[0];
                else *(V*)p = x1[u];
            }
        }
    }
}

template <typename T, bool INTERLEAVED>
void rope_launch(int vec, unsigned blocks, const RopeArgs& a, hipStream_t st) {
    constexpr int most = 16 / (int)sizeof(T) / (INTERLEAVED ? 2 : 1);
    switch (vec) {
        case 8: if constexpr (most >= 8) { rope_apply_kernel<T, INTERLEAVED, 8><<<blocks, kRopeWaves * 64, 0, st>>>(a); } break;
        case 4: if constexpr (most >= 4) { rope_apply_kernel<T, INTERLEAVED, 4><<<blocks, kRopeWaves * 64, 0, st>>>(a); } break;
        case 2: rope_apply_kernel<T, INTERLEAVED, 2><<<blocks, kRopeWaves * 64, 0, st>>>(a); break;
        default: rope_apply_kernel<T, INTERLEAVED, 1><<<blocks, kRopeWaves * 64, 0, st>>>(a);
    }
}

}  // namespace

hipError_t launch_rope_apply(const hr_rope_cfg& c, const double* freqs, int dtype, int64_t n_tokens, const int32_t* positions, int32_t first,
                             int32_t period, const hr_rope_tensor* tensors, int32_t n_tensors, bool inverse, hipStream_t st) {
    RopeArgs a{};
    bool in_place = true;
    for (int i = 0; i < n_tensors; ++i) {
        a.side[i] = RopeSide{tensors[i].in, tensors[i].out, tensors[i].in_token_stride, tensors[i].in_head_stride, tensors[i].out_token_stride,
                             tensors[i].out_head_stride};
        in_place = in_place && tensors[i].in == tensors[i].out;
    }
    a.n_heads[0] = tensors[0].n_heads;
    a.n_heads[1] = a.n_heads[0] + (n_tensors > 1 ? tensors[1].n_heads : 0);
    const RopeShape s = rope_shape(c.head_dim, c.rotary_dim, c.layout, (int)dtype_size(dtype), in_place, a.n_heads[1]);
    a.positions = positions;
    a.n_tokens = n_tokens;
    a.first = first;
    a.period = period;
    a.rot_chunks = c.rotary_dim / 2 / s.vec;
    a.chunks = s.chunks;
    a.heads = s.heads;
    a.tokens = s.tokens;
    a.rotary = c.rotary_dim;
    a.head_dim = c.head_dim;
    a.amplitude = c.amplitude;
    a.sign = inverse ? -1.0f : 1.0f;
    for (int i = 0; i < c.rotary_dim / 2; ++i) a.quarters[i] = freqs[i] * 0.63661977236758134308;      // 2 / pi
    const unsigned blocks = (unsigned)((n_tokens + (int64_t)s.tokens * kRopeWaves - 1) / ((int64_t)s.tokens * kRopeWaves));
    if (dtype == HR_F32) {
        if (c.layout == HR_ROPE_INTERLEAVED) rope_launch<float, true>(s.vec, blocks, a, st);
        else rope_launch<float, false>(s.vec, blocks, a, st);
    } else {
        if (c.layout == HR_ROPE_INTERLEAVED) rope_launch<bf16_t, true>(s.vec, blocks, a, st);
        else rope_launch<bf16_t, false>(s.vec, blocks, a, st);
    }
    return hipGetLastError();
}

}  // namespace hr
