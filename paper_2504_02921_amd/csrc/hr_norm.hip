// The norm of a residual stream with its addition, and codes with scales (hr_rms_norm, hr_block_quantize).
//
// y = s / sqrt(mean(s^2) + eps) * (gain + offset), s = x + add: one pass over a head whose channels stay in registers between the sum of their squares and
// what is made of them, so every input is read and every output written once.  A block of 128 channels has its scale from 16 lanes of a row (four lane
// swaps away), and its codes leave in 8 bytes a lane.  All values and sums are fp32; out and total are rounded once each.
//
// What bounds it is those bytes, if everything is requested before anything is waited for and addresses are scalar: bf16, sums and codes written, 12800 x 4096
// 69 us (5.3 TB/s; a copy of 4 GiB reaches 4.8 read and written), 12800 x 896 15.4 (5.2), 25600 x 32 heads of 128 77 (5.5), fp32 3000 x 4096 39 (5.0); of
// 65 x 896 (3.1 us) the launch and one way to memory and back.  bf16 rows that begin at odd elements: 8000 x 5003 93 us (3.0).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "hr_block8.h"
#include "hr_block8_device.h"
#include "hr_kernels.h"

namespace hr {

namespace {

constexpr int kVec = 8;                      // channels of a lane: 16 lanes have a block of 128
constexpr int kThreads = 256, kWideThreads = 1024;
constexpr int kBlockLanes = kBlockCols / kVec;
constexpr int64_t kMostGroups = 1 << 20;     // workgroups of a launch; more rows are walked

struct NormSide { const void* p; int64_t ts, hs; };
struct NormArgs {
    NormSide x, add, total, out;
    const float* gain;
    uint8_t* codes;
    float* scales;
    int64_t rows, code_stride, scale_stride;
    int32_t heads, channels;
    float eps, offset;
};

template <typename T>
__device__ __forceinline__ T* at(const NormSide& s, int64_t token, int head) { return (T*)s.p + token * s.ts + head * s.hs; }

// Channels c .. c + 7 as they lie there.  WHOLE: the number of channels is a multiple of 8; a lane behind the last one has others then, which must not count,
// else those behind the last one are zeros
template <typename T, bool WHOLE>
__device__ __forceinline__ Loose<T, kVec> load8(const T* p, int c, int channels) {
    if constexpr (WHOLE) return *(const Loose<T, kVec>*)(p + (c < channels ? c : 0));
    Loose<T, kVec> w;
    if (c + kVec <= channels) {
        w = *(const Loose<T, kVec>*)(p + c);
    } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) w.w[e] = c + e < channels ? p[c + e] : (T)0.0f;
    }
    return w;
}
template <typename T>
__device__ __forceinline__ void values8(const Loose<T, kVec>& w, float (&v)[kVec]) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = to_float<T>(w.w[e]);
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void store8(T* p, int c, int channels, const float (&v)[kVec]) {
    if (c + kVec <= channels) {
        Loose<T, kVec> w;
#pragma unroll
        for (int e = 0; e < kVec; ++e) w.w[e] = from_float<T>(v[e]);
        *(Loose<T, kVec>*)(p + c) = w;
    } else if (!WHOLE) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            if (c + e < channels) p[c + e] = from_float<T>(v[e]);
    }
}
// Codes c .. c + 7 of a row; c is a multiple of 8 and rows begin at multiples of 16
template <bool WHOLE>
__device__ __forceinline__ void store_codes8(uint8_t* p, int c, int cols, const float (&v)[kVec], float by) {
    const uint2 w = {codes4(v[0] * by, v[1] * by, v[2] * by, v[3] * by), codes4(v[4] * by, v[5] * by, v[6] * by, v[7] * by)};
    if (c + kVec <= cols) {
        *(uint2*)(p + c) = w;
    } else if (!WHOLE) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            if (c + e < cols) p[c + e] = (uint8_t)((e < 4 ? w.x : w.y) >> (e % 4 * 8));
    }
}

// What becomes of eight channels of a head; 16 lanes in a row come here together for a block of 128
template <typename T, bool WHOLE>
__device__ __forceinline__ void finish8(const NormArgs& a, int64_t token, int head, int c, bool on, const float (&s)[kVec], float up, float r,
                                        const Loose<float, kVec>& gain) {
    if (c / kBlockCols * kBlockCols >= a.channels) return;
    const bool any = c < a.channels;
    float y[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) y[e] = s[e] * up * r;
    if (a.gain) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) y[e] *= gain.w[e] + a.offset;
    }
    if (a.codes) {
        if (!WHOLE && c + kVec > a.channels)
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (c + e >= a.channels) y[e] = 0.0f;             // an infinite 1 / root makes NaN of them
        const float scale = scale_of(max16(any ? finite_top(y) : 0.0f));
        if (on && any) {
            store_codes8<WHOLE>(a.codes + token * a.code_stride, c, a.channels, y, 1.0f / scale);
            if (c % kBlockCols == 0) a.scales[token * a.scale_stride + c / kBlockCols] = scale;
        }
    }
    if (on && any) {
        if (a.total.p) store8<T, WHOLE>(at<T>(a.total, token, head), c, a.channels, s);
        if (a.out.p) store8<T, WHOLE>(at<T>(a.out, token, head), c, a.channels, y);
    }
}

// Squares of values below 1e-19 leave fp32's normal range, where each is off by 2^-150 at most.  Where mean + eps is below 2^-120, of which that is more than
// 2^-30, a head is summed once more, its values times 2^100 (at most 2^48 then, and 2^-49 or more): y = (s 2^100) / root of mean and eps times 2^200.  A branch that
// heads of usual sizes do not take: 12800 x 4096 is as fast without it
constexpr float kSmallMean = 0x1p-120f, kUp = 0x1p100f;
__device__ __forceinline__ float mean_of(float squares, float up, const NormArgs& a) { return squares / (float)a.channels + a.eps * up * up; }
__device__ __forceinline__ float root_of(float mean) { return mean == 0.0f ? 0.0f : rsqrtf(mean); }

// LANES lanes have a head, CHUNKS times 8 channels each
template <typename T, bool WHOLE, int LANES, int CHUNKS>
__global__ void __launch_bounds__(LANES > kThreads ? LANES : kThreads) norm_kernel(NormArgs a) {
    constexpr int UNITS = LANES > kThreads ? 1 : kThreads / LANES, WAVES = LANES / 64;
    __shared__ float part[2][UNITS][LANES > 64 ? WAVES : 1];
    const int lane = threadIdx.x % LANES, unit = threadIdx.x / LANES;
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * UNITS; first < a.rows; first += (int64_t)gridDim.x * UNITS) {
        const bool on = first + unit < a.rows;
        const int64_t row = on ? first + unit : a.rows - 1;
        int64_t token = row;
        int head = 0;
        if (a.heads > 1) {
            token = a.rows <= 0xFFFFFFFFll ? (int64_t)((uint32_t)row / (uint32_t)a.heads) : row / a.heads;
            head = (int)(row - token * a.heads);
        }
        if constexpr (LANES >= 64) {                     // the same in a wavefront's lanes: scalar addresses (tokens are at most 2^30)
            token = __builtin_amdgcn_readfirstlane((int)token);
            head = __builtin_amdgcn_readfirstlane(head);
        }
        // everything is requested before anything is waited for
        Loose<T, kVec> x[CHUNKS], add[CHUNKS];
        Loose<float, kVec> gain[CHUNKS];
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) x[k] = load8<T, WHOLE>(at<const T>(a.x, token, head), (k * LANES + lane) * kVec, a.channels);
        if (a.add.p) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) add[k] = load8<T, WHOLE>(at<const T>(a.add, token, head), (k * LANES + lane) * kVec, a.channels);
        }
        if (CHUNKS == 1 && a.gain) gain[0] = load8<float, WHOLE>(a.gain, lane * kVec, a.channels);
        float s[CHUNKS][kVec];
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) values8<T>(x[k], s[k]);
        if (a.add.p) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                for (int e = 0; e < kVec; ++e) s[k][e] += to_float<T>(add[k].w[e]);
        }
        // mean + eps of the head; low: that of one of the workgroup's heads, where these meet at barriers, is small
        auto mean = [&](auto again, bool& low) {
            constexpr float up = decltype(again)::value ? kUp : 1.0f;
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                float part = 0.0f;
#pragma unroll
                for (int e = 0; e < kVec; ++e) part = fmaf(s[k][e] * up, s[k][e] * up, part);
                sum += !WHOLE || (k * LANES + lane) * kVec < a.channels ? part : 0.0f;
            }
            float m;
            if constexpr (LANES <= 64) {
                if constexpr (LANES == 64) sum = wave_sum(sum);
                else sum = sum16(sum);
                if constexpr (LANES == 32) sum += __shfl_xor(sum, 16, 64);
                m = mean_of(sum, up, a);
                low = m < kSmallMean;
            } else {
                sum = wave_sum(sum);
                if (lane % 64 == 0) part[turn][unit][lane / 64] = sum;
                __syncthreads();                    // one a turn: the other half of `part` is written next
                low = false;
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    sum = 0.0f;
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) sum += part[turn][u][w];
                    const float of = mean_of(sum, up, a);
                    low = low || of < kSmallMean;
                    if (u == unit) m = of;
                }
                turn ^= 1;
            }
            return m;
        };
        float up = 1.0f;
        bool low;
        float m = mean(std::false_type{}, low);
        if (low) {                                  // the same in all lanes that meet in mean()
            bool unused;
            const float more = mean(std::true_type{}, unused);
            if (m < kSmallMean) {
                m = more;
                up = kUp;
            }
        }
        const float r = root_of(m);
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            if (CHUNKS > 1 && a.gain) gain[k] = load8<float, WHOLE>(a.gain, (k * LANES + lane) * kVec, a.channels);
            finish8<T, WHOLE>(a, token, head, (k * LANES + lane) * kVec, on, s[k], up, r, gain[k]);
        }
    }
}

// Heads of more channels than registers are kept for: read once for the sum and once more, mostly from a cache
template <typename T>
__global__ void __launch_bounds__(kWideThreads) norm_wide_kernel(NormArgs a) {
    __shared__ float part[2][kWideThreads / 64];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t token = row / a.heads;
        const int head = (int)(row - token * a.heads);
        auto load = [&](int c, float (&s)[kVec]) {
            values8<T>(load8<T, false>(at<const T>(a.x, token, head), c, a.channels), s);
            if (!a.add.p) return;
            const Loose<T, kVec> add = load8<T, false>(at<const T>(a.add, token, head), c, a.channels);
#pragma unroll
            for (int e = 0; e < kVec; ++e) s[e] += to_float<T>(add.w[e]);
        };
        float s[kVec];
        auto mean = [&](float up) {
            float sum = 0.0f;
            for (int c = threadIdx.x * kVec; c < a.channels; c += kWideThreads * kVec) {
                load(c, s);
#pragma unroll
                for (int e = 0; e < kVec; ++e) sum = fmaf(s[e] * up, s[e] * up, sum);
            }
            sum = wave_sum(sum);
            if (threadIdx.x % 64 == 0) part[turn][threadIdx.x / 64] = sum;
            __syncthreads();
            sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWideThreads / 64; ++w) sum += part[turn][w];
            turn ^= 1;
            return mean_of(sum, up, a);
        };
        float up = 1.0f, m = mean(up);
        if (m < kSmallMean) m = mean(up = kUp);
        const float r = root_of(m);
        const int64_t padded = blocks_of(a.channels) * kBlockCols;        // whole groups of lanes look for a block's largest
        for (int c = threadIdx.x * kVec; c < padded; c += kWideThreads * kVec) {
            load(c, s);
            Loose<float, kVec> gain;
            if (a.gain) gain = load8<float, false>(a.gain, c, a.channels);
            finish8<T, false>(a, token, head, c, true, s, up, r, gain);
        }
    }
}

template <typename T, int LANES, int CHUNKS>
void norm_go(const NormArgs& a, hipStream_t st) {
    constexpr int64_t units = LANES > kThreads ? 1 : kThreads / LANES;
    const unsigned groups = (unsigned)std::min((a.rows + units - 1) / units, kMostGroups);
    if (a.channels % kVec == 0) norm_kernel<T, true, LANES, CHUNKS><<<groups, LANES > kThreads ? LANES : kThreads, 0, st>>>(a);
    else norm_kernel<T, false, LANES, CHUNKS><<<groups, LANES > kThreads ? LANES : kThreads, 0, st>>>(a);
}

template <typename T>
void norm_launch(const NormArgs& a, hipStream_t st) {
    const NormShape s = norm_shape(a.channels, a.rows);
    switch (s.lanes) {
        case 16: norm_go<T, 16, 1>(a, st); break;
        case 32: norm_go<T, 32, 1>(a, st); break;
        case 64: norm_go<T, 64, 1>(a, st); break;
        case 128: norm_go<T, 128, 1>(a, st); break;
        case 256: norm_go<T, 256, 1>(a, st); break;
        case 512: s.chunks == 1 ? norm_go<T, 512, 1>(a, st) : norm_go<T, 512, 2>(a, st); break;
        default:
            if (s.chunks == 1) norm_go<T, 1024, 1>(a, st);
            else if (s.chunks) norm_go<T, 1024, 2>(a, st);
            else norm_wide_kernel<T><<<(unsigned)std::min(a.rows, kMostGroups), kWideThreads, 0, st>>>(a);
    }
}

struct QuantizeArgs {
    const void* x;
    uint8_t* codes;
    float* scales;
    int64_t rows, x_stride, code_stride, scale_stride;
    int32_t cols, blocks;            // blocks of 128 columns
};

// Rows of activations: 16 lanes have 128 columns of a row.  12800 x 4096 bf16: 32 us (4.9 TB/s)
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(QuantizeArgs a) {
    constexpr int UNITS = kThreads / kBlockLanes;
    const int64_t n = a.rows * a.blocks;
    for (int64_t first = (int64_t)blockIdx.x * UNITS; first < n; first += (int64_t)gridDim.x * UNITS) {
        const int64_t u = first + threadIdx.x / kBlockLanes;
        const bool on = u < n;
        const int64_t row = n <= 0xFFFFFFFFll ? (int64_t)((uint32_t)(on ? u : 0) / (uint32_t)a.blocks) : (on ? u : 0) / a.blocks;
        const int b = (int)((on ? u : 0) - row * a.blocks), c = b * kBlockCols + threadIdx.x % kBlockLanes * kVec;
        float v[kVec];
        values8<T>(load8<T, WHOLE>((const T*)a.x + row * a.x_stride, c, a.cols), v);
        const float scale = scale_of(max16(!WHOLE || c < a.cols ? finite_top(v) : 0.0f));
        if (on && c < a.cols) {
            store_codes8<WHOLE>(a.codes + row * a.code_stride, c, a.cols, v, 1.0f / scale);
            if (c % kBlockCols == 0) a.scales[row * a.scale_stride + b] = scale;
        }
    }
}

// Weights: a workgroup has a tile of 128 x 128, its lanes 8 columns of every 16th row, all eight of them under way at once and kept in registers until the
// tile's largest is known.  28672 x 4096 bf16: 63 us (5.6 TB/s)
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kThreads) quantize_tiles_kernel(QuantizeArgs a) {
    constexpr int STEP = kThreads / kBlockLanes, PASSES = kBlockCols / STEP;
    __shared__ float tops[kThreads / 64];
    const int64_t tile_row = blockIdx.x / a.blocks, b = blockIdx.x % a.blocks;
    const int c = (int)b * kBlockCols + threadIdx.x % kBlockLanes * kVec;
    const int64_t row0 = tile_row * kBlockCols + threadIdx.x / kBlockLanes;
    Loose<T, kVec> x[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) x[p] = load8<T, WHOLE>((const T*)a.x + min(row0 + p * STEP, a.rows - 1) * a.x_stride, c, a.cols);
    float v[PASSES][kVec], top = 0.0f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        values8<T>(x[p], v[p]);
        top = fmaxf(top, finite_top(v[p]));
    }
    top = wave_max(!WHOLE || c < a.cols ? top : 0.0f);
    if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) top = fmaxf(top, tops[w]);
    const float scale = scale_of(top), by = 1.0f / scale;
    if (c >= a.cols) return;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int64_t row = row0 + p * STEP;
        if (row < a.rows) store_codes8<WHOLE>(a.codes + row * a.code_stride, c, a.cols, v[p], by);
    }
    if (threadIdx.x == 0) a.scales[tile_row * a.scale_stride + b] = scale;
}

template <typename T>
void quantize_launch(const QuantizeArgs& a, int block_rows, hipStream_t st) {
    constexpr int64_t units = kThreads / kBlockLanes;
    const unsigned groups = (unsigned)(block_rows == 1 ? std::min((a.rows * a.blocks + units - 1) / units, kMostGroups) : blocks_of(a.rows) * a.blocks);
    const auto kernel = block_rows == 1 ? (a.cols % kVec == 0 ? quantize_rows_kernel<T, true> : quantize_rows_kernel<T, false>)
                                        : (a.cols % kVec == 0 ? quantize_tiles_kernel<T, true> : quantize_tiles_kernel<T, false>);
    kernel<<<groups, kThreads, 0, st>>>(a);
}

}  // namespace

hipError_t launch_rms_norm(const hr_norm_args& n, hipStream_t st) {
    NormArgs a{};
    a.x = NormSide{n.x, n.x_token_stride, n.x_head_stride};
    a.add = NormSide{n.add, n.add_token_stride, n.add_head_stride};
    a.total = NormSide{n.total, n.total_token_stride, n.total_head_stride};
    a.out = NormSide{n.out, n.out_token_stride, n.out_head_stride};
    a.gain = n.gain;
    if (n.block8) {
        a.codes = (uint8_t*)n.block8->codes;
        a.scales = n.block8->scales;
        a.code_stride = n.block8->row_stride;
        a.scale_stride = n.block8->scale_stride;
    }
    a.rows = n.tokens * n.heads;
    a.heads = n.heads;
    a.channels = n.channels;
    a.eps = n.eps;
    a.offset = n.gain_offset;
    if (n.dtype == HR_F32) norm_launch<float>(a, st);
    else norm_launch<bf16_t>(a, st);
    return hipGetLastError();
}

hipError_t launch_block_quantize(int dtype, const void* x, int64_t x_stride, const hr_block8& out, hipStream_t st) {
    QuantizeArgs a{x, (uint8_t*)out.codes, out.scales, out.rows, x_stride, out.row_stride, out.scale_stride, out.cols, (int32_t)blocks_of(out.cols)};
    if (dtype == HR_F32) quantize_launch<float>(a, out.block_rows, st);
    else quantize_launch<bf16_t>(a, out.block_rows, st);
    return hipGetLastError();
}

}  // namespace hr
