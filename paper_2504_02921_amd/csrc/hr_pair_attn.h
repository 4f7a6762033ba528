// Device pieces that the kernels of hr_pair_attention share: their parameters, a block's rows and what they see, scores, softmax.
//
// A block is 32 rows of a group (the pairs of one document): (token in order, query head of the kv head's group of heads), heads fastest, so that
// the rows of several short queries share a block.  Scores are computed transposed, S^T = K Q^T, in sub-tiles of 32 keys: lane l
// of a wavefront owns row l & 31 and the keys 8 (r >> 2) + 4 (l >> 5) + (r & 3), r < 16, of a sub-tile; P is then in operand order for
// O^T += V^T P^T, of which the lane holds channels 8 (r >> 2) + 4 (l >> 5) + (r & 3) of every 32.
// What a row sees is two intervals: document keys [dlo, D) and, numbered by their place in order, own keys [olo, ohi).  So a mask is two
// comparisons, and a sub-tile that all rows see whole needs none.
#pragma once

#include <hip/hip_runtime.h>

#include "hr_attn_common.h"
#include "hr_device_types.h"
#include "hr_pair.h"

namespace hr {

typedef const __attribute__((address_space(4))) int32_t* const_int_t;       // read through the scalar cache: uniform, written by an earlier launch
typedef const __attribute__((address_space(4))) float* const_float_t;

struct PairAttnArgs {
    // what finds a workgroup's rows comes first: those words are in scalar registers when a wavefront starts
    const int32_t* hdr;
    const int4 *rec, *rec_tiles;      // records of the work list, two int4 each: blocks, tiles
    const int4* ord;
    const int32_t* page_table;
    int32_t pt_stride, n_kv, g, most_splits;
    int32_t num_pages, d, window, own_keys;
    int32_t n_pairs, max_tokens, chunk;
    int64_t cap_blk, cap_tile;        // records of the work list
    const int32_t *q_cu, *prefix;
    const char* pool;                 // page 0 of the layer
    const float* scales;              // fp8: of page 0 of the layer
    const void *q, *k, *v;
    void* out;
    float* lse;
    const float* slopes;
    int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;
    float scale_log2;                 // scale times log2 e: scores are in log2 units
    float cap_log2, cap_in;           // cap: s = cap_log2 tanh(s), where s is the scaled score times cap_in; 0: none
    float* part_o;                    // pieces: [piece][token row][query head][d], unscaled
    float2* part_ml;                  // ... and maximum and sum
    int64_t part_rows;                // rows of a piece
    int32_t blocks_only;              // work items are blocks (kernels that know no tiles)
};

// What scores need before they are compared, a kernel's form for each: a positive factor alone, or also a cap, a bias or a factor below 0.  The quotient
// of a cap is off by 2^-23 of it, whatever the score: with wide caps, from kWideCap on, small arguments take the series of tanh, and in the
// fp32 kernels (EXACT) under any cap.  Below kWideCap the quotient leaves 2^-17 in a score, a 64th of what the weight loses in half.
// Quotient alone / with the series: 200 documents of 2048 x 64 tokens, 128 channels 742 / 793 us, 640 of 512 x 32, 64 channels 104 / 108
enum PairScores { PS_FACTOR = 0, PS_EXTRA = 1, PS_WIDE_CAP = 2, PS_EXACT = 3 };
constexpr float kWideCap = 64.0f;
constexpr float kLn2 = 0.69314718055994531f, kLog2e = 1.4426950408889634f;

inline PairScores pair_scores_of(const PairAttnArgs& a) {
    if (a.cap_log2 >= kWideCap * kLog2e) return PS_WIDE_CAP;
    return a.cap_in != 0.0f || a.slopes || a.scale_log2 < 0.0f ? PS_EXTRA : PS_FACTOR;
}

__device__ __forceinline__ int rows_min(int v) {          // over the 32 rows of a wavefront
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int rows_max(int v) { return -rows_min(-v); }

// Consecutive workgroups go to the 8 XCDs in turn: of every 8 << c items XCD x takes 1 << c that follow each other, so that the kv heads and
// the neighbouring tiles of a group, which share pages, meet in one L2.  (Eighths of all items would take a look at their number first.)
// chunk = c; 0 where keys are cut into pieces: few items, that are to be spread.
__device__ __forceinline__ int item_of(int wg, int chunk) {
    return (wg >> (3 + chunk) << (3 + chunk)) + ((wg & 7) << chunk) + (wg >> 3 & ((1 << chunk) - 1));
}

__device__ __forceinline__ int list_items(const PairAttnArgs& a, bool tiles) {
    const const_int_t hdr = (const_int_t)a.hdr;
    return (int)min((int64_t)max(hdr[tiles ? SH_TILES : SH_BLOCKS], 0), tiles ? a.cap_tile : a.cap_blk) * a.n_kv;
}
__device__ __forceinline__ PairItem list_item(const PairAttnArgs& a, bool tiles, int at) {
    const const_int_t r = (const_int_t)((tiles ? a.rec_tiles : a.rec) + 2 * min((int64_t)at, (tiles ? a.cap_tile : a.cap_blk) - 1));
    return pair_item(r[0], r[1], r[2], r[3], r[4], a.n_pairs, a.max_tokens, a.pt_stride, a.g);
}

// A lane's row
struct PairRow {
    int token, head;                  // row of q, query head within the kv head's group
    int place, start;                 // of its token and of its pair's first token, in order
    int pos;                          // D + index within the query
    int dlo, olo, ohi;                // see above
    bool on;                          // the row exists (the others repeat the last one)
    float slope;                      // slopes[a] log2 e, or 0
};

__device__ __forceinline__ PairRow pair_row(const PairAttnArgs& a, int h, const PairItem& it, int row) {
    PairRow r;
    r.on = row < it.rows;
    const PairPlace at = pair_place(it, row, a.g, a.max_tokens);
    r.head = at.head;
    r.place = at.place;
    const int4 o = a.ord[r.place];    // token row, start, pair, D
    r.token = min(max(o.x, 0), a.max_tokens - 1);
    r.start = min(max(o.y, 0), r.place);
    const int i = r.place - r.start, pair = min(max(o.z, 0), a.n_pairs - 1);
    r.pos = it.D + i;
    const int first = a.window > 0 ? r.pos - a.window + 1 : 0;      // the first position the row sees
    r.dlo = min(max(first, 0), it.D);
    int all = 0;
    if (a.prefix) all = pair_prefix(a.prefix[pair], a.q_cu[pair], a.q_cu[pair + 1], a.max_tokens);
    r.olo = r.start + min(max(first - it.D, 0), i);
    r.ohi = min(r.start + max(i + 1, all), a.max_tokens);
    r.slope = a.slopes ? a.slopes[h * a.g + r.head] * kLog2e : 0.0f;
    return r;
}
// A lane's own key: its place's token row
__device__ __forceinline__ int64_t own_token(const PairAttnArgs& a, int place) { return min(max(a.ord[place].x, 0), a.max_tokens - 1); }

// The scaled scores of a sub-tile in log2 units: cap, then distance.  first: position (document) or place (own) of its first key as seen from
// the row, i.e. minus the row's own
template <int FORM>
__device__ __forceinline__ void pair_scores(floatx16& s, const PairAttnArgs& a, const PairRow& row, int first, int hh) {
    if (a.cap_in != 0.0f) {
        // tanh x = 1 - 2 / (e^2x + 1); 2 log2 e is in cap_in
        auto quotient = [&](float y) { return fmaf(-2.0f * a.cap_log2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y) + 1.0f), a.cap_log2); };
        constexpr float h = 0.5f * kLn2;                                // x = h y
        if (FORM == PS_EXACT) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                // x - x^3 / 3 + 2 x^5 / 15 - ..: behind the seventh of these terms 10^-8 of the value is left at 1/2
                const float x = s[r] * a.cap_in * h, u = x * x;
                float t = fmaf(u, 1.4558344e-3f, -3.5921280e-3f);
                t = fmaf(u, t, 8.8632355e-3f);
                t = fmaf(u, t, -2.1869489e-2f);
                t = fmaf(u, t, 5.3968254e-2f);
                t = fmaf(u, t, -1.3333333e-1f);
                t = fmaf(u, t, 3.3333333e-1f);
                s[r] = fabsf(x) < 0.5f ? a.cap_log2 * fmaf(-x * u, t, x) : quotient(s[r] * a.cap_in);
            }
        } else if (FORM == PS_WIDE_CAP) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                // cap and its reciprocal make one: s (1 - x^2 / 3 + 2 x^4 / 15), of which 2^-22 is left at 1/8; the quotient is 2^-20 of its value off there
                const float y = s[r] * a.cap_in, u = y * y, t = fmaf(u, fmaf(u, 2.0f * h * h * h * h / 15.0f, -h * h / 3.0f), 1.0f);
                s[r] = fabsf(y) < 0.125f / h ? s[r] * t : quotient(y);
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = quotient(s[r] * a.cap_in);
        }
    }
    if (a.slopes) {
        const float f = (float)(first + 4 * hh);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = fmaf(-row.slope, fabsf(f + (float)(8 * (r >> 2) + (r & 3))), s[r]);
    }
}

// Running softmax of a row over its keys (both lanes of the row hold the same)
struct PairSoftmax {
    float m = -INFINITY, l = 0.0f;    // maximum (log2 units), this lane's share of the sum

    // takes in the row's largest new score; the factor on what has been summed so far.  The maximum follows only scores that exceed it by
    // kLazyMax: see hr_attn_mfma.hip
    __device__ __forceinline__ float follow(float mx) {
        const float cand = fmaxf(m, mx);
        if (!(cand > m + kLazyMax)) return 1.0f;
        const float alpha = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - cand);
        m = cand;
        return alpha;
    }
    __device__ __forceinline__ float used() const { return m == -INFINITY ? 0.0f : m; }      // a row that has seen nothing keeps p = 0
};

// s -> probabilities against the running maximum; the factor on what has been summed so far
__device__ __forceinline__ float pair_softmax(PairSoftmax& sm, floatx16& s) {
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
    const float alpha = sm.follow(row_max2(mx)), use = sm.used();
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s[r] = __builtin_amdgcn_exp2f(s[r] - use);
        sum += s[r];
    }
    sm.l = fmaf(sm.l, alpha, sum);
    return alpha;
}

// A row's log-sum: nothing seen is -infinity, a score that is NaN (which no maximum takes in) leaves NaN in the sum
__device__ __forceinline__ float pair_lse(float m, float sum) { return sum == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * kLn2; }

// Joins a row's pieces: what the results of one with maximum m count for under the common maximum
__device__ __forceinline__ float piece_factor(float m, float all) { return m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - all); }

// Joins what the NW wavefronts of a workgroup have of a block's rows, in the wavefronts' order, and writes the rows (or, of a call cut into
// pieces, the piece's).  HD: channels that the accumulators hold, a.d or more.  smem: pair_join_bytes.
constexpr size_t pair_join_bytes(int nw, int hd) {
    return (size_t)nw * 32 * (hd + 4) * sizeof(float) + (size_t)nw * 32 * 2 * sizeof(float) + 32 * sizeof(int2);
}
template <int NW, int HD, typename QT>
__device__ __forceinline__ void pair_join_waves(const PairAttnArgs& a, float* smem, const floatx16 (&o)[HD / 32], const PairSoftmax& sm,
                                                const PairRow& row, int h, int pieces) {
    constexpr int LD = HD + 4;
    const int lane = threadIdx.x & 63, ln = lane & 31, hh = lane >> 5, wave = threadIdx.x >> 6, d = a.d;
    float* ml = smem + NW * 32 * LD;                                // [wave][row][maximum, sum]
    const float l = row_sum2(sm.l);
    if (hh == 0) {
        ml[(wave * 32 + ln) * 2] = sm.m;
        ml[(wave * 32 + ln) * 2 + 1] = l;
    }
#pragma unroll
    for (int mb = 0; mb < HD / 32; ++mb)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *(float4*)(smem + (wave * 32 + ln) * LD + mb * 32 + 8 * (r >> 2) + 4 * hh) = make_float4(o[mb][r], o[mb][r + 1], o[mb][r + 2], o[mb][r + 3]);
    // where the rows go
    int2* where = (int2*)(ml + NW * 32 * 2);
    if (wave == 0 && hh == 0) where[ln] = make_int2(row.on ? row.token : -1, row.head);
    __syncthreads();
    const int piece = d / 4;
    for (int u = threadIdx.x; u < 32 * piece; u += NW * 64) {
        const int rw = u / piece, c = (u - rw * piece) * 4;
        const int2 to = where[rw];
        if (to.x < 0) continue;
        float m = -INFINITY, sum = 0.0f, f[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w) m = fmaxf(m, ml[(w * 32 + rw) * 2]);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            f[w] = piece_factor(ml[(w * 32 + rw) * 2], m);
            sum = fmaf(f[w], ml[(w * 32 + rw) * 2 + 1], sum);
            const float4 x = *(const float4*)(smem + (w * 32 + rw) * LD + c);
            if (f[w] == 0.0f) continue;                                 // nothing seen there
            acc.x = fmaf(f[w], x.x, acc.x);
            acc.y = fmaf(f[w], x.y, acc.y);
            acc.z = fmaf(f[w], x.z, acc.z);
            acc.w = fmaf(f[w], x.w, acc.w);
        }
        const int head = h * a.g + to.y;
        if (pieces > 1) {
            const int64_t at = (int64_t)blockIdx.y * a.part_rows + (int64_t)to.x * a.g * a.n_kv + head;
            if (c == 0) a.part_ml[at] = make_float2(m, sum);
            if (m != -INFINITY) *(float4*)(a.part_o + at * d + c) = acc;
            continue;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        QT* out = (QT*)a.out + to.x * a.o_ts + head * a.o_hs + c;
        using W = Loose<QT, 4>;
        W y;
        y.w[0] = from_float<QT>(acc.x * inv);
        y.w[1] = from_float<QT>(acc.y * inv);
        y.w[2] = from_float<QT>(acc.z * inv);
        y.w[3] = from_float<QT>(acc.w * inv);
        *(W*)out = y;
        if (c == 0 && a.lse) a.lse[(int64_t)to.x * a.g * a.n_kv + head] = pair_lse(m, sum);
    }
}


}  // namespace hr
