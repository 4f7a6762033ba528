// Host part of the operators of a layer's projections in 8 bits: argument checks and the choice of launches.  No HIP calls here, so every refusal can
// be exercised on a machine without a GPU.
#include <algorithm>
#include <cmath>

#include "hr_block8.h"

namespace hr {

namespace {

constexpr int64_t kMaxRows = 1 << 30, kMaxStride = (int64_t)1 << 60;
constexpr int32_t kMaxCols = 1 << 22, kMaxScaleStride = 1 << 20, kMaxChannels = 65536, kMaxHeads = 65536;

bool aligned(const void* p, uintptr_t to) { return (uintptr_t)p % to == 0; }

// [tokens][heads][channels] whose offsets fit 62 bits; negative strides are not meant
bool strides_fit(int64_t tokens, int64_t heads, int64_t token_stride, int64_t head_stride) {
    if (heads > 1 && (head_stride < 0 || head_stride > kMaxStride / heads)) return false;
    return tokens <= 1 || (token_stride >= 0 && token_stride <= kMaxStride / tokens);
}

// ... and whose heads share no element: those of one index lie inside a step of the other
bool rows_apart(int64_t tokens, int64_t heads, int64_t token_stride, int64_t head_stride, int64_t channels) {
    if ((tokens > 1 && token_stride < channels) || (heads > 1 && head_stride < channels)) return false;
    if (tokens <= 1 || heads <= 1) return true;
    return token_stride >= (heads - 1) * head_stride + channels || head_stride >= (tokens - 1) * token_stride + channels;
}

bool same_strides(const hr_norm_args& a, int64_t t0, int64_t h0, int64_t t1, int64_t h1) {
    return (a.tokens <= 1 || t0 == t1) && (a.heads <= 1 || h0 == h1);
}

}  // namespace

int block8_check(const hr_block8* b, int block_rows) {
    if (!b || b->block_rows != block_rows || b->rows < 0 || b->cols < 1) return HR_ERR_INVALID_ARG;
    if (b->rows > kMaxRows || b->cols > kMaxCols) return HR_ERR_LEN_RANGE;
    if (b->row_stride % 16 != 0 || b->row_stride < b->cols || b->row_stride > kMaxCols) return HR_ERR_INVALID_ARG;
    if (b->scale_stride < blocks_of(b->cols) || b->scale_stride > kMaxScaleStride) return HR_ERR_INVALID_ARG;
    if (b->rows == 0) return HR_OK;
    if (!b->codes || !b->scales || !aligned(b->codes, 16) || !aligned(b->scales, 4)) return HR_ERR_INVALID_ARG;
    return HR_OK;
}

// Lanes of a head and, for each, chunks of 8 channels (0: as many as there are, read twice).  One chunk wherever a workgroup of 512 has the lanes (bf16, sums
// and codes: 8000 x 4096 by 512 lanes 45 us, by 256 lanes of two chunks 46, by 1024 74; 4 rows 3.2, 3.5, 3.4).  Of 1024 lanes only two workgroups fit a compute
// unit, so rows that fill the chip take 512 lanes of two chunks (8000 x 8192 84 us for 110, fp32 65 x 5003 5.0 for 4.4), and 1024 of two where that is needed
// (8000 x 14336 149 us, by 512 lanes of four chunks 149, fp32 286 and 304).
NormShape norm_shape(int channels, int64_t rows) {
    for (int lanes : {16, 32, 64, 128, 256, 512})
        if (channels <= lanes * 8) return {lanes, 1};
    if (channels <= 8192) return rows < 256 ? NormShape{1024, 1} : NormShape{512, 2};
    return {1024, channels <= 16384 ? 2 : 0};
}

int norm_check(const hr_norm_args* a) {
    if (!a || (a->dtype != HR_F32 && a->dtype != HR_BF16)) return HR_ERR_INVALID_ARG;
    if (a->heads < 1 || a->heads > kMaxHeads || a->channels < 1 || a->channels > kMaxChannels || a->tokens < 0) return HR_ERR_INVALID_ARG;
    if (!std::isfinite(a->eps) || a->eps < 0.0f || !std::isfinite(a->gain_offset)) return HR_ERR_INVALID_ARG;
    if (a->tokens > kMaxRows) return HR_ERR_LEN_RANGE;
    if (!a->total && !a->out && !a->block8) return HR_ERR_INVALID_ARG;
    if (a->block8) {
        const int rc = block8_check(a->block8, 1);
        if (rc != HR_OK) return rc;
        if (a->heads != 1) return HR_ERR_INVALID_ARG;
        if (a->block8->rows != a->tokens || a->block8->cols != a->channels) return HR_ERR_MISMATCH;
    }
    if (a->tokens == 0) return HR_OK;
    const uintptr_t esz = dtype_size(a->dtype);
    if (!a->x || !aligned(a->x, esz) || !aligned(a->add, esz) || !aligned(a->total, esz) || !aligned(a->out, esz) || !aligned(a->gain, 4)) return HR_ERR_INVALID_ARG;
    const int64_t T = a->tokens, H = a->heads, C = a->channels;
    if (!strides_fit(T, H, a->x_token_stride, a->x_head_stride)) return HR_ERR_INVALID_ARG;
    if (a->add && !strides_fit(T, H, a->add_token_stride, a->add_head_stride)) return HR_ERR_INVALID_ARG;
    struct Side { const void* p; int64_t t, h; };
    const Side x{a->x, a->x_token_stride, a->x_head_stride}, add{a->add, a->add_token_stride, a->add_head_stride};
    for (const Side& o : {Side{a->total, a->total_token_stride, a->total_head_stride}, Side{a->out, a->out_token_stride, a->out_head_stride}}) {
        if (!o.p) continue;
        if (!strides_fit(T, H, o.t, o.h) || !rows_apart(T, H, o.t, o.h, C)) return HR_ERR_INVALID_ARG;
        // a head is read by the lanes that write it, before they do: in place is fine, another arrangement of the same memory is not
        for (const Side& in : {x, add})
            if (in.p == o.p && !same_strides(*a, in.t, in.h, o.t, o.h)) return HR_ERR_INVALID_ARG;
        if (o.p == (const void*)a->gain) return HR_ERR_INVALID_ARG;
    }
    if (a->total && a->total == a->out) return HR_ERR_INVALID_ARG;
    if (a->block8) {
        if (a->block8->codes == (void*)a->block8->scales) return HR_ERR_INVALID_ARG;
        for (const void* p : {a->x, a->add, (const void*)a->total, (const void*)a->out, (const void*)a->gain})
            if (p && (p == a->block8->codes || p == (const void*)a->block8->scales)) return HR_ERR_INVALID_ARG;
    }
    return HR_OK;
}

int quantize_check(int dtype, const void* x, int64_t x_stride, const hr_block8* out) {
    if ((dtype != HR_F32 && dtype != HR_BF16) || !out || (out->block_rows != 1 && out->block_rows != kBlockCols)) return HR_ERR_INVALID_ARG;
    const int rc = block8_check(out, out->block_rows);
    if (rc != HR_OK) return rc;
    if (out->rows == 0) return HR_OK;
    if (!x || !aligned(x, dtype_size(dtype)) || !strides_fit(out->rows, 1, x_stride, 0)) return HR_ERR_INVALID_ARG;
    if (x == out->codes || x == (const void*)out->scales || out->codes == (void*)out->scales) return HR_ERR_INVALID_ARG;
    return out->block_rows > 1 && blocks_of(out->rows) * blocks_of(out->cols) > kMaxWorkgroups ? HR_ERR_LEN_RANGE : HR_OK;
}

int matmul_check(const hr_block8* a, const hr_block8* w, const hr_matmul_args* m) {
    int rc = block8_check(a, 1);
    if (rc != HR_OK) return rc;
    rc = block8_check(w, kBlockCols);
    if (rc != HR_OK) return rc;
    if (!m || (m->dtype != HR_F32 && m->dtype != HR_BF16) || m->gate < HR_GATE_NONE || m->gate > HR_GATE_GELU) return HR_ERR_INVALID_ARG;
    if (a->cols != w->cols) return HR_ERR_MISMATCH;
    if (m->gate != HR_GATE_NONE && w->rows % (2 * kBlockCols) != 0) return HR_ERR_MISMATCH;
    const int64_t wide = m->gate != HR_GATE_NONE ? w->rows / 2 : w->rows;
    if (m->block8) {
        if (m->out || m->add) return HR_ERR_INVALID_ARG;
        if (wide > 0) {                            // a matrix without columns is none
            rc = block8_check(m->block8, 1);
            if (rc != HR_OK) return rc;
            if (m->block8->rows != a->rows || m->block8->cols != wide) return HR_ERR_MISMATCH;
        }
    }
    if (a->rows == 0 || w->rows == 0) return HR_OK;
    if (!aligned(m->bias, 4)) return HR_ERR_INVALID_ARG;
    const void* outs[2] = {m->out, nullptr};
    if (m->block8) {
        outs[0] = m->block8->codes;
        outs[1] = m->block8->scales;
        if (outs[0] == outs[1]) return HR_ERR_INVALID_ARG;
    } else {
        const uintptr_t esz = dtype_size(m->dtype);
        if (!m->out || !aligned(m->out, esz) || !aligned(m->add, esz)) return HR_ERR_INVALID_ARG;
        if (!strides_fit(a->rows, 1, m->out_stride, 0) || !rows_apart(a->rows, 1, m->out_stride, 0, wide)) return HR_ERR_INVALID_ARG;
        if (m->add && !strides_fit(a->rows, 1, m->add_stride, 0)) return HR_ERR_INVALID_ARG;
        // a value's addend is read by the lane that writes it
        if (m->add == m->out && a->rows > 1 && m->add_stride != m->out_stride) return HR_ERR_INVALID_ARG;
    }
    for (const void* out : outs)
        for (const void* in : {(const void*)a->codes, (const void*)a->scales, (const void*)w->codes, (const void*)w->scales, (const void*)m->bias})
            if (out && out == in) return HR_ERR_INVALID_ARG;
    const MatmulArgs r = matmul_args(*a, *w, *m);
    const MatmulPlan plan = matmul_plan(r);
    if (matmul_tiles(plan.shape, r, plan.rows) > kMaxWideWorkgroups) return HR_ERR_LEN_RANGE;
    return HR_OK;
}

MatmulArgs matmul_args(const hr_block8& a, const hr_block8& w, const hr_matmul_args& m) {
    MatmulArgs r{};
    r.a = (const uint8_t*)a.codes;
    r.w = (const uint8_t*)w.codes;
    r.a_scales = a.scales;
    r.w_scales = w.scales;
    r.a_stride = a.row_stride;
    r.w_stride = w.row_stride;
    r.a_scale_stride = a.scale_stride;
    r.w_scale_stride = w.scale_stride;
    r.M = a.rows;
    r.K = a.cols;
    r.half = m.gate != HR_GATE_NONE ? (int32_t)(w.rows / 2) : 0;
    r.N = r.half > 0 ? r.half : (int32_t)w.rows;
    r.gate = m.gate;
    r.eight = m.fast != 0;
    r.bias = m.bias;
    r.add = m.add;
    r.out = m.out;
    r.add_stride = m.add_stride;
    r.out_stride = m.out_stride;
    if (m.block8) {
        r.codes = (uint8_t*)m.block8->codes;
        r.scales = m.block8->scales;
        r.code_stride = m.block8->row_stride;
        r.scale_stride = m.block8->scale_stride;
    }
    return r;
}

namespace {

// What a shape's launch takes in us: start + turns * first with a tile a CU at most, turns being its blocks of k by its groups along k; where a CU holds
// two workgroups, start + turns * pair with up to two; and turns * more + again for each further round of as many (the last of two may be half a round).
// By results: out with the 8-bit instruction (fitted into bf16) and with halves (into fp32), codes with either, codes of a gate with either.  Fitted to 5872 launches of 1 to 6000 rows with
// weights of 896 x 896 to 28672 x 4096 and 4096 x 14336, operands from memory, gates among them for codes only.  Over 21480 launches of other sizes, gated ones of
// every kind among them, what it picks takes 1.2 % more than the fastest shape in the mean and 30 % at most, with the 8-bit instruction 39 %, gated 78 % (17 to 250 rows, few
// columns).  The kernels without LDS: at 16 rows, with a gate by factors set by hand.
struct Times { float start, first, pair, more, again; };
struct Cost { int bm, bn, groups, held; Times t[6]; };
constexpr Cost kCost[MM_SHAPES] = {
    {16, 16, 8, 1, {{2.3f, 1.05f, 0.0f, 1.10f, 0.0f}, {2.3f, 1.05f, 0.0f, 1.10f, 0.0f}}},      // MM_FEW_16
    {16, 32, 8, 1, {{3.2f, 1.50f, 0.0f, 1.60f, 0.0f}, {3.2f, 1.50f, 0.0f, 1.60f, 0.0f}}},
    {16, 32, 8, 1, {{3.9f, 0.64f, 0.00f, 0.65f, 2.9f}, {3.9f, 0.76f, 0.00f, 0.76f, 2.9f}, {}, {}, {}, {}}},      // MM_16x32_8
    {32, 32, 8, 1, {{4.4f, 0.89f, 0.00f, 1.06f, 3.4f}, {4.7f, 1.00f, 0.00f, 1.05f, 3.7f}, {}, {}, {}, {}}},      // MM_32x32_8
    {16, 64, 4, 1, {{4.0f, 0.58f, 0.00f, 0.78f, 2.8f}, {4.0f, 0.73f, 0.00f, 0.87f, 3.0f}, {}, {}, {}, {}}},      // MM_16x64_4
    {32, 64, 2, 2, {{3.1f, 0.37f, 0.79f, 0.66f, 2.3f}, {3.2f, 0.53f, 1.04f, 0.79f, 2.8f}, {}, {}, {}, {}}},      // MM_32x64_2
    {64, 64, 1, 2, {{3.2f, 0.28f, 0.48f, 0.46f, 2.5f}, {3.1f, 0.47f, 0.77f, 0.66f, 2.7f}, {}, {}, {}, {}}},      // MM_64x64
    {64, 64, 2, 1, {{3.9f, 0.43f, 0.00f, 0.47f, 3.3f}, {3.5f, 0.79f, 0.00f, 0.74f, 3.2f}, {}, {}, {}, {}}},      // MM_64x64_2
    {64, 128, 1, 2, {{3.3f, 0.37f, 0.70f, 0.70f, 2.7f}, {4.3f, 0.72f, 1.23f, 1.12f, 3.4f}, {4.0f, 0.35f, 0.69f, 0.73f, 2.7f}, {3.8f, 0.80f, 1.25f, 1.12f, 2.9f}, {}, {}}},      // MM_64x128
    {64, 128, 2, 1, {{4.5f, 0.62f, 0.00f, 0.73f, 3.6f}, {4.6f, 1.25f, 0.00f, 1.21f, 3.5f}, {5.7f, 0.55f, 0.00f, 0.74f, 4.9f}, {5.4f, 1.24f, 0.00f, 1.19f, 4.4f}, {}, {}}},      // MM_64x128_2
    {64, 256, 1, 1, {{4.2f, 0.55f, 0.00f, 0.64f, 2.8f}, {5.0f, 1.17f, 0.00f, 1.16f, 3.4f}, {4.1f, 0.56f, 0.00f, 0.64f, 3.3f}, {4.3f, 1.20f, 0.00f, 1.19f, 3.2f}, {5.3f, 0.51f, 0.00f, 0.67f, 3.8f}, {4.8f, 1.18f, 0.00f, 1.18f, 3.7f}}},      // MM_64x256
    {128, 128, 1, 2, {{4.1f, 0.69f, 1.13f, 1.25f, 2.8f}, {7.9f, 1.17f, 1.84f, 1.92f, 4.7f}, {5.1f, 0.70f, 1.11f, 1.23f, 3.0f}, {7.1f, 1.18f, 1.83f, 1.92f, 4.4f}, {}, {}}},      // MM_128x128
    {128, 128, 2, 1, {{6.0f, 1.12f, 0.00f, 1.27f, 5.1f}, {8.2f, 1.71f, 0.00f, 1.83f, 5.5f}, {8.0f, 1.14f, 0.00f, 1.22f, 7.5f}, {9.6f, 1.73f, 0.00f, 1.83f, 7.6f}, {}, {}}},      // MM_128x128_2
    {128, 256, 1, 1, {{5.5f, 0.81f, 0.00f, 1.01f, 4.5f}, {9.1f, 1.61f, 0.00f, 1.78f, 6.3f}, {5.8f, 0.82f, 0.00f, 1.01f, 4.6f}, {6.8f, 1.64f, 0.00f, 1.75f, 5.1f}, {7.1f, 0.81f, 0.00f, 1.03f, 5.4f}, {8.2f, 1.65f, 0.00f, 1.77f, 6.3f}}},      // MM_128x256
    {256, 256, 1, 1, {{8.7f, 1.39f, 0.00f, 1.72f, 5.9f}, {14.7f, 2.85f, 0.00f, 3.09f, 11.0f}, {13.2f, 1.45f, 0.00f, 1.62f, 12.0f}, {12.7f, 3.03f, 0.00f, 3.16f, 9.1f}, {12.1f, 1.43f, 0.00f, 1.65f, 9.5f}, {14.6f, 2.90f, 0.00f, 3.02f, 11.8f}}},      // MM_256x256
    {16, 128, 4, 1, {{}, {}, {3.7f, 1.08f, 0.00f, 1.35f, 2.4f}, {4.0f, 1.13f, 0.00f, 1.28f, 2.9f}, {}, {}}},      // MM_16x128_4
    {32, 128, 2, 1, {{}, {}, {4.3f, 0.46f, 0.00f, 0.54f, 3.4f}, {4.6f, 0.79f, 0.00f, 0.77f, 4.0f}, {}, {}}},      // MM_32x128_2
    {16, 256, 1, 1, {{}, {}, {}, {}, {3.5f, 0.50f, 0.00f, 0.51f, 2.4f}, {3.6f, 0.66f, 0.00f, 0.64f, 3.1f}}},      // MM_16x256
    {32, 256, 1, 1, {{}, {}, {}, {}, {4.8f, 0.46f, 0.00f, 0.49f, 4.1f}, {5.0f, 0.78f, 0.00f, 0.78f, 4.4f}}},      // MM_32x256
};
constexpr int kCus = 256;

bool covers(int shape, bool codes, bool gate) {
    const int bn = kCost[shape].bn;
    if (!codes) return shape < MM_16x128_4 && !(gate && shape >= MM_16x32_8 && shape <= MM_16x64_4);      // whose wavefronts have 16 rows of w
    return shape > MM_FEW_32 && (gate ? bn >= 2 * kBlockCols : bn == kBlockCols || (bn > kBlockCols && kCost[shape].bm >= 64));
}

float cost_of(int shape, const MatmulArgs& a, int64_t rows, int results) {
    const Cost& c = kCost[shape];
    const Times& t = c.t[results];
    const int64_t tiles = matmul_tiles(shape, a, rows), rounds = (tiles + kCus - 1) / kCus, blocks = blocks_of(a.K);
    const float turns = (float)((blocks + c.groups - 1) / c.groups), further = std::max((float)(rounds - c.held) / (float)c.held, 0.0f);
    float first = rounds > 1 && c.held > 1 ? t.pair : t.first, more = t.more;
    if (shape <= MM_FEW_32) {
        if (a.half > 0) {                           // reads two pieces of w
            first *= 1.4f;
            more *= 1.5f;
        }
        first *= 0.6f + 0.025f * (float)std::min<int64_t>(rows, 16);      // lanes without a row read what others read
    }
    return t.start + turns * first + further * (turns * more + t.again);
}

}  // namespace

int64_t matmul_tiles(int shape, const MatmulArgs& a, int64_t rows) {
    const Cost& c = kCost[shape];
    const int wide = shape > MM_FEW_32 && a.half > 0 ? c.bn / 2 : c.bn;
    return (rows + c.bm - 1) / c.bm * ((a.N + wide - 1) / wide);
}

// The shape that costs least.  Rows that fill whole rounds of the largest tiles may go ahead of the others, which are then tiled for themselves where a launch can have
// that many tiles (matmul_check counts those of the first launch)
MatmulPlan matmul_plan(const MatmulArgs& a) {
    const bool codes = a.codes != nullptr, gate = a.half > 0;
    const int results = (codes ? (gate ? 4 : 2) : 0) + (a.eight ? 0 : 1);
    auto best = [&](int64_t rows, float& cost) {
        int shape = -1;
        for (int s = 0; s < MM_SHAPES; ++s) {
            if (!covers(s, codes, gate)) continue;
            const float t = cost_of(s, a, rows, results);
            if (shape < 0 || t < cost) {
                shape = s;
                cost = t;
            }
        }
        return shape;
    };
    float cost = 0.0f, rest_cost = 0.0f;
    MatmulPlan p{best(a.M, cost), a.M, 0};
    const Cost& large = kCost[MM_256x256];
    const int wide = gate ? large.bn / 2 : large.bn;
    const int64_t columns = (a.N + wide - 1) / wide, rounds = a.M / large.bm * columns / kCus;
    const int64_t rows = rounds * kCus / columns * large.bm;
    if (rows > 0 && rows < a.M) {
        const int rest = best(a.M - rows, rest_cost);
        if (rest != MM_256x256 && matmul_tiles(rest, a, a.M - rows) <= kMaxWideWorkgroups && cost_of(MM_256x256, a, rows, results) + rest_cost < 0.98f * cost)
            p = MatmulPlan{MM_256x256, rows, rest};
    }
    return p;
}

MatmulArgs matmul_rows(const MatmulArgs& a, int dtype, int64_t first, int64_t rows) {
    MatmulArgs r = a;
    const int64_t esz = (int64_t)dtype_size(dtype);
    r.M = rows;
    r.a += first * a.a_stride;
    r.a_scales += first * a.a_scale_stride;
    if (a.add) r.add = (const char*)a.add + first * a.add_stride * esz;
    if (a.out) r.out = (char*)a.out + first * a.out_stride * esz;
    if (a.codes) {
        r.codes += first * a.code_stride;
        r.scales += first * a.scale_stride;
    }
    return r;
}

}  // namespace hr
