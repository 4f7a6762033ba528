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

NormShape norm_shape(int channels, int64_t rows) {
    NormShape s{256, 0};
    auto fits = [&](int lanes, int most) {
        const int chunks = (channels + lanes * 8 - 1) / (lanes * 8);
        if (chunks > most) return false;
        s.lanes = lanes;
        s.chunks = chunks <= 1 ? 1 : chunks <= 2 ? 2 : chunks <= 4 ? 4 : 8;
        return true;
    };
    if (fits(16, 1) || fits(32, 1)) return s;
    if (rows >= 1024 ? fits(64, 8) : fits(64, 1)) return s;
    if (fits(256, 8)) return s;
    return s;
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
    const MatmulTile t = matmul_tile(a->rows, (int)wide, a->cols, m->dtype, m->gate, m->block8 != nullptr);
    if ((a->rows + t.bm - 1) / t.bm * ((wide + t.bn - 1) / t.bn) > kMaxWorkgroups) return HR_ERR_LEN_RANGE;
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

MatmulTile matmul_tile(int64_t M, int N, int K, int dtype, int gate, bool block8) {
    (void)K; (void)dtype;
    const bool gated = gate != HR_GATE_NONE;
    if (M > 64) {
        const bool large = M >= 2048 && N >= 1024;
        const int bm = large ? 256 : 128, bn = large ? 256 : 128;
        return MatmulTile{bm, gated ? (block8 && bn < 256 ? 128 : bn / 2) : bn, false};
    }
    const int bm = M <= 16 ? 16 : M <= 32 ? 32 : 64;
    return MatmulTile{bm, block8 ? 128 : gated ? 16 : 32, true};
}

}  // namespace hr
