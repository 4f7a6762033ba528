// Host part of the operators for models whose layers the caller runs: argument checks, frequencies, the layout of the work list.
// No HIP calls here, so every refusal can be exercised on a machine without a GPU.
#include <algorithm>
#include <cmath>

#include "hr_pair.h"

namespace hr {

namespace {

constexpr int32_t kMaxTokens = 1 << 30, kMaxStride = 1 << 26;
constexpr int64_t kMaxGroups = (1 << 24) - 512;      // workgroups of 256 threads in a launch, of which items are rounded up to 256

bool finite_positive(float v) { return v > 0.0f && std::isfinite(v); }

// The largest offset that [tokens][heads][channels] reaches must fit 62 bits; negative strides are not meant
bool strides_fit(int64_t tokens, int64_t heads, int64_t token_stride, int64_t head_stride) {
    if (token_stride < 0 || head_stride < 0) return false;
    constexpr int64_t most = (int64_t)1 << 60;
    return (tokens <= 1 || token_stride <= most / tokens) && (heads <= 1 || head_stride <= most / heads);
}

// Rows of `channels` elements at token * token_stride + head * head_stride share no element: the rows of one index lie inside a step of the other
bool rows_apart(int64_t tokens, int64_t heads, int64_t token_stride, int64_t head_stride, int64_t channels) {
    if ((tokens > 1 && token_stride < channels) || (heads > 1 && head_stride < channels)) return false;
    if (tokens <= 1 || heads <= 1) return true;
    return token_stride >= (heads - 1) * head_stride + channels || head_stride >= (tokens - 1) * token_stride + channels;
}

}  // namespace

int rope_check(const hr_rope_cfg* c) {
    if (!c) return HR_ERR_INVALID_ARG;
    if (c->head_dim < 2 || c->head_dim > 1024) return HR_ERR_INVALID_ARG;
    if (c->rotary_dim < 2 || c->rotary_dim % 2 != 0 || c->rotary_dim > c->head_dim || c->rotary_dim > 2 * kMaxRotaryPairs) return HR_ERR_INVALID_ARG;
    if (c->layout != HR_ROPE_HALF && c->layout != HR_ROPE_INTERLEAVED) return HR_ERR_INVALID_ARG;
    if (!finite_positive(c->amplitude)) return HR_ERR_INVALID_ARG;
    return HR_OK;
}

int rope_apply_check(const hr_rope_cfg* c, const double* freqs, int dtype, int64_t n_tokens, const int32_t* positions, int32_t first_position,
                     int32_t period, const hr_rope_tensor* tensors, int32_t n_tensors) {
    if (rope_check(c) != HR_OK || !freqs || n_tokens < 0 || (dtype != HR_F32 && dtype != HR_BF16)) return HR_ERR_INVALID_ARG;
    if (!tensors || n_tensors < 1 || n_tensors > 2) return HR_ERR_INVALID_ARG;
    for (int i = 0; i < c->rotary_dim / 2; ++i)
        if (!(freqs[i] >= 0.0) || !(freqs[i] < 6.283185307179586)) return HR_ERR_INVALID_ARG;
    if (n_tokens > kMaxTokens) return HR_ERR_LEN_RANGE;
    if (!positions) {
        if (first_position < 0 || period < 0) return HR_ERR_INVALID_ARG;
        const int64_t last = period > 0 ? std::min<int64_t>(period, n_tokens) - 1 : n_tokens - 1;
        if (first_position + last > INT32_MAX) return HR_ERR_LEN_RANGE;
    }
    int64_t heads = 0;
    for (int i = 0; i < n_tensors; ++i) {
        const hr_rope_tensor& t = tensors[i];
        if (!t.in || !t.out || t.n_heads < 1 || t.n_heads > 65536) return HR_ERR_INVALID_ARG;
        if (!strides_fit(n_tokens, t.n_heads, t.in_token_stride, t.in_head_stride)) return HR_ERR_INVALID_ARG;
        if (!strides_fit(n_tokens, t.n_heads, t.out_token_stride, t.out_head_stride)) return HR_ERR_INVALID_ARG;
        if (t.in == t.out && (t.in_token_stride != t.out_token_stride || t.in_head_stride != t.out_head_stride)) return HR_ERR_INVALID_ARG;
        if (!rows_apart(n_tokens, t.n_heads, t.out_token_stride, t.out_head_stride, c->head_dim)) return HR_ERR_INVALID_ARG;
        const uintptr_t esz = dtype_size(dtype);
        if ((uintptr_t)t.in % esz != 0 || (uintptr_t)t.out % esz != 0) return HR_ERR_INVALID_ARG;
        heads += t.n_heads;
    }
    // what one tensor's rows are turned into, nothing else is read or written
    if (n_tensors == 2 && (tensors[0].out == tensors[1].out || tensors[0].out == tensors[1].in || tensors[1].out == tensors[0].in)) return HR_ERR_INVALID_ARG;
    const RopeShape s = rope_shape(c->head_dim, c->rotary_dim, c->layout, (int)dtype_size(dtype), false, (int)heads);
    if (n_tokens / ((int64_t)s.tokens * kRopeWaves) > kMaxGroups) return HR_ERR_LEN_RANGE;
    return HR_OK;
}

RopeShape rope_shape(int head_dim, int rotary_dim, int layout, int esz, bool in_place, int n_heads) {
    const int rest = in_place ? 0 : head_dim - rotary_dim;         // channels that are only copied
    // pairs a lane takes: one load brings vec channels (half) or 2 vec (interleaved), 16 bytes at most
    const int wide = layout == HR_ROPE_INTERLEAVED ? 2 : 1;
    int vec = 16 / (esz * wide);
    while (vec > 1 && (rotary_dim / 2 % vec != 0 || rest % (vec * wide) != 0)) vec /= 2;
    RopeShape s;
    s.vec = vec;
    s.chunks = rotary_dim / 2 / vec + (rest + vec * wide - 1) / (vec * wide);
    const int per = std::max(1, 64 / s.chunks);                    // heads side by side in a wavefront
    s.heads = std::min(per, n_heads);
    s.tokens = std::max(1, per / s.heads);
    return s;
}

SchedLayout make_sched_layout(int64_t n_pairs, int64_t max_tokens, int g) {
    SchedLayout s;
    int64_t o = 0;
    auto take = [&](int64_t ints) {
        const int64_t at = o;
        o = (o + ints + 15) / 16 * 16;
        return at;
    };
    const int64_t groups = std::min(n_pairs, max_tokens);          // groups with a token: one partly filled block each
    s.cap_blk = max_tokens * g / kPairBlkRows + groups;
    s.cap_tile = max_tokens * g / kPairTileRows + groups;
    s.hdr = take(16);
    s.ord_first = take(n_pairs);
    s.grp_pair = take(n_pairs + 1);
    s.grp_tok = take(n_pairs + 1);
    s.blk_cu = take(n_pairs + 1);
    s.tile_cu = take(n_pairs + 1);
    s.key[0] = take(n_pairs);
    s.key[1] = take(n_pairs);
    s.idx = take(n_pairs);
    s.ord = take(max_tokens * 4);
    s.blk = take(s.cap_blk * kSchedRec);
    s.tile = take(s.cap_tile * kSchedRec);
    s.total = o;
    return s;
}

static int tables_sizes_check(const hr_pool* pool, int32_t n_pairs, int32_t max_tokens, int32_t n_q_heads) {
    if (!pool || n_pairs < 0 || max_tokens < 0 || n_q_heads < 1 || n_q_heads % pool->cfg.n_kv_heads != 0) return HR_ERR_INVALID_ARG;
    if (n_pairs > kMaxTokens || (int64_t)max_tokens * (n_q_heads / pool->cfg.n_kv_heads) > kMaxTokens) return HR_ERR_LEN_RANGE;
    return HR_OK;
}

int tables_check(const hr_pool* pool, const hr_pair_tables* t) {
    if (!t) return HR_ERR_INVALID_ARG;
    const int rc = tables_sizes_check(pool, t->n_pairs, t->max_tokens, t->n_q_heads);
    if (rc != HR_OK) return rc;
    if (t->pt_stride < 0 || t->pt_stride > kMaxStride) return t->pt_stride < 0 ? HR_ERR_INVALID_ARG : HR_ERR_LEN_RANGE;
    if (t->n_pairs == 0) return HR_OK;
    if (!t->q_cu || !t->doc_lens || !t->order || !t->report || !t->sched || (t->pt_stride > 0 && !t->page_table)) return HR_ERR_INVALID_ARG;
    if (t->max_tokens > 0 && (!t->tok_pos || !t->tok_pair)) return HR_ERR_INVALID_ARG;
    if ((uintptr_t)t->sched % 16 != 0) return HR_ERR_INVALID_ARG;
    const SchedLayout s = make_sched_layout(t->n_pairs, t->max_tokens, t->n_q_heads / pool->cfg.n_kv_heads);
    if (t->sched_bytes < (size_t)s.total * sizeof(int32_t)) return HR_ERR_WORKSPACE_SMALL;
    return HR_OK;
}

int tables_build_check(const hr_pool* pool, const hr_doc_list* docs, const int32_t* pair_doc, const int32_t* query_lens, const hr_pair_tables* t) {
    const int rc = tables_check(pool, t);
    if (rc != HR_OK) return rc;
    if (!docs || docs->n_docs < 0 || docs->n_pages < 0 || docs->n_docs == INT32_MAX) return HR_ERR_INVALID_ARG;
    if (t->n_pairs == 0) return HR_OK;
    if (!pair_doc || !query_lens) return HR_ERR_INVALID_ARG;
    if (docs->n_docs > 0 && (!docs->doc_lens || !docs->page_cu)) return HR_ERR_INVALID_ARG;
    if (docs->n_pages > 0 && !docs->pages) return HR_ERR_INVALID_ARG;
    return HR_OK;
}

int pair_most_splits(int64_t n_pairs, int64_t max_tokens, int n_q, int n_kv, int d, int64_t pt_stride) {
    const int64_t keys = pt_stride * kPageTokens, rows = max_tokens * (n_q / n_kv);
    if (keys < kPairSplitLeast) return 1;
    // items of a full batch: blocks are fewest with all pairs in one group and most with a group each; tiles hold at most four blocks, and
    // are taken from a number of blocks on
    const int64_t blocks = (rows + kPairBlkRows - 1) / kPairBlkRows * n_kv, most_blocks = (rows / kPairBlkRows + std::min(n_pairs, max_tokens)) * n_kv;
    int64_t s = kPairSplitWgs / std::max<int64_t>(blocks, 1);
    const int64_t from = pair_tile_blocks(d);
    if (most_blocks > from) s = std::max<int64_t>(s, kPairSplitWgs / std::max((blocks + 3) / 4, (from + 3) / 4));
    s = std::min<int64_t>(s, std::min<int64_t>((keys + kPairSplitKeys - 1) / kPairSplitKeys, kPairSplitMost));
    return (int)std::max<int64_t>(s, 1);
}

PairWorkspace make_pair_workspace(int64_t n_pairs, int64_t max_tokens, int n_q, int n_kv, int d, int64_t pt_stride) {
    PairWorkspace w;
    w.most = pair_most_splits(n_pairs, max_tokens, n_q, n_kv, d, pt_stride);
    if (w.most == 1) return w;
    const size_t rows = (size_t)w.most * (size_t)max_tokens * n_q;
    w.o = align_up(rows * 2 * sizeof(float));
    w.total = align_up(w.o + rows * d * sizeof(float));
    return w;
}

int attention_check(const hr_pool* pool, const hr_pair_tables* t, const hr_attention_args* a) {
    int rc = tables_check(pool, t);
    if (rc != HR_OK) return rc;
    if (!a) return HR_ERR_INVALID_ARG;
    if (a->dtype != HR_F32 && a->dtype != HR_BF16) return HR_ERR_INVALID_ARG;
    if ((a->dtype == HR_F32) != (pool->cfg.kv_dtype == HR_F32)) return HR_ERR_MISMATCH;
    if (a->layer < 0 || a->layer >= pool->cfg.n_layers) return HR_ERR_INVALID_ARG;
    if (!std::isfinite(a->scale) || !std::isfinite(a->cap) || a->cap < 0.0f || a->window < 0) return HR_ERR_INVALID_ARG;
    if (a->cap > 0.0f && !(a->cap >= 1e-18f && a->cap <= 1e18f)) return HR_ERR_INVALID_ARG;      // its reciprocal is used
    if (t->n_pairs == 0 || t->max_tokens == 0) return HR_OK;
    if (!a->q || !a->out || (a->k != nullptr) != (a->v != nullptr)) return HR_ERR_INVALID_ARG;
    const int n_q = t->n_q_heads, n_kv = pool->cfg.n_kv_heads, d = pool->cfg.head_dim;
    const uintptr_t esz = dtype_size(a->dtype);
    if ((uintptr_t)a->q % esz != 0 || (uintptr_t)a->k % esz != 0 || (uintptr_t)a->v % esz != 0 || (uintptr_t)a->out % esz != 0) return HR_ERR_INVALID_ARG;
    if (!strides_fit(t->max_tokens, n_q, a->q_token_stride, a->q_head_stride) || !strides_fit(t->max_tokens, n_q, a->out_token_stride, a->out_head_stride))
        return HR_ERR_INVALID_ARG;
    if (a->k && (!strides_fit(t->max_tokens, n_kv, a->k_token_stride, a->k_head_stride) ||
                 !strides_fit(t->max_tokens, n_kv, a->v_token_stride, a->v_head_stride)))
        return HR_ERR_INVALID_ARG;
    if (!rows_apart(t->max_tokens, n_q, a->out_token_stride, a->out_head_stride, d)) return HR_ERR_INVALID_ARG;
    if (make_sched_layout(t->n_pairs, t->max_tokens, n_q / n_kv).cap_blk * n_kv > kMaxGroups) return HR_ERR_LEN_RANGE;
    return HR_OK;
}

int attention_outputs_check(const hr_attention_args* a) {
    // workgroups write their rows while others still read keys and values, and lse is not rows of out
    for (const void* in : {a->q, a->k, a->v, (const void*)a->lse})
        if (a->out == in) return HR_ERR_INVALID_ARG;
    for (const void* in : {a->q, a->k, a->v, (const void*)a->slopes, (const void*)a->prefix_lens})
        if (a->lse && a->lse == in) return HR_ERR_INVALID_ARG;
    return HR_OK;
}

}  // namespace hr

extern "C" {

int hr_rope_frequencies(const hr_rope_cfg* c, double* out) {
    if (hr::rope_check(c) != HR_OK || !out) return HR_ERR_INVALID_ARG;
    const int s = c->scaling, r = c->rotary_dim;
    if (s < HR_ROPE_SCALE_NONE || s > HR_ROPE_SCALE_RAMP || !(c->base > 1.0f) || !std::isfinite(c->base)) return HR_ERR_INVALID_ARG;
    if (s != HR_ROPE_SCALE_NONE && (!(c->factor >= 1.0f) || !std::isfinite(c->factor))) return HR_ERR_INVALID_ARG;
    if (s == HR_ROPE_SCALE_BASE && r <= 2) return HR_ERR_INVALID_ARG;
    const bool turns = s == HR_ROPE_SCALE_BANDS || s == HR_ROPE_SCALE_RAMP;
    if (turns && (!hr::finite_positive(c->original_len) || !hr::finite_positive(c->low) || !(c->high > c->low) || !std::isfinite(c->high)))
        return HR_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586, factor = c->factor, len = c->original_len;
    const double base = s == HR_ROPE_SCALE_BASE ? c->base * std::pow(factor, r / (r - 2.0)) : (double)c->base;
    // RAMP: the index at which a pair makes n turns over the original length, len base^(-2 i / r) = 2 pi n solved for i
    auto index = [&](double n) { return r * std::log(len / (two_pi * n)) / (2.0 * std::log(base)); };
    double first = 0.0, last = 0.0;
    if (s == HR_ROPE_SCALE_RAMP) {
        first = std::max(std::floor(index(c->high)), 0.0);
        last = std::max(std::min(std::ceil(index(c->low)), r - 1.0), first);
    }
    for (int i = 0; i < r / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / r);
        double keep = 1.0;                                          // share of f itself, the rest is f / factor
        if (s == HR_ROPE_SCALE_LINEAR) keep = 0.0;
        if (s == HR_ROPE_SCALE_BANDS) keep = std::clamp((len * f / two_pi - c->low) / ((double)c->high - c->low), 0.0, 1.0);
        if (s == HR_ROPE_SCALE_RAMP) keep = 1.0 - std::clamp((i - first) / (last != first ? last - first : 0.001), 0.0, 1.0);
        out[i] = keep == 1.0 ? f : keep * f + (1.0 - keep) * f / factor;
    }
    return HR_OK;
}

size_t hr_pair_tables_sched_bytes(const hr_pool* pool, int32_t n_pairs, int32_t max_tokens, int32_t n_q_heads) {
    if (hr::tables_sizes_check(pool, n_pairs, max_tokens, n_q_heads) != HR_OK) return 0;
    return (size_t)hr::make_sched_layout(n_pairs, max_tokens, n_q_heads / pool->cfg.n_kv_heads).total * sizeof(int32_t);
}

size_t hr_pair_attention_workspace_bytes(const hr_pool* pool, const hr_pair_tables* t) {
    if (hr::tables_check(pool, t) != HR_OK || t->n_pairs == 0) return 0;
    return hr::make_pair_workspace(t->n_pairs, t->max_tokens, t->n_q_heads, pool->cfg.n_kv_heads, pool->cfg.head_dim, t->pt_stride).total;
}

}  // extern "C"
