// hr_pair_attention in fp32 arithmetic: fp32 pools, and 16-bit and fp8 pools whose head size the half kernels do not take; and the join of
// the pieces that long documents are cut into.
//
// A workgroup takes one block of 32 rows of one kv head, its four wavefronts every fourth sub-tile of 32 keys, each with a softmax of its own;
// they are joined through LDS in a fixed order.  K, V and the rows go from memory straight into the operands of the fp32 matrix instruction (a page
// holds them as a lane wants them: 8 channels of a key, 8 keys of a channel).  What bounds small calls is the chain of loads: work list, rows and
// page numbers, keys, own keys (8 queries of 16 tokens, documents of 128, 4 heads of 64: 14 us, of which the products are 4).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "hr_kernels.h"
#include "hr_pair_attn.h"
#include "hr_pair_launch.h"

namespace hr {

namespace {

constexpr int kWaves = 4;

typedef __attribute__((ext_vector_type(8))) float floatx8;

template <typename T>
__device__ __forceinline__ floatx8 load8(const T* p) {
    const Loose<T, 8> x = *(const Loose<T, 8>*)p;
    floatx8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = to_float<T>(x.w[e]);
    return r;
}
template <>
__device__ __forceinline__ floatx8 load8<uint8_t>(const uint8_t* p) {
    const uint2 x = *(const uint2*)p;
    floatx8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = e4m3_to_float((uint8_t)((e < 4 ? x.x : x.y) >> (8 * (e & 3))));
    return r;
}

template <int MB, typename PT, typename QT>
__global__ void __launch_bounds__(kWaves * 64) pair_attn_f32_kernel(PairAttnArgs a) {
    constexpr bool FP8 = sizeof(PT) == 1;
    extern __shared__ __attribute__((aligned(16))) float smem[];
    const int items = list_items(a, false);
    const int item = item_of((int)blockIdx.x, a.chunk);
    const int pieces = pair_choice(items, items, a.d, a.most_splits).pieces;
    if (item >= items || (int)blockIdx.y >= pieces) return;
    const int blk = item / a.n_kv, h = item - blk * a.n_kv;
    const PairItem it = list_item(a, false, blk);
    const int D = it.D, d = a.d;
    const int lane = threadIdx.x & 63, ln = lane & 31, hh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PairRow row = pair_row(a, h, it, it.row + ln);
    const int32_t* pt = a.page_table + (int64_t)it.pair * a.pt_stride;
    const int block = kPageTokens * d;                                  // elements of a K or V block
    const PT* pool = (const PT*)a.pool + (int64_t)h * 2 * block;
    const int64_t page_stride = (int64_t)a.n_kv * 2 * block;
    const QT *kn = (const QT*)a.k + h * a.k_hs, *vn = (const QT*)a.v + h * a.v_hs;

    // the sub-tiles that some row of the block sees, and this piece's share of them
    const int dlo = rows_min(row.dlo), dlo_all = rows_max(row.dlo), olo = rows_min(row.olo), ohi = rows_max(row.ohi);
    const int doc0 = dlo / 32, n_doc = max((D + 31) / 32 - doc0, 0), n_own = a.own_keys ? (ohi - olo + 31) / 32 : 0;
    const int n_sub = n_doc + n_own, share = (n_sub + pieces - 1) / pieces;
    const int j0 = (int)blockIdx.y * share, j1 = min(j0 + share, n_sub);

    floatx8 qf[2 * MB];                                                 // lane: row ln, channels 16 m + 8 hh ..
    {
        const QT* qr = (const QT*)a.q + row.token * a.q_ts + (h * a.g + row.head) * a.q_hs;
#pragma unroll
        for (int m = 0; m < 2 * MB; ++m) {
            if (16 * m < d) qf[m] = load8<QT>(qr + 16 * m + 8 * hh);
            else qf[m] = floatx8{};
        }
    }
    floatx16 o[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[mb] = floatx16{};
    PairSoftmax sm;

    for (int j = j0 + wave; j < j1; j += kWaves) {
        const bool doc = j < n_doc;
        const int key0 = doc ? (doc0 + j) * 32 : olo + (j - n_doc) * 32;
        // K: lane = key ln of the sub-tile
        floatx16 s = {};
        float ks[2] = {1.0f, 1.0f}, vs[2] = {1.0f, 1.0f};
        const PT* page[2] = {pool, pool};
        const QT* kr = kn;
        if (doc) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int at = min(key0 / kPageTokens + e, (D - 1) / kPageTokens);
                const int id = min(max(pt[at], 0), a.num_pages - 1);
                page[e] = pool + id * page_stride;
                if (FP8) {
                    const float2 sc = *(const float2*)(a.scales + ((int64_t)id * a.n_kv + h) * 2);
                    ks[e] = sc.x;
                    vs[e] = sc.y;
                }
            }
        } else {
            kr += own_token(a, min(key0 + ln, ohi - 1)) * a.k_ts;
        }
        const PT* kp = (ln >> 4) ? page[1] : page[0];
#pragma unroll
        for (int m = 0; m < 2 * MB; ++m) {
            if (16 * m >= d) break;
            const floatx8 kf = doc ? load8<PT>(kp + k_elem(ln & 15, 16 * m + 8 * hh, d, (int)sizeof(PT))) : load8<QT>(kr + 16 * m + 8 * hh);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[m][e], s, 0, 0, 0);
        }
        const float c0 = a.scale_log2 * ks[0], c1 = a.scale_log2 * ks[1];
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= r < 8 ? c0 : c1;
        pair_scores<PS_EXACT>(s, a, row, key0 - (doc ? row.pos : row.place), hh);
        const bool whole = doc && key0 >= dlo_all && key0 + 32 <= D;
        unsigned seen = 0xFFFFu;                                        // of the lane's 16 keys
        if (!whole) {
            const int lo = (doc ? row.dlo : row.olo) - key0 - 4 * hh, hi = (doc ? D : row.ohi) - key0 - 4 * hh;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = 8 * (r >> 2) + (r & 3);
                const bool on = key >= lo && key < hi;
                s[r] = on ? s[r] : -INFINITY;
                seen = on ? seen : seen & ~(1u << r);
            }
        }
        const float alpha = pair_softmax(sm, s);
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) o[mb] *= alpha;
        }
        // V: lane = channel ln of every 32, keys {0..3, 8..11} + 4 hh of a page
        const int exist = min(doc ? D - key0 : ohi - key0, 32);         // keys of the sub-tile that there are
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            if (32 * mb >= d) break;
            const int ch = min(32 * mb + ln, d - 1);
            floatx8 vf[2];
#pragma unroll
            for (int e2 = 0; e2 < 2; ++e2) {
                if (doc) {
                    vf[e2] = load8<PT>(page[e2] + block + (hh * d + ch) * 8);
                    if (FP8) vf[e2] *= vs[e2];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int x = min(key0 + 16 * e2 + (e & 3) + 2 * (e & 4) + 4 * hh, ohi - 1);
                        vf[e2][e] = to_float<QT>(vn[own_token(a, x) * a.v_ts + ch]);
                    }
                }
            }
            if (whole) {
#pragma unroll
                for (int e = 0; e < 16; ++e) o[mb] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[e >> 3][e & 7], s[e], o[mb], 0, 0, 0);
                continue;
            }
            // Some row does not see some key: that key's V counts for nothing there, whatever it holds, and 0 times infinity is not nothing.
            // Values that are not finite are counted where they are seen, as ones, kind by kind; the product has zeros for them.
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float v = 8 * (e >> 2) + (e & 3) + 4 * hh < exist ? vf[e >> 3][e & 7] : 0.0f;
                vf[e >> 3][e & 7] = v;
                odd = odd || !(fabsf(v) < INFINITY);
            }
            if (__any(odd)) {
#pragma unroll 1
                for (int kind = 0; kind < 3; ++kind) {                  // infinities of either sign, NaN
                    floatx16 n = {};
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float v = vf[e >> 3][e & 7];
                        const bool is = kind == 2 ? v != v : v == (kind == 0 ? INFINITY : -INFINITY);
                        n = __builtin_amdgcn_mfma_f32_32x32x2f32(is ? 1.0f : 0.0f, seen >> e & 1 ? 1.0f : 0.0f, n, 0, 0, 0);
                    }
                    const float add = kind == 2 ? NAN : kind == 0 ? INFINITY : -INFINITY;
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[mb][r] += n[r] > 0.0f ? add : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) vf[e >> 3][e & 7] = fabsf(vf[e >> 3][e & 7]) < INFINITY ? vf[e >> 3][e & 7] : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) o[mb] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[e >> 3][e & 7], s[e], o[mb], 0, 0, 0);
        }
    }

    pair_join_waves<kWaves, MB * 32, QT>(a, smem, o, sm, row, h, pieces);
}

// A row's pieces, joined in a fixed order: few pieces by one wavefront, many by the four of a workgroup, a quarter each.  Bound by reading them:
// 9824 rows of 6 pieces of 128 channels, 30 MB, 8.4 us (a workgroup for each row took 29); 14 rows of 128 pieces 5.7 us.
constexpr int kJoinAlone = 16;      // pieces that one wavefront joins: two rounds of loads

template <typename QT>
__device__ __forceinline__ void join_store(const PairAttnArgs& a, int64_t row, int c, float v) {
    const int n_q = a.g * a.n_kv;
    const int64_t token = row / n_q;
    ((QT*)a.out)[token * a.o_ts + (row - token * n_q) * a.o_hs + c] = from_float<QT>(v);
}

template <typename QT>
__global__ void __launch_bounds__(256) pair_join_kernel(PairAttnArgs a) {
    __shared__ float part[4][256], piece_m[kPairSplitMost], piece_l[kPairSplitMost];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int blocks = list_items(a, false), tiles = a.blocks_only ? blocks : list_items(a, true);
    const int pieces = pair_choice(blocks, tiles, a.d, a.most_splits).pieces;
    if (pieces == 1) return;                                            // the rows are there
    const int64_t rows = pair_join_rows(a.hdr[SH_TOKENS], a.max_tokens, a.g * a.n_kv);
    constexpr int AHEAD = 8;
    if (pieces <= kJoinAlone) {
        const int64_t row = (int64_t)blockIdx.x * 4 + wave;
        if (row >= rows) return;
        const float2 x = lane < pieces ? a.part_ml[lane * a.part_rows + row] : make_float2(-INFINITY, 0.0f);
        const float m = wave_max(x.x), f = piece_factor(x.x, m), sum = wave_sum(f * x.y), inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        for (int c = lane; c < a.d; c += 128) {
            const int c2 = min(c + 64, a.d - 1);
            float acc = 0.0f, acc2 = 0.0f;
            for (int p0 = 0; p0 < pieces; p0 += AHEAD) {
                float v[AHEAD], v2[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const float* o = a.part_o + (min(p0 + u, pieces - 1) * a.part_rows + row) * a.d;
                    v[u] = o[c];
                    v2[u] = o[c2];
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const float fu = p0 + u < pieces ? __shfl(f, p0 + u, 64) : 0.0f;
                    acc = fu != 0.0f ? fmaf(fu, v[u], acc) : acc;       // nothing is written of a piece that sees nothing
                    acc2 = fu != 0.0f ? fmaf(fu, v2[u], acc2) : acc2;
                }
            }
            join_store<QT>(a, row, c, acc * inv);
            if (c + 64 < a.d) join_store<QT>(a, row, c + 64, acc2 * inv);
        }
        if (lane == 0 && a.lse) a.lse[row] = pair_lse(m, sum);
        return;
    }
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        if (threadIdx.x < kPairSplitMost) {
            const float2 x = (int)threadIdx.x < pieces ? a.part_ml[threadIdx.x * a.part_rows + row] : make_float2(-INFINITY, 0.0f);
            piece_m[threadIdx.x] = x.x;
            piece_l[threadIdx.x] = x.y;
        }
        __syncthreads();
        static_assert(kPairSplitMost == 128, "two pieces a lane");
        const float m0 = piece_m[lane], m1 = piece_m[lane + 64], m = wave_max(fmaxf(m0, m1));
        const float sum = wave_sum(fmaf(piece_factor(m0, m), piece_l[lane], piece_factor(m1, m) * piece_l[lane + 64]));
        for (int c = lane; c < a.d; c += 64) {
            float acc = 0.0f;
            for (int p0 = wave; p0 < pieces; p0 += 4 * AHEAD) {
                float x[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) x[u] = a.part_o[(min(p0 + 4 * u, pieces - 1) * a.part_rows + row) * a.d + c];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const float f = p0 + 4 * u < pieces ? piece_factor(piece_m[min(p0 + 4 * u, pieces - 1)], m) : 0.0f;
                    acc = f != 0.0f ? fmaf(f, x[u], acc) : acc;
                }
            }
            part[wave][c] = acc;
        }
        __syncthreads();
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int c = threadIdx.x;
        if (c < a.d) join_store<QT>(a, row, c, (part[0][c] + part[1][c] + part[2][c] + part[3][c]) * inv);
        if (c == 0 && a.lse) a.lse[row] = pair_lse(m, sum);
        __syncthreads();                                                // the next row writes where this one reads
    }
}

template <int MB, typename PT, typename QT>
hipError_t f32_launch(const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    const size_t lds = pair_join_bytes(kWaves, MB * 32);
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)pair_attn_f32_kernel<MB, PT, QT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    pair_attn_f32_kernel<MB, PT, QT><<<grid, kWaves * 64, lds, st>>>(a);
    return hipGetLastError();
}
template <typename PT, typename QT>
hipError_t f32_by_size(const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    if (a.d <= 32) return f32_launch<1, PT, QT>(a, grid, st);
    if (a.d <= 64) return f32_launch<2, PT, QT>(a, grid, st);
    if (a.d <= 128) return f32_launch<4, PT, QT>(a, grid, st);
    return f32_launch<8, PT, QT>(a, grid, st);
}

}  // namespace

static hipError_t launch_pair_join(int dtype, const PairAttnArgs& a, int64_t max_tokens, hipStream_t st) {
    const unsigned blocks = (unsigned)pair_join_groups(max_tokens * a.g * a.n_kv);
    if (dtype == HR_F32) pair_join_kernel<float><<<blocks, 256, 0, st>>>(a);
    else pair_join_kernel<bf16_t><<<blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_pair_attention(const hr_pool* pool, const hr_pair_tables* t, const hr_attention_args* g, void* workspace, hipStream_t st) {
    const PoolLayout& lay = pool->lay;
    const int heads = t->n_q_heads / lay.n_kv;
    const SchedLayout s = make_sched_layout(t->n_pairs, t->max_tokens, heads);
    const int32_t* S = (const int32_t*)t->sched;
    PairAttnArgs a{};
    a.hdr = S + s.hdr;
    a.rec = (const int4*)(S + s.blk);
    a.ord = (const int4*)(S + s.ord);
    a.page_table = t->page_table;
    a.pt_stride = t->pt_stride;
    a.n_kv = lay.n_kv;
    a.g = heads;
    a.num_pages = lay.num_pages;
    a.d = lay.d;
    a.window = g->window;
    a.own_keys = g->k != nullptr;
    a.n_pairs = t->n_pairs;
    a.max_tokens = t->max_tokens;
    a.cap_blk = s.cap_blk;
    a.cap_tile = s.cap_tile;
    a.q_cu = t->q_cu;
    a.prefix = g->prefix_lens;
    a.pool = pool->base + (size_t)g->layer * lay.num_pages * lay.n_kv * 2 * lay.block_elems * lay.esz;
    a.scales = lay.kv_dtype == HR_FP8_E4M3 ? (const float*)(pool->base + lay.data_bytes) + lay.scale_index(g->layer, 0, 0, 0) : nullptr;
    a.q = g->q; a.k = g->k; a.v = g->v; a.out = g->out; a.lse = g->lse; a.slopes = g->slopes;
    a.q_ts = g->q_token_stride; a.q_hs = g->q_head_stride; a.k_ts = g->k_token_stride; a.k_hs = g->k_head_stride;
    a.v_ts = g->v_token_stride; a.v_hs = g->v_head_stride; a.o_ts = g->out_token_stride; a.o_hs = g->out_head_stride;
    a.scale_log2 = (g->scale != 0.0f ? g->scale : 1.0f / sqrtf((float)lay.d)) * kLog2e;
    if (g->cap > 0.0f) {
        a.cap_log2 = g->cap * kLog2e;
        a.cap_in = 2.0f / g->cap;                        // x = s / (cap log2 e); e^2x = 2^(2 log2 e x) = 2^(2 s / cap)
    }
    const PairWorkspace w = make_pair_workspace(t->n_pairs, t->max_tokens, t->n_q_heads, lay.n_kv, lay.d, t->pt_stride);
    a.most_splits = w.most;
    a.part_ml = (float2*)workspace;
    a.part_o = (float*)((char*)workspace + w.o);
    a.part_rows = (int64_t)t->max_tokens * t->n_q_heads;
    const int64_t items = s.cap_blk * lay.n_kv;
    while (w.most == 1 && a.chunk < 5 && 1 << a.chunk < 2 * lay.n_kv) ++a.chunk;
    const int64_t round = 8 << a.chunk;
    const dim3 grid((unsigned)((items + round - 1) / round * round), (unsigned)w.most);
    hipError_t e;
    a.rec_tiles = (const int4*)(S + s.tile);
    const bool half = lay.kv_dtype != HR_F32 && (lay.d == 64 || lay.d == 96 || lay.d == 128);
    a.blocks_only = !half;
    if (half) e = launch_pair_half(lay.kv_dtype == HR_FP8_E4M3, a, grid, st);
    else if (lay.kv_dtype == HR_F32) e = f32_by_size<float, float>(a, grid, st);
    else if (lay.kv_dtype == HR_BF16) e = f32_by_size<half_t, bf16_t>(a, grid, st);
    else e = f32_by_size<uint8_t, bf16_t>(a, grid, st);
    if (e != hipSuccess || w.most == 1) return e;
    return launch_pair_join(g->dtype, a, t->max_tokens, st);
}

}  // namespace hr
