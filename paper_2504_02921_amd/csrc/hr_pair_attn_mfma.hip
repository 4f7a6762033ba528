// hr_pair_attention on the half matrix instructions: 16-bit and fp8 pools with heads of 64 or 128 channels.
//
// A workgroup of four wavefronts goes about its work item in one of two ways; the device, which knows the items, chooses (pair_choice):
//   few rows   the item is one block of 32 rows, a wavefront has every fourth sub-tile of 32 keys and a softmax of its own, and they are joined
//              through LDS in a fixed order.  K and V go from memory straight into operand registers: V pages hold a channel's 8 keys as a lane
//              wants them, and a K instruction takes 32 bytes of each of 32 rows, whose lines the next ones take the rest of.
//   many rows  the item is a tile of up to four blocks, one per wavefront, and keys go through LDS in stages of 64 (four pages), double
//              buffered, in the pool's own arrangement: half pages straight from memory, fp8 pages by way of a wavefront's registers, which
//              expands them once for all rows.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "hr_kernels.h"
#include "hr_pair_half.h"
#include "hr_pair_launch.h"

namespace hr {

namespace {

constexpr int kPairWaves = 4;
constexpr int kStageKeys = 64, kStagePages = kStageKeys / kPageTokens;

template <int HD>
struct TileGeo {
    static constexpr int HBLOCK = kPageTokens * HD * 2, HPAGE = 2 * HBLOCK, STAGE = kStagePages * HPAGE;      // bytes, as half
    static constexpr int TURN = HD * 2 + 16;      // bytes between the rows of a block on its way out: they start at other banks
    static constexpr int LDS = std::max(2 * STAGE, kPairWaves * 32 * TURN);
};

// What rows of a group see together (row, row + 1, .. last of them), without asking each
struct PairSpan {
    int dlo, dlo_all;                 // document keys that some row sees begin at dlo, those that all see at dlo_all
    int olo, ohi;                     // own keys that some row sees, by place
};
// mine: the rows of this wavefront, one per lane of a half
__device__ __forceinline__ PairSpan pair_span(const PairAttnArgs& a, const PairRow& mine, int4 rec, int first, int last) {
    PairSpan s;
    if (a.window > 0) {
        s.dlo = rows_min(mine.dlo);
        s.dlo_all = rows_max(mine.dlo);
        s.olo = rows_min(mine.olo);
        s.ohi = rows_max(mine.ohi);
        return s;
    }
    // without a window: the first row's query from its first token, the last row's as far as that row sees
    const int t0 = rec.z + first / a.g, t1 = rec.z + last / a.g;
    const const_int_t f = (const_int_t)(a.ord + t0), l = (const_int_t)(a.ord + t1);
    s.dlo = s.dlo_all = 0;
    s.olo = f[1];
    s.ohi = t1 + 1;
    if (a.prefix) {
        const int pair = l[2], n = ((const_int_t)a.q_cu)[pair + 1] - ((const_int_t)a.q_cu)[pair];
        s.ohi = max(s.ohi, l[1] + min(((const_int_t)a.prefix)[pair], n));
    }
    return s;
}

// by value: a conditional of two members of an array would keep the array in memory
__device__ __forceinline__ float pick(bool second, float a, float b) { return second ? b : a; }
__device__ __forceinline__ int pick(bool second, int a, int b) { return second ? b : a; }

template <int HD>
__device__ __forceinline__ void load_q(const PairAttnArgs& a, const PairRow& row, int h, int hh, halfx8 (&q)[HD / 16]) {
    const bf16_t* qr = (const bf16_t*)a.q + row.token * a.q_ts + (h * a.g + row.head) * a.q_hs;
#pragma unroll
    for (int kk = 0; kk < HD / 16; ++kk) q[kk] = bf16x8_to_half(qr + 16 * kk + 8 * hh);
}

// ---- few rows
template <int HD, bool FP8, bool EXTRA>
__device__ __forceinline__ void pair_rows(const PairAttnArgs& a, float* smem, int4 rec, int rows, int h, int pieces) {
    using G = PairGeo<HD, FP8>;
    using Piece = typename G::Piece;
    constexpr int KC = G::KC, MB = G::MB, NW = kPairWaves;
    const int D = rec.y;
    const int lane = threadIdx.x & 63, ln = lane & 31, hh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PairRow row = pair_row(a, h, rec, rows, rec.w + ln);
    const const_int_t pt = (const_int_t)(a.page_table + (int64_t)rec.x * a.pt_stride);
    const char* pool = a.pool + (int64_t)h * 2 * G::BLOCK;
    const int64_t page_stride = (int64_t)a.n_kv * 2 * G::BLOCK;

    // The sub-tiles that some row of the block sees: document sub-tiles that all rows see whole, then those at an edge (the window's, the
    // document's end), then the pairs' own keys; and this piece's share of them
    const PairSpan span = pair_span(a, row, rec, rec.w, min(rec.w + 32, rows) - 1);
    const int dlo = span.dlo, dlo_all = span.dlo_all, olo = span.olo, ohi = span.ohi;
    const int doc0 = dlo / 32, doc1 = (D + 31) / 32, whole0 = (dlo_all + 31) / 32, whole1 = max(D / 32, whole0);
    const int n_whole = whole1 - whole0, n_doc = max(doc1 - doc0, 0), n_own = a.own_keys ? (ohi - olo + 31) / 32 : 0;
    const int n_sub = n_doc + n_own, share = (n_sub + pieces - 1) / pieces;
    const int j0 = (int)blockIdx.y * share, j1 = min(j0 + share, n_sub);
    const int last_page = (D - 1) / kPageTokens;

    floatx16 o[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[mb] = floatx16{};
    PairSoftmax sm;
    halfx8 qf[KC];                                                      // lane: row ln, channels 16 kk + 8 hh ..

    // a sub-tile's pages, and its K and V as they lie there; a lane's key is ln: page ln >> 4, token ln & 15
    const int t = ln & 15;
    const char* page[2];
    auto find = [&](int sub, float (&k_scale)[2], float (&v_scale)[2]) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int id = min(max(pt[min(2 * sub + e, last_page)], 0), a.num_pages - 1);
            page[e] = pool + id * page_stride;
            if constexpr (FP8) {
                const const_float_t sc = (const_float_t)(a.scales + ((int64_t)id * a.n_kv + h) * 2);
                k_scale[e] = sc[0];
                v_scale[e] = sc[1];
            }
        }
    };
    auto load_k = [&](Piece (&kr)[KC]) {
        const char* p = ln >> 4 ? page[1] : page[0];
#pragma unroll
        for (int kk = 0; kk < KC; ++kk) kr[kk] = *(const Piece*)(p + (t * HD + (((2 * kk + hh) ^ k_swizzle(t, HD, G::ESZ)) << 3)) * G::ESZ);
    };
    auto load_v = [&](Piece (&vr)[MB][2]) {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int e = 0; e < 2; ++e) vr[mb][e] = *(const Piece*)(page[e] + G::BLOCK + (hh * HD + mb * 32 + ln) * 8 * G::ESZ);
    };
    auto rescale = [&](float alpha) {
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) o[mb] *= alpha;
        }
    };
    auto half_k = [&](const Piece& x) {
        if constexpr (FP8) return fp8x8_to_half(x, fp8_expand_factor(1.0f));
        else return x;
    };
    auto half_v = [&](const Piece& x, float scale) {
        if constexpr (FP8) return fp8x8_to_half(x, fp8_expand_factor(scale));
        else return x;
    };

    int j = j0 + wave;
    const int jw = min(j1, n_whole);
    if (j >= jw) {
        load_q<HD>(a, row, h, hh, qf);
    } else {
        Piece kr[KC], vr[MB][2];
        float ks[2] = {1.0f, 1.0f}, vs[2] = {1.0f, 1.0f}, vs_next[2] = {1.0f, 1.0f};
        find(whole0 + j, ks, vs);
        load_k(kr);
        load_v(vr);
        load_q<HD>(a, row, h, hh, qf);
        for (; j < jw; j += NW) {
            floatx16 s = {};
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(half_k(kr[kk]), qf[kk], s, 0, 0, 0);
            const float c0 = a.scale_log2 * ks[0], c1 = a.scale_log2 * ks[1];
            // the next sub-tile's; behind the last one, that one's again (the requests are counted, so they are made in any case)
            find(whole0 + min(j + NW, jw - 1), ks, vs_next);
            load_k(kr);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] *= r < 8 ? c0 : c1;
            if (EXTRA) pair_scores<false>(s, a, row, (whole0 + j) * 32 - row.pos, hh);
            rescale(pair_softmax(sm, s));
            halfx8 pf[2];
            pack_p(s, pf, FP8 ? fp8_scale_mantissa(vs[0]) : 1.0f, FP8 ? fp8_scale_mantissa(vs[1]) : 1.0f);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int e = 0; e < 2; ++e) o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(half_v(vr[mb][e], vs[e]), pf[e], o[mb], 0, 0, 0);
            load_v(vr);
            vs[0] = vs_next[0];
            vs[1] = vs_next[1];
        }
    }
#pragma unroll 1
    for (; j < j1; j += NW) {
        const bool doc = j < n_doc;
        float ks[2] = {1.0f, 1.0f}, vs[2] = {1.0f, 1.0f};
        floatx16 s = {};
        char* stay = (char*)(smem + wave * 32 * (HD + 4));                    // V of the sub-tile as two half pages' V blocks
        constexpr int STAY = kPageTokens * HD * 2;
        int key0, exist;
        if (doc) {
            const int sub = j - n_whole < whole0 - doc0 ? doc0 + j - n_whole : doc0 + j;        // the edge in front, the edge behind
            key0 = 32 * sub;
            exist = min(D - key0, 32);
            Piece x[KC];
            find(sub, ks, vs);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int i = 0; i < HD / 32; ++i) x[i] = *(const Piece*)(page[e] + G::BLOCK + (i * 64 + lane) * 8 * G::ESZ);
#pragma unroll
                for (int i = 0; i < HD / 32; ++i) *(halfx8*)(stay + e * STAY + (i * 64 + lane) * 16) = half_v(x[i], vs[e]);
            }
            load_k(x);
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(half_k(x[kk]), qf[kk], s, 0, 0, 0);
        } else {
            key0 = olo + (j - n_doc) * 32;
            exist = min(ohi - key0, 32);
            const int64_t token = a.ord[min(key0 + ln, ohi - 1)].x;
            const bf16_t *kp = (const bf16_t*)a.k + token * a.k_ts + h * a.k_hs, *vp = (const bf16_t*)a.v + token * a.v_ts + h * a.v_hs;
            halfx8 x[KC];
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) x[kk] = bf16x8_to_half(vp + 16 * kk + 8 * hh);
#pragma unroll
            for (int kk = 0; kk < KC; ++kk)
#pragma unroll
                for (int e = 0; e < 8; ++e) ((half_t*)(stay + (ln >> 4) * STAY))[v_elem(t, 16 * kk + 8 * hh + e, HD)] = x[kk][e];
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) x[kk] = bf16x8_to_half(kp + 16 * kk + 8 * hh);
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[kk], qf[kk], s, 0, 0, 0);
        }
        const float c0 = a.scale_log2 * ks[0], c1 = a.scale_log2 * ks[1];
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= r < 8 ? c0 : c1;
        if (EXTRA) pair_scores<false>(s, a, row, key0 - (doc ? row.pos : row.place), hh);
        const int lo = (doc ? row.dlo : row.olo) - key0, hi = (doc ? D : row.ohi) - key0;
        hide_keys(s, lo - 4 * hh, hi - 4 * hh);
        rescale(pair_softmax(sm, s));
        halfx8 pf[2];
        pack_p(s, pf, FP8 ? fp8_scale_mantissa(vs[0]) : 1.0f, FP8 ? fp8_scale_mantissa(vs[1]) : 1.0f);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");          // LDS accesses of a wavefront are done in order
        add_pv_masked<MB>(o, pf, lo, hi, exist, hh, [&](int mb, int e) { return *(const halfx8*)(stay + e * STAY + (hh * HD + mb * 32 + ln) * 16); },
                          [&](int key, int ch) { return ((const half_t*)(stay + (key >> 4) * STAY))[v_elem(key & 15, ch, HD)]; });
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    pair_join_waves<NW, HD, bf16_t>(a, smem, o, sm, row, h, pieces);
}

// ---- many rows
template <int HD, bool FP8, bool EXTRA>
__device__ __forceinline__ void pair_tile(const PairAttnArgs& a, char* smem, int4 rec, int rows, int h, int pieces) {
    using G = PairGeo<HD, FP8>;
    using T = TileGeo<HD>;
    constexpr int KC = G::KC, MB = G::MB, NW = kPairWaves;
    const int D = rec.y;
    const int lane = threadIdx.x & 63, ln = lane & 31, hh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const const_int_t pt = (const_int_t)(a.page_table + (int64_t)rec.x * a.pt_stride);
    const char* pool = a.pool + (int64_t)h * 2 * G::BLOCK;
    const int64_t page_stride = (int64_t)a.n_kv * 2 * G::BLOCK;
    const int last_page = (D - 1) / kPageTokens, last_row = min(rec.w + kPairTileRows, rows) - 1;

    // ---- the wavefront's block; without rows of its own it only brings pages
    const int first = rec.w + wave * 32;
    const bool active = first <= last_row;
    const PairRow row = pair_row(a, h, rec, rows, first + ln);
    const PairSpan mine = pair_span(a, row, rec, min(first, last_row), min(first + 31, last_row));
    PairSpan wg = pair_span(a, row, rec, rec.w, last_row);
    if (a.window > 0) {                                                 // the wavefronts' together
        int* range = (int*)smem;
        if (lane == 0) {
            range[wave] = mine.dlo;
            range[NW + wave] = mine.olo;
            range[2 * NW + wave] = mine.ohi;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            wg.dlo = min(wg.dlo, range[w]);
            wg.olo = min(wg.olo, range[NW + w]);
            wg.ohi = max(wg.ohi, range[2 * NW + w]);
        }
        wg.dlo = __builtin_amdgcn_readfirstlane(wg.dlo);
        wg.olo = __builtin_amdgcn_readfirstlane(wg.olo);
        wg.ohi = __builtin_amdgcn_readfirstlane(wg.ohi);
        __syncthreads();
    }
    // this piece's stages: the document's, then the own keys'
    const int doc0 = wg.dlo / kStageKeys, n_doc = wg.dlo < D ? (D + kStageKeys - 1) / kStageKeys - doc0 : 0;
    const int n_own = a.own_keys ? (wg.ohi - wg.olo + kStageKeys - 1) / kStageKeys : 0;
    const int share = (n_doc + n_own + pieces - 1) / pieces, u0 = (int)blockIdx.y * share, u1 = min(u0 + share, n_doc + n_own);
    const int j0 = doc0 + u0, j1 = doc0 + min(u1, n_doc);               // document stages

    // ---- a stage's K and V blocks, page after page, K first: a wavefront brings one page
    auto id_at = [&](int at) { return min(max(pt[min(at, last_page)], 0), a.num_pages - 1); };
    auto request = [&](int id, int buf) {                               // a half page, verbatim
        const char* src = pool + id * page_stride + lane * 16;
        char* dst = smem + buf * T::STAGE + wave * T::HPAGE;
#pragma unroll
        for (int e = 0; e < T::HPAGE / 1024; ++e)
            __builtin_amdgcn_global_load_lds((gbl_ptr_t)(src + e * 1024), (lds_ptr_t)(dst + e * 1024), 16, 0, 0);
    };
    constexpr int RAW = FP8 ? 2 * G::BLOCK / 512 : 1;                   // fp8: 8-byte words of a page that a lane has
    uint2 raw[RAW];
    auto fetch = [&](int id) {
        const char* src = pool + id * page_stride + lane * 8;
#pragma unroll
        for (int e = 0; e < RAW; ++e) raw[e] = *(const uint2*)(src + e * 512);
    };
    auto expand = [&](int buf, float v_scale) {
        char* dst = smem + buf * T::STAGE + wave * T::HPAGE;
#pragma unroll
        for (int e = 0; e < RAW; ++e) {
            const int w = (e % (RAW / 2)) * 64 + lane, t = w / (HD / 8), c8 = (w % (HD / 8)) ^ k_swizzle(t, HD, 1);
            if (e < RAW / 2) *(halfx8*)(dst + (t * HD + ((c8 ^ k_swizzle(t, HD, 2)) << 3)) * 2) = fp8x8_to_half(raw[e], fp8_expand_factor(1.0f));
            else *(halfx8*)(dst + T::HBLOCK + w * 16) = fp8x8_to_half(raw[e], fp8_expand_factor(v_scale));
        }
    };
    // What is needed of a stage's pages, asked for ahead of it: ids (the wavefront's own, fp8: all), and, fp8, the factors of its scores, and of its
    // probabilities what the expansion leaves of the V scales
    struct Ids { int own, all[FP8 ? kStagePages : 1]; };
    auto ids_of = [&](int stage) {
        Ids r;
        stage = min(stage, j1 - 1);                                     // behind the last stage its pages again, which nobody reads
        if constexpr (FP8) {
#pragma unroll
            for (int e = 0; e < kStagePages; ++e) r.all[e] = id_at(kStagePages * stage + e);
            r.own = pick(wave >= 2, pick(wave == 1, r.all[0], r.all[1]), pick(wave == 3, r.all[2], r.all[3]));
        } else {
            r.own = id_at(kStagePages * stage + wave);
        }
        return r;
    };
    struct Scales { float k[kStagePages], v[kStagePages]; };
    auto scales_of = [&](const Ids& ids) {
        Scales r;
#pragma unroll
        for (int e = 0; e < kStagePages; ++e) {
            r.k[e] = r.v[e] = 1.0f;
            if constexpr (FP8) {
                const const_float_t sc = (const_float_t)(a.scales + ((int64_t)ids.all[e] * a.n_kv + h) * 2);
                r.k[e] = sc[0];
                r.v[e] = sc[1];
            }
        }
        return r;
    };
    auto own_scale = [&](const Scales& s) { return pick(wave >= 2, pick(wave == 1, s.v[0], s.v[1]), pick(wave == 3, s.v[2], s.v[3])); };
    // own keys from place key0 on: a thread has one key and its wavefront's share of the channels
    auto own_stage = [&](int key0, int buf) {
        constexpr int CH = HD / NW;
        const int64_t token = a.ord[min(key0 + lane, wg.ohi - 1)].x;
        const bf16_t *kp = (const bf16_t*)a.k + token * a.k_ts + h * a.k_hs + wave * CH, *vp = (const bf16_t*)a.v + token * a.v_ts + h * a.v_hs + wave * CH;
        char* page = smem + buf * T::STAGE + (lane >> 4) * T::HPAGE;
        const int t = lane & 15;
        halfx8 kx[CH / 8], vx[CH / 8];
#pragma unroll
        for (int e = 0; e < CH / 8; ++e) {
            kx[e] = bf16x8_to_half(kp + e * 8);
            vx[e] = bf16x8_to_half(vp + e * 8);
        }
#pragma unroll
        for (int e = 0; e < CH / 8; ++e) {
            const int c = wave * CH + e * 8;
            *(halfx8*)(page + k_elem(t, c, HD, 2) * 2) = kx[e];
#pragma unroll
            for (int i = 0; i < 8; ++i) *(half_t*)(page + T::HBLOCK + v_elem(t, c + i, HD) * 2) = vx[e][i];
        }
    };

    // the first pages are on their way while the rows are read
    Ids ids;                          // of the stage that is asked for next
    Scales sc_now, sc_next;           // of this stage and the one behind it
    if (j0 < j1) {
        ids = ids_of(j0);
        if constexpr (FP8) fetch(ids.own);
        else request(ids.own, 0);
        sc_now = scales_of(ids);
        ids = ids_of(j0 + 1);
        sc_next = scales_of(ids);
    }
    halfx8 q[KC];
    load_q<HD>(a, row, h, hh, q);
    floatx16 o[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[mb] = floatx16{};
    PairSoftmax sm;

    // ---- sub: the first of a sub-tile's two pages in LDS
    auto k_frag = [&](const char* sub, int kk) {
        const int t = ln & 15;
        return *(const halfx8*)(sub + (ln >> 4) * T::HPAGE + (t * HD + (((2 * kk + hh) ^ k_swizzle(t, HD, 2)) << 3)) * 2);
    };
    auto v_frag = [&](const char* sub, int mb, int e) { return *(const halfx8*)(sub + e * T::HPAGE + T::HBLOCK + (hh * HD + mb * 32 + ln) * 16); };
    auto rescale = [&](float alpha) {
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) o[mb] *= alpha;
        }
    };
    constexpr bool SCALED = EXTRA || FP8;      // scores are scaled before they are compared
    constexpr int SUBS = HD == 64 || FP8 ? 1 : 2;     // sub-tiles at a time: at 64 channels a second one's scores would cost the fourth wavefront of a SIMD

    // SUBS sub-tiles that the wavefront's rows see whole, the stage's first-th and on
    auto whole = [&](const char* buf, int first, int key0, const Scales& sc) {
        floatx16 s[SUBS];
#pragma unroll
        for (int st = 0; st < SUBS; ++st) {
            const char* sub = buf + (first + st) * 2 * T::HPAGE;
            s[st] = floatx16{};
            halfx8 k[KC];
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) k[kk] = k_frag(sub, kk);
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) s[st] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[kk], q[kk], s[st], 0, 0, 0);
        }
        float mx = -INFINITY;
#pragma unroll
        for (int st = 0; st < SUBS; ++st) {
            const bool behind = first + st > 0;
            if (SCALED) {
                const float c0 = a.scale_log2 * pick(behind, sc.k[0], sc.k[2]), c1 = a.scale_log2 * pick(behind, sc.k[1], sc.k[3]);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[st][r] *= r < 8 ? c0 : c1;
            }
            if (EXTRA) pair_scores<false>(s[st], a, row, key0 + 32 * (first + st) - row.pos, hh);
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[st][r]);
        }
        const float c = SCALED ? 1.0f : a.scale_log2;
        const float alpha = sm.follow(row_max2(mx) * c), use = sm.used();
        rescale(alpha);
        float sum = 0.0f;
        halfx8 p[SUBS][2];
#pragma unroll
        for (int st = 0; st < SUBS; ++st) {
            const bool behind = first + st > 0;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[st][r] = __builtin_amdgcn_exp2f(fmaf(s[st][r], c, -use));
                sum += s[st][r];
            }
            pack_p(s[st], p[st], FP8 ? fp8_scale_mantissa(pick(behind, sc.v[0], sc.v[2])) : 1.0f, FP8 ? fp8_scale_mantissa(pick(behind, sc.v[1], sc.v[3])) : 1.0f);
        }
        sm.l = fmaf(sm.l, alpha, sum);
#pragma unroll
        for (int st = 0; st < SUBS; ++st)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v_frag(buf + (first + st) * 2 * T::HPAGE, mb, e), p[st][e], o[mb], 0, 0, 0);
    };
    // 32 keys at an edge: document keys from key0 on, or own keys from place key0 on; end: behind the last key there is
    auto edge = [&](const char* sub, bool doc, int key0, int end, float ks0, float ks1, float vs0, float vs1) {
        if (doc ? key0 + 32 <= mine.dlo : key0 + 32 <= mine.olo || key0 >= mine.ohi) return;      // seen by none of the rows
        floatx16 s = {};
#pragma unroll
        for (int kk = 0; kk < KC; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(k_frag(sub, kk), q[kk], s, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= a.scale_log2 * (r < 8 ? ks0 : ks1);
        if (EXTRA) pair_scores<false>(s, a, row, key0 - (doc ? row.pos : row.place), hh);
        const int lo = (doc ? row.dlo : row.olo) - key0, hi = (doc ? D : row.ohi) - key0;
        hide_keys(s, lo - 4 * hh, hi - 4 * hh);
        rescale(pair_softmax(sm, s));
        halfx8 pf[2];
        pack_p(s, pf, FP8 ? fp8_scale_mantissa(vs0) : 1.0f, FP8 ? fp8_scale_mantissa(vs1) : 1.0f);
        add_pv_masked<MB>(o, pf, lo, hi, min(end - key0, 32), hh, [&](int mb, int e) { return v_frag(sub, mb, e); },
                          [&](int key, int ch) { return ((const half_t*)(sub + (key >> 4) * T::HPAGE + T::HBLOCK))[v_elem(key & 15, ch, HD)]; });
    };

    // ---- own keys, in the second buffer, while the document's first pages come
    for (int u = max(u0, n_doc); u < u1; ++u) {
        const int key0 = wg.olo + (u - n_doc) * kStageKeys;
        own_stage(key0, 1);
        __syncthreads();
        if (active) {
#pragma unroll 1
            for (int st = 0; st < 2; ++st) edge(smem + T::STAGE + st * 2 * T::HPAGE, false, key0 + 32 * st, wg.ohi, 1.0f, 1.0f, 1.0f, 1.0f);
        }
        __syncthreads();
    }
    // ---- the document
    if (j0 < j1) {
        if constexpr (FP8) {
            expand(0, own_scale(sc_now));
            fetch(ids.own);
            ids = ids_of(j0 + 2);
        }
        for (int j = j0; j < j1; ++j) {
            const int buf = (j - j0) & 1;
            const char* at = smem + buf * T::STAGE;
            if constexpr (!FP8) __builtin_amdgcn_s_waitcnt(0x0F70);     // this wavefront's page has landed
            __syncthreads();                                            // everyone's has; and everyone is past the stage before
            Scales sc_after;
            if constexpr (FP8) {
                expand(buf ^ 1, own_scale(sc_next));
                fetch(ids.own);
                sc_after = scales_of(ids);
                ids = ids_of(j + 3);
            } else {
                request(ids.own, buf ^ 1);
                sc_after = sc_now;
                ids = ids_of(j + 2);
            }
            const int key0 = j * kStageKeys;
            if (active) {
                if (key0 >= mine.dlo_all && key0 + kStageKeys <= D) {
#pragma unroll 1
                    for (int st = 0; st < 2; st += SUBS) whole(at, st, key0, sc_now);
                } else {
#pragma unroll 1
                    for (int st = 0; st < 2; ++st)
                        if (key0 + 32 * st < D)
                            edge(at + st * 2 * T::HPAGE, true, key0 + 32 * st, D, pick(st, sc_now.k[0], sc_now.k[2]), pick(st, sc_now.k[1], sc_now.k[3]),
                                 pick(st, sc_now.v[0], sc_now.v[2]), pick(st, sc_now.v[1], sc_now.v[3]));
                }
            }
            sc_now = sc_next;
            sc_next = sc_after;
        }
    }
    // ---- out
    __builtin_amdgcn_s_waitcnt(0x0F70);                                 // nothing is on its way into LDS
    __syncthreads();
    if (!active) return;
    const float l = row_sum2(sm.l);
    const int head = h * a.g + row.head;
    const int64_t at = (int64_t)row.token * a.g * a.n_kv + head;
    if (pieces > 1) {
        if (!row.on) return;
        const int64_t part = (int64_t)blockIdx.y * a.part_rows + at;
        if (hh == 0) a.part_ml[part] = make_float2(sm.m, l);
        if (sm.m == -INFINITY) return;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(float4*)(a.part_o + part * HD + mb * 32 + 8 * (r >> 2) + 4 * hh) = make_float4(o[mb][r], o[mb][r + 1], o[mb][r + 2], o[mb][r + 3]);
        return;
    }
    // rows turned in LDS, so that a store writes whole pieces of rows
    char* turn = smem + wave * 32 * T::TURN;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    using W = __attribute__((ext_vector_type(4))) bf16_t;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            W y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (bf16_t)(o[mb][r + e] * inv);
            *(W*)(turn + ln * T::TURN + (mb * 32 + 8 * (r >> 2) + 4 * hh) * 2) = y;
        }
    if (row.on && hh == 0 && a.lse) a.lse[at] = sm.m == -INFINITY ? -INFINITY : (sm.m + __builtin_amdgcn_logf(l)) * kLn2;
    const int64_t out_at = row.on ? row.token * a.o_ts + head * a.o_hs : -1;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");              // LDS accesses of a wavefront are done in order
    constexpr int PIECES = HD / 8;                                      // 16-byte pieces of a row
#pragma unroll
    for (int e = 0; e < 32 * PIECES / 64; ++e) {
        const int u = e * 64 + lane, rw = u / PIECES, c = u % PIECES;
        const int64_t to = __shfl(out_at, rw, 64);
        using P8 = Loose<bf16_t, 8>;
        const auto x = *(const VecN<bf16_t, 8>*)(turn + rw * T::TURN + c * 16);
        if (to >= 0) *(P8*)((bf16_t*)a.out + to + c * 8) = P8{x};
    }
}

template <int HD, bool FP8, bool EXTRA>
__global__ void __launch_bounds__(kPairWaves * 64) __attribute__((amdgpu_waves_per_eu(HD == 64 ? 3 : 2, 8))) pair_attn_half_kernel(PairAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const const_int_t hdr = (const_int_t)a.hdr;
    const PairChoice ch = pair_choice(hdr[SH_BLOCKS] * a.n_kv, hdr[SH_TILES] * a.n_kv, HD, a.most_splits);
    const int item = item_of((int)blockIdx.x, (ch.tiles ? hdr[SH_TILES] : hdr[SH_BLOCKS]) * a.n_kv);
    if (item < 0 || (int)blockIdx.y >= ch.pieces) return;
    const int at = item / a.n_kv, h = item - at * a.n_kv;
    const const_int_t rp = (const_int_t)((ch.tiles ? a.rec_tiles : a.rec) + 2 * at);
    const int4 rec = make_int4(rp[0], rp[1], rp[2], rp[3]);
    if (ch.tiles) pair_tile<HD, FP8, EXTRA>(a, smem, rec, rp[4], h, ch.pieces);
    else pair_rows<HD, FP8, EXTRA>(a, (float*)smem, rec, rp[4], h, ch.pieces);
}

template <int HD, bool FP8, bool EXTRA>
hipError_t half_launch_as(const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    constexpr size_t lds = std::max<size_t>(TileGeo<HD>::LDS, pair_join_bytes(kPairWaves, HD));
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)pair_attn_half_kernel<HD, FP8, EXTRA>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    pair_attn_half_kernel<HD, FP8, EXTRA><<<grid, kPairWaves * 64, lds, st>>>(a);
    return hipGetLastError();
}
template <int HD, bool FP8>
hipError_t half_launch(const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    return pair_extra(a) ? half_launch_as<HD, FP8, true>(a, grid, st) : half_launch_as<HD, FP8, false>(a, grid, st);
}

}  // namespace

hipError_t launch_pair_half(bool fp8, const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    if (a.d == 64) return fp8 ? half_launch<64, true>(a, grid, st) : half_launch<64, false>(a, grid, st);
    return fp8 ? half_launch<128, true>(a, grid, st) : half_launch<128, false>(a, grid, st);
}

}  // namespace hr
