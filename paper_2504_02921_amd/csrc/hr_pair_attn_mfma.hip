// hr_pair_attention on the half matrix instructions: 16-bit and fp8 pools with heads of 64, 96 or 128 channels.
//
// A workgroup of four wavefronts goes about its work item in one of two ways; the device, which knows the items, chooses (pair_choice):
//   few rows   the item is one block of 32 rows, a wavefront has every fourth sub-tile of 32 keys and a softmax of its own, and they are joined
//              through LDS in a fixed order.  K and V go from memory straight into operand registers: V pages hold a channel's 8 keys as a lane
//              wants them, and a K instruction takes 32 bytes of each of 32 rows, whose lines the next ones take the rest of.  Bound by reading:
//              640 documents of 512 keys, one token, 64 channels, 41 us, 4.1 TB/s (31 us again and again, out of the last-level cache); 100 of
//              2048, 128 channels, fp8, 97 us, 4.3 TB/s (VALU 39 % busy, MFMA 11 %; a second sub-tile ahead, a third wavefront a SIMD and more pieces each measured slower).
//   many rows  the item is a tile of up to four blocks, one per wavefront, and keys go through LDS in a ring of four sub-tiles of 32, in the arrangement
//              of half pages: half pages straight from memory, fp8 pages by way of a wavefront's registers, which expands them once for all rows.
//              S of a sub-tile is computed next to the exponentials of the one before.  Bound by what a wavefront issues and, with 128 channels, by
//              power: 640 x 512 keys x 32 tokens, 64 channels, 81 us, 479 TFLOP/s; 400 x 2048 x 64, 128 channels, 1150 us, 758 TFLOP/s (MFMA 44 % of the
//              cycles of a clock that falls to 1.3 GHz), the same in fp8 1250 to 1280 us, 682 to 698 TFLOP/s (VALU 65 %, MFMA 33 %, 1.7 GHz).
//              Heads of 96 channels have no swizzle in their pages, and their K reads meet in banks: 640 x 512 x 32 155 us, 321 TFLOP/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "hr_kernels.h"
#include "hr_pair_half.h"
#include "hr_pair_launch.h"

namespace hr {

namespace {

constexpr int kPairWaves = 4;

// The ring of sub-tiles that tiles read: four slots of 32 keys, as half
template <int HD>
struct TileGeo {
    static constexpr int HBLOCK = kPageTokens * HD * 2, SLOT = 4 * HBLOCK;      // bytes
    static constexpr int LOADS = HBLOCK / 1024;   // of a wavefront for a block
    static constexpr int TURN = HD * 2 + 16;      // bytes between the rows of a block on its way out: they start at other banks
    static constexpr int LDS = std::max(4 * SLOT, kPairWaves * 32 * TURN);
};

// What rows of a group see together (row, row + 1, .. last of them), without asking each
struct PairSpan {
    int dlo, dlo_all;                 // document keys that some row sees begin at dlo, those that all see at dlo_all
    int olo, ohi;                     // own keys that some row sees, by place
};
// mine: the rows of this wavefront, one per lane of a half
__device__ __forceinline__ PairSpan pair_span(const PairAttnArgs& a, const PairRow& mine, const PairItem& it, int first, int last) {
    PairSpan s;
    if (a.window > 0) {
        s.dlo = rows_min(mine.dlo);
        s.dlo_all = rows_max(mine.dlo);
        s.olo = rows_min(mine.olo);
        s.ohi = rows_max(mine.ohi);
        return s;
    }
    // without a window: the first row's query from its first token, the last row's as far as that row sees
    const int t0 = pair_place(it, first, a.g, a.max_tokens).place, t1 = pair_place(it, last, a.g, a.max_tokens).place;
    const const_int_t f = (const_int_t)(a.ord + t0), l = (const_int_t)(a.ord + t1);
    s.dlo = s.dlo_all = 0;
    s.olo = min(max(f[1], 0), t0);
    s.ohi = t1 + 1;
    if (a.prefix) {
        const int pair = min(max(l[2], 0), a.n_pairs - 1);
        const const_int_t cu = (const_int_t)a.q_cu + pair;
        s.ohi = min(max(s.ohi, min(max(l[1], 0), t1) + pair_prefix(((const_int_t)a.prefix)[pair], cu[0], cu[1], a.max_tokens)), a.max_tokens);
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
template <int HD, bool FP8, int FORM>
__device__ __forceinline__ void pair_rows(const PairAttnArgs& a, float* smem, const PairItem& it, int h, int pieces) {
    using G = PairGeo<HD, FP8>;
    using Piece = typename G::Piece;
    constexpr int KC = G::KC, MB = G::MB, NW = kPairWaves;
    const int D = it.D;
    const int lane = threadIdx.x & 63, ln = lane & 31, hh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PairRow row = pair_row(a, h, it, it.row + ln);
    const const_int_t pt = (const_int_t)(a.page_table + (int64_t)it.pair * a.pt_stride);
    const char* pool = a.pool + (int64_t)h * 2 * G::BLOCK;
    const int64_t page_stride = (int64_t)a.n_kv * 2 * G::BLOCK;

    // The sub-tiles that some row of the block sees: document sub-tiles that all rows see whole, then those at an edge (the window's, the
    // document's end), then the pairs' own keys; and this piece's share of them
    const PairSpan span = pair_span(a, row, it, it.row, min(it.row + 32, it.rows) - 1);
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
                k_scale[e] = sc[0] * kFp8Low;
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
        if constexpr (FP8) return fp8x8_low(x);
        else return x;
    };
    auto half_v = [&](const Piece& x, float scale) {
        if constexpr (FP8) return fp8x8_times(x, fp8_expand_factor(scale));
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
            if (FORM) pair_scores<FORM>(s, a, row, (whole0 + j) * 32 - row.pos, hh);
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
            const int64_t token = own_token(a, min(key0 + ln, ohi - 1));
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
        if (FORM) pair_scores<FORM>(s, a, row, key0 - (doc ? row.pos : row.place), hh);
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
template <int HD, bool FP8, int FORM>
__device__ __forceinline__ void pair_tile(const PairAttnArgs& a, char* smem, const PairItem& it, int h, int pieces) {
    using G = PairGeo<HD, FP8>;
    using T = TileGeo<HD>;
    constexpr int KC = G::KC, MB = G::MB, NW = kPairWaves;
    const int D = it.D;
    const int lane = threadIdx.x & 63, ln = lane & 31, hh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t page_stride = (int64_t)a.n_kv * 2 * G::BLOCK;
    const int last_page = (D - 1) / kPageTokens, last_row = min(it.row + kPairTileRows, it.rows) - 1;

    // ---- the wavefront's block; without rows of its own it only brings pages
    const int first = it.row + wave * 32;
    const bool active = first <= last_row;
    const PairRow row = pair_row(a, h, it, first + ln);
    const PairSpan mine = pair_span(a, row, it, min(first, last_row), min(first + 31, last_row));
    PairSpan wg = pair_span(a, row, it, it.row, last_row);
    if (a.window > 0) {                                                 // the wavefronts' together
        int* range = (int*)smem;
        if (lane == 0) {
            range[wave] = mine.dlo;
            range[NW + wave] = mine.dlo_all;
            range[2 * NW + wave] = mine.olo;
            range[3 * NW + wave] = mine.ohi;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            wg.dlo = min(wg.dlo, range[w]);
            wg.dlo_all = max(wg.dlo_all, range[NW + w]);
            wg.olo = min(wg.olo, range[2 * NW + w]);
            wg.ohi = max(wg.ohi, range[3 * NW + w]);
        }
        wg.dlo = __builtin_amdgcn_readfirstlane(wg.dlo);
        wg.dlo_all = __builtin_amdgcn_readfirstlane(wg.dlo_all);
        wg.olo = __builtin_amdgcn_readfirstlane(wg.olo);
        wg.ohi = __builtin_amdgcn_readfirstlane(wg.ohi);
        __syncthreads();
    }
    // this piece's sub-tiles, in the order of pair_rows: whole ones, those at the window's edge, the document's last if it is not whole, own keys
    const int doc0 = wg.dlo / 32, doc1 = (D + 31) / 32, whole0 = (wg.dlo_all + 31) / 32, whole1 = max(D / 32, whole0);
    const int n_whole = whole1 - whole0, n_doc = max(doc1 - doc0, 0), n_own = a.own_keys ? (wg.ohi - wg.olo + 31) / 32 : 0;
    const int share = (n_doc + n_own + pieces - 1) / pieces, u0 = (int)blockIdx.y * share, u1 = min(u0 + share, n_doc + n_own);
    const int own0 = max(u0, n_doc);
    // those of the document go through the ring: n_ring of them, whole ones first
    const int n_ring = max(min(u1, n_doc) - u0, 0), n_ring_whole = max(min(u1, n_whole) - u0, 0);
    auto sub_of = [&](int at) {
        const int u = u0 + at;
        return u < n_whole ? whole0 + u : u - n_whole < whole0 - doc0 ? doc0 + u - n_whole : doc0 + u;
    };

    // ---- a sub-tile in the ring: K of its two pages, V of its two pages; wavefront w brings page w & 1's K (w < 2) or V
    const int my_page = wave & 1;
    const char* block0 = a.pool + ((int64_t)h * 2 + (wave >> 1)) * G::BLOCK;
    char* const my_part = smem + (wave >> 1) * 2 * T::HBLOCK + my_page * T::HBLOCK;
    auto request = [&](int id, int slot) {                              // a half block, verbatim
        const char* src = block0 + id * page_stride + lane * 16;
        char* dst = my_part + slot * T::SLOT;
#pragma unroll
        for (int e = 0; e < T::LOADS; ++e)
            __builtin_amdgcn_global_load_lds((gbl_ptr_t)(src + e * 1024), (lds_ptr_t)(dst + e * 1024), 16, 0, 0);
    };
    struct Raw { uint2 w[FP8 ? G::BLOCK / 512 : 1]; };                  // fp8: a block as it lies there
    auto fetch = [&](int id, Raw& r) {
        const char* src = block0 + id * page_stride + lane * 8;
#pragma unroll
        for (int e = 0; e < G::BLOCK / 512; ++e) r.w[e] = *(const uint2*)(src + e * 512);
    };
    auto expand = [&](const Raw& r, int slot, float v_scale) {
        char* dst = my_part + slot * T::SLOT;
        const halfx2 f = fp8_expand_factor(v_scale);                        // K's scale goes into the scores
#pragma unroll
        for (int e = 0; e < G::BLOCK / 512; ++e) {
            const int w = e * 64 + lane, t = w / (HD / 8), c8 = (w % (HD / 8)) ^ k_swizzle(t, HD, 1);
            if (wave < 2) *(halfx8*)(dst + (t * HD + ((c8 ^ k_swizzle(t, HD, 2)) << 3)) * 2) = fp8x8_low(r.w[e]);
            else *(halfx8*)(dst + w * 16) = fp8x8_times(r.w[e], f);
        }
    };
    // fp8: scales of a sub-tile's two pages
    struct Scales { float k0 = 1.0f, k1 = 1.0f, v0 = 1.0f, v1 = 1.0f; };      // half pages: one
    // The pages of the sub-tiles, a window of 32 sub-tiles that moves on by 16: a lane has the id and the scales of one page.  Lane reads cost the loop
    // no wait; requests through the scalar cache would share the counter of the LDS reads, and out of order, so that each of those waited for all.
    struct Pages { int id; float k, v; };
    const int lane_sub = lane >> 1;
    auto pages_of = [&](int at) {
        Pages r;
        const int sub = sub_of(min(at, n_ring - 1));                    // behind the last one that one's again
        r.id = min(max(a.page_table[(int64_t)it.pair * a.pt_stride + min(2 * sub + (lane & 1), last_page)], 0), a.num_pages - 1);
        return r;
    };
    auto scale_pages = [&](Pages& r) {
        if constexpr (FP8) {
            const float2 x = *(const float2*)(a.scales + ((int64_t)r.id * a.n_kv + h) * 2);
            r.k = x.x * kFp8Low;
            r.v = x.y;
        }
    };
    Pages pages, later;                                                 // the window, and what half of it becomes next
    auto lane_float = [&](float x, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l & 63)); };
    auto page_of = [&](int at) { return __builtin_amdgcn_readlane(pages.id, 2 * at + my_page & 63); };
    auto v_scale_of = [&](int at) { return FP8 ? lane_float(pages.v, 2 * at + my_page) : 1.0f; };
    auto scales_at = [&](int at) {
        Scales r;
        if constexpr (FP8) {
            r.k0 = lane_float(pages.k, 2 * at);
            r.k1 = lane_float(pages.k, 2 * at + 1);
            r.v0 = lane_float(pages.v, 2 * at);
            r.v1 = lane_float(pages.v, 2 * at + 1);
        }
        return r;
    };
    // 32 own keys from place key0 on: eight threads have a key, every eighth chunk of eight channels each
    constexpr int CHUNKS = HD / 8, MINE = (CHUNKS + 7) / 8;
    const int own_key = threadIdx.x & 31, own_c = threadIdx.x >> 5;
    struct Own { VecN<bf16_t, 8> k[MINE], v[MINE]; };
    auto load_own = [&](int key0, Own& x) {
        const int64_t token = own_token(a, min(key0 + own_key, wg.ohi - 1));
        const bf16_t *kp = (const bf16_t*)a.k + token * a.k_ts + h * a.k_hs, *vp = (const bf16_t*)a.v + token * a.v_ts + h * a.v_hs;
#pragma unroll
        for (int e = 0; e < MINE; ++e) {
            const int c = min(own_c + 8 * e, CHUNKS - 1) * 8;
            x.k[e] = ((const Loose<bf16_t, 8>*)(kp + c))->w;
            x.v[e] = ((const Loose<bf16_t, 8>*)(vp + c))->w;
        }
    };
    auto store_own = [&](const Own& x, int slot) {
        const int t = own_key & 15;
        half_t* dst = (half_t*)(smem + slot * T::SLOT + (own_key >> 4) * T::HBLOCK);
#pragma unroll
        for (int e = 0; e < MINE; ++e) {
            const int c = (own_c + 8 * e) * 8;
            if (c >= HD) break;
            *(halfx8*)(dst + k_elem(t, c, HD, 2)) = to_half8(x.k[e]);
            const halfx8 v = to_half8(x.v[e]);
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[T::HBLOCK + v_elem(t, c + i, HD)] = v[i];      // V two blocks on
        }
    };
    auto k_frag = [&](int slot, int kk) {
        const int t = ln & 15;
        return *(const halfx8*)(smem + slot * T::SLOT + (ln >> 4) * T::HBLOCK + (t * HD + (((2 * kk + hh) ^ k_swizzle(t, HD, 2)) << 3)) * 2);
    };
    auto v_frag = [&](int slot, int mb, int e) { return *(const halfx8*)(smem + slot * T::SLOT + (2 + e) * T::HBLOCK + (hh * HD + mb * 32 + ln) * 16); };

    // ---- the first sub-tiles are on their way while the rows are read.  Behind the last one that one's again, which nobody reads: what is asked for
    // does not hang on a branch.
    Raw raw[2];
    if (n_ring > 0) {
        pages = pages_of(lane_sub);
        scale_pages(pages);
        if constexpr (FP8) {
            fetch(page_of(0), raw[0]);
            fetch(page_of(1), raw[1]);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e) request(page_of(e), e);
        }
        later = pages_of(32 + (lane_sub & 15));
        scale_pages(later);
    }
    Own own;                                                            // needed behind the document
    if (own0 < u1) load_own(wg.olo + 32 * (own0 - n_doc), own);
    halfx8 q[KC];
    load_q<HD>(a, row, h, hh, q);
    floatx16 o[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[mb] = floatx16{};
    PairSoftmax sm;
    auto rescale = [&](float alpha) {
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) o[mb] *= alpha;
        }
    };

    // At the at-th sub-tile: everyone has the next one, and is past the one before, whose slot is free
    auto advance = [&](int at, int slot, Raw& r) {
        if constexpr (!FP8) __builtin_amdgcn_s_waitcnt(0x0F70 | T::LOADS);
        __syncthreads();
        if ((at & 15) == 0 && at > 0) {                                 // the half that is past
            const bool mine = lane_sub >> 4 == (at - 16 >> 4 & 1);
            pages.id = mine ? later.id : pages.id;
            if constexpr (FP8) {
                pages.k = mine ? later.k : pages.k;
                pages.v = mine ? later.v : pages.v;
            }
            later = pages_of(at + 32 + (lane_sub & 15));
        }
        if (FP8 && (at & 15) == 8 && at > 8) scale_pages(later);        // their ids are there
        if constexpr (FP8) {
            expand(r, (slot + 2) & 3, v_scale_of(at + 2));
            fetch(page_of(at + 4), r);
        } else {
            request(page_of(at + 3), (slot + 3) & 3);
        }
    };
    if (n_ring > 0) {
        if constexpr (FP8) {
            expand(raw[0], 0, v_scale_of(0));
            expand(raw[1], 1, v_scale_of(1));
            fetch(page_of(2), raw[0]);
            fetch(page_of(3), raw[1]);
        } else {
            __builtin_amdgcn_s_waitcnt(0x0F70);                         // the pages' numbers came behind the first blocks
        }
        __syncthreads();
    }
    // ---- whole sub-tiles.  S of one is computed next to the exponentials of the one before, and its maxima next to that one's V P: a wavefront issues in
    // order, and without the other's arithmetic between them it would wait 32 cycles for each of its matrix instructions
    if (n_ring_whole > 0) {
        floatx16 s = {};
        float mx = 0.0f;
        Scales c = scales_at(0);
        // the largest of a lane's raw scores, scaled where they are scaled later; FORM: scaled, capped and biased in place
        auto largest = [&](floatx16& x, int key0, const Scales& c) {
            if (FORM) {
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] *= a.scale_log2 * (r < 8 ? c.k0 : c.k1);
                pair_scores<FORM>(x, a, row, key0 - row.pos, hh);
            }
            float m0 = x[0], m1 = x[8];
#pragma unroll
            for (int r = 1; r < 8; ++r) {
                m0 = fmaxf(m0, x[r]);
                m1 = fmaxf(m1, x[8 + r]);
            }
            return FORM ? fmaxf(m0, m1) : FP8 ? fmaxf(m0 * (a.scale_log2 * c.k0), m1 * (a.scale_log2 * c.k1)) : fmaxf(m0, m1) * a.scale_log2;
        };
        // by = at & 3: known where it is called, so that a slot's place is part of the LDS instructions
        auto step = [&](int at, auto by, Raw& r) {
            constexpr int vs = decltype(by)::value, ks = (vs + 1) & 3;
            advance(at, vs, r);
            if (!active) return;
            const Scales cn = scales_at(at + 1);
            const float alpha = sm.follow(row_max2(mx)), use = sm.used();
            rescale(alpha);
            const float c0 = FORM ? 1.0f : a.scale_log2 * c.k0, c1 = FORM ? 1.0f : a.scale_log2 * c.k1;
            floatx16 sn = {};
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) sn = __builtin_amdgcn_mfma_f32_32x32x16_f16(k_frag(ks, kk), q[kk], sn, 0, 0, 0);
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], e < 8 ? c0 : c1, -use));
                sum += s[e];
            }
            sm.l = fmaf(sm.l, alpha, sum);
            halfx8 p[2];
            pack_p(s, p, FP8 ? fp8_scale_mantissa(c.v0) : 1.0f, FP8 ? fp8_scale_mantissa(c.v1) : 1.0f);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int e = 0; e < 2; ++e) o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v_frag(vs, mb, e), p[e], o[mb], 0, 0, 0);
            mx = largest(sn, 32 * (whole0 + u0 + at + 1), cn);
            s = sn;
            c = cn;
        };
        if (active) {
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(k_frag(0, kk), q[kk], s, 0, 0, 0);
            mx = largest(s, 32 * (whole0 + u0), c);
        }
        constexpr std::integral_constant<int, 0> s0{};
        constexpr std::integral_constant<int, 1> s1{};
        constexpr std::integral_constant<int, 2> s2{};
        constexpr std::integral_constant<int, 3> s3{};
        constexpr int odd = FP8 ? 1 : 0;
        int at = 0;
        for (; at + 3 < n_ring_whole; at += 4) {
            step(at, s0, raw[0]);
            step(at + 1, s1, raw[odd]);
            step(at + 2, s2, raw[0]);
            step(at + 3, s3, raw[odd]);
        }
        if (at < n_ring_whole) step(at, s0, raw[0]);
        if (at + 1 < n_ring_whole) step(at + 1, s1, raw[odd]);
        if (at + 2 < n_ring_whole) step(at + 2, s2, raw[0]);
    }
    // ---- sub-tiles at an edge, and own keys
#pragma unroll 1
    for (int u = u0 + n_ring_whole; u < u1; ++u) {
        const bool doc = u < n_doc;
        const int at = u - u0, slot = doc ? at & 3 : 0;
        const int key0 = 32 * (doc ? sub_of(at) : u - n_doc) + (doc ? 0 : wg.olo), end = doc ? D : wg.ohi;
        Scales c;
        if (doc) {
            if (FP8 && (at & 1)) advance(at, slot, raw[1]);
            else advance(at, slot, raw[0]);
            c = scales_at(at);
        } else {
            __builtin_amdgcn_s_waitcnt(0x0F70);                         // nothing is on its way into LDS
            __syncthreads();                                            // everyone is past the sub-tile before
            store_own(own, slot);
            if (u + 1 < u1) load_own(key0 + 32, own);
            __syncthreads();
        }
        if (!active || (doc ? key0 + 32 <= mine.dlo : key0 + 32 <= mine.olo || key0 >= mine.ohi)) continue;      // seen by none of the rows
        floatx16 s = {};
#pragma unroll
        for (int kk = 0; kk < KC; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(k_frag(slot, kk), q[kk], s, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= a.scale_log2 * (r < 8 ? c.k0 : c.k1);
        if (FORM) pair_scores<FORM>(s, a, row, key0 - (doc ? row.pos : row.place), hh);
        const int lo = (doc ? row.dlo : row.olo) - key0, hi = (doc ? D : row.ohi) - key0;
        hide_keys(s, lo - 4 * hh, hi - 4 * hh);
        rescale(pair_softmax(sm, s));
        halfx8 p[2];
        pack_p(s, p, FP8 ? fp8_scale_mantissa(c.v0) : 1.0f, FP8 ? fp8_scale_mantissa(c.v1) : 1.0f);
        add_pv_masked<MB>(o, p, lo, hi, min(end - key0, 32), hh, [&](int mb, int e) { return v_frag(slot, mb, e); },
                          [&](int key, int ch) { return ((const half_t*)(smem + slot * T::SLOT + (2 + (key >> 4)) * T::HBLOCK))[v_elem(key & 15, ch, HD)]; });
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
    if (row.on && hh == 0 && a.lse) a.lse[at] = pair_lse(sm.m, l);
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

template <int HD, bool FP8, int FORM>
__global__ void __launch_bounds__(kPairWaves * 64) __attribute__((amdgpu_waves_per_eu(HD == 64 ? 3 : 2, 8))) pair_attn_half_kernel(PairAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    // the item's record as either kind is asked for together with the counts that say which kind it is
    const int item = item_of((int)blockIdx.x, a.chunk), at = item / a.n_kv, h = item - at * a.n_kv;
    const PairItem block = list_item(a, false, at), tile = list_item(a, true, at);
    const int blocks = list_items(a, false), tiles = list_items(a, true);
    const PairChoice ch = pair_choice(blocks, tiles, HD, a.most_splits);
    if (item >= (ch.tiles ? tiles : blocks) || (int)blockIdx.y >= ch.pieces) return;
    const PairItem it = ch.tiles ? tile : block;
    if (ch.tiles) pair_tile<HD, FP8, FORM>(a, smem, it, h, ch.pieces);
    else pair_rows<HD, FP8, FORM>(a, (float*)smem, it, h, ch.pieces);
}

template <int HD, bool FP8, int FORM>
hipError_t half_launch_as(const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    constexpr size_t lds = std::max<size_t>(TileGeo<HD>::LDS, pair_join_bytes(kPairWaves, HD));
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)pair_attn_half_kernel<HD, FP8, FORM>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    pair_attn_half_kernel<HD, FP8, FORM><<<grid, kPairWaves * 64, lds, st>>>(a);
    return hipGetLastError();
}
template <int HD, bool FP8>
hipError_t half_launch(const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    switch (pair_scores_of(a)) {
        case PS_FACTOR: return half_launch_as<HD, FP8, PS_FACTOR>(a, grid, st);
        case PS_EXTRA: return half_launch_as<HD, FP8, PS_EXTRA>(a, grid, st);
        default: return half_launch_as<HD, FP8, PS_WIDE_CAP>(a, grid, st);
    }
}

}  // namespace

hipError_t launch_pair_half(bool fp8, const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    if (a.d == 64) return fp8 ? half_launch<64, true>(a, grid, st) : half_launch<64, false>(a, grid, st);
    if (a.d == 96) return fp8 ? half_launch<96, true>(a, grid, st) : half_launch<96, false>(a, grid, st);
    return fp8 ? half_launch<128, true>(a, grid, st) : half_launch<128, false>(a, grid, st);
}

}  // namespace hr
