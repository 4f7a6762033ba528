// hr_pair_attention on the half matrix instructions: 16-bit and fp8 pools with heads of 64 or 128 channels.
//
// Few rows (pair_rows_kernel): a workgroup takes one block of 32 rows of one kv head, its wavefronts every NW-th sub-tile of 32 keys, each with a
// softmax of its own; they are joined through LDS in a fixed order.  K and V go from memory straight into operand registers: V pages hold
// a channel's 8 keys as a lane wants them, and a K instruction takes 32 bytes of each of 32 rows, whose lines the next ones take the rest of.
// K of the next sub-tile is requested when S is there, V when O is.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "hr_kernels.h"
#include "hr_pair_attn.h"
#include "hr_pair_launch.h"

namespace hr {

namespace {

typedef const __attribute__((address_space(4))) int32_t* const_int_t;       // read through the scalar cache: uniform, written by an earlier launch
typedef const __attribute__((address_space(4))) float* const_float_t;

template <int HD, bool FP8>
struct PairGeo {
    static constexpr int KC = HD / 16, MB = HD / 32;
    static constexpr int ESZ = FP8 ? 1 : 2;
    static constexpr int BLOCK = kPageTokens * HD * ESZ;      // bytes of a K or V block
    using Piece = std::conditional_t<FP8, uint2, halfx8>;     // 8 elements of a page
};

__device__ __forceinline__ halfx8 bf16x8_to_half(const bf16_t* p) {
    const Loose<bf16_t, 8> x = *(const Loose<bf16_t, 8>*)p;
    halfx8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (half_t)(float)x.w[e];       // beyond the half range: infinity
    return r;
}

// the lane's 16 probabilities as the B operands of two products over 16 keys each
__device__ __forceinline__ void pack_p(const floatx16& s, halfx8 (&pf)[2], float f0, float f1) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const halfx2 x = __builtin_convertvector(floatx2{s[e] * f0, s[e + 1] * f0}, halfx2);
        const halfx2 y = __builtin_convertvector(floatx2{s[8 + e] * f1, s[9 + e] * f1}, halfx2);
        pf[0][e] = x[0]; pf[0][e + 1] = x[1];
        pf[1][e] = y[0]; pf[1][e + 1] = y[1];
    }
}

// Which of the lane's 16 keys of a sub-tile are in [lo, hi), relative to the lane's first
__device__ __forceinline__ unsigned hide_keys(floatx16& s, int lo, int hi) {
    unsigned seen = 0xFFFFu;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int key = 8 * (r >> 2) + (r & 3);
        const bool on = key >= lo && key < hi;
        s[r] = on ? s[r] : -INFINITY;
        seen = on ? seen : seen & ~(1u << r);
    }
    return seen;
}

// O^T += V^T P^T over a sub-tile that not every row sees whole.  A hidden key's V counts for nothing, whatever it holds, and 0 times infinity is
// not nothing: finite values go through the product, the others are counted where they are seen, as ones.  exist: keys that there are.
template <int MB>
__device__ __forceinline__ void add_pv_masked(floatx16 (&o)[MB], halfx8 (&vf)[MB][2], const halfx8 (&pf)[2], unsigned seen, int exist, int hh) {
    bool odd = false;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const half_t v = 8 * (e >> 2) + (e & 3) + 4 * hh < exist ? vf[mb][e >> 3][e & 7] : (half_t)0.0f;
            vf[mb][e >> 3][e & 7] = v;
            odd = odd || !(__builtin_fabsf16(v) < (half_t)INFINITY);
        }
    if (__any(odd)) {
        // counted kind by kind (rare: as few registers as may be)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
#pragma unroll 1
            for (int kind = 0; kind < 3; ++kind) {                      // infinities of either sign, NaN
                floatx16 n = {};
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2) {
                    halfx8 x, p;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const half_t v = vf[mb][s2][e];
                        const bool is = kind == 2 ? v != v : v == (half_t)(kind == 0 ? INFINITY : -INFINITY);
                        x[e] = (half_t)(is ? 1.0f : 0.0f);
                        p[e] = (half_t)(seen >> (8 * s2 + e) & 1 ? 1.0f : 0.0f);
                    }
                    n = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, p, n, 0, 0, 0);
                }
                const float add = kind == 2 ? NAN : kind == 0 ? INFINITY : -INFINITY;
#pragma unroll
                for (int r = 0; r < 16; ++r) o[mb][r] += n[r] > 0.0f ? add : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const half_t v = vf[mb][e >> 3][e & 7];
                vf[mb][e >> 3][e & 7] = __builtin_fabsf16(v) < (half_t)INFINITY ? v : (half_t)0.0f;
            }
        }
    }
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[mb][0], pf[0], o[mb], 0, 0, 0);
        o[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[mb][1], pf[1], o[mb], 0, 0, 0);
    }
}

template <int HD, bool FP8, bool EXTRA, int NW>
__global__ void __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(HD == 64 ? 4 : 2, 8))) pair_rows_kernel(PairAttnArgs a) {
    using G = PairGeo<HD, FP8>;
    constexpr int KC = G::KC, MB = G::MB, LD = HD + 4;
    extern __shared__ __attribute__((aligned(16))) float smem[];        // [wave][row][channels, and 4 more so that rows start at other banks]
    const int items = ((const_int_t)a.hdr)[SH_BLOCKS] * a.n_kv;
    const int item = item_of((int)blockIdx.x, items);
    const int pieces = pair_splits(items, a.most_splits);
    if (item < 0 || (int)blockIdx.y >= pieces) return;
    const int blk = item / a.n_kv, h = item - blk * a.n_kv;
    const const_int_t rp = (const_int_t)(a.rec + 2 * blk);
    const int4 rec = make_int4(rp[0], rp[1], rp[2], rp[3]);
    const int rows = rp[4], D = rec.y;
    const int lane = threadIdx.x & 63, ln = lane & 31, hh = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PairRow row = pair_row(a, h, rec, rows, rec.w + ln);
    const const_int_t pt = (const_int_t)(a.page_table + (int64_t)rec.x * a.pt_stride);
    const char* pool = a.pool + (int64_t)h * 2 * G::BLOCK;
    const int64_t page_stride = (int64_t)a.n_kv * 2 * G::BLOCK;

    halfx8 qf[KC];                                                      // lane: row ln, channels 16 kk + 8 hh ..
    {
        const bf16_t* qr = (const bf16_t*)a.q + row.token * a.q_ts + (h * a.g + row.head) * a.q_hs;
#pragma unroll
        for (int kk = 0; kk < KC; ++kk) qf[kk] = bf16x8_to_half(qr + 16 * kk + 8 * hh);
    }
    // The sub-tiles that some row of the block sees: document sub-tiles that all rows see whole, then those at an edge (the window's, the
    // document's end), then the pairs' own keys; and this piece's share of them
    const int dlo = rows_min(row.dlo), dlo_all = rows_max(row.dlo), olo = rows_min(row.olo), ohi = rows_max(row.ohi);
    const int doc0 = dlo / 32, doc1 = (D + 31) / 32, whole0 = (dlo_all + 31) / 32, whole1 = max(D / 32, whole0);
    const int n_whole = whole1 - whole0, n_doc = max(doc1 - doc0, 0), n_own = a.own_keys ? (ohi - olo + 31) / 32 : 0;
    const int n_sub = n_doc + n_own, share = (n_sub + pieces - 1) / pieces;
    const int j0 = (int)blockIdx.y * share, j1 = min(j0 + share, n_sub);
    const int last_page = (D - 1) / kPageTokens;

    floatx16 o[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[mb] = floatx16{};
    PairSoftmax sm;

    // a sub-tile's pages, and its K and V as they lie there; a lane's key is ln: page ln >> 4, token ln & 15
    using Piece = typename G::Piece;
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
    if (j < jw) {
        Piece kr[KC], vr[MB][2];
        float ks[2] = {1.0f, 1.0f}, vs[2] = {1.0f, 1.0f}, vs_next[2] = {1.0f, 1.0f};
        find(whole0 + j, ks, vs);
        load_k(kr);
        load_v(vr);
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
        halfx8 kf[KC], vf[MB][2];
        int key0, exist;
        if (doc) {
            const int sub = j - n_whole < whole0 - doc0 ? doc0 + j - n_whole : doc0 + j;        // the edge in front, the edge behind
            key0 = 32 * sub;
            exist = D - key0;
            Piece kr[KC], vr[MB][2];
            find(sub, ks, vs);
            load_k(kr);
            load_v(vr);
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) kf[kk] = half_k(kr[kk]);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int e = 0; e < 2; ++e) vf[mb][e] = half_v(vr[mb][e], vs[e]);
        } else {
            key0 = olo + (j - n_doc) * 32;
            exist = ohi - key0;
            const int64_t token = a.ord[min(key0 + ln, ohi - 1)].x;
            const bf16_t *kp = (const bf16_t*)a.k + token * a.k_ts + h * a.k_hs, *vp = (const bf16_t*)a.v + token * a.v_ts + h * a.v_hs;
            halfx8 vt[KC];
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) vt[kk] = bf16x8_to_half(vp + 16 * kk + 8 * hh);
#pragma unroll
            for (int kk = 0; kk < KC; ++kk) kf[kk] = bf16x8_to_half(kp + 16 * kk + 8 * hh);
            // V is turned in the wavefront's part of LDS, into the arrangement of two pages' V blocks
            half_t* turn = (half_t*)(smem + wave * 32 * LD);
#pragma unroll
            for (int kk = 0; kk < KC; ++kk)
#pragma unroll
                for (int e = 0; e < 8; ++e) turn[(ln >> 4) * kPageTokens * HD + v_elem(t, 16 * kk + 8 * hh + e, HD)] = vt[kk][e];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // LDS accesses of a wavefront are done in order
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int e = 0; e < 2; ++e) vf[mb][e] = *(const halfx8*)(turn + e * kPageTokens * HD + (hh * HD + mb * 32 + ln) * 8);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        floatx16 s = {};
#pragma unroll
        for (int kk = 0; kk < KC; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[kk], qf[kk], s, 0, 0, 0);
        const float c0 = a.scale_log2 * ks[0], c1 = a.scale_log2 * ks[1];
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= r < 8 ? c0 : c1;
        if (EXTRA) pair_scores<false>(s, a, row, key0 - (doc ? row.pos : row.place), hh);
        const unsigned seen = hide_keys(s, (doc ? row.dlo : row.olo) - key0 - 4 * hh, (doc ? D : row.ohi) - key0 - 4 * hh);
        rescale(pair_softmax(sm, s));
        halfx8 pf[2];
        pack_p(s, pf, FP8 ? fp8_scale_mantissa(vs[0]) : 1.0f, FP8 ? fp8_scale_mantissa(vs[1]) : 1.0f);
        add_pv_masked<MB>(o, vf, pf, seen, exist, hh);
    }
    pair_join_waves<NW, HD, bf16_t>(a, smem, o, sm, row, h, pieces);
}

template <int HD, bool FP8, bool EXTRA, int NW>
hipError_t rows_launch_as(const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    const size_t lds = pair_join_bytes(NW, HD);
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)pair_rows_kernel<HD, FP8, EXTRA, NW>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    pair_rows_kernel<HD, FP8, EXTRA, NW><<<grid, NW * 64, lds, st>>>(a);
    return hipGetLastError();
}

// EXTRA: scores are capped or biased
template <int HD, bool FP8>
hipError_t rows_launch(const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    if (a.cap_in != 0.0f || a.slopes) return rows_launch_as<HD, FP8, true, 8>(a, grid, st);
    return rows_launch_as<HD, FP8, false, 8>(a, grid, st);
}

}  // namespace

hipError_t launch_pair_rows(bool fp8, const PairAttnArgs& a, dim3 grid, hipStream_t st) {
    if (a.d == 64) return fp8 ? rows_launch<64, true>(a, grid, st) : rows_launch<64, false>(a, grid, st);
    return fp8 ? rows_launch<128, true>(a, grid, st) : rows_launch<128, false>(a, grid, st);
}

}  // namespace hr
