// The tables of a batch of pairs, built on the device from the pairs' documents and query lengths (hr_pair_tables_build).
//
// Two parts.  What goes over all pairs in turn (offsets, the stable order by document, groups, their row blocks) is a few passes of scans of
// one workgroup: a launch of many would wait at a grid barrier for each of them, and the passes are short (a pair is 8 bytes).  What is written
// per pair, token and block goes to as many workgroups as there is work for; a small batch has the one workgroup do that too, in the same launch.
// The order is a radix sort of 8 bits a pass, least first, each wavefront with a run of its own: equal documents keep the pairs' order, and no
// result depends on which wavefront is first.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "hr_kernels.h"
#include "hr_pair.h"

namespace hr {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kDigits = 256;

struct TablesArgs {
    const int32_t *pair_doc, *query_lens;
    const int32_t *list_lens, *list_cu, *list_pages;      // hr_doc_list
    int32_t n_docs, n_list_pages, num_pages;
    int32_t n_pairs, max_tokens, pt_stride, g;
    int32_t *q_cu, *doc_lens, *page_table, *tok_pos, *tok_pair, *order, *report;
    int32_t* sched;
    SchedLayout lay;
    int32_t passes;                                       // of the sort
};

struct Shared {
    unsigned scan[2][kWaves];
    unsigned carry[2];
    int unsorted, bits;
    unsigned count[kWaves][kDigits];
};

// exclusive sum over the workgroup of values whose sums saturate at `cap` (at most 2^30 + 2^30 meets before the cap is applied); total: of all
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned cap, unsigned* s, unsigned& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned inc = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned up = __shfl_up(inc, o, 64);
        if (lane >= o) inc = min(inc + up, cap);
    }
    __syncthreads();                                      // the last scan's sums have been read
    if (lane == 63) s[wave] = inc;
    __syncthreads();
    unsigned before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) before = all;
        all = min(all + s[w], cap);
    }
    total = all;
    const unsigned ex = __shfl_up(inc, 1, 64);
    return min(before + (lane == 0 ? 0u : ex), cap);
}

__device__ __forceinline__ int key_of(const TablesArgs& a, int doc) { return doc < 0 || doc >= a.n_docs ? 0 : doc + 1; }

struct Doc { int first, len, bits; };                     // place in the page list, tokens, what was wrong
__device__ __forceinline__ Doc doc_of(const TablesArgs& a, int doc) {
    Doc r{0, 0, 0};
    if (doc < 0 || doc >= a.n_docs) {
        r.bits = doc == -1 ? 0 : HR_TABLES_BAD_DOC;
        return r;
    }
    const int lo = min(max(a.list_cu[doc], 0), a.n_list_pages), hi = min(max(a.list_cu[doc + 1], lo), a.n_list_pages);
    const int len = a.list_lens[doc];
    const int64_t room = (int64_t)min(hi - lo, a.pt_stride) * kPageTokens;
    r.first = lo;
    r.len = len < 0 ? 0 : (int)min((int64_t)len, room);
    r.bits = r.len != len ? HR_TABLES_CUT : 0;
    return r;
}

constexpr int kPer = 4;                                   // consecutive pairs of a thread in a scan

// Everything that goes over the pairs in turn.  One workgroup.
__device__ void tables_scan(const TablesArgs& a, Shared& sh) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_pairs;
    int32_t* const S = a.sched;
    if (tid == 0) {
        sh.unsorted = 0;
        sh.bits = 0;
        a.q_cu[0] = 0;
    }
    // offsets of the queries; are the pairs in the documents' order as they stand?
    unsigned carry = 0;
    int bits = 0, unsorted = 0;
    const unsigned cap = (unsigned)a.max_tokens + 1;      // the first sum past max_tokens is told from the last that fits
    for (int base = 0; base < n; base += kThreads * kPer) {
        unsigned q[kPer], sum = 0;
        const int p0 = base + tid * kPer;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int p = p0 + e;
            int len = p < n ? a.query_lens[p] : 0;
            if (len < 0) bits |= HR_TABLES_BAD_LENGTH;
            q[e] = (unsigned)min(max(len, 0), a.max_tokens + 1);
            sum = min(sum + q[e], cap);
            if (p < n && p > 0) unsorted |= key_of(a, a.pair_doc[p]) < key_of(a, a.pair_doc[p - 1]);
        }
        unsigned total;
        unsigned at = min(carry + block_scan(sum, cap, sh.scan[0], total), cap);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            at = min(at + q[e], cap);
            if (at == cap) bits |= HR_TABLES_BAD_LENGTH;
            if (p0 + e < n) a.q_cu[p0 + e + 1] = (int)min(at, (unsigned)a.max_tokens);
        }
        carry = min(carry + total, cap);
    }
    if (bits) atomicOr(&sh.bits, bits);
    if (unsorted) atomicOr(&sh.unsorted, 1);
    __syncthreads();
    const int tokens = (int)min(carry, (unsigned)a.max_tokens);

    // order by document
    int32_t *key = S + a.lay.key[0], *key2 = S + a.lay.key[1], *idx = S + a.lay.idx;
    if (!sh.unsorted) {
        for (int p = tid; p < n; p += kThreads) {
            a.order[p] = p;
            key[p] = key_of(a, a.pair_doc[p]);
        }
    } else {
        const int run = ((n + kWaves - 1) / kWaves + 63) / 64 * 64;      // a wavefront's pairs
        const int lo = min(wave * run, n), hi = min(lo + run, n);
        for (int pass = 0; pass < a.passes; ++pass) {
            // the last pass writes `order` and key
            const bool even = (a.passes - 1 - pass) % 2 == 0;
            int32_t *ki = even ? key2 : key, *ko = even ? key : key2, *xi = even ? idx : a.order, *xo = even ? a.order : idx;
            const int shift = 8 * pass;
            for (int i = tid; i < kWaves * kDigits; i += kThreads) (&sh.count[0][0])[i] = 0;
            __syncthreads();
            for (int i = lo + lane; i < hi; i += 64) {
                const int k = pass == 0 ? key_of(a, a.pair_doc[i]) : ki[i];
                atomicAdd(&sh.count[wave][(k >> shift) & (kDigits - 1)], 1u);      // a count: the order of the additions does not show
            }
            __syncthreads();
            // first place of every digit of every wavefront: digits in turn, in a digit the wavefronts in turn
            unsigned c[kPer], sum = 0;
            static_assert(kWaves * kDigits == kThreads * kPer, "a thread scans kPer counts");
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int i = tid * kPer + e;
                c[e] = sh.count[i % kWaves][i / kWaves];
                sum += c[e];
            }
            unsigned total, at = block_scan(sum, 0xFFFFFFFFu, sh.scan[0], total);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int i = tid * kPer + e;
                sh.count[i % kWaves][i / kWaves] = at;
                at += c[e];
            }
            __syncthreads();
            for (int i0 = lo; i0 < hi; i0 += 64) {
                const int i = i0 + lane;
                const bool on = i < hi;
                const int k = on ? pass == 0 ? key_of(a, a.pair_doc[i]) : ki[i] : 0, x = on ? pass == 0 ? i : xi[i] : 0;
                const unsigned digit = (unsigned)(k >> shift) & (kDigits - 1);
                uint64_t same = __ballot(on);
#pragma unroll
                for (int b = 0; b < 8; ++b) {
                    const uint64_t has = __ballot(digit >> b & 1);
                    same &= digit >> b & 1 ? has : ~has;
                }
                const unsigned rank = __popcll(same & (((uint64_t)1 << lane) - 1));
                const unsigned first = sh.count[wave][digit];
                // every lane has its place before one of them moves it on, and sees that in the next step
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                if (on && rank == 0) sh.count[wave][digit] = first + (unsigned)__popcll(same);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                if (on) {
                    ko[first + rank] = k;
                    xo[first + rank] = x;
                }
            }
            __syncthreads();
        }
    }
    __syncthreads();

    // groups: pairs of one document
    unsigned tok_carry = 0, grp_carry = 0;
    for (int base = 0; base < n; base += kThreads * kPer) {
        const int i0 = base + tid * kPer;
        unsigned q[kPer], qs = 0, gs = 0;
        int p[kPer];
        bool head[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int i = i0 + e;
            p[e] = i < n ? a.order[i] : 0;
            q[e] = i < n ? (unsigned)(a.q_cu[p[e] + 1] - a.q_cu[p[e]]) : 0u;
            head[e] = i < n && (i == 0 || key[i] != key[i - 1]);
            qs += q[e];
            gs += head[e] ? 1u : 0u;
        }
        unsigned q_all, g_all;
        unsigned t = tok_carry + block_scan(qs, 0xFFFFFFFFu, sh.scan[0], q_all), g = grp_carry + block_scan(gs, 0xFFFFFFFFu, sh.scan[1], g_all);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (i0 + e >= n) break;
            S[a.lay.ord_first + p[e]] = (int)t;
            if (head[e]) {
                S[a.lay.grp_pair + g] = i0 + e;
                S[a.lay.grp_tok + g] = (int)t;
                ++g;
            }
            t += q[e];
        }
        tok_carry += q_all;
        grp_carry += g_all;
    }
    const int groups = (int)grp_carry;
    if (tid == 0) {
        S[a.lay.grp_pair + groups] = n;
        S[a.lay.grp_tok + groups] = tokens;
    }
    __syncthreads();

    // row blocks of the groups
    unsigned b_carry = 0, t_carry = 0;
    for (int base = 0; base < groups; base += kThreads * kPer) {
        const int g0 = base + tid * kPer;
        unsigned b[kPer], t[kPer], bs = 0, ts = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int gi = g0 + e;
            const int rows = gi < groups ? (S[a.lay.grp_tok + gi + 1] - S[a.lay.grp_tok + gi]) * a.g : 0;
            b[e] = (unsigned)(rows + kPairBlkRows - 1) / kPairBlkRows;
            t[e] = (unsigned)(rows + kPairTileRows - 1) / kPairTileRows;
            bs += b[e];
            ts += t[e];
        }
        unsigned b_all, t_all;
        unsigned bo = b_carry + block_scan(bs, 0xFFFFFFFFu, sh.scan[0], b_all), to = t_carry + block_scan(ts, 0xFFFFFFFFu, sh.scan[1], t_all);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (g0 + e >= groups) break;
            S[a.lay.blk_cu + g0 + e] = (int)bo;
            S[a.lay.tile_cu + g0 + e] = (int)to;
            bo += b[e];
            to += t[e];
        }
        b_carry += b_all;
        t_carry += t_all;
    }
    if (tid == 0) {
        S[a.lay.blk_cu + groups] = (int)b_carry;
        S[a.lay.tile_cu + groups] = (int)t_carry;
        int32_t* hdr = S + a.lay.hdr;
        hdr[SH_TOKENS] = tokens;
        hdr[SH_GROUPS] = groups;
        hdr[SH_BLOCKS] = (int)b_carry;
        hdr[SH_TILES] = (int)t_carry;
        a.report[0] = tokens;
        a.report[1] = groups;
        a.report[2] = sh.bits;
        a.report[3] = 0;
    }
    __syncthreads();
}

// What belongs to single pairs, tokens and blocks, by `threads` threads (whole wavefronts)
__device__ void tables_fill(const TablesArgs& a, int64_t tid, int64_t threads) {
    int32_t* const S = a.sched;
    const int lane = (int)(tid & 63);
    const int tokens = S[a.lay.hdr + SH_TOKENS], groups = S[a.lay.hdr + SH_GROUPS];
    int bits = 0;
    for (int64_t p = tid / 64; p < a.n_pairs; p += threads / 64) {
        const Doc d = doc_of(a, a.pair_doc[p]);
        bits |= d.bits;
        if (lane == 0) a.doc_lens[p] = d.len;
        const int n_pages = (d.len + kPageTokens - 1) / kPageTokens;
        int32_t* row = a.page_table + p * a.pt_stride;
        for (int j = lane; j < a.pt_stride; j += 64) {
            int id = -1;
            if (j < n_pages) {
                id = a.list_pages[d.first + j];
                if (id < 0 || id >= a.num_pages) {
                    id = -1;
                    bits |= HR_TABLES_BAD_PAGE;
                }
            }
            row[j] = id;
        }
        const int t0 = a.q_cu[p], n = a.q_cu[p + 1] - t0, first = S[a.lay.ord_first + p];
        int4* ord = (int4*)(S + a.lay.ord) + first;
        for (int i = lane; i < n; i += 64) {
            a.tok_pos[t0 + i] = d.len + i;
            a.tok_pair[t0 + i] = (int)p;
            ord[i] = make_int4(t0 + i, first, (int)p, d.len);
        }
    }
    for (int64_t t = tokens + tid; t < a.max_tokens; t += threads) {
        a.tok_pos[t] = -1;
        a.tok_pair[t] = -1;
    }
    // a block's group: the last one that begins at or before it
    auto records = [&](int64_t cu_at, int64_t rec_at, int n, int unit) {
        const int32_t* cu = S + cu_at;
        for (int64_t b = tid; b < n; b += threads) {
            int lo = 0, hi = groups;                      // cu[lo] <= b < cu[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (cu[mid] <= b) lo = mid;
                else hi = mid;
            }
            const int pair = a.order[S[a.lay.grp_pair + lo]], tok = S[a.lay.grp_tok + lo];
            int4* rec = (int4*)(S + rec_at) + 2 * b;
            rec[0] = make_int4(pair, doc_of(a, a.pair_doc[pair]).len, tok, (int)(b - cu[lo]) * unit);
            rec[1] = make_int4((S[a.lay.grp_tok + lo + 1] - tok) * a.g, 0, 0, 0);
        }
    };
    records(a.lay.blk_cu, a.lay.blk, S[a.lay.hdr + SH_BLOCKS], kPairBlkRows);
    records(a.lay.tile_cu, a.lay.tile, S[a.lay.hdr + SH_TILES], kPairTileRows);
    if (bits) atomicOr(&a.report[2], bits);
}

__global__ void __launch_bounds__(kThreads) tables_scan_kernel(TablesArgs a, int with_fill) {
    __shared__ Shared sh;
    tables_scan(a, sh);
    if (with_fill) tables_fill(a, threadIdx.x, kThreads);
}
__global__ void __launch_bounds__(256) tables_fill_kernel(TablesArgs a) {
    tables_fill(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

}  // namespace

hipError_t launch_pair_tables(const hr_pool* pool, const hr_doc_list* docs, const int32_t* pair_doc, const int32_t* query_lens,
                              const hr_pair_tables* t, hipStream_t st) {
    TablesArgs a{};
    a.pair_doc = pair_doc;
    a.query_lens = query_lens;
    a.list_lens = docs->doc_lens;
    a.list_cu = docs->page_cu;
    a.list_pages = docs->pages;
    a.n_docs = docs->n_docs;
    a.n_list_pages = docs->n_pages;
    a.num_pages = pool->cfg.num_pages;
    a.n_pairs = t->n_pairs;
    a.max_tokens = t->max_tokens;
    a.pt_stride = t->pt_stride;
    a.g = t->n_q_heads / pool->cfg.n_kv_heads;
    a.q_cu = t->q_cu;
    a.doc_lens = t->doc_lens;
    a.page_table = t->page_table;
    a.tok_pos = t->tok_pos;
    a.tok_pair = t->tok_pair;
    a.order = t->order;
    a.report = t->report;
    a.sched = (int32_t*)t->sched;
    a.lay = make_sched_layout(t->n_pairs, t->max_tokens, a.g);
    while (a.passes < 4 && (int64_t)docs->n_docs >> (8 * a.passes)) ++a.passes;      // keys are 0 .. n_docs
    if (a.passes == 0) a.passes = 1;
    // entries written; one workgroup writes a few thousand in the time of a launch
    const int64_t work = (int64_t)t->n_pairs * (t->pt_stride + 64) + t->max_tokens;
    const bool one = work <= 16384;
    tables_scan_kernel<<<1, kThreads, 0, st>>>(a, one ? 1 : 0);
    if (!one) {
        const int64_t blocks = std::min<int64_t>((std::max<int64_t>(t->n_pairs * 64, t->max_tokens) + 255) / 256, 2048);
        tables_fill_kernel<<<(unsigned)blocks, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace hr
