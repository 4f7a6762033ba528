// The tables of a batch of pairs, built on the device from the pairs' documents and query lengths (hr_pair_tables_build).
//
// Three ways; no result depends on which wavefront is first.
//   small    one workgroup, a thread a pair, everything that one step hands to the next in LDS: what it costs is the loads that depend on each other
//            (document, its place in the list, its pages).  20 pairs 6 us on the device, 200 of 4 tokens 18.0 (256, the second way: 20.0).
//   sorted   one workgroup goes over the pairs in turn (offsets, a stable radix sort by document of up to 8 bits a pass, least first, each wavefront
//            with a run of its own, groups, row blocks): passes of scans, which are short (a pair is 8 bytes).  Many workgroups, with a
//            launch or a grid barrier for each pass, have not been measured.  What is written per pair, token and block goes to the whole chip in a second launch.
//   counted  many pairs: that workgroup only counts the pairs and tokens of every document, kWindow of them at a time in LDS, which gives groups and
//            row blocks; the order of the pairs, most of the sort's time, is found by many workgroups (tables_place_kernel).
// Sorted / counted, in us: 4096 pairs over 1000 documents 33.9 / 34.4, 8192 over 1000 43.6 / 36.7, 25600 over 8192 129 / 65 (counts 30, places 18,
// what is written, 21 MB, 17); windows cost a look at the pairs each: 4096 over 30000 37 / 55, 16384 over 40000 94 / 77, 60000 over 200000 337 / 372.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "hr_kernels.h"
#include "hr_pair.h"

namespace hr {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kDigits = 256;
constexpr int kChipWaves = 8192;                          // wavefronts that the chip holds; more pairs than that share them, four at a time (25600: 19.7 to 17 us)
constexpr int kSmallPairs = 256, kSmallWork = 16384;      // of a small batch; work: entries written
constexpr int kWindow = 16384, kWindowPairs = 5000;       // documents that are counted in LDS at a time, and the pairs for which that pays
constexpr int kCountPairs = 65535;                        // pairs and groups share a word there
constexpr int kPlacePairs = 128;                          // pairs whose groups begin in a workgroup's share of the order

struct TablesArgs {
    const int32_t *pair_doc, *query_lens;
    const int32_t *list_lens, *list_cu, *list_pages;      // hr_doc_list
    int32_t n_docs, n_list_pages, num_pages;
    int32_t n_pairs, max_tokens, pt_stride, g;
    int32_t *q_cu, *doc_lens, *page_table, *tok_pos, *tok_pair, *order, *report;
    int32_t* sched;
    SchedLayout lay;
    int32_t passes, bits;                                 // of the sort: passes, bits of a digit
    int32_t wide;                                         // log2 of the lanes that write a pair
};

struct Shared {
    unsigned scan[4][kWaves];
    int unsorted, bits;
    unsigned count[kWaves][kDigits];
};

// a lane's value of the lane before it; the first lane has `first`
__device__ __forceinline__ int lane_before(int v, int first) { return __builtin_amdgcn_update_dpp(first, v, 0x138, 0xf, 0xf, false); }
__device__ __forceinline__ int lane_last(int v) { return __builtin_amdgcn_readlane(v, 63); }

// inclusive sum over the wavefront, saturating at `cap`: in rows of 16 lanes, then over the rows
__device__ __forceinline__ unsigned wave_scan(unsigned v, unsigned cap) {
    v = min(v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false), cap);
    v = min(v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false), cap);
    v = min(v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false), cap);
    v = min(v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false), cap);
    v = min(v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false), cap);
    return min(v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false), cap);
}

// exclusive sums over the workgroup of PER values a thread, of NV kinds, saturating at `cap` (at most 2^30 + 2^30 meets before the cap is applied);
// total: of all.  A wavefront's 64 PER values stand together, 64 beside each other, so that what they come from is read in whole lines.
template <int NV, int PER>
__device__ __forceinline__ void block_scan(const unsigned (&v)[NV][PER], unsigned (&ex)[NV][PER], unsigned cap, unsigned (*s)[kWaves],
                                           unsigned (&total)[NV]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned carry[NV] = {};
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const unsigned inc = wave_scan(v[n][e], cap);
            ex[n][e] = min(carry[n] + (unsigned)lane_before((int)inc, 0), cap);
            carry[n] = min(carry[n] + (unsigned)lane_last((int)inc), cap);
        }
    __syncthreads();                                      // the last scan's sums have been read
    if (lane == 0) {
#pragma unroll
        for (int n = 0; n < NV; ++n) s[n][wave] = carry[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const unsigned inc = wave_scan(lane < kWaves ? s[n][lane] : 0u, cap);
        const unsigned before = wave == 0 ? 0u : (unsigned)__builtin_amdgcn_readlane((int)inc, wave - 1);
        total[n] = (unsigned)lane_last((int)inc);
#pragma unroll
        for (int e = 0; e < PER; ++e) ex[n][e] = min(before + ex[n][e], cap);
    }
}
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned cap, unsigned (*s)[kWaves], unsigned& total) {
    const unsigned one[1][1] = {{v}};
    unsigned ex[1][1], all[1];
    block_scan(one, ex, cap, s, all);
    total = all[0];
    return ex[0][0];
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

constexpr int kPer = 8;                                   // pairs of a thread in a scan

struct __attribute__((packed, aligned(4))) Ends { int lo, hi; };      // of a pair's queries, in one load

// the lanes whose digit is this lane's, among those that are on
__device__ __forceinline__ uint64_t same_digit(unsigned digit, int bits, bool on) {
    uint64_t same = __ballot(on);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        if (b == bits) break;
        const int mine = (int)(digit << (31 - b)) >> 31;      // the bit, 32 times
        const uint64_t has = __ballot(mine);
        same &= ~(has ^ ((uint64_t)(unsigned)mine << 32 | (unsigned)mine));
    }
    return same;
}

// counts per wavefront and digit become first places: digits in turn, in a digit the wavefronts in turn
__device__ __forceinline__ void digit_places(Shared& sh) {
    constexpr int PER = kWaves * kDigits / kThreads;
    unsigned c[PER], sum = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int i = threadIdx.x * PER + e;
        c[e] = sh.count[i % kWaves][i / kWaves];
        sum += c[e];
    }
    unsigned total, at = block_scan(sum, 0xFFFFFFFFu, sh.scan, total);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int i = threadIdx.x * PER + e;
        sh.count[i % kWaves][i / kWaves] = at;
        at += c[e];
    }
    __syncthreads();
}

// place of this lane's element in the sorted order; the wavefront's next elements of that digit come behind it
__device__ __forceinline__ unsigned take_place(unsigned* count, unsigned digit, int bits, bool on) {
    const uint64_t same = same_digit(digit, bits, on);
    const unsigned rank = __popcll(same & (((uint64_t)1 << (threadIdx.x & 63)) - 1)), first = count[digit];
    // every lane has its place before one of them moves it on, and sees that in the next step
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (on && rank == 0) count[digit] = first + (unsigned)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return first + rank;
}

__device__ __forceinline__ void clear_counts(Shared& sh) {
    for (int i = threadIdx.x; i < kWaves * kDigits; i += kThreads) (&sh.count[0][0])[i] = 0;
    __syncthreads();
}

// put(i, get(i)) for i = first, first + step, .. below n, with the loads of eight at a time in flight: get sees clamped places, without a branch
template <typename Get, typename Put>
__device__ __forceinline__ void stream(int first, int step, int n, Get get, Put put) {
    constexpr int AHEAD = 8;
    for (int i0 = first; i0 < n; i0 += step * AHEAD) {
        decltype(get(0)) v[AHEAD];
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) v[e] = get(min(i0 + step * e, n - 1));
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            if (i0 + step * e < n) put(i0 + step * e, v[e]);
        }
    }
}

// The pairs in the documents' order: keys in key[0], pairs in `order`
__device__ void sort_memory(const TablesArgs& a, Shared& sh) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_pairs;
    int32_t *key = a.sched + a.lay.key[0], *key2 = a.sched + a.lay.key[1], *idx = a.sched + a.lay.idx;
    if (!sh.unsorted) {
        for (int p = tid; p < n; p += kThreads) {
            a.order[p] = p;
            key[p] = key_of(a, a.pair_doc[p]);
        }
        __syncthreads();
        return;
    }
    const int run = ((n + kWaves - 1) / kWaves + 63) / 64 * 64;      // a wavefront's pairs
    const int lo = min(wave * run, n), hi = min(lo + run, n);
    for (int pass = 0; pass < a.passes; ++pass) {
        // the last pass writes `order` and key
        const bool even = (a.passes - 1 - pass) % 2 == 0;
        int32_t *ki = even ? key2 : key, *ko = even ? key : key2, *xi = even ? idx : a.order, *xo = even ? a.order : idx;
        const int shift = a.bits * pass;
        const unsigned mask = (1u << a.bits) - 1;
        clear_counts(sh);
        for (int i = lo + lane; i < hi; i += 64) {
            const int k = pass == 0 ? key_of(a, a.pair_doc[i]) : ki[i];
            atomicAdd(&sh.count[wave][((unsigned)k >> shift) & mask], 1u);      // a count: the order of the additions does not show
        }
        __syncthreads();
        digit_places(sh);
        for (int i0 = lo; i0 < hi; i0 += 64) {
            const int i = i0 + lane;
            const bool on = i < hi;
            const int k = on ? pass == 0 ? key_of(a, a.pair_doc[i]) : ki[i] : 0, x = on ? pass == 0 ? i : xi[i] : 0;
            const unsigned at = take_place(sh.count[wave], ((unsigned)k >> shift) & mask, a.bits, on);
            if (on) {
                ko[at] = k;
                xo[at] = x;
            }
        }
        __syncthreads();
    }
}

// Offsets of the queries; the tokens.  unsorted: whether the pairs are not in the documents' order as they stand
__device__ int tables_offsets(const TablesArgs& a, Shared& sh) {
    constexpr int PER = 2 * kPer;                         // fewer rounds of loads
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_pairs;
    if (tid == 0) {
        sh.unsorted = 0;
        sh.bits = 0;
        a.q_cu[0] = 0;
    }
    unsigned carry = 0;
    int bits = 0, unsorted = 0;
    const unsigned cap = (unsigned)a.max_tokens + 1;      // the first sum past max_tokens is told from the last that fits
    for (int base = 0; base < n; base += kThreads * PER) {
        unsigned q[1][PER], at[1][PER], total[1];
        const int p0 = base + wave * 64 * PER + lane;
        int len[PER], doc[PER];                         // clamped places: loads without a branch between them
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            len[e] = a.query_lens[min(p0 + 64 * e, n - 1)];
            doc[e] = a.pair_doc[min(p0 + 64 * e, n - 1)];
        }
        int k0 = key_of(a, a.pair_doc[min(max(p0 - 1, 0), n - 1)]);      // of the pair before, in a run's first lane
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const bool on = p0 + 64 * e < n;
            const int k = key_of(a, doc[e]), up = lane_before(k, k0);
            q[0][e] = on ? (unsigned)min(max(len[e], 0), a.max_tokens + 1) : 0u;
            if (on && len[e] < 0) bits |= HR_TABLES_BAD_LENGTH;
            unsorted |= on && k < up;
            k0 = lane_last(k);
        }
        block_scan(q, at, cap, sh.scan, total);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const unsigned end = min(min(carry + at[0][e], cap) + q[0][e], cap);
            if (end == cap) bits |= HR_TABLES_BAD_LENGTH;
            if (p0 + 64 * e < n) a.q_cu[p0 + 64 * e + 1] = (int)min(end, (unsigned)a.max_tokens);
        }
        carry = min(carry + total[0], cap);
    }
    if (bits) atomicOr(&sh.bits, bits);
    if (unsorted) atomicOr(&sh.unsorted, 1);
    __syncthreads();
    return (int)min(carry, (unsigned)a.max_tokens);
}

__device__ __forceinline__ int blocks_of(int rows) { return (rows + kPairBlkRows - 1) / kPairBlkRows; }
__device__ __forceinline__ int tiles_of(int rows) { return (rows + kPairTileRows - 1) / kPairTileRows; }

// What is written once: the lists' ends, header and report
__device__ __forceinline__ void tables_close(const TablesArgs& a, int bits, int tokens, int groups, int blocks, int tiles) {
    int32_t* const S = a.sched;
    S[a.lay.grp_pair + groups] = a.n_pairs;
    S[a.lay.grp_tok + groups] = tokens;
    S[a.lay.blk_cu + groups] = blocks;
    S[a.lay.tile_cu + groups] = tiles;
    int32_t* hdr = S + a.lay.hdr;
    hdr[SH_TOKENS] = tokens;
    hdr[SH_GROUPS] = groups;
    hdr[SH_BLOCKS] = blocks;
    hdr[SH_TILES] = tiles;
    a.report[0] = tokens;
    a.report[1] = groups;
    a.report[2] = bits;
    a.report[3] = 0;
}

// Offsets, the pairs sorted, groups and their row blocks.  One workgroup.
__global__ void __launch_bounds__(kThreads) tables_sort_kernel(TablesArgs a) {
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_pairs;
    int32_t* const S = a.sched;
    const int tokens = tables_offsets(a, sh);
    sort_memory(a, sh);
    const int32_t* key = S + a.lay.key[0];
    // groups: pairs of one document
    unsigned tok_carry = 0, grp_carry = 0;
    for (int base = 0; base < n; base += kThreads * kPer) {
        const int i0 = base + wave * 64 * kPer + lane;
        unsigned v[2][kPer], ex[2][kPer], all[2];         // tokens, heads of groups
        Ends ends[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int i = min(i0 + 64 * e, n - 1);
            ends[e] = *(const Ends*)(a.q_cu + a.order[i]);
            v[1][e] = (i == 0) | (key[i] != key[max(i - 1, 0)]) ? 1u : 0u;
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const bool on = i0 + 64 * e < n;
            v[0][e] = on ? (unsigned)(ends[e].hi - ends[e].lo) : 0u;
            v[1][e] = on ? v[1][e] : 0u;
        }
        block_scan(v, ex, 0xFFFFFFFFu, sh.scan, all);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int i = i0 + 64 * e;
            if (i >= n) break;
            S[a.lay.ord_first + i] = (int)(tok_carry + ex[0][e]);
            if (v[1][e]) {
                S[a.lay.grp_pair + grp_carry + ex[1][e]] = i;
                S[a.lay.grp_tok + grp_carry + ex[1][e]] = (int)(tok_carry + ex[0][e]);
            }
        }
        tok_carry += all[0];
        grp_carry += all[1];
    }
    const int groups = (int)grp_carry;
    if (tid == 0) S[a.lay.grp_tok + groups] = tokens;
    __syncthreads();
    // row blocks of the groups
    unsigned b_carry = 0, t_carry = 0;
    for (int base = 0; base < groups; base += kThreads * kPer) {
        const int g0 = base + wave * 64 * kPer + lane;
        unsigned v[2][kPer], ex[2][kPer], all[2];
        Ends ends[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) ends[e] = *(const Ends*)(S + a.lay.grp_tok + min(g0 + 64 * e, groups - 1));
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int rows = g0 + 64 * e < groups ? (ends[e].hi - ends[e].lo) * a.g : 0;
            v[0][e] = (unsigned)blocks_of(rows);
            v[1][e] = (unsigned)tiles_of(rows);
        }
        block_scan(v, ex, 0xFFFFFFFFu, sh.scan, all);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (g0 + 64 * e >= groups) break;
            S[a.lay.blk_cu + g0 + 64 * e] = (int)(b_carry + ex[0][e]);
            S[a.lay.tile_cu + g0 + 64 * e] = (int)(t_carry + ex[1][e]);
        }
        b_carry += all[0];
        t_carry += all[1];
    }
    if (tid == 0) tables_close(a, sh.bits, tokens, groups, (int)b_carry, (int)t_carry);
}

// The same from counts: pairs and tokens of every document, kWindow documents at a time in LDS, give groups and row blocks without an order of the
// pairs, which many workgroups then find (tables_place_kernel).  One workgroup.
__global__ void __launch_bounds__(kThreads) tables_count_kernel(TablesArgs a) {
    __shared__ Shared sh;
    extern __shared__ unsigned counts[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_pairs, n_keys = a.n_docs + 1, width = min(n_keys, kWindow);
    unsigned *pairs = counts, *toks = counts + width;
    int32_t* const S = a.sched;
    const int tokens = tables_offsets(a, sh);
    unsigned pair_carry = 0, tok_carry = 0, b_carry = 0, t_carry = 0;      // pair_carry: groups in the upper half
    if (tid == 0) S[a.lay.idx] = 0;
    for (int first = 0; first < n_keys; first += kWindow) {
        for (int i = tid; i < width; i += kThreads) pairs[i] = toks[i] = 0;
        __syncthreads();
        struct Pair { int doc; Ends ends; };
        stream(tid, kThreads, n, [&](int p) { return Pair{a.pair_doc[p], *(const Ends*)(a.q_cu + p)}; }, [&](int, const Pair& x) {
            const int k = key_of(a, x.doc) - first;
            if (k < 0 || k >= width) return;
            atomicAdd(&pairs[k], 1u);                     // counts: the order of the additions does not show
            atomicAdd(&toks[k], (unsigned)(x.ends.hi - x.ends.lo));
        });
        __syncthreads();
        for (int base = 0; base < width; base += kThreads * kPer) {
            const int k0 = base + wave * 64 * kPer + lane;
            unsigned v[4][kPer], ex[4][kPer], all[4];     // pairs and groups, tokens, blocks, tiles
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int k = min(k0 + 64 * e, width - 1);
                const bool on = k0 + 64 * e < width && first + k < n_keys;
                const unsigned c = on ? pairs[k] : 0u, t = on ? toks[k] : 0u;
                v[0][e] = c | (c ? 1u << 16 : 0u);
                v[1][e] = t;
                v[2][e] = (unsigned)blocks_of((int)t * a.g);
                v[3][e] = (unsigned)tiles_of((int)t * a.g);
            }
            block_scan(v, ex, 0xFFFFFFFFu, sh.scan, all);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int c = (int)(v[0][e] & 0xFFFFu);
                if (c == 0) continue;
                const unsigned both = pair_carry + ex[0][e];
                const int g = (int)(both >> 16), p = (int)(both & 0xFFFFu);
                S[a.lay.grp_pair + g] = p;
                S[a.lay.grp_tok + g] = (int)(tok_carry + ex[1][e]);
                S[a.lay.blk_cu + g] = (int)(b_carry + ex[2][e]);
                S[a.lay.tile_cu + g] = (int)(t_carry + ex[3][e]);
                S[a.lay.key[0] + g] = first + k0 + 64 * e;
                for (int m = p / kPlacePairs + 1; m <= (p + c) / kPlacePairs; ++m) S[a.lay.idx + m] = g + 1;      // the first group from there on
            }
            pair_carry += all[0];
            tok_carry += all[1];
            b_carry += all[2];
            t_carry += all[3];
        }
        __syncthreads();                                  // counts have been read
    }
    if (tid == 0) tables_close(a, sh.bits, tokens, (int)(pair_carry >> 16), (int)b_carry, (int)t_carry);
}

// The pairs' places in the order, and their first tokens': a workgroup has the groups that begin in its kPlacePairs places and looks through all pairs
// for theirs.  They are ranked by counting.  If the last of these groups, the only one that may be long, is longer than kPlacePairs, its pairs are taken
// one behind the other instead, in a second look: they are of one document.
__global__ void __launch_bounds__(kThreads) tables_place_kernel(TablesArgs a) {
    constexpr int MOST = 2 * kPlacePairs, AHEAD = 16, EACH = kThreads / MOST;
    __shared__ int list_key[kWaves][MOST], list_pair[kWaves][MOST], list_len[kWaves][MOST];
    __shared__ int key[MOST], pair[MOST], len[MOST];
    __shared__ int wave_few[kWaves], wave_last[kWaves], wave_tok[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_pairs, w = blockIdx.x;
    int32_t* const S = a.sched;
    const int groups = S[a.lay.hdr + SH_GROUPS];
    const int g0 = min(S[a.lay.idx + w], groups), g1 = (int64_t)(w + 1) * kPlacePairs > n ? groups : min(S[a.lay.idx + w + 1], groups);
    if (g0 >= g1) return;
    const int key_lo = S[a.lay.key[0] + g0], key_last = S[a.lay.key[0] + g1 - 1];
    const int place0 = S[a.lay.grp_pair + g0], place_last = S[a.lay.grp_pair + g1 - 1], place1 = S[a.lay.grp_pair + g1];
    const int tok0 = S[a.lay.grp_tok + g0], tok_last = S[a.lay.grp_tok + g1 - 1];
    const bool is_long = place1 - place_last > kPlacePairs;
    const int key_hi = key_last + (is_long ? 0 : 1);      // keys that are ranked: below it
    const int run = (n + kThreads - 1) / kThreads * 64, lo = min(wave * run, n), hi = min(lo + run, n);      // a wavefront's pairs
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    int few = 0, last = 0, toks = 0;
    auto look = [&](auto each) {                          // each(pair, key or -1, tokens), for 64 pairs beside each other
        for (int i0 = lo; i0 < hi; i0 += 64 * AHEAD) {
            int doc[AHEAD];
            Ends ends[AHEAD];
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const int i = min(i0 + 64 * e + lane, n - 1);
                doc[e] = a.pair_doc[i];
                ends[e] = *(const Ends*)(a.q_cu + i);
            }
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const int i = i0 + 64 * e + lane;
                each(i, i < hi ? key_of(a, doc[e]) : -1, ends[e].hi - ends[e].lo);
            }
        }
    };
    look([&](int i, int k, int tokens) {
        const bool is_few = k >= key_lo && k < key_hi;
        const uint64_t f = __ballot(is_few);
        if (f) {
            const int at = few + (int)__popcll(f & below);
            if (is_few && at < MOST) {
                list_key[wave][at] = k;
                list_pair[wave][at] = i;
                list_len[wave][at] = tokens;
            }
            few += (int)__popcll(f);
        }
        if (is_long) {
            const uint64_t l = __ballot(k == key_last);
            last += (int)__popcll(l);
            if (l) toks += lane_last((int)wave_scan(k == key_last ? (unsigned)tokens : 0u, 0xFFFFFFFFu));
        }
    });
    if (lane == 0) {
        wave_few[wave] = min(few, MOST);
        wave_last[wave] = last;
        wave_tok[wave] = toks;
    }
    __syncthreads();
    int at0 = 0, m = 0;
    last = place_last;
    toks = tok_last;
    for (int v = 0; v < kWaves; ++v) {
        if (v < wave) {
            at0 += wave_few[v];
            last += wave_last[v];
            toks += wave_tok[v];
        }
        m += wave_few[v];
    }
    m = min(m, MOST);
    for (int i = lane; i < wave_few[wave] && at0 + i < MOST; i += 64) {
        key[at0 + i] = list_key[wave][i];
        pair[at0 + i] = list_pair[wave][i];
        len[at0 + i] = list_len[wave][i];
    }
    __syncthreads();
    const int mine = tid / EACH;
    int before = 0, tok = 0;
    if (mine < m) {
        const int k = key[mine];
        for (int j = tid % EACH; j < m; j += EACH) {
            const bool is = key[j] < k || (key[j] == k && j < mine);
            before += is ? 1 : 0;
            tok += is ? len[j] : 0;
        }
    }
#pragma unroll
    for (int o = 1; o < EACH; o <<= 1) {
        before += __shfl_xor(before, o, 64);
        tok += __shfl_xor(tok, o, 64);
    }
    if (mine < m && tid % EACH == 0 && place0 + before < n) {
        a.order[place0 + before] = pair[mine];
        S[a.lay.ord_first + place0 + before] = tok0 + tok;
    }
    if (!is_long) return;
    look([&](int i, int k, int tokens) {
        const bool is_last = k == key_last;
        const uint64_t l = __ballot(is_last);
        if (!l) return;
        const int inc = (int)wave_scan(is_last ? (unsigned)tokens : 0u, 0xFFFFFFFFu), at = last + (int)__popcll(l & below);
        if (is_last && at < n) {
            a.order[at] = i;
            S[a.lay.ord_first + at] = toks + inc - tokens;
        }
        last += (int)__popcll(l);
        toks += lane_last(inc);
    });
}

// What the parts that write pairs, tokens and blocks take from the part before them, from memory or LDS
struct Found {
    const int32_t *q_cu, *order, *ord_first, *grp_pair, *grp_tok, *blk_cu, *tile_cu;
    int tokens, groups, blocks, tiles;
};

// What belongs to single pairs, tokens and blocks, by `threads` threads (whole wavefronts); what was wrong with them
__device__ __forceinline__ int tables_fill(const TablesArgs& a, const Found& f, int64_t tid, int64_t threads) {
    int32_t* const S = a.sched;
    const int wide = 1 << a.wide, lane = (int)tid & (wide - 1);
    int bits = 0;
    for (int64_t i = tid >> a.wide; i < a.n_pairs; i += threads >> a.wide) {
        const int p = f.order[i];
        const Doc d = doc_of(a, a.pair_doc[p]);
        bits |= d.bits;
        if (lane == 0) a.doc_lens[p] = d.len;
        const int n_pages = (d.len + kPageTokens - 1) / kPageTokens;
        int32_t* row = a.page_table + (int64_t)p * a.pt_stride;
        for (int j = lane; j < a.pt_stride; j += wide) {
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
        const int t0 = f.q_cu[p], n = f.q_cu[p + 1] - t0, first = f.ord_first[i];
        int4* ord = (int4*)(S + a.lay.ord) + first;
        for (int k = lane; k < n; k += wide) {
            a.tok_pos[t0 + k] = d.len + k;
            a.tok_pair[t0 + k] = p;
            ord[k] = make_int4(t0 + k, first, p, d.len);
        }
    }
    for (int64_t t = f.tokens + tid; t < a.max_tokens; t += threads) {
        a.tok_pos[t] = -1;
        a.tok_pair[t] = -1;
    }
    // a block's group: the last one that begins at or before it
    auto records = [&](const int32_t* cu, int64_t rec_at, int n, int unit) {
        for (int64_t b = tid; b < n; b += threads) {
            int lo = 0, hi = f.groups;                    // cu[lo] <= b < cu[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (cu[mid] <= b) lo = mid;
                else hi = mid;
            }
            const int pair = f.order[f.grp_pair[lo]], tok = f.grp_tok[lo];
            int4* rec = (int4*)(S + rec_at) + 2 * b;
            rec[0] = make_int4(pair, doc_of(a, a.pair_doc[pair]).len, tok, (int)(b - cu[lo]) * unit);
            rec[1] = make_int4((f.grp_tok[lo + 1] - tok) * a.g, 0, 0, 0);
        }
    };
    records(f.blk_cu, a.lay.blk, f.blocks, kPairBlkRows);
    records(f.tile_cu, a.lay.tile, f.tiles, kPairTileRows);
    return bits;
}

__global__ void __launch_bounds__(256) tables_fill_kernel(TablesArgs a) {
    const int32_t* S = a.sched;
    const int32_t* hdr = S + a.lay.hdr;
    const Found f{a.q_cu, a.order, S + a.lay.ord_first, S + a.lay.grp_pair, S + a.lay.grp_tok, S + a.lay.blk_cu, S + a.lay.tile_cu,
                  hdr[SH_TOKENS], hdr[SH_GROUPS], hdr[SH_BLOCKS], hdr[SH_TILES]};
    const int bits = tables_fill(a, f, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
    if (bits) atomicOr(&a.report[2], bits);
}

struct SmallShared {
    unsigned scan[2][kWaves];
    int bits;
    int key[kSmallPairs];
    int q_cu[kSmallPairs + 1], order[kSmallPairs], ord_first[kSmallPairs];
    int grp_pair[kSmallPairs + 1], grp_tok[kSmallPairs + 1], blk_cu[kSmallPairs + 1], tile_cu[kSmallPairs + 1];
};

// A small batch: a thread a pair.  The order comes from counting, for every pair, those before it.
__global__ void __launch_bounds__(kThreads) tables_small_kernel(TablesArgs a) {
    __shared__ SmallShared s;
    static_assert(kSmallPairs * 4 == kThreads, "four threads count for a pair");
    const int tid = threadIdx.x, n = a.n_pairs;
    if (tid == 0) {
        s.bits = 0;
        s.q_cu[0] = 0;
        a.q_cu[0] = 0;
    }
    int bits = 0;
    const unsigned cap = (unsigned)a.max_tokens + 1;
    const int len = tid < n ? a.query_lens[tid] : 0;
    if (tid < n) s.key[tid] = key_of(a, a.pair_doc[tid]);
    const unsigned q = (unsigned)min(max(len, 0), a.max_tokens + 1);
    unsigned total;
    const unsigned end = min(block_scan(q, cap, s.scan, total) + q, cap);
    if (len < 0 || end == cap) bits |= HR_TABLES_BAD_LENGTH;
    if (tid < n) a.q_cu[tid + 1] = s.q_cu[tid + 1] = (int)min(end, (unsigned)a.max_tokens);
    const int tokens = (int)min(total, (unsigned)a.max_tokens), pair = tid >> 2;
    int before = 0;
    if (pair < n) {
        const int k = s.key[pair];
        for (int j = tid & 3; j < n; j += 4) {
            const int other = s.key[j];
            before += other < k || (other == k && j < pair) ? 1 : 0;
        }
    }
    before += __shfl_xor(before, 1, 64);
    before += __shfl_xor(before, 2, 64);
    if (pair < n && (tid & 3) == 0) a.order[before] = s.order[before] = pair;
    if (bits) atomicOr(&s.bits, bits);
    __syncthreads();
    // groups: tokens and heads of groups share a word of the scan
    static_assert(kSmallWork < 1 << 20 && kSmallPairs < 1 << 12, "");
    unsigned mine = 0;
    bool head = false;
    if (tid < n) {
        const int p = s.order[tid];
        head = tid == 0 || s.key[p] != s.key[s.order[tid - 1]];
        mine = (unsigned)(s.q_cu[p + 1] - s.q_cu[p]) << 12 | (head ? 1u : 0u);
    }
    const unsigned at = block_scan(mine, 0xFFFFFFFFu, s.scan, total);
    const int groups = (int)(total & 0xFFFu);
    if (tid < n) {
        s.ord_first[tid] = (int)(at >> 12);
        if (head) {
            s.grp_pair[at & 0xFFFu] = tid;
            s.grp_tok[at & 0xFFFu] = (int)(at >> 12);
        }
    }
    if (tid == 0) {
        s.grp_pair[groups] = n;
        s.grp_tok[groups] = tokens;
    }
    __syncthreads();
    // row blocks of the groups
    const int rows = tid < groups ? (s.grp_tok[tid + 1] - s.grp_tok[tid]) * a.g : 0;
    const unsigned both[2][1] = {{(unsigned)blocks_of(rows)}, {(unsigned)tiles_of(rows)}};
    unsigned ex[2][1], all[2];
    block_scan(both, ex, 0xFFFFFFFFu, s.scan, all);
    const unsigned b0 = ex[0][0], t0 = ex[1][0], blocks = all[0], tiles = all[1];
    if (tid < groups) {
        s.blk_cu[tid] = (int)b0;
        s.tile_cu[tid] = (int)t0;
    }
    if (tid == 0) {
        s.blk_cu[groups] = (int)blocks;
        s.tile_cu[groups] = (int)tiles;
        int32_t* hdr = a.sched + a.lay.hdr;
        hdr[SH_TOKENS] = tokens;
        hdr[SH_GROUPS] = groups;
        hdr[SH_BLOCKS] = (int)blocks;
        hdr[SH_TILES] = (int)tiles;
        a.report[0] = tokens;
        a.report[1] = groups;
        a.report[3] = 0;
    }
    __syncthreads();
    const Found f{s.q_cu, s.order, s.ord_first, s.grp_pair, s.grp_tok, s.blk_cu, s.tile_cu, tokens, groups, (int)blocks, (int)tiles};
    bits = tables_fill(a, f, tid, kThreads);
    if (bits) atomicOr(&s.bits, bits);
    __syncthreads();
    if (tid == 0) a.report[2] = s.bits;
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
    int key_bits = 1;                                     // keys are 0 .. n_docs
    while (docs->n_docs >> key_bits) ++key_bits;
    a.passes = (key_bits + 7) / 8;                        // digits of one width: the last one is as cheap as the others
    a.bits = (key_bits + a.passes - 1) / a.passes;
    a.wide = t->n_pairs > kChipWaves ? 4 : 6;
    const int64_t work = (int64_t)t->n_pairs * (t->pt_stride + 64) + t->max_tokens;
    if (t->n_pairs <= kSmallPairs && work <= kSmallWork) {
        tables_small_kernel<<<1, kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    if (t->n_pairs <= kCountPairs && docs->n_docs < kWindow * (t->n_pairs / kWindowPairs)) {
        const size_t lds = (size_t)std::min(docs->n_docs + 1, kWindow) * 2 * sizeof(unsigned);
        if (lds + sizeof(Shared) > 65536) {
            const hipError_t e = hipFuncSetAttribute((const void*)tables_count_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) return e;
        }
        tables_count_kernel<<<1, kThreads, lds, st>>>(a);
        tables_place_kernel<<<(unsigned)((t->n_pairs + kPlacePairs - 1) / kPlacePairs), kThreads, 0, st>>>(a);
    } else {
        tables_sort_kernel<<<1, kThreads, 0, st>>>(a);
    }
    const int64_t blocks = std::min<int64_t>((std::max<int64_t>((int64_t)t->n_pairs << a.wide, t->max_tokens) + 255) / 256, kChipWaves / 4);
    tables_fill_kernel<<<(unsigned)blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace hr
