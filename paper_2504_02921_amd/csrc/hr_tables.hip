// The tables of a batch of pairs, built on the device from the pairs' documents and query lengths (hr_pair_tables_build).
//
// Three ways.  A small batch is one workgroup's, a thread a pair, with everything that one step hands to the next in LDS: what it costs is the
// loads that depend on each other (document, its place in the list, its pages).  Else two launches.  What goes over all pairs in turn (offsets,
// the stable order by document, groups, their row blocks) is a few passes of scans of one workgroup, which are short (a pair is 8 bytes), while a
// launch of many would wait at a grid barrier for each of them; what is written per pair, token and block goes to the whole chip.  The order is a
// radix sort of up to 8 bits a pass, least first, each wavefront with a run of its own: equal documents keep the pairs' order, and no result depends on
// which wavefront is first.  It runs in registers and LDS where key and place share a word, else through memory, whose scattered stores take a
// cache line each.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "hr_kernels.h"
#include "hr_pair.h"

namespace hr {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kDigits = 256;
constexpr int kChipWaves = 8192;                          // wavefronts that the chip holds; more pairs than that share them, four at a time
constexpr int kSmallPairs = 256, kSmallWork = 16384;      // of a batch that one workgroup builds; work: entries written
constexpr int kPlaceBits = 15, kKeyBits = 32 - kPlaceBits;      // of a word of the sort in LDS
constexpr int kLdsPairs = 1 << kPlaceBits;

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
    unsigned scan[2][kWaves];
    unsigned carry[2];
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

// exclusive sums over the workgroup of PER values a thread, saturating at `cap` (at most 2^30 + 2^30 meets before the cap is applied); total: of
// all.  A wavefront's 64 PER values stand together, 64 beside each other, so that what they come from is read in whole lines.
template <int PER>
__device__ __forceinline__ void block_scan(const unsigned (&v)[PER], unsigned (&ex)[PER], unsigned cap, unsigned* s, unsigned& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned carry = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const unsigned inc = wave_scan(v[e], cap);
        ex[e] = min(carry + (unsigned)lane_before((int)inc, 0), cap);
        carry = min(carry + (unsigned)lane_last((int)inc), cap);
    }
    __syncthreads();                                      // the last scan's sums have been read
    if (lane == 0) s[wave] = carry;
    __syncthreads();
    const unsigned inc = wave_scan(lane < kWaves ? s[lane] : 0u, cap);
    const unsigned before = wave == 0 ? 0u : (unsigned)__builtin_amdgcn_readlane((int)inc, wave - 1);
    total = (unsigned)lane_last((int)inc);
#pragma unroll
    for (int e = 0; e < PER; ++e) ex[e] = min(before + ex[e], cap);
}
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned cap, unsigned* s, unsigned& total) {
    const unsigned one[1] = {v};
    unsigned ex[1];
    block_scan(one, ex, cap, s, total);
    return ex[0];
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
    unsigned total, at = block_scan(sum, 0xFFFFFFFFu, sh.scan[0], total);
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

// The pairs in the documents' order, words [key | pair] in LDS.  A pass deals out from memory what the one before left in LDS.
__device__ void sort_lds(const TablesArgs& a, Shared& sh, unsigned* word) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_pairs;
    int32_t* copy = a.sched + a.lay.idx;
    stream(tid, kThreads, n, [&](int p) { return a.pair_doc[p]; }, [&](int p, int doc) {
        word[p] = (unsigned)key_of(a, doc) << kPlaceBits | (unsigned)p;
        copy[p] = (int)word[p];
    });
    if (!sh.unsorted) {
        __syncthreads();
        return;
    }
    const int run = (n + kThreads - 1) / kThreads * 64, lo = min(wave * run, n), hi = min(lo + run, n);      // a wavefront's pairs
    constexpr int AHEAD = 8;
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = kPlaceBits + a.bits * pass;
        const unsigned mask = (1u << a.bits) - 1;
        clear_counts(sh);
        stream(lo + lane, 64, hi, [&](int i) { return word[i]; }, [&](int, unsigned w) {
            atomicAdd(&sh.count[wave][(w >> shift) & mask], 1u);      // a count: the order of the additions does not show
        });
        __syncthreads();
        digit_places(sh);
        for (int i0 = lo + lane; i0 - lane < hi; i0 += 64 * AHEAD) {
            unsigned w[AHEAD];                            // clamped places: loads without a branch between them
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) w[e] = (unsigned)copy[min(i0 + 64 * e, n - 1)];
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                if (i0 - lane + 64 * e >= hi) break;
                const bool on = i0 + 64 * e < hi;
                const unsigned at = take_place(sh.count[wave], (w[e] >> shift) & mask, a.bits, on);
                if (on) word[at] = w[e];
            }
        }
        __syncthreads();
        if (pass + 1 < a.passes) {
            stream(tid, kThreads, n, [&](int p) { return word[p]; }, [&](int p, unsigned w) { copy[p] = (int)w; });
        }
    }
}

// The same through memory: keys in key[0], pairs in `order`
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

// Everything that goes over the pairs in turn.  One workgroup.
template <bool LDS>
__device__ void tables_scan(const TablesArgs& a, Shared& sh, unsigned* word) {
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
        unsigned q[kPer], at[kPer], total;
        const int p0 = base + wave * 64 * kPer + lane;
        int len[kPer], doc[kPer];                         // clamped places: loads without a branch between them
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            len[e] = a.query_lens[min(p0 + 64 * e, n - 1)];
            doc[e] = a.pair_doc[min(p0 + 64 * e, n - 1)];
        }
        int k0 = key_of(a, a.pair_doc[min(max(p0 - 1, 0), n - 1)]);      // of the pair before, in a run's first lane
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const bool on = p0 + 64 * e < n;
            const int k = key_of(a, doc[e]), up = lane_before(k, k0);
            q[e] = on ? (unsigned)min(max(len[e], 0), a.max_tokens + 1) : 0u;
            if (on && len[e] < 0) bits |= HR_TABLES_BAD_LENGTH;
            unsorted |= on && k < up;
            k0 = lane_last(k);
        }
        block_scan(q, at, cap, sh.scan[0], total);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const unsigned end = min(min(carry + at[e], cap) + q[e], cap);
            if (end == cap) bits |= HR_TABLES_BAD_LENGTH;
            if (p0 + 64 * e < n) a.q_cu[p0 + 64 * e + 1] = (int)min(end, (unsigned)a.max_tokens);
        }
        carry = min(carry + total, cap);
    }
    if (bits) atomicOr(&sh.bits, bits);
    if (unsorted) atomicOr(&sh.unsorted, 1);
    __syncthreads();
    const int tokens = (int)min(carry, (unsigned)a.max_tokens);

    if constexpr (LDS) {
        sort_lds(a, sh, word);
        stream(tid, kThreads, n, [&](int i) { return word[i]; }, [&](int i, unsigned w) { a.order[i] = (int)(w & (kLdsPairs - 1)); });
    } else {
        sort_memory(a, sh);
    }
    const int32_t* key = S + a.lay.key[0];
    auto pair_at = [&](int i) { return LDS ? (int)(word[i] & (kLdsPairs - 1)) : a.order[i]; };
    auto key_at = [&](int i) { return LDS ? (int)(word[max(i, 0)] >> kPlaceBits) : key[max(i, 0)]; };

    // groups: pairs of one document
    unsigned tok_carry = 0, grp_carry = 0;
    for (int base = 0; base < n; base += kThreads * kPer) {
        const int i0 = base + wave * 64 * kPer + lane;
        unsigned q[kPer], head[kPer], t[kPer], g[kPer], q_all, g_all;
        Ends ends[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int i = min(i0 + 64 * e, n - 1);
            ends[e] = *(const Ends*)(a.q_cu + pair_at(i));
            head[e] = (i == 0) | (key_at(i) != key_at(i - 1)) ? 1u : 0u;
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const bool on = i0 + 64 * e < n;
            q[e] = on ? (unsigned)(ends[e].hi - ends[e].lo) : 0u;
            head[e] = on ? head[e] : 0u;
        }
        block_scan(q, t, 0xFFFFFFFFu, sh.scan[0], q_all);
        block_scan(head, g, 0xFFFFFFFFu, sh.scan[1], g_all);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int i = i0 + 64 * e;
            if (i >= n) break;
            S[a.lay.ord_first + i] = (int)(tok_carry + t[e]);
            if (head[e]) {
                S[a.lay.grp_pair + grp_carry + g[e]] = i;
                S[a.lay.grp_tok + grp_carry + g[e]] = (int)(tok_carry + t[e]);
            }
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
        const int g0 = base + wave * 64 * kPer + lane;
        unsigned b[kPer], t[kPer], bo[kPer], to[kPer], b_all, t_all;
        Ends ends[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) ends[e] = *(const Ends*)(S + a.lay.grp_tok + min(g0 + 64 * e, groups - 1));
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int rows = g0 + 64 * e < groups ? (ends[e].hi - ends[e].lo) * a.g : 0;
            b[e] = (unsigned)(rows + kPairBlkRows - 1) / kPairBlkRows;
            t[e] = (unsigned)(rows + kPairTileRows - 1) / kPairTileRows;
        }
        block_scan(b, bo, 0xFFFFFFFFu, sh.scan[0], b_all);
        block_scan(t, to, 0xFFFFFFFFu, sh.scan[1], t_all);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (g0 + 64 * e >= groups) break;
            S[a.lay.blk_cu + g0 + 64 * e] = (int)(b_carry + bo[e]);
            S[a.lay.tile_cu + g0 + 64 * e] = (int)(t_carry + to[e]);
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

template <bool LDS>
__global__ void __launch_bounds__(kThreads) tables_scan_kernel(TablesArgs a) {
    __shared__ Shared sh;
    extern __shared__ unsigned word[];
    tables_scan<LDS>(a, sh, word);
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
    const unsigned end = min(block_scan(q, cap, s.scan[0], total) + q, cap);
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
    const unsigned at = block_scan(mine, 0xFFFFFFFFu, s.scan[1], total);
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
    unsigned blocks, tiles;
    const unsigned b0 = block_scan((unsigned)(rows + kPairBlkRows - 1) / kPairBlkRows, 0xFFFFFFFFu, s.scan[0], blocks);
    const unsigned t0 = block_scan((unsigned)(rows + kPairTileRows - 1) / kPairTileRows, 0xFFFFFFFFu, s.scan[1], tiles);
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
    // entries written; one workgroup writes a few thousand in the time of a launch
    const int64_t work = (int64_t)t->n_pairs * (t->pt_stride + 64) + t->max_tokens;
    if (t->n_pairs <= kSmallPairs && work <= kSmallWork) {
        tables_small_kernel<<<1, kThreads, 0, st>>>(a);
        return hipGetLastError();
    }
    if (t->n_pairs <= kLdsPairs && docs->n_docs < 1 << kKeyBits) {
        const size_t lds = (size_t)t->n_pairs * sizeof(unsigned);
        if (lds + sizeof(Shared) > 65536) {
            const hipError_t e = hipFuncSetAttribute((const void*)tables_scan_kernel<true>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e != hipSuccess) return e;
        }
        tables_scan_kernel<true><<<1, kThreads, lds, st>>>(a);
    } else {
        tables_scan_kernel<false><<<1, kThreads, 0, st>>>(a);
    }
    const int64_t blocks = std::min<int64_t>((std::max<int64_t>((int64_t)t->n_pairs << a.wide, t->max_tokens) + 255) / 256, kChipWaves / 4);
    tables_fill_kernel<<<(unsigned)blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace hr
