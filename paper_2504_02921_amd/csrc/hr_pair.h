// The operators for models whose layers the caller runs (hr_rope_apply, hr_pair_tables_build, hr_pair_attention): what their host
// and device parts share.
#pragma once

#include <cstddef>
#include <cstdint>

#include "hr_internal.h"
#include "hr_layout.h"

namespace hr {

// ---- rotary positions
constexpr int kMaxRotaryPairs = 128, kRopeWaves = 4;
int rope_check(const hr_rope_cfg* c);
int rope_apply_check(const hr_rope_cfg* c, const double* freqs, int dtype, int64_t n_tokens, const int32_t* positions, int32_t first_position,
                     int32_t period, const hr_rope_tensor* tensors, int32_t n_tensors);

// How a wavefront's lanes are spread over a token's heads: a lane has `vec` pairs (or, behind the rotated channels, as many others as one of its
// loads brings) of one head, `chunks` lanes have a head, `heads` heads and `tokens` tokens are taken at a time.
struct RopeShape { int vec, chunks, heads, tokens; };
RopeShape rope_shape(int head_dim, int rotary_dim, int layout, int esz, bool in_place, int n_heads);

// The channels of a lane's chunk: `n` from `at` on and, where a half layout is turned, as many a half further.  rot_chunks: chunks of rotated channels
struct RopeChunk { int at, n; };
HR_HD RopeChunk rope_chunk(int chunk, int rot_chunks, int vec, int layout, int rotary_dim, int head_dim) {
    const int wide = layout == HR_ROPE_INTERLEAVED ? 2 * vec : vec;
    if (chunk < rot_chunks) return RopeChunk{chunk * wide, wide};
    const int at = rotary_dim + (chunk - rot_chunks) * wide;
    return RopeChunk{at, wide < head_dim - at ? wide : head_dim - at};      // neighbours are taken two at a time: an odd head's last channel stands alone
}

// ---- tables of a batch of pairs
// The attention's work list, in int32 units from hr_pair_tables.sched.  "In order": the pairs by document, token behind token.
// A group is the pairs of one document; its rows for a kv head are (token in order, query head of the group of heads), heads fastest.
struct SchedLayout {
    int64_t hdr = 0;           // SchedHdr
    int64_t ord_first = 0;     // [n_pairs] place of the first token of every pair, pairs in order
    int64_t grp_pair = 0;      // [n_pairs + 1] a group's first place in `order`
    int64_t grp_tok = 0;       // [n_pairs + 1] its first token's place
    int64_t blk_cu = 0;        // [n_pairs + 1] blocks of kPairBlkRows rows before a group
    int64_t tile_cu = 0;       // [n_pairs + 1] ... of kPairTileRows rows
    int64_t key[2] = {0, 0}, idx = 0;      // [n_pairs] each: the sort
    int64_t ord = 0;           // [max_tokens] int4: token's row, place of its pair's first token, pair, document length
    int64_t blk = 0, tile = 0; // records of 8: a pair of the group, document length, group's first place, first row, rows of the group
    int64_t total = 0;
    int64_t cap_blk = 0, cap_tile = 0;
};
enum SchedHdr { SH_TOKENS = 0, SH_GROUPS = 1, SH_BLOCKS = 2, SH_TILES = 3 };
constexpr int kPairBlkRows = 32, kPairTileRows = 128;
constexpr int kSchedRec = 8;
SchedLayout make_sched_layout(int64_t n_pairs, int64_t max_tokens, int g);
int tables_check(const hr_pool* pool, const hr_pair_tables* t);       // sizes and pointers that building and reading have in common
int tables_build_check(const hr_pool* pool, const hr_doc_list* docs, const int32_t* pair_doc, const int32_t* query_lens, const hr_pair_tables* t);

// ---- attention
int attention_check(const hr_pool* pool, const hr_pair_tables* t, const hr_attention_args* a);
int attention_outputs_check(const hr_attention_args* a);      // ... of a call that has something to write: its outputs are not its inputs
// Few rows and long documents: an item's keys are cut into up to `most` pieces, each a workgroup's, whose results are joined by a second
// launch.  How many is decided on the device, which knows the items (pair_choice); `most` bounds grid and workspace.
// Whole / in pieces, with the join: 16 blocks of 304 keys 10.6 / 11.8 us, of 544 12.7 / 12.4, of 1025 18.1 / 12.5, of 2049 28.7 / 12.7.
constexpr int kPairSplitMost = 128, kPairSplitKeys = 256, kPairSplitLeast = 768;      // keys of a piece, of documents that are cut, at least
int pair_most_splits(int64_t n_pairs, int64_t max_tokens, int n_q, int n_kv, int d, int64_t pt_stride);
constexpr int kPairSplitWgs = 512;                            // workgroups that a launch wants
// Whether an attention's work items are blocks of 32 rows, each streaming its keys for itself, or tiles of four, which share a stream (see
// hr_pair_attn_mfma.hip), and their pieces.  blocks, tiles: of all kv heads.  Tiles read and expand keys once for up to four blocks, blocks fill
// the chip sooner: tiles pay where they are more than a third full and the blocks more than the chip takes at once.  Blocks / tiles, in us:
// 64 channels, 280 blocks of 544 keys 11.2 / 15.3, 320 of 2064 24.6 / 41.0, 700 of 544 17.9 / 15.9, 1120 of 544 27.7 / 21.2, 4480 of 544 84.8 / 44.4, two
// a tile 2560 of 520 51.3 / 41.9; 96 channels, 240 of 544 13.2 / 18.2, 360 18.1 / 18.4, 540 23.4 / 19.6, 240 of 4128 51.1 / 48.3; 128 channels, 128 blocks of 4112 33.3 / 44.2, 256 of 4128 45.7 / 45.3, 312 of 8200 95.0 / 75.2, 640 of 288 24.7 / 17.3;
// one block a tile, 1280 of 516 (64 channels) 37.0 / 37.1, 3200 of 520 183 / 190, 800 of 2049 (fp8) 101 / 159.
HR_HD int pair_tile_blocks(int d) { return d == 64 ? 512 : 256; }
struct PairChoice { bool tiles; int pieces; };
HR_HD PairChoice pair_choice(int blocks, int tiles, int d, int most) {
    PairChoice c;
    c.tiles = blocks > pair_tile_blocks(d) && 2 * (int64_t)blocks > 3 * (int64_t)tiles;
    const int items = c.tiles ? tiles : blocks, s = kPairSplitWgs / (items > 0 ? items : 1);
    c.pieces = s < 1 ? 1 : s > most ? most : s;
    return c;
}
// What the work list says of an item, from the first five words of its record.  Tables that were not built, or not for this call, are taken for what
// they can at most be: every index stays inside its array and every loop ends, whatever they hold.
struct PairItem {
    int pair, D;                      // a pair of the group, and its document's length
    int tok, row, rows;               // place of the group's first token, the item's first row, rows of the group
};
HR_HD int within(int lo, int v, int hi) { return v < lo ? lo : v > hi ? hi : v; }
HR_HD PairItem pair_item(int pair, int D, int tok, int row, int rows, int n_pairs, int max_tokens, int pt_stride, int g) {
    PairItem it;
    it.pair = within(0, pair, n_pairs - 1);
    it.D = within(0, D, pt_stride * kPageTokens);
    it.tok = within(0, tok, max_tokens - 1);
    it.row = within(0, row, max_tokens * g - 1);
    it.rows = within(it.row + 1, rows, max_tokens * g);
    return it;
}
// A row's query head within its kv head's group and its token's place in order; rows behind the item's last one repeat that
struct PairPlace { int head, place; };
HR_HD PairPlace pair_place(const PairItem& it, int row, int g, int max_tokens) {
    const int rc = row < it.rows ? row : it.rows - 1, t = rc / g;
    return PairPlace{rc - t * g, it.tok + t < max_tokens ? it.tok + t : max_tokens - 1};
}
// Own keys that a whole query sees, by the caller's prefix and the query's offsets
HR_HD int pair_prefix(int prefix, int begin, int end, int max_tokens) {
    const int64_t n = (int64_t)end - begin, all = prefix < n ? prefix : n;
    return all < 0 ? 0 : (int)(all < max_tokens ? all : max_tokens);
}

// The launch that joins the pieces: its workgroups, four rows each where a row has few pieces and one by one where it has many; and the rows that there
// are when the tables say `tokens`.  Tables that were not built say anything
inline int64_t pair_join_groups(int64_t rows) {
    const int64_t fours = (rows + 3) / 4, few = rows < kPairSplitWgs ? rows : kPairSplitWgs;
    return fours > few ? fours : few;
}
HR_HD int64_t pair_join_rows(int tokens, int max_tokens, int n_q) {
    return (int64_t)(tokens < 0 ? 0 : tokens > max_tokens ? max_tokens : tokens) * n_q;
}
struct PairWorkspace { size_t ml = 0, o = 0, total = 0; int most = 1; };
PairWorkspace make_pair_workspace(int64_t n_pairs, int64_t max_tokens, int n_q, int n_kv, int d, int64_t pt_stride);

}  // namespace hr
