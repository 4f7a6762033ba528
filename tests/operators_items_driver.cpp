// What a work item of the attention makes of its record, built or not: rows and places inside the call's arrays, in blocks and in tiles, with numbers
// that do not run over.
#include <climits>
#include <cstdio>
#include <cstdlib>

#include "hr_pair.h"

#define REQUIRE(x)                                                                                                              \
    do {                                                                                                                        \
        if (!(x)) {                                                                                                             \
            std::printf("record %d %d %d %d %d of %d pairs, %d tokens, %d pages, %d heads: %s\n", r[0], r[1], r[2], r[3], r[4], \
                        n_pairs, max_tokens, pt_stride, g, #x);                                                                 \
            std::exit(1);                                                                                                       \
        }                                                                                                                       \
    } while (0)

int main() {
    const int odd[] = {0, 1, 7, 31, 1000, 1 << 30, INT_MAX - 127, INT_MAX - 31, INT_MAX - 1, INT_MAX, -1, -77, INT_MIN, INT_MIN + 1};
    const int sizes[][4] = {{1, 1, 0, 1}, {3, 40, 4, 7}, {1000, 1 << 20, 2048, 16}, {1 << 30, 1 << 30, 1 << 26, 1}, {5, 1 << 26, 1 << 26, 16}};
    for (const auto& c : sizes) {
        const int n_pairs = c[0], max_tokens = c[1], pt_stride = c[2], g = c[3];
        for (int pair : odd)
            for (int D : odd)
                for (int tok : odd)
                    for (int row : odd)
                        for (int rows : odd) {
                            const int r[5] = {pair, D, tok, row, rows};
                            const hr::PairItem it = hr::pair_item(pair, D, tok, row, rows, n_pairs, max_tokens, pt_stride, g);
                            REQUIRE(it.pair >= 0 && it.pair < n_pairs);
                            REQUIRE(it.D >= 0 && it.D <= (int64_t)pt_stride * hr::kPageTokens);
                            REQUIRE(it.tok >= 0 && it.tok < max_tokens);
                            REQUIRE(it.row >= 0 && it.row < it.rows && it.rows <= (int64_t)max_tokens * g);
                            for (int at = 0; at < hr::kPairTileRows; at += 31) {
                                const hr::PairPlace p = hr::pair_place(it, it.row + at, g, max_tokens);
                                REQUIRE(p.head >= 0 && p.head < g && p.place >= 0 && p.place < max_tokens);
                            }
                            // a record that the tables can hold is taken as it is
                            if (pair >= 0 && pair < n_pairs && D >= 0 && D <= (int64_t)pt_stride * hr::kPageTokens && tok >= 0 && row >= 0 && row < rows && tok < max_tokens &&
                                rows <= (int64_t)(max_tokens - tok) * g)
                                REQUIRE(it.pair == pair && it.D == D && it.tok == tok && it.row == row && it.rows == rows);
                        }
    }
    // a prefix and a pair's offsets: what is added to a place stays a place's
    for (int prefix : odd)
        for (int begin : odd)
            for (int end : odd) {
                const int max_tokens = 1 << 30, all = hr::pair_prefix(prefix, begin, end, max_tokens);
                if (all < 0 || all > max_tokens || (begin >= 0 && end >= begin && end <= max_tokens && prefix >= 0 && all != (prefix < end - begin ? prefix : end - begin))) {
                    std::printf("prefix %d of %d .. %d: %d\n", prefix, begin, end, all);
                    return 1;
                }
            }
    std::printf("inside\n");
    return 0;
}
