// The rows that the joining launch of the attention goes over, walked as the kernel does: whatever the tables hold, none lies behind the workspace's,
// and tables that were built have every one.
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "hr_pair.h"

int main() {
    for (int max_tokens : {1, 3, 17, 300})
        for (int n_q : {1, 14, 32}) {
            const int64_t room = (int64_t)max_tokens * n_q, groups = hr::pair_join_groups(room);
            for (int said : {0, 1, max_tokens - 1, max_tokens, max_tokens + 1, 4 * max_tokens, 1 << 20, INT_MAX, -1, -77, INT_MIN}) {
                const int64_t rows = hr::pair_join_rows(said, max_tokens, n_q);
                // few pieces: a wavefront a row; many: a workgroup a row, and on by the grid's size
                std::vector<int> few(room, 0), many(room, 0);
                for (int64_t group = 0; group < groups; ++group) {
                    for (int wave = 0; wave < 4; ++wave)
                        if (group * 4 + wave < rows) {
                            if (group * 4 + wave >= room) { std::printf("%d tokens said of %d: row %lld of %lld\n", said, max_tokens, (long long)(group * 4 + wave), (long long)room); return 1; }
                            ++few[group * 4 + wave];
                        }
                    for (int64_t row = group; row < rows; row += groups) {
                        if (row >= room) { std::printf("%d tokens said of %d: row %lld of %lld\n", said, max_tokens, (long long)row, (long long)room); return 1; }
                        ++many[row];
                    }
                }
                for (int64_t r = 0; r < room; ++r)
                    if (few[r] != (r < rows) || many[r] != (r < rows) || (said >= 0 && said <= max_tokens && rows != (int64_t)said * n_q)) { std::printf("row %lld\n", (long long)r); return 1; }
            }
        }
    std::printf("every row once\n");
    return 0;
}
