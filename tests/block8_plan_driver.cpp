// Prints what a product's arguments lead to, for lines of: into codes, hr_dtype of out, fast, gate, rows, rows of w, columns.  8-bit instruction, shape of the tiles, its rows, shape of the
// rows behind them (-1: none), tiles of both, number of shapes
#include <cstdio>

#include "hr_block8.h"

int main() {
    int codes, dtype, fast, gate;
    long long m, n, k;
    while (std::scanf("%d %d %d %d %lld %lld %lld", &codes, &dtype, &fast, &gate, &m, &n, &k) == 7) {
        const hr_block8 a{(void*)0x1000, (float*)0x2000, m, (int32_t)k, 1, (k + 15) / 16 * 16, hr::blocks_of(k)}, w{(void*)0x3000, (float*)0x4000, n, (int32_t)k, 128, (k + 15) / 16 * 16, hr::blocks_of(k)};
        const long long wide = gate ? n / 2 : n;
        const hr_block8 out{(void*)0x5000, (float*)0x6000, m, (int32_t)wide, 1, (wide + 15) / 16 * 16, hr::blocks_of(wide)};
        hr_matmul_args g{};
        g.dtype = dtype;
        g.gate = gate;
        g.fast = fast;
        if (codes) g.block8 = &out;
        else g.out = (void*)0x7000;
        const hr::MatmulArgs r = hr::matmul_args(a, w, g);
        const hr::MatmulPlan p = hr::matmul_plan(r);
        const bool rest = p.rows < m;
        std::printf("%d %d %lld %d %lld %lld %d\n", (int)r.eight, p.shape, (long long)p.rows, rest ? p.rest : -1, (long long)hr::matmul_tiles(p.shape, r, p.rows),
                    rest ? (long long)hr::matmul_tiles(p.rest, r, m - p.rows) : 0ll, (int)hr::MM_SHAPES);
    }
    return 0;
}
