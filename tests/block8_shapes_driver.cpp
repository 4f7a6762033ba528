// Prints the shape that a product's tile takes, and that of the rows behind the largest tiles (-1: none), for lines of: into codes, 8-bit instruction, gate, rows, rows of w, columns
#include <cstdio>

#include "hr_block8.h"

int main() {
    int codes, eight, gate;
    long long m, n, k;
    unsigned char anything = 0;
    while (std::scanf("%d %d %d %lld %lld %lld", &codes, &eight, &gate, &m, &n, &k) == 6) {
        hr::MatmulArgs a{};
        a.M = m;
        a.half = gate ? (int)(n / 2) : 0;
        a.N = gate ? a.half : (int)n;
        a.K = (int)k;
        a.eight = eight != 0;
        if (codes) a.codes = &anything;
        const hr::MatmulPlan p = hr::matmul_plan(a);
        if (p.rows < 1 || p.rows > m || hr::matmul_tiles(p.shape, a, p.rows) < 1) return 1;
        std::printf("%d %d %d\n", p.shape, p.rows < m ? p.rest : -1, (int)hr::MM_SHAPES);
    }
    return 0;
}
