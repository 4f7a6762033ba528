// Prints the shape that a product's tile takes, and that of the rows behind the largest tiles (-1: none), for lines of: into codes, fp32, gate, rows, rows of w, columns
#include <cstdio>

#include "hr_block8.h"

int main() {
    int codes, f32, gate;
    long long m, n, k;
    unsigned char anything = 0;
    while (std::scanf("%d %d %d %lld %lld %lld", &codes, &f32, &gate, &m, &n, &k) == 6) {
        hr::MatmulArgs a{};
        a.M = m;
        a.half = gate ? (int)(n / 2) : 0;
        a.N = gate ? a.half : (int)n;
        a.K = (int)k;
        if (codes) a.codes = &anything;
        const hr::MatmulPlan p = hr::matmul_plan(a, f32 ? HR_F32 : HR_BF16);
        if (p.rows < 1 || p.rows > m || hr::matmul_tiles(p.shape, a, p.rows) < 1) return 1;
        std::printf("%d %d %d\n", p.shape, p.rows < m ? p.rest : -1, (int)hr::MM_SHAPES);
    }
    return 0;
}
