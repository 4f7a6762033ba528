// Host part of the operators of a layer under sanitizers: frequencies into buffers of exactly their size, checks, layouts and workspaces over ranges
// of sizes, with what the layouts must hold.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "hr_pair.h"

#define REQUIRE(x)                                                   \
    do {                                                             \
        if (!(x)) {                                                  \
            std::printf("line %d: %s\n", __LINE__, #x);              \
            std::exit(1);                                            \
        }                                                            \
    } while (0)

int main() {
    for (int r = 2; r <= 256; r += 2)
        for (int scaling = HR_ROPE_SCALE_NONE; scaling <= HR_ROPE_SCALE_RAMP; ++scaling) {
            hr_rope_cfg c{256, r, HR_ROPE_HALF, scaling, 1.0f, 10000.0f, 8.0f, 4096.0f, 1.0f, 32.0f};
            std::vector<double> f(r / 2);
            const int rc = hr_rope_frequencies(&c, f.data());
            REQUIRE(rc == (scaling == HR_ROPE_SCALE_BASE && r == 2 ? HR_ERR_INVALID_ARG : HR_OK));
            if (rc == HR_OK)
                for (double x : f) REQUIRE(x > 0.0 && x <= 1.0);
        }
    // every channel belongs to one lane's chunk, and a wavefront's lanes to one token, head and chunk each
    for (int layout = 0; layout < 2; ++layout)
        for (int esz = 2; esz <= 4; esz += 2)
            for (int d = 2; d <= 300; ++d)
                for (int r = 2; r <= d && r <= 256; r += 2)
                    for (int heads : {1, 3, 40})
                        for (bool in_place : {false, true}) {
                            const hr::RopeShape s = hr::rope_shape(d, r, layout, esz, in_place, heads);
                            const int wide = layout == HR_ROPE_INTERLEAVED ? 2 : 1, rest = in_place ? 0 : d - r;
                            REQUIRE(r / 2 % s.vec == 0 && s.vec * wide * esz <= 16);
                            REQUIRE((s.chunks - r / 2 / s.vec) * s.vec * wide >= rest);
                            REQUIRE(s.vec == 1 ? rest <= (s.chunks - r / 2) * wide : (s.chunks - r / 2 / s.vec) * s.vec * wide == rest);
                            REQUIRE(s.heads >= 1 && s.tokens >= 1 && (s.chunks > 64 || s.chunks * s.heads * s.tokens <= 64));
                        }
    // the parts of a work list lie apart, and the workspace holds what the pieces write
    for (int64_t pairs : {1, 2, 255, 257, 5000, 1 << 20})
        for (int64_t tokens : {0, 1, 31, 33, 4096, 1 << 20})
            for (int g : {1, 4, 7, 16}) {
                const hr::SchedLayout s = hr::make_sched_layout(pairs, tokens, g);
                const int64_t at[] = {s.hdr, s.ord_first, s.grp_pair, s.grp_tok, s.blk_cu, s.tile_cu, s.key[0], s.key[1], s.idx, s.ord, s.blk, s.tile, s.total};
                const int64_t n[] = {16, pairs, pairs + 1, pairs + 1, pairs + 1, pairs + 1, pairs, pairs, pairs, 4 * tokens, 8 * s.cap_blk, 8 * s.cap_tile};
                for (int i = 0; i < 12; ++i) REQUIRE(at[i] % 4 == 0 && at[i] + n[i] <= at[i + 1]);
                for (int d : {16, 64, 128, 256})
                    for (int64_t stride : {0, 1, 48, 47, 4096}) {
                        const hr::PairWorkspace w = hr::make_pair_workspace(pairs, tokens, 2 * g, 2, d, stride);
                        REQUIRE(w.most >= 1 && w.most <= hr::kPairSplitMost && (w.most == 1 || tokens == 0) == (w.total == 0));      // no rows, no bytes
                        REQUIRE(w.most == 1 || (w.o >= (size_t)w.most * tokens * 2 * g * 8 && w.total >= w.o + (size_t)w.most * tokens * 2 * g * d * 4));
                        for (int blocks : {0, 1, 16, 300, 5000}) {
                            const hr::PairChoice c = hr::pair_choice(blocks, (blocks + 3) / 4, d, w.most);
                            REQUIRE(c.pieces >= 1 && c.pieces <= w.most);
                        }
                    }
            }
    std::printf("clean under sanitizers\n");
    return 0;
}
