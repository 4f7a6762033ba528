// Rotary positions: the channels that a token's lanes read and write, walked as the kernel does, for every head size, rotated part and type that a
// call accepts.  Each channel of a head belongs to one chunk, and none lies outside the head.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "hr_pair.h"

int main() {
    for (int layout = 0; layout < 2; ++layout)
        for (int esz = 2; esz <= 4; esz += 2)
            for (int d = 2; d <= 1024; d += d < 300 ? 1 : 37)
                for (int r = 2; r <= d && r <= 256; r += 2)
                    for (bool in_place : {false, true}) {
                        const hr_rope_cfg c{d, r, layout, HR_ROPE_SCALE_NONE, 1.0f, 10000.0f, 1.0f, 0.0f, 1.0f, 4.0f};
                        if (hr::rope_check(&c) != HR_OK) continue;
                        const hr::RopeShape s = hr::rope_shape(d, r, layout, esz, in_place, 3);
                        const int rot_chunks = r / 2 / s.vec;
                        std::vector<int> times(d, 0);
                        for (int chunk = 0; chunk < s.chunks; ++chunk) {
                            const hr::RopeChunk x = hr::rope_chunk(chunk, rot_chunks, s.vec, layout, r, d);
                            const bool twice = layout == HR_ROPE_HALF && chunk < rot_chunks;
                            for (int i = 0; i < x.n; ++i)
                                for (int ch : {x.at + i, x.at + i + r / 2}) {
                                    if (ch != x.at + i && !twice) continue;
                                    if (ch < 0 || ch >= d) {
                                        std::printf("layout %d, %d bytes, %d of %d channels rotated: chunk %d reaches channel %d\n", layout, esz, r, d, chunk, ch);
                                        return 1;
                                    }
                                    ++times[ch];
                                }
                        }
                        for (int ch = 0; ch < d; ++ch)
                            if (times[ch] != (in_place && ch >= r ? 0 : 1)) {
                                std::printf("layout %d, %d bytes, %d of %d channels rotated: channel %d %d times\n", layout, esz, r, d, ch, times[ch]);
                                return 1;
                            }
                    }
    std::printf("every channel once\n");
    return 0;
}
