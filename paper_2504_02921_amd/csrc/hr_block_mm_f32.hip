// Products of 8-bit matrices with fp32 results: codes as halves.
#include "hr_block_mm_tiles.h"

namespace hr {

namespace {

// DEPTH: stages; TURNS: groups along k
template <int BM, int BN, int WM, int WN, int DEPTH, int TURNS>
hipError_t launch_shape(const MatmulArgs& a, hipStream_t st) {
    if constexpr (BN / WN < 32) {                    // a wavefront has no 16 columns of either half
        if (a.half > 0) return hipErrorInvalidValue;
    } else {
        if (a.half > 0) return launch_tile<BM, BN, WM, WN, DEPTH, TURNS, false, true, float, false>(a, st);
    }
    return launch_tile<BM, BN, WM, WN, DEPTH, TURNS, false, false, float, false>(a, st);
}

}  // namespace

hipError_t launch_block_matmul_f32(const MatmulArgs& a, int shape, hipStream_t st) {
    switch (shape) {
        case MM_16x64_4: return launch_shape<16, 64, 1, 4, 3, 4>(a, st);
        case MM_32x64_2: return launch_shape<32, 64, 2, 2, 3, 2>(a, st);
        case MM_64x64: return launch_shape<64, 64, 2, 2, 4, 1>(a, st);
        case MM_64x64_2: return launch_shape<64, 64, 2, 2, 4, 2>(a, st);
        case MM_64x128: return launch_shape<64, 128, 2, 2, 3, 1>(a, st);
        case MM_64x128_2: return launch_shape<64, 128, 2, 2, 3, 2>(a, st);
        case MM_64x256: return launch_shape<64, 256, 2, 4, 3, 1>(a, st);
        case MM_128x128: return launch_shape<128, 128, 2, 2, 2, 1>(a, st);
        case MM_128x256: return launch_shape<128, 256, 2, 4, 2, 1>(a, st);
        case MM_256x256: return launch_shape<256, 256, 2, 4, 2, 1>(a, st);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace hr
