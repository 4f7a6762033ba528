// Products of 8-bit matrices into codes and scales: codes as halves, tiles with whole blocks of 128 columns of y.
#include "hr_block_mm_tiles.h"

namespace hr {

namespace {

// DEPTH: stages; TURNS: groups along k
template <int BM, int BN, int WM, int WN, int DEPTH, int TURNS>
hipError_t launch_shape(const MatmulArgs& a, hipStream_t st) {
    if constexpr (BN >= 2 * kBlockCols) {
        if (a.half > 0) return launch_tile<BM, BN, WM, WN, DEPTH, TURNS, false, true, float, true>(a, st);
    }
    if constexpr (BN == kBlockCols || BM >= 64) {
        if (a.half == 0) return launch_tile<BM, BN, WM, WN, DEPTH, TURNS, false, false, float, true>(a, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_block_matmul_codes(const MatmulArgs& a, int shape, hipStream_t st) {
    switch (shape) {
        case MM_16x128_4: return launch_shape<16, 128, 1, 4, 2, 4>(a, st);
        case MM_32x128_2: return launch_shape<32, 128, 1, 4, 3, 2>(a, st);
        case MM_16x256: return launch_shape<16, 256, 1, 8, 4, 1>(a, st);
        case MM_32x256: return launch_shape<32, 256, 1, 8, 4, 1>(a, st);
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
