// Products of 8-bit matrices: fp32 results, codes as halves.
#include "hr_block_mm_tiles.h"

namespace hr {

hipError_t launch_block_matmul_f32(const MatmulArgs& a, int shape, hipStream_t st) { return launch_out_shape<false, float>(a, shape, st); }

}  // namespace hr
