// Products of 8-bit matrices: bf16 results, codes as halves.
#include "hr_block_mm_tiles.h"

namespace hr {

hipError_t launch_block_matmul_bf16(const MatmulArgs& a, int shape, hipStream_t st) { return launch_out_shape<false, bf16_t>(a, shape, st); }

}  // namespace hr
