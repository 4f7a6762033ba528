// Products of 8-bit matrices: codes and scales as results, 8-bit instruction.
#include "hr_block_mm_tiles.h"

namespace hr {

hipError_t launch_block_matmul_codes_fast(const MatmulArgs& a, int shape, hipStream_t st) { return launch_codes_shape<true>(a, shape, st); }

}  // namespace hr
