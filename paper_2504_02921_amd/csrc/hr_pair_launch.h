// Launchers of the attention kernels of hr_pair_attention, by the pool's kind.
#pragma once

#include "hr_pair_attn.h"

namespace hr {

// 16-bit and fp8 pools with heads of 64, 96 or 128 channels; grid: (work items of either kind, pieces)
hipError_t launch_pair_half(bool fp8, const PairAttnArgs& a, dim3 grid, hipStream_t st);

}  // namespace hr
