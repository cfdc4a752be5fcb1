// Walks of 16-bit operands on the tensor cores: whether a call's operands suit them, and their launch.
#pragma once
#include <cuda_runtime.h>

#include "../../include/pcr.h"

namespace pcr {

struct WalkArgs;
bool tiles_fit(const pcr_decay_args& a, bool back);
// `of`: which of q, k, v, out (0 .. 3) are a, b, c of each walk; `parts`: 16-bit parts in which what goes into a memory is kept.
int launch_tiles(const WalkArgs& walks, const int (*of)[3], const pcr_decay_args& a, unsigned keys, int parts, int sms, cudaStream_t st);

}  // namespace pcr
