// What the host side of the decoder uses of the paged caches besides the C entry points.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/nt.h"

namespace nt {
// nt_cache_attend after its checks, with k and v written; out_type: IoType, lo_offset: of the tails with IO_PLANES
int cache_attend(nt_cache *c, const nt_attend_args &a, int out_type, long lo_offset, hipStream_t s);
}  // namespace nt
