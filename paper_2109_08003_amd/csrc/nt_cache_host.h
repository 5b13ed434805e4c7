// What the host side of the decoder uses of the paged caches besides the C entry points.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/nt.h"
#include "nt_cache.h"

namespace nt {
// The calls after their checks.  cache_attend, out_type: IoType, lo_offset: of the tails with IO_PLANES
hipError_t cache_reserve(nt_cache *c, const CacheRows &r, hipStream_t s);
hipError_t cache_end(nt_cache *c, int n, const int32_t *seq, hipStream_t s);  // seq: distinct ids, or the caller clears the marks
hipError_t cache_write(nt_cache *c, int layer, const CacheRows &r, const void *k, const void *v, long ld, int type, hipStream_t s);
hipError_t cache_attend(nt_cache *c, const nt_attend_args &a, int out_type, long lo_offset, hipStream_t s);
}  // namespace nt
