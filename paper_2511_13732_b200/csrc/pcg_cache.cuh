// Checks of arguments that the cache's entry points and the attention's share.
#pragma once

#include "pcg_common.cuh"

namespace pcg {

// The pointer is memory of the current device.
pcg_status check_here(const char *who, const void *p);
bool valid_block_size(int32_t n);
pcg_status check_cache(const char *who, const pcg_cache *c);
// Packed rows [rows, heads, d]: base and stride.
pcg_status check_rows(const char *who, const char *name, const void *p, int64_t stride, int32_t heads, int32_t d,
                      pcg_dtype dtype);

}  // namespace pcg
