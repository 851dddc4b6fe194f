// Attention over a paged cache, many rows a request: fp16.
#include "paged_tile_impl.h"

namespace fs {
hipError_t paged_tile_launch_f16(const PagedArgs& a, int dim, hipStream_t s) { return paged_tile_launch_type<f16_t>(a, dim, s); }
}  // namespace fs
