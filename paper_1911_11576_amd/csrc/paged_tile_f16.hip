// Attention over a paged cache, many rows a request: fp16.
#include "paged_tile_impl.h"

namespace fs {
hipError_t paged_mixed_launch_f16(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) { return paged_mixed_launch_type<f16_t>(a, dim, row_tiles, s); }
}  // namespace fs
