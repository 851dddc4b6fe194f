// Attention over a paged cache, many rows a request: bf16.
#include "paged_tile_impl.h"

namespace fs {
hipError_t paged_mixed_launch_bf16(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) { return paged_mixed_launch_type<bf16_t>(a, dim, row_tiles, s); }
hipError_t paged_mixed_join_launch_bf16(const PagedArgs& a, int dim, int row_tiles, hipStream_t s) { return paged_mixed_join_launch_type<bf16_t>(a, dim, row_tiles, s); }
}  // namespace fs
