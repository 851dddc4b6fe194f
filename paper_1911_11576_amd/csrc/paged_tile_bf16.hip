// Attention over a paged cache, many rows a request: bf16.
#include "paged_tile_impl.h"

namespace fs {
hipError_t paged_tile_launch_bf16(const PagedArgs& a, int dim, hipStream_t s) { return paged_tile_launch_type<bf16_t>(a, dim, s); }
}  // namespace fs
